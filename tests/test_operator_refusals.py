"""Arguments that the head norms, the 8-bit layers and their quantisers refuse: found on the host, before any launch (no GPU needed)."""
import ctypes

import pytest

from paper_2506_05096_b200 import binding as A, build

P = 0x1000                                       # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def L():
    build.build_library()
    return A.lib()


def rows(x=P, y=P + 4096, idx=None, M=0, H=2, d=64, flags=0, weight=None, bias=None, xs=None, ys=None):
    st = (16 * H * d, d, H * d)
    return A.HeadRows(x, *(xs or st), y, *(ys or st), idx, weight, bias, M, H, flags)


def test_head_norm(L):
    def call(*ts, cos=P, sin=P, n_rot=16, B=1, N=16, d=64, norm=0, rotation=0, eps=1e-6, ws=None):
        return L.astraea_qk_norm_rotate((A.HeadRows * max(1, len(ts)))(*ts), len(ts), cos, sin, n_rot, B, N, d, norm, rotation, eps, ws, None)

    assert call() == A.ERR_INVALID_ARG and call(rows(), rows(), rows()) == A.ERR_INVALID_ARG
    assert L.astraea_qk_norm_rotate(None, 1, P, P, 16, 1, 16, 64, 0, 0, 0.0, None, None) == A.ERR_INVALID_ARG
    assert call(rows(), d=80) == A.ERR_UNSUPPORTED
    assert call(rows(), norm=2) == A.ERR_UNSUPPORTED and call(rows(), rotation=-1) == A.ERR_UNSUPPORTED
    assert call(rows(flags=4)) == A.ERR_UNSUPPORTED
    for bad in (dict(n_rot=17), dict(n_rot=-1), dict(cos=None), dict(sin=P + 4), dict(eps=-1.0), dict(ws=2), dict(B=0), dict(N=0), dict(B=1 << 11, N=1 << 20)):
        assert call(rows(), **bad) == A.ERR_INVALID_ARG, bad
    for bad in (dict(x=None), dict(y=None), dict(x=P + 2), dict(y=P + 8), dict(H=0), dict(weight=P + 4), dict(bias=P), dict(idx=P, M=17),
                dict(idx=P, M=-1), dict(flags=A.ROWS_COMPACT_IN), dict(xs=(2048, 64, 132)), dict(ys=(2048, 32, 128)), dict(xs=(-8, 64, 128))):
        assert call(rows(**bad)) == A.ERR_INVALID_ARG, bad
        assert call(rows(), rows(**bad)) == A.ERR_INVALID_ARG, bad
    assert call(rows(x=P, y=P, idx=P, M=3, flags=A.ROWS_COMPACT_IN)) == A.ERR_INVALID_ARG and b"in place" in L.astraea_last_error()
    assert call(rows(x=P, y=P, ys=(4096, 64, 256))) == A.ERR_INVALID_ARG
    assert call(rows(idx=P, M=0, x=None, y=None)) == A.OK                                 # an empty list: nothing to do
    assert L.astraea_workspace_bytes(A.OP_QK_NORM_ROTATE, 1, 1, 1, 1, 64) == 256


def test_quantisers(L):
    def call(x=P, idx=P, M=4, xq=P, s=P, B=1, N=16, K=128, flags=0, ws=None):
        return L.astraea_quantize_fp8(x, idx, M, xq, s, B, N, K, flags, ws, None)

    assert call(K=192) == A.ERR_INVALID_ARG and b"128" in L.astraea_last_error()
    assert call(flags=A.LINEAR_COMPACT_OUT) == A.ERR_UNSUPPORTED
    for bad in (dict(x=None), dict(xq=None), dict(s=None), dict(x=P + 8), dict(xq=P + 4), dict(s=P + 2), dict(M=17), dict(M=-1), dict(B=0), dict(K=0),
                dict(ws=3), dict(idx=None, flags=A.LINEAR_COMPACT_IN)):
        assert call(**bad) == A.ERR_INVALID_ARG, bad
    assert call(M=0, x=None) == A.OK
    w = lambda w=P, q=P, s=P, N_out=8, K=128: L.astraea_quantize_fp8_weight(w, q, s, N_out, K, None)
    for bad in (dict(w=None), dict(q=P + 1), dict(s=P + 1), dict(N_out=0), dict(K=64), dict(K=0), dict(N_out=128 * 65536)):
        assert w(**bad) == A.ERR_INVALID_ARG, bad


def test_linear(L):
    def call(xq=P, xs=P, idx=P, M=4, wq=P, ws=P, bias=None, res=None, gate=None, y=P, B=1, N=16, K=128, N_out=64, flags=0, work=P, size=256):
        return L.astraea_gathered_linear_fp8(xq, xs, idx, M, wq, ws, bias, res, gate, y, B, N, K, N_out, flags, work, size, None)

    assert call(flags=A.LINEAR_COMPACT_IN) == A.ERR_UNSUPPORTED and call(flags=16) == A.ERR_UNSUPPORTED
    assert call(work=None) == A.ERR_WORKSPACE_TOO_SMALL and call(size=255) == A.ERR_WORKSPACE_TOO_SMALL
    for bad in (dict(K=64), dict(K=192), dict(N_out=12), dict(M=17), dict(B=0), dict(xq=None), dict(xs=None), dict(wq=None), dict(ws=None), dict(y=None),
                dict(xq=P + 8), dict(wq=P + 8), dict(y=P + 8), dict(bias=P + 8), dict(res=P + 8), dict(gate=P + 8), dict(xs=P + 2), dict(ws=P + 2),
                dict(work=P + 16), dict(flags=A.LINEAR_COMPACT_RES), dict(idx=None, flags=A.LINEAR_COMPACT_OUT),
                dict(B=1 << 20, N=1 << 16, M=1 << 16)):
        assert call(**bad) == A.ERR_INVALID_ARG, bad
    assert call(M=0, xq=None) == A.OK
    assert L.astraea_workspace_bytes(A.OP_GATHERED_LINEAR_FP8, 1, 1, 1, 1, 64) == 256


def test_binding_raises_and_an_empty_list_is_not_all_rows(L):
    import torch
    h = A.head_rows(torch.zeros(8), (8, 8, 8), torch.zeros(8), (8, 8, 8), 1, torch.zeros(1, 0, dtype=torch.int32), 0)
    assert h.idx and h.M == 0
    assert ctypes.sizeof(A.HeadRows) == 8 * 11 + 16


def test_window_attention(L):
    def call(q=P, k=P, v=P, out=P, qs=(1024, 64, 128), ks=(1024, 64, 128), idx=P, M=4, kv_len=None, B=1, H=2, H_kv=2, N=16, d=64, n_first=0, n_last=0,
             left=1, right=1, scale=0.0, flags=0, ws=P, size=256):
        return L.astraea_window_attn(q, k, v, *qs, *ks, *ks, idx, M, kv_len, out, None, B, H, H_kv, N, d, n_first, n_last, left, right, scale, flags,
                                     ws, size, None)

    assert call(d=96) == A.ERR_UNSUPPORTED and call(flags=16) == A.ERR_UNSUPPORTED
    assert call(ws=None) == A.ERR_WORKSPACE_TOO_SMALL and call(size=255) == A.ERR_WORKSPACE_TOO_SMALL
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(q=P + 8), dict(out=P + 8), dict(qs=(1024, 64, 100)), dict(ks=(1024, 60, 128)),
                dict(qs=(1024, 64, 32)), dict(ks=(-8, 64, 128)), dict(M=17), dict(M=-1), dict(B=0), dict(H=3), dict(H_kv=0), dict(N=0), dict(N=(1 << 30) + 1),
                dict(n_first=-1), dict(n_last=-1), dict(left=-1), dict(right=-1), dict(scale=-1.0), dict(ws=P + 128),
                dict(N=1 << 29, M=1 << 29, H=8, H_kv=2)):
        assert call(**bad) == A.ERR_INVALID_ARG, bad
    assert call(M=0) == A.OK
    # room for the key shares: one unit's at least, no more than 296 shares
    assert 256 + 16 * 256 * 516 <= L.astraea_workspace_bytes(A.OP_WINDOW_ATTN, 1, 1, 1000, 1, 128) < 3 << 20
    assert L.astraea_workspace_bytes(A.OP_WINDOW_ATTN, 8, 64, 1 << 20, 1 << 20, 128) < 40 << 20


def test_sizes_at_the_limits(L):
    assert L.astraea_quantize_fp8_weight(P, P, P, 65535 * 128 + 1, 128, None) == A.ERR_INVALID_ARG
    assert L.astraea_quantize_fp8_weight(P, P, P, 0x7fffffff, 128, None) == A.ERR_INVALID_ARG
    for n_out in (65535 * 128 + 8, 0x7ffffff8):
        assert L.astraea_gathered_linear_fp8(P, P, P, 4, P, P, None, None, None, P, 1, 16, 128, n_out, 0, P, 256, None) == A.ERR_INVALID_ARG
        assert b"65535" in L.astraea_last_error()
    s = (1 << 20, 64, 128)
    for h, h_kv in ((4097, 1), (8194, 2)):                 # query heads of a key head
        assert L.astraea_window_attn(P, P, P, *s, *s, *s, P, 4, None, P, None, 1, h, h_kv, 16, 64, 0, 0, 1, 1, 0.0, 0, P, 256, None) == A.ERR_INVALID_ARG
        assert b"4096" in L.astraea_last_error()
