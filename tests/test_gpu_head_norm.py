"""astraea_qk_norm_rotate against the formula in 64 bits: head widths, lists, strides, in place, a cache that rows are appended to."""
import pytest
import torch

from helpers import Guarded
from paper_2506_05096_b200 import binding as A

pytestmark = pytest.mark.gpu
EPS = 1e-6


def reference(x, tok, n_rot, cos, sin, weight, bias, norm, rotation, eps=EPS):
    """x [B, M, H, d] fp64, tok [B, M]."""
    x = x.double()
    if norm == A.NORM_LAYER:
        x = x - x.mean(-1, keepdim=True)
    z = x / ((x * x).mean(-1, keepdim=True) + eps).sqrt()
    if weight is not None:
        z = z * weight.double()
    if bias is not None:
        z = z + bias.double()
    d = x.shape[-1]
    first, second = (torch.arange(d // 2), torch.arange(d // 2, d)) if rotation == A.ROTATE_HALF else (torch.arange(0, d, 2), torch.arange(1, d, 2))
    out = z.clone()
    for b in range(x.shape[0]):
        for r in range(x.shape[1]):
            t = int(tok[b, r])
            if t < n_rot:
                c, s = cos[t].double(), sin[t].double()
                out[b, r][:, first] = z[b, r][:, first] * c - z[b, r][:, second] * s
                out[b, r][:, second] = z[b, r][:, first] * s + z[b, r][:, second] * c
    return out, z


def close(got, want, z, layer):
    # one rounding to bf16 (2^-8 of the value), and fp32 arithmetic: the sum, the mean, rsqrt, three products and a sum are each within a
    # few 2^-24 of the largest channel of the head; a mean of up to four standard deviations costs two more bits
    big = z.abs().amax(-1, keepdim=True)
    excess = (got.double() - want).abs() - (2.0 ** -8 * want.abs() + (2.0 ** -18 if layer else 2.0 ** -20) * big)
    assert excess.max() <= 0, float(excess.max())


def table(n, d, g):
    a = torch.rand(n, d // 2, generator=g, device="cuda", dtype=torch.float64) * 1000
    return a.cos().float(), a.sin().float()


@pytest.mark.parametrize("d,H", [(64, 1), (64, 8), (64, 9), (64, 48), (72, 1), (72, 4), (72, 16), (128, 1), (128, 5), (128, 24), (128, 25)])
@pytest.mark.parametrize("norm", [A.NORM_RMS, A.NORM_LAYER])
@pytest.mark.parametrize("rotation", [A.ROTATE_INTERLEAVED, A.ROTATE_HALF])
def test_listed_queries_and_all_keys_in_one_launch(d, H, norm, rotation):
    g = torch.Generator("cuda").manual_seed(d * 100 + H)
    B, N, M, H_kv, n_rot = 2, 37, 13, max(1, H // 2), 30
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    q, k = 2 + 3 * rnd(B, N, H, d), 3 * rnd(B, N, H_kv, d)
    k[1, 5] = 0                                                    # a head of zeros: the norm's eps keeps it finite
    wq, wk = 1 + 0.3 * rnd(d), rnd(d)
    bq = rnd(d) if norm == A.NORM_LAYER else None
    cos, sin = table(n_rot, d, g)
    idx = torch.stack([torch.randperm(N, device="cuda", generator=g)[:M].sort().values for _ in range(B)]).int()
    before = rnd(B, N, H, d)
    qo, ko = Guarded((B, N, H, d), torch.bfloat16, before), Guarded((B, N, H_kv, d), torch.bfloat16)
    ws = A.new_workspace(A.OP_QK_NORM_ROTATE, B, H, N, M, d)
    sq, sk = A.bhnd_strides(N, H, d), A.bhnd_strides(N, H_kv, d)
    A.astraea_qk_norm_rotate([A.head_rows(q, sq, qo.t, sq, H, idx, M, wq, bq), A.head_rows(k, sk, ko.t, sk, H_kv, weight=wk)], cos, sin, n_rot,
                             B, N, d, norm, rotation, EPS, ws)
    A.astraea_poll_error(ws)
    rows = torch.arange(B, device="cuda")[:, None]
    want, z = reference(q[rows, idx.long()], idx, n_rot, cos, sin, wq, bq, norm, rotation)
    close(qo.t[rows, idx.long()], want, z, norm == A.NORM_LAYER)
    rest = torch.ones(B, N, dtype=torch.bool, device="cuda")
    rest[rows, idx.long()] = False
    assert torch.equal(qo.t[rest], before[rest])
    want, z = reference(k, torch.arange(N).expand(B, -1), n_rot, cos, sin, wk, None, norm, rotation)
    close(ko.t, want, z, norm == A.NORM_LAYER)
    qo.check(); ko.check()


@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("rotation", [A.ROTATE_INTERLEAVED, A.ROTATE_HALF])
def test_one_token_appended_to_a_cache(d, rotation):
    g = torch.Generator("cuda").manual_seed(d)
    B, N, H, H_kv = 3, 500, 12, 3
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    q, k, cache = rnd(B, 1, H, d), rnd(B, 1, H_kv, d), rnd(B, N, H_kv, d)
    was = cache.clone()
    cos, sin = table(N, d, g)
    idx = torch.tensor([[0], [499], [77]], device="cuda", dtype=torch.int32)
    s1, s2, sc = A.bhnd_strides(1, H, d), A.bhnd_strides(1, H_kv, d), A.bhnd_strides(N, H_kv, d)
    qo = torch.empty_like(q)
    A.astraea_qk_norm_rotate([A.head_rows(q, s1, qo, s1, H, idx, 1, flags=A.ROWS_COMPACT_IN | A.ROWS_COMPACT_OUT),
                              A.head_rows(k, s2, cache, sc, H_kv, idx, 1, flags=A.ROWS_COMPACT_IN)], cos, sin, N, B, N, d, rotation=rotation)
    want, z = reference(q, idx, N, cos, sin, None, None, A.NORM_RMS, rotation)
    close(qo, want, z, False)
    want, z = reference(k, idx, N, cos, sin, None, None, A.NORM_RMS, rotation)
    b = torch.arange(B, device="cuda")
    close(cache[b, idx[:, 0].long()][:, None], want, z, False)
    was[b, idx[:, 0].long()] = cache[b, idx[:, 0].long()]
    assert torch.equal(cache, was)


@pytest.mark.parametrize("d", [64, 72, 128])
def test_in_place_on_a_slice_of_fused_projections_and_head_major(d):
    g = torch.Generator("cuda").manual_seed(7)
    B, N, H = 2, 19, 6
    qkv = (3 * torch.randn(B, N, 3, H, d, device="cuda", generator=g)).bfloat16()
    was = qkv.clone()
    cos, sin = table(N, d, g)
    st = (N * 3 * H * d, d, 3 * H * d)
    k_major = torch.empty(B, H, N, d, device="cuda", dtype=torch.bfloat16)
    A.astraea_qk_norm_rotate([A.head_rows(qkv, st, qkv, st, H), A.head_rows(qkv[:, :, 1], st, k_major, (H * N * d, N * d, d), H)], cos, sin, N, B, N, d)
    tok = torch.arange(N).expand(B, -1)
    for got, i in ((qkv[:, :, 0], 0), (k_major.transpose(1, 2), 1)):
        want, z = reference(was[:, :, i], tok, N, cos, sin, None, None, A.NORM_RMS, A.ROTATE_INTERLEAVED)
        close(got, want, z, False)
    assert torch.equal(qkv[:, :, 1:], was[:, :, 1:])


def test_bad_entries_are_skipped_and_reported_and_nan_stays_in_its_head():
    B, N, H, d = 1, 8, 2, 64
    x = torch.randn(B, N, H, d, device="cuda").bfloat16()
    x[0, 3, 1, 5] = float("nan")
    y = torch.full_like(x, 7.0)
    idx = torch.tensor([[1, 3, 3, 99, 5]], device="cuda", dtype=torch.int32)           # a duplicate, out of range, 5 after 99
    ws = A.new_workspace(A.OP_QK_NORM_ROTATE, B, H, N, 5, d)
    st = A.bhnd_strides(N, H, d)
    A.astraea_qk_norm_rotate([A.head_rows(x, st, y, st, H, idx, 5)], None, None, 0, B, N, d, workspace=ws)
    with pytest.raises(A.AstraeaError) as e:
        A.astraea_poll_error(ws)
    assert e.value.code == A.ERR_BAD_INDEX
    assert bool((y[0, [0, 2, 4, 5, 6, 7]] == 7).all()) and not bool((y[0, [1]] == 7).all())
    assert bool(y[0, 3, 1].isnan().all()) and bool(y[0, 3, 0].isfinite().all())
    empty = torch.zeros(1, 0, device="cuda", dtype=torch.int32)
    y.fill_(7)
    A.astraea_qk_norm_rotate([A.head_rows(x, st, y, st, H, empty, 0)], None, None, 0, B, N, d, workspace=ws)
    A.astraea_poll_error(ws)
    assert bool((y == 7).all())


@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("norm", [A.NORM_RMS, A.NORM_LAYER])
@pytest.mark.parametrize("rotation", [A.ROTATE_INTERLEAVED, A.ROTATE_HALF])
@pytest.mark.parametrize("H,H_kv", [(8, 1), (2, 1), (1, 16)])
def test_few_heads_of_many_tokens(d, norm, rotation, H, H_kv):
    g = torch.Generator("cuda").manual_seed(d + H)
    B, N, M, n_rot = 2, 6007, 5001, 5990
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    q, k, wq, wk = 3 * rnd(B, N, H, d), 3 * rnd(B, N, H_kv, d), 1 + 0.3 * rnd(d), rnd(d)
    bk = rnd(d) if norm == A.NORM_LAYER else None
    cos, sin = table(n_rot, d, g)
    idx = torch.stack([torch.randperm(N, device="cuda", generator=g)[:M].sort().values for _ in range(B)]).int()
    idx[1, 77] = idx[1, 76]                                        # a row that is skipped
    before = rnd(B, N, H, d)
    qo, ko = Guarded((B, N, H, d), torch.bfloat16, before), Guarded((B, N, H_kv, d), torch.bfloat16)
    ws = A.new_workspace(A.OP_QK_NORM_ROTATE, B, H, N, M, d)
    sq, sk = A.bhnd_strides(N, H, d), A.bhnd_strides(N, H_kv, d)
    A.astraea_qk_norm_rotate([A.head_rows(q, sq, qo.t, sq, H, idx, M, wq), A.head_rows(k, sk, ko.t, sk, H_kv, weight=wk, bias=bk)], cos, sin, n_rot,
                             B, N, d, norm, rotation, EPS, ws)
    with pytest.raises(A.AstraeaError) as e:
        A.astraea_poll_error(ws)
    assert e.value.code == A.ERR_BAD_INDEX

    def want(x, w, b):
        x = x.double() - (x.double().mean(-1, keepdim=True) if norm == A.NORM_LAYER else 0)
        z = x / ((x * x).mean(-1, keepdim=True) + EPS).sqrt() * w.double() + (0 if b is None else b.double())
        c, s = torch.ones(N, d // 2, device="cuda", dtype=torch.float64), torch.zeros(N, d // 2, device="cuda", dtype=torch.float64)
        c[:n_rot], s[:n_rot] = cos.double(), sin.double()
        c, s = c[None, :, None], s[None, :, None]
        if rotation == A.ROTATE_HALF:
            u, v = z.chunk(2, -1)
            return torch.cat([u * c - v * s, u * s + v * c], -1), z
        u, v = z[..., 0::2], z[..., 1::2]
        return torch.stack([u * c - v * s, u * s + v * c], -1).flatten(-2), z

    y, z = want(k, wk, bk)
    close(ko.t, y, z, norm == A.NORM_LAYER)
    y, z = want(q, wq, None)
    rows = torch.zeros(B, N, dtype=torch.bool, device="cuda")
    rows[torch.arange(B, device="cuda")[:, None], idx.long()] = True
    close(qo.t[rows], y[rows], z[rows], norm == A.NORM_LAYER)
    assert torch.equal(qo.t[~rows], before[~rows])
    qo.check(); ko.check()


def test_many_rows_and_another_stream():
    g = torch.Generator("cuda").manual_seed(3)
    B, N, H, d = 1, 4999, 24, 128                                  # more rows than warps: every warp takes several
    x = torch.randn(B, N, H, d, device="cuda", generator=g).bfloat16()
    y = torch.empty_like(x)
    a = torch.rand(N, d // 2, device="cuda", generator=g) * 6.28
    cos, sin = a.cos(), a.sin()
    st = A.bhnd_strides(N, H, d)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    A.astraea_qk_norm_rotate([A.head_rows(x, st, y, st, H)], cos, sin, N, B, N, d, stream=side)
    side.synchronize()
    z = x.double() / ((x.double() ** 2).mean(-1, keepdim=True) + EPS).sqrt()
    c, s = cos.double()[None, :, None], sin.double()[None, :, None]
    want = torch.stack([z[..., 0::2] * c - z[..., 1::2] * s, z[..., 0::2] * s + z[..., 1::2] * c], -1).flatten(-2)
    close(y, want, z, False)


@pytest.mark.parametrize("d,H", [(64, 49), (72, 21), (72, 41), (128, 50)])
@pytest.mark.parametrize("norm,rotation", [(A.NORM_RMS, A.ROTATE_HALF), (A.NORM_LAYER, A.ROTATE_INTERLEAVED)])
def test_heads_that_take_several_rounds(d, H, norm, rotation):
    test_listed_queries_and_all_keys_in_one_launch(d, H, norm, rotation)
    # and in a launch that gives a warp more than one token, each with all its heads
    g = torch.Generator("cuda").manual_seed(H)
    B, N = 1, 5003
    x = 3 * torch.randn(B, N, H, d, device="cuda", generator=g).bfloat16()
    y = Guarded((B, N, H, d), torch.bfloat16)
    w = torch.randn(d, device="cuda", generator=g).bfloat16()
    cos, sin = table(N - 3, d, g)
    st = A.bhnd_strides(N, H, d)
    A.astraea_qk_norm_rotate([A.head_rows(x, st, y.t, st, H, weight=w)], cos, sin, N - 3, B, N, d, norm, rotation, EPS)
    some = torch.cat([torch.arange(40), torch.arange(2500, 2540), torch.arange(N - 40, N)])
    want, z = reference(x[:, some], some[None], N - 3, cos, sin, w, None, norm, rotation)
    close(y.t[:, some], want, z, norm == A.NORM_LAYER)
    y.check()


@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("H,H_kv", [(1, 16), (16, 1), (1, 1)])
@pytest.mark.parametrize("empty", [0, 1])
def test_an_empty_list_beside_all_rows_in_place(d, H, H_kv, empty):
    g = torch.Generator("cuda").manual_seed(d + H)
    B, N, n_rot = 2, 5500, 5400
    heads = (H, H_kv)
    x = [3 * torch.randn(B, N, h, d, device="cuda", generator=g).bfloat16() for h in heads]
    y = [Guarded((B, N, h, d), torch.bfloat16, v) for h, v in zip(heads, x)]
    w = [torch.randn(d, device="cuda", generator=g).bfloat16() for _ in heads]
    cos, sin = table(n_rot, d, g)
    nothing = torch.zeros(B, 0, dtype=torch.int32, device="cuda")
    rows = []
    for i in (0, 1):
        st = A.bhnd_strides(N, heads[i], d)
        rows.append(A.head_rows(y[i].t, st, y[i].t, st, heads[i], nothing if i == empty else None, 0, w[i]))
    A.astraea_qk_norm_rotate(rows, cos, sin, n_rot, B, N, d, A.NORM_RMS, A.ROTATE_HALF, EPS)
    assert torch.equal(y[empty].t, x[empty])
    full = 1 - empty
    some = torch.cat([torch.arange(60), torch.arange(5380, 5420), torch.arange(N - 20, N)])
    want, z = reference(x[full][:, some], some.expand(B, -1), n_rot, cos, sin, w[full], None, A.NORM_RMS, A.ROTATE_HALF)
    close(y[full].t[:, some], want, z, False)
    y[0].check(); y[1].check()
