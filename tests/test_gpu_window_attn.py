"""astraea_window_attn against the definition in 64 bits: windows, first and last keys, lengths, shared heads, single tokens, masked NaN."""
import math

import pytest
import torch

from helpers import Guarded, assert_attn_close
from paper_2506_05096_b200 import binding as A

pytestmark = pytest.mark.gpu


def visible(tok, N, n_first, n_last, left, right, length):
    j, i = torch.arange(N, device="cuda"), tok.long()[:, None]
    return (j < length) & ((j < n_first) | (j >= N - n_last) | ((j >= i - left) & (j <= i + right)))


def reference(q, k, v, tok, N, n_first, n_last, left, right, kv_len, scale):
    """q [B, M, H, d], k, v [B, N, H_kv, d], tok [B, M]: out [B, M, H, d], lse [B, H, M] in fp64; a value counts where it is seen only."""
    B, M, H, d = q.shape
    G = H // k.shape[2]
    out, lse = torch.zeros(B, M, H, d, device="cuda", dtype=torch.float64), torch.zeros(B, H, M, device="cuda", dtype=torch.float64)
    for b in range(B):
        see = visible(tok[b], N, n_first, n_last, left, right, N if kv_len is None else int(kv_len[b]))
        for h in range(H):
            s = torch.where(see, q[b, :, h].double() @ torch.where(see.any(0)[:, None], k[b, :, h // G].double(), 0.0).t() * scale, -math.inf)
            z = torch.logsumexp(s, 1)
            p = torch.where(see, torch.exp(s - torch.where(z == -math.inf, 0.0, z)[:, None]), 0.0)
            val = v[b, :, h // G].double()
            odd = ~val.isfinite()
            o = p @ torch.where(odd, 0.0, val)
            for j in odd.any(1).nonzero()[:, 0].tolist():
                o = o + torch.where(see[:, j, None] & odd[j], val[j], 0.0)
            out[b, :, h], lse[b, h] = o, z
    return out, lse


def lists(g, B, N, M):
    return torch.stack([torch.randperm(N, device="cuda", generator=g)[:M].sort().values for _ in range(B)]).int()


def check(out, lse, want, want_lse, what=""):
    empty = want_lse == -math.inf
    assert torch.equal(lse == -math.inf, empty), what
    # A logit is a sum of d products in fp32: d roundings of 2^-24 of it.  The exponentials' arguments are differences of numbers that reach 1.44
    # |logit| + 48, rounded four times (the scale in log2 units, the reference's product, the difference, the LSE's own sum), where the reference may
    # lie 100 above a row that does not see its key: 4 * 2^-24 * 200 = 5e-5.  The exponentials themselves are good to 2e-7.
    err = (lse.double() - want_lse)[~empty].abs() - (5e-5 + (out.shape[-1] + 8) * 2.0 ** -24 * want_lse[~empty].abs())
    assert err.max() <= 0 if (~empty).any() else True, (what, float(err.max()))
    rows = (~empty).transpose(1, 2)
    assert (out.double()[~rows] == 0).all(), what
    if rows.any():
        assert_attn_close(out.double()[rows].cpu().numpy(), want[rows].cpu().numpy(), what=what)


def run(g, B, N, M, H, H_kv, d, n_first=0, n_last=0, left=0, right=0, kv_len=None, compact=False, flags=0, amp=1.0, idx=None, small_ws=False, qkv=None):
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    idx = lists(g, B, N, M) if idx is None else idx
    q, k, v = qkv or (amp * rnd(B, M if compact else N, H, d), rnd(B, N, H_kv, d), rnd(B, N, H_kv, d))
    before, before_lse = rnd(*q.shape), torch.randn(B, H, q.shape[1], device="cuda", generator=g)
    out, lse = Guarded(q.shape, torch.bfloat16, before), Guarded((B, H, q.shape[1]), torch.float32, before_lse)
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda") if small_ws else A.new_workspace(A.OP_WINDOW_ATTN, B, H, N, M, d)
    kv = A.bhnd_strides(N, H_kv, d)
    A.astraea_window_attn(q, k, v, A.bhnd_strides(q.shape[1], H, d), kv, kv, idx, M, out.t, lse.t, B, H, H_kv, N, d, n_first, n_last, left, right, kv_len,
                          flags=flags | (A.ATTN_COMPACT_Q | A.ATTN_COMPACT_OUT if compact else 0), workspace=ws)
    A.astraea_poll_error(ws)
    rows = torch.arange(B, device="cuda")[:, None]
    got, got_lse, ql = out.t, lse.t, q
    if not compact:
        got, ql = out.t[rows, idx.long()], q[rows, idx.long()]
        got_lse = lse.t.transpose(1, 2)[rows, idx.long()].transpose(1, 2)
        rest = torch.ones(B, N, dtype=torch.bool, device="cuda")
        rest[rows, idx.long()] = False
        assert torch.equal(out.t[rest], before[rest]) and torch.equal(lse.t.transpose(1, 2)[rest], before_lse.transpose(1, 2)[rest])
    want, want_lse = reference(ql, k, v, idx, N, n_first, n_last, left, right, kv_len, 1 / math.sqrt(d))
    out.check(); lse.check()
    return got, got_lse, want, want_lse


@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("N,M,left,right,n_first,n_last", [
    (1, 1, 0, 0, 0, 0), (64, 64, 0, 0, 0, 0), (65, 65, 5, 3, 0, 0), (300, 140, 20, 0, 7, 0), (300, 140, 0, 40, 0, 9), (700, 700, 100, 100, 64, 64),
    (1000, 129, 63, 64, 1, 1), (1000, 257, 1000, 0, 0, 0), (1000, 31, 2000000000, 2000000000, 0, 0), (513, 300, 17, 17, 513, 0), (513, 300, 17, 17, 0, 513),
    (2000, 600, 300, 300, 100, 77), (9000, 500, 8000, 500, 0, 0)])
@pytest.mark.parametrize("flags", [0, A.ATTN_SMALL_CTAS])
def test_windows(d, N, M, left, right, n_first, n_last, flags):
    g = torch.Generator("cuda").manual_seed(N + d)
    check(*run(g, 2, N, M, 3, 3, d, n_first, n_last, left, right, flags=flags))


@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("H,H_kv", [(4, 2), (6, 2), (8, 1), (40, 1)])
@pytest.mark.parametrize("M,compact", [(1, True), (3, True), (90, False)])
def test_shared_heads(d, H, H_kv, M, compact):
    g = torch.Generator("cuda").manual_seed(H + d)
    check(*run(g, 2, 777, M, H, H_kv, d, 5, 11, 200, 30, compact=compact))


@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("small_ws", [False, True])
def test_single_tokens_over_caches_of_different_lengths(d, small_ws):
    g = torch.Generator("cuda").manual_seed(d)
    B, N = 6, 5000
    kv_len = torch.tensor([1, 64, 65, 4999, 5000, 2500], device="cuda", dtype=torch.int32)
    idx = (kv_len - 1)[:, None].contiguous()
    for left, n_first in ((4999, 0), (1023, 16), (100, 300), (0, 0)):
        check(*run(g, B, N, 1, 8, 2, d, n_first, 0, left, 0, kv_len, compact=True, idx=idx, small_ws=small_ws), what=(left, n_first))


@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_see_nothing(d):
    g = torch.Generator("cuda").manual_seed(d)
    # lengths of zero, out of range, and shorter than most windows begin
    kv_len = torch.tensor([0, -3, 150, 9999], device="cuda", dtype=torch.int32)
    check(*run(g, 4, 900, 400, 2, 1, d, 0, 0, 50, 10, kv_len))
    check(*run(g, 4, 900, 400, 2, 1, d, 3, 20, 50, 10, kv_len))
    check(*run(g, 4, 900, 1, 2, 1, d, 0, 0, 600, 0, torch.tensor([0, 1, 100, 900], device="cuda", dtype=torch.int32), compact=True,
               idx=torch.tensor([[899], [0], [750], [899]], device="cuda", dtype=torch.int32)))


@pytest.mark.parametrize("d", [64, 72, 128])
def test_what_is_not_seen_may_be_nan_and_what_is_seen_counts(d):
    g = torch.Generator("cuda").manual_seed(d)
    B, N, M, H = 2, 1500, 1000, 2
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    q, k, v = rnd(B, N, H, d), rnd(B, N, H, d), rnd(B, N, H, d)
    kv_len = torch.tensor([700, 1500], device="cuda", dtype=torch.int32)
    k[0, 700:], v[0, 700:] = float("nan"), float("inf")            # memory behind a length
    # values that some rows of a tile see and others do not
    v[1, 400, 0, 3], v[1, 401, 1, 4], v[1, 777, 0, d - 1] = float("nan"), float("inf"), float("-inf")
    v[1, 402, 1, 4] = float("-inf")                                # rows that see both: NaN
    v[1, 2, 0, 5] = float("inf")                                   # a first key that all see
    got, lse, want, want_lse = run(g, B, N, M, H, H, d, 4, 0, 40, 0, kv_len, qkv=(q, k, v))
    assert torch.equal(got.double().isnan(), want.isnan()) and torch.equal(got.double().isinf(), want.isinf())
    assert torch.equal(got.double()[want.isinf()], want[want.isinf()])
    fine = want.isfinite()
    check(torch.where(fine, got, 0), lse, torch.where(fine, want, 0.0), want_lse)
    # a key of NaN makes the rows that see it NaN and no other
    k[1, 900, 1, 0] = float("nan")
    got, lse, want, want_lse = run(g, B, N, M, H, H, d, 4, 0, 40, 0, kv_len, qkv=(q, k, v.nan_to_num(0, 0, 0)))
    assert torch.equal(lse.isnan(), want_lse.isnan()) and int(lse.isnan().sum()) > 0
    assert torch.equal(got.isnan().any(-1), want.isnan().any(-1)) and torch.equal(got.isnan().all(-1), want.isnan().all(-1))
    fine = ~want_lse.isnan()
    check(torch.where(fine.transpose(1, 2)[..., None], got, 0), torch.where(fine, lse, 0.0), torch.where(fine.transpose(1, 2)[..., None], want, 0.0), torch.where(fine, want_lse, 0.0))


@pytest.mark.parametrize("d", [64, 72, 128])
def test_hidden_logits_far_above_the_seen_ones(d):
    """The running reference comes from keys that a row may not see: where those lie hundreds of nats above what it sees, its terms would
    all be zero against it."""
    g = torch.Generator("cuda").manual_seed(d)
    B, N, M, H = 1, 400, 400, 2
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    q, k, v = rnd(B, N, H, d), rnd(B, N, H, d), rnd(B, N, H, d)
    q[..., 0] = 8.0
    k[0, :, 0, 0] = 0.25
    k[0, 5, 0, 0] = 60 * math.sqrt(d)                              # hidden from the rows behind it; 480 nats
    k[0, 200, 1, 0] = -60 * math.sqrt(d)
    check(*run(g, B, N, M, H, H, d, 0, 0, 3, 3, qkv=(q, k, v)))
    check(*run(g, B, N, M, H, H, d, 1, 0, 100, 0, qkv=(q, k, v)))


def test_lists_that_are_null_bad_or_empty():
    g = torch.Generator("cuda").manual_seed(1)
    B, N, H, d = 1, 600, 2, 64
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    q, k, v = rnd(B, N, H, d), rnd(B, N, H, d), rnd(B, N, H, d)
    st = A.bhnd_strides(N, H, d)
    ws = A.new_workspace(A.OP_WINDOW_ATTN, B, H, N, N, d)
    out, lse = torch.full_like(q, 7.0), torch.zeros(B, H, N, device="cuda")
    A.astraea_window_attn(q, k, v, st, st, st, None, 300, out, lse, B, H, H, N, d, left=30, right=5, workspace=ws)     # rows 0 .. 299
    A.astraea_poll_error(ws)
    tok = torch.arange(300, device="cuda")[None]
    want, want_lse = reference(q[:, :300], k, v, tok, N, 0, 0, 30, 5, None, 1 / 8)
    check(out[:, :300], lse[:, :, :300], want, want_lse)
    assert bool((out[:, 300:] == 7).all())
    out.fill_(7)
    idx = torch.tensor([[3, 590, 50, 50, 700, -1, 599]], device="cuda", dtype=torch.int32)      # 50 after 590, twice, out of range
    A.astraea_window_attn(q, k, v, st, st, st, idx, 7, out, lse, B, H, H, N, d, left=30, right=5, workspace=ws)
    with pytest.raises(A.AstraeaError) as e:
        A.astraea_poll_error(ws)
    assert e.value.code == A.ERR_BAD_INDEX
    good = [3, 590, 599]
    want, want_lse = reference(q[:, good], k, v, torch.tensor([good], device="cuda"), N, 0, 0, 30, 5, None, 1 / 8)
    check(out[:, good], lse[:, :, good], want, want_lse)
    assert bool((out[:, [i for i in range(N) if i not in good]] == 7).all())
    A.astraea_window_attn(q, k, v, st, st, st, idx, 0, out, lse, B, H, H, N, d, workspace=ws)
    A.astraea_poll_error(ws)


def test_strides_scale_and_no_lse():
    g = torch.Generator("cuda").manual_seed(2)
    B, N, H, d = 2, 500, 3, 128
    qkv = torch.randn(B, 3, H, N, d, device="cuda", generator=g).bfloat16()           # head-major, fused
    st = (3 * H * N * d, N * d, d)
    out = torch.zeros(B, N, H, d, device="cuda", dtype=torch.bfloat16)
    ws = A.new_workspace(A.OP_WINDOW_ATTN, B, H, N, N, d)
    A.astraea_window_attn(qkv[:, 0], qkv[:, 1], qkv[:, 2], st, st, st, None, N, out, None, B, H, H, N, d, left=70, right=70, scale=0.3, workspace=ws)
    A.astraea_poll_error(ws)
    q, k, v = (qkv[:, i].transpose(1, 2) for i in range(3))
    want, want_lse = reference(q, k, v, torch.arange(N, device="cuda").expand(B, -1), N, 0, 0, 70, 70, None, 0.3)
    check(out, want_lse.float(), want, want_lse)


@pytest.mark.parametrize("d", [64, 128])
def test_split_by_keys_is_the_unsplit_launch_and_repeats(d):
    g = torch.Generator("cuda").manual_seed(d)
    B, N, M, H = 1, 6000, 700, 4
    args = dict(B=B, N=N, M=M, H=H, H_kv=H, d=d, n_first=50, left=2000, right=2000)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    qkv, idx = (rnd(B, N, H, d), rnd(B, N, H, d), rnd(B, N, H, d)), lists(g, B, N, M)
    split = run(g, **args, qkv=qkv, idx=idx)
    whole = run(g, **args, qkv=qkv, idx=idx, flags=A.ATTN_WHOLE_KEYS)
    again = run(g, **args, qkv=qkv, idx=idx)
    check(*split); check(*whole)
    assert torch.equal(split[0], again[0]) and torch.equal(split[1], again[1])
    assert (split[0].float() - whole[0].float()).abs().max() <= 2.0 ** -7 * whole[0].float().abs().max()


@pytest.mark.parametrize("d", [64, 72, 128])
def test_keys_shared_by_the_batch_and_offsets_past_32_bits(d):
    g = torch.Generator("cuda").manual_seed(d)
    B, N, M, H, H_kv, left, right = 2, 2100, 40, 4, 2, 150, 90
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    q, k, v = rnd(B, N, H, d), rnd(1, N, H_kv, d).expand(B, -1, -1, -1), rnd(1, N, H_kv, d)
    v[0, N - 30, 1, 3] = math.inf                                   # in the last windows
    v = v.expand(B, -1, -1, -1)
    idx = lists(g, B, N, M)
    idx[:, -1] = N - 1
    apart = 1 << 20                                                 # elements between two tokens: the last ones lie 2.2e9 elements in
    room = torch.empty(N * apart, device="cuda", dtype=torch.bfloat16)
    far_k = room.as_strided((N, H_kv, d), (apart, d, 1))
    far_v = room.as_strided((N, H_kv, d), (apart, d, 1), 4 * 128)
    far_k.copy_(k[0]); far_v.copy_(v[0])
    out, lse = torch.zeros(B, M, H, d, device="cuda", dtype=torch.bfloat16), torch.zeros(B, H, M, device="cuda")
    ws = A.new_workspace(A.OP_WINDOW_ATTN, B, H, N, M, d)
    st = (0, d, apart)
    A.astraea_window_attn(q, far_k, far_v, A.bhnd_strides(N, H, d), st, st, idx, M, out, lse, B, H, H_kv, N, d, 0, 0, left, right,
                          flags=A.ATTN_COMPACT_OUT, workspace=ws)
    A.astraea_poll_error(ws)
    rows = torch.arange(B, device="cuda")[:, None]
    want, want_lse = reference(q[rows, idx.long()], k, v, idx, N, 0, 0, left, right, None, 1 / math.sqrt(d))
    odd = ~want.isfinite()
    assert odd.any() and torch.equal(~out.isfinite(), odd)
    check(torch.where(odd, 0.0, out.float()).bfloat16(), lse, torch.where(odd, 0.0, want), want_lse)
