"""Window attention in CTAs some of whose rows do not exist: behind the last row of a list, or entries that are skipped."""
import math

import pytest
import torch

from helpers import Guarded
from paper_2506_05096_b200 import binding as A
from test_gpu_window_attn import check, reference

pytestmark = pytest.mark.gpu


def call(q, k, v, idx, kv_len, N, n_first, left, right, flags=A.ATTN_COMPACT_Q | A.ATTN_COMPACT_OUT, bad=False):
    B, M, H, d = q.shape
    H_kv = k.shape[2]
    out, lse = torch.full_like(q, 7.0), torch.full((B, H, M), 7.0, device="cuda")
    ws = A.new_workspace(A.OP_WINDOW_ATTN, B, H, N, M, d)
    kv = A.bhnd_strides(N, H_kv, d)
    A.astraea_window_attn(q, k, v, A.bhnd_strides(M, H, d), kv, kv, idx, M, out, lse, B, H, H_kv, N, d, n_first, 0, left, right, kv_len, flags=flags, workspace=ws)
    if bad:
        with pytest.raises(A.AstraeaError) as e:
            A.astraea_poll_error(ws)
        assert e.value.code == A.ERR_BAD_INDEX
    else:
        A.astraea_poll_error(ws)
    return out, lse


@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("H,H_kv", [(4, 1), (2, 2), (40, 1)])
@pytest.mark.parametrize("N,p,left,n_first", [(400, 130, 100, 16), (400, 130, 100, 0), (400, 130, 399, 0), (3000, 2100, 2040, 7), (3000, 2100, 64, 1), (3000, 2100, 2999, 64)])
@pytest.mark.parametrize("fill", [float("nan"), float("inf")])
def test_single_tokens_before_keys_that_were_never_written(d, H, H_kv, N, p, left, n_first, fill):
    """Windows that begin at key 0, within the first 64 keys and behind them."""
    g = torch.Generator("cuda").manual_seed(d + N)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    q, k, v = rnd(2, 1, H, d), rnd(2, N, H_kv, d), rnd(2, N, H_kv, d)
    kv_len = torch.tensor([p + 1, p - 20], device="cuda", dtype=torch.int32)
    for b in range(2):
        k[b, int(kv_len[b]):], v[b, int(kv_len[b]):] = fill, fill
    idx = (kv_len - 1)[:, None].contiguous()
    out, lse = call(q, k, v, idx, kv_len, N, n_first, left, 0)
    for b in range(2):                                            # (no row sees them)
        k[b, int(kv_len[b]):], v[b, int(kv_len[b]):] = 0, 0
    want, want_lse = reference(q, k, v, idx, N, n_first, 0, left, 0, kv_len, 1 / math.sqrt(d))
    check(out, lse, want, want_lse)


@pytest.mark.parametrize("d", [64, 72, 128])
def test_skipped_entries_hold_nothing_back(d):
    """Their query rows are NaN, and their positions out of every other row's reach."""
    g = torch.Generator("cuda").manual_seed(d)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    B, N, H, M = 1, 2000, 2, 300
    q, k, v = rnd(B, M, H, d), rnd(B, N, H, d), rnd(B, N, H, d)
    idx = torch.arange(M, device="cuda", dtype=torch.int32)[None].contiguous() + 1500
    skipped = [10, 100, 200]
    idx[0, 10], idx[0, 100], idx[0, 200] = 40, -1, N             # below its predecessor, out of range on either side
    good = [r for r in range(M) if r not in skipped + [201]]      # (the entry behind N does not exceed it)
    q[0, skipped] = float("nan")
    kv_len = torch.tensor([1700], device="cuda", dtype=torch.int32)
    k[0, 1700:], v[0, 1700:] = float("nan"), float("nan")
    out, lse = call(q, k, v, idx, kv_len, N, 3, 90, 10, bad=True)
    k[0, 1700:], v[0, 1700:] = 0, 0
    want, want_lse = reference(q[:, good], k, v, idx[:, good], N, 3, 0, 90, 10, kv_len, 1 / math.sqrt(d))
    check(out[:, good], lse[:, :, good], want, want_lse)
    rest = skipped + [201]
    assert bool((out[:, rest] == 7).all()) and bool((lse[:, :, rest] == 7).all())


@pytest.mark.parametrize("d", [64, 72])
@pytest.mark.parametrize("M", [129, 200, 256])
def test_the_workspace_asked_for_holds_every_share_of_small_ctas(d, M):
    """A call of two units of 128 rows is shared out as far with the bytes of astraea_workspace_bytes as with any more, and stays inside them."""
    g = torch.Generator("cuda").manual_seed(M + d)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    N = 9000
    q, k, v = rnd(1, M, 1, d), rnd(1, N, 1, d), rnd(1, N, 1, d)
    idx = (torch.arange(M, device="cuda", dtype=torch.int32)[None] * 35).contiguous()
    asked = A.new_workspace(A.OP_WINDOW_ATTN, 1, 1, N, M, d).numel()
    results = []
    for size in (asked, asked + (64 << 20)):
        ws = Guarded((size + 4096,), torch.uint8)                 # (a workspace begins at a multiple of 256 bytes)
        skip = -ws.t.data_ptr() % 256
        ws.t[skip:skip + size] = 0
        behind = ws.t[skip + size:].clone()
        out, lse = torch.zeros_like(q), torch.zeros(1, 1, M, device="cuda")
        st = A.bhnd_strides(N, 1, d)
        A.astraea_window_attn(q, k, v, A.bhnd_strides(M, 1, d), st, st, idx, M, out, lse, 1, 1, 1, N, d, 0, 0, N, N,
                              flags=A.ATTN_COMPACT_Q | A.ATTN_COMPACT_OUT | A.ATTN_SMALL_CTAS, workspace=ws.t[skip:skip + size])
        A.astraea_poll_error(ws.t[skip:skip + size])
        ws.check()
        assert torch.equal(ws.t[skip + size:], behind)
        want, want_lse = reference(q, k, v, idx, N, 0, 0, N, N, None, 1 / math.sqrt(d))
        check(out, lse, want, want_lse)
        results.append((out, lse))
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])
