"""astraea_quantize_fp8(_weight) and astraea_gathered_linear_fp8 against their formulas in 64 bits."""
import pytest
import torch

from helpers import Guarded
from paper_2506_05096_b200 import binding as A

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


def lists(g, B, N, M):
    return torch.stack([torch.randperm(N, device="cuda", generator=g)[:M].sort().values for _ in range(B)]).int()


def check_codes(q, scale, x):
    """q, x [R, K]; scale [R, K / 128]: a scale is off by two roundings of fp32, a code by half a step of e4m3 (2^-4 of the value, 2^-10
    below 2^-6) and what fp32 adds to it."""
    blocks = x.double().unflatten(1, (-1, 128))
    want = blocks.abs().amax(2).clamp(min=2.0 ** -100) / 448
    assert ((scale.double() - want).abs() <= 2.0 ** -22 * want).all()
    v = blocks / want[..., None]
    err = (q.double().unflatten(1, (-1, 128)) - v).abs()
    assert (err <= torch.maximum(2.0 ** -4 * v.abs(), torch.tensor(2.0 ** -10, device="cuda", dtype=torch.float64)) * (1 + 2.0 ** -18)).all()
    assert (q.double().abs() <= 448).all()


@pytest.mark.parametrize("B,N,M,K", [(1, 1, 1, 128), (2, 9, 5, 256), (1, 300, 77, 1152), (3, 50, 50, 384), (1, 40, 3, 12288), (2, 5000, 4001, 640)])
def test_rows(B, N, M, K):
    g = torch.Generator("cuda").manual_seed(K + M)
    x = (torch.randn(B, N, K, device="cuda", generator=g) * torch.exp(3 * torch.randn(B, N, 1, device="cuda", generator=g))).bfloat16()
    x[0, :, :128] = 0                                              # a block of zeros
    if K > 128:
        x[-1, 0, 128:256] = 2.0 ** -130                             # one below the least scale
    idx = lists(g, B, N, M)
    q, s = Guarded((B * M, K), torch.uint8), Guarded((K // 128, B * M), torch.float32)
    ws = A.new_workspace(A.OP_QUANTIZE_FP8, B, 0, N, M, K)
    A.astraea_quantize_fp8(x, idx, M, q.t, s.t, B, N, K, workspace=ws)
    A.astraea_poll_error(ws)
    rows = x[torch.arange(B, device="cuda")[:, None], idx.long()].flatten(0, 1)
    check_codes(q.t.view(F8), s.t.t(), rows)
    q.check(); s.check()
    q2, s2 = torch.zeros_like(q.t), torch.zeros_like(s.t)          # the same rows, compact
    A.astraea_quantize_fp8(rows.contiguous(), idx, M, q2, s2, B, N, K, flags=A.LINEAR_COMPACT_IN)
    assert torch.equal(q2, q.t) and torch.equal(s2, s.t)
    if M == N:
        A.astraea_quantize_fp8(x, None, 0, q2.zero_(), s2.zero_(), B, N, K)
        assert torch.equal(q2, q.t) and torch.equal(s2, s.t)


def test_ties_go_to_the_even_code_and_nothing_saturates_early():
    """With a largest value of 448 the scale is one, so that codes are the values rounded: all ties between neighbours, both signs."""
    codes = torch.arange(127, device="cuda", dtype=torch.uint8).view(F8).float()
    ties = (codes[1:] + codes[:-1]) / 2                            # exact in bf16: five significant bits
    x = torch.zeros(2, 128, device="cuda")
    x[0, :126], x[0, 127] = ties, 448
    x[1, :126], x[1, 127] = -ties, 448
    q, s = torch.zeros(2, 128, device="cuda", dtype=torch.uint8), torch.zeros(1, 2, device="cuda")
    A.astraea_quantize_fp8(x.bfloat16(), None, 0, q, s, 1, 2, 128)
    assert (s == 1).all()
    even = torch.arange(126, device="cuda") // 2 * 2
    even = torch.where(torch.arange(126, device="cuda") % 2 == 0, even, even + 2).to(torch.uint8)
    assert torch.equal(q[0, :126], even) and torch.equal(q[1, :126], even + 128) and int(q[0, 127]) == 126


def test_nan_and_infinity_stay_in_their_blocks():
    x = torch.ones(1, 3, 256, device="cuda").bfloat16()
    x[0, 0, 3], x[0, 1, 200], x[0, 2, :128] = float("nan"), float("inf"), float("nan")
    q, s = torch.zeros(3, 256, device="cuda", dtype=torch.uint8), torch.zeros(2, 3, device="cuda")
    A.astraea_quantize_fp8(x, None, 0, q, s, 1, 3, 256)
    v = q.view(F8).float().unflatten(1, (2, 128)) * s.t()[..., None]
    assert bool(v[0, 0, 3].isnan()) and int(v[0].isnan().sum()) == 1 and bool((v[0, 0, :3] - 1).abs().max() < 0.01)
    assert bool(v[1, 1].isnan().all()) and bool(v[1, 0].isfinite().all())
    assert bool(v[2, 0].isnan().all()) and bool(v[2, 1].isfinite().all())


@pytest.mark.parametrize("N_out,K", [(8, 128), (128, 256), (136, 384), (1000, 1152)])
def test_weights(N_out, K):
    g = torch.Generator("cuda").manual_seed(N_out)
    w = (torch.randn(N_out, K, device="cuda", generator=g) * torch.exp(torch.randn(N_out, 1, device="cuda", generator=g))).bfloat16()
    nb = -(-N_out // 128)
    q, s = Guarded((N_out, K), torch.uint8), Guarded((nb, K // 128), torch.float32)
    A.astraea_quantize_fp8_weight(w, q.t, s.t, N_out, K)
    q.check(); s.check()
    padded = torch.zeros(nb * 128, K, device="cuda", dtype=torch.float64)
    padded[:N_out] = w.double()
    tiles = padded.unflatten(0, (nb, 128)).unflatten(2, (-1, 128)).permute(0, 2, 1, 3).flatten(2)      # [nb, kb, 128 * 128]
    want = tiles.abs().amax(2) / 448
    assert ((s.t.double() - want).abs() <= 2.0 ** -22 * want).all()
    v = w.double() / want.repeat_interleave(128, 0)[:N_out].repeat_interleave(128, 1)
    err = (q.t.view(F8).double() - v).abs()
    assert (err <= torch.maximum(2.0 ** -4 * v.abs(), torch.tensor(2.0 ** -10, device="cuda", dtype=torch.float64)) * (1 + 2.0 ** -18)).all()


def operands(g, R, N_out, K):
    e4m3 = lambda r: (torch.randn(r, K, device="cuda", generator=g) * 120).clamp(-448, 448).to(F8)
    xq, wq = e4m3(R), e4m3(N_out)
    xs = torch.exp(torch.randn(K // 128, R, device="cuda", generator=g)) / 100
    ws = torch.exp(torch.randn(-(-N_out // 128), K // 128, device="cuda", generator=g)) / 100 / K ** 0.5
    return xq, xs, wq, ws


def product(xq, xs, wq, ws, N_out):
    x = xq.double() * xs.double().t().repeat_interleave(128, 1)
    w = wq.double() * ws.double().repeat_interleave(128, 0)[:N_out].repeat_interleave(128, 1)
    return x @ w.t(), x.abs() @ w.abs().t()


def close(got, want, mass, K, factor=1.0):
    # one rounding to bf16; sums of 128 products in fp32 and K / 128 sums of those, each within 2^-24 of the sum of the magnitudes
    bound = 2.0 ** -8 * want.abs() + factor * (128 + 2 * K / 128 + 4) * 2.0 ** -24 * mass + 1e-30
    excess = (got.double() - want).abs() - bound
    assert excess.max() <= 0, (float(excess.max()), float(((got.double() - want).abs() / bound).max()))


@pytest.mark.parametrize("B,N,M,K,N_out", [(1, 4, 1, 128, 8), (1, 300, 77, 384, 200), (2, 150, 130, 1152, 264), (1, 600, 513, 256, 520),
                                           (3, 40, 33, 2432, 64), (1, 9, 2, 12288, 24), (2, 20, 4, 1152, 4608), (1, 30, 9, 256, 136), (2, 40, 8, 640, 2056),
                                           (1, 40, 32, 384, 1000), (3, 30, 21, 1408, 72), (1, 64, 64, 4096, 520), (1, 80, 65, 4096, 520), (1, 256, 256, 128, 256), (1, 20000, 19000, 256, 1000), (2, 3000, 2999, 512, 2056),
                                           (1, 9000, 8200, 3200, 1032), (1, 9000, 8999, 128, 2048), (1, 5000, 4999, 1408, 2056)])
def test_layer(B, N, M, K, N_out):
    g = torch.Generator("cuda").manual_seed(N_out + K)
    xq, xs, wq, ws = operands(g, B * M, N_out, K)
    idx = lists(g, B, N, M)
    before = torch.randn(B, N, N_out, device="cuda", generator=g).bfloat16()
    y = Guarded((B, N, N_out), torch.bfloat16, before)
    work = A.new_workspace(A.OP_GATHERED_LINEAR_FP8, B, 0, N, M, K)
    A.astraea_gathered_linear_fp8(xq, xs, idx, M, wq, ws, None, None, None, y.t, B, N, K, N_out, workspace=work)
    A.astraea_poll_error(work)
    want, mass = product(xq, xs, wq, ws, N_out)
    rows = torch.arange(B, device="cuda")[:, None]
    close(y.t[rows, idx.long()].flatten(0, 1), want, mass, K)
    rest = torch.ones(B, N, dtype=torch.bool, device="cuda")
    rest[rows, idx.long()] = False
    assert torch.equal(y.t[rest], before[rest])
    y.check()


@pytest.mark.parametrize("N_out", [72, 264, 2056])
@pytest.mark.parametrize("bias,gelu,gate,residual", [(1, 0, 0, 0), (1, 1, 0, 0), (0, 1, 0, 0), (0, 0, 1, 0), (0, 0, 0, 1), (1, 0, 1, 1), (1, 1, 1, 1)])
@pytest.mark.parametrize("compact", [False, True])
@pytest.mark.parametrize("M", [150, 7])
def test_epilogue(N_out, bias, gelu, gate, residual, compact, M):
    g = torch.Generator("cuda").manual_seed(N_out)
    B, N, K = 3, 200, 384                                           # tiles that hold rows of two batch elements
    xq, xs, wq, ws = operands(g, B * M, N_out, K)
    idx = lists(g, B, N, M)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    bi, ga = rnd(N_out) if bias else None, rnd(B, N_out) if gate else None
    re = rnd(B, M if compact else N, N_out) if residual else None
    y = Guarded((B, M if compact else N, N_out), torch.bfloat16)
    work = A.new_workspace(A.OP_GATHERED_LINEAR_FP8, B, 0, N, M, K)
    flags = (A.LINEAR_GELU if gelu else 0) | (A.LINEAR_COMPACT_OUT if compact else 0) | (A.LINEAR_COMPACT_RES if compact and residual else 0)
    A.astraea_gathered_linear_fp8(xq, xs, idx, M, wq, ws, bi, re, ga, y.t, B, N, K, N_out, flags=flags, workspace=work)
    A.astraea_poll_error(work)
    y.check()
    rows = torch.arange(B, device="cuda")[:, None]
    want, mass = product(xq, xs, wq, ws, N_out)
    if bias:
        want, mass = want + bi.double(), mass + bi.double().abs()
    if gelu:                                                        # slope at most 1.13, erf within 1.5e-7
        want, mass = want * torch.special.ndtr(want), 1.13 * mass + 2.0 ** 17 * 1.5e-7 * want.abs()
    want, mass = want.unflatten(0, (B, M)), mass.unflatten(0, (B, M))
    if gate:
        want, mass = want * ga.double()[:, None], mass * ga.double().abs()[:, None] + want.abs() * 2.0 ** -6
    if residual:
        r = (re if compact else re[rows, idx.long()]).double()
        want, mass = want + r, mass + r.abs() * 2.0 ** -6
    close(y.t if compact else y.t[rows, idx.long()], want, mass, K)


def test_all_rows_without_a_list_and_a_whole_run_from_bf16():
    g = torch.Generator("cuda").manual_seed(5)
    B, N, K, N_out = 2, 333, 640, 392
    x = torch.randn(B, N, K, device="cuda", generator=g).bfloat16()
    w = (torch.randn(N_out, K, device="cuda", generator=g) / K ** 0.5).bfloat16()
    xq, xs = torch.empty(B * N, K, device="cuda", dtype=torch.uint8), torch.empty(K // 128, B * N, device="cuda")
    wq, ws = torch.empty(N_out, K, device="cuda", dtype=torch.uint8), torch.empty(4, K // 128, device="cuda")
    y = torch.empty(B, N, N_out, device="cuda", dtype=torch.bfloat16)
    work = A.new_workspace(A.OP_GATHERED_LINEAR_FP8, B, 0, N, N, K)
    A.astraea_quantize_fp8(x, None, 0, xq, xs, B, N, K)
    A.astraea_quantize_fp8_weight(w, wq, ws, N_out, K)
    A.astraea_gathered_linear_fp8(xq, xs, None, 0, wq, ws, None, None, None, y, B, N, K, N_out, workspace=work)
    want, mass = product(xq.view(F8), xs, wq.view(F8), ws, N_out)
    close(y.flatten(0, 1), want, mass, K)
    # against the layer in bf16: every operand is off by at most 2^-4 of itself, two of them, errors of random sign
    full = x.double().flatten(0, 1) @ w.double().t()
    assert (y.double().flatten(0, 1) - full).norm() < 0.05 * full.norm()


def test_bad_entries_are_skipped_and_reported():
    g = torch.Generator("cuda").manual_seed(6)
    N, M, K, N_out = 16, 5, 128, 64
    xq, xs, wq, ws = operands(g, M, N_out, K)
    idx = torch.tensor([[1, 4, 4, 77, 9]], device="cuda", dtype=torch.int32)
    y = torch.full((1, N, N_out), 7.0, device="cuda").bfloat16()
    work = A.new_workspace(A.OP_GATHERED_LINEAR_FP8, 1, 0, N, M, K)
    A.astraea_gathered_linear_fp8(xq, xs, idx, M, wq, ws, None, None, None, y, 1, N, K, N_out, workspace=work)
    with pytest.raises(A.AstraeaError) as e:
        A.astraea_poll_error(work)
    assert e.value.code == A.ERR_BAD_INDEX
    want, mass = product(xq, xs, wq, ws, N_out)
    close(y[0, [1, 4]], want[:2], mass[:2], K)
    assert bool((y[0, [i for i in range(N) if i not in (1, 4)]] == 7).all())
    x = torch.randn(1, N, K, device="cuda").bfloat16()
    q, s = torch.full((M, K), 9, device="cuda", dtype=torch.uint8), torch.full((1, M), 9.0, device="cuda")
    A.astraea_quantize_fp8(x, idx, M, q, s, 1, N, K, workspace=work)
    with pytest.raises(A.AstraeaError) as e:
        A.astraea_poll_error(work)
    assert e.value.code == A.ERR_BAD_INDEX
    check_codes(q[:2].view(F8), s[:, :2].t(), x[0, [1, 4]])
    assert bool((q[2:] == 9).all()) and bool((s[0, 2:] == 9).all())
    A.astraea_gathered_linear_fp8(xq, xs, idx[:, :0].contiguous(), 0, wq, ws, None, None, None, y, 1, N, K, N_out, workspace=work)
    A.astraea_poll_error(work)


@pytest.mark.parametrize("R", [300, 50])
def test_a_row_of_nan_stays_alone_and_runs_repeat(R):
    g = torch.Generator("cuda").manual_seed(8)
    K, N_out = 1152, 520
    xq, xs, wq, ws = operands(g, R, N_out, K)
    y, again = (torch.empty(1, R, N_out, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    work = A.new_workspace(A.OP_GATHERED_LINEAR_FP8, 1, 0, R, R, K)
    call = lambda out: A.astraea_gathered_linear_fp8(xq, xs, None, 0, wq, ws, None, None, None, out, 1, R, K, N_out, workspace=work)
    call(y); call(again)
    assert torch.equal(y, again)
    xq.view(torch.uint8)[17, 5] = 0x7F
    xs[3, 44] = float("inf")
    call(again)
    assert bool(again[0, 17].isnan().all()) and not bool(again[0, 44].isfinite().any())
    others = [r for r in range(R) if r not in (17, 44)]
    assert torch.equal(again[0, others], y[0, others])


@pytest.mark.parametrize("N_out", [40, 264, 2056])
@pytest.mark.parametrize("residual", [False, True])
def test_bad_entries_among_compact_rows(N_out, residual):
    """Compact rows go out 32 at a time, unless one of them is not to be written."""
    g = torch.Generator("cuda").manual_seed(N_out)
    B, N, M, K = 2, 900, 700, 384
    xq, xs, wq, ws = operands(g, B * M, N_out, K)
    idx = lists(g, B, N, M)
    bad = {(0, 5): N, (0, 40): -1, (1, 699): 1 << 20, (1, 0): N + 3}
    for (b, r), v in bad.items():
        idx[b, r] = v
    idx[0, 300] = idx[0, 299]                                       # does not exceed its predecessor
    skipped = torch.zeros(B, M, dtype=torch.bool, device="cuda")
    for b, r in list(bad) + [(0, 300)]:
        skipped[b, r] = True
    # the entry behind one that is too large does not exceed it either; the one behind -1 does
    for b, r in ((0, 5), (1, 0)):
        skipped[b, r + 1] = True
    before = torch.randn(B, M, N_out, device="cuda", generator=g).bfloat16()
    y = Guarded((B, M, N_out), torch.bfloat16, before)
    work = A.new_workspace(A.OP_GATHERED_LINEAR_FP8, B, 0, N, M, K)
    flags = A.LINEAR_COMPACT_OUT | (A.LINEAR_COMPACT_RES if residual else 0)
    A.astraea_gathered_linear_fp8(xq, xs, idx, M, wq, ws, None, y.t if residual else None, None, y.t, B, N, K, N_out, flags=flags, workspace=work)
    with pytest.raises(A.AstraeaError):
        A.astraea_poll_error(work)
    want, mass = product(xq, xs, wq, ws, N_out)
    want, mass = want.unflatten(0, (B, M)), mass.unflatten(0, (B, M))
    if residual:                                                    # in place
        want, mass = want + before.double(), mass + before.double().abs() * 2.0 ** -6
    close(y.t[~skipped], want[~skipped], mass[~skipped], K)
    assert torch.equal(y.t[skipped], before[skipped])
    y.check()


@pytest.mark.parametrize("B,N,K,N_out", [(1, 4097, 256, 1160), (3, 700, 1152, 520), (1, 20000, 128, 264)])
def test_all_rows_in_place_over_many_tiles(B, N, K, N_out):
    g = torch.Generator("cuda").manual_seed(N)
    xq, xs, wq, ws = operands(g, B * N, N_out, K)
    before = torch.randn(B, N, N_out, device="cuda", generator=g).bfloat16()
    y = Guarded((B, N, N_out), torch.bfloat16, before)
    work = A.new_workspace(A.OP_GATHERED_LINEAR_FP8, B, 0, N, N, K)
    A.astraea_gathered_linear_fp8(xq, xs, None, 0, wq, ws, None, y.t, None, y.t, B, N, K, N_out, workspace=work)
    A.astraea_poll_error(work)
    want, mass = product(xq, xs, wq, ws, N_out)
    close(y.t.flatten(0, 1), want + before.double().flatten(0, 1), mass + before.double().flatten(0, 1).abs() * 2.0 ** -6, K)
    y.check()
