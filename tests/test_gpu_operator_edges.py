"""Calls of the operators beside the path that their limits allow and that an ordinary block does not make: many heads on one key head, rows without a
list, sums over many blocks of channels, tensors of a few heads between caches and compact rows, captured calls on shared inputs."""
import math

import pytest
import torch

from helpers import Guarded
from paper_2506_05096_b200 import binding as A
from test_gpu_head_norm import close as norm_close, reference as norm_reference, table
from test_gpu_linear_fp8 import close as layer_close, lists, operands, product
from test_gpu_window_attn import check, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,group,M", [(64, 4096, 2), (128, 4095, 1), (72, 1000, 3), (64, 257, 5), (128, 129, 7), (72, 127, 9)])
def test_many_query_heads_on_one_key_head(d, group, M):
    """Units of one token's heads, of several tokens', and tokens whose heads straddle units."""
    g = torch.Generator("cuda").manual_seed(group)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    N = 333
    q, k, v = rnd(1, M, group, d), rnd(1, N, 1, d), rnd(1, N, 1, d)
    idx = (torch.arange(M, device="cuda", dtype=torch.int32)[None] * 30 + 5).contiguous()
    out, lse = Guarded(q.shape, torch.bfloat16), Guarded((1, group, M), torch.float32)
    ws = A.new_workspace(A.OP_WINDOW_ATTN, 1, group, N, M, d)
    kv = A.bhnd_strides(N, 1, d)
    A.astraea_window_attn(q, k, v, A.bhnd_strides(M, group, d), kv, kv, idx, M, out.t, lse.t, 1, group, 1, N, d, 4, 2, 60, 9,
                          flags=A.ATTN_COMPACT_Q | A.ATTN_COMPACT_OUT, workspace=ws)
    A.astraea_poll_error(ws)
    want, want_lse = reference(q, k, v, idx, N, 4, 2, 60, 9, None, 1 / math.sqrt(d))
    check(out.t, lse.t, want, want_lse)
    out.check(); lse.check()


@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("scale", [1e-6, 0.02, 3.0])
def test_compact_rows_without_a_list_and_scales(d, scale):
    """Rows 0 .. M - 1, logits all alike and logits of hundreds."""
    g = torch.Generator("cuda").manual_seed(d)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    B, N, M, H = 2, 500, 270, 2
    q, k, v = rnd(B, M, H, d), rnd(B, N, H, d), rnd(B, N, H, d)
    out, lse = torch.zeros_like(q), torch.zeros(B, H, M, device="cuda")
    ws = A.new_workspace(A.OP_WINDOW_ATTN, B, H, N, M, d)
    kv = A.bhnd_strides(N, H, d)
    A.astraea_window_attn(q, k, v, A.bhnd_strides(M, H, d), kv, kv, None, M, out, lse, B, H, H, N, d, 0, 3, 100, 40, scale=scale,
                          flags=A.ATTN_COMPACT_Q | A.ATTN_COMPACT_OUT, workspace=ws)
    A.astraea_poll_error(ws)
    idx = torch.arange(M, device="cuda", dtype=torch.int32).expand(B, -1)
    want, want_lse = reference(q, k, v, idx, N, 0, 3, 100, 40, None, scale)
    check(out, lse, want, want_lse)


@pytest.mark.parametrize("d", [64, 72, 128])
def test_one_window_call_captured_on_inputs_that_change(d):
    """Lengths, lists and rows are read when the graph runs; two graphs have workspaces of their own and run at the same time."""
    g = torch.Generator("cuda").manual_seed(d)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    B, N, H, H_kv = 3, 3000, 8, 2
    k, v = rnd(B, N, H_kv, d), rnd(B, N, H_kv, d)
    kv, row = A.bhnd_strides(N, H_kv, d), A.bhnd_strides(1, H, d)
    calls = []
    for _ in range(2):
        s = dict(q=rnd(B, 1, H, d), kv_len=torch.full((B,), N, device="cuda", dtype=torch.int32), idx=torch.full((B, 1), N - 1, device="cuda", dtype=torch.int32),
                 out=torch.zeros(B, 1, H, d, device="cuda", dtype=torch.bfloat16), lse=torch.zeros(B, H, 1, device="cuda"),
                 ws=A.new_workspace(A.OP_WINDOW_ATTN, B, H, N, 1, d), graph=torch.cuda.CUDAGraph())
        run = lambda s=s: A.astraea_window_attn(s["q"], k, v, row, kv, kv, s["idx"], 1, s["out"], s["lse"], B, H, H_kv, N, d, 8, 0, 1700, 0, s["kv_len"],
                                                flags=A.ATTN_COMPACT_Q | A.ATTN_COMPACT_OUT, workspace=s["ws"])
        run()
        torch.cuda.synchronize()
        with torch.cuda.graph(s["graph"]):
            for _ in range(3):
                run()
        calls.append(s)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for lengths in ([[1, 2000, 2999], [64, 65, 0]], [[3000, 1701, 1709], [1710, 8, 9]]):
        for s, n in zip(calls, lengths):
            s["kv_len"].copy_(torch.tensor(n, dtype=torch.int32))
            s["idx"].copy_((s["kv_len"] - 1).clamp(min=0)[:, None])
            s["q"].copy_(rnd(B, 1, H, d))
        torch.cuda.synchronize()
        for _ in range(4):
            for s, st in zip(calls, streams):
                with torch.cuda.stream(st):
                    s["graph"].replay()
        torch.cuda.synchronize()
        for s in calls:
            A.astraea_poll_error(s["ws"])
            want, want_lse = reference(s["q"], k, v, s["idx"], N, 8, 0, 1700, 0, s["kv_len"], 1 / math.sqrt(d))
            check(s["out"], s["lse"], want, want_lse)


@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("norm,rotation", [(A.NORM_RMS, A.ROTATE_HALF), (A.NORM_LAYER, A.ROTATE_INTERLEAVED)])
def test_few_heads_of_many_tokens_between_compact_rows_and_caches(d, norm, rotation):
    """Both tensors take the kernel for few heads: listed rows of a head-major cache to compact rows, and compact rows to their places in one."""
    g = torch.Generator("cuda").manual_seed(d)
    B, N, M, H, H_kv, n_rot = 2, 8000, 6000, 3, 1, 7900
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    q, k = 3 * rnd(B, H, N, d), 3 * rnd(B, M, H_kv, d)
    idx = lists(g, B, N, M)
    cos, sin = table(n_rot, d, g)
    w, b = rnd(d), rnd(d) if norm == A.NORM_LAYER else None
    before = rnd(B, N, H_kv, d)
    qo, cache = Guarded((B, M, H, d), torch.bfloat16), Guarded((B, N, H_kv, d), torch.bfloat16, before)
    ws = A.new_workspace(A.OP_QK_NORM_ROTATE, B, H, N, M, d)
    A.astraea_qk_norm_rotate([A.head_rows(q, (H * N * d, N * d, d), qo.t, A.bhnd_strides(M, H, d), H, idx, M, w, b, flags=A.ROWS_COMPACT_OUT),
                              A.head_rows(k, A.bhnd_strides(M, H_kv, d), cache.t, A.bhnd_strides(N, H_kv, d), H_kv, idx, M, None, None, flags=A.ROWS_COMPACT_IN)],
                             cos, sin, n_rot, B, N, d, norm, rotation, 1e-6, ws)
    A.astraea_poll_error(ws)
    rows, at = torch.arange(B, device="cuda")[:, None], torch.cat([torch.arange(30), torch.arange(M - 60, M)]).cuda()
    some = idx[:, at]
    want, z = norm_reference(q.transpose(1, 2)[rows, some.long()], some, n_rot, cos, sin, w, b, norm, rotation)
    norm_close(qo.t[:, at], want, z, norm == A.NORM_LAYER)
    want, z = norm_reference(k[:, at], some, n_rot, cos, sin, None, None, norm, rotation)
    norm_close(cache.t[rows, some.long()], want, z, norm == A.NORM_LAYER)
    rest = torch.ones(B, N, dtype=torch.bool, device="cuda")
    rest[rows, idx.long()] = False
    assert torch.equal(cache.t[rest], before[rest])
    # every other row: the one-launch kernel does the same arithmetic (a tensor of this many tokens in pieces that are too short for the other)
    whole = torch.zeros(B, N, H, d, device="cuda", dtype=torch.bfloat16)
    for n0 in range(0, N, 2000):
        piece = q[:, :, n0:n0 + 2000].transpose(1, 2).contiguous()
        out = torch.zeros_like(piece)
        st = A.bhnd_strides(2000, H, d)
        turned = max(0, min(n_rot - n0, 2000))
        A.astraea_qk_norm_rotate([A.head_rows(piece, st, out, st, H, None, 0, w, b)], cos[n0:n0 + turned].contiguous(), sin[n0:n0 + turned].contiguous(), turned,
                                 B, 2000, d, norm, rotation, 1e-6, ws)
        whole[:, n0:n0 + 2000] = out
    assert torch.equal(qo.t, whole[rows, idx.long()])
    qo.check(); cache.check()


@pytest.mark.parametrize("R,K,N_out", [(33, 33 * 128, 136), (300, 65 * 128, 264), (70, 48 * 128, 520), (8, 65 * 128, 40), (1, 33 * 128, 1000), (257, 36 * 128, 2056)])
@pytest.mark.parametrize("gelu", [False, True])
def test_layers_over_many_blocks_of_channels(R, K, N_out, gelu):
    """More than the 32 blocks whose scales of W a warp holds at a time."""
    g = torch.Generator("cuda").manual_seed(K + R)
    xq, xs, wq, ws = operands(g, R, N_out, K)
    y = Guarded((1, R, N_out), torch.bfloat16)
    work = A.new_workspace(A.OP_GATHERED_LINEAR_FP8, 1, 0, R, R, K)
    A.astraea_gathered_linear_fp8(xq, xs, None, 0, wq, ws, None, None, None, y.t, 1, R, K, N_out, flags=A.LINEAR_GELU if gelu else 0, workspace=work)
    A.astraea_poll_error(work)
    want, mass = product(xq, xs, wq, ws, N_out)
    if gelu:                                                       # slope at most 1.13, Phi within 7.5e-8
        want, mass = want * torch.special.ndtr(want), 1.13 * mass + 2.0 ** 17 * 7.5e-8 * want.abs()
    layer_close(y.t[0], want, mass, K)
    y.check()


@pytest.mark.parametrize("B,N,gate", [(8, 1, True), (1, 8, False), (4, 2, True), (9, 1, True), (3, 3, True)])
def test_a_handful_of_rows_without_a_list(B, N, gate):
    """On both sides of the line between the kernels, a gate for each batch element, in place."""
    g = torch.Generator("cuda").manual_seed(B * 10 + N)
    K, N_out = 640, 1000
    xq, xs, wq, ws = operands(g, B * N, N_out, K)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    bias, ga, before = rnd(N_out), rnd(B, N_out) if gate else None, rnd(B, N, N_out)
    y = Guarded((B, N, N_out), torch.bfloat16, before)
    work = A.new_workspace(A.OP_GATHERED_LINEAR_FP8, B, 0, N, N, K)
    A.astraea_gathered_linear_fp8(xq, xs, None, 0, wq, ws, bias, y.t, ga, y.t, B, N, K, N_out, workspace=work)
    A.astraea_poll_error(work)
    want, mass = product(xq, xs, wq, ws, N_out)
    want, mass = (want + bias.double()).view(B, N, -1), (mass + bias.double().abs()).view(B, N, -1)
    if gate:
        want, mass = want * ga.double()[:, None], mass * ga.double().abs()[:, None] + want.abs() * 2.0 ** -6
    layer_close(y.t, want + before.double(), mass + before.double().abs() * 2.0 ** -6, K)
    y.check()
