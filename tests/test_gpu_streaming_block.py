"""The self-attention group of a block as a stream runs it, in 8 bits: layer norm, quantiser, projections, head norms with rotation and the new
keys' way into the cache, window attention over the cache, output projection with gate and residual.  Every stage is checked against its
formula in 64 bits on what the stage before left; a captured run is replayed on new inputs."""
import math

import pytest
import torch

from helpers import assert_attn_close, bf16_dev_to_f64
from paper_2506_05096_b200 import binding as A

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


class Block:
    def __init__(self, B, N, M, H, H_kv, d, seed):
        g = torch.Generator("cuda").manual_seed(seed)
        self.g, self.B, self.N, self.M, self.H, self.H_kv, self.d, self.D = g, B, N, M, H, H_kv, d, H * d
        rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
        D, kv = self.D, H_kv * d
        self.w = {n: (rnd(o, D) / math.sqrt(D)).bfloat16() for n, o in (("q", D), ("k", kv), ("v", kv), ("o", D))}
        self.bias, self.gate = rnd(D), rnd(B, D)
        self.qw, self.kw = 1 + 0.1 * rnd(d), 1 + 0.1 * rnd(d)
        a = torch.rand(N, d // 2, device="cuda", generator=g, dtype=torch.float64) * 100
        self.cos, self.sin = a.cos().float(), a.sin().float()
        self.k_cache, self.v_cache = rnd(B, N, H_kv, d), rnd(B, N, H_kv, d)
        self.x = rnd(B, N, D)
        self.idx = torch.stack([torch.randperm(N, device="cuda", generator=g)[:M].sort().values for _ in range(B)]).int()
        self.wq, self.ws = {}, {}
        for n, w in self.w.items():
            self.wq[n] = torch.empty(w.shape, device="cuda", dtype=torch.uint8)
            self.ws[n] = torch.empty(-(-w.shape[0] // 128), D // 128, device="cuda")
            A.astraea_quantize_fp8_weight(w, self.wq[n], self.ws[n], w.shape[0], D)
        z = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, device="cuda", dtype=dtype)
        self.h, self.xq, self.xs = z(B, M, D), z(B * M, D, dtype=torch.uint8), z(D // 128, B * M, dtype=torch.float32)
        self.q, self.k_new, self.v_new = z(B, M, D), z(B, M, kv), z(B, M, kv)
        self.qr, self.o, self.lse = z(B, M, D), z(B, M, D), z(B, H, M, dtype=torch.float32)
        self.oq, self.os = z(B * M, D, dtype=torch.uint8), z(D // 128, B * M, dtype=torch.float32)
        self.y = self.x.clone()
        self.work = A.new_workspace(A.OP_WINDOW_ATTN, B, H, N, M, d)

    def run(self):
        B, N, M, H, H_kv, d, D = self.B, self.N, self.M, self.H, self.H_kv, self.d, self.D
        ws, kv = self.work, self.H_kv * self.d
        A.astraea_layernorm_modulate(self.x, self.idx, M, None, None, self.h, B, N, D, flags=A.LN_COMPACT_OUT, workspace=ws)
        A.astraea_quantize_fp8(self.h, self.idx, M, self.xq, self.xs, B, N, D, flags=A.LINEAR_COMPACT_IN, workspace=ws)
        for n, out, o in (("q", self.q, D), ("k", self.k_new, kv), ("v", self.v_new, kv)):
            A.astraea_gathered_linear_fp8(self.xq, self.xs, self.idx, M, self.wq[n], self.ws[n], None, None, None, out, B, N, D, o,
                                          flags=A.LINEAR_COMPACT_OUT, workspace=ws)
        rows_q, rows_k, cache = A.bhnd_strides(M, H, d), A.bhnd_strides(M, H_kv, d), A.bhnd_strides(N, H_kv, d)
        A.astraea_qk_norm_rotate([A.head_rows(self.q, rows_q, self.qr, rows_q, H, self.idx, M, self.qw, flags=A.ROWS_COMPACT_IN | A.ROWS_COMPACT_OUT),
                                  A.head_rows(self.k_new, rows_k, self.k_cache, cache, H_kv, self.idx, M, self.kw, flags=A.ROWS_COMPACT_IN)],
                                 self.cos, self.sin, N, B, N, d, workspace=ws)
        A.astraea_scatter_reuse(self.v_cache, self.v_new, self.idx, B, N, M, kv, workspace=ws)
        A.astraea_window_attn(self.qr, self.k_cache, self.v_cache, rows_q, cache, cache, self.idx, M, self.o, self.lse, B, H, H_kv, N, d,
                              n_first=16, left=300, right=0, flags=A.ATTN_COMPACT_Q | A.ATTN_COMPACT_OUT, workspace=ws)
        A.astraea_quantize_fp8(self.o, self.idx, M, self.oq, self.os, B, N, D, flags=A.LINEAR_COMPACT_IN, workspace=ws)
        A.astraea_gathered_linear_fp8(self.oq, self.os, self.idx, M, self.wq["o"], self.ws["o"], self.bias, self.x, self.gate, self.y, B, N, D, D, workspace=ws)

    def values(self, codes, scale, weight):
        v = codes.view(F8).double()
        if weight:
            return v * scale.double().repeat_interleave(128, 0)[:v.shape[0]].repeat_interleave(128, 1)
        return v * scale.double().t().repeat_interleave(128, 1)

    def check(self, k_before, v_before):
        B, N, M, H, H_kv, d, D = self.B, self.N, self.M, self.H, self.H_kv, self.d, self.D
        rows, idx = torch.arange(B, device="cuda")[:, None], self.idx.long()
        x = self.x[rows, idx].double()
        h = (x - x.mean(-1, keepdim=True)) / (x.var(-1, unbiased=False, keepdim=True) + 1e-6).sqrt()
        assert ((self.h.double() - h).abs() <= 2.0 ** -8 * h.abs() + 1e-5).all()
        xv = self.values(self.xq, self.xs, False)
        # codes are within half a step of their values: 2^-4 of them, and 2^-10 steps of the scale (amax / 448) near zero
        assert ((xv - self.h.double().flatten(0, 1)).abs() <= 2.0 ** -4 * 1.001 * xv.abs() + 2.0 ** -10 * self.xs.double().max() * 1.001).all()
        for n, got in (("q", self.q), ("k", self.k_new), ("v", self.v_new)):
            wv = self.values(self.wq[n], self.ws[n], True)
            want, mass = (xv @ wv.t()).view_as(got), (xv.abs() @ wv.abs().t()).view_as(got)
            assert ((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + (132 + D // 64) * 2.0 ** -24 * mass).all(), n
        for got, new, heads, w in ((self.qr, self.q, H, self.qw), (self.k_cache[rows, idx], self.k_new, H_kv, self.kw)):
            z = new.double().view(B, M, heads, d)
            z = z / ((z * z).mean(-1, keepdim=True) + 1e-6).sqrt() * w.double()
            c, s = self.cos.double()[idx][:, :, None], self.sin.double()[idx][:, :, None]
            want = torch.stack([z[..., 0::2] * c - z[..., 1::2] * s, z[..., 0::2] * s + z[..., 1::2] * c], -1).flatten(-2)
            big = z.abs().amax(-1, keepdim=True)
            assert ((got.double().view_as(want) - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -20 * big).all()
        rest = torch.ones(B, N, dtype=torch.bool, device="cuda")
        rest[rows, idx] = False
        assert torch.equal(self.k_cache[rest], k_before[rest]) and torch.equal(self.v_cache[rest], v_before[rest])
        assert torch.equal(self.v_cache[rows, idx].flatten(2), self.v_new)
        j = torch.arange(N, device="cuda")
        for b in range(B):
            p = idx[b][:, None]
            see = (j < 16) | ((j >= p - 300) & (j <= p))
            for hh in range(H):
                logit = (self.qr[b].view(M, H, d)[:, hh].double() @ self.k_cache[b, :, hh * H_kv // H].double().t() / math.sqrt(d)).masked_fill(~see, -math.inf)
                want = logit.softmax(1) @ self.v_cache[b, :, hh * H_kv // H].double()
                assert (self.lse[b, hh].double() - logit.logsumexp(1)).abs().max() < 1e-3
                assert_attn_close(bf16_dev_to_f64(self.o[b].view(M, H, d)[:, hh]), want.cpu().numpy(), what=(b, hh))
        ov, wv = self.values(self.oq, self.os, False), self.values(self.wq["o"], self.ws["o"], True)
        res, gate = self.x[rows, idx].double(), self.gate.double()[:, None]
        act, mass = (ov @ wv.t()).view(B, M, D) + self.bias.double(), (ov.abs() @ wv.abs().t()).view(B, M, D) + self.bias.double().abs()
        want = res + gate * act
        bound = 2.0 ** -8 * want.abs() + (136 + D // 64) * 2.0 ** -24 * (mass * gate.abs() + res.abs())
        assert ((self.y[rows, idx].double() - want).abs() <= bound).all()
        assert torch.equal(self.y[rest], self.x[rest])


# few rows and many, both kinds of linear layer; grouped heads; every head width (72 x 16 channels are nine blocks of 128)
@pytest.mark.parametrize("B,N,M,H,H_kv,d", [(1, 700, 500, 6, 2, 64), (2, 600, 300, 16, 16, 72), (2, 900, 1, 8, 2, 128), (3, 400, 2, 4, 4, 64), (1, 2000, 777, 4, 1, 128)])
def test_a_stream_step(B, N, M, H, H_kv, d):
    s = Block(B, N, M, H, H_kv, d, 11)
    k, v = s.k_cache.clone(), s.v_cache.clone()
    s.run()
    A.astraea_poll_error(s.work)
    s.check(k, v)


@pytest.mark.parametrize("M", [1, 300])
def test_captured_and_replayed_on_new_inputs(M):
    s = Block(2, 900, M, 8, 2, 128, 12)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.run()                                                     # set-up that happens once per kernel
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for _ in range(2):
        s.x.copy_(torch.randn(s.x.shape, device="cuda", generator=s.g))
        s.y.copy_(s.x)
        s.idx.copy_(torch.stack([torch.randperm(s.N, device="cuda", generator=s.g)[:M].sort().values for _ in range(s.B)]).int())
        k, v = s.k_cache.clone(), s.v_cache.clone()
        graph.replay()
        torch.cuda.synchronize()
        A.astraea_poll_error(s.work)
        s.check(k, v)


def test_two_streams_at_once():
    a, b = Block(1, 1500, 400, 4, 4, 64, 13), Block(1, 1500, 600, 4, 2, 128, 14)
    keep = [(s.k_cache.clone(), s.v_cache.clone()) for s in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, st in zip((a, b), streams):
            with torch.cuda.stream(st):
                s.run()
    torch.cuda.synchronize()
    for s, (k, v) in zip((a, b), keep):
        A.astraea_poll_error(s.work)
        s.check(k, v)
