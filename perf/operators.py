"""The operators of a streaming, quantised transformer block, as cases to be timed: what a block does between its projections
and its attention when its model rotates positions, when the video is too long for attention over all of it, and when its
linear layers run in 8 bits.

A case is a dict of plain values.  `op` says which operator it is:

    rotate      astraea_qk_norm_rotate: every head of the listed query rows and of the key rows is normalised (RMS or layer
                norm over the head's channels, learned weight) and rotated by its token's position
    window      astraea_window_attn: attention of the listed query rows over a window of keys around each, and over a few first
                and last keys that every query sees
    quantize    astraea_quantize_fp8: listed rows to e4m3 with a scale for each row and 128 channels
    linear      astraea_gathered_linear_fp8: a linear layer of such rows with e4m3 weights that have a scale for each block of
                128 x 128, with bias, GELU, gate and residual

Sizes: B batch elements, H query heads and H_kv key heads of d channels, N tokens, M listed ones, K and N_out channels of a
linear layer.  The plain forms work in 32 bits and round once.
"""
import math

import torch

own = False

E4M3_MAX = 448.0
LEAST_AMAX = 2.0 ** -100           # a block of smaller values is scaled as if this were its largest
BLOCK = 128
EPS = 1e-6


# ------------------------------------------------------------------ the cases
def _rotate(name, B, N, M, H, H_kv, d, n_rot, norm, rotation, append=False):
    return _named(name, {"op": "rotate", "B": B, "N": N, "M": M, "H": H, "H_kv": H_kv, "d": d, "n_rot": n_rot, "norm": norm,
                         "rotation": rotation, "append": append})


def _window(name, B, N, M, H, H_kv, d, n_first, n_last, left, right, lengths=False):
    return _named(name, {"op": "window", "B": B, "N": N, "M": M, "H": H, "H_kv": H_kv, "d": d, "n_first": n_first, "n_last": n_last,
                         "left": left, "right": right, "lengths": lengths})


def _quantize(name, B, N, M, K):
    return _named(name, {"op": "quantize", "B": B, "N": N, "M": M, "K": K})


def _linear(name, B, N, M, K, N_out, bias=True, gelu=False, residual=False):
    return _named(name, {"op": "linear", "B": B, "N": N, "M": M, "K": K, "N_out": N_out, "bias": bias, "gelu": gelu, "residual": residual})


def _named(name, c):
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the HunyuanVideo shape at a keep-ratio of 0.6: queries of the selected tokens, keys of all, the largest call
        _rotate("rotate_hunyuan_600", 1, 118800, 71280, 24, 24, 128, 118800, "rms", "interleaved"),
        # the Open-Sora shape with layer norm and the half-split rotation: a batch of two, 72 channels a head
        _rotate("rotate_opensora_400", 2, 16384, 6553, 16, 16, 72, 16384, "layer", "half"),
        # one new token for each of eight streams, its key appended to a cache: the smallest call
        _rotate("rotate_append", 8, 32768, 1, 32, 8, 128, 32768, "rms", "half", append=True),
        # the 65536-token shape on one of four GPUs that share its heads, a fifth of the tokens, a window of one eighth of the video
        _window("window_64k_200", 1, 65536, 13107, 6, 6, 128, 1024, 0, 4096, 4096),
        # the Open-Sora shape: a batch of two, 72 channels a head, the first frame stays visible
        _window("window_opensora_400", 2, 16384, 6553, 16, 16, 72, 1024, 0, 2048, 2048),
        # one token for each of eight streams over long caches filled to different lengths, four query heads a key head
        _window("window_decode_long", 8, 32768, 1, 32, 8, 128, 128, 0, 16383, 0, lengths=True),
        # one token of one stream over a short window: where latency counts
        _window("window_decode_short", 1, 4276, 1, 24, 24, 64, 16, 226, 1023, 0),
        # the MLP's input rows of the Open-Sora shape, and a handful of rows of a small model
        _quantize("quantize_opensora_400", 2, 16384, 6553, 4608),
        _quantize("quantize_small", 1, 4276, 77, 1536),
        # the largest layer, the Open-Sora shape's first MLP layer, the output projection of a handful of rows
        _linear("linear_large", 1, 17776, 16384, 6144, 6144),
        _linear("linear_opensora_mlp", 2, 16384, 6553, 1152, 4608, gelu=True),
        _linear("linear_small", 1, 4276, 77, 1536, 1536, residual=True),
    ]


def draw(rng):
    def size(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return max(lo, min(hi, n | 1 if rng.random() < 0.5 else n))

    op = rng.choice(["rotate", "window", "window", "quantize", "linear"])
    B = rng.choice([1, 1, 2, 3])
    d = rng.choice([64, 72, 128])
    H_kv = rng.choice([1, 2, 3, 4, 8, 16])
    if op == "rotate":
        H = H_kv * rng.choice([1, 1, 1, 2, 4])
        N = size(4, 350_000_000 // (B * (H + H_kv) * d * 2))
        N = min(N, 60000)
        M = size(1, N)
        return _rotate("", B, N, M, H, H_kv, d, rng.choice([N, N, max(1, N - size(1, 300))]), rng.choice(["rms", "rms", "layer"]),
                       rng.choice(["interleaved", "half"]), append=rng.random() < 0.3)
    if op == "window":
        if rng.random() < 0.3:                                    # single tokens and short lists over a cache
            M, N, H = rng.choice([1, 1, 2, 5]), size(1 << 8, 1 << 15), H_kv * rng.choice([1, 2, 4])
            return _window("", B, max(N, 8), M, H, H_kv, d, rng.choice([0, 4, 64, 200]), 0, size(15, N), 0, lengths=rng.random() < 0.7)
        H = H_kv * rng.choice([1, 1, 1, 2])
        N = size(64, 20000)
        M = min(N, size(1, max(2, min(N, 1_500_000_000 // (B * H * N)))))
        return _window("", B, N, M, H, H_kv, d, rng.choice([0, 1, 17, N // 16]), rng.choice([0, 0, 77, 226]) % N, size(1, N),
                       rng.choice([0, size(1, N)]), lengths=rng.random() < 0.2)
    if op == "quantize":
        K = 128 * rng.randint(1, 64)
        N = size(8, 30_000_000 // K)
        return _quantize("", B, N, size(1, N), K)
    K, N_out = 128 * rng.randint(1, 48), 8 * rng.randint(8, 768)
    N = size(16, 16000)
    return _linear("", B, N, size(1, N // B), K, N_out, bias=rng.random() < 0.7, gelu=rng.random() < 0.4, residual=rng.random() < 0.4)


# ------------------------------------------------------------------ inputs
def _indices(g, B, N, M):
    """M of N tokens for each batch element, ascending."""
    if M == N:
        return torch.arange(N, device="cuda", dtype=torch.int32).repeat(B, 1).contiguous()
    r = torch.rand(B, N, device="cuda", generator=g)
    return r.topk(M, dim=1).indices.sort(dim=1).values.to(torch.int32).contiguous()


def _angles(n, d, dtype):
    """Angles of n tokens in a latent of frames of 45 x 80, the channel pairs shared out over time, height and width."""
    pos = torch.arange(n, device="cuda")
    t, y, x = pos // 3600, pos // 80 % 45, pos % 80
    half = d // 2
    n_y = n_x = half * 3 // 8
    parts = []
    for p, m in ((t, half - n_y - n_x), (y, n_y), (x, n_x)):
        parts.append(p.to(dtype)[:, None] * 256.0 ** (-torch.arange(m, device="cuda", dtype=dtype) / m))
    return torch.cat(parts, 1)


def _blocks_amax(x):
    return x.unflatten(-1, (-1, BLOCK)).abs().amax(-1)


def _random_fp8(g, rows, cols, amp):
    """e4m3 values as a quantiser leaves them: normal numbers whose blocks reach the top of the range."""
    return (torch.randn(rows, cols, device="cuda", generator=g) * amp).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, device="cuda", dtype=torch.bfloat16, generator=g)

    B, N, M = c["B"], c["N"], c["M"]
    if c["op"] == "rotate":
        H, H_kv, d = c["H"], c["H_kv"], c["d"]
        a = _angles(c["n_rot"], d, torch.float64)
        s = {"cos": a.cos().float(), "sin": a.sin().float(), "q_weight": 1 + 0.2 * randn(d), "k_weight": 1 + 0.2 * randn(d)}
        if c["norm"] == "layer":
            s["q_bias"], s["k_bias"] = 0.1 * randn(d), 0.1 * randn(d)
        s["idx"] = _indices(g, B, N, M)
        if c["append"]:                          # rows of the listed tokens alone; keys go to their places in a cache
            s["q"], s["k"] = 3 * randn(B, M, H, d), 3 * randn(B, M, H_kv, d)
            s["q_out"], s["k_out"] = torch.zeros_like(s["q"]), randn(B, N, H_kv, d)
        else:                                    # listed rows of a cache of queries, all rows of the keys
            s["q"], s["k"] = 3 * randn(B, N, H, d), 3 * randn(B, N, H_kv, d)
            s["q_out"], s["k_out"] = randn(B, N, H, d), torch.zeros_like(s["k"])
    elif c["op"] == "window":
        H, H_kv, d = c["H"], c["H_kv"], c["d"]
        s = {"k": randn(B, N, H_kv, d), "v": randn(B, N, H_kv, d)}
        s["compact"] = M <= 8                    # single tokens come and go as rows of their own
        s["q"] = randn(B, M if s["compact"] else N, H, d)
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(B, H, s["q"].shape[1], device="cuda")
        s["kv_len"] = None
        if c["lengths"]:
            s["kv_len"] = torch.randint(max(1, N // 2), N + 1, (B,), device="cuda", dtype=torch.int32, generator=g)
        if s["compact"] and M == 1:              # the newest token
            s["idx"] = (s["kv_len"][:, None] - 1).contiguous() if c["lengths"] else torch.full((B, 1), N - 1, device="cuda", dtype=torch.int32)
        else:
            s["idx"] = _indices(g, B, N, M)
    elif c["op"] == "quantize":
        K = c["K"]
        s = {"x": randn(B, N, K) * torch.exp(0.5 * randn(B, N, 1)), "idx": _indices(g, B, N, M)}
        s["xq"] = torch.zeros(B * M, K, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn)
        s["x_scale"] = torch.zeros(K // BLOCK, B * M, device="cuda")
    else:
        K, N_out, R = c["K"], c["N_out"], B * M
        s = {"xq": _random_fp8(g, R, K, 140.0), "wq": _random_fp8(g, N_out, K, 140.0)}
        s["x_scale"] = (3 / E4M3_MAX) * torch.exp(0.5 * torch.randn(K // BLOCK, R, device="cuda", generator=g))
        s["w_scale"] = (3 / E4M3_MAX / math.sqrt(K)) * torch.exp(0.3 * torch.randn(-(-N_out // BLOCK), K // BLOCK, device="cuda", generator=g))
        s["bias"] = 0.1 * randn(N_out) if c["bias"] else None
        s["residual"] = randn(B, N, N_out) if c["residual"] else None
        s["gate"] = randn(B, N_out) if c["residual"] else None
        s["idx"] = _indices(g, B, N, M)
        s["y"] = randn(B, N, N_out)
    s["case"] = c
    return s


# ------------------------------------------------------------------ the plain forms
def _listed_rows(x, idx):
    return x[torch.arange(x.shape[0], device=x.device)[:, None], idx.long()]


def _put_rows(y, idx, rows):
    y[torch.arange(y.shape[0], device=y.device)[:, None], idx.long()] = rows.to(y.dtype)
    return y


def _norm_rotate(c, x, tok, weight, bias, cos, sin):
    """x: rows of heads [B, M, H, d] of the tokens tok [B, M]."""
    x = x.float()
    if c["norm"] == "layer":
        x = x - x.mean(-1, keepdim=True)
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    if bias is not None:
        x = x + bias.float()
    turned = tok < c["n_rot"]
    at = torch.where(turned, tok, 0).long()
    co = torch.where(turned[..., None], cos[at], 1.0)[:, :, None, :]
    si = torch.where(turned[..., None], sin[at], 0.0)[:, :, None, :]
    if c["rotation"] == "half":
        a, b = x.chunk(2, -1)
        return torch.cat([a * co - b * si, b * co + a * si], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * co - b * si, b * co + a * si], -1).flatten(-2)


def _plain_rotate(s):
    c, tok = s["case"], s["idx"]
    everything = torch.arange(c["N"], device="cuda").expand(c["B"], -1)
    q = s["q"] if c["append"] else _listed_rows(s["q"], tok)
    q = _norm_rotate(c, q, tok, s["q_weight"], s.get("q_bias"), s["cos"], s["sin"])
    k = _norm_rotate(c, s["k"], tok if c["append"] else everything, s["k_weight"], s.get("k_bias"), s["cos"], s["sin"])
    if c["append"]:
        return q.to(torch.bfloat16), _put_rows(s["k_out"], tok, k)
    return _put_rows(s["q_out"], tok, q), k.to(torch.bfloat16)


def _plain_window(s):
    c, tok = s["case"], s["idx"]
    B, N, H, H_kv, d = c["B"], c["N"], c["H"], c["H_kv"], c["d"]
    q = s["q"] if s["compact"] else _listed_rows(s["q"], tok)
    q = q.float().mul(1 / math.sqrt(d)).unflatten(2, (H_kv, H // H_kv)).permute(0, 2, 3, 1, 4).flatten(2, 3)      # [B, H_kv, G M, d]
    p = torch.matmul(q, s["k"].float().permute(0, 2, 3, 1))
    p = p.unflatten(2, (H // H_kv, -1))                                               # [B, H_kv, G, M, N]
    j, i = torch.arange(N, device="cuda"), tok.long()[..., None]
    hidden = ~((j < c["n_first"]) | (j >= N - c["n_last"]) | ((j >= i - c["left"]) & (j <= i + c["right"])))
    if s["kv_len"] is not None:
        hidden = hidden | (j >= s["kv_len"][:, None, None])
    p.masked_fill_(hidden[:, None, None], -math.inf)
    top = p.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.flatten(2, 3), s["v"].float().permute(0, 2, 1, 3)).unflatten(2, (H // H_kv, -1))
    out = torch.where(total > 0, out / total, 0.0).permute(0, 3, 1, 2, 4).flatten(2, 3)          # [B, M, H, d]
    lse = (top + total.log())[..., 0].flatten(1, 2)                                   # [B, H, M]
    if s["compact"]:
        return out.to(torch.bfloat16), lse
    b = torch.arange(B, device="cuda")[:, None, None]
    h = torch.arange(H, device="cuda")[None, :, None]
    s["lse"][b, h, tok.long()[:, None, :]] = lse
    return _put_rows(s["out"], tok, out), s["lse"]


def _plain_quantize(s):
    x = _listed_rows(s["x"], s["idx"]).flatten(0, 1).float()
    scale = _blocks_amax(x).clamp(min=LEAST_AMAX) / E4M3_MAX
    xq = (x.unflatten(-1, (-1, BLOCK)) / scale[..., None]).flatten(-2).to(torch.float8_e4m3fn)
    return xq, scale.t().contiguous()


def _plain_linear(s):
    c = s["case"]
    x = s["xq"].float() * s["x_scale"].t().repeat_interleave(BLOCK, 1)
    w = s["wq"].float() * s["w_scale"].repeat_interleave(BLOCK, 0)[:c["N_out"]].repeat_interleave(BLOCK, 1)
    y = torch.matmul(x, w.t())
    if s["bias"] is not None:
        y = y + s["bias"].float()
    if c["gelu"]:
        y = 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    y = y.unflatten(0, (c["B"], -1))
    if s["residual"] is not None:
        y = _listed_rows(s["residual"], s["idx"]).float() + s["gate"].float()[:, None] * y
    return _put_rows(s["y"], s["idx"], y)


# ------------------------------------------------------------------ the framework's calls
def _workspace(s, A, op, *sizes):
    if "workspace" not in s:
        s["workspace"] = A.new_workspace(op, *sizes)
    return s["workspace"]


def _own_rotate(s, A):
    c = s["case"]
    B, N, M, H, H_kv, d = c["B"], c["N"], c["M"], c["H"], c["H_kv"], c["d"]
    ws = _workspace(s, A, A.OP_QK_NORM_ROTATE, B, H, N, M, d)
    all_q, all_k = A.bhnd_strides(N, H, d), A.bhnd_strides(N, H_kv, d)
    if c["append"]:
        row_q, row_k = A.bhnd_strides(M, H, d), A.bhnd_strides(M, H_kv, d)
        rows = [A.head_rows(s["q"], row_q, s["q_out"], row_q, H, s["idx"], M, s["q_weight"], s.get("q_bias"),
                            flags=A.ROWS_COMPACT_IN | A.ROWS_COMPACT_OUT),
                A.head_rows(s["k"], row_k, s["k_out"], all_k, H_kv, s["idx"], M, s["k_weight"], s.get("k_bias"), flags=A.ROWS_COMPACT_IN)]
    else:
        rows = [A.head_rows(s["q"], all_q, s["q_out"], all_q, H, s["idx"], M, s["q_weight"], s.get("q_bias")),
                A.head_rows(s["k"], all_k, s["k_out"], all_k, H_kv, None, N, s["k_weight"], s.get("k_bias"))]
    A.astraea_qk_norm_rotate(rows, s["cos"], s["sin"], c["n_rot"], B, N, d, norm=A.NORM_LAYER if c["norm"] == "layer" else A.NORM_RMS,
                             rotation=A.ROTATE_HALF if c["rotation"] == "half" else A.ROTATE_INTERLEAVED, eps=EPS, workspace=ws)
    return s["q_out"], s["k_out"]


def _own_window(s, A):
    c = s["case"]
    B, N, M, H, H_kv, d = c["B"], c["N"], c["M"], c["H"], c["H_kv"], c["d"]
    ws = _workspace(s, A, A.OP_WINDOW_ATTN, B, H, N, M, d)
    rows = M if s["compact"] else N
    kv = A.bhnd_strides(N, H_kv, d)
    A.astraea_window_attn(s["q"], s["k"], s["v"], A.bhnd_strides(rows, H, d), kv, kv, s["idx"], M, s["out"], s["lse"], B, H, H_kv, N, d,
                          n_first=c["n_first"], n_last=c["n_last"], left=c["left"], right=c["right"], kv_len=s["kv_len"],
                          flags=A.ATTN_COMPACT_Q | A.ATTN_COMPACT_OUT if s["compact"] else 0, workspace=ws)
    return s["out"], s["lse"]


def _own_quantize(s, A):
    c = s["case"]
    ws = _workspace(s, A, A.OP_QUANTIZE_FP8, c["B"], 0, c["N"], c["M"], c["K"])
    A.astraea_quantize_fp8(s["x"], s["idx"], c["M"], s["xq"], s["x_scale"], c["B"], c["N"], c["K"], workspace=ws)
    return s["xq"], s["x_scale"]


def _own_linear(s, A):
    c = s["case"]
    ws = _workspace(s, A, A.OP_GATHERED_LINEAR_FP8, c["B"], 0, c["N"], c["M"], c["K"])
    A.astraea_gathered_linear_fp8(s["xq"], s["x_scale"], s["idx"], c["M"], s["wq"], s["w_scale"], s["bias"], s["residual"], s["gate"], s["y"],
                                  c["B"], c["N"], c["K"], c["N_out"], flags=A.LINEAR_GELU if c["gelu"] else 0, workspace=ws)
    return s["y"]


def run(state):
    op = state["case"]["op"]
    if own:
        from paper_2506_05096_b200 import binding as A
        return {"rotate": _own_rotate, "window": _own_window, "quantize": _own_quantize, "linear": _own_linear}[op](state, A)
    return {"rotate": _plain_rotate, "window": _plain_window, "quantize": _plain_quantize, "linear": _plain_linear}[op](state)


# ------------------------------------------------------------------ what a pass cannot do without
def _visible(c, p):
    """Keys that the queries at positions p see (lengths at their mean), and how many different ones."""
    N, n_first, n_last = c["N"], c["n_first"], c["n_last"]
    length = N * 3 // 4 if c["lengths"] else N
    lo = torch.clamp(p - c["left"], min=min(n_first, N))
    hi = torch.clamp(p + c["right"] + 1, max=min(length, N - n_last))
    fixed = min(n_first, length) + max(0, length - max(N - n_last, n_first))
    return (hi - lo).clamp(min=0) + fixed, min(length, fixed + int(max(0, hi.max() - lo.min())))


def work(case):
    c = case
    B, N, M = c["B"], c["N"], c["M"]
    if c["op"] == "rotate":
        rows = B * (M * c["H"] + (M if c["append"] else N) * c["H_kv"])
        return {"bytes": rows * c["d"] * 4 + min(c["n_rot"], B * M if c["append"] else N) * c["d"] * 4, "flops": rows * c["d"] * 9}
    if c["op"] == "window":
        length = N * 3 // 4 if c["lengths"] else N
        p = torch.full((1,), length - 1) if M == 1 else (torch.arange(M, dtype=torch.float64) * (N / M)).long()
        seen, keys = _visible(c, p)
        pairs = B * c["H"] * float(seen.double().sum())
        return {"bytes": B * (M * c["H"] * (4 * c["d"] + 4) + keys * c["H_kv"] * 4 * c["d"]), "flops": 4 * c["d"] * pairs}
    if c["op"] == "quantize":
        return {"bytes": B * M * (3 * c["K"] + c["K"] // 32), "flops": B * M * c["K"] * 3}
    R, K, N_out = B * M, c["K"], c["N_out"]
    return {"bytes": R * (K + K // 32) + N_out * (K + K // 4096) + R * N_out * (4 if c["residual"] else 2), "flops": 2 * R * K * N_out}


# ------------------------------------------------------------------ the definitions, in 64 bits
def _exact_rotate(c, s):
    B, N, M, d = c["B"], c["N"], c["M"], c["d"]
    half = d // 2
    first, second = (list(range(half)), list(range(half, d))) if c["rotation"] == "half" else (list(range(0, d, 2)), list(range(1, d, 2)))
    outs = []
    for x, y, w, b, listed_rows in ((s["q"], s["q_out"], s["q_weight"], s.get("q_bias"), True), (s["k"], s["k_out"], s["k_weight"], s.get("k_bias"), c["append"])):
        y = y.double()
        for e in range(B):
            tok = s["idx"][e].long() if listed_rows else torch.arange(N, device="cuda")
            z = (x[e] if c["append"] or not listed_rows else x[e, tok]).double()
            if c["norm"] == "layer":
                z = z - z.sum(-1, keepdim=True) / d
            z = z / ((z ** 2).sum(-1, keepdim=True) / d + EPS).sqrt() * w.double()
            if b is not None:
                z = z + b.double()
            r = torch.empty_like(z)
            n = torch.clamp(tok, max=c["n_rot"] - 1)
            still = (tok >= c["n_rot"])[:, None]
            co = s["cos"].double()[n].masked_fill(still, 1.0)[:, None]
            si = s["sin"].double()[n].masked_fill(still, 0.0)[:, None]
            r[..., first] = z[..., first] * co - z[..., second] * si
            r[..., second] = z[..., first] * si + z[..., second] * co
            if c["append"] and y.shape[1] == M and x is s["q"]:
                y[e] = r
            else:
                y[e, tok] = r
        outs.append(y)
    return tuple(outs)


def _exact_window(c, s):
    B, N, M, H, H_kv, d = c["B"], c["N"], c["M"], c["H"], c["H_kv"], c["d"]
    out, lse = s["out"].double(), s["lse"].double()
    for e in range(B):
        length = N if s["kv_len"] is None else int(s["kv_len"][e])
        always = torch.cat([torch.arange(0, min(c["n_first"], N)), torch.arange(max(N - c["n_last"], min(c["n_first"], N)), N)])
        for m0 in range(0, M, 1024):
            tok = s["idx"][e, m0:m0 + 1024].long()
            lo, hi = max(0, int(tok[0]) - c["left"]), min(N, int(tok[-1]) + c["right"] + 1)
            keys = torch.cat([always, torch.arange(lo, hi)]).unique()
            keys = keys[keys < length].cuda()
            near = (keys[None] >= tok[:, None] - c["left"]) & (keys[None] <= tok[:, None] + c["right"])
            seen = near | (keys < c["n_first"])[None] | (keys >= N - c["n_last"])[None]
            rows = slice(m0, m0 + tok.numel()) if s["compact"] else tok
            for h in range(H):
                kv = h // (H // H_kv)
                logit = s["q"][e, rows, h].double() @ s["k"][e, keys, kv].double().t() / math.sqrt(d)
                logit = torch.where(seen, logit, -math.inf)
                z = torch.logsumexp(logit, 1) if keys.numel() else torch.full((tok.numel(),), -math.inf, device="cuda", dtype=torch.float64)
                weight = torch.where(seen, torch.exp(logit - torch.where(z == -math.inf, 0.0, z)[:, None]), 0.0)
                out[e, rows, h] = weight @ s["v"][e, keys, kv].double()
                lse[e, h, rows] = z
    return out, lse


def _to_e4m3(v):
    """The nearest e4m3 value, ties to the even one: three bits behind the leading one, down to steps of 2^-9."""
    exponent = torch.frexp(v).exponent - 1
    step = torch.ldexp(torch.ones_like(v), exponent.clamp(min=-6) - 3)
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def _exact_quantize(c, s):
    x = torch.cat([s["x"][e][s["idx"][e].long()] for e in range(c["B"])]).double().reshape(-1, c["K"] // BLOCK, BLOCK)
    scale = torch.maximum(x.abs().max(2).values, torch.tensor(LEAST_AMAX, device="cuda", dtype=torch.float64)) / E4M3_MAX
    return _to_e4m3(x / scale[:, :, None]).reshape(-1, c["K"]), scale.t()


def _exact_linear(c, s):
    B, N, M, K, N_out = c["B"], c["N"], c["M"], c["K"], c["N_out"]
    acc = torch.zeros(B * M, N_out, device="cuda", dtype=torch.float64)
    col = torch.arange(N_out, device="cuda") // BLOCK
    for kb in range(K // BLOCK):
        ks = slice(kb * BLOCK, (kb + 1) * BLOCK)
        acc += (s["xq"][:, ks].double() @ s["wq"][:, ks].double().t()) * s["x_scale"][kb].double()[:, None] * s["w_scale"][:, kb].double()[col]
    if s["bias"] is not None:
        acc += s["bias"].double()
    if c["gelu"]:
        acc *= torch.special.ndtr(acc)
    y = s["y"].double()
    for e in range(B):
        tok, rows = s["idx"][e].long(), acc[e * M:(e + 1) * M]
        y[e, tok] = rows if s["residual"] is None else s["residual"][e, tok].double() + rows * s["gate"][e].double()
    return y


def exact(case, seed):
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "window": _exact_window, "quantize": _exact_quantize, "linear": _exact_linear}[case["op"]](s["case"], s)
