// astraea_qk_norm_rotate: every head of the listed rows of a tensor of heads (queries, keys) is normalised over its d channels and
// rotated by the position of its token,
//     z = norm(x[b, i, h, :]) * weight + bias,   y[b, i, h, (p, p')] = (z_p cos_i,p - z_p' sin_i,p,  z_p sin_i,p + z_p' cos_i,p),
// what a block that normalises its queries and keys and encodes positions by rotation does between its projections and its attention
// (Section 3.2: such layers act on every token by itself, so queries are needed for the selected tokens only; keys for all).
//
// HBM-bound: every value is read once and written once, in one launch for queries and keys.  A warp takes one token's heads (a share of
// them in short launches); what weights, cosines and sines make of a channel pair is two products and a sum, whose factors are computed
// once per token and used for all of its heads.  A lane owns the same channels of the first and of the second half of a head (16 bytes
// each; three times 8 bytes at head_dim 72, whose halves are 72 bytes), so that both ways of pairing channels, (2p, 2p + 1) and
// (p, p + d/2), stay inside a lane and only the sums of the norm go round: over 4, 3 or 8 lanes.
// fp32 arithmetic, one rounding to bf16 at the end.
#include "common.cuh"

namespace astraea {
namespace {

constexpr int kWarps = 4;                                          // per block

struct HeadTensor {
    const __nv_bfloat16 *x;
    __nv_bfloat16 *y;
    int64_t x_sb, x_sh, x_sn, y_sb, y_sh, y_sn;
    const int32_t *idx;
    const __nv_bfloat16 *weight, *bias;
    int M, H, compact_in, compact_out;
    int parts, part_heads;                                         // a token's heads are shared out over `parts` warps
};
struct HeadNormParams {
    HeadTensor t[2];
    int units0, units;                                             // of t[0], of both: B * M * parts each
    const float *cos, *sin;
    int n_rot, N;
    float eps;
    int *err_word;
};

template <int DH, bool LAYER = false> struct Lanes {
    static constexpr int kUnit = DH == 72 ? 4 : 8;                 // channels of one access
    static constexpr int kUnits = DH == 72 ? 3 : 1;                // accesses of a lane to each half of a head
    static constexpr int kGroup = DH / 2 / (kUnit * kUnits);       // lanes of a head: 4, 3, 8
    static constexpr int kHeads = 32 / kGroup;                     // heads that a warp takes at once: 8, 10, 4
    static constexpr int kUnroll = DH == 72 ? 2 : LAYER ? 3 : 6;              // and how often before it waits (24 x 128, 16 x 72, 48 x 64 are one round)
};

// one access to a head: 16 or 8 bytes
template <int U> __device__ __forceinline__ void load_unit(const __nv_bfloat16 *p, uint32_t *r) {
    if constexpr (U == 8) {
        const uint4 v = ld_stream(reinterpret_cast<const uint4 *>(p));
        r[0] = v.x; r[1] = v.y; r[2] = v.z; r[3] = v.w;
    } else asm volatile("ld.global.v2.u32 {%0,%1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "l"(p));
}
template <int U> __device__ __forceinline__ void store_unit(__nv_bfloat16 *p, const f32x2 *f) {
    uint32_t w[U / 2];
#pragma unroll
    for (int i = 0; i < U / 2; ++i) {
        float lo, hi;
        unpack2(f[i], lo, hi);
        __nv_bfloat162 v2 = __floats2bfloat162_rn(lo, hi);
        w[i] = *reinterpret_cast<uint32_t *>(&v2);
    }
    if constexpr (U == 8) *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
}
// N consecutive values of a table
template <int N> __device__ __forceinline__ void load_table(const float *p, float *f) {
    if constexpr (N == 2) asm volatile("ld.global.v2.f32 {%0,%1}, [%2];" : "=f"(f[0]), "=f"(f[1]) : "l"(p));
    else {
#pragma unroll
        for (int i = 0; i < N; i += 4)
            asm volatile("ld.global.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(f[i]), "=f"(f[i + 1]), "=f"(f[i + 2]), "=f"(f[i + 3]) : "l"(p + i));
    }
}
__device__ __forceinline__ f32x2 widen(uint32_t w) { return pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ f32x2 swapped(uint32_t w) { return pack2(__uint_as_float(w & 0xffff0000u), __uint_as_float(w << 16)); }
__device__ __forceinline__ f32x2 swapped(f32x2 v) { float lo, hi; unpack2(v, lo, hi); return pack2(hi, lo); }
__device__ __forceinline__ f32x2 twice(float v) { return pack2(v, v); }

// the sum over the lanes of a head
template <int G> __device__ __forceinline__ float group_sum(float s, int lane) {
    if constexpr (G == 3) {
        const int l = lane % 3, base = lane - l;                   // lanes 30 and 31 hold no head: their sums are not used
        return s + __shfl_sync(0xffffffffu, s, base + (l + 1) % 3) + __shfl_sync(0xffffffffu, s, base + (l + 2) % 3);
    } else {
#pragma unroll
        for (int o = G / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        return s;
    }
}

// LAYER: layer norm with a bias (RMS norm without one otherwise); HALF: channels are paired (p, p + DH/2) and not (2p, 2p + 1)
template <int DH, bool LAYER, bool HALF>
__global__ void __launch_bounds__(kWarps * 32, LAYER && DH == 72 ? 3 : 4) head_norm_kernel(const __grid_constant__ HeadNormParams p)
{
    using L = Lanes<DH, LAYER>;
    constexpr int U = L::kUnit, G = L::kGroup, kPairs = L::kUnits * U / 2;      // (f32x2 pairs of a half)
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int sub = lane / G, l = lane - sub * G;                  // head of the warp's kHeads, lane of the head
    const bool on = sub < L::kHeads;
    grid_launch_dependents();
    grid_dependency_wait();
    struct Unit { int which, row, part, b, r, tok, before; };
    auto unit_at = [&](int u) {
        Unit n = {};
        if (u >= p.units) return n;
        n.which = u >= p.units0 ? 1 : 0;
        const HeadTensor &t = p.t[n.which];
        const int v = n.which ? u - p.units0 : u;
        n.row = t.parts == 1 ? v : v / t.parts; n.part = v - n.row * t.parts;
        n.b = n.row / t.M; n.r = n.row - n.b * t.M;
        n.tok = t.idx ? __ldcg(t.idx + n.row) : n.r;
        n.before = (t.idx && n.r > 0) ? __ldcg(t.idx + n.row - 1) : -1;
        return n;
    };
    int u = blockIdx.x * kWarps + warp;
    Unit next = unit_at(u);                                        // list entries are fetched a token ahead
    for (; u < p.units; u += gridDim.x * kWarps) {
        const int which = next.which, part = next.part, b = next.b, r = next.r, tok = next.tok, before = next.before;
        const HeadTensor &t = p.t[which];
        next = unit_at(u + gridDim.x * kWarps);
        if ((unsigned)tok >= (unsigned)p.N || before >= tok) {     // see astraea_scatter_reuse
            if (lane == 0 && part == 0 && p.err_word) atomicExch(p.err_word, kErrBadIndex);
            continue;
        }
        const __nv_bfloat16 *src = t.x + b * t.x_sb + (int64_t)(t.compact_in ? r : tok) * t.x_sn + l * U;
        __nv_bfloat16 *dst = t.y + b * t.y_sb + (int64_t)(t.compact_out ? r : tok) * t.y_sn + l * U;
        const int h0 = part * t.part_heads, h1 = min(t.H, h0 + t.part_heads);
        // the first round of heads is sent for before the tables are
        uint32_t raw[L::kUnroll][2][kPairs];
        auto fetch = [&](int hb) {
#pragma unroll
            for (int k = 0; k < L::kUnroll; ++k) {
                const int h = hb + k * L::kHeads;
                if (on && h < h1) {
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int j = 0; j < L::kUnits; ++j) load_unit<U>(src + h * t.x_sh + s * (DH / 2) + G * j * U, &raw[k][s][j * (U / 2)]);
                } else {
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) raw[k][0][i] = raw[k][1][i] = 0u;
                }
            }
        };
        fetch(h0 + sub);
        // y = r (x by + x' cross) + plus for channel pairs x and their partners x': by = weight cos, cross = -+ partner's weight sin
        f32x2 by[2][kPairs], cross[2][kPairs], plus[2][LAYER ? kPairs : 1];
        {
            const bool turned = on && tok < p.n_rot;
            const float *pc = p.cos + (size_t)(turned ? tok : 0) * (DH / 2), *ps = p.sin + (size_t)(turned ? tok : 0) * (DH / 2);
#pragma unroll
            for (int j = 0; j < L::kUnits; ++j) {
                const int c0 = (l + G * j) * U;                    // first channel of the access, in its half
                uint32_t ww[2][U / 2], wb[2][U / 2];
#pragma unroll
                for (int s = 0; s < 2; ++s) {
#pragma unroll
                    for (int i = 0; i < U / 2; ++i) { ww[s][i] = 0x3F803F80u; wb[s][i] = 0u; }
                    if (on && t.weight) load_unit<U>(t.weight + s * (DH / 2) + c0, ww[s]);
                    if (LAYER && on && t.bias) load_unit<U>(t.bias + s * (DH / 2) + c0, wb[s]);
                }
                float co[U], si[U];                                // HALF: of the channels; else of the pairs of both halves
#pragma unroll
                for (int i = 0; i < U; ++i) { co[i] = 1.f; si[i] = 0.f; }
                if (turned) {
                    if (HALF) { load_table<U>(pc + c0, co); load_table<U>(ps + c0, si); }
                    else {
#pragma unroll
                        for (int s = 0; s < 2; ++s) {
                            load_table<U / 2>(pc + s * (DH / 4) + c0 / 2, co + s * (U / 2));
                            load_table<U / 2>(ps + s * (DH / 4) + c0 / 2, si + s * (U / 2));
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < U / 2; ++i) {
                    const int k = j * (U / 2) + i;
                    if (HALF) {
                        const f32x2 c = pack2(co[2 * i], co[2 * i + 1]), n = pack2(si[2 * i], si[2 * i + 1]), m = pack2(-si[2 * i], -si[2 * i + 1]);
                        by[0][k] = mul2(widen(ww[0][i]), c); cross[0][k] = mul2(widen(ww[1][i]), m);
                        by[1][k] = mul2(widen(ww[1][i]), c); cross[1][k] = mul2(widen(ww[0][i]), n);
                        if (LAYER) {
                            plus[0][LAYER ? k : 0] = fma2(widen(wb[0][i]), c, mul2(widen(wb[1][i]), m));
                            plus[1][LAYER ? k : 0] = fma2(widen(wb[1][i]), c, mul2(widen(wb[0][i]), n));
                        }
                    } else {
#pragma unroll
                        for (int s = 0; s < 2; ++s) {
                            const f32x2 c = twice(co[s * (U / 2) + i]), n = pack2(-si[s * (U / 2) + i], si[s * (U / 2) + i]);
                            by[s][k] = mul2(widen(ww[s][i]), c); cross[s][k] = mul2(swapped(ww[s][i]), n);
                            if (LAYER) plus[s][LAYER ? k : 0] = fma2(widen(wb[s][i]), c, mul2(swapped(wb[s][i]), n));
                        }
                    }
                }
            }
        }
        for (int hb = h0 + sub; hb - sub < h1; hb += L::kUnroll * L::kHeads) {
            if (hb != h0 + sub) fetch(hb);
#pragma unroll
            for (int k = 0; k < L::kUnroll; ++k) {
                const int h = hb + k * L::kHeads;
                if (h - sub >= h1) break;                          // the whole warp: no head of this step is left
                f32x2 z[2][kPairs];
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) z[s][i] = widen(raw[k][s][i]);
                float lo, hi;
                if (LAYER) {
                    f32x2 a = 0ull;
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) a = add2(a, add2(z[0][i], z[1][i]));
                    unpack2(a, lo, hi);
                    const f32x2 minus_mean = twice(group_sum<G>(lo + hi, lane) * (-1.0f / DH));
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int i = 0; i < kPairs; ++i) z[s][i] = add2(z[s][i], minus_mean);
                }
                f32x2 a = 0ull;
#pragma unroll
                for (int i = 0; i < kPairs; ++i) a = fma2(z[1][i], z[1][i], fma2(z[0][i], z[0][i], a));
                unpack2(a, lo, hi);
                const f32x2 rstd = twice(rsqrtf(group_sum<G>(lo + hi, lane) * (1.0f / DH) + p.eps));
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    const f32x2 x0 = z[0][i], x1 = z[1][i];
                    z[0][i] = fma2(x0, by[0][i], mul2(HALF ? x1 : swapped(x0), cross[0][i]));
                    z[1][i] = fma2(x1, by[1][i], mul2(HALF ? x0 : swapped(x1), cross[1][i]));
#pragma unroll
                    for (int s = 0; s < 2; ++s) z[s][i] = LAYER ? fma2(z[s][i], rstd, plus[s][LAYER ? i : 0]) : mul2(z[s][i], rstd);
                }
                if (on && h < h1) {
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int j = 0; j < L::kUnits; ++j) store_unit<U>(dst + h * t.y_sh + s * (DH / 2) + G * j * U, &z[s][j * (U / 2)]);
                }
            }
        }
    }
}

template <int DH>
int32_t launch_dim(HeadNormParams &p, const astraea_head_rows *rows, int n, int B, bool layer, bool half, cudaStream_t stream)
{
    // A token's heads go to one warp where that gives every SM its 32 warps, and are shared out in steps of a warp's heads where it does
    // not: one token of 32 + 8 heads is then 10 warps and not 2.
    long long all_rows = 0;
    for (int i = 0; i < n; ++i) all_rows += (long long)B * p.t[i].M;
    const long long slots = (long long)sm_count() * 32;
    long long units[2] = {0, 0};
    for (int i = 0; i < n; ++i) {
        HeadTensor &t = p.t[i];
        const int steps = (t.H + Lanes<DH>::kHeads - 1) / Lanes<DH>::kHeads;
        long long want = all_rows > 0 ? slots / all_rows : 1;
        want = want < 1 ? 1 : want > steps ? steps : want;
        const int part_steps = (int)((steps + want - 1) / want);
        t.part_heads = part_steps * Lanes<DH>::kHeads;
        t.parts = (steps + part_steps - 1) / part_steps;
        units[i] = (long long)B * t.M * t.parts;
    }
    if (units[0] + units[1] > 0x3fffffffll) return fail(ASTRAEA_ERR_INVALID_ARG, "astraea_qk_norm_rotate: too many rows");
    p.units0 = (int)units[0];
    p.units = (int)(units[0] + units[1]);
    if (p.units == 0) return ASTRAEA_OK;
    const long long want = (p.units + kWarps - 1) / kWarps, cap = (long long)sm_count() * 16;
    const int grid = (int)(want < cap ? want : cap);
    auto kernel = layer ? (half ? head_norm_kernel<DH, true, true> : head_norm_kernel<DH, true, false>)
                        : (half ? head_norm_kernel<DH, false, true> : head_norm_kernel<DH, false, false>);
    launch_overlapped(kernel, grid, kWarps * 32, 0, stream, p);
    return check_launch("astraea_qk_norm_rotate");
}

}  // namespace

int32_t launch_qk_norm_rotate(const astraea_head_rows *rows, int n, const float *cos, const float *sin, int n_rot, int B, int N, int d,
                              bool layer, bool half, float eps, int *err_word, cudaStream_t stream)
{
    HeadNormParams p = {};
    for (int i = 0; i < n; ++i) {
        HeadTensor &t = p.t[i];
        const astraea_head_rows &a = rows[i];
        t.x = reinterpret_cast<const __nv_bfloat16 *>(a.x);
        t.y = reinterpret_cast<__nv_bfloat16 *>(a.y);
        t.x_sb = a.x_sb; t.x_sh = a.x_sh; t.x_sn = a.x_sn;
        t.y_sb = a.y_sb; t.y_sh = a.y_sh; t.y_sn = a.y_sn;
        t.idx = a.idx; t.M = a.idx ? a.M : N; t.H = a.H;
        t.weight = reinterpret_cast<const __nv_bfloat16 *>(a.weight);
        t.bias = reinterpret_cast<const __nv_bfloat16 *>(a.bias);
        t.compact_in = (a.flags & ASTRAEA_ROWS_COMPACT_IN) ? 1 : 0;
        t.compact_out = (a.flags & ASTRAEA_ROWS_COMPACT_OUT) ? 1 : 0;
    }
    p.cos = cos; p.sin = sin; p.n_rot = n_rot; p.N = N; p.eps = eps; p.err_word = err_word;
    switch (d) {
    case 64: return launch_dim<64>(p, rows, n, B, layer, half, stream);
    case 72: return launch_dim<72>(p, rows, n, B, layer, half, stream);
    default: return launch_dim<128>(p, rows, n, B, layer, half, stream);
    }
}

}  // namespace astraea
