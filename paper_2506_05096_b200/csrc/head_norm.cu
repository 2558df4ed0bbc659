// astraea_qk_norm_rotate: every head of the listed rows of a tensor of heads (queries, keys) is normalised over its d channels and
// rotated by the position of its token,
//     z = norm(x[b, i, h, :]) * weight + bias,   y[b, i, h, (p, p')] = (z_p cos_i,p - z_p' sin_i,p,  z_p sin_i,p + z_p' cos_i,p),
// what a block that normalises its queries and keys and encodes positions by rotation does between its projections and its attention
// (Section 3.2: such layers act on every token by itself, so queries are needed for the selected tokens only; keys for all).
//
// HBM-bound: every value is read once and written once, in one launch for queries and keys.  A warp takes one token's heads (a share of
// them in short launches), whose cosines and sines it reads once.  A lane owns the same channels of the first and of the second half of a
// head (16 bytes each; three times 8 bytes at head_dim 72, whose halves are 72 bytes), so that both ways of pairing channels, (2p, 2p + 1)
// and (p, p + d/2), stay inside a lane and only the sums of the norm go round: over 4, 3 or 8 lanes.  The rows come through shared memory by
// cp.async, a round of heads ahead, so that the loads of the next token run under the arithmetic of this one and cost no registers
// (with loads into registers 71280 query and 118800 key rows of 24 x 128 took 412 us, now 383 = 6.3 TB/s).  Weights, biases and angles are
// read from shared memory where they are used: at head_dim 72 they were 72 of 154 registers, and there is latency to hide (us with them in
// registers / now: 13106 query and 32768 key rows of 16 x 72, layer norm 70 / 60, RMS norm 67 / 50; 80000 rows of 8 x 128 75 / 72; five blocks a SM,
// with spills, 78, 58 and 75; with four, the layer norm at head_dim 72 still spills 76 bytes a thread, the others nothing).
// fp32 arithmetic, one rounding to bf16 at the end.
#include <initializer_list>

#include "common.cuh"

namespace astraea {
namespace {

constexpr int kWarps = 4;                                          // per block
constexpr int kBlocksSM = 4;                                       // blocks of head_norm_kernel on an SM: 128 registers a thread, 54 KB at head_dim 128

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

template <int DH> struct Lanes {
    static constexpr int kUnit = DH == 72 ? 4 : 8;                 // channels of one access
    static constexpr int kUnits = DH == 72 ? 3 : 1;                // accesses of a lane to each half of a head
    static constexpr int kGroup = DH / 2 / (kUnit * kUnits);       // lanes of a head: 4, 3, 8
    static constexpr int kHeads = 32 / kGroup;                     // heads that a warp takes at once: 8, 10, 4
    static constexpr int kUnroll = DH == 72 ? 2 : 6;              // and how often before it waits (24 x 128, 16 x 72, 48 x 64 are one round)
};

// What a warp keeps of a round in shared memory: kUnroll * kHeads heads as they lie in memory, and the cosines and sines of their token.
// Two of them: the next round is on its way while one is worked on.
template <int DH> struct Round {
    using L = Lanes<DH>;
    static constexpr int kHeadVecs = DH / 8, kHeads = L::kUnroll * L::kHeads, kVecs = kHeads * kHeadVecs;      // 16-byte pieces
    static constexpr int kTableVecs = DH / 8;                      // of the cosines; as many of the sines
    static constexpr int kBytes = (kVecs + 2 * kTableVecs) * 16;
};
__device__ __forceinline__ void copy_async(uint32_t dst, const void *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// one access to a head: 16 or 8 bytes
template <int U> __device__ __forceinline__ void load_shared(const void *p, uint32_t *r) {
    if constexpr (U == 8) { const uint4 v = *reinterpret_cast<const uint4 *>(p); r[0] = v.x; r[1] = v.y; r[2] = v.z; r[3] = v.w; }
    else { const uint2 v = *reinterpret_cast<const uint2 *>(p); r[0] = v.x; r[1] = v.y; }
}
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
    else asm volatile("ld.global.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(f[0]), "=f"(f[1]), "=f"(f[2]), "=f"(f[3]) : "l"(p));
}
__device__ __forceinline__ f32x2 widen(uint32_t w) { return pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
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

// The weights and biases of a lane's channels.
template <int DH, bool LAYER, int PAIRS, int BIAS>
__device__ __forceinline__ void load_weights(const HeadTensor &t, int l, bool on, uint32_t (&w)[2][PAIRS], uint32_t (&bi)[2][BIAS])
{
    using L = Lanes<DH>;
    constexpr int U = L::kUnit, G = L::kGroup;
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int j = 0; j < L::kUnits; ++j) {
                            uint32_t ww[U / 2], wb[U / 2];
#pragma unroll
                            for (int i = 0; i < U / 2; ++i) { ww[i] = 0x3F803F80u; wb[i] = 0u; }       // ones, zeros
                            const int c = s * (DH / 2) + (l + G * j) * U;
                            if (on && t.weight) load_unit<U>(t.weight + c, ww);
                            if (LAYER && on && t.bias) load_unit<U>(t.bias + c, wb);
#pragma unroll
                            for (int i = 0; i < U / 2; ++i) {
                                w[s][j * (U / 2) + i] = ww[i];
                                if (LAYER) bi[s][LAYER ? j * (U / 2) + i : 0] = wb[i];
                            }
                        }
}
// A head: z is a lane's channels of its first and second half; co and si the cosines and sines of its channels (HALF) or of its pairs.
template <int DH, bool LAYER, bool HALF, int PAIRS, int BIAS>
__device__ __forceinline__ void norm_rotate(f32x2 (&z)[2][PAIRS], const uint32_t (&w)[2][PAIRS], const uint32_t (&bi)[2][BIAS], const float (&co)[2 * PAIRS],
                                            const float (&si)[2 * PAIRS], float eps, int lane)
{
    constexpr int G = Lanes<DH>::kGroup, kPairs = PAIRS;
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
                    const f32x2 rstd = twice(rsqrtf(group_sum<G>(lo + hi, lane) * (1.0f / DH) + eps));
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int i = 0; i < kPairs; ++i) {
                            z[s][i] = mul2(z[s][i], rstd);
                            z[s][i] = LAYER ? fma2(z[s][i], widen(w[s][i]), widen(bi[s][LAYER ? i : 0])) : mul2(z[s][i], widen(w[s][i]));
                        }
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) {
                        const f32x2 x0 = z[0][i], x1 = z[1][i];
                        if (HALF) {
                            const f32x2 c = pack2(co[2 * i], co[2 * i + 1]);
                            z[0][i] = fma2(x0, c, mul2(x1, pack2(-si[2 * i], -si[2 * i + 1])));
                            z[1][i] = fma2(x1, c, mul2(x0, pack2(si[2 * i], si[2 * i + 1])));
                        } else {
                            z[0][i] = fma2(x0, twice(co[i]), mul2(swapped(x0), pack2(-si[i], si[i])));
                            z[1][i] = fma2(x1, twice(co[kPairs + i]), mul2(swapped(x1), pack2(-si[kPairs + i], si[kPairs + i])));
                        }
                    }
}

// LAYER: layer norm with a bias (RMS norm without one otherwise); HALF: channels are paired (p, p + DH/2) and not (2p, 2p + 1)
template <int DH, bool LAYER, bool HALF>
__global__ void __launch_bounds__(kWarps * 32, kBlocksSM) head_norm_kernel(const __grid_constant__ HeadNormParams p)
{
    using L = Lanes<DH>;
    constexpr int U = L::kUnit, G = L::kGroup, kPairs = L::kUnits * U / 2;      // (f32x2 pairs of a half)
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int sub = lane / G, l = lane - sub * G;                  // head of the warp's kHeads, lane of the head
    const bool on = sub < L::kHeads;
    grid_launch_dependents();
    grid_dependency_wait();
    // weights and biases, ones and zeros where there are none
    __shared__ __align__(16) uint16_t weights[2][2 * DH];
    for (int i = threadIdx.x; i < 4 * DH; i += kWarps * 32) {
        const HeadTensor &t = p.t[i / (2 * DH)];
        const int c = i % (2 * DH);
        const __nv_bfloat16 *src = c < DH ? t.weight : t.bias;
        weights[i / (2 * DH)][c] = src ? __ldcg(reinterpret_cast<const uint16_t *>(src) + c % DH) : c < DH ? 0x3F80 : 0;
    }
    __syncthreads();
    // A unit is one token's heads of one tensor, or a share of them; it is gone through in rounds.  The list's entries are fetched a unit ahead
    // of the copies.
    struct Unit { int which, part, b, r, tok, before, h0, h1; };   // heads h0 .. h1 - 1; none behind the last unit
    auto unit_at = [&](int u) {
        Unit n = {};
        if (u >= p.units) return n;
        n.which = u >= p.units0 ? 1 : 0;
        const HeadTensor &t = p.t[n.which];
        const int v = n.which ? u - p.units0 : u;
        const int row = t.parts == 1 ? v : v / t.parts;
        n.part = v - row * t.parts;
        n.b = row / t.M; n.r = row - n.b * t.M;
        n.tok = t.idx ? __ldcg(t.idx + row) : n.r;
        n.before = (t.idx && n.r > 0) ? __ldcg(t.idx + row - 1) : -1;
        n.h0 = n.part * t.part_heads; n.h1 = min(t.H, n.h0 + t.part_heads);
        return n;
    };
    auto bad = [&](const Unit &n) { return (unsigned)n.tok >= (unsigned)p.N || n.before >= n.tok; };      // see astraea_scatter_reuse
    using R = Round<DH>;
    extern __shared__ __align__(16) uint8_t smem[];
    const uint8_t *rounds = smem + warp * (2 * R::kBytes);
    const uint32_t s_rounds = static_cast<uint32_t>(__cvta_generic_to_shared(rounds));
    auto send = [&](const Unit &n, int h0, int slot) {
        if (h0 < n.h1 && !bad(n)) {
            const HeadTensor &t = p.t[n.which];
            const __nv_bfloat16 *src = t.x + n.b * t.x_sb + (int64_t)(t.compact_in ? n.r : n.tok) * t.x_sn + h0 * t.x_sh;
            const uint32_t to = s_rounds + slot * R::kBytes;
            const int left = n.h1 - h0;
#pragma unroll
            for (int i = 0; i < (R::kVecs + 31) / 32; ++i) {
                const int c = lane + 32 * i, head = c / R::kHeadVecs;
                if (c < R::kVecs && head < left) copy_async(to + c * 16, src + head * t.x_sh + (c - head * R::kHeadVecs) * 8);
            }
            if (n.tok < p.n_rot && lane < 2 * R::kTableVecs) {
                const float *table = lane < R::kTableVecs ? p.cos : p.sin;
                copy_async(to + (R::kVecs + lane) * 16, table + (size_t)n.tok * (DH / 2) + (lane % R::kTableVecs) * 4);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    const int stride = gridDim.x * kWarps;
    int u = blockIdx.x * kWarps + warp, slot = 0;
    Unit now = unit_at(u), ahead = unit_at(u + stride);
    int hr = now.h0;                                               // first head of the round
    send(now, hr, 0);
    while (u < p.units) {
        Unit next = now;
        int next_hr = hr + R::kHeads, next_u = u;
        if (next_hr >= now.h1 || bad(now)) {
            next_u = u + stride;
            next = ahead; next_hr = next.h0;
            ahead = unit_at(next_u + stride);
        }
        __syncwarp();                                              // the other slot has been read by all lanes
        send(next, next_hr, slot ^ 1);
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        __syncwarp();
        if (bad(now)) {
            if (lane == 0 && now.part == 0 && p.err_word) atomicExch(p.err_word, kErrBadIndex);
        } else {
            const HeadTensor &t = p.t[now.which];
            const uint8_t *mine = rounds + slot * R::kBytes;
            const bool turned = on && now.tok < p.n_rot;
            const float *pc = reinterpret_cast<const float *>(mine + R::kVecs * 16), *ps = pc + DH / 2;
            __nv_bfloat16 *dst = t.y + now.b * t.y_sb + (int64_t)(t.compact_out ? now.r : now.tok) * t.y_sn + l * U;
            const int hb = hr + sub, h1 = now.h1;
#pragma unroll
            for (int k = 0; k < L::kUnroll; ++k) {
                const int h = hb + k * L::kHeads;
                if (h - sub >= h1) break;                          // the whole warp: no head of this step is left
                uint32_t raw[2][kPairs];
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int j = 0; j < L::kUnits; ++j) {
                        load_shared<U>(mine + (k * L::kHeads + (on ? sub : 0)) * (DH * 2) + s * DH + (l + G * j) * (U * 2), &raw[s][j * (U / 2)]);
                    }
                uint32_t w[2][kPairs], bi[2][LAYER ? kPairs : 1];
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int j = 0; j < L::kUnits; ++j) {
                        const uint16_t *pw = weights[now.which] + s * (DH / 2) + (l + G * j) * U;
                        load_shared<U>(pw, &w[s][j * (U / 2)]);
                        if constexpr (LAYER) load_shared<U>(pw + DH, &bi[s][j * (U / 2)]);
                    }
                float co[kPairs * 2], si[kPairs * 2];              // HALF: of the lane's channels; else of the pairs of both of its halves
#pragma unroll
                for (int j = 0; j < L::kUnits; ++j)
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        const int c0 = (l + G * j) * U;             // first channel of the access, in its half
                        const int from = HALF ? c0 + s * (U / 2) : s * (DH / 4) + c0 / 2, to = HALF ? j * U + s * (U / 2) : s * kPairs + j * (U / 2);
#pragma unroll
                        for (int i = 0; i < U / 2; ++i) { co[to + i] = turned ? pc[from + i] : 1.f; si[to + i] = turned ? ps[from + i] : 0.f; }
                    }
                f32x2 z[2][kPairs];
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) z[s][i] = widen(raw[s][i]);
                norm_rotate<DH, LAYER, HALF>(z, w, bi, co, si, p.eps, lane);
                if (on && h < h1) {
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int j = 0; j < L::kUnits; ++j) store_unit<U>(dst + h * t.y_sh + s * (DH / 2) + G * j * U, &z[s][j * (U / 2)]);
                }
            }
        }
        now = next; hr = next_hr; u = next_u;
        slot ^= 1;
    }
}

// Tensors of few heads (keys that many query heads share): a warp's lanes hold heads of several tokens, each with angles of its own, two steps
// of them in flight.  A warp for each token would leave most of its lanes idle.  118800 tokens of 4 x 128, RMS norm, angles for each: 79 us for 304
// MB, 3.9 TB/s; 2 x 32768 of 4 x 72, layer norm, 28 us for 85 MB.  Registers bind it: 119 to 160 a thread, three or four
// blocks a SM.
template <int DH, bool LAYER, bool HALF>
__global__ void __launch_bounds__(kWarps * 32, 3) few_heads_kernel(const __grid_constant__ HeadNormParams p, int which, int B)
{
    using L = Lanes<DH>;
    constexpr int U = L::kUnit, G = L::kGroup, kPairs = L::kUnits * U / 2, kSteps = 2;
    const int lane = threadIdx.x & 31, sub = lane / G, l = lane - sub * G;
    const bool on = sub < L::kHeads;
    grid_launch_dependents();
    grid_dependency_wait();
    const HeadTensor &t = p.t[which];
    const long long rows = (long long)B * t.M * t.H;               // (token, head) pairs
    uint32_t w[2][kPairs], bi[2][LAYER ? kPairs : 1];
    load_weights<DH, LAYER>(t, l, on, w, bi);
    const long long step = (long long)gridDim.x * kWarps * kSteps * L::kHeads;
    for (long long base = ((long long)blockIdx.x * kWarps + (threadIdx.x >> 5)) * kSteps * L::kHeads; base < rows; base += step) {
        uint32_t raw[kSteps][2][kPairs];
        float co[kSteps][kPairs * 2], si[kSteps][kPairs * 2];
        __nv_bfloat16 *dst[kSteps];
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const long long row = base + k * L::kHeads + sub;
            const bool there = on && row < rows;
            const int token = there ? (int)(row / t.H) : 0, h = there ? (int)(row - (long long)token * t.H) : 0;      // (fewer than 2^30 tokens)
            const int b = token / t.M, r = token - b * t.M;
            const int tok = t.idx ? __ldcg(t.idx + token) : r, before = t.idx && r > 0 ? __ldcg(t.idx + token - 1) : -1;
            const bool bad = (unsigned)tok >= (unsigned)p.N || before >= tok;                      // see astraea_scatter_reuse
            if (there && bad && h == 0 && l == 0 && p.err_word) atomicExch(p.err_word, kErrBadIndex);
            const bool good = there && !bad;
            dst[k] = good ? t.y + b * t.y_sb + (int64_t)(t.compact_out ? r : tok) * t.y_sn + h * t.y_sh + l * U : nullptr;
            const __nv_bfloat16 *src = good ? t.x + b * t.x_sb + (int64_t)(t.compact_in ? r : tok) * t.x_sn + h * t.x_sh + l * U : nullptr;
            const bool turned = good && tok < p.n_rot;
            const float *pc = p.cos + (size_t)(turned ? tok : 0) * (DH / 2), *ps = p.sin + (size_t)(turned ? tok : 0) * (DH / 2);
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int j = 0; j < L::kUnits; ++j) {
#pragma unroll
                    for (int i = 0; i < U / 2; ++i) raw[k][s][j * (U / 2) + i] = 0u;
                    if (good) load_unit<U>(src + s * (DH / 2) + G * j * U, &raw[k][s][j * (U / 2)]);
                    const int c0 = (l + G * j) * U;                 // first channel of the access, in its half
                    const int from = HALF ? c0 + s * (U / 2) : s * (DH / 4) + c0 / 2, to = HALF ? j * U + s * (U / 2) : s * kPairs + j * (U / 2);
#pragma unroll
                    for (int i = 0; i < U / 2; ++i) { co[k][to + i] = 1.f; si[k][to + i] = 0.f; }
                    if (turned) { load_table<U / 2>(pc + from, &co[k][to]); load_table<U / 2>(ps + from, &si[k][to]); }
                }
        }
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            f32x2 z[2][kPairs];
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < kPairs; ++i) z[s][i] = widen(raw[k][s][i]);
            norm_rotate<DH, LAYER, HALF>(z, w, bi, co[k], si[k], p.eps, lane);
            if (dst[k]) {
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int j = 0; j < L::kUnits; ++j) store_unit<U>(dst[k] + s * (DH / 2) + G * j * U, &z[s][j * (U / 2)]);
            }
        }
    }
}

template <int DH>
int32_t launch_dim(HeadNormParams &p, int n, int B, bool layer, bool half, cudaStream_t stream)
{
    // a tensor of few heads and many tokens goes by itself (a short one is not worth a launch of its own)
    bool alone[2] = {false, false};
    for (int i = 0; i < n; ++i) alone[i] = p.t[i].H <= Lanes<DH>::kHeads && (long long)B * p.t[i].M > (long long)sm_count() * 64;
    for (int i = 0; i < n; ++i) {
        if (!alone[i]) continue;
        const long long want = ((long long)B * p.t[i].M * p.t[i].H + kWarps * 2 * Lanes<DH>::kHeads - 1) / (kWarps * 2 * Lanes<DH>::kHeads), cap = (long long)sm_count() * 12;
        auto kernel = layer ? (half ? few_heads_kernel<DH, true, true> : few_heads_kernel<DH, true, false>)
                            : (half ? few_heads_kernel<DH, false, true> : few_heads_kernel<DH, false, false>);
        launch_overlapped(kernel, (int)(want < cap ? want : cap), kWarps * 32, 0, stream, p, i, B);
        const int32_t rc = check_launch("astraea_qk_norm_rotate");
        if (rc != ASTRAEA_OK) return rc;
    }
    if (alone[0]) { p.t[0] = p.t[1]; alone[0] = alone[1]; --n; }
    if (n == 2 && alone[1]) n = 1;
    if (n == 0 || (n == 1 && alone[0])) return ASTRAEA_OK;
    // A token's heads go to one warp where that gives every SM the warps that it holds, and are shared out in steps of a warp's heads where it
    // does not: one token of 32 + 8 heads is then 10 warps and not 2.  More shares than there is room for wait, and each reads its token's
    // angles again (us for 600 / 1500 / 2300 rows of 24 x 128 with twice as many 5.9 / 7.2 / 8.2, now 4.3 / 5.9 / 6.2; of 16 x 72, layer norm, 3.8 /
    // 6.3 / 7.6 and 3.8 / 5.1 / 5.3; of 32 x 128 5.7 / 8.3 / 9.7 and 4.9 / 8.4 / 8.6).
    long long all_rows = 0;
    for (int i = 0; i < n; ++i) all_rows += (long long)B * p.t[i].M;
    const long long slots = (long long)sm_count() * (kWarps * kBlocksSM);
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
    constexpr int kSmem = kWarps * 2 * Round<DH>::kBytes;           // 52 KB at head_dim 128
    static_assert(kBlocksSM * (kSmem + 8 * DH + 1024) <= 228 * 1024, "shared memory of the blocks of an SM");
    static PerDeviceOnce attrs;                   // the attribute is per device (all four kernels of the width at once)
    if (attrs.run([] {
            cudaError_t e = cudaSuccess;
            for (auto k : {head_norm_kernel<DH, true, true>, head_norm_kernel<DH, true, false>, head_norm_kernel<DH, false, true>, head_norm_kernel<DH, false, false>})
                if (e == cudaSuccess) e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
            return e;
        }) != cudaSuccess)
        return check_launch("astraea_qk_norm_rotate (shared memory attribute)");
    launch_overlapped(kernel, grid, kWarps * 32, kSmem, stream, p);
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
    case 64: return launch_dim<64>(p, n, B, layer, half, stream);
    case 72: return launch_dim<72>(p, n, B, layer, half, stream);
    default: return launch_dim<128>(p, n, B, layer, half, stream);
    }
}

}  // namespace astraea
