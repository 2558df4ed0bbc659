// astraea_quantize_fp8: the listed rows of x as e4m3 with a scale for each row and 128 channels; astraea_quantize_fp8_weight: a weight
// matrix as e4m3 with a scale for each block of 128 x 128.  The operands of astraea_gathered_linear_fp8.
//     scale = max(largest magnitude of the block, 2^-100) / 448,    q = x / scale rounded to e4m3 (ties to even)
// so that the largest value of a block takes the largest code (448) and the scales of all-zero blocks stay normal numbers.
//
// HBM-bound: two bytes in and one out for every value.  A warp takes a row; a block of 128 channels is 16 lanes with 16 bytes each, whose
// largest magnitude goes round by four shuffles.  Four pairs of blocks are in flight per warp.  The quotient by the stored scale is x times both
// parts of 1 / scale, which is the correctly rounded fp32 quotient for all but a few operands.  bf16 values have many quotients x 448 / amax that are
// ties of e4m3, or so close to one that the roundings to fp32 of the scale and of the quotient decide: a code is within half a step and 2^-22 of
// the value, and about 1 in 1000 codes of normal values is the other neighbour of a tie than in exact arithmetic (a plain
// product moves 1 in 2000 more).
#include "common.cuh"

namespace astraea {
namespace {

constexpr float kE4M3Max = 448.0f, kLeastAmax = 7.888609052210118e-31f;       // 2^-100
constexpr int kWarps = 8;
constexpr int kUnroll = 4;

// the larger magnitude of each half, NaN left out (signs are of no account until the end)
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
    uint32_t m;
    asm("max.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
    return m;
}
__device__ __forceinline__ uint32_t largest(const uint4 &v) { return larger(larger(v.x, v.y), larger(v.z, v.w)); }
// of both halves, as fp32
__device__ __forceinline__ float magnitude(uint32_t m) { return fmaxf(fabsf(__uint_as_float(m << 16)), fabsf(__uint_as_float(m & 0xffff0000u))); }

// The scale: a product with 1 / 448 and a step by its residual.  1 / scale as the sum of two numbers: a step of Newton's iteration behind an
// approximate reciprocal, and the residual that it leaves.
struct BlockScale { float scale, inv, low; };
__device__ __forceinline__ BlockScale scale_of(float amax) {
    BlockScale s;
    const float a = fmaxf(amax, kLeastAmax), q = a * (1.0f / kE4M3Max);
    s.scale = fmaf(fmaf(q, -kE4M3Max, a), 1.0f / kE4M3Max, q);
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s.scale));
    s.inv = fmaf(fmaf(-s.scale, r, 1.0f), r, r);
    s.low = fmaf(-s.scale, s.inv, 1.0f) * s.inv;
    // an infinity in the block: 0 for what is finite, NaN for what is not
    if (a == INFINITY) { s.scale = a; s.inv = 0.f; s.low = 0.f; }
    return s;
}
// eight values as e4m3
__device__ __forceinline__ uint2 encode8(const uint4 &v, const BlockScale &s) {
    f32x2 x[4];
    unpack8(v, x);
    const f32x2 inv = pack2(s.inv, s.inv), low = pack2(s.low, s.low);
    uint32_t out[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 q = fma2(x[i], inv, mul2(x[i], low));
        float lo, hi;
        unpack2(q, lo, hi);
        uint16_t c;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(hi), "f"(lo));
        if (i & 1) out[i >> 1] |= (uint32_t)c << 16; else out[i >> 1] = c;
    }
    return make_uint2(out[0], out[1]);
}

__global__ void __launch_bounds__(kWarps * 32)
quantize_rows_kernel(const uint4 *__restrict__ x, const int32_t *__restrict__ idx, int M, uint2 *__restrict__ xq, float *__restrict__ scale,
                     int B, int N, int blocks, int parts, int part_blocks, int compact_in, int *__restrict__ err_word)
{
    grid_launch_dependents();
    grid_dependency_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, vecs = blocks * 16;
    const long long rows = (long long)B * M, units = rows * parts;
    // neighbouring warps take neighbouring rows: the scales of a block of channels lie side by side by row
    for (long long u = (long long)blockIdx.x * kWarps + warp; u < units; u += (long long)gridDim.x * kWarps) {
        const int part = (int)(u / rows);
        const long long t = u - part * rows;
        const int b = (int)(t / M), r = (int)(t - (long long)b * M);
        const int tok = idx ? __ldcg(idx + t) : r;
        const int before = (idx && r > 0) ? __ldcg(idx + t - 1) : -1;
        const bool bad = (unsigned)tok >= (unsigned)N || before >= tok;
        if (bad && lane == 0 && part == 0 && err_word) atomicExch(err_word, kErrBadIndex);
        if (bad) continue;                                          // its row of codes and scales is left as it was
        const uint4 *src = x + (compact_in ? t : (long long)b * N + tok) * vecs;
        uint2 *dst = xq + t * vecs;
        const int k0 = part * part_blocks, k1 = min(blocks, k0 + part_blocks);
        uint4 v[kUnroll], ahead[kUnroll];
        auto fetch = [&](int kb) {
#pragma unroll
            for (int i = 0; i < kUnroll; ++i) {
                const int c = (kb + 2 * i) * 16 + lane;
                ahead[i] = c < k1 * 16 ? ld_stream(src + c) : make_uint4(0, 0, 0, 0);
            }
        };
        fetch(k0);
        for (int kb = k0; kb < k1; kb += 2 * kUnroll) {
#pragma unroll
            for (int i = 0; i < kUnroll; ++i) v[i] = ahead[i];
            if (kb + 2 * kUnroll < k1) fetch(kb + 2 * kUnroll);
#pragma unroll
            for (int i = 0; i < kUnroll; ++i) {
                const int c = (kb + 2 * i) * 16 + lane;
                uint32_t m = largest(v[i]);
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) m = larger(m, __shfl_xor_sync(0xffffffffu, m, o));
                const BlockScale s = scale_of(magnitude(m));
                if (c < k1 * 16) {
                    dst[c] = encode8(v[i], s);
                    if ((lane & 15) == 0) scale[(long long)(c >> 4) * rows + t] = s.scale;
                }
            }
        }
    }
}

// one CTA per block of 128 x 128: 256 threads, eight 16-byte vectors each (12288 x 12288 68 us, 6.4 TB/s; 4608 x 1152 4.3 us)
__global__ void __launch_bounds__(256)
quantize_weight_kernel(const uint4 *__restrict__ w, uint2 *__restrict__ wq, float *__restrict__ scale, int N_out, int blocks)
{
    __shared__ float part[8];
    grid_launch_dependents();
    grid_dependency_wait();
    const int kb = blockIdx.x, nb = blockIdx.y, lane = threadIdx.x & 31, c = threadIdx.x & 15, r0 = threadIdx.x >> 4;
    uint4 v[8];
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = nb * 128 + r0 + 16 * i;
        v[i] = row < N_out ? ld_stream(w + ((long long)row * blocks + kb) * 16 + c) : make_uint4(0, 0, 0, 0);
        m = fmaxf(m, magnitude(largest(v[i])));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (lane == 0) part[threadIdx.x >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, part[i]);
    const BlockScale s = scale_of(m);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = nb * 128 + r0 + 16 * i;
        if (row < N_out) wq[((long long)row * blocks + kb) * 16 + c] = encode8(v[i], s);
    }
    if (threadIdx.x == 0) scale[(long long)nb * blocks + kb] = s.scale;
}

}  // namespace

int32_t launch_quantize_fp8(const void *x, const int32_t *idx, int M, void *xq, float *x_scale, int B, int N, int K, bool compact_in,
                            int *err_word, cudaStream_t stream)
{
    const int rows_each = idx ? M : N, blocks = K / 128;
    const long long rows = (long long)B * rows_each;
    if (rows == 0) return ASTRAEA_OK;
    // A row is one warp's, but in short launches its blocks are shared out over warps, a pair of blocks at least
    const long long slots = (long long)sm_count() * 32;
    const int pairs = (blocks + 1) / 2;
    long long want = slots / rows;
    want = want < 1 ? 1 : want > pairs ? pairs : want;
    const int part_blocks = (int)((pairs + want - 1) / want) * 2, parts = (blocks + part_blocks - 1) / part_blocks;
    const long long ctas = (rows * parts + kWarps - 1) / kWarps, cap = (long long)sm_count() * 8;
    launch_overlapped(quantize_rows_kernel, (int)(ctas < cap ? ctas : cap), kWarps * 32, 0, stream, reinterpret_cast<const uint4 *>(x), idx, rows_each,
                      reinterpret_cast<uint2 *>(xq), x_scale, B, N, blocks, parts, part_blocks, compact_in ? 1 : 0, err_word);
    return check_launch("astraea_quantize_fp8");
}

int32_t launch_quantize_fp8_weight(const void *w, void *wq, float *w_scale, int N_out, int K, cudaStream_t stream)
{
    launch_overlapped(quantize_weight_kernel, dim3(K / 128, (N_out + 127) / 128), 256, 0, stream, reinterpret_cast<const uint4 *>(w),
                      reinterpret_cast<uint2 *>(wq), w_scale, N_out, K / 128);
    return check_launch("astraea_quantize_fp8_weight");
}

}  // namespace astraea
