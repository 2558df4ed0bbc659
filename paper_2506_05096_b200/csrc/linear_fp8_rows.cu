// astraea_gathered_linear_fp8 for a handful of rows (a new token of each of a few streams): the same sums as in linear_fp8.cu, but bound by
// the bytes of W, which are read once.
//
// A tile of 256 rows would be nearly empty, and its columns a long chain: one block of 128 channels after the other.  Here a CTA takes 16
// rows of W (output channels), its sixteen warps every sixteenth half of a block each, and a lane's loads of W are 16 bytes, four in flight,
// 32 warps on an SM.  The products are mma.sync m16n8k32 (W's rows as A, rows of x as B): a tensor-memory MMA has 128 rows at least, and at up
// to eight rows its rate is not what is short.  k is permuted so that a lane's 16 contiguous bytes are two of its fragments: lane t of a row
// holds channels 16 t .. 16 t + 15 of a half block of 64, the same ones of W and of x.  A half block's products are scaled by its block's
// scales on the way to fp32 sums, and the warps' sums meet in shared memory.
// us at one / eight rows, and of a tile kernel's launch: 4096 x 4096 7.7 / 8.9, 13.6; 1152 x 4608 3.1 / 4.9, 7.5; 6144 x 1536 5.0 / 6.1, 14.3; 256 x
// 1000 1.8 / 1.9, 4.3.  (Rows and scales of x fetched with W's cost registers and with them resident warps: 4096 x 4096, one row, 10.6 us; eight
// channels a CTA 12.6; at 16 rows the tiles are as fast.)
#include "common.cuh"
#include "epilogue_math.cuh"

namespace astraea {
namespace {

constexpr int kWarps = 16, kOut = 16, kRows = 8;                   // output channels of a CTA, rows of x
constexpr int kUnroll = 2;                                         // half blocks whose loads of W are in flight

struct RowsParams {
    const uint8_t *xq, *wq;
    const float *x_scale, *w_scale;
    const int32_t *idx;
    int M, B, N, K, N_out;
    const __nv_bfloat16 *bias, *residual, *gate;
    __nv_bfloat16 *y;
    int compact, res_compact, gelu;
    int *err_word;
};

__device__ __forceinline__ void mma_e4m3(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__global__ void __launch_bounds__(kWarps * 32, 2) linear_fp8_rows_kernel(const __grid_constant__ RowsParams p)
{
    __shared__ float part[kWarps][kRows][kOut + 1];
    grid_launch_dependents();
    grid_dependency_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int rows = p.B * p.M, n0 = blockIdx.x * kOut, halves = p.K / 64, blocks = p.K / 128;
    const bool low = n0 + g < p.N_out, high = n0 + g + 8 < p.N_out;
    const uint8_t *w0 = p.wq + (size_t)(low ? n0 + g : 0) * p.K + t * 16, *w1 = p.wq + (size_t)(high ? n0 + g + 8 : 0) * p.K + t * 16;
    const uint8_t *x = p.xq + (size_t)(g < rows ? g : 0) * p.K + t * 16;
    const float *ws = p.w_scale + (size_t)(n0 / 128) * blocks;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};                            // channels g, g + 8 for rows 2 t, 2 t + 1
    const uint4 none = make_uint4(0, 0, 0, 0);
    for (int h0 = warp; h0 < halves; h0 += kWarps * kUnroll) {
        uint4 a[kUnroll], b[kUnroll];
        float sw[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int h = h0 + u * kWarps;
            const bool there = h < halves;
            a[u] = there && low ? ld_stream(reinterpret_cast<const uint4 *>(w0 + h * 64)) : none;
            b[u] = there && high ? ld_stream(reinterpret_cast<const uint4 *>(w1 + h * 64)) : none;
            sw[u] = there ? __ldcg(ws + (h >> 1)) : 0.f;
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int h = h0 + u * kWarps;
            if (h >= halves) break;
            const uint4 v = g < rows ? __ldcg(reinterpret_cast<const uint4 *>(x + h * 64)) : none;
            const float *xs = p.x_scale + (size_t)(h >> 1) * rows + 2 * t;
            const float s0 = 2 * t < rows ? sw[u] * __ldcg(xs) : 0.f, s1 = 2 * t + 1 < rows ? sw[u] * __ldcg(xs + 1) : 0.f;
            float c[4] = {0.f, 0.f, 0.f, 0.f};
            mma_e4m3(c, a[u].x, b[u].x, a[u].y, b[u].y, v.x, v.y);
            mma_e4m3(c, a[u].z, b[u].z, a[u].w, b[u].w, v.z, v.w);
            sum[0] = fmaf(c[0], s0, sum[0]); sum[1] = fmaf(c[1], s1, sum[1]);
            sum[2] = fmaf(c[2], s0, sum[2]); sum[3] = fmaf(c[3], s1, sum[3]);
        }
    }
    part[warp][2 * t][g] = sum[0]; part[warp][2 * t + 1][g] = sum[1];
    part[warp][2 * t][g + 8] = sum[2]; part[warp][2 * t + 1][g + 8] = sum[3];
    __syncthreads();
    for (int i = threadIdx.x; i < kRows * kOut; i += kWarps * 32) {
        const int r = i / kOut, n = i % kOut, col = n0 + n;
        if (r >= rows || col >= p.N_out) continue;
        const int b = r / p.M, m = r - b * p.M;
        const int tok = p.idx ? __ldcg(p.idx + r) : m, before = p.idx && m > 0 ? __ldcg(p.idx + r - 1) : -1;
        if ((unsigned)tok >= (unsigned)p.N || before >= tok) {         // see astraea_scatter_reuse
            if (col == 0) atomicExch(p.err_word, kErrBadIndex);
            continue;
        }
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) v += part[w][r][n];
        const long long full = (long long)b * p.N + tok;
        if (p.bias) v += __bfloat162float(p.bias[col]);
        if (p.gelu) {
            float unused;
            unpack2(gelu2(pack2(v, v)), v, unused);
        }
        if (p.gate) v *= __bfloat162float(p.gate[(long long)b * p.N_out + col]);
        if (p.residual) v += __bfloat162float(p.residual[(p.res_compact ? r : full) * p.N_out + col]);
        p.y[(p.compact ? r : full) * p.N_out + col] = __float2bfloat16(v);
    }
}

}  // namespace

int32_t launch_linear_fp8_rows(const void *xq, const float *x_scale, const int32_t *idx, int M, const void *wq, const float *w_scale,
                               const void *bias, const void *residual, const void *gate, void *y, int B, int N, int K, int N_out,
                               uint32_t flags, int *err_word, cudaStream_t stream)
{
    RowsParams p = {};
    p.xq = reinterpret_cast<const uint8_t *>(xq); p.wq = reinterpret_cast<const uint8_t *>(wq);
    p.x_scale = x_scale; p.w_scale = w_scale; p.idx = idx;
    p.M = M; p.B = B; p.N = N; p.K = K; p.N_out = N_out;
    p.bias = reinterpret_cast<const __nv_bfloat16 *>(bias);
    p.residual = reinterpret_cast<const __nv_bfloat16 *>(residual);
    p.gate = reinterpret_cast<const __nv_bfloat16 *>(gate);
    p.y = reinterpret_cast<__nv_bfloat16 *>(y);
    p.compact = (flags & ASTRAEA_LINEAR_COMPACT_OUT) ? 1 : 0;
    p.res_compact = (flags & ASTRAEA_LINEAR_COMPACT_RES) ? 1 : 0;
    p.gelu = (flags & ASTRAEA_LINEAR_GELU) ? 1 : 0;
    p.err_word = err_word;
    launch_overlapped(linear_fp8_rows_kernel, (N_out + kOut - 1) / kOut, kWarps * 32, 0, stream, p);
    return check_launch("astraea_gathered_linear_fp8");
}

}  // namespace astraea
