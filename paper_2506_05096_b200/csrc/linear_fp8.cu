// astraea_gathered_linear_fp8: y[b, idx[b,r], :] = residual + gate * act(x W^T + bias) for rows of x and a W held as e4m3 with a scale for
// each 128 channels of a row and for each block of 128 x 128 of W: the 8-bit form of astraea_gathered_linear(_residual).
//     (x W^T)[r, n] = sum over blocks kb of 128 channels:  x_scale[kb, r] w_scale[n / 128, kb] (xq[r, kb] . wq[n, kb])
// The dot product of a block is the tensor cores' (exact products, fp32 sums); its scale is applied on the way to the sum over blocks,
// which is kept in fp32 registers.
//
// Layout of the launch as in linear.cu: persistent CTA pairs on 256-row x BN-column tiles, tcgen05.mma.cta_group::2 (kind::f8f6f4,
// 256 x BN x 32), rows of x (always one contiguous matrix: the quantiser has gathered them) and W by TMA, one pipeline stage being one
// block of 128 channels = 128 bytes, rows of y scattered by the epilogue.  What differs is where the sum lives: every block gets an
// accumulator of its own in TMEM (two in turn at BN = 256), and eight warps read it, scale it and add it to their registers while the
// tensor cores are at the next block.  (A sum over blocks in the tensor cores would need the scales to be powers of two.)
//
// At BN = 256 the MMAs of a block take 512 clocks and its 32768 FMAs half the FMA pipe's time.  What is scarce is the round trip of an
// accumulator (512 of MMAs, 234 from their end to the warps that wait for it, the reads, 143 for the arrival at the other CTA) and the
// issue slots of the warps that do all this, so: eight warps of 128 columns and not sixteen of 64 (the loop around the FMAs is paid half
// as often), loads of 64 columns, the accumulator released when the last load has landed and before its FMAs, descriptors and phases
// counted on, not computed, scales fetched four blocks ahead.  16384 x 6144 x 6144: 588 -> 413 us on zeros (clocks at their maximum); on
// random codes 503 us = 2.46 PFLOP/s in bursts of a few calls, where the power cap takes the clocks to 1.6 GHz, and 555-605 us = 2.04-2.23 PFLOP/s
// in calls without a pause.  (128-column tiles by two sets of warps in turn, whose epilogues
// overlap, are slower: an MMA of 128 columns takes 80 clocks of the 64 that it should, and a commit for each block more.)
// Warp roles of each CTA:
//   warps 0-7  sums and epilogue: a thread has one row (TMEM lane) and BN / 2 columns, which share the scale of W;
//   warp 8     TMA producer, warp 9 (even CTA) MMA issuer for the pair; warps 10-11 only give their registers away.
// Every mbarrier wait is bounded, and a CTA that gives up leaves as described in linear.cu.
#include "common.cuh"
#include "sm100_ptx.cuh"
#include "bounded_wait.cuh"
#include "epilogue_math.cuh"

namespace astraea {
namespace {

using namespace ptx;

constexpr int kTileRows = 256, kRowsCta = kTileRows / 2, kBK = 128;    // bytes = channels of a stage, and of a scale
constexpr int kSumWarps = 8;
constexpr int kTmaWarp = kSumWarps, kMmaWarp = kTmaWarp + 1;
constexpr int kThreads = (kSumWarps + 4) * 32;
constexpr int kStages = 5;                                              // (six are no faster)
constexpr int kABytes = kRowsCta * kBK, kBBytes = 128 * kBK;           // (B: half of at most 256 columns)
constexpr int kBufBytes = 32 * 64;                                     // 32 rows x 32 bf16 columns on their way to / from global memory
constexpr int kStageBytes = 2 * kBufBytes;                             // per sum warp: two of them in turn
constexpr int kMaxAcc = 4;
constexpr int kAhead = 4;                                              // blocks between the load of a row's scale and its use
constexpr int kBarBytes = 256;
static_assert(8 * (2 * kStages + 2 * kMaxAcc + 1) <= kBarBytes, "barrier area too small");
constexpr int kVecBytes = 2 * 256;                                     // per sum warp: its columns of the bias and of a gate
constexpr int kSmemBytes = kStages * (kABytes + kBBytes) + kBarBytes + kSumWarps * (kStageBytes + kVecBytes) + 1024;
static_assert(kSmemBytes + 512 <= 227 * 1024, "shared memory of one CTA");
constexpr uint32_t kTmemCols = 512;
// registers: 128 sums, 64 values on their way out of TMEM and the addresses of a sum warp against 168 a thread at launch
constexpr int kRegsLaunch = 65536 / kThreads / 8 * 8, kRegsSum = 232, kRegsOther = 40;
static_assert(kRegsSum * kSumWarps * 32 + kRegsOther * 128 <= kRegsLaunch * kThreads, "setmaxnreg budget");

struct Fp8Params {
    const float *x_scale, *w_scale;      // [K / 128][rows], [ceil(N_out / 128)][K / 128]
    const int32_t *idx;
    int M, B, N, K, N_out;
    const __nv_bfloat16 *bias, *residual, *gate;
    __nv_bfloat16 *y;
    int compact, res_compact, gelu;
    int whole;                           // the rows of y lie one behind the other: a warp's go out by TMA
    int *err_word;
};

// C columns of an accumulator, waited for, as pairs.  (One piece of assembly: with single registers that the wait then names, 16384 x 6144 x 6144
// took 590 us instead of 440.)
template <int C> __device__ __forceinline__ void load_pairs(uint32_t t, f32x2 (&a)[C / 2]);
template <> __device__ __forceinline__ void load_pairs<32>(uint32_t t, f32x2 (&a)[16]) {
    asm volatile("{\n\t.reg .b32 t<32>;\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {t0,t1,t2,t3,t4,t5,t6,t7,t8,t9,t10,t11,t12,t13,t14,t15,t16,t17,t18,t19,t20,t21,t22,t23,t24,t25,t26,t27,t28,t29,t30,t31}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;\n\t"
        "mov.b64 %0, {t0,t1}; mov.b64 %1, {t2,t3}; mov.b64 %2, {t4,t5}; mov.b64 %3, {t6,t7}; mov.b64 %4, {t8,t9}; mov.b64 %5, {t10,t11}; mov.b64 %6, {t12,t13}; mov.b64 %7, {t14,t15};"
        "mov.b64 %8, {t16,t17}; mov.b64 %9, {t18,t19}; mov.b64 %10, {t20,t21}; mov.b64 %11, {t22,t23}; mov.b64 %12, {t24,t25}; mov.b64 %13, {t26,t27}; mov.b64 %14, {t28,t29}; mov.b64 %15, {t30,t31};"
        "}"
        : "=l"(a[0]), "=l"(a[1]), "=l"(a[2]), "=l"(a[3]), "=l"(a[4]), "=l"(a[5]), "=l"(a[6]), "=l"(a[7]),
          "=l"(a[8]), "=l"(a[9]), "=l"(a[10]), "=l"(a[11]), "=l"(a[12]), "=l"(a[13]), "=l"(a[14]), "=l"(a[15])
        : "r"(t) : "memory");
}
template <> __device__ __forceinline__ void load_pairs<64>(uint32_t t, f32x2 (&a)[32]) {
    asm volatile("{\n\t.reg .b32 t<64>;\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 {t0,t1,t2,t3,t4,t5,t6,t7,t8,t9,t10,t11,t12,t13,t14,t15,t16,t17,t18,t19,t20,t21,t22,t23,t24,t25,t26,t27,t28,t29,t30,t31,t32,t33,t34,t35,t36,t37,t38,t39,t40,t41,t42,t43,t44,t45,t46,t47,t48,t49,t50,t51,t52,t53,t54,t55,t56,t57,t58,t59,t60,t61,t62,t63}, [%32];\n\t"
        "tcgen05.wait::ld.sync.aligned;\n\t"
        "mov.b64 %0, {t0,t1}; mov.b64 %1, {t2,t3}; mov.b64 %2, {t4,t5}; mov.b64 %3, {t6,t7}; mov.b64 %4, {t8,t9}; mov.b64 %5, {t10,t11}; mov.b64 %6, {t12,t13}; mov.b64 %7, {t14,t15};"
        "mov.b64 %8, {t16,t17}; mov.b64 %9, {t18,t19}; mov.b64 %10, {t20,t21}; mov.b64 %11, {t22,t23}; mov.b64 %12, {t24,t25}; mov.b64 %13, {t26,t27}; mov.b64 %14, {t28,t29}; mov.b64 %15, {t30,t31};"
        "mov.b64 %16, {t32,t33}; mov.b64 %17, {t34,t35}; mov.b64 %18, {t36,t37}; mov.b64 %19, {t38,t39}; mov.b64 %20, {t40,t41}; mov.b64 %21, {t42,t43}; mov.b64 %22, {t44,t45}; mov.b64 %23, {t46,t47};"
        "mov.b64 %24, {t48,t49}; mov.b64 %25, {t50,t51}; mov.b64 %26, {t52,t53}; mov.b64 %27, {t54,t55}; mov.b64 %28, {t56,t57}; mov.b64 %29, {t58,t59}; mov.b64 %30, {t60,t61}; mov.b64 %31, {t62,t63};"
        "}"
        : "=l"(a[0]), "=l"(a[1]), "=l"(a[2]), "=l"(a[3]), "=l"(a[4]), "=l"(a[5]), "=l"(a[6]), "=l"(a[7]),
          "=l"(a[8]), "=l"(a[9]), "=l"(a[10]), "=l"(a[11]), "=l"(a[12]), "=l"(a[13]), "=l"(a[14]), "=l"(a[15]),
          "=l"(a[16]), "=l"(a[17]), "=l"(a[18]), "=l"(a[19]), "=l"(a[20]), "=l"(a[21]), "=l"(a[22]), "=l"(a[23]),
          "=l"(a[24]), "=l"(a[25]), "=l"(a[26]), "=l"(a[27]), "=l"(a[28]), "=l"(a[29]), "=l"(a[30]), "=l"(a[31])
        : "r"(t) : "memory");
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *m, uint32_t bar, int c0, int c1) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4}], [%2];"
        ::"r"(dst), "l"(m), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
// GELU(x) = x Phi(x) of two elements, Phi(x) = 1 / (1 + 2^-g(x)) with g the log2 of Phi(x) / Phi(-x): odd and smooth, x times a polynomial of degree six
// in x^2 over |x| < 5.75 (fitted here for the least error of Phi: 5.4e-8 with fp32 arithmetic) and linear beyond, where Phi(-|x|) is below
// 5e-9.  One reciprocal for both, of the product of their divisors (up to 2^60 each): three XU operations a pair instead of the four of
// gelu2, and 23 clocks of the FMA pipe instead of 27, which an epilogue has more of than anything else.  From a divisor that is held at
// 2^60 (x below -11.7, where Phi is under 2^-100) a factor of 2^-60 would be left, and with it a result that grows with x: 2^-59 is taken off
// both factors, which are zero from there down (for nothing; a select for each takes 13106 x 1152 x 4608 from 115 to 120 us).
__device__ __forceinline__ f32x2 gelu2_odds(f32x2 x) {
    float t0, t1, a0, a1, d0, d1, e0, e1, r;
    unpack2(mul2(x, x), t0, t1);
    const f32x2 t = pack2(fminf(t0, 33.0625f), fminf(t1, 33.0625f));
    f32x2 g = fma2(both(-5.067235e-9f), t, both(3.8163125e-7f));                          // minus the polynomial
    g = fma2(g, t, both(-1.1439834e-5f));
    g = fma2(g, t, both(1.5957994e-4f));
    g = fma2(g, t, both(9.404923e-5f));
    g = fma2(g, t, both(-0.10483512f));
    g = fma2(g, t, both(-2.3022094f));
    unpack2(mul2(x, g), a0, a1);
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(fminf(a0, 60.0f)));                  // (NaN: 60)
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(fminf(a1, 60.0f)));
    unpack2(add2(pack2(e0, e1), both(1.0f)), d0, d1);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d0 * d1));
    return mul2(x, pack2(__saturatef(fmaf(r, d1, -0x1p-59f)), __saturatef(fmaf(r, d0, -0x1p-59f))));
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap *m, uint32_t src, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];"
                 ::"l"(m), "r"(src), "r"(c0), "r"(c1) : "memory");
}
enum { kNothing = 0, kGelu = 1, kAnything = 2 };                       // as in linear.cu

template <int BN, int EPI>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
linear_fp8_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ CUtensorMap tmap_y,
                  const __grid_constant__ Fp8Params p)
{
    constexpr int kAcc = 512 / BN < kMaxAcc ? 512 / BN : kMaxAcc;      // accumulators in turn
    constexpr int kCols = BN / 2;                                      // columns of a sum warp
    constexpr int kLoad = kCols < 64 ? kCols : 64;                     // columns of a load
    constexpr int kChunk = 32, kChunks = kCols / kChunk;               // and of a step of the epilogue
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    __shared__ int stop;                                               // the stages that were sent for before the CTA gave up

    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t sA = smem_base, sB = sA + kStages * kABytes, sBufs = sB + kStages * kBBytes, bars = sBufs + kSumWarps * kStageBytes;
    const uint32_t bar_full = bars, bar_empty = bars + 8 * kStages, bar_acc_full = bars + 16 * kStages,
                   bar_acc_empty = bar_acc_full + 8 * kMaxAcc, bar_end = bar_acc_empty + 8 * kMaxAcc;

    const int tid = threadIdx.x;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);            // warp-uniform
    const int lane = tid & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
    const long long total_rows = (long long)p.B * p.M;
    const int tiles_m = (int)((total_rows + kTileRows - 1) / kTileRows), tiles_n = (p.N_out + BN - 1) / BN;
    const int total_tiles = tiles_m * tiles_n, k_steps = p.K / kBK;

    if (tid == 0) {
        abort_flag = 0;
        stop = 0x7fffffff;
        mbar_init(bar_end, 1);
        for (int s = 0; s < kStages; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_empty + 8 * s, 1); }
        for (int a = 0; a < kMaxAcc; ++a) { mbar_init(bar_acc_full + 8 * a, 1); mbar_init(bar_acc_empty + 8 * a, 2 * kSumWarps); }
        fence_barrier_init();
    }
    if (warp == kTmaWarp && elect_one()) { prefetch_tensormap(&tmap_w); prefetch_tensormap(&tmap_x); prefetch_tensormap(&tmap_y); }
    if (warp == kMmaWarp) {
        tmem_alloc_pair(smem_u32(&tmem_slot), kTmemCols);
        tmem_relinquish_pair();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                                                // the barriers of both CTAs are set up
    tc_fence_after();
    grid_dependency_wait();
    const uint32_t tmem = tmem_slot;

    if (warp < kSumWarps) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSum));
        // ------------------------------------------------ sums over the blocks, epilogue
        const int part = warp >> 2, c0 = part * kCols;
        const int row = (int)rank * kRowsCta + (warp & 3) * 32 + lane;
        const uint32_t t_row = tmem + ((uint32_t)((warp & 3) * 32) << 16) + c0;
        uint8_t *bufs = smem_raw + (sBufs - smem_u32(smem_raw)) + warp * kStageBytes;
        const uint32_t s_bufs = smem_u32(bufs);
        int buf = 0;                                                   // the one that is next
        uint8_t *vectors = smem_raw + (bars + kBarBytes - smem_u32(smem_raw)) + warp * kVecBytes;
        // A thread owns a row of the tile.  Where the rows of y lie one behind the other, a warp's 32 x 32 results go out of shared memory by TMA,
        // under the next step: stores by the warp wait for the L2, which all SMs write to at the same time (13106 x 1152 x 4608: 84 us with
        // them, 72 by TMA, 69 without any).  Rows at places of a list are stored by the warp, in 16-byte pieces: piece q of rows r0 + kStep j (see
        // linear.cu; bulk copies of each row's 64 bytes took 1.4 times as long, TMA scatters of four rows were no faster: 90 us against 87).
        constexpr int kPieces = kChunk / 8, kStep = 32 / kPieces;
        const int q = lane % kPieces, r0 = lane / kPieces;
        auto swizzled = [](int r, int piece) { return r * (kChunk * 2) + ((piece ^ ((kPieces == 8 ? r : r >> 1) & (kPieces - 1))) << 4); };
        // the buffer that is next has been read by the copy before the last
        auto buf_free = [&] {
            bulk_wait_read<1>();
            __syncwarp();
        };
        int acc = 0;
        uint32_t acc_phase = 0;
        // What a tile needs before its first block: the list's entries for its rows, the scales of the first blocks.  They are fetched in
        // front of the epilogue of the tile before (behind it, they were 1500 clocks of every tile).
        // (Loads that no branch guards, from places that exist: what stands for rows, columns and vectors that there are not is not used.  With
        // branches the values were waited for here; 13106 x 1152 x 4608 with GELU 102 -> 98 us.)
        int tok_next = 0, before_next = 0;
        uint4 vec_next = make_uint4(0, 0, 0, 0);                       // lanes 0-15: 8 columns of the bias each, 16-31: of the gate
        int vec_batch = 0;                                             // the batch element that the gate belongs to
        float xs_next[kAhead], ws_lane = 0.f;                          // scales of the row, kAhead blocks ahead (an L2 round trip is longer than a block)
        const int *list = p.idx ? p.idx : reinterpret_cast<const int *>(p.x_scale);
        const __nv_bfloat16 *vec_src = lane < 16 ? (p.bias ? p.bias : p.y) : (EPI == kAnything && p.gate ? p.gate : p.y);
        const bool vec_gate = EPI == kAnything && p.gate && lane >= 16;
        auto fetch = [&](int tile) {
            const int there = tile < total_tiles ? tile : pair;
            const int tm = there / tiles_n, n0 = (there - tm * tiles_n) * BN + c0;
            const long long first = (long long)tm * kTileRows + (int)rank * kRowsCta + (warp & 3) * 32, grow = min(first + lane, total_rows - 1);
            tok_next = __ldcg(list + grow);
            before_next = __ldcg(list + (grow > 0 ? grow - 1 : 0));
#pragma unroll
            for (int u = 0; u < kAhead; ++u) xs_next[u] = __ldcg(p.x_scale + (long long)min(u, k_steps - 1) * total_rows + grow);
            ws_lane = __ldcg(p.w_scale + (long long)(n0 < p.N_out ? n0 / 128 : 0) * k_steps + min(lane, k_steps - 1));
            if (EPI == kAnything) vec_batch = (unsigned)min(first, total_rows - 1) / (unsigned)p.M;
            const int col = n0 + (lane & 15) * 8;
            vec_next = ld_cached(reinterpret_cast<const uint4 *>(vec_src + (vec_gate ? (long long)vec_batch * p.N_out : 0) + (col < p.N_out ? col : 0)));
        };
        fetch(pair);
        for (int tile = pair; tile < total_tiles; tile += n_pairs) {
            const int tm = tile / tiles_n, tn = tile - tm * tiles_n, n0 = tn * BN + c0;
            const long long grow = (long long)tm * kTileRows + row;
            const bool in_range = grow < total_rows;
            // the row of a [B, N, *] tensor; -1: past the end, an entry out of range or one that does not exceed its predecessor
            const int batch = in_range ? (int)((unsigned)grow / (unsigned)p.M) : 0;
            const int place = in_range ? (int)grow - batch * p.M : 0;       // of the row in its list
            const int tok = p.idx ? tok_next : place, before = p.idx && place > 0 ? before_next : -1;
            const bool bad = in_range && ((unsigned)tok >= (unsigned)p.N || before >= tok);
            const long long full_row = in_range && !bad ? (long long)batch * p.N + tok : -1;
            if (bad && tn == 0 && part == 0) atomicExch(p.err_word, kErrBadIndex);
            // the vectors go to shared memory, where every row's thread finds them (the last tile's have been used: the warp has met since)
            *reinterpret_cast<uint4 *>(vectors + lane * 16) = vec_next;
            const bool one_batch = __all_sync(0xffffffffu, full_row < 0 || batch == vec_batch);       // (a gate belongs to a batch element)
            // the first columns of the residual are fetched while the blocks are summed
            uint4 rr[kPieces];
            auto residual_at = [&](int j, int col) -> const __nv_bfloat16 * {
                const int rrow = __shfl_sync(0xffffffffu, full_row < 0 ? -1 : p.res_compact ? (int)grow : (int)full_row, r0 + kStep * j);
                return rrow >= 0 && col < p.N_out ? p.residual + (long long)rrow * p.N_out + col : nullptr;
            };
            if (EPI == kAnything && p.residual) {
                buf_free();
#pragma unroll
                for (int j = 0; j < kPieces; ++j) {
                    const __nv_bfloat16 *src = residual_at(j, n0 + q * 8);
                    cp_async_16(s_bufs + buf * kBufBytes + swizzled(r0 + kStep * j, q), src ? src : p.residual, src != nullptr);
                }
            }
            const float *xs = p.x_scale + (in_range ? grow : 0), *ws = p.w_scale + (long long)(n0 < p.N_out ? n0 / 128 : 0) * k_steps;
            f32x2 sum[kCols / 2];
#pragma unroll
            for (int i = 0; i < kCols / 2; ++i) sum[i] = 0ull;
            for (int ks0 = 0; ks0 < k_steps; ks0 += kAhead) {
                if (ks0 > 0 && (ks0 & 31) == 0) ws_lane = ks0 + lane < k_steps ? __ldcg(ws + ks0 + lane) : 0.f;
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const int ks = ks0 + u;
                    if (ks >= k_steps) break;
                    const float s1 = xs_next[u] * __shfl_sync(0xffffffffu, ws_lane, ks & 31);
                    const f32x2 s = pack2(s1, s1);
                    if (in_range && ks + kAhead < k_steps) xs_next[u] = __ldcg(xs + (long long)(ks + kAhead) * total_rows);
                    wait_bar(bar_acc_full + 8 * acc, acc_phase, &abort_flag, p.err_word);
                    tc_fence_after();
                    const uint32_t t = t_row + acc * BN;
                    auto release = [&] {                               // this warp's part of the accumulator has been read
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_cluster(map_to_rank(bar_acc_empty + 8 * acc, 0));
                    };
#pragma unroll
                    for (int c = 0; c < kCols; c += kLoad) {
                        f32x2 v[kLoad / 2];
                        load_pairs<kLoad>(t + c, v);
                        if (c + kLoad == kCols) release();
#pragma unroll
                        for (int i = 0; i < kLoad / 2; ++i) sum[c / 2 + i] = fma2(v[i], s, sum[c / 2 + i]);
                    }
                    if (++acc == kAcc) { acc = 0; acc_phase ^= 1; }
                }
            }
            if (tile + n_pairs >= total_tiles) grid_launch_dependents();       // the last epilogue of this CTA
            fetch(tile + n_pairs);
            const bool whole = __all_sync(0xffffffffu, p.whole && !bad && !abort_flag);
            int out_row[kPieces];                                           // rows r0 + kStep j of y
#pragma unroll
            for (int j = 0; j < kPieces; ++j)
                out_row[j] = __shfl_sync(0xffffffffu, full_row < 0 || abort_flag ? -1 : p.compact ? (int)grow : (int)full_row, r0 + kStep * j);
            const __nv_bfloat16 *gate = p.gate ? p.gate + (long long)batch * p.N_out : nullptr;
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                const int col0 = n0 + c * kChunk, colq = col0 + q * 8;      // this chunk's columns, the 8 that this lane moves
                uint8_t *stage = bufs + buf * kBufBytes;
                if (!(EPI == kAnything && p.residual) || c > 0) buf_free();
                if (EPI == kAnything && p.residual) {
                    if (c == 0) asm volatile("cp.async.wait_all;" ::: "memory");
                    else {
#pragma unroll
                        for (int j = 0; j < kPieces; ++j) *reinterpret_cast<uint4 *>(stage + swizzled(r0 + kStep * j, q)) = rr[j];
                    }
                    __syncwarp();
                    if (c + 1 < kChunks) {
#pragma unroll
                        for (int j = 0; j < kPieces; ++j) {
                            const __nv_bfloat16 *src = residual_at(j, colq + kChunk);
                            rr[j] = src ? __ldcg(reinterpret_cast<const uint4 *>(src)) : make_uint4(0, 0, 0, 0);
                        }
                    }
                }
                // (all of a step's loads first, then its arithmetic: there are two warps on a scheduler to hide latencies)
                f32x2 f[kChunk / 2];
                uint4 vec[kPieces];
                if (p.bias) {
#pragma unroll
                    for (int v = 0; v < kPieces; ++v) vec[v] = *reinterpret_cast<const uint4 *>(vectors + (c * kPieces + v) * 16);
#pragma unroll
                    for (int v = 0; v < kPieces; ++v) {
                        f32x2 t[4];
                        unpack8(vec[v], t);
#pragma unroll
                        for (int i = 0; i < 4; ++i) f[v * 4 + i] = add2(sum[c * 16 + v * 4 + i], t[i]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < kChunk / 2; ++i) f[i] = sum[c * 16 + i];
                }
                if (EPI == kGelu || (EPI == kAnything && p.gelu)) {
#pragma unroll
                    for (int i = 0; i < kChunk / 2; ++i) f[i] = gelu2_odds(f[i]);
                }
                if (EPI == kAnything && gate) {
#pragma unroll
                    for (int v = 0; v < kPieces; ++v)
                        vec[v] = one_batch ? *reinterpret_cast<const uint4 *>(vectors + 256 + (c * kPieces + v) * 16)
                               : col0 + v * 8 < p.N_out ? ld_cached(reinterpret_cast<const uint4 *>(gate + col0 + v * 8)) : make_uint4(0, 0, 0, 0);
#pragma unroll
                    for (int v = 0; v < kPieces; ++v) {
                        f32x2 t[4];
                        unpack8(vec[v], t);
#pragma unroll
                        for (int i = 0; i < 4; ++i) f[v * 4 + i] = mul2(f[v * 4 + i], t[i]);
                    }
                }
#pragma unroll
                for (int v = 0; v < kPieces; ++v) {
                    uint4 *mine = reinterpret_cast<uint4 *>(stage + swizzled(lane, v));     // residual in, result out
                    if (EPI == kAnything && p.residual) {
                        f32x2 t[4];
                        unpack8(*mine, t);
#pragma unroll
                        for (int i = 0; i < 4; ++i) f[v * 4 + i] = add2(f[v * 4 + i], t[i]);
                    }
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float lo, hi;
                        unpack2(f[v * 4 + i], lo, hi);
                        __nv_bfloat162 v2 = __floats2bfloat162_rn(lo, hi);
                        w[i] = *reinterpret_cast<uint32_t *>(&v2);
                    }
                    *mine = make_uint4(w[0], w[1], w[2], w[3]);
                }
                if (whole) {
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0 && col0 < p.N_out && grow < total_rows) tma_store_2d(&tmap_y, s_bufs + buf * kBufBytes, col0, (int)grow);
                } else {
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < kPieces; ++j) {
                        const uint4 t = *reinterpret_cast<const uint4 *>(stage + swizzled(r0 + kStep * j, q));
                        if (out_row[j] >= 0 && colq < p.N_out) *reinterpret_cast<uint4 *>(p.y + (long long)out_row[j] * p.N_out + colq) = t;
                    }
                    __syncwarp();
                }
                bulk_commit();                           // (a group for every step, so that buf_free can count them)
                buf ^= 1;
            }
        }
        bulk_wait<0>();
    } else if (warp == kTmaWarp) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
        // ------------------------------------------------ TMA producer (the bytes of both CTAs are counted on the even one's barrier)
        const uint32_t full0 = map_to_rank(bar_full, 0);
        auto gave_up = [&] { return *static_cast<volatile int *>(&abort_flag) != 0; };
        auto going = [&](int g) -> bool {                              // once the CTA has given up, stage g and those after it are not sent for
            if (gave_up()) stop = min(stop, g);
            return stop > g;
        };
        int g = 0, st = 0;
        uint32_t phase = 1;
        for (int tile = pair; tile < total_tiles; tile += n_pairs) {
            const int tm = tile / tiles_n, tn = tile - tm * tiles_n;
            for (int ks = 0; ks < k_steps; ++ks, ++g) {
                wait_bar(bar_empty + 8 * st, phase, &abort_flag, p.err_word);
                if (elect_one() && going(g)) {
                    if (rank == 0) mbar_arrive_expect_tx(bar_full + 8 * st, 2 * (BN / 2 * kBK + kABytes));
                    tma_load_2d(sB + st * kBBytes, &tmap_w, full0 + 8 * st, ks * kBK, tn * BN + (int)rank * (BN / 2));
                    tma_load_2d(sA + st * kABytes, &tmap_x, full0 + 8 * st, ks * kBK, tm * kTileRows + (int)rank * kRowsCta);
                }
                __syncwarp();
                if (++st == kStages) { st = 0; phase ^= 1; }
            }
        }
        // every copy issued above must have landed before either CTA's shared memory is released (see linear.cu)
        if (gave_up()) { __syncwarp(); g = min(g, stop) + 1; }
        for (int gs = (g > kStages ? g - kStages : 0); rank == 0 && gs < g; ++gs)
            drain_bar(bar_full + 8 * (gs % kStages), (gs / kStages) & 1);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
        if (warp == kMmaWarp && rank == 0) {
            // -------------------------------------------- MMA issuer of the pair
            constexpr uint32_t idesc = idesc_e4m3(kTileRows, BN);
            const uint64_t desc_a = smem_desc(sA, 16, 1024, kSwizzle128B), desc_b = smem_desc(sB, 16, 1024, kSwizzle128B);    // of the first stage
            int st = 0, acc = 0;
            uint32_t phase = 0, acc_phase = 1;
            for (int tile = pair; tile < total_tiles; tile += n_pairs) {
                for (int ks = 0; ks < k_steps; ++ks) {
                    // (what TMA has brought to either CTA is there for the MMAs once its bytes are counted: no fence between)
                    wait_bar(bar_full + 8 * st, phase, &abort_flag, p.err_word);
                    wait_bar<true>(bar_acc_empty + 8 * acc, acc_phase, &abort_flag, p.err_word);
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t a = desc_a + (uint32_t)st * (kABytes / 16), b = desc_b + (uint32_t)st * (kBBytes / 16);
#pragma unroll
                        for (int kk = 0; kk < kBK / 32; ++kk) mma_ss_pair_f8(tmem + acc * BN, a + kk * 2, b + kk * 2, idesc, kk > 0 ? 1u : 0u);
                        tc_commit_pair(bar_acc_full + 8 * acc);
                        tc_commit_pair(bar_empty + 8 * st);
                    }
                    __syncwarp();
                    if (++st == kStages) { st = 0; phase ^= 1; }
                    if (++acc == kAcc) { acc = 0; acc_phase ^= 1; }
                }
            }
        }
    }

    // neither CTA leaves (or gives up its TMEM) while the other may still arrive on its barriers or read its shared memory
    tc_fence_before();
    __syncthreads();
    if (abort_flag && rank == 0 && warp == kMmaWarp) {                 // MMAs that are under way end before their memory is given up
        if (elect_one()) { tc_commit_pair(bar_end); drain_bar(bar_end, 0); }
        __syncwarp();
    }
    cluster_sync_all();
    if (warp == kMmaWarp) tmem_dealloc_pair(tmem, kTmemCols);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// a row-major matrix of bytes [rows, K] with 128-byte-swizzled boxes of 128 columns x box_rows; rows past the end read as zero
int32_t make_byte_map(CUtensorMap *map, const void *base, long long rows, int K, int box_rows, const char *what)
{
    const EncodeTiledFn enc = reinterpret_cast<EncodeTiledFn>(tensor_map_encoder());
    if (!enc) return fail(ASTRAEA_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
    cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)K};
    cuuint32_t box[2] = {(cuuint32_t)kBK, (cuuint32_t)box_rows};
    cuuint32_t estr[2] = {1, 1};
    CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, estr,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(ASTRAEA_ERR_INVALID_ARG, "astraea_gathered_linear_fp8: tensor map of %s rejected (CUresult %d)", what, (int)r);
    return ASTRAEA_OK;
}

// y as a matrix of rows one behind the other, by boxes of 32 columns x 32 rows; what lies outside is not written
int32_t make_y_map(CUtensorMap *map, void *base, long long rows, int N_out)
{
    const EncodeTiledFn enc = reinterpret_cast<EncodeTiledFn>(tensor_map_encoder());
    cuuint64_t dims[2] = {(cuuint64_t)N_out, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)N_out * 2};
    cuuint32_t box[2] = {32, 32};
    cuuint32_t estr[2] = {1, 1};
    CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, dims, strides, box, estr,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(ASTRAEA_ERR_INVALID_ARG, "astraea_gathered_linear_fp8: tensor map of y rejected (CUresult %d)", (int)r);
    return ASTRAEA_OK;
}

template <int BN, int EPI>
int32_t launch_tiles(const Fp8Params &p, const void *xq, const void *wq, int pairs, cudaStream_t stream)
{
    CUtensorMap mw, mx;
    int32_t rc = make_byte_map(&mw, wq, p.N_out, p.K, BN / 2, "wq");
    if (rc == ASTRAEA_OK) rc = make_byte_map(&mx, xq, (long long)p.B * p.M, p.K, kRowsCta, "xq");
    CUtensorMap my = mx;                          // (not used for rows that are not one behind the other)
    if (rc == ASTRAEA_OK && p.whole) rc = make_y_map(&my, p.y, (long long)p.B * p.M, p.N_out);
    if (rc != ASTRAEA_OK) return rc;
    static PerDeviceOnce attrs;                   // the attribute is per device
    if (attrs.run([] { return cudaFuncSetAttribute(linear_fp8_kernel<BN, EPI>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes); }) != cudaSuccess)
        return check_launch("astraea_gathered_linear_fp8 (shared memory attribute)");
    const long long tiles = (((long long)p.B * p.M + kTileRows - 1) / kTileRows) * ((p.N_out + BN - 1) / BN);
    launch_overlapped(linear_fp8_kernel<BN, EPI>, 2 * (int)(tiles < pairs ? tiles : pairs), kThreads, kSmemBytes, stream, mw, mx, my, p);
    return check_launch("astraea_gathered_linear_fp8");
}

template <int BN>
int32_t launch_epi(const Fp8Params &p, const void *xq, const void *wq, int pairs, cudaStream_t stream)
{
    if (p.residual || p.gate) return launch_tiles<BN, kAnything>(p, xq, wq, pairs, stream);
    return p.gelu ? launch_tiles<BN, kGelu>(p, xq, wq, pairs, stream) : launch_tiles<BN, kNothing>(p, xq, wq, pairs, stream);
}

}  // namespace

int32_t launch_gathered_linear_fp8(const void *xq, const float *x_scale, const int32_t *idx, int M, const void *wq, const float *w_scale,
                                   const void *bias, const void *residual, const void *gate, void *y, int B, int N, int K, int N_out,
                                   uint32_t flags, int *err_word, cudaStream_t stream)
{
    if ((long long)B * (idx ? M : N) <= kFewRows)
        return launch_linear_fp8_rows(xq, x_scale, idx, idx ? M : N, wq, w_scale, bias, residual, gate, y, B, N, K, N_out, flags, err_word, stream);
    Fp8Params p = {};
    p.x_scale = x_scale; p.w_scale = w_scale; p.idx = idx;
    p.M = idx ? M : N; p.B = B; p.N = N; p.K = K; p.N_out = N_out;
    p.bias = reinterpret_cast<const __nv_bfloat16 *>(bias);
    p.residual = reinterpret_cast<const __nv_bfloat16 *>(residual);
    p.gate = reinterpret_cast<const __nv_bfloat16 *>(gate);
    p.y = reinterpret_cast<__nv_bfloat16 *>(y);
    p.compact = (flags & ASTRAEA_LINEAR_COMPACT_OUT) ? 1 : 0;
    p.res_compact = (flags & ASTRAEA_LINEAR_COMPACT_RES) ? 1 : 0;
    p.gelu = (flags & ASTRAEA_LINEAR_GELU) ? 1 : 0;
    p.whole = !idx || p.compact ? 1 : 0;
    p.err_word = err_word;
    const int pairs = sm_count() / 2 > 0 ? sm_count() / 2 : 1;
    const long long tiles_m = ((long long)B * p.M + kTileRows - 1) / kTileRows;
    // A round of narrower tiles costs less, but not in proportion; 256 columns, unless narrower ones make up for it by the rounds.  us with 256 /
    // 128 / 64 columns: 16384 x 6144 x 6144 517 / 592 / 823, 13106 x 1152 x 4608 94 / 101 / 139, 1846 x 6144 x 1536 26.5 / 29.4 / 33.2; 256 x
    // 4096 x 4096 18.4 / 12.4 / 11.4, 77 x 1536 x 1536 9.8 / 7.1 / 6.4.
    int bn = 256;
    double best = 0.0;
    for (int w = 256; w >= 64; w /= 2) {
        const long long tiles = tiles_m * ((N_out + w - 1) / w);
        const double t = (double)((tiles + pairs - 1) / pairs) * (w == 256 ? 1.0 : w == 128 ? 0.62 : 0.42);
        if (best == 0.0 || t < 0.97 * best) { best = t; bn = w; }
    }
    switch (bn) {
    case 256: return launch_epi<256>(p, xq, wq, pairs, stream);
    case 128: return launch_epi<128>(p, xq, wq, pairs, stream);
    default: return launch_epi<64>(p, xq, wq, pairs, stream);
    }
}

}  // namespace astraea
