// astraea_gathered_linear_fp8: y[b, idx[b,r], :] = residual + gate * act(x W^T + bias) for rows of x and a W held as e4m3 with a scale for
// each 128 channels of a row and for each block of 128 x 128 of W: the 8-bit form of astraea_gathered_linear(_residual).
//     (x W^T)[r, n] = sum over blocks kb of 128 channels:  x_scale[kb, r] w_scale[n / 128, kb] (xq[r, kb] . wq[n, kb])
// The dot product of a block is the tensor cores' (exact products, fp32 sums); its scale is applied on the way to the sum over blocks,
// which is kept in fp32 registers.
//
// Layout of the launch as in linear.cu: persistent CTA pairs on 256-row x BN-column tiles, tcgen05.mma.cta_group::2 (kind::f8f6f4,
// 256 x BN x 32), rows of x (always one contiguous matrix: the quantiser has gathered them) and W by TMA, one pipeline stage being one
// block of 128 channels = 128 bytes, rows of y scattered by the epilogue.  What differs is where the sum lives: every block gets an
// accumulator of its own in TMEM (512 / BN of them, in turn), and sixteen warps read it, scale it and add it to their registers while the
// tensor cores are at the next blocks.  Four MMAs of a block at BN = 256 take 512 clocks of the tensor pipe; reading its 128 x 256 values
// and the 16384 packed FMAs on them take half the issue slots of that time.  (A sum over blocks in the tensor cores would need the scales
// to be powers of two.)
// Warp roles of each CTA:
//   warps 0-15  sums and epilogue: a thread has one row (TMEM lane) and BN / 4 columns; a warp's columns share the scale of W;
//   warp 16     TMA producer, warp 17 (even CTA) MMA issuer for the pair; warps 18-19 only give their registers away.
// Every mbarrier wait is bounded, and a CTA that gives up leaves as described in linear.cu.
#include "common.cuh"
#include "sm100_ptx.cuh"
#include "bounded_wait.cuh"
#include "epilogue_math.cuh"

namespace astraea {
namespace {

using namespace ptx;

constexpr int kTileRows = 256, kRowsCta = kTileRows / 2, kBK = 128;    // bytes = channels of a stage, and of a scale
constexpr int kSumWarps = 16;
constexpr int kTmaWarp = kSumWarps, kMmaWarp = kTmaWarp + 1;
constexpr int kThreads = (kSumWarps + 4) * 32;
constexpr int kStages = 6;
constexpr int kABytes = kRowsCta * kBK, kBBytes = 128 * kBK;           // (B: half of at most 256 columns)
constexpr int kStageBytes = 32 * 64;                                   // per sum warp: 32 rows x 32 bf16 columns on their way to / from global memory
constexpr int kMaxAcc = 4;
constexpr int kBarBytes = 256;
static_assert(8 * (2 * kStages + 2 * kMaxAcc + 1) <= kBarBytes, "barrier area too small");
constexpr int kSmemBytes = kStages * (kABytes + kBBytes) + kBarBytes + kSumWarps * kStageBytes + 1024;
static_assert(kSmemBytes + 512 <= 227 * 1024, "shared memory of one CTA");
constexpr uint32_t kTmemCols = 512;
// registers: 64 sums, 32 values on their way out of TMEM and the addresses of a sum warp against 96 a thread at launch
constexpr int kRegsLaunch = 65536 / kThreads / 8 * 8, kRegsSum = 112, kRegsOther = 32;
static_assert(kRegsSum * kSumWarps * 32 + kRegsOther * 128 <= kRegsLaunch * kThreads, "setmaxnreg budget");

struct Fp8Params {
    const float *x_scale, *w_scale;      // [K / 128][rows], [ceil(N_out / 128)][K / 128]
    const int32_t *idx;
    int M, B, N, K, N_out;
    const __nv_bfloat16 *bias, *residual, *gate;
    __nv_bfloat16 *y;
    int compact, res_compact, gelu;
    int *err_word;
};

// columns [col, col + 32) or [col, col + 16) of an accumulator
template <int C> __device__ __forceinline__ void tmem_ld(uint32_t taddr, uint32_t (&r)[C]) {
    if constexpr (C == 32) tmem_ld32(taddr, r); else tmem_ld16(taddr, r);
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *m, uint32_t bar, int c0, int c1) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4}], [%2];"
        ::"r"(dst), "l"(m), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
// one output row: of a [B, N, *] tensor, or -1 (past the end, an entry out of range or not ascending)
__device__ __forceinline__ long long target_row(const Fp8Params &p, long long g, long long total, int *batch, bool *bad) {
    *bad = false;
    if (g >= total) return -1;
    const int b = (int)((unsigned)g / (unsigned)p.M), r = (int)((unsigned)g - (unsigned)b * (unsigned)p.M);
    const int tok = p.idx ? __ldcg(p.idx + g) : r;
    const int before = (p.idx && r > 0) ? __ldcg(p.idx + g - 1) : -1;
    if ((unsigned)tok >= (unsigned)p.N || (r > 0 && before >= tok)) { *bad = true; return -1; }
    *batch = b;
    return (long long)b * p.N + tok;
}

enum { kNothing = 0, kGelu = 1, kAnything = 2 };                       // as in linear.cu

template <int BN, int EPI>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
linear_fp8_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ Fp8Params p)
{
    constexpr int kAcc = 512 / BN < kMaxAcc ? 512 / BN : kMaxAcc;      // accumulators in turn
    constexpr int kCols = BN / 4;                                      // columns of a sum warp
    constexpr int kChunk = kCols < 32 ? kCols : 32, kChunks = kCols / kChunk;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    __shared__ int stop;                                               // the stages that were sent for before the CTA gave up

    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t sA = smem_base, sB = sA + kStages * kABytes, bars = sB + kStages * kBBytes;
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
    if (warp == kTmaWarp && elect_one()) { prefetch_tensormap(&tmap_w); prefetch_tensormap(&tmap_x); }
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
        uint8_t *stage = smem_raw + (bars + kBarBytes - smem_u32(smem_raw)) + warp * kStageBytes;
        const uint32_t s_stage = smem_u32(stage);
        // a thread owns a row of the tile, and global memory is touched in 16-byte pieces: piece q of rows r0 + kStep j (see linear.cu)
        constexpr int kPieces = kChunk / 8, kStep = 32 / kPieces, kRowBytes = kChunk * 2;
        const int q = lane % kPieces, r0 = lane / kPieces;
        auto swizzled = [](int r, int piece) { return r * kRowBytes + ((piece ^ ((r >> (kPieces == 4 ? 1 : 2)) & (kPieces - 1))) << 4); };
        int g = 0;
        for (int tile = pair; tile < total_tiles; tile += n_pairs) {
            const int tm = tile / tiles_n, tn = tile - tm * tiles_n, n0 = tn * BN + c0;
            const long long grow = (long long)tm * kTileRows + row;
            int batch = 0;
            bool bad;
            long long full_row = target_row(p, grow, total_rows, &batch, &bad);
            if (bad && tn == 0 && part == 0) atomicExch(p.err_word, kErrBadIndex);
            const unsigned in_list = __ballot_sync(0xffffffffu, full_row >= 0);
            const int batch0 = __shfl_sync(0xffffffffu, batch, in_list ? __ffs(in_list) - 1 : 0);
            const bool one_batch = __all_sync(0xffffffffu, full_row < 0 || batch == batch0);       // (a gate belongs to a batch element)
            // fetched while the blocks are summed: 8 columns of the bias (lanes 0-7) and of the gate (8-15), the first columns of the residual
            uint4 vec = make_uint4(0, 0, 0, 0);
            {
                const int col = n0 + (lane & 7) * 8;
                const __nv_bfloat16 *src = lane < 8 ? p.bias : EPI == kAnything && lane < 16 && p.gate ? p.gate + (long long)batch0 * p.N_out : nullptr;
                if (src && (lane & 7) * 8 < kCols && col < p.N_out) vec = ld_cached(reinterpret_cast<const uint4 *>(src + col));
            }
            const long long res_row = (full_row >= 0 && p.res_compact) ? grow : full_row;
            if (EPI == kAnything && p.residual) {
#pragma unroll
                for (int j = 0; j < kPieces; ++j) {
                    const int r = r0 + kStep * j;
                    const long long rrow = __shfl_sync(0xffffffffu, res_row, r);
                    const bool there = rrow >= 0 && n0 + q * 8 < p.N_out;
                    cp_async_16(s_stage + swizzled(r, q), p.residual + (there ? rrow * p.N_out + n0 + q * 8 : 0), there);
                }
            }
            const bool in_range = grow < total_rows;
            const float *xs = p.x_scale + (in_range ? grow : 0);
            const float *ws = p.w_scale + (long long)(n0 < p.N_out ? n0 / 128 : 0) * k_steps;
            float xs_next = in_range ? __ldcg(xs) : 0.f, ws_lane = 0.f;
            f32x2 sum[kCols / 2];
#pragma unroll
            for (int i = 0; i < kCols / 2; ++i) sum[i] = 0ull;
            for (int ks = 0; ks < k_steps; ++ks, ++g) {
                if ((ks & 31) == 0) ws_lane = ks + lane < k_steps ? __ldcg(ws + ks + lane) : 0.f;
                const float s = xs_next * __shfl_sync(0xffffffffu, ws_lane, ks & 31);
                if (ks + 1 < k_steps && in_range) xs_next = __ldcg(xs + (long long)(ks + 1) * total_rows);
                const int acc = g % kAcc;
                wait_bar(bar_acc_full + 8 * acc, (g / kAcc) & 1, &abort_flag, p.err_word);
                tc_fence_after();
                const f32x2 s2 = pack2(s, s);
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    uint32_t v[kChunk];
                    tmem_ld<kChunk>(t_row + acc * BN + c * kChunk, v);
                    tc_wait_ld();
                    if (c == kChunks - 1) {                            // this warp's part of the accumulator has been read
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_cluster(map_to_rank(bar_acc_empty + 8 * acc, 0));
                    }
#pragma unroll
                    for (int i = 0; i < kChunk / 2; ++i)
                        sum[c * (kChunk / 2) + i] = fma2(pack2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), s2, sum[c * (kChunk / 2) + i]);
                }
            }
            if (tile + n_pairs >= total_tiles) grid_launch_dependents();       // the last epilogue of this CTA
            if (abort_flag) full_row = -1;
            const long long out_row = (full_row >= 0 && p.compact) ? grow : full_row;
            uint4 rr[kPieces];                                          // the residual of the next columns
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                const int colq = n0 + c * kChunk + q * 8;               // the 8 columns this lane moves
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
                            const long long rrow = __shfl_sync(0xffffffffu, res_row, r0 + kStep * j);
                            rr[j] = (rrow >= 0 && colq + kChunk < p.N_out) ? __ldcg(reinterpret_cast<const uint4 *>(p.residual + rrow * p.N_out + colq + kChunk))
                                                                           : make_uint4(0, 0, 0, 0);
                        }
                    }
                }
#pragma unroll
                for (int v = 0; v < kPieces; ++v) {
                    const int col = n0 + c * kChunk + v * 8;
                    uint4 *mine = reinterpret_cast<uint4 *>(stage + swizzled(lane, v));     // residual in, result out
                    f32x2 f[4], t[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) f[i] = sum[c * (kChunk / 2) + v * 4 + i];
                    if (p.bias) {
                        unpack8(shfl_vec(vec, c * kPieces + v), t);
#pragma unroll
                        for (int i = 0; i < 4; ++i) f[i] = add2(f[i], t[i]);
                    }
                    if (EPI == kGelu || (EPI == kAnything && p.gelu)) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) f[i] = gelu2(f[i]);
                    }
                    if (EPI == kAnything && p.gate) {
                        uint4 gv = shfl_vec(vec, 8 + c * kPieces + v);
                        if (!one_batch && col < p.N_out) gv = ld_cached(reinterpret_cast<const uint4 *>(p.gate + (long long)batch * p.N_out + col));
                        unpack8(gv, t);
#pragma unroll
                        for (int i = 0; i < 4; ++i) f[i] = mul2(f[i], t[i]);
                    }
                    if (EPI == kAnything && p.residual) {
                        unpack8(*mine, t);
#pragma unroll
                        for (int i = 0; i < 4; ++i) f[i] = add2(f[i], t[i]);
                    }
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float lo, hi;
                        unpack2(f[i], lo, hi);
                        __nv_bfloat162 v2 = __floats2bfloat162_rn(lo, hi);
                        w[i] = *reinterpret_cast<uint32_t *>(&v2);
                    }
                    *mine = make_uint4(w[0], w[1], w[2], w[3]);
                }
                __syncwarp();
#pragma unroll
                for (int j = 0; j < kPieces; ++j) {
                    const int r = r0 + kStep * j;
                    const long long orow = __shfl_sync(0xffffffffu, out_row, r);
                    const uint4 t = *reinterpret_cast<const uint4 *>(stage + swizzled(r, q));
                    if (orow >= 0 && colq < p.N_out) *reinterpret_cast<uint4 *>(p.y + orow * p.N_out + colq) = t;
                }
                __syncwarp();
            }
        }
    } else if (warp == kTmaWarp) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
        // ------------------------------------------------ TMA producer (the bytes of both CTAs are counted on the even one's barrier)
        const uint32_t full0 = map_to_rank(bar_full, 0);
        auto gave_up = [&] { return *static_cast<volatile int *>(&abort_flag) != 0; };
        auto going = [&](int g) -> bool {                              // once the CTA has given up, stage g and those after it are not sent for
            if (gave_up()) stop = min(stop, g);
            return stop > g;
        };
        int g = 0;
        for (int tile = pair; tile < total_tiles; tile += n_pairs) {
            const int tm = tile / tiles_n, tn = tile - tm * tiles_n;
            for (int ks = 0; ks < k_steps; ++ks, ++g) {
                const int st = g % kStages;
                wait_bar(bar_empty + 8 * st, ((g / kStages) & 1) ^ 1, &abort_flag, p.err_word);
                if (elect_one() && going(g)) {
                    if (rank == 0) mbar_arrive_expect_tx(bar_full + 8 * st, 2 * (BN / 2 * kBK + kABytes));
                    tma_load_2d(sB + st * kBBytes, &tmap_w, full0 + 8 * st, ks * kBK, tn * BN + (int)rank * (BN / 2));
                    tma_load_2d(sA + st * kABytes, &tmap_x, full0 + 8 * st, ks * kBK, tm * kTileRows + (int)rank * kRowsCta);
                }
                __syncwarp();
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
            int g = 0;
            for (int tile = pair; tile < total_tiles; tile += n_pairs) {
                for (int ks = 0; ks < k_steps; ++ks, ++g) {
                    const int st = g % kStages, acc = g % kAcc;
                    wait_bar<true>(bar_acc_empty + 8 * acc, ((g / kAcc) & 1) ^ 1, &abort_flag, p.err_word);
                    wait_bar(bar_full + 8 * st, (g / kStages) & 1, &abort_flag, p.err_word);
                    fence_acquire_smem();                              // what landed in the odd CTA is in order before the MMAs too
                    tc_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (int kk = 0; kk < kBK / 32; ++kk)
                            mma_ss_pair_f8(tmem + acc * BN, smem_desc(sA + st * kABytes + kk * 32, 16, 1024, kSwizzle128B),
                                           smem_desc(sB + st * kBBytes + kk * 32, 16, 1024, kSwizzle128B), idesc, kk > 0 ? 1u : 0u);
                        tc_commit_pair(bar_acc_full + 8 * acc);
                        tc_commit_pair(bar_empty + 8 * st);
                    }
                    __syncwarp();
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

template <int BN, int EPI>
int32_t launch_tiles(const Fp8Params &p, const void *xq, const void *wq, int pairs, cudaStream_t stream)
{
    CUtensorMap mw, mx;
    int32_t rc = make_byte_map(&mw, wq, p.N_out, p.K, BN / 2, "wq");
    if (rc == ASTRAEA_OK) rc = make_byte_map(&mx, xq, (long long)p.B * p.M, p.K, kRowsCta, "xq");
    if (rc != ASTRAEA_OK) return rc;
    static PerDeviceOnce attrs;                   // the attribute is per device
    if (attrs.run([] { return cudaFuncSetAttribute(linear_fp8_kernel<BN, EPI>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes); }) != cudaSuccess)
        return check_launch("astraea_gathered_linear_fp8 (shared memory attribute)");
    const long long tiles = (((long long)p.B * p.M + kTileRows - 1) / kTileRows) * ((p.N_out + BN - 1) / BN);
    launch_overlapped(linear_fp8_kernel<BN, EPI>, 2 * (int)(tiles < pairs ? tiles : pairs), kThreads, kSmemBytes, stream, mw, mx, p);
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
    p.err_word = err_word;
    const int pairs = sm_count() / 2 > 0 ? sm_count() / 2 : 1;
    const long long tiles_m = ((long long)B * p.M + kTileRows - 1) / kTileRows;
    // a round of narrower tiles costs less, but not in proportion
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
