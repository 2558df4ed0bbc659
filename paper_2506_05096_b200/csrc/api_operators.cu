// extern "C" entry points of the operators that stand beside the path: attention over a window of keys, head norms with the rotation by
// position, linear layers in 8 bits.  Argument validation on the host, then the kernel launchers, as in api.cu.
#include <math.h>

#include "common.cuh"

using namespace astraea;

#define REQUIRE(cond, ...) do { if (!(cond)) return fail(ASTRAEA_ERR_INVALID_ARG, __VA_ARGS__); } while (0)

extern "C" {

int32_t astraea_window_attn(const void *q, const void *k, const void *v,
                            int64_t q_sb, int64_t q_sh, int64_t q_sn,
                            int64_t k_sb, int64_t k_sh, int64_t k_sn,
                            int64_t v_sb, int64_t v_sh, int64_t v_sn,
                            const int32_t *q_idx, int M, const int32_t *kv_len, void *out, float *lse_out,
                            int B, int H, int H_kv, int N, int d, int n_first, int n_last, int left, int right,
                            float scale, uint32_t flags, void *workspace, size_t workspace_bytes, void *stream)
{
    const char *fn = "astraea_window_attn";
    REQUIRE(B > 0 && H > 0 && H_kv > 0 && N > 0, "%s: B, H, H_kv, N must be positive", fn);
    REQUIRE(N <= 1 << 30, "%s: N=%d is above 2^30", fn, N);
    REQUIRE(H % H_kv == 0 && H / H_kv <= 4096, "%s: H=%d must be a multiple of H_kv=%d, up to 4096 times it", fn, H, H_kv);
    REQUIRE(M >= 0 && M <= N, "%s: M=%d outside [0, N=%d]", fn, M, N);
    REQUIRE((long long)M * (H / H_kv) <= 1 << 30, "%s: too many rows", fn);
    if (d != 64 && d != 72 && d != 128) return fail(ASTRAEA_ERR_UNSUPPORTED, "%s: head_dim %d not in {64, 72, 128}", fn, d);
    if (flags & ~(ASTRAEA_ATTN_COMPACT_OUT | ASTRAEA_ATTN_COMPACT_Q | ASTRAEA_ATTN_SMALL_CTAS | ASTRAEA_ATTN_WHOLE_KEYS)) return fail(ASTRAEA_ERR_UNSUPPORTED, "%s: unknown flags 0x%x", fn, flags);
    REQUIRE(n_first >= 0 && n_last >= 0 && left >= 0 && right >= 0, "%s: n_first, n_last, left, right must not be negative", fn);
    REQUIRE(q && k && v && out, "%s: null q, k, v or out", fn);
    REQUIRE(aligned16(q) && aligned16(k) && aligned16(v) && aligned16(out), "%s: q, k, v, out must be 16-byte aligned", fn);
    REQUIRE(q_sn % 8 == 0 && k_sn % 8 == 0 && v_sn % 8 == 0 && q_sh % 8 == 0 && k_sh % 8 == 0 && v_sh % 8 == 0 &&
            q_sb % 8 == 0 && k_sb % 8 == 0 && v_sb % 8 == 0,
            "%s: strides must be multiples of 8 elements (16 bytes)", fn);
    REQUIRE(q_sn >= d && k_sn >= d && v_sn >= d && q_sh > 0 && k_sh > 0 && v_sh > 0 && q_sb >= 0 && k_sb >= 0 && v_sb >= 0,
            "%s: strides must be positive and token stride >= head_dim", fn);
    REQUIRE(scale >= 0.f, "%s: scale must be >= 0 (0 selects 1/sqrt(d))", fn);
    if (!workspace || workspace_bytes < 256)
        return fail(ASTRAEA_ERR_WORKSPACE_TOO_SMALL, "%s: workspace of %zu bytes, need %d", fn, workspace_bytes, 256);
    REQUIRE((reinterpret_cast<uintptr_t>(workspace) & 255u) == 0, "%s: workspace must be 256-byte aligned", fn);
    if (M == 0) return ASTRAEA_OK;
    WindowArgs w;
    AttnArgs &a = w.a;
    a.q = q; a.k = k; a.v = v;
    a.q_sb = q_sb; a.q_sh = q_sh; a.q_sn = q_sn;
    a.k_sb = k_sb; a.k_sh = k_sh; a.k_sn = k_sn;
    a.v_sb = v_sb; a.v_sh = v_sh; a.v_sn = v_sn;
    a.q_idx = q_idx; a.M = M; a.out = out; a.lse_out = lse_out;
    a.B = B; a.H = H; a.N = N; a.N_tok = N; a.d = d;
    a.scale = (scale == 0.f) ? 1.0f / sqrtf((float)d) : scale;
    a.flags = flags;
    a.err_word = reinterpret_cast<int *>(workspace);
    if (workspace_bytes > 256) { a.split_ws = static_cast<char *>(workspace) + 256; a.split_ws_bytes = workspace_bytes - 256; }
    w.group = H / H_kv;
    w.left = left < N ? left : N - 1; w.right = right < N ? right : N - 1;      // (position + right + 1 stays below 2^31)
    w.n_first = n_first < N ? n_first : N; w.n_last = n_last < N ? n_last : N;
    w.kv_len = kv_len;
    return launch_window_attn(w, (cudaStream_t)stream);
}

int32_t astraea_qk_norm_rotate(const astraea_head_rows *rows, int n, const float *cos, const float *sin, int n_rot,
                               int B, int N, int d, int norm, int rotation, float eps, void *err_workspace, void *stream)
{
    const char *fn = "astraea_qk_norm_rotate";
    REQUIRE(rows && (n == 1 || n == 2), "%s: one or two tensors, got %d", fn, rows ? n : 0);
    REQUIRE(B > 0 && N > 0, "%s: B and N must be positive", fn);
    REQUIRE((long long)B * N <= 1 << 30, "%s: too many rows", fn);
    if (d != 64 && d != 72 && d != 128) return fail(ASTRAEA_ERR_UNSUPPORTED, "%s: head_dim %d not in {64, 72, 128}", fn, d);
    if (norm != ASTRAEA_NORM_RMS && norm != ASTRAEA_NORM_LAYER) return fail(ASTRAEA_ERR_UNSUPPORTED, "%s: unknown norm %d", fn, norm);
    if (rotation != ASTRAEA_ROTATE_INTERLEAVED && rotation != ASTRAEA_ROTATE_HALF) return fail(ASTRAEA_ERR_UNSUPPORTED, "%s: unknown rotation %d", fn, rotation);
    REQUIRE(n_rot >= 0 && n_rot <= N, "%s: n_rot=%d outside [0, N=%d]", fn, n_rot, N);
    REQUIRE(n_rot == 0 || (cos && sin && aligned16(cos) && aligned16(sin)), "%s: cos and sin must be 16-byte aligned and not null", fn);
    REQUIRE(eps >= 0.f, "%s: eps must be >= 0", fn);
    REQUIRE((reinterpret_cast<uintptr_t>(err_workspace) & 3u) == 0, "%s: err_workspace must be 4-byte aligned", fn);
    for (int i = 0; i < n; ++i) {
        const astraea_head_rows &t = rows[i];
        if (t.flags & ~(ASTRAEA_ROWS_COMPACT_IN | ASTRAEA_ROWS_COMPACT_OUT)) return fail(ASTRAEA_ERR_UNSUPPORTED, "%s: unknown flags 0x%x", fn, t.flags);
        REQUIRE(t.H > 0, "%s: H must be positive", fn);
        REQUIRE(!t.idx || (t.M >= 0 && t.M <= N), "%s: M=%d outside [0, N=%d]", fn, t.M, N);
        REQUIRE(!t.flags || t.idx, "%s: compact rows need an index list", fn);
        if (t.idx && t.M == 0) continue;
        REQUIRE(t.x && t.y, "%s: null x or y", fn);
        REQUIRE(aligned16(t.x) && aligned16(t.y) && aligned16(t.weight) && aligned16(t.bias), "%s: x, y, weight, bias must be 16-byte aligned", fn);
        REQUIRE(t.x_sb % 8 == 0 && t.x_sh % 8 == 0 && t.x_sn % 8 == 0 && t.y_sb % 8 == 0 && t.y_sh % 8 == 0 && t.y_sn % 8 == 0,
                "%s: strides must be multiples of 8 elements (16 bytes)", fn);
        REQUIRE(t.x_sb >= 0 && t.x_sh > 0 && t.x_sn >= 0 && t.y_sb >= 0 && t.y_sh >= d && t.y_sn >= d, "%s: strides must be positive and those of y at least head_dim", fn);
        REQUIRE(B == 1 || t.y_sb >= d, "%s: the batch stride of y must be at least head_dim", fn);
        REQUIRE(t.x != t.y || (t.x_sb == t.y_sb && t.x_sh == t.y_sh && t.x_sn == t.y_sn &&
                               ((t.flags & ASTRAEA_ROWS_COMPACT_IN) != 0) == ((t.flags & ASTRAEA_ROWS_COMPACT_OUT) != 0)),
                "%s: in place, x and y must have the same strides and rows", fn);
        REQUIRE(!t.bias || norm == ASTRAEA_NORM_LAYER, "%s: a bias goes with the layer norm", fn);
    }
    return launch_qk_norm_rotate(rows, n, cos, sin, n_rot, B, N, d, norm == ASTRAEA_NORM_LAYER, rotation == ASTRAEA_ROTATE_HALF, eps,
                                 reinterpret_cast<int *>(err_workspace), (cudaStream_t)stream);
}

int32_t astraea_quantize_fp8(const void *x, const int32_t *idx, int M, void *xq, float *x_scale, int B, int N, int K,
                             uint32_t flags, void *err_workspace, void *stream)
{
    const char *fn = "astraea_quantize_fp8";
    REQUIRE(B > 0 && N > 0 && K > 0, "%s: B, N, K must be positive", fn);
    REQUIRE(K % 128 == 0, "%s: K=%d must be a multiple of 128", fn, K);
    REQUIRE(!idx || (M >= 0 && M <= N), "%s: M=%d outside [0, N=%d]", fn, M, N);
    if (flags & ~ASTRAEA_LINEAR_COMPACT_IN) return fail(ASTRAEA_ERR_UNSUPPORTED, "%s: unknown flags 0x%x", fn, flags);
    REQUIRE(!flags || idx, "%s: compact rows need an index list", fn);
    if (idx && M == 0) return ASTRAEA_OK;
    REQUIRE(x && xq && x_scale, "%s: null x, xq or x_scale", fn);
    REQUIRE(aligned16(x) && aligned16(xq), "%s: x and xq must be 16-byte aligned", fn);
    REQUIRE((reinterpret_cast<uintptr_t>(x_scale) & 3u) == 0 && (reinterpret_cast<uintptr_t>(err_workspace) & 3u) == 0,
            "%s: x_scale and err_workspace must be 4-byte aligned", fn);
    return launch_quantize_fp8(x, idx, M, xq, x_scale, B, N, K, (flags & ASTRAEA_LINEAR_COMPACT_IN) != 0, reinterpret_cast<int *>(err_workspace),
                               (cudaStream_t)stream);
}

int32_t astraea_quantize_fp8_weight(const void *w, void *wq, float *w_scale, int N_out, int K, void *stream)
{
    const char *fn = "astraea_quantize_fp8_weight";
    REQUIRE(N_out > 0 && K > 0 && K % 128 == 0, "%s: N_out must be positive, K=%d a positive multiple of 128", fn, K);
    REQUIRE(N_out <= 65535 * 128, "%s: N_out=%d is too large", fn, N_out);
    REQUIRE(w && wq && w_scale, "%s: null w, wq or w_scale", fn);
    REQUIRE(aligned16(w) && aligned16(wq) && (reinterpret_cast<uintptr_t>(w_scale) & 3u) == 0, "%s: w and wq must be 16-byte aligned, w_scale 4-byte", fn);
    return launch_quantize_fp8_weight(w, wq, w_scale, N_out, K, (cudaStream_t)stream);
}

int32_t astraea_gathered_linear_fp8(const void *xq, const float *x_scale, const int32_t *idx, int M,
                                    const void *wq, const float *w_scale, const void *bias, const void *residual, const void *gate,
                                    void *y, int B, int N, int K, int N_out, uint32_t flags,
                                    void *workspace, size_t workspace_bytes, void *stream)
{
    const char *fn = "astraea_gathered_linear_fp8";
    REQUIRE(B > 0 && N > 0 && K > 0 && N_out > 0, "%s: B, N, K, N_out must be positive", fn);
    REQUIRE(!idx || (M >= 0 && M <= N), "%s: M=%d outside [0, N=%d]", fn, M, N);
    REQUIRE(K % 128 == 0, "%s: K=%d must be a multiple of 128", fn, K);
    REQUIRE(N_out % 8 == 0 && N_out <= 65535 * 128, "%s: N_out=%d must be a multiple of 8 and is limited to 65535 * 128", fn, N_out);
    if (flags & ~(ASTRAEA_LINEAR_COMPACT_OUT | ASTRAEA_LINEAR_GELU | ASTRAEA_LINEAR_COMPACT_RES)) return fail(ASTRAEA_ERR_UNSUPPORTED, "%s: unknown flags 0x%x", fn, flags);
    REQUIRE(!(flags & (ASTRAEA_LINEAR_COMPACT_OUT | ASTRAEA_LINEAR_COMPACT_RES)) || idx, "%s: compact rows need an index list", fn);
    REQUIRE(!(flags & ASTRAEA_LINEAR_COMPACT_RES) || residual, "%s: ASTRAEA_LINEAR_COMPACT_RES without a residual", fn);
    if (!workspace || workspace_bytes < linear_workspace_bytes())
        return fail(ASTRAEA_ERR_WORKSPACE_TOO_SMALL, "%s: workspace of %zu bytes, need %zu", fn, workspace_bytes, linear_workspace_bytes());
    REQUIRE((reinterpret_cast<uintptr_t>(workspace) & 255u) == 0, "%s: workspace must be 256-byte aligned", fn);
    const long long rows = (long long)B * (idx ? M : N);
    if (rows == 0) return ASTRAEA_OK;
    REQUIRE((long long)B * N <= 0x7fffffffll - 256, "%s: too many rows", fn);
    REQUIRE((rows + 255) / 256 * ((N_out + 63) / 64) <= 0x7fffffffll, "%s: too many tiles", fn);
    REQUIRE(xq && x_scale && wq && w_scale && y, "%s: null xq, x_scale, wq, w_scale or y", fn);
    REQUIRE(aligned16(xq) && aligned16(wq) && aligned16(y) && aligned16(bias) && aligned16(residual) && aligned16(gate),
            "%s: xq, wq, bias, residual, gate, y must be 16-byte aligned", fn);
    REQUIRE((reinterpret_cast<uintptr_t>(x_scale) & 3u) == 0 && (reinterpret_cast<uintptr_t>(w_scale) & 3u) == 0, "%s: scales must be 4-byte aligned", fn);
    return launch_gathered_linear_fp8(xq, x_scale, idx, M, wq, w_scale, bias, residual, gate, y, B, N, K, N_out, flags,
                                      reinterpret_cast<int *>(workspace), (cudaStream_t)stream);
}

}  // extern "C"
