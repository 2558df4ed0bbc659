// Attention over a window of keys (astraea_window_attn): which key tiles a CTA of the attention kernel walks over and which keys of a tile a
// row sees.  (Included by attn.cu behind its Params.)
//
// A query at position p sees key j if j < len and (j < n_first, or j >= N - n_last, or p - left <= j <= p + right).  The keys that any of a
// CTA's rows sees are at most three ranges: the first keys, the windows of its first to its last row, the last keys; ranges that touch or
// overlap are one.  Each is cut into tiles from its own first key (TMA takes any first row), so that a range of n keys is ceil(n / 64)
// tiles whatever its place, and the tiles are numbered through.
#pragma once

#include <limits.h>

constexpr int kKeyTile = 64;
// A row's sum of exponentials against the speculative reference below which it is redone against its exact maximum
constexpr float kLeastSum = 8.271806125530277e-25f;              // 2^-80

struct KeyList {
    int a1, b0, b1, c0, c1;              // ranges [0, a1), [b0, b1), [c0, c1), empty ones with no tile
    int b_tile, c_tile, n;               // number of the first tile of the second and third, tiles in all
    int all_lo, all_hi;                  // keys in reach of every row of the CTA
    int w_base, w_tile, w_end;           // the range that holds the windows: its first key, its first tile, its end (none: 0, 0, 0)
    int l_base, l_tile, l_end;           // and the one that holds the last keys
    __device__ __forceinline__ int key(int j) const { return j < b_tile ? kKeyTile * j : j < c_tile ? b0 + kKeyTile * (j - b_tile) : c0 + kKeyTile * (j - c_tile); }
    __device__ __forceinline__ int end(int j) const { return j < b_tile ? a1 : j < c_tile ? b1 : c1; }
};

// What a row of the CTA that does not exist (behind the last one, a bad entry of the list) reaches: neutral where a warp takes the largest lo and
// the smallest hi of its rows.  It sees no key, and a warp of such rows takes no tile for whole.
constexpr int kNoRowLo = INT_MIN, kNoRowHi = INT_MAX;

struct GroupRow { int m, rest; };        // row m * group + rest of a key head's (query, head) pairs
struct WindowParams : Params {
    int group;                           // query heads of a key head: `heads` of the launch are key heads, a unit's rows are (query, head) pairs
    uint64_t group_inv;                  // 2^32 / group, rounded up
    // x / group for x below 256 + group, exact while that times the group is below 2^32 (the group is at most 4096)
    __host__ __device__ __forceinline__ int div_group(int x) const { return (int)((uint32_t)x * group_inv >> 32); }
    __device__ __forceinline__ GroupRow group_row(int row) const { const int m = row / group; return {m, row - m * group}; }
    int left, right, n_first, last0;     // last0 = N - n_last
    const int32_t *kv_len;               // keys of a batch element that exist (NULL: all N)
    int q_compact;                       // q holds the listed rows only
    const __nv_bfloat16 *v;              // for values that are not finite (see spread_odd_values)
    int64_t v_sb, v_sh, v_sn;
    __device__ __forceinline__ int token(int b, int m) const { return q_idx ? __ldcg(q_idx + (size_t)b * M + m) : m; }
};

// The key tiles of a CTA whose rows stand at positions first .. last (last < first: it has none), by all lanes of a warp alike.
__device__ __forceinline__ KeyList list_keys(const WindowParams &p, int b, int first, int last)
{
    KeyList k;
    const int len = p.kv_len ? min(max(__ldcg(p.kv_len + b), 0), p.N) : p.N;
    const bool rows = first <= last;
    k.a1 = rows ? min(p.n_first, len) : 0;
    k.b0 = rows ? min(max(first - p.left, k.a1), len) : 0;
    k.b1 = rows ? max(k.b0, min(last + p.right + 1, len)) : 0;
    if (p.last0 <= k.b0) k.b1 = k.b0;                             // the last keys hold the window
    if (k.b0 == k.a1) { k.a1 = k.b1; k.b0 = k.b1; }              // the window begins where the first keys end
    const int top = k.b0 < k.b1 ? k.b1 : k.a1;
    k.c0 = rows ? min(max(p.last0, top), len) : 0;
    k.c1 = rows ? len : 0;
    if (k.c0 == top) {                                             // the last keys begin where the window ends
        if (k.b0 < k.b1) k.b1 = k.c1; else k.a1 = k.c1;
        k.c0 = k.c1;
    }
    k.b_tile = (k.a1 + kKeyTile - 1) / kKeyTile;
    k.c_tile = k.b_tile + (k.b1 - k.b0 + kKeyTile - 1) / kKeyTile;
    k.n = k.c_tile + (k.c1 - k.c0 + kKeyTile - 1) / kKeyTile;
    const bool b_there = k.b0 < k.b1, c_there = k.c0 < k.c1;
    k.w_base = b_there ? k.b0 : 0; k.w_tile = b_there ? k.b_tile : 0; k.w_end = b_there ? k.b1 : k.a1;
    k.l_base = c_there ? k.c0 : k.w_base; k.l_tile = c_there ? k.c_tile : k.w_tile; k.l_end = c_there ? k.c1 : k.w_end;
    k.all_lo = last - p.left; k.all_hi = rows ? first + p.right : -1;
    return k;
}

// The tiles of which rows that all reach keys lo .. hi see every key: up to three runs of tile numbers (a tile that is seen whole only
// because two reasons meet in it is not among them).  None where there is no row (lo = kNoRowLo).
struct WholeTiles {
    int first, w0, w_n, l0, l_n;         // tiles below `first`, w_n from w0 on, l_n from l0 on
    __device__ __forceinline__ bool has(int j) const { return j < first || (unsigned)(j - w0) < (unsigned)w_n || (unsigned)(j - l0) < (unsigned)l_n; }
};
__device__ __forceinline__ WholeTiles whole_tiles(const KeyList &k, int lo, int hi, int n_first, int last0)
{
    WholeTiles t = {};
    if (lo == kNoRowLo) return t;
    t.first = min(n_first, k.a1) / kKeyTile;
    auto run = [](int from, int to, int base, int tile, int &t0, int &n) {      // keys from .. to - 1 of a range
        const int a = (max(from - base, 0) + kKeyTile - 1) / kKeyTile, b = max(to - base, 0) / kKeyTile;
        t0 = tile + a; n = max(b - a, 0);
    };
    run(lo, hi < k.w_end ? hi + 1 : k.w_end, k.w_base, k.w_tile, t.w0, t.w_n);
    run(last0, k.l_end, k.l_base, k.l_tile, t.l0, t.l_n);
    return t;
}
// bits [a, b) of a word, both clipped to [0, 64]
__device__ __forceinline__ uint64_t bits_between(int a, int b)
{
    a = max(a, 0); b = min(b, 64);
    return b > a ? (~0ull >> (64 - (b - a))) << a : 0ull;
}
// The keys of that tile that a row which reaches lo .. hi sees, a bit each (none for a row that does not exist).
__device__ __forceinline__ uint64_t visible_bits(int k0, int end, int lo, int hi, int n_first, int last0)
{
    if (lo == kNoRowLo) return 0ull;
    return (bits_between(0, n_first - k0) | bits_between(lo - k0, hi + 1 - k0) | bits_between(last0 - k0, 64)) & bits_between(0, end - k0);
}
template <int NS> __device__ __forceinline__ void hide(float (&s)[NS], uint64_t visible, float with)
{
    const uint32_t w[2] = {(uint32_t)visible, (uint32_t)(visible >> 32)};
#pragma unroll
    for (int i = 0; i < NS; ++i) if (!(w[i >> 5] >> (i & 31) & 1u)) s[i] = with;
}

// the two warpgroups of a query tile meet
__device__ __forceinline__ void pair_sync(int tile)
{
    if (tile == 0) asm volatile("bar.sync 1, 256;" ::: "memory");
    else asm volatile("bar.sync 2, 256;" ::: "memory");
}
// whether any thread of the two says yes (they meet here, too)
__device__ __forceinline__ bool pair_any(int tile, bool yes)
{
    uint32_t any;
    if (tile == 0)
        asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, 1, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(any) : "r"((uint32_t)yes) : "memory");
    else
        asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, 2, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(any) : "r"((uint32_t)yes) : "memory");
    return any != 0;
}

// A probability of zero does not keep a value of NaN or infinity out of the product (0 * inf = NaN), and rows of a tile need not see the
// same keys.  So in tiles that some row does not see whole, one warp looks at the values in shared memory before the MMAs do: it clears the
// rows behind the end of the range (real keys, or memory that was never written, behind the length of a batch element) and every element
// that is not finite, and says whether there was one.  bits of eight bf16 (in a 16-byte vector) that are not finite: all ones, else 0.
__device__ __forceinline__ uint4 clear_odd(uint4 v, bool &odd)
{
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t t = ((w[i] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;       // the exponent is all ones
        if (t) { odd = true; w[i] &= ~((t >> 15) * 0xffffu); }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Whether eight bf16 hold one that is not finite shows in the largest magnitude so far, NaN counting as the largest: one instruction a word.
__device__ __forceinline__ void largest(uint32_t &m, const uint4 &v)
{
    asm("max.NaN.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(v.x));
    asm("max.NaN.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(v.y));
    asm("max.NaN.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(v.z));
    asm("max.NaN.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(v.w));
}
// A tile of values in shared memory (a row is 128 bytes in each of the chunks of CHUNK_BYTES and 32 in what is left of LOAD_BYTES behind
// them; the swizzle keeps a row's bytes in its row) by one warp: rows from `rows` on and elements that are not finite become zero.  True if
// there were such elements in the rows before.  Written only where there is something to clear.  Two loads are in flight: the warp has 32
// registers, and a load takes four of them (us with one / two / four / eight: 4613 of 17776 queries, 2048 keys either way, 24 heads of 64 216 / 216 /
// 223 / 220; 1000 of them, 300 keys either way 63 / 63 / 70 / 67, with heads of 128 92 / 92 / 92 / 94).
constexpr int kCleanLoads = 2;
template <int CHUNK_BYTES, int CHUNKS, int LOAD_BYTES>
__device__ __forceinline__ bool clean_values(uint4 *v, int rows, int lane)
{
    constexpr int kVecs = LOAD_BYTES / 16, kMain = CHUNKS * CHUNK_BYTES / 16, kRound = kCleanLoads;
    static_assert(kVecs % (32 * kRound) == 0, "whole rounds");
    auto row_of = [](int i) { return i < kMain ? i / 8 % kKeyTile : (i - kMain) / 2; };
    bool odd = false;
    uint32_t m = 0;
    for (int i0 = lane; i0 < kVecs; i0 += 32 * kRound) {
        uint4 x[kRound];
#pragma unroll
        for (int u = 0; u < kRound; ++u) x[u] = v[i0 + 32 * u];
#pragma unroll
        for (int u = 0; u < kRound; ++u) largest(m, x[u]);
    }
    const bool look = (m & 0x7f80u) == 0x7f80u || (m & 0x7f800000u) == 0x7f800000u;
    if (__any_sync(0xffffffffu, look) || rows < kKeyTile) {
        for (int i = lane; i < kVecs; i += 32) {
            if (row_of(i) >= rows) v[i] = make_uint4(0, 0, 0, 0);
            else if (look) v[i] = clear_odd(v[i], odd);
        }
    }
    return odd;
}

// What was cleared is put back behind the rows' epilogue, by each row's own thread and for the keys that it sees: an element of +-inf or NaN
// times a probability above zero is that element, whatever is added to it, so it is added to the row that has been written.  Rows of
// values that are not finite are not met in a program that works: this is slow and need not be fast.
template <class T, int DH>
__device__ __noinline__ void spread_odd_values(const WindowParams &p, const KeyList &keys, int tile0, int n_tiles, int b, int kv_head, int tok, T *row)
{
    const WholeTiles whole = whole_tiles(keys, keys.all_lo, keys.all_hi, p.n_first, p.last0);
    for (int j = 0; j < n_tiles; ++j) {
        if (whole.has(tile0 + j)) continue;
        const int k0 = keys.key(tile0 + j), end = keys.end(tile0 + j);
        const uint64_t visible = visible_bits(k0, end, tok - p.left, tok + p.right, p.n_first, p.last0);
        for (int i = 0; i < kKeyTile; ++i) {
            if (!(visible >> i & 1)) continue;
            const __nv_bfloat16 *v = p.v + b * p.v_sb + kv_head * p.v_sh + (int64_t)(k0 + i) * p.v_sn;
            for (int c = 0; c < DH; c += 8) {
                const uint4 x = __ldcg(reinterpret_cast<const uint4 *>(v + c));
                bool odd = false;
                clear_odd(x, odd);
                if (!odd) continue;
                for (int e = 0; e < 8; ++e) {
                    const float f = __bfloat162float(v[c + e]);
                    if (!isfinite(f)) row[c + e] = static_cast<T>(static_cast<float>(row[c + e]) + f);
                }
            }
        }
    }
}
