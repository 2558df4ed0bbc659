// The key tiles of a window (window_keys.cuh) on the host: for random sizes, every row's visible keys come out of the CTA's tiles exactly
// once, tiles that are taken unmasked hold nothing that a row does not see, and what is not finite is found in every position.
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <random>
#include <vector>

using std::max;
using std::min;
#define __device__
#define __host__
#define __forceinline__ inline
#define __noinline__
struct uint4 { uint32_t x, y, z, w; };
static uint4 make_uint4(uint32_t x, uint32_t y, uint32_t z, uint32_t w) { return {x, y, z, w}; }
struct __nv_bfloat16 { uint16_t b; };
static float __bfloat162float(__nv_bfloat16 v) { uint32_t u = (uint32_t)v.b << 16; float f; memcpy(&f, &u, 4); return f; }
template <class T> static T __ldcg(const T *p) { return *p; }
struct Params { const int32_t *q_idx; int M, N, N_tok; };
static bool __any_sync(unsigned, bool b) { return b; }
#define asm(...)
#define volatile
#include "../paper_2506_05096_b200/csrc/window_keys.cuh"
#undef asm
#undef volatile

#define CHECK(c) do { if (!(c)) { printf("failed: %s (line %d, case %d)\n", #c, __LINE__, n_case); return 1; } } while (0)

int main()
{
    std::mt19937 rng(1);
    auto upto = [&](int n) { return (int)(rng() % (unsigned)(n + 1)); };
    int n_case = 0;
    long long runs = 0, missed = 0;                                // tiles seen whole that are in the runs, and that are not
    for (; n_case < 20000; ++n_case) {
        WindowParams p = {};
        p.N = p.N_tok = 1 + upto(n_case % 3 ? 700 : 60);
        p.left = upto(3) ? upto(upto(1) ? 30 : 400) : upto(1) ? 0 : p.N;
        p.right = upto(2) ? upto(200) : upto(1) ? 0 : p.N;
        p.left = min(p.left, p.N - 1); p.right = min(p.right, p.N - 1);
        p.n_first = min(p.N, upto(2) ? upto(150) : 0);
        p.last0 = p.N - min(p.N, upto(2) ? upto(150) : 0);
        int32_t len = upto(3) ? p.N : upto(p.N + 20) - 10;
        p.kv_len = upto(1) ? &len : nullptr;
        const int L = p.kv_len ? min(max(len, 0), p.N) : p.N;
        std::vector<int> rows(1 + upto(40));
        for (int &r : rows) r = upto(p.N - 1);
        const int first = *std::min_element(rows.begin(), rows.end()), last = *std::max_element(rows.begin(), rows.end());
        const KeyList k = list_keys(p, 0, first, last);
        const WholeTiles whole = whole_tiles(k, k.all_lo, k.all_hi, p.n_first, p.last0);
        for (int r : rows) {
            std::vector<int> seen(p.N, 0);
            const WholeTiles own = whole_tiles(k, r - p.left, r + p.right, p.n_first, p.last0);
            for (int j = 0; j < k.n; ++j) {
                const int k0 = k.key(j), end = k.end(j);
                CHECK(k0 >= 0 && k0 < end && end <= L);
                const uint64_t bits = visible_bits(k0, end, r - p.left, r + p.right, p.n_first, p.last0);
                if (whole.has(j)) CHECK(bits == ~0ull);
                if (own.has(j)) { CHECK(bits == ~0ull); ++runs; }
                if (bits == ~0ull && !own.has(j)) ++missed;
                for (int i = 0; i < 64; ++i) if (bits >> i & 1) ++seen[k0 + i];
            }
            for (int j = 0; j < p.N; ++j) {
                const bool want = j < L && (j < p.n_first || j >= p.last0 || (j >= r - p.left && j <= r + p.right));
                CHECK(seen[j] == (want ? 1 : 0));
            }
        }
        // no more tiles than the three ranges need
        const int a = min(p.n_first, L), b0 = min(max(first - p.left, 0), L), b1 = max(b0, min(last + p.right + 1, L)), c0 = min(p.last0, L);
        CHECK(k.n <= (a + 63) / 64 + (b1 - b0 + 63) / 64 + (L - c0 + 63) / 64);
        float s[64];
        const uint64_t v = ((uint64_t)rng() << 32) | rng();
        for (int i = 0; i < 64; ++i) s[i] = (float)i;
        hide<64>(s, v, -1.f);
        for (int i = 0; i < 64; ++i) CHECK(s[i] == ((v >> i & 1) ? (float)i : -1.f));
    }
    CHECK(runs > 100000 && missed * 20 < runs);
    for (int g = 1; g <= 4096; ++g) {                              // a row's query and head
        WindowParams q = {};
        q.group = g; q.group_inv = ((1ull << 32) + g - 1) / g;
        for (int x = 0; x < g + 256; ++x) CHECK(q.div_group(x) == x / g);
        CHECK(q.group_row((1 << 30) - 1).m == ((1 << 30) - 1) / g);
    }
    WindowParams p = {};
    p.N = 100; p.last0 = 90; p.n_first = 5; p.left = p.right = 3;
    CHECK(list_keys(p, 0, 0x7fffffff, -1).n == 0);                // a unit whose rows are all bad entries
    // the largest sizes: no overflow
    p.N = p.N_tok = 1 << 30; p.left = p.right = (1 << 30) - 1; p.last0 = 1 << 30; p.n_first = 0;
    const KeyList k = list_keys(p, 0, 0, (1 << 30) - 1);
    CHECK(k.n == 1 << 24 && k.key(k.n - 1) == (1 << 30) - 64 && k.end(0) == 1 << 30);
    // every bf16 in every place of a vector
    for (int e = 0; e < 8; ++e)
        for (uint32_t code = 0; code < 65536; ++code) {
            uint16_t h[8];
            for (int i = 0; i < 8; ++i) h[i] = (uint16_t)(0x3F80 + i);
            h[e] = (uint16_t)code;
            uint4 v;
            memcpy(&v, h, 16);
            bool odd = false;
            const uint4 r = clear_odd(v, odd);
            uint16_t g[8];
            memcpy(g, &r, 16);
            const bool finite = (code & 0x7f80) != 0x7f80;
            CHECK(odd == !finite);
            for (int i = 0; i < 8; ++i) CHECK(g[i] == (i == e && !finite ? 0 : h[i]));
        }
    // what was cleared reaches the rows that see it, in its channels
    {
        WindowParams q = {};
        q.N = q.N_tok = 200; q.left = 10; q.right = 0; q.n_first = 0; q.last0 = 200;
        std::vector<__nv_bfloat16> v(200 * 64, __nv_bfloat16{0x3F80});
        v[60 * 64 + 7].b = 0x7F80; v[61 * 64 + 8].b = 0xFF80; v[62 * 64 + 9].b = 0x7FC0;
        q.v = v.data(); q.v_sb = 0; q.v_sh = 0; q.v_sn = 64;
        const KeyList kl = list_keys(q, 0, 50, 90);
        for (int tok : {50, 60, 61, 62, 70, 71, 72, 73, 90}) {
            float row[64] = {};
            spread_odd_values<float, 64>(q, kl, 0, kl.n, 0, 0, tok, row);
            CHECK((row[7] == INFINITY) == (tok >= 60 && tok <= 70));
            CHECK((row[8] == -INFINITY) == (tok >= 61 && tok <= 71));
            CHECK(isnan(row[9]) == (tok >= 62 && tok <= 72));
            for (int c = 0; c < 64; ++c) if (c < 7 || c > 9) CHECK(row[c] == 0.f);
        }
    }
    printf("window keys ok\n");
    return 0;
}
