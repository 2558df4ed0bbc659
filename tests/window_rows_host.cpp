// Rows that do not exist among a CTA's rows (window_keys.cuh) on the host: behind the last row of a list, or entries that are skipped.  They
// see no key, hold no other row back, and a warp of nothing but such rows takes no tile for whole, wherever its CTA's key ranges begin.
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>
#include <climits>
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
    std::mt19937 rng(7);
    auto upto = [&](int n) { return (int)(rng() % (unsigned)(n + 1)); };
    int n_case = 0, begins[3] = {0, 0, 0};                        // CTAs whose window begins at key 0, at 1 .. 63, behind that
    for (; n_case < 20000; ++n_case) {
        WindowParams p = {};
        p.N = p.N_tok = 200 + upto(900);
        p.left = upto(400); p.right = upto(1) ? 0 : upto(100);
        p.n_first = upto(1) ? 0 : upto(150);
        p.last0 = p.N - (upto(1) ? 0 : upto(100));
        const int32_t len = upto(p.N);
        p.kv_len = &len;
        const int row = upto(p.N - 1);
        const KeyList k = list_keys(p, 0, row, row);
        ++begins[k.w_base == 0 ? 0 : k.w_base < 64 ? 1 : 2];
        // a warp of rows that do not exist: the largest of their lo, the smallest of their hi
        const WholeTiles none = whole_tiles(k, kNoRowLo, kNoRowHi, p.n_first, p.last0);
        // one that holds the row beside them
        const WholeTiles mixed = whole_tiles(k, max(kNoRowLo, row - p.left), min(kNoRowHi, row + p.right), p.n_first, p.last0);
        const WholeTiles own = whole_tiles(k, row - p.left, row + p.right, p.n_first, p.last0);
        for (int j = 0; j < k.n; ++j) {
            CHECK(!none.has(j));
            CHECK(visible_bits(k.key(j), k.end(j), kNoRowLo, kNoRowHi, p.n_first, p.last0) == 0);
            CHECK(mixed.has(j) == own.has(j));
            if (own.has(j)) CHECK(k.end(j) - k.key(j) >= kKeyTile);
        }
    }
    CHECK(begins[0] > 500 && begins[1] > 500 && begins[2] > 500);
    CHECK(kNoRowLo == INT_MIN && kNoRowHi == INT_MAX);
    printf("window rows ok\n");
    return 0;
}
