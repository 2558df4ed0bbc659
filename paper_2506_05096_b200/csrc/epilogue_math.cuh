// What the epilogues of the two GEMMs (linear.cu, linear_fp8.cu) share.
#pragma once

#include "common.cuh"

namespace astraea {

__device__ __forceinline__ void cp_async_16(uint32_t dst, const void *src, bool valid) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}

// GELU(x) = x (1 + erf(x / sqrt 2)) / 2 of two elements, with erf to 1.5e-7 absolute (rational approximation 7.1.26 of Abramowitz
// and Stegun: erf(z) = 1 - (a1 t + ... + a5 t^5) e^{-z^2} for z >= 0, t = 1 / (1 + p z)): with w = 1/2 + copysign(1/2 - (a1 t +
// ... + a5 t^5) e^{-z^2} / 2, z) it is x w.  Issue slots bind it (the epilogue of a tile has four warps on each SM sub-partition,
// and a main loop of K = 1152 is over in 5 us), so all but the XU operations and the signs are packed pairs: 10 instructions per
// element instead of 17.  z is rounded before it is squared and the halves only scale by powers of two, so the result is that of the
// same formula element by element, bit for bit (with 1 / sqrt 2 folded into the constants 9001 x 3072 x 12288 takes 488 us instead
// of 491, but outputs of a block move by single bf16 roundings; with |z| masked out of a packed product 493).  13106 x 1152 x 4608 took
// 110.0 us with the erf element by element and the epilogue's loads behind its wait, 101.6 now; 1846 x 1536 x 6144 32.2 -> 30.7.
__device__ __forceinline__ f32x2 both(float v) { return pack2(v, v); }
__device__ __forceinline__ f32x2 gelu2(f32x2 x) {
    float x0, x1, d0, d1, a0, a1, t0, t1, e0, e1;
    unpack2(x, x0, x1);
    const f32x2 az = pack2(__fmul_rn(fabsf(x0), 0.70710678118654752f), __fmul_rn(fabsf(x1), 0.70710678118654752f));     // |z|
    unpack2(fma2(az, both(0.3275911f), both(1.0f)), d0, d1);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t0) : "f"(d0));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t1) : "f"(d1));
    unpack2(mul2(mul2(az, az), both(-1.4426950408889634f)), a0, a1);
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(a0));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(a1));
    const f32x2 t = pack2(t0, t1);
    f32x2 pl = fma2(both(-0.5f * 1.061405429f), t, both(0.5f * 1.453152027f));           // minus half the polynomial
    pl = fma2(pl, t, both(-0.5f * 1.421413741f));
    pl = fma2(pl, t, both(0.5f * 0.284496736f));
    pl = fma2(pl, t, both(-0.5f * 0.254829592f));
    const f32x2 half_erf = fma2(mul2(pl, t), pack2(e0, e1), both(0.5f));                // of |z|
    return mul2(x, add2(both(0.5f), (half_erf & 0x7fffffff7fffffffull) | (x & 0x8000000080000000ull)));
}

__device__ __forceinline__ uint4 shfl_vec(const uint4 &v, int lane) {
    return make_uint4(__shfl_sync(0xffffffffu, v.x, lane), __shfl_sync(0xffffffffu, v.y, lane), __shfl_sync(0xffffffffu, v.z, lane),
                      __shfl_sync(0xffffffffu, v.w, lane));
}

}  // namespace astraea
