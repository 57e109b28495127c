// Rows of values as 8-bit integers with a scale each (int8_dense.cu, few_rows.cu).
#pragma once

#include "common.cuh"
#include "dense_math.cuh"

namespace tfjsb {
namespace dense {

// q = 127 x / amax rounded to nearest, halves to even.  Whether a value lies above, on or below the middle between two integers is decided
// exactly: 127 |x| is t + t_low (a product and its fma rest), q0 the integer nearest to t / amax as computed, and the sign of
// 127 |x| - (q0 +- 1/2) amax, of which t - q0 amax is exact (one fma; the terms nearly cancel), settles whether q0 is it.
// Rows of very small or large values are scaled by a power of two first, so that nothing here overflows or loses bits.
struct RowScale {
    float pre, amax, inverse;  // of pre * x
    bool none;                 // q = 0: amax is 0, infinite or NaN
};
__device__ __forceinline__ RowScale row_scale(float amax) {
    RowScale r;
    r.none = !(amax > 0.f) || !isfinite(amax);
    r.pre = amax < 7.8886091e-31f ? 1.2676506e30f : amax > 1.2676506e30f ? 7.8886091e-31f : 1.f;  // 2^-100, 2^100
    r.amax = amax * r.pre;
    r.inverse = 1.f / r.amax;
    return r;
}
__device__ __forceinline__ int quantize(float x, const RowScale& r) {
    if (r.none) return 0;
    const float v = fabsf(x * r.pre);
    const float t = v * 127.f, t_low = fmaf(v, 127.f, -t);
    float q = rintf(t * r.inverse);
    const float e = fmaf(-q, r.amax, t), middle = 0.5f * r.amax;
    const bool odd = ((int)q & 1) != 0;
    const float above = (e - middle) + t_low, below = (e + middle) + t_low;
    if (above > 0.f || (above == 0.f && odd)) q += 1.f;
    else if (below < 0.f || (below == 0.f && odd)) q -= 1.f;
    return x < 0.f ? -(int)q : (int)q;
}
// The larger of two magnitudes; a NaN wins over all.
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// Eight values from element i on, of which `left` exist.
template <bool F32>
__device__ __forceinline__ void values8(const void* x, int64_t i, int left, float (&v)[8]) {
    if (F32) {
        load_f32(static_cast<const float*>(x) + i, v, left);
        return;
    }
    const unsigned short* p = static_cast<const unsigned short*>(x) + i;
    if (left >= 8 && aligned(p, 16)) {
        uint32_t w[4];
        asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = __uint_as_float(w[e] << 16);
            v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < left ? __uint_as_float((uint32_t)load_global(p + e) << 16) : 0.f;
    }
}
__device__ __forceinline__ uint2 quantize8(const float (&v)[8], const RowScale& r) {
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e / 4] |= (uint32_t)(quantize(v[e], r) & 0xff) << (e % 4 * 8);
    return make_uint2(w[0], w[1]);
}

}  // namespace dense
}  // namespace tfjsb
