// Rows of values as 8-bit integers with a scale each (int8_dense.cu, few_rows.cu).
#pragma once

#include "common.cuh"
#include "dense_math.cuh"

namespace tfjsb {
namespace dense {

// q = 127 x / amax rounded to nearest, halves to even.  Whether a value lies above, on or below the middle between two integers is decided
// exactly.
//
// The quotient r is t / amax with t = 127 x, corrected by its own remainder (an fma), which leaves it within an ulp and exact where it can be: a bfloat16
// x makes t exact (15 bits), a middle between two integers is representable, and no other quotient comes nearer to one than 2^-8 / 255 of
// the larger of 1 and its own size, which is more than an ulp.  So for bfloat16 rounding r is right.  For fp32 values t is rounded;
// there a quotient within 2^-9 of a middle is decided again: 127 |x| is t + t_low (a product and its fma rest), t - q amax
// is exact for the integer q next to it (one fma, the terms nearly cancel), and the sign of what remains of 127 |x| - (q +- 1/2) amax settles it.
//
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
// |x| in [0, 1] times amax: the integer next to 127 |x| / amax
static __device__ __noinline__ int quantize_near_middle(float x, float pre, float amax, float inverse) {
    const float v = fabsf(x * pre);
    const float t = v * 127.f, t_low = fmaf(v, 127.f, -t);
    float q = rintf(t * inverse);
    const float e = fmaf(-q, amax, t), middle = 0.5f * amax;
    const bool odd = ((int)q & 1) != 0;
    const float above = (e - middle) + t_low, below = (e + middle) + t_low;
    if (above > 0.f || (above == 0.f && odd)) q += 1.f;
    else if (below < 0.f || (below == 0.f && odd)) q -= 1.f;
    return x < 0.f ? -(int)q : (int)q;
}
// Eight values as eight bytes.
template <bool F32>
__device__ __forceinline__ uint2 quantize8(const float (&v)[8], const RowScale& s) {
    if (s.none) return make_uint2(0u, 0u);
    const float c = 127.f * s.pre;
    uint32_t q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float t = v[e] * c, r0 = t * s.inverse;
        const float r = fmaf(fmaf(-r0, s.amax, t), s.inverse, r0);
        const float m = r + 12582912.f;  // 1.5 * 2^23: the integer nearest to r in the low bits, halves to even
        q[e] = __float_as_uint(m);
        if (F32) {
            const float d = fabsf(r - (m - 12582912.f));
            if (fabsf(d - 0.5f) < 0.001953125f) q[e] = (uint32_t)quantize_near_middle(v[e], s.pre, s.amax, s.inverse);
        }
    }
    uint2 w;
    w.x = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
    w.y = __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410);
    return w;
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

}  // namespace dense
}  // namespace tfjsb
