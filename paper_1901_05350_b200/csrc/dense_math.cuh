// The gates of the gated feed-forward block, and rows of values to and from global memory, a group of 32 bytes at a time.
#pragma once

#include <cuda_bf16.h>

#include "common.cuh"

namespace tfjsb {
namespace dense {

// ---- gates -------------------------------------------------------------------------------------------------
//   silu       g s(g)              s(g) = 1 / (1 + e^-g)
//   gelu       g F(g)              F: the normal distribution function, erfc(-g / sqrt 2) / 2
//   gelu_tanh  g s(2 v(g))         v = sqrt(2 / pi) (g + 0.044715 g^3); 1 + tanh(v) = 2 s(2 v)
//   sigmoid    s(g)
//   relu       max(g, 0)           NaN stays NaN; slope 0 at 0
// EXACT: for fp32 results, with functions that are good to an ulp or two; the others go into bfloat16, to which the fast
// exponential's 2^-21 is nothing.  Slopes take 1 - s(v) = s(-v) from the same exponential: subtracted from 1, what is left of a large
// v is s's rounding (at v = 12 1 % of it, at 17 all).
template <bool EXACT>
__device__ __forceinline__ float logistic(float v) {
    if (EXACT) {
        float r;
        asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(1.f + expf(-v)));  // within an ulp; 0 of an infinity
        return r;
    }
    return __fdividef(1.f, 1.f + __expf(-v));  // e^-v = inf: 0
}

// s(v) and s(-v), both to their own last bits
template <bool EXACT>
__device__ __forceinline__ void logistics(float v, float& s, float& other) {
    float e, r;
    if (EXACT) {
        e = expf(-fabsf(v));
        asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    } else {
        e = __expf(-fabsf(v));
        r = __fdividef(1.f, 1.f + e);
    }
    const float small = e * r;
    s = v < 0.f ? small : r;  // a NaN stays one
    other = v < 0.f ? r : small;
}

// a = gate(g) and, with SLOPE, its derivative
template <int GATE, bool EXACT, bool SLOPE>
__device__ __forceinline__ void gate_of(float g, float& a, float& slope) {
    if (GATE == TFJSB_GATE_SILU) {
        float s, other = 0.f;
        if (SLOPE) logistics<EXACT>(g, s, other);
        else s = logistic<EXACT>(g);
        a = g * s;
        if (SLOPE) slope = s * (1.f + g * other);
    } else if (GATE == TFJSB_GATE_SIGMOID) {
        float other = 0.f;
        if (SLOPE) logistics<EXACT>(g, a, other);
        else a = logistic<EXACT>(g);
        if (SLOPE) slope = a * other;
    } else if (GATE == TFJSB_GATE_RELU) {
        a = relu_nan(g);
        if (SLOPE) slope = g > 0.f ? 1.f : 0.f;
    } else if (GATE == TFJSB_GATE_GELU) {
        float f, e;
        if (EXACT) {
            f = 0.5f * erfcf(g * -0.70710678118654752f);
            if (SLOPE) e = expf(-0.5f * g * g);
        } else {
            // Abramowitz and Stegun 7.1.26: erfc(x) = (a1 t + .. + a5 t^5) e^(-x^2), t = 1 / (1 + p x), off by 1.5e-7 at most; here
            // x = |g| / sqrt 2 and the coefficients are halved
            const float t = __fdividef(1.f, fmaf(0.23164189f, fabsf(g), 1.f));
            e = __expf(-0.5f * g * g);
            const float tail = t * e * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 0.5307027145f, -0.7265760135f), 0.7107068705f), -0.142248368f), 0.127414796f);
            f = g < 0.f ? tail : 1.f - tail;  // a NaN stays one
        }
        a = g * f;
        if (SLOPE) slope = fmaf(g * 0.39894228040143268f, e, f);
    } else {
        const float g2 = fminf(g * g, 1e30f);  // finite, so that s(-v) = 0 makes the slope of large g what it is
        const float v = 1.5957691216057308f * g * fmaf(0.044715f, g2, 1.f);
        float s, other = 0.f;
        if (SLOPE) logistics<EXACT>(v, s, other);
        else s = logistic<EXACT>(v);
        a = g * s;
        if (SLOPE) slope = s + a * other * 1.5957691216057308f * fmaf(0.134145f, g2, 1.f);
    }
}

template <int GATE, bool EXACT, int W>
__device__ __forceinline__ void gated_as(const float (&g)[W], const float (&u)[W], float (&h)[W]) {
#pragma unroll
    for (int i = 0; i < W; ++i) {
        float a, unused;
        gate_of<GATE, EXACT, false>(g[i], a, unused);
        h[i] = a * u[i];
    }
}
// h = gate(g) u
template <bool EXACT, int W>
__device__ __forceinline__ void gated(int gate, const float (&g)[W], const float (&u)[W], float (&h)[W]) {
    if (gate == TFJSB_GATE_SILU) gated_as<TFJSB_GATE_SILU, EXACT>(g, u, h);
    else if (gate == TFJSB_GATE_GELU) gated_as<TFJSB_GATE_GELU, EXACT>(g, u, h);
    else if (gate == TFJSB_GATE_GELU_TANH) gated_as<TFJSB_GATE_GELU_TANH, EXACT>(g, u, h);
    else if (gate == TFJSB_GATE_SIGMOID) gated_as<TFJSB_GATE_SIGMOID, EXACT>(g, u, h);
    else gated_as<TFJSB_GATE_RELU, EXACT>(g, u, h);
}

template <int GATE, bool EXACT, int W>
__device__ __forceinline__ void gradient_as(const float (&g)[W], const float (&u)[W], float (&d)[W], float (&du)[W]) {
#pragma unroll
    for (int i = 0; i < W; ++i) {
        float a, slope;
        gate_of<GATE, EXACT, true>(g[i], a, slope);
        du[i] = d[i] * a;
        d[i] = d[i] * u[i] * slope;
    }
}
// d: the gradient of h on entry, that of g on return; du: that of u
template <bool EXACT, int W>
__device__ __forceinline__ void gated_gradient(int gate, const float (&g)[W], const float (&u)[W], float (&d)[W], float (&du)[W]) {
    if (gate == TFJSB_GATE_SILU) gradient_as<TFJSB_GATE_SILU, EXACT>(g, u, d, du);
    else if (gate == TFJSB_GATE_GELU) gradient_as<TFJSB_GATE_GELU, EXACT>(g, u, d, du);
    else if (gate == TFJSB_GATE_GELU_TANH) gradient_as<TFJSB_GATE_GELU_TANH, EXACT>(g, u, d, du);
    else if (gate == TFJSB_GATE_SIGMOID) gradient_as<TFJSB_GATE_SIGMOID, EXACT>(g, u, d, du);
    else gradient_as<TFJSB_GATE_RELU, EXACT>(g, u, d, du);
}

// ---- rows of W values, of which `left` exist ---------------------------------------------------------------
__host__ __device__ __forceinline__ bool aligned(const void* p, uint32_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
__device__ __forceinline__ uint32_t pack_bf16(float x, float y) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void st32(void* p, const uint32_t* v) {  // 32 bytes, one sector
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]),
                 "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
__device__ __forceinline__ void st16(void* p, const uint32_t* v) {
    asm volatile("st.global.v4.b32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}

template <int W>
__device__ __forceinline__ void store_f32(float* p, const float (&v)[W], int left) {
    const bool sector = aligned(p, 32), quad = aligned(p, 16);
#pragma unroll
    for (int j = 0; j < W; j += 8) {
        const uint32_t* bits = reinterpret_cast<const uint32_t*>(&v[j]);
        if (j + 8 <= left && sector) {
            st32(p + j, bits);
        } else if (j + 8 <= left && quad) {
            st16(p + j, bits);
            st16(p + j + 4, bits + 4);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (j + i < left) p[j + i] = v[j + i];
        }
    }
}
template <int W>
__device__ __forceinline__ void load_f32(const float* p, float (&v)[W], int left) {
    const bool sector = aligned(p, 32);
#pragma unroll
    for (int j = 0; j < W; j += 8) {
        if (j + 8 <= left && sector) {
            asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=f"(v[j]), "=f"(v[j + 1]), "=f"(v[j + 2]), "=f"(v[j + 3]), "=f"(v[j + 4]), "=f"(v[j + 5]), "=f"(v[j + 6]), "=f"(v[j + 7])
                         : "l"(p + j));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[j + i] = j + i < left ? ld_global(p + j + i) : 0.f;
        }
    }
}
// Pairs of bfloat16.
template <int W>
__device__ __forceinline__ void store_pairs(__nv_bfloat16* p, const uint32_t (&w)[W / 2], int left) {
    const bool sector = aligned(p, 32), quad = aligned(p, 16);
    constexpr int G = W < 16 ? 8 : 16;
#pragma unroll
    for (int j = 0; j < W; j += G) {
        if (G == 16 && j + G <= left && sector) {
            st32(p + j, &w[j / 2]);
        } else if (j + G <= left && quad) {
            st16(p + j, &w[j / 2]);
            if (G == 16) st16(p + j + 8, &w[j / 2 + G / 4]);
        } else {
#pragma unroll
            for (int i = 0; i < G; ++i)
                if (j + i < left) p[j + i] = __ushort_as_bfloat16((unsigned short)(w[(j + i) / 2] >> (i % 2 * 16)));
        }
    }
}
template <int W>
__device__ __forceinline__ void store_bf16(__nv_bfloat16* p, const float (&v)[W], int left) {
    uint32_t w[W / 2];
#pragma unroll
    for (int i = 0; i < W / 2; ++i) w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    store_pairs<W>(p, w, left);
}

// Values as P bfloat16 planes: themselves, rounded to nearest (P = 1), or three whose sum they are, each the rest of the one before
// rounded to nearest.  Of a value beyond the largest bfloat16 the first plane is that, so that the sum holds; of an infinity or a NaN the planes'
// sum is a NaN.
template <int P, int W>
__device__ __forceinline__ void store_planes(__nv_bfloat16* p, int64_t plane, const float (&v)[W], int left) {
    if constexpr (P == 1) {
        store_bf16(p, v, left);
    } else {
        const float most = __uint_as_float(0x7f7f0000u);
        uint32_t w[W / 2];
        float r[W];
#pragma unroll
        for (int i = 0; i < W / 2; ++i) w[i] = pack_bf16(fminf(fmaxf(v[2 * i], -most), most), fminf(fmaxf(v[2 * i + 1], -most), most));
#pragma unroll
        for (int i = 0; i < W; ++i) r[i] = v[i] - __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        store_pairs<W>(p, w, left);
#pragma unroll
        for (int i = 0; i < W / 2; ++i) w[i] = pack_bf16(r[2 * i], r[2 * i + 1]);
#pragma unroll
        for (int i = 0; i < W; ++i) r[i] -= __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        store_pairs<W>(p + plane, w, left);
#pragma unroll
        for (int i = 0; i < W / 2; ++i) w[i] = pack_bf16(r[2 * i], r[2 * i + 1]);
        store_pairs<W>(p + 2 * plane, w, left);
    }
}

// ---- parts of a sum ----------------------------------------------------------------------------------------
template <int KIND>
__device__ __forceinline__ void add_part(uint32_t (&s)[8], int i, const uint4& x) {
    if (KIND == 1) {  // 32-bit integers
        s[i] += x.x; s[i + 1] += x.y; s[i + 2] += x.z; s[i + 3] += x.w;
    } else {
        s[i] = __float_as_uint(__uint_as_float(s[i]) + __uint_as_float(x.x));
        s[i + 1] = __float_as_uint(__uint_as_float(s[i + 1]) + __uint_as_float(x.y));
        s[i + 2] = __float_as_uint(__uint_as_float(s[i + 2]) + __uint_as_float(x.z));
        s[i + 3] = __float_as_uint(__uint_as_float(s[i + 3]) + __uint_as_float(x.w));
    }
}

}  // namespace dense
}  // namespace tfjsb
