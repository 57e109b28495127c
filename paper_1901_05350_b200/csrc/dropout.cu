// tf.dropout with a mask that is made from a counter and never stored, forward (with the residual that follows it, if any) and backward.
//
// The generator is Philox-4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3",
// 2011): a bijection of a 128-bit counter under a 64-bit key, here (index of a block of four words, offset) and the seed.  Words
// are whole numbers, so keeping one is a comparison, word >= ceil(rate 2^32), and needs no conversion.
//
// A thread has eight consecutive elements, 16 or 32 bytes of each tensor.  Without broadcasting their words are two whole blocks.  With
// it (a mask of fewer dimensions) an element's index in the mask is worked out for the first of the eight; those that lie in one row of the
// innermost dimension share one word (that dimension is broadcast) or have words in a row, out of two or three blocks (it is not).
#include <cmath>

#include <cuda_bf16.h>

#include "common.cuh"
#include "dense.cuh"
#include "dense_math.cuh"
#include "ptx_sm100.cuh"

namespace tfjsb {
namespace {

constexpr int PER_THREAD = 8, BLOCK = 256;
constexpr uint32_t MULTIPLIER_0 = 0xD2511F53u, MULTIPLIER_1 = 0xCD9E8D57u, KEY_STEP[2] = {0x9E3779B9u, 0xBB67AE85u};
constexpr int ROUNDS = 10;

struct DropoutArgs {
    const void *x, *residual;
    void* out;
    int64_t n;
    uint32_t threshold;
    float scale;
    uint32_t keys[ROUNDS][2];
    uint32_t offset[2];
    // what the first two rounds make of the offset alone: see philox
    uint32_t high1, low1, high2, low2;
    // broadcast masks: the dimensions, neighbours of one kind merged, innermost first; a dimension's step in the mask is 0
    // where it is broadcast
    int dims = 0;
    uint64_t extent[4], step[4];
};

__device__ __forceinline__ void multiply(uint32_t a, uint32_t m, uint32_t& high, uint32_t& low) {
    uint64_t p;
    asm("mul.wide.u32 %0, %1, %2;" : "=l"(p) : "r"(a), "r"(m));
    asm("mov.b64 {%0, %1}, %2;" : "=r"(low), "=r"(high) : "l"(p));
}
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0x96;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}

// The four words of a block.  The offset is the same for all, so one product of the first round is worked out before the launch, and so is one of
// the second where the upper half of the block's index is 0 (SMALL: less than 2^34 elements).  The products that make 64 bits of 32
// are what the words cost most: 18 of them a block instead of 20.
template <bool SMALL>
__device__ __forceinline__ void philox(const DropoutArgs& a, uint64_t block, uint32_t (&w)[4]) {
    uint32_t h0, l0, h1, l1;
    multiply((uint32_t)block, MULTIPLIER_0, h0, l0);
    uint32_t c0 = a.high1, c1 = a.low1, c2 = xor3(h0, a.offset[1], a.keys[0][1]), c3 = l0;
    if (!SMALL) c0 ^= (uint32_t)(block >> 32);
#pragma unroll
    for (int r = 1; r < ROUNDS; ++r) {
        multiply(c2, MULTIPLIER_1, h1, l1);
        if (SMALL && r == 1) {
            h0 = a.high2;
            l0 = a.low2;
        } else {
            multiply(c0, MULTIPLIER_0, h0, l0);
        }
        c0 = xor3(h1, c1, a.keys[r][0]);
        c2 = xor3(h0, c3, a.keys[r][1]);
        c1 = l1;
        c3 = l0;
    }
    w[0] = c0; w[1] = c1; w[2] = c2; w[3] = c3;
}

// Index in the mask of element i, and where i lies in the innermost dimension.
template <typename I>
__device__ __forceinline__ uint64_t mask_index(const DropoutArgs& a, uint64_t i, uint64_t* inner) {
    I rest = (I)i;
    uint64_t m = 0;
    for (int d = 0; d < a.dims; ++d) {
        const I e = (I)a.extent[d], q = rest / e, at = rest - q * e;
        if (d == 0) *inner = at;
        m += (uint64_t)at * a.step[d];
        rest = q;
    }
    return m;
}

// Eight words of the stream from word m on (m may be "negative": words before the first mean nothing), out of two blocks or,
// where m is no multiple of four, three.
template <bool SMALL>
__device__ __forceinline__ void run_of_words(const DropoutArgs& a, uint64_t m, uint32_t (&w)[8]) {
    uint32_t v[12];
    const uint64_t block = (uint64_t)((int64_t)m >> 2);
    const uint32_t r = (uint32_t)m & 3u;
#pragma unroll
    for (int b = 0; b < 3; ++b) {
        if (b == 2 && r == 0) break;
        uint32_t q[4];
        philox<SMALL>(a, block + b, q);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * b + e] = q[e];
    }
    if (r & 1u) {
#pragma unroll
        for (int e = 0; e < 11; ++e) v[e] = v[e + 1];
    }
    if (r & 2u) {
#pragma unroll
        for (int e = 0; e < 9; ++e) v[e] = v[e + 2];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = v[e];
}

// The words of the `left` (at most eight) elements from i on.
template <bool BROADCAST, typename I>
__device__ __forceinline__ void words_of(const DropoutArgs& a, uint64_t i, int left, uint32_t (&w)[8]) {
    constexpr bool SMALL = sizeof(I) == 4;
    if (!BROADCAST) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            uint32_t q[4];
            philox<SMALL>(a, (i >> 2) + b, q);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[4 * b + e] = q[e];
        }
        return;
    }
    // run by run: the elements that lie in one row of the innermost dimension
    for (int e0 = 0; e0 < left;) {
        uint64_t inner = 0;
        const uint64_t m = mask_index<I>(a, i + e0, &inner);
        const int end = (uint64_t)(left - e0) < a.extent[0] - inner ? left : e0 + (int)(a.extent[0] - inner);
        uint32_t u[8];
        if (a.step[0] == 0) {
            uint32_t q[4];
            philox<SMALL>(a, m >> 2, q);
            const uint32_t v = (m & 2) ? ((m & 1) ? q[3] : q[2]) : ((m & 1) ? q[1] : q[0]);
#pragma unroll
            for (int e = 0; e < 8; ++e) u[e] = v;
        } else {
            run_of_words<SMALL>(a, m - (uint64_t)e0, u);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e >= e0 && e < end) w[e] = u[e];
        e0 = end;
    }
}

template <bool F32>
__device__ __forceinline__ void load8(const void* p, int64_t i, int left, float (&v)[8]) {
    if (F32) {
        dense::load_f32(static_cast<const float*>(p) + i, v, left);
    } else {
        const unsigned short* q = static_cast<const unsigned short*>(p) + i;
        if (left >= 8) {  // tensors are 16-byte aligned, i is a multiple of eight
            uint32_t w[4];
            asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(q));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[2 * e] = __uint_as_float(w[e] << 16);
                v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = e < left ? __uint_as_float((uint32_t)load_global(q + e) << 16) : 0.f;
        }
    }
}

// A block has STEPS pieces of 2048 elements: many more blocks than are resident, so that those on SMs with less to wait for take more of
// them (one wave of blocks that each did the same share left the SMs at 70 % of their warps, 73 us for 67 M bfloat16 values against 67).
constexpr int STEPS = 4;
template <bool F32, bool BROADCAST, bool RESIDUAL, typename I>
__global__ void __launch_bounds__(BLOCK) dropout_kernel(const __grid_constant__ DropoutArgs a) {
    ptx::pdl_wait();
    int64_t i = (int64_t)blockIdx.x * (STEPS * BLOCK * PER_THREAD) + threadIdx.x * PER_THREAD;
#pragma unroll 1
    for (int step = 0; step < STEPS && i < a.n; ++step, i += BLOCK * PER_THREAD) {
        const int left = a.n - i < 8 ? (int)(a.n - i) : 8;
        float x[8], r[8];
        load8<F32>(a.x, i, left, x);
        if (RESIDUAL) load8<F32>(a.residual, i, left, r);
        uint32_t w[8];
        words_of<BROADCAST, I>(a, (uint64_t)i, left, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (RESIDUAL) x[e] = w[e] >= a.threshold ? fmaf(x[e], a.scale, r[e]) : r[e];
            else x[e] = w[e] >= a.threshold ? x[e] * a.scale : 0.f;
        }
        if (F32) dense::store_f32(static_cast<float*>(a.out) + i, x, left);
        else dense::store_bf16(static_cast<__nv_bfloat16*>(a.out) + i, x, left);
    }
}

// A mask shared by many positions: [outer][positions][channels], one row of the mask for all positions of an outer index (spatial dropout of
// a sequence or an image).  A thread has four channels, whose words it makes once, of `share` positions: next to no arithmetic is left, so
// this is bound by memory where making each word again was bound by the generator (64 x 197 x 771 fp32: 28 us).  VECTOR: rows of
// channels are whole groups of four, which a thread loads at once.  Otherwise a warp has 124 channels, a thread every 32nd of them: their words
// lie in 32 blocks wherever the first begins, a block a thread (four neighbours a thread, value by value, kept an SM's loads busy with four
// lines each and took two or three blocks: 64 x 197 x 771 fp32 19 us, now 11.3).
struct Positions {
    int64_t outer, positions, groups;  // groups of four channels, or (not VECTOR) of 124
    int share;
};
template <bool F32, bool RESIDUAL, bool VECTOR>
__global__ void __launch_bounds__(BLOCK) dropout_positions_kernel(const __grid_constant__ DropoutArgs a, const __grid_constant__ Positions s) {
    ptx::pdl_wait();
    constexpr int NEXT = VECTOR ? 1 : 32, GROUP = VECTOR ? 4 : 124;  // from one channel of a thread to the next; channels of a group
    const int lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * BLOCK + threadIdx.x, g = VECTOR ? t : t >> 5, o = g / s.groups;
    if (o >= s.outer) return;  // not VECTOR: all of a warp
    const int64_t channels = (int64_t)a.extent[0], group = (g - o * s.groups) * GROUP, c = group + (VECTOR ? 0 : lane);
    const int64_t end = channels - group < GROUP ? channels : group + GROUP;  // of the group
    uint64_t m = (uint64_t)group, rest = (uint64_t)o;
    for (int d = 2; d < a.dims; ++d) {
        const uint64_t q = rest / a.extent[d];
        m += (rest - q * a.extent[d]) * a.step[d];
        rest = q;
    }
    uint32_t w[4];
    philox<false>(a, (m >> 2) + (VECTOR ? 0 : lane), w);
    bool keep[4];
    int left = 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) keep[e] = w[e] >= a.threshold;
    if (!VECTOR) {
        const uint32_t own = (keep[0] ? 1u : 0u) | (keep[1] ? 2u : 0u) | (keep[2] ? 4u : 0u) | (keep[3] ? 8u : 0u);
        left = c < end ? (int)((end - c + 31) / 32) : 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {  // word i of the group's first block and those after it
            const int i = (int)(m & 3u) + lane + 32 * e;
            keep[e] = __shfl_sync(0xffffffffu, own, i >> 2) >> (i & 3) & 1u;
        }
    }
    const int64_t first = (int64_t)blockIdx.y * s.share, last = first + s.share < s.positions ? first + s.share : s.positions;
    auto load4 = [&](const void* p, int64_t i, float (&v)[4]) {
        if (F32) {
            const float* q = static_cast<const float*>(p) + i;
            if (VECTOR) {
                const float4 f = ld_global4(q);
                v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = e < left ? load_global(q + e * NEXT) : 0.f;
            }
        } else {
            const unsigned short* q = static_cast<const unsigned short*>(p) + i;
            if (VECTOR) {
                const uint2 f = load_global(reinterpret_cast<const uint2*>(q));
                v[0] = __uint_as_float(f.x << 16); v[1] = __uint_as_float(f.x & 0xffff0000u);
                v[2] = __uint_as_float(f.y << 16); v[3] = __uint_as_float(f.y & 0xffff0000u);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = e < left ? __uint_as_float((uint32_t)load_global(q + e * NEXT) << 16) : 0.f;
            }
        }
    };
    constexpr int U = 4;  // positions on their way at a time
    for (int64_t p = first; p < last; p += U) {
        float x[U][4], r[U][4];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (p + u < last) {
                const int64_t i = (o * s.positions + p + u) * channels + c;
                load4(a.x, i, x[u]);
                if (RESIDUAL) load4(a.residual, i, r[u]);
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (p + u < last) {
                const int64_t i = (o * s.positions + p + u) * channels + c;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (RESIDUAL) x[u][e] = keep[e] ? fmaf(x[u][e], a.scale, r[u][e]) : r[u][e];
                    else x[u][e] = keep[e] ? x[u][e] * a.scale : 0.f;
                }
                if (F32) {
                    float* q = static_cast<float*>(a.out) + i;
                    if (VECTOR) *reinterpret_cast<float4*>(q) = make_float4(x[u][0], x[u][1], x[u][2], x[u][3]);
                    else
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (e < left) q[e * NEXT] = x[u][e];
                } else {
                    __nv_bfloat16* q = static_cast<__nv_bfloat16*>(a.out) + i;
                    if (VECTOR) *reinterpret_cast<uint2*>(q) = make_uint2(dense::pack_bf16(x[u][0], x[u][1]), dense::pack_bf16(x[u][2], x[u][3]));
                    else
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (e < left) q[e * NEXT] = __float2bfloat16_rn(x[u][e]);
                }
            }
    }
}

template <bool F32, bool BROADCAST, bool RESIDUAL, typename I>
cudaError_t launch(const DropoutArgs& a, cudaStream_t s) {
    const int64_t blocks = (a.n + STEPS * BLOCK * PER_THREAD - 1) / (STEPS * BLOCK * PER_THREAD);
    return launch_k(&dropout_kernel<F32, BROADCAST, RESIDUAL, I>, dim3((unsigned)blocks), dim3(BLOCK), 0, s, a);
}
template <bool F32, bool RESIDUAL>
cudaError_t launch_any(const DropoutArgs& a, int sm_count, cudaStream_t s) {
    // One row of the mask for at least eight positions, and enough threads with four channels of eight or more positions to fill the GPU
    if (a.dims >= 2 && a.step[0] == 1 && a.step[1] == 0 && a.extent[1] >= 8) {
        Positions p;
        p.positions = (int64_t)a.extent[1];
        const bool vector = a.extent[0] % 4 == 0;
        p.groups = ((int64_t)a.extent[0] + (vector ? 3 : 123)) / (vector ? 4 : 124);
        p.outer = a.n / (int64_t)(a.extent[0] * a.extent[1]);
        const int64_t threads = p.outer * p.groups * (vector ? 1 : 32), blocks = (threads + BLOCK - 1) / BLOCK;
        p.share = 32;
        while (p.share > 8 && blocks * ((p.positions + p.share - 1) / p.share) < (int64_t)sm_count * 8) p.share /= 2;
        const int64_t shares = (p.positions + p.share - 1) / p.share;
        if (a.extent[0] >= 32 && blocks < (1LL << 31) && shares <= 65535) {
            auto* kernel = vector ? &dropout_positions_kernel<F32, RESIDUAL, true> : &dropout_positions_kernel<F32, RESIDUAL, false>;
            return launch_k(kernel, dim3((unsigned)blocks, (unsigned)shares), dim3(BLOCK), 0, s, a, p);
        }
    }
    const bool small = a.n < (1LL << 31);
    if (a.dims == 0) return small ? launch<F32, false, RESIDUAL, uint32_t>(a, s) : launch<F32, false, RESIDUAL, uint64_t>(a, s);
    return small ? launch<F32, true, RESIDUAL, uint32_t>(a, s) : launch<F32, true, RESIDUAL, uint64_t>(a, s);
}

bool overlaps_partly(const void* a, const void* b, int64_t bytes) {
    const char *x = static_cast<const char*>(a), *y = static_cast<const char*>(b);
    return x != y && x < y + bytes && y < x + bytes;
}

tfjsb_status run(tfjsb_ctx* ctx, tfjsb_dtype dtype, const void* x, const char* x_name, const void* residual, void* out, const char* out_name, int32_t rank,
                 const int64_t* dims, const int64_t* noise, double rate, uint64_t seed, uint64_t offset, void* stream) {
    if (!ctx) return TFJSB_ERR_INVALID_ARG;
    const dense::OnDevice on(ctx);
    if (dtype != TFJSB_DTYPE_F32 && dtype != TFJSB_DTYPE_BF16) return fail(ctx, TFJSB_ERR_INVALID_ARG, "unknown dtype");
    if (rank < 1 || rank > 4) return fail(ctx, TFJSB_ERR_INVALID_ARG, "rank " + std::to_string(rank) + ", expected 1..4");
    if (!dims) return fail(ctx, TFJSB_ERR_INVALID_ARG, "dims is null");
    if (!(rate >= 0.0 && rate < 1.0)) return fail(ctx, TFJSB_ERR_INVALID_ARG, "rate must be in [0, 1)");
    DropoutArgs a;
    a.n = 1;
    bool empty = false;
    for (int d = 0; d < rank; ++d) {
        if (dims[d] < 0) return fail(ctx, TFJSB_ERR_SHAPE, std::string(x_name) + " has a negative dimension");
        if (noise && noise[d] != dims[d] && noise[d] != 1)
            return fail(ctx, TFJSB_ERR_SHAPE, "each dimension of the mask must be that of " + std::string(x_name) + " or 1");
        if (dims[d] == 0) empty = true;
    }
    if (empty) return TFJSB_OK;
    for (int d = 0; d < rank; ++d) {
        if (dims[d] > (1LL << 40) / a.n) return fail(ctx, TFJSB_ERR_SHAPE, "more than 2^40 elements");
        a.n *= dims[d];
    }
    if (!x || !out) return fail(ctx, TFJSB_ERR_INVALID_ARG, std::string(x_name) + " / " + out_name + " is null");
    if (!dense::aligned(x, 16) || !dense::aligned(out, 16) || (residual && !dense::aligned(residual, 16)))
        return fail(ctx, TFJSB_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
    const int64_t bytes = a.n * (dtype == TFJSB_DTYPE_F32 ? 4 : 2);
    if (overlaps_partly(x, out, bytes) || (residual && overlaps_partly(residual, out, bytes)))
        return fail(ctx, TFJSB_ERR_INVALID_ARG, std::string(out_name) + " overlaps an input that it is not");
    a.x = x;
    a.residual = residual;
    a.out = out;
    a.threshold = (uint32_t)std::ceil(std::ldexp(rate, 32));  // rate < 1: at most 2^32 - 1 unless within 2^-32 of 1
    if (std::ceil(std::ldexp(rate, 32)) >= 4294967296.0) return fail(ctx, TFJSB_ERR_INVALID_ARG, "rate is within 2^-32 of 1");
    a.scale = (float)(1.0 / (1.0 - rate));
    for (int r = 0; r < ROUNDS; ++r)
        for (int k = 0; k < 2; ++k) a.keys[r][k] = (uint32_t)(seed >> (32 * k)) + (uint32_t)r * KEY_STEP[k];
    a.offset[0] = (uint32_t)offset;
    a.offset[1] = (uint32_t)(offset >> 32);
    const uint64_t p1 = (uint64_t)a.offset[0] * MULTIPLIER_1;
    a.high1 = (uint32_t)(p1 >> 32) ^ a.keys[0][0];
    a.low1 = (uint32_t)p1;
    const uint64_t p2 = (uint64_t)a.high1 * MULTIPLIER_0;
    a.high2 = (uint32_t)(p2 >> 32);
    a.low2 = (uint32_t)p2;
    if (noise) {
        // dimensions innermost first; those of extent 1 say nothing, neighbours of one kind are one dimension
        uint64_t in_mask = 1;
        for (int d = rank - 1; d >= 0; --d) {
            if (dims[d] == 1) continue;
            const bool shared = noise[d] == 1;
            if (a.dims > 0 && (a.step[a.dims - 1] == 0) == shared) {
                a.extent[a.dims - 1] *= (uint64_t)dims[d];
            } else {
                a.extent[a.dims] = (uint64_t)dims[d];
                a.step[a.dims] = shared ? 0 : in_mask;
                ++a.dims;
            }
            if (!shared) in_mask *= (uint64_t)dims[d];
        }
        if (a.dims == 1 && a.step[0] == 1) a.dims = 0;  // nothing is broadcast
    }
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (dtype == TFJSB_DTYPE_F32) e = residual ? launch_any<true, true>(a, ctx->sm_count, s) : launch_any<true, false>(a, ctx->sm_count, s);
    else e = residual ? launch_any<false, true>(a, ctx->sm_count, s) : launch_any<false, false>(a, ctx->sm_count, s);
    if (e != cudaSuccess) return cuda_fail(ctx, e, "dropout launch");
    count_launch(&ctx->launches);
    return TFJSB_OK;
}

}  // namespace
}  // namespace tfjsb

extern "C" {

tfjsb_status tfjsb_dropout(tfjsb_ctx* ctx, tfjsb_dtype dtype, const void* x, const void* residual, void* out, int32_t rank, const int64_t* dims,
                           const int64_t* noise_dims, double rate, uint64_t seed, uint64_t offset, void* stream) {
    return tfjsb::run(ctx, dtype, x, "x", residual, out, "out", rank, dims, noise_dims, rate, seed, offset, stream);
}

tfjsb_status tfjsb_dropout_backprop(tfjsb_ctx* ctx, tfjsb_dtype dtype, const void* dy, void* dx, int32_t rank, const int64_t* dims,
                                    const int64_t* noise_dims, double rate, uint64_t seed, uint64_t offset, void* stream) {
    return tfjsb::run(ctx, dtype, dy, "dy", nullptr, dx, "dx", rank, dims, noise_dims, rate, seed, offset, stream);
}

}  // extern "C"
