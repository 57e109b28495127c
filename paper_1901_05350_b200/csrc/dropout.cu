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
constexpr uint32_t MULTIPLIER[2] = {0xD2511F53u, 0xCD9E8D57u}, KEY_STEP[2] = {0x9E3779B9u, 0xBB67AE85u};
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

// The four words of a block.  The offset is the same for all, so one product of the first round is worked out before the launch, and so is one of
// the second where the upper half of the block's index is 0 (SMALL: less than 2^34 elements).  The multiplier that makes 64 bits of 32 is
// what bounds the kernel next to memory: 18 of them a block instead of 20.
template <bool SMALL>
__device__ __forceinline__ void philox(const DropoutArgs& a, uint64_t block, uint32_t (&w)[4]) {
    const uint64_t first = (uint64_t)(uint32_t)block * MULTIPLIER[0];
    uint32_t c0 = a.high1, c1 = a.low1, c2 = (uint32_t)(first >> 32) ^ a.offset[1] ^ a.keys[0][1], c3 = (uint32_t)first;
    if (!SMALL) c0 ^= (uint32_t)(block >> 32);
#pragma unroll
    for (int r = 1; r < ROUNDS; ++r) {
        const uint64_t p1 = (uint64_t)c2 * MULTIPLIER[1];
        uint32_t h0, l0;
        if (SMALL && r == 1) {
            h0 = a.high2;
            l0 = a.low2;
        } else {
            const uint64_t p0 = (uint64_t)c0 * MULTIPLIER[0];
            h0 = (uint32_t)(p0 >> 32);
            l0 = (uint32_t)p0;
        }
        c0 = (uint32_t)(p1 >> 32) ^ c1 ^ a.keys[r][0];
        c2 = h0 ^ c3 ^ a.keys[r][1];
        c1 = (uint32_t)p1;
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

template <bool F32, bool BROADCAST, bool RESIDUAL, typename I>
__global__ void __launch_bounds__(BLOCK) dropout_kernel(const __grid_constant__ DropoutArgs a) {
    ptx::pdl_wait();
    const int64_t step = (int64_t)gridDim.x * BLOCK * PER_THREAD;
    for (int64_t i = ((int64_t)blockIdx.x * BLOCK + threadIdx.x) * PER_THREAD; i < a.n; i += step) {
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

template <bool F32, bool BROADCAST, bool RESIDUAL, typename I>
cudaError_t launch(const DropoutArgs& a, int sm_count, cudaStream_t s) {
    auto* kernel = &dropout_kernel<F32, BROADCAST, RESIDUAL, I>;
    // One wave of blocks, so that none is left over for a second.
    static const int resident = [kernel] {
        int n = 0;
        return cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, BLOCK, 0) == cudaSuccess && n > 0 ? n : 1;
    }();
    const int64_t needed = (a.n + BLOCK * PER_THREAD - 1) / (BLOCK * PER_THREAD), most = (int64_t)sm_count * resident;
    return launch_k(kernel, dim3((unsigned)(needed < most ? needed : most)), dim3(BLOCK), 0, s, a);
}
template <bool F32, bool RESIDUAL>
cudaError_t launch_any(const DropoutArgs& a, int sm_count, cudaStream_t s) {
    const bool small = a.n < (1LL << 31);
    if (a.dims == 0) return small ? launch<F32, false, RESIDUAL, uint32_t>(a, sm_count, s) : launch<F32, false, RESIDUAL, uint64_t>(a, sm_count, s);
    return small ? launch<F32, true, RESIDUAL, uint32_t>(a, sm_count, s) : launch<F32, true, RESIDUAL, uint64_t>(a, sm_count, s);
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
        if (dims[d] > (1LL << 42) / a.n) return fail(ctx, TFJSB_ERR_SHAPE, "more than 2^42 elements");
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
    const uint64_t p1 = (uint64_t)a.offset[0] * MULTIPLIER[1];
    a.high1 = (uint32_t)(p1 >> 32) ^ a.keys[0][0];
    a.low1 = (uint32_t)p1;
    const uint64_t p2 = (uint64_t)a.high1 * MULTIPLIER[0];
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
    ++ctx->launches;
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
