// Dense layers on 8-bit integers: rows quantised with a scale of their own, products with exact 32-bit sums (dense_tcgen05.cu, kind::i8), and
// the epilogue act(sum a_scale b_scale + bias).
#include <cuda_bf16.h>

#include "common.cuh"
#include "dense.cuh"
#include "dense_math.cuh"
#include "ptx_sm100.cuh"
#include "quantize.cuh"

namespace tfjsb {
namespace dense {
namespace {

constexpr int64_t MAX_K = 131072;  // 2^17 products of at most 2^14: sums fit 32 bits
constexpr int QUANTIZE_THREADS = 256;

// A block has a row.  Its first HELD groups of 2048 values stay in registers between the maximum and the rounding, the others are read again.
template <bool F32, int HELD>
__global__ void __launch_bounds__(QUANTIZE_THREADS) quantize_kernel(const void* x, int64_t columns, int64_t pitch, int8_t* q, float* scale) {
    ptx::pdl_wait();
    ptx::pdl_launch_dependents();
    __shared__ float part[QUANTIZE_THREADS / 32];
    constexpr int STEP = QUANTIZE_THREADS * 8;
    const int64_t row = blockIdx.x, base = row * columns;
    auto left_at = [&](int64_t c) { return columns - c < 8 ? (int)(columns - c) : 8; };
    float held[HELD][8];
    float amax = 0.f;
#pragma unroll
    for (int j = 0; j < HELD; ++j) {
        const int64_t c = (int64_t)j * STEP + threadIdx.x * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) held[j][e] = 0.f;
        if (c < columns) values8<F32>(x, base + c, left_at(c), held[j]);
    }
#pragma unroll
    for (int j = 0; j < HELD; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = max_nan(amax, fabsf(held[j][e]));
    for (int64_t c = (int64_t)HELD * STEP + threadIdx.x * 8; c < columns; c += STEP) {
        float v[8];
        values8<F32>(x, base + c, left_at(c), v);
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = max_nan(amax, fabsf(v[e]));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = amax;
    __syncthreads();
    amax = part[0];
#pragma unroll
    for (int w = 1; w < QUANTIZE_THREADS / 32; ++w) amax = max_nan(amax, part[w]);
    const RowScale r = row_scale(amax);
    if (threadIdx.x == 0) scale[row] = amax / 127.f;
    int8_t* out = q + row * pitch;  // the pitch is a multiple of 16
#pragma unroll
    for (int j = 0; j < HELD; ++j) {
        const int64_t c = (int64_t)j * STEP + threadIdx.x * 8;
        if (c < pitch) *reinterpret_cast<uint2*>(out + c) = quantize8<F32>(held[j], r);
    }
    for (int64_t c = (int64_t)HELD * STEP + threadIdx.x * 8; c < pitch; c += STEP) {
        float v[8] = {};
        if (c < columns) values8<F32>(x, base + c, left_at(c), v);
        *reinterpret_cast<uint2*>(out + c) = quantize8<F32>(v, r);
    }
}

// A warp has a row, which it holds as it is stored: many rows whose length is a multiple of eight, up to GROUPS * 256 bfloat16 or GROUPS * 128
// fp32 values.  No block waits for its slowest load, and an SM has 160 KiB of rows on their way (8192 x 4096 bfloat16: a block a row 32 us).
template <bool F32, int GROUPS>
__global__ void __launch_bounds__(128) quantize_rows_kernel(const void* x, int64_t rows, int64_t columns, int64_t pitch, int8_t* q, float* scale) {
    ptx::pdl_wait();
    ptx::pdl_launch_dependents();
    constexpr int PER = F32 ? 4 : 8;  // values of 16 bytes
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (row >= rows) return;
    const uint4* in = reinterpret_cast<const uint4*>(static_cast<const char*>(x) + row * columns * (F32 ? 4 : 2));
    const int pieces = (int)(columns / PER);
    uint4 v[GROUPS];
#pragma unroll
    for (int j = 0; j < GROUPS; ++j) {
        v[j] = make_uint4(0u, 0u, 0u, 0u);
        if (j * 32 + lane < pieces)
            asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[j].x), "=r"(v[j].y), "=r"(v[j].z), "=r"(v[j].w) : "l"(in + j * 32 + lane));
    }
    float amax;
    if (F32) {
        amax = 0.f;
#pragma unroll
        for (int j = 0; j < GROUPS; ++j) {
            amax = max_nan(amax, max_nan(fabsf(__uint_as_float(v[j].x)), fabsf(__uint_as_float(v[j].y))));
            amax = max_nan(amax, max_nan(fabsf(__uint_as_float(v[j].z)), fabsf(__uint_as_float(v[j].w))));
        }
    } else {
        uint32_t m = 0u;  // two bfloat16
        auto more = [&](uint32_t w) { asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(w & 0x7fff7fffu)); };
#pragma unroll
        for (int j = 0; j < GROUPS; ++j) { more(v[j].x); more(v[j].y); more(v[j].z); more(v[j].w); }
        amax = max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    const RowScale r = row_scale(amax);
    if (lane == 0) scale[row] = amax / 127.f;
    int8_t* out = q + row * pitch;
#pragma unroll
    for (int j = 0; j < GROUPS; ++j) {
        const int at = j * 32 + lane;
        if (at >= pieces) continue;
        const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
        float f[8];
        if (F32) {
#pragma unroll
            for (int e = 0; e < 4; ++e) { f[e] = __uint_as_float(w[e]); f[e + 4] = 0.f; }
            *reinterpret_cast<uint32_t*>(out + at * 4) = quantize8<true>(f, r).x;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) { f[2 * e] = __uint_as_float(w[e] << 16); f[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u); }
            *reinterpret_cast<uint2*>(out + at * 8) = quantize8<false>(f, r);
        }
    }
    if (columns + lane * 4 < pitch) *reinterpret_cast<uint32_t*>(out + columns + lane * 4) = 0u;  // a filled-up end of 4 or 8
}

template <bool F32>
cudaError_t launch_quantize_as(int sm_count, const void* x, int64_t rows, int64_t columns, int8_t* q, float* scale, cudaStream_t s) {
    const int64_t pitch = (columns + 15) / 16 * 16;
    // a warp a row where that is enough warps for the GPU: eight an SM
    if (rows >= (int64_t)sm_count * 8 && columns % 8 == 0 && columns <= (F32 ? 2048 : 4096)) {
        constexpr int ALL = 16;
        auto* kernel = columns <= (F32 ? 512 : 1024) ? &quantize_rows_kernel<F32, ALL / 4>
                       : columns <= (F32 ? 1024 : 2048) ? &quantize_rows_kernel<F32, ALL / 2>
                                                        : &quantize_rows_kernel<F32, ALL>;
        return launch_k(kernel, dim3((unsigned)((rows + 3) / 4)), dim3(128), 0, s, x, rows, columns, pitch, q, scale);
    }
    auto* kernel = columns <= 2048 ? &quantize_kernel<F32, 1> : columns <= 4096 ? &quantize_kernel<F32, 2> : &quantize_kernel<F32, 4>;
    return launch_k(kernel, dim3((unsigned)rows), dim3(QUANTIZE_THREADS), 0, s, x, columns, pitch, q, scale);
}
cudaError_t launch_quantize(tfjsb_ctx* ctx, bool f32, const void* x, int64_t rows, int64_t columns, int8_t* q, float* scale, cudaStream_t s) {
    const cudaError_t e = f32 ? launch_quantize_as<true>(ctx->sm_count, x, rows, columns, q, scale, s)
                              : launch_quantize_as<false>(ctx->sm_count, x, rows, columns, q, scale, s);
    if (e == cudaSuccess) count_launch(&ctx->launches);
    return e;
}

// One kernel on CUDA cores instead of two launches: a single row, and layers so small that launching takes longest.  A warp of it takes 0.2 ns of the
// GPU's time for each output, and 0.1 ns more per 1000 values of K: it is taken where that is less than 2.6 us in all.
// M x N x K of bfloat16, us in a captured graph, one kernel | two; within the rule: 2 x 2048 x 1024 3.9 | 6.7, 8 x 256 x 4096 3.9 | 6.9, 32 x 256 x 256
// 4.7 | 5.5, 2 x 1000 x 8192 6.0 | 8.7, 8 x 1024 x 1024 5.1 | 6.7, 128 x 64 x 1024 5.2 | 7.0, 256 x 40 x 256 5.7 | 5.4; beyond it: 128 x 100 x 128 6.6 | 6.7,
// 8 x 1024 x 2048 5.9 | 6.8, 64 x 256 x 256 7.0 | 5.6, 16 x 1024 x 512 7.0 | 6.0, 64 x 64 x 8192 8.2 | 9.2, 2 x 8192 x 1024 7.3 | 6.9.
bool few_products(int64_t M, int64_t N, int64_t K) { return M == 1 || M * N <= 26000000 / (K + 2048); }

bool known(tfjsb_dtype d) { return d == TFJSB_DTYPE_F32 || d == TFJSB_DTYPE_BF16; }
bool overlap(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
    if (!a || !b || a_bytes <= 0 || b_bytes <= 0) return false;
    const char *x = static_cast<const char*>(a), *y = static_cast<const char*>(b);
    return x < y + b_bytes && y < x + a_bytes;
}
int64_t up16(int64_t v) { return (v + 15) / 16 * 16; }
int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }

tfjsb_status check_product(tfjsb_ctx* ctx, const void* bt, const float* b_scale, const float* bias, tfjsb_act act, void* out, tfjsb_dtype out_dtype,
                           int64_t M, int64_t N, int64_t K) {
    if (!known(out_dtype)) return fail(ctx, TFJSB_ERR_INVALID_ARG, "unknown dtype");
    if (act != TFJSB_ACT_NONE && act != TFJSB_ACT_RELU && act != TFJSB_ACT_RELU6) return fail(ctx, TFJSB_ERR_INVALID_ARG, "unknown activation");
    if (M < 0 || N < 0 || K < 1 || M > (1LL << 30) || N > (1LL << 30)) return fail(ctx, TFJSB_ERR_SHAPE, "sizes: 0 <= M, N <= 2^30, K >= 1");
    if (K > MAX_K) return fail(ctx, TFJSB_ERR_UNSUPPORTED, "K is above 131072: 32-bit sums could overflow");
    if (M == 0 || N == 0) return TFJSB_OK;
    if (!bt || !b_scale || !out) return fail(ctx, TFJSB_ERR_INVALID_ARG, "bt / b_scale / out is null");
    if (!aligned(bt, 16) || !aligned(out, 16) || !aligned(b_scale, 16) || (bias && !aligned(bias, 16)))
        return fail(ctx, TFJSB_ERR_INVALID_ARG, "pointers must be 16-byte aligned");
    const int64_t bytes = M * N * (out_dtype == TFJSB_DTYPE_F32 ? 4 : 2);
    if (overlap(out, bytes, bt, N * up16(K)) || overlap(out, bytes, b_scale, 4 * N) || overlap(out, bytes, bias, 4 * N))
        return fail(ctx, TFJSB_ERR_INVALID_ARG, "out overlaps an input");
    return TFJSB_OK;
}

tfjsb_status product(tfjsb_ctx* ctx, const int8_t* a, const float* a_scale, const int8_t* bt, const float* b_scale, const float* bias, tfjsb_act act,
                     void* out, tfjsb_dtype out_dtype, int64_t M, int64_t N, int64_t K, bool quantized_before, cudaStream_t s) {
    if (M == 1) return rows_int8(ctx, 0, a, a_scale, bt, b_scale, bias, act, out, out_dtype == TFJSB_DTYPE_BF16, M, N, K, s);
    Product p;
    p.kind = KIND_INT8;
    p.epilogue = EPI_SCALE;
    p.a.base = a;
    p.a.pitch = K;
    p.b[0].base = bt;
    p.b[0].pitch = K;
    p.args.M = (int)M; p.args.N = (int)N; p.args.K = (int)K;
    p.args.out[0] = out;
    p.args.out_pitch = N;
    p.args.out_bf16 = out_dtype == TFJSB_DTYPE_BF16;
    p.args.act = act;
    p.args.a_scale = a_scale;
    p.args.b_scale = b_scale;
    p.args.bias = bias;
    p.args.early_b = quantized_before;  // the kernel before is the one that quantised A
    return run_product(ctx, p, s);
}

}  // namespace
}  // namespace dense
}  // namespace tfjsb

using namespace tfjsb;
using namespace tfjsb::dense;

extern "C" {

tfjsb_status tfjsb_quantize_int8(tfjsb_ctx* ctx, tfjsb_dtype dtype, const void* x, int64_t rows, int64_t columns, int8_t* q, float* scale, void* stream) {
    if (!ctx) return TFJSB_ERR_INVALID_ARG;
    const dense::OnDevice on(ctx);
    if (!known(dtype)) return fail(ctx, TFJSB_ERR_INVALID_ARG, "unknown dtype");
    if (rows < 0 || rows > (1LL << 30) || columns < 1) return fail(ctx, TFJSB_ERR_SHAPE, "sizes: 0 <= rows <= 2^30, columns >= 1");
    if (columns > MAX_K) return fail(ctx, TFJSB_ERR_UNSUPPORTED, "more than 131072 columns");
    if (rows == 0) return TFJSB_OK;
    if (!x || !q || !scale) return fail(ctx, TFJSB_ERR_INVALID_ARG, "x / q / scale is null");
    if (!aligned(x, 16) || !aligned(q, 16) || !aligned(scale, 16)) return fail(ctx, TFJSB_ERR_INVALID_ARG, "pointers must be 16-byte aligned");
    const int64_t in = rows * columns * (dtype == TFJSB_DTYPE_F32 ? 4 : 2), out = rows * up16(columns);
    if (overlap(x, in, q, out) || overlap(x, in, scale, 4 * rows) || overlap(q, out, scale, 4 * rows))
        return fail(ctx, TFJSB_ERR_INVALID_ARG, "x, q and scale overlap");
    const cudaError_t e = launch_quantize(ctx, dtype == TFJSB_DTYPE_F32, x, rows, columns, q, scale, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? TFJSB_OK : cuda_fail(ctx, e, "quantize launch");
}

tfjsb_status tfjsb_matmul_int8(tfjsb_ctx* ctx, const int8_t* a, const float* a_scale, const int8_t* bt, const float* b_scale, const float* bias,
                               tfjsb_act act, void* out, tfjsb_dtype out_dtype, int64_t M, int64_t N, int64_t K, void* stream) {
    if (!ctx) return TFJSB_ERR_INVALID_ARG;
    const dense::OnDevice on(ctx);
    ran().count = 0;
    const tfjsb_status st = check_product(ctx, bt, b_scale, bias, act, out, out_dtype, M, N, K);
    if (st != TFJSB_OK) return st;
    if (K % 16) return fail(ctx, TFJSB_ERR_UNSUPPORTED, "K must be a multiple of 16: fill rows up with zeros");
    if (M == 0 || N == 0) return TFJSB_OK;
    if (!a || !a_scale) return fail(ctx, TFJSB_ERR_INVALID_ARG, "a / a_scale is null");
    if (!aligned(a, 16) || !aligned(a_scale, 16)) return fail(ctx, TFJSB_ERR_INVALID_ARG, "pointers must be 16-byte aligned");
    const int64_t bytes = M * N * (out_dtype == TFJSB_DTYPE_F32 ? 4 : 2);
    if (overlap(out, bytes, a, M * K) || overlap(out, bytes, a_scale, 4 * M)) return fail(ctx, TFJSB_ERR_INVALID_ARG, "out overlaps an input");
    return product(ctx, a, a_scale, bt, b_scale, bias, act, out, out_dtype, M, N, K, false, static_cast<cudaStream_t>(stream));
}

int64_t tfjsb_dense_int8_workspace(int64_t M, int64_t K) {
    if (M < 0 || K < 1 || M > (1LL << 30) || K > MAX_K) return 0;
    return up256(M * up16(K)) + up256(4 * M);
}

tfjsb_status tfjsb_dense_int8(tfjsb_ctx* ctx, tfjsb_dtype dtype, const void* x, const int8_t* bt, const float* b_scale, const float* bias, tfjsb_act act,
                              void* out, tfjsb_dtype out_dtype, int64_t M, int64_t N, int64_t K, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!ctx) return TFJSB_ERR_INVALID_ARG;
    const dense::OnDevice on(ctx);
    ran().count = 0;
    if (!known(dtype)) return fail(ctx, TFJSB_ERR_INVALID_ARG, "unknown dtype");
    const tfjsb_status st = check_product(ctx, bt, b_scale, bias, act, out, out_dtype, M, N, K);
    if (st != TFJSB_OK) return st;
    if (M == 0 || N == 0) return TFJSB_OK;
    const int64_t needed = tfjsb_dense_int8_workspace(M, K);
    if (workspace_bytes < needed) return fail(ctx, TFJSB_ERR_INVALID_ARG, "the workspace needs " + std::to_string(needed) + " bytes");
    if (!x || !workspace) return fail(ctx, TFJSB_ERR_INVALID_ARG, "x / workspace is null");
    if (!aligned(x, 16) || !aligned(workspace, 16)) return fail(ctx, TFJSB_ERR_INVALID_ARG, "pointers must be 16-byte aligned");
    const int64_t x_bytes = M * K * (dtype == TFJSB_DTYPE_F32 ? 4 : 2), out_bytes = M * N * (out_dtype == TFJSB_DTYPE_F32 ? 4 : 2);
    if (overlap(out, out_bytes, x, x_bytes) || overlap(out, out_bytes, workspace, needed) || overlap(workspace, needed, x, x_bytes) ||
        overlap(workspace, needed, bt, N * up16(K)) || overlap(workspace, needed, b_scale, 4 * N) || overlap(workspace, needed, bias, 4 * N))
        return fail(ctx, TFJSB_ERR_INVALID_ARG, "out or the workspace overlaps another argument");
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (few_products(M, N, K))
        return rows_int8(ctx, dtype == TFJSB_DTYPE_F32 ? 2 : 1, x, nullptr, bt, b_scale, bias, act, out, out_dtype == TFJSB_DTYPE_BF16, M, N, K, s);
    int8_t* q = static_cast<int8_t*>(workspace);
    float* scale = reinterpret_cast<float*>(q + up256(M * up16(K)));
    const cudaError_t e = launch_quantize(ctx, dtype == TFJSB_DTYPE_F32, x, M, K, q, scale, s);
    if (e != cudaSuccess) return cuda_fail(ctx, e, "quantize launch");
    return product(ctx, q, scale, bt, b_scale, bias, act, out, out_dtype, M, N, up16(K), true, s);
}

}  // extern "C"
