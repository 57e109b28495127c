// Products of few rows with large weights, on CUDA cores: the dense layers of transformer blocks when they serve single tokens.
//
// With a few rows nothing but reading the weights costs time (a byte of them is used in 1 to 8 multiply-adds), so what counts is
// that every SM has enough loads in flight and that the launches are short.  Each weight is read once, 16 bytes a load, all rows are
// multiplied with it, and long sums are cut among the threads, the warps and the CTAs of a cluster, whose parts are added in a fixed
// order through shared and distributed shared memory.
//
//   matrices [K, N] (the gated block): a block has 64 columns, a thread 8 of them and every 32nd k; K is cut among the CTAs of a cluster
//   matrices [N, K] of 8-bit integers: a block has one row of x, which it quantises, or copies, into shared memory; a warp has a row of
//   weights, a lane 16 bytes of each 512
#include <cuda_bf16.h>

#include "common.cuh"
#include "dense.cuh"
#include "dense_math.cuh"
#include "ptx_sm100.cuh"
#include "quantize.cuh"

namespace tfjsb {
namespace dense {

using namespace ptx;

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int COLUMNS = 64;   // of a block: 8 groups of 8
constexpr int K_LANES = 32;   // threads of a column group
constexpr int CHUNK = 2048;   // values of a row of x in shared memory at a time

__device__ __forceinline__ void st_cluster(uint32_t addr, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}
__device__ __forceinline__ uint4 ld_weights(const void* p) {  // read once: not kept in L1
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// Eight weights of a row: 16 bytes of bfloat16 or 32 of fp32.
template <bool F32>
struct Eight {
    uint4 a[F32 ? 2 : 1];
    __device__ __forceinline__ float operator[](int i) const {  // i: a constant
        const uint4& v = a[F32 ? i / 4 : 0];
        const int e = F32 ? i % 4 : i / 2;
        const uint32_t w = e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w;
        if (F32) return __uint_as_float(w);
        return __uint_as_float(i % 2 ? w & 0xffff0000u : w << 16);
    }
    // of row k, columns c ..; VECTOR: rows are a multiple of 16 bytes and all eight exist
    template <bool VECTOR>
    __device__ __forceinline__ void load(const void* w, int64_t k, int64_t N, int64_t c, int left) {
        const int64_t at = k * N + c;
        if (VECTOR) {
            const char* p = static_cast<const char*>(w) + at * (F32 ? 4 : 2);
            a[0] = ld_weights(p);
            if (F32) a[F32 ? 1 : 0] = ld_weights(p + 16);
        } else {
            uint32_t v[8] = {};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) v[i] = F32 ? __float_as_uint(ld_global(static_cast<const float*>(w) + at + i)) : (uint32_t)load_global(static_cast<const unsigned short*>(w) + at + i);
            if (F32) {
                a[0] = make_uint4(v[0], v[1], v[2], v[3]);
                a[F32 ? 1 : 0] = make_uint4(v[4], v[5], v[6], v[7]);
            } else {
                a[0] = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
            }
        }
    }
};

struct FewArgs {
    const void* x;        // [rows, K]: of the weights' type, or fp32 (X32)
    const void *w0, *w1;  // [K, N]
    void* out;            // [rows, N]
    int64_t N;
    int K, rows, k_per_slice, splits, gate;
};

// out = x w0, or gate(x w0) (x w1) in fp32.  T rows at most; a cluster of `splits` CTAs for every 64 columns.
template <bool F32, bool X32, bool GATED, int T, bool VECTOR>
__global__ void __launch_bounds__(THREADS) few_rows_kernel(const __grid_constant__ FewArgs a) {
    constexpr int M = GATED ? 2 : 1;
    constexpr int U = T >= 8 ? 4 : 8;  // rows of weights in flight a thread and matrix
    extern __shared__ float xs[];      // [k][T] of this slice, a chunk at a time
    __shared__ float part[WARPS][M][T * 8][8];
    __shared__ float sums[M][T][COLUMNS];  // [slice][column of this CTA's share]: every CTA of the cluster writes its slice's part
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = lane & 7, k_lane = warp * 4 + (lane >> 3);
    const uint32_t slice = a.splits > 1 ? cluster_ctarank() : 0u;
    const int64_t c0 = (int64_t)(blockIdx.x / a.splits) * COLUMNS, c = c0 + group * 8;
    const int left = (int)min((int64_t)8, a.N - c);
    const int k_begin = (int)slice * a.k_per_slice, k_end = min(a.K, k_begin + a.k_per_slice);
    float acc[M][T][8] = {};
    if (a.splits > 1) cluster_arrive();  // "has begun", which the others wait for before they write here
    Eight<F32> w[M][U];
    auto fetch_half = [&](int k0, int count, int k, int half) {
#pragma unroll
        for (int v = 0; v < U / 2; ++v) {
            const int u = half * (U / 2) + v;
            if (k + u * K_LANES < count && left > 0) {
                w[0][u].template load<VECTOR>(a.w0, k0 + k + u * K_LANES, a.N, c, left);
                if (GATED) w[M - 1][u].template load<VECTOR>(a.w1, k0 + k + u * K_LANES, a.N, c, left);
            }
        }
    };
    auto fetch = [&](int k0, int count, int k) {
        fetch_half(k0, count, k, 0);
        fetch_half(k0, count, k, 1);
    };
    // The second kernel of a block follows the first, which writes no weights and lets this one start once everything before it is
    // done: its first weights are on their way while the first kernel runs.
    if (!GATED) fetch(k_begin, min(CHUNK, k_end - k_begin), k_lane);
    pdl_wait();
    pdl_launch_dependents();

    for (int k0 = k_begin; k0 < k_end; k0 += CHUNK) {
        const int count = min(CHUNK, k_end - k0);
        if (k0 != k_begin) __syncthreads();
        if (GATED || k0 != k_begin) fetch(k0, count, k_lane);  // on its way while x is
        for (int i = threadIdx.x; i < count * T; i += THREADS) {
            const int t = i / count, k = i - t * count;  // rows of x along threads
            float v = 0.f;
            if (t < a.rows) {
                const int64_t at = (int64_t)t * a.K + k0 + k;
                v = F32 || X32 ? load_global(static_cast<const float*>(a.x) + at)
                               : __uint_as_float((uint32_t)load_global(static_cast<const unsigned short*>(a.x) + at) << 16);
            }
            xs[k * T + t] = v;
        }
        __syncthreads();
        for (int k = k_lane; k < count; k += U * K_LANES) {
            // one half is used while the other, and then its own successor, is on its way
#pragma unroll
            for (int half = 0; half < 2; ++half) {
#pragma unroll
                for (int v = 0; v < U / 2; ++v) {
                    const int u = half * (U / 2) + v;
                    if (k + u * K_LANES < count && left > 0) {
                        float x[T];
#pragma unroll
                        for (int t = 0; t < T; ++t) x[t] = xs[(k + u * K_LANES) * T + t];
#pragma unroll
                        for (int m = 0; m < M; ++m)
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const float value = w[m][u][i];
#pragma unroll
                                for (int t = 0; t < T; ++t) acc[m][t][i] = fmaf(x[t], value, acc[m][t][i]);
                            }
                    }
                }
                if (k + U * K_LANES < count) fetch_half(k0, count, k + U * K_LANES, half);
            }
        }
    }

    // four k-lanes of a warp: each step halves what a lane has to add, lane bit 3 and then bit 4 saying which half is its own
    constexpr int Q = T * 8 / 4;
    const bool hi0 = lane & 8, hi1 = lane & 16;
#pragma unroll
    for (int m = 0; m < M; ++m) {
        float* v = &acc[m][0][0];
        float half[T * 4];
#pragma unroll
        for (int j = 0; j < T * 4; ++j) {
            const float give = hi0 ? v[j] : v[j + T * 4], keep = hi0 ? v[j + T * 4] : v[j];
            half[j] = keep + __shfl_xor_sync(0xffffffffu, give, 8);
        }
#pragma unroll
        for (int j = 0; j < Q; ++j) {
            const float give = hi1 ? half[j] : half[j + Q], keep = hi1 ? half[j + Q] : half[j];
            part[warp][m][(hi0 ? T * 4 : 0) + (hi1 ? Q : 0) + j][group] = keep + __shfl_xor_sync(0xffffffffu, give, 16);
        }
    }
    __syncthreads();
    // A CTA of the cluster has COLUMNS / splits columns to finish; the parts of each are written into its shared memory.
    const int share = COLUMNS / a.splits;
    if (a.splits > 1) cluster_wait();
    for (int i = threadIdx.x; i < M * T * COLUMNS; i += THREADS) {
        const int m = i / (T * COLUMNS), t = i / COLUMNS % T, col = i % COLUMNS;
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) s += part[w][m][t * 8 + col % 8][col / 8];
        if (a.splits > 1) {
            const int owner = col / share;
            st_cluster(map_to_cta(smem_u32(&sums[m][t][(int)slice * share + col - owner * share]), (uint32_t)owner), s);
        } else {
            sums[m][t][col] = s;
        }
    }
    if (a.splits > 1) {  // after this nothing touches another CTA's memory
        cluster_arrive();
        cluster_wait();
    } else {
        __syncthreads();
    }
    for (int i = threadIdx.x; i < a.rows * share; i += THREADS) {
        const int t = i / share, own = i - t * share;
        const int64_t col = c0 + (int64_t)slice * share + own;
        if (col < a.N) {
            float s[M];
#pragma unroll
            for (int m = 0; m < M; ++m) {
                s[m] = 0.f;
                for (int r = 0; r < a.splits; ++r) s[m] += sums[m][t][r * share + own];
            }
            const int64_t at = (int64_t)t * a.N + col;
            if (GATED) {
                float g[1] = {s[0]}, u[1] = {s[M - 1]}, h[1];
                gated<F32>(a.gate, g, u, h);
                static_cast<float*>(a.out)[at] = h[0];
            } else if (F32) {
                static_cast<float*>(a.out)[at] = s[0];
            } else {
                static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(s[0]);
            }
        }
    }
}

template <typename... KArgs, typename... A>
cudaError_t launch_clusters(void (*kernel)(KArgs...), dim3 grid, int cluster, size_t smem, cudaStream_t s, int64_t* launches, A&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = cluster;
        attr[n].val.clusterDim.y = 1;
        attr[n].val.clusterDim.z = 1;
        ++n;
    }
    if (g_launch_pdl) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, std::forward<A>(args)...);
    if (e == cudaSuccess) count_launch(launches);
    return e;
}

template <bool F32, bool X32, bool GATED, int T>
cudaError_t launch_few(const FewArgs& a, bool vector, int64_t grid, cudaStream_t s, int64_t* launches) {
    const int chunk = a.k_per_slice < CHUNK ? a.k_per_slice : CHUNK;
    const size_t smem = (size_t)chunk * T * 4;
    auto* kernel = vector ? &few_rows_kernel<F32, X32, GATED, T, true> : &few_rows_kernel<F32, X32, GATED, T, false>;
    const cudaError_t e = smem_attr_once(reinterpret_cast<const void*>(kernel), CHUNK * T * 4);
    if (e != cudaSuccess) return e;
    return launch_clusters(kernel, dim3((unsigned)grid), a.splits, smem, s, launches, a);
}

template <bool F32, bool X32, bool GATED>
tfjsb_status few(tfjsb_ctx* ctx, const void* x, const void* w0, const void* w1, int gate, void* out, int64_t rows, int64_t N, int64_t K, cudaStream_t s) {
    FewArgs a = {x, w0, w1, out, N, (int)K, (int)rows, 0, 1, gate};
    // As many slices as give each SM two blocks at most and each thread at least 4 rows of weights.
    const int64_t blocks = (N + COLUMNS - 1) / COLUMNS;
    while (a.splits < 8 && blocks * a.splits * 2 <= 2 * ctx->sm_count && K / (a.splits * 2) >= 4 * K_LANES) a.splits *= 2;
    a.k_per_slice = (int)((K + a.splits - 1) / a.splits);
    const bool vector = N % 8 == 0;  // pointers are 16-byte aligned
    const int64_t grid = blocks * a.splits;
    if (grid >= (1LL << 31)) return fail(ctx, TFJSB_ERR_UNSUPPORTED, "too many columns");
    cudaError_t e;
    if (rows == 1) e = launch_few<F32, X32, GATED, 1>(a, vector, grid, s, &ctx->launches);
    else if (!F32 || rows == 2) e = launch_few<F32, X32, GATED, 2>(a, vector, grid, s, &ctx->launches);  // bfloat16: two rows at most
    else if (rows <= 4) e = launch_few<F32, X32, GATED, F32 ? 4 : 2>(a, vector, grid, s, &ctx->launches);
    else e = launch_few<F32, X32, GATED, F32 ? 8 : 2>(a, vector, grid, s, &ctx->launches);
    return e == cudaSuccess ? TFJSB_OK : cuda_fail(ctx, e, "few rows launch");
}

// ---- 8-bit weights -------------------------------------------------------------------------------------------

struct FewInt8Args {
    const void* x;         // QUANTIZE: rows of K values; otherwise [pitch] 8-bit
    const float* a_scale;  // not with QUANTIZE
    const int8_t* bt;      // [N, pitch]
    const float *b_scale, *bias;
    void* out;
    int64_t N;
    int K, pitch, act, out_bf16;
};

// A row of x for every blockIdx.y.  QUANTIZE: 0 x is 8-bit already (one row), 1 bfloat16, 2 fp32.
template <int QUANTIZE>
__global__ void __launch_bounds__(THREADS, 4) few_rows_int8_kernel(const __grid_constant__ FewInt8Args a) {
    extern __shared__ __align__(16) int8_t q[];  // [pitch]
    __shared__ float largest[WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_wait();
    pdl_launch_dependents();
    const uint32_t x_at = QUANTIZE == 0 ? 0u : blockIdx.y * (uint32_t)a.K;  // several rows are small layers'
    constexpr int U = 8;     // pieces of 512 bytes of a row of weights in flight a warp
    constexpr int HELD = 2;  // groups of eight values of x that a thread holds between the maximum and the rounding
    const int64_t step = (int64_t)gridDim.x * WARPS;
    int64_t n = (int64_t)blockIdx.x * WARPS + warp;
    uint4 w[U];
    auto fetch = [&](int64_t row, int k) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            w[u] = make_uint4(0u, 0u, 0u, 0u);
            if (row < a.N && k + u * 512 < a.pitch) w[u] = ld_weights(a.bt + row * a.pitch + k + u * 512);
        }
    };
    fetch(n, lane * 16);  // on its way while x is laid out

    float scale;
    if (QUANTIZE == 0) {
        for (int i = threadIdx.x * 16; i < a.pitch; i += THREADS * 16)
            *reinterpret_cast<uint4*>(q + i) = load_global(reinterpret_cast<const uint4*>(static_cast<const int8_t*>(a.x) + i));
        scale = load_global(a.a_scale);
    } else {
        auto left_at = [&](int k) { return a.K - k < 8 ? a.K - k : 8; };
        float v[HELD][8], m = 0.f;
#pragma unroll
        for (int j = 0; j < HELD; ++j) {
            const int k = (j * THREADS + threadIdx.x) * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[j][e] = 0.f;
            if (k < a.K) values8<QUANTIZE == 2>(a.x, (int64_t)(x_at + k), left_at(k), v[j]);
        }
#pragma unroll
        for (int j = 0; j < HELD; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) m = max_nan(m, fabsf(v[j][e]));
        for (int k = (HELD * THREADS + threadIdx.x) * 8; k < a.K; k += THREADS * 8) {
            float more[8];
            values8<QUANTIZE == 2>(a.x, (int64_t)(x_at + k), left_at(k), more);
#pragma unroll
            for (int e = 0; e < 8; ++e) m = max_nan(m, fabsf(more[e]));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (lane == 0) largest[warp] = m;
        __syncthreads();
        m = largest[0];
#pragma unroll
        for (int i = 1; i < WARPS; ++i) m = max_nan(m, largest[i]);
        const RowScale rs = row_scale(m);
        scale = m / 127.f;
#pragma unroll
        for (int j = 0; j < HELD; ++j) {
            const int k = (j * THREADS + threadIdx.x) * 8;
            if (k < a.pitch) *reinterpret_cast<uint2*>(q + k) = quantize8<QUANTIZE == 2>(v[j], rs);
        }
        for (int k = (HELD * THREADS + threadIdx.x) * 8; k < a.pitch; k += THREADS * 8) {
            float more[8] = {};
            if (k < a.K) values8<QUANTIZE == 2>(a.x, (int64_t)(x_at + k), left_at(k), more);
            *reinterpret_cast<uint2*>(q + k) = quantize8<QUANTIZE == 2>(more, rs);
        }
    }
    __syncthreads();

    for (; n < a.N; n += step) {
        int sum = 0;
        for (int k = lane * 16; k < a.pitch; k += U * 512) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (k + u * 512 < a.pitch) {
                    const int4 x = *reinterpret_cast<const int4*>(q + k + u * 512);
                    sum = __dp4a((int)w[u].x, x.x, sum);
                    sum = __dp4a((int)w[u].y, x.y, sum);
                    sum = __dp4a((int)w[u].z, x.z, sum);
                    sum = __dp4a((int)w[u].w, x.w, sum);
                }
            if (k + U * 512 < a.pitch) fetch(n, k + U * 512);  // the last pieces differ from lane to lane
        }
        __syncwarp();
        fetch(n + step, lane * 16);
        sum = __reduce_add_sync(0xffffffffu, sum);
        if (lane == 0) {
            // as the tensor-core product's epilogue does it, to the bit
            float v = fmaf((float)sum * scale, load_global(a.b_scale + n), a.bias ? load_global(a.bias + n) : 0.f);
            v = apply_act(v, a.act);
            const int64_t at = n + (QUANTIZE == 0 ? 0 : (int64_t)(blockIdx.y * (uint32_t)a.N));
            if (a.out_bf16) static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(v);
            else static_cast<float*>(a.out)[at] = v;
        }
    }
}

template <int QUANTIZE>
cudaError_t launch_int8(const FewInt8Args& a, int64_t rows, int sm_count, cudaStream_t s, int64_t* launches) {
    auto* kernel = &few_rows_int8_kernel<QUANTIZE>;
    const cudaError_t e = smem_attr_once(reinterpret_cast<const void*>(kernel), ROW_INT8_BYTES);
    if (e != cudaSuccess) return e;
    // a row of weights a warp; blocks of 64 registers a thread are four to an SM
    const int64_t needed = (a.N + WARPS - 1) / WARPS, most = rows < (int64_t)sm_count * 4 ? sm_count * 4 / rows : 1;
    return launch_clusters(kernel, dim3((unsigned)(needed < most ? needed : most), (unsigned)rows), 1, (size_t)a.pitch, s, launches, a);
}

}  // namespace

tfjsb_status few_rows_gated(tfjsb_ctx* ctx, bool f32, const void* x, const void* w_gate, const void* w_up, int gate, float* h, int64_t rows, int64_t N,
                            int64_t K, cudaStream_t s) {
    return f32 ? few<true, true, true>(ctx, x, w_gate, w_up, gate, h, rows, N, K, s) : few<false, false, true>(ctx, x, w_gate, w_up, gate, h, rows, N, K, s);
}
tfjsb_status few_rows_down(tfjsb_ctx* ctx, bool f32, const float* h, const void* w, void* y, int64_t rows, int64_t N, int64_t K, cudaStream_t s) {
    return f32 ? few<true, true, false>(ctx, h, w, nullptr, 0, y, rows, N, K, s) : few<false, true, false>(ctx, h, w, nullptr, 0, y, rows, N, K, s);
}

tfjsb_status rows_int8(tfjsb_ctx* ctx, int x_kind, const void* x, const float* a_scale, const int8_t* bt, const float* b_scale, const float* bias, int act,
                      void* out, bool out_bf16, int64_t M, int64_t N, int64_t K, cudaStream_t s) {
    const FewInt8Args a = {x, a_scale, bt, b_scale, bias, out, N, (int)K, (int)((K + 15) / 16 * 16), act, out_bf16 ? 1 : 0};
    const cudaError_t e = x_kind == 0   ? launch_int8<0>(a, M, ctx->sm_count, s, &ctx->launches)
                          : x_kind == 1 ? launch_int8<1>(a, M, ctx->sm_count, s, &ctx->launches)
                                        : launch_int8<2>(a, M, ctx->sm_count, s, &ctx->launches);
    return e == cudaSuccess ? TFJSB_OK : cuda_fail(ctx, e, "8-bit rows launch");
}

}  // namespace dense
}  // namespace tfjsb
