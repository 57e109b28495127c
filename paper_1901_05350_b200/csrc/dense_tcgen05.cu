// Tensor-core products of the dense layers of transformer blocks: bfloat16 operands (tcgen05 kind::f16), fp32 operands as three
// bfloat16 planes each, or 8-bit integers (kind::i8), with the layers' own epilogues.
//
//     sum[M,N] = sum over passes p and k of  A_p[M,K] B_p[K,N]
//
// Operands are read as they are stored: with K contiguous (128-byte-swizzled rows of 128 bytes) or with rows or columns
// contiguous (boxes of 64 k x 64 columns in the same swizzle).  A k-block is 128 bytes of K: 64 bfloat16 or 128 8-bit values,
// four MMAs.  The gated block's two projections are ONE product: half of a tile's columns come from Wg and half from Wu, so that g and u of
// an element are in the same tensor-memory lane and h = gate(g) u needs no exchange; in a CTA pair each CTA fetches the
// columns of one of them.  The gradient of x is one product too, over dg Wg^T and then du Wu^T in the same accumulator, and the
// gradients of Wg and Wu are one launch over the tiles of both.
//
// Structure (CTA pairs, CG = 2, as in gemm_pair.cu; single CTAs, CG = 1, without the cluster): warp 0 copies A and warp 18 B (TMA), warp
// 1 issues the MMAs, warps 2-17 are the epilogue, which works on one accumulator stage while the next tile is summed in the
// other.  Stored results leave through shared memory (TMA), h and the gradients of g and u from registers, 32 bytes of a row a thread, so that
// every sector is written once and whole; g and u are in blocks of 32 rows x 8 columns, which a warp moves in one piece.
//
// What bounds it: at large sizes what an SM can fetch from L2 (50 to 60 bytes a cycle), so the widest tile is 512 x 256 for a CTA pair, two parts
// of 256 rows that share B (SUBS = 2): h Wd of 8192 x 4096 x 16384 took 1.62-1.64 PFLOP/s in a burst, with 256 x 256 tiles 1.35.  Epilogues
// with more to do take their share: x Wg and x Wu, whose gates and copies of g and u hold up the next tile, 1.45-1.48 (tensor pipe 72 % active),
// the gradients of g and u, which read 8 bytes an element and have tiles of one part, 1.28 (64 %).  At small sizes
// latency: a launch, the first copies (2 us) and the epilogue.
// Persistent over tiles in bands of `band` tile rows, so that the tiles in flight share operand rows and columns in L2.
//
// Few tiles: K is cut among the CTAs of a cluster (CG = 1, one tile each).  Each has a share of the tile's columns to finish and gets the
// other slices' sums of them written into its shared memory, which it adds, after a cluster barrier, in the order of the slices: no
// atomics, results do not depend on scheduling.  (Sums left where they are made and read from there cost a round trip more: 64 x 512 x 2048 on
// eight slices 10.2 us, now 7.3.  Blocks of half the registers and shared memory, so that the next kernel's could begin
// beside them, made 1000 x 1024 x 2730 in training 120 us instead of 106: blocks come to lie two on an SM beside empty ones.)
//
// fp32: v = p0 + p1 + p2 (bfloat16, rounded to nearest each, exact), a b = p0 q0 + (p0 q1 + p1 q0 + p1 q1 + p0 q2 + p2 q0), what is left out is
// below 2^-26 of it.  The tensor core cuts every sum towards zero, so the error of an accumulator grows with the number of
// additions: the large products go to an accumulator of their own for `seg_kb` k-blocks only (8 additions), the small ones
// to another, and the epilogue adds both to fp32 sums in registers, rounded to nearest.
#include <atomic>
#include <cstdio>
#include <cstdlib>

#include <cuda_bf16.h>

#include "dense.cuh"
#include "dense_math.cuh"
#include "ptx_sm100.cuh"
#include "umma_tile.cuh"

namespace tfjsb {
namespace dense {

using namespace ptx;
using tile::give_up;
using tile::drain;

namespace {

constexpr int EPI_WARPS = 16;  // four for each quadrant of tensor-memory lanes
constexpr int B_WARP = 2 + EPI_WARPS;
constexpr int THREADS = 32 * (B_WARP + 1);  // producer warp of A, MMA warp, epilogue warps, producer warp of B
constexpr int MAX_STAGES = 8;
constexpr int STAGES_AT_LEAST = 192 * 1024;  // bytes of all stages, whatever a tile's columns and planes
constexpr int ROWS = 128;     // of a CTA's tile
constexpr int A_BYTES = ROWS * 128;
constexpr int GROUP_BYTES = 64 * 128;  // a box of 64 k x 64 columns

// Operand tile whose memory runs along M or N: descriptor of boxes of 64 columns x 64 k in the 128-byte swizzle.  Eight k are
// 1024 bytes (stride byte offset), groups of 64 columns 8192 bytes apart (leading byte offset); an MMA's 16 k are 2048 bytes.
__device__ __forceinline__ uint64_t mn_desc(uint32_t addr) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(GROUP_BYTES >> 4) << 16) | ((uint64_t)(1024u >> 4) << 32) | (1ull << 46) |
           (2ull << 61);
}

// Descriptors come as their lower words, which change from MMA to MMA, and their upper words, which do not: 32-bit additions on the
// uniform datapath are most of what a k-block costs the issuing warp.
#define TFJSB_DENSE_MMA(FORM)                                                                                                      \
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tmov.b64 a, {%1, %2};\n\tmov.b64 b, {%3, %4};\n\tsetp.ne.b32 p, %6, 0;\n\t"     \
                 "tcgen05.mma." FORM " [%0], a, b, %5, p;\n\t}" ::"r"(d), "r"(a), "r"(a_hi), "r"(b), "r"(b_hi), "r"(idesc), "r"(accumulate) \
                 : "memory")
template <int CG, int KIND>
__device__ __forceinline__ void mma(uint32_t d, uint32_t a, uint32_t a_hi, uint32_t b, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
    if (KIND == KIND_BF16) {
        if (CG == 2) TFJSB_DENSE_MMA("cta_group::2.kind::f16");
        else TFJSB_DENSE_MMA("cta_group::1.kind::f16");
    } else {
        if (CG == 2) TFJSB_DENSE_MMA("cta_group::2.kind::i8");
        else TFJSB_DENSE_MMA("cta_group::1.kind::i8");
    }
}
#undef TFJSB_DENSE_MMA
template <int CG>
__device__ __forceinline__ void commit(uint32_t bar) {  // to this CTA, or to the same barrier of both
    if (CG == 2) tc_commit_pair(bar, (uint16_t)3);
    else tc_commit(bar);
}
// Copy whose bytes are counted on `bar`: of this CTA, or (CG = 2) a shared::cluster address of the even one.
template <int CG>
__device__ __forceinline__ void load3(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2) {
    if (CG == 2)
        asm volatile(
            "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
            "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
    else tma_load_3d(dst, map, bar, c0, c1, c2);
}

// Arrival on the even CTA's barrier that orders no memory: what it hands back is tensor memory, whose reads are complete.  One that releases
// waits for the stores before it, which took 900 cycles.
__device__ __forceinline__ void arrive_relaxed(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ void sts16_cluster(uint32_t at, const uint32_t* v) {
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}

// bounded_wait with more than one limit after the other, where the time may be somebody else's.
//   A role that begins before the kernel before has ended (its operands are not that kernel's, or it waits for a role that does wait for
//   that kernel) may spend a limit on it: few tiles with an enormous K keep a handful of SMs busy while the others are this kernel's
//   already.  So that kernel is waited for, and then the limit is this kernel's own.
//   An epilogue, which has been through that wait, waits for all of a tile's k-blocks: it has a limit for each 65536 of them (of 250 ns each where K is
//   cut eight ways and a tile is small: 2^30 terms take 0.52 s).
// One function and no calls from it: calls of bounded_wait_slow, or of a second function after it, made short products 1 to 2 % slower.
__device__ __noinline__ bool patient_wait_slow(uint32_t bar, uint32_t parity, volatile int* abort_flag, int limits) {
#pragma unroll 1
    for (;;) {
        const unsigned long long t0 = global_ns();
#pragma unroll 1
        for (uint32_t it = 1; it < (1u << 26); ++it) {
            if (mbar_try_wait(bar, parity)) return true;
            if (*abort_flag) return false;
            if ((it & 63u) == 0u && global_ns() - t0 > WAIT_LIMIT_NS) break;
        }
        if (--limits <= 0) return false;
        pdl_wait();
    }
}
__device__ __forceinline__ bool patient_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, int limits = 2) {
    return mbar_try_wait(bar, parity) || patient_wait_slow(bar, parity, abort_flag, limits);
}

__device__ __forceinline__ uint4 lds4u(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}

__device__ __forceinline__ void ld_columns(uint32_t at, uint32_t (&r)[16]) { tc_ld_cols(at, r); }
__device__ __forceinline__ void ld_columns(uint32_t at, uint32_t (&r)[8]) { tc_ld_cols(at, r); }

// Where the slices of a tile (few tiles, K cut among the CTAs of a cluster) put their sums: the tile's columns are shared out among the CTAs, and
// each has room for its share of every slice's rows, in rows of `pitch` values; a gated tile's for g and then for u.
struct Share {
    int columns, pitch, rows, planes;  // of a CTA's share; the last CTAs' may be smaller, or nothing
    __host__ __device__ Share(int block_n, int splits, int M, bool gated) {
        planes = gated ? 2 : 1;
        columns = (block_n / planes / 8 + splits - 1) / splits * 8;
        pitch = columns + 4;  // consecutive rows start in other banks
        rows = M < ROWS ? M : ROWS;
    }
    __host__ __device__ int at(int slice, int plane, int row) const { return ((slice * planes + plane) * rows + row) * pitch; }
    __host__ __device__ int bytes(int slices) const { return at(slices, 0, 0) * 4; }
};
// The sum of eight columns, added in the order of the slices, `step` bytes apart.
template <int KIND>
__device__ __forceinline__ void sum_parts(uint32_t at, uint32_t step, int splits, uint32_t (&sum)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0u;
#pragma unroll 4
    for (int r = 0; r < splits; ++r) {
        add_part<KIND>(sum, 0, lds4u(at + (uint32_t)r * step));
        add_part<KIND>(sum, 4, lds4u(at + (uint32_t)r * step + 16u));
    }
}

struct Maps {
    CUtensorMap a, b[2];
    CUtensorMap out[2];  // results that are stored from shared memory
};

// Shared memory of an epilogue warp: a chunk of 32 rows of a result on its way out, rows of 64 bytes, or g and u of 32 rows and 16
// columns on their way in.
template <int P, int EPI> constexpr int SLAB_BYTES = P == 3 || EPI == EPI_GATED ? 0 : EPI == EPI_GRAD ? 4096 : 2048;

// 16-byte piece j of row r of a chunk whose rows are B bytes, in the swizzle of B bytes.
template <int B>
__device__ __forceinline__ uint32_t piece(int r, int j) {
    return (uint32_t)(r * B + ((j ^ (B == 32 ? r >> 2 & 1 : B == 64 ? r >> 1 & 3 : r & 7)) << 4));
}
__device__ __forceinline__ void sts16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// Where eight values of g (plane 0) or u of row `row` from column `col` on, a multiple of eight, are in z.  Neighbouring rows' eights are
// neighbours, in blocks of 32 rows, so that a warp whose lanes have a row each reads or writes 1 KiB in one piece.
__device__ __forceinline__ float* z_at(const Args& a, int64_t row, int col, int plane) {
    return a.z + (((row >> 5) * (a.z_pitch >> 3) + (col >> 3)) * 2 + plane) * 256 + (row & 31) * 8;
}

// Tile number -> (tile row, tile column), in bands of `band` tile rows, down a band's columns one after the other.
__device__ __forceinline__ void tile_at(const Args& a, int tile, int* m, int* n) {
    const int columns = a.n_tiles * a.outputs;
    const int per_band = a.band * columns;
    const int b = tile / per_band, in = tile - b * per_band;
    const int rows = min(a.band, a.m_tiles - b * a.band);
    *n = in / rows;
    *m = b * a.band + in - *n * rows;
}

// A work item: a tile, and the first and the number of its 256-row parts (SUBS = 2).
struct Item {
    int tm, tn, sub, subs;
};
template <int SUBS>
__device__ __forceinline__ Item item_at(const Args& a, int item) {
    Item it;
    if (SUBS == 1) {
        tile_at(a, item, &it.tm, &it.tn);
        it.sub = 0;
        it.subs = 1;
        return it;
    }
    const bool whole = item < a.whole_tiles;
    tile_at(a, whole ? item : a.whole_tiles + ((item - a.whole_tiles) >> 1), &it.tm, &it.tn);
    it.sub = whole ? 0 : (item - a.whole_tiles) & 1;
    it.subs = whole && (int64_t)it.tm * (2 * SUBS * ROWS) + 2 * ROWS < a.M ? 2 : 1;
    return it;
}

// Eight of W values.
template <int W>
__device__ __forceinline__ float (&eight(float (&v)[W], int j))[8] {
    return reinterpret_cast<float(&)[8]>(v[j]);
}

// ---- what becomes of W sums of a row -------------------------------------------------------------------
// act(sum a_scale b_scale + bias); bias is 0 where there is none
template <int W>
__device__ __forceinline__ void scaled(const Args& a, float row_scale, const uint32_t (&sum)[W], const float (&scale)[W], const float (&bias)[W],
                                       float (&v)[W]) {
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = fmaf((float)(int)sum[i] * row_scale, scale[i], bias[i]);
    if (a.act == TFJSB_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = relu_nan(v[i]);
    } else if (a.act == TFJSB_ACT_RELU6) {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = relu6_nan(v[i]);
    }
}

// Sixteen columns of a warp's 32 rows of an fp32 result, a lane's row each, where rows begin anywhere: a store of one value a lane would touch 32
// rows, so the 16 x 16 values of each half warp change places first (lane and index swap, one bit at a time) and a lane has a column, row after
// row.  515 x 512 x 1365, gradients of g's and u's weights: 16.4 us, with stores along rows 22.5.
__device__ __forceinline__ void store_across(float* out, int64_t pitch, int64_t row0, int64_t rows, int col, int columns, uint32_t (&v)[16]) {
    const int lane = threadIdx.x & 31, c = lane & 15;
#pragma unroll
    for (int b = 8; b > 0; b >>= 1) {
        const bool up = lane & b;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (i & b) continue;
            const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? v[i] : v[i + b], b);
            if (up) v[i] = got;
            else v[i + b] = got;
        }
    }
    if (col + c >= columns) return;
    const int64_t first = row0 + (lane & 16);
    float* to = out + first * pitch + col + c;
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (first + i < rows) to[i * pitch] = __uint_as_float(v[i]);
}

// `first` and, for EPI_GATED, `second` are the sums (g and u) of columns col .. col + W - 1 of row `row`; W is 8 or 16.
template <int P, int EPI, int W>
__device__ __forceinline__ void finish(const Args& a, int which, int64_t row, int col, const uint32_t (&first)[W], const uint32_t (&second)[W]) {
    const int left = a.N - col;  // columns that exist
    if (row >= a.M || left <= 0) return;
    float v[W];
    if constexpr (EPI == EPI_STORE) {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = __uint_as_float(first[i]);
        if constexpr (P == 1) store_bf16(static_cast<__nv_bfloat16*>(a.out[which]) + row * a.out_pitch + col, v, left);
        else store_f32(static_cast<float*>(a.out[which]) + row * a.out_pitch + col, v, left);
    } else if constexpr (EPI == EPI_SCALE) {
        float scale[W], bias[W];
        load_f32(a.b_scale + col, scale, left);
        load_f32(a.bias + col, bias, a.bias ? left : 0);
        scaled(a, load_global(a.a_scale + row), first, scale, bias, v);
        if (a.out_bf16) store_bf16(static_cast<__nv_bfloat16*>(a.out[0]) + row * a.out_pitch + col, v, left);
        else store_f32(static_cast<float*>(a.out[0]) + row * a.out_pitch + col, v, left);
    } else if constexpr (EPI == EPI_GATED) {
        float g[W], u[W];
#pragma unroll
        for (int i = 0; i < W; ++i) { g[i] = __uint_as_float(first[i]); u[i] = __uint_as_float(second[i]); }
        if (a.z) {
#pragma unroll
            for (int j = 0; j < W; j += 8) {
                if (j >= left) break;
                store_f32(z_at(a, row, col + j, 0), eight(g, j), 8);
                store_f32(z_at(a, row, col + j, 1), eight(u, j), 8);
            }
        }
        gated<P == 3>(a.gate, g, u, v);
        store_planes<P>(static_cast<__nv_bfloat16*>(a.out[0]) + row * a.out_pitch + col, a.out_plane, v, left);
    } else {
        float g[W], u[W];
#pragma unroll
        for (int j = 0; j < W; j += 8) {
            if (j >= left) break;
            load_f32(z_at(a, row, col + j, 0), eight(g, j), 8);
            load_f32(z_at(a, row, col + j, 1), eight(u, j), 8);
        }
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = __uint_as_float(first[i]);
        float du[W];
        gated_gradient<P == 3>(a.gate, g, u, v, du);  // v: dh -> dg
        __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(a.out[0]) + row * a.out_pitch + col;
        store_planes<P>(dst, a.out_plane, v, left);
        store_planes<P>(dst + P * a.out_plane, a.out_plane, du, left);
    }
}

template <int CG, int P, int KIND, int EPI, int SUBS, bool A_MN, bool B_MN>
__global__ void __launch_bounds__(THREADS, 1)
dense_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Args args) {
    const CUtensorMap &map_a = maps.a, &map_b0 = maps.b[0], &map_b1 = maps.b[1];
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bar_full[MAX_STAGES];  // CG = 2: used in the even CTA only
    __shared__ __align__(8) uint64_t bar_empty[MAX_STAGES];
    __shared__ __align__(8) uint64_t bar_acc_full[2];
    __shared__ __align__(8) uint64_t bar_acc_empty[2];      // CG = 2: used in the even CTA only
    __shared__ __align__(8) uint64_t bar_drain;
    constexpr int SLAB = SLAB_BYTES<P, EPI>;
    __shared__ __align__(8) uint64_t bar_z[EPI == EPI_GRAD && P == 1 ? EPI_WARPS : 1];
    __shared__ uint32_t tmem_base_slot;
    __shared__ int abort_flag_s;

    volatile int* abort_flag = &abort_flag_s;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? cluster_ctarank() : 0u;
    const uint32_t slice = CG == 1 && args.splits > 1 ? cluster_ctarank() : 0u;
    const bool leader = rank == 0;
    const int block_n = args.block_n, stages = args.stages;
    const int own_n = block_n / CG;  // columns of B that this CTA fetches
    const uint32_t a_plane = A_BYTES, b_plane = (uint32_t)own_n * 128u;
    constexpr int TILE_M = CG * ROWS * SUBS;
    const uint32_t stage_bytes = SUBS * P * a_plane + P * b_plane;
    const uint32_t a_tx = CG * P * (uint32_t)args.a_rows * 128u, b_tx = CG * P * b_plane;
    const int first_tile = args.splits > 1 ? (int)blockIdx.x / args.splits : (int)blockIdx.x / CG;
    const int tile_step = args.splits > 1 ? args.num_tiles : (int)gridDim.x / CG;  // a slice has one tile
    const int kb_total = args.passes * args.num_kb;
    const int kb_begin = (int)slice * args.kb_per_split;
    const int kb_end = args.splits > 1 ? min(kb_total, kb_begin + args.kb_per_split) : kb_total;
    constexpr int BK = KIND == KIND_BF16 ? 64 : 128;
    const uint32_t acc_cols = (uint32_t)block_n * (P == 3 ? 2u : 1u);  // of an accumulator stage: large | small
    const uint32_t stage_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t parts_base = stage_base + (args.parts_apart ? (uint32_t)stages * stage_bytes : 0u);  // see Share

    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) {
            mbar_init(smem_u32(&bar_full[s]), 1);
            mbar_init(smem_u32(&bar_empty[s]), 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(smem_u32(&bar_acc_full[s]), 1);
            mbar_init(smem_u32(&bar_acc_empty[s]), EPI_WARPS * CG);
        }
        mbar_init(smem_u32(&bar_drain), 1);
        if (EPI == EPI_GRAD && P == 1)
            for (int i = 0; i < EPI_WARPS; ++i) mbar_init(smem_u32(&bar_z[i]), 1);
        abort_flag_s = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_b0) : "memory");
    }
    constexpr uint32_t TMEM_COLS = 512;
    if (warp == 1) {
        if (CG == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_slot)), "r"(TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_slot)), "r"(TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    if (CG == 2) {  // the partner's barriers must be initialised before anything of this CTA can signal them
        cluster_arrive();
        cluster_wait();
    }
    tc_fence_after();
    if (CG == 1 && args.splits > 1 && args.parts_apart)  // "has begun": others may put their sums here
        asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
    const uint32_t tmem_base = tmem_base_slot;
    // Each role waits for the kernel before on its own: the producers only where that kernel may still write what they read (args.early_*), the
    // epilogue always, before it reads or writes anything, and the next kernel is let go after that wait.  So when a kernel of a chain
    // starts, everything but the kernel right before it is complete: it may read what the one before that wrote, and as SMs run out of tiles
    // of one product they sum those of the next.

    if (warp == 0 || warp == B_WARP) {
        // ---------------------------------------------------------------- producers: of A (which arms the barriers) and of B
        // One thread issues a copy in 150 to 250 cycles, so the two operands have a warp each, and everything that an issue takes is
        // worked out by the whole warp outside the branch (see elect_one).
        const bool is_a = warp == 0;
        if (!(is_a ? args.early_a : args.early_b)) pdl_wait();
        int stage = 0;
        uint32_t phase = 0;
        int issued = 0;
        const bool elected = elect_one();
        bool ok = true;  // the elected thread's
        constexpr int A_GROUPS = A_MN ? ROWS / 64 : 1, A_COPIES = SUBS * P * A_GROUPS;
        constexpr int B_MATS = EPI == EPI_GATED && CG == 1 ? 2 : 1, B_GROUPS = B_MN ? 4 / B_MATS / CG : 1, B_COPIES = P * B_MATS * B_GROUPS;
        const int mat_n = own_n / B_MATS, groups = B_MN ? mat_n / 64 : 1;
        const uint32_t full_0 = smem_u32(&bar_full[0]), empty_0 = smem_u32(&bar_empty[0]), full_leader = CG == 2 ? map_to_cta(full_0, 0u) : full_0;
        const uint32_t dst_0 = stage_base + (is_a ? 0u : SUBS * P * a_plane);
        uint32_t dst = dst_0;
        bool ready = false;  // the elected thread's: the stage was seen free while the one before was filled
        for (int tile = first_tile; tile < args.num_tiles; tile += tile_step) {
            const Item it = item_at<SUBS>(args, tile);
            const int tn = it.tn;
            const int which = EPI == EPI_STORE && tn >= args.n_tiles ? 1 : 0;
            const int m0 = it.tm * TILE_M + it.sub * (CG * ROWS) + (int)rank * ROWS;
            const int n0 = EPI == EPI_GATED ? tn * (block_n >> 1) : (tn - which * args.n_tiles) * block_n + (int)rank * own_n;
            const uint32_t tx = (uint32_t)it.subs * a_tx + b_tx;
            int pass = kb_begin >= args.num_kb ? 1 : 0, k0 = (kb_begin - pass * args.num_kb) * BK;
            for (int kb = kb_begin; kb < kb_end; ++kb) {
                const uint32_t own_full = full_0 + 8u * stage, empty = empty_0 + 8u * stage, full = full_leader + 8u * stage;
                const int next = stage + 1 == stages ? 0 : stage + 1;
                const uint32_t next_empty = empty_0 + 8u * next, next_phase = phase ^ (next == 0 ? 1u : 0u);
                if (is_a) {
                    uint32_t to[A_COPIES];
                    int c0[A_COPIES], c1[A_COPIES], c2[A_COPIES];
#pragma unroll
                    for (int i = 0; i < A_COPIES; ++i) {
                        const int g = i % A_GROUPS, u = i / A_GROUPS % SUBS, p = i / A_GROUPS / SUBS;
                        const int row = m0 + u * (CG * ROWS) + 64 * g;
                        to[i] = dst + (uint32_t)((p * SUBS + u) * A_BYTES + g * GROUP_BYTES);
                        c0[i] = A_MN ? row : k0;
                        c1[i] = A_MN ? k0 : row;
                        c2[i] = pass * P + p;
                    }
                    if (elected && ok && (ready || (ok = patient_wait(empty, phase ^ 1u, abort_flag)))) {
                        ready = mbar_test_wait(next_empty, next_phase ^ 1u);
                        if (leader) mbar_arrive_expect_tx(own_full, tx);
#pragma unroll
                        for (int i = 0; i < A_COPIES; ++i)
                            if (SUBS == 1 || i / A_GROUPS % SUBS < it.subs) load3<CG>(to[i], &map_a, full, c0[i], c1[i], c2[i]);
                        ++issued;
                    }
                } else {
                    // the weights of this half of the columns, of this pass, or one and the same
                    const CUtensorMap* map_b = (EPI == EPI_GATED ? (CG == 2 && rank == 1) : pass == 1) ? &map_b1 : &map_b0;
                    uint32_t to[B_COPIES];
                    int c0[B_COPIES], c1[B_COPIES], c2[B_COPIES];
#pragma unroll
                    for (int i = 0; i < B_COPIES; ++i) {
                        const int g = i % B_GROUPS, w = i / B_GROUPS % B_MATS, p = i / B_GROUPS / B_MATS;
                        const int row = n0 + 64 * g;
                        to[i] = dst + (uint32_t)p * b_plane + (uint32_t)(w * mat_n) * 128u + (uint32_t)g * GROUP_BYTES;
                        c0[i] = B_MN ? row : k0;
                        c1[i] = B_MN ? k0 : row;
                        c2[i] = which * P + p;
                    }
                    if (elected && ok && (ready || (ok = patient_wait(empty, phase ^ 1u, abort_flag)))) {
                        ready = mbar_test_wait(next_empty, next_phase ^ 1u);
#pragma unroll
                        for (int i = 0; i < B_COPIES; ++i)
                            if (i % B_GROUPS < groups) load3<CG>(to[i], B_MATS == 2 && i / B_GROUPS % B_MATS ? &map_b1 : map_b, full, c0[i], c1[i], c2[i]);
                        ++issued;
                    }
                }
                stage = next;
                phase = next_phase;
                dst = next == 0 ? dst_0 : dst + stage_bytes;
                k0 += BK;
                if (kb + 1 == args.num_kb) { pass = 1; k0 = 0; }
            }
        }
        if (!ok) {
            give_up(abort_flag, args.dev_status, DEV_STATUS_TIMEOUT_PRODUCER);
            // copies in flight must land before this CTA's shared memory goes away; the odd CTA of a pair has no barrier of
            // its own to watch and waits out the longest that a copy can take
            if (leader && is_a) {
                for (int k = (issued > stages ? issued - stages : 0); k < issued; ++k)
                    drain(smem_u32(&bar_full[k % stages]), (uint32_t)((k / stages) & 1), args.dev_status);
            } else {
                const unsigned long long t0 = global_ns();
                while (global_ns() - t0 < 2000000ull) {}  // 2 ms
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---------------------------------------------------------------- MMA issuer (the even CTA's)
        if (leader) {
            const uint32_t formats = KIND == KIND_BF16 ? (1u << 4) | (1u << 7) | (1u << 10)   // fp32 sums of bfloat16
                                                       : (2u << 4) | (1u << 7) | (1u << 10);  // 32-bit sums of signed 8-bit
            const uint32_t idesc = formats | ((uint32_t)(block_n >> 3) << 17) | ((uint32_t)(CG * ROWS >> 4) << 24) |
                                   (A_MN ? IDESC_A_MN : 0u) | (B_MN ? IDESC_B_MN : 0u);
            constexpr uint32_t a_step = A_MN ? 128 : 2, b_step = B_MN ? 128 : 2;  // of an MMA along K, in 16 bytes
            const uint64_t a_desc = A_MN ? mn_desc(stage_base) : make_kmajor_sw128_desc(stage_base);
            const uint64_t b_desc = B_MN ? mn_desc(stage_base + SUBS * P * a_plane) : make_kmajor_sw128_desc(stage_base + SUBS * P * a_plane);
            const uint32_t a_hi = (uint32_t)(a_desc >> 32), b_hi = (uint32_t)(b_desc >> 32), a_0 = (uint32_t)a_desc, b_0 = (uint32_t)b_desc;
            const uint32_t stage_step = stage_bytes >> 4;
            const uint32_t full_0 = smem_u32(&bar_full[0]), empty_0 = smem_u32(&bar_empty[0]), acc_full_0 = smem_u32(&bar_acc_full[0]), acc_empty_0 = smem_u32(&bar_acc_empty[0]);
            int stage = 0;
            uint32_t phase = 0;
            uint32_t offset = 0;  // of the stage, in 16 bytes
            const bool elected = elect_one();
            bool ok = true, issued_any = false, ready = false;  // the elected thread's; ready: the stage was seen filled
            auto advance = [&]() {
                const bool wrap = stage + 1 == stages;
                stage = wrap ? 0 : stage + 1;
                phase ^= wrap ? 1u : 0u;
                offset = wrap ? 0u : offset + stage_step;
            };
            if constexpr (SUBS == 2) {
                // Both parts of a tile use each stage.  At its beginning and its end a part's MMAs of LEAD k-blocks go one after
                // the other: the first part is complete, and read by the epilogue, while the second is still summed, and the
                // next tile begins in the first part's columns while the second part's are read.
                constexpr int LEAD = 2;
                uint32_t part_phase[2] = {0u, 0u};
                for (int tile = first_tile; tile < args.num_tiles; tile += tile_step) {
                    const int subs = item_at<SUBS>(args, tile).subs;
                    for (int kb = kb_begin; kb < kb_end;) {
                        // k-blocks of one part in a row
                        const int run = kb == kb_begin || kb_end - kb <= LEAD ? min(LEAD, kb_end - kb) : 1;
                        const int stage_was = stage;
                        const uint32_t phase_was = phase, offset_was = offset;
#pragma unroll
                        for (int part = 0; part < 2; ++part) {
                            if (part >= subs) break;
                            if (kb == kb_begin) {
                                if (elected && ok) ok = patient_wait(acc_empty_0 + 8u * part, part_phase[part] ^ 1u, abort_flag);
                                part_phase[part] ^= 1u;
                                tc_fence_after();
                            }
                            stage = stage_was;
                            phase = phase_was;
                            offset = offset_was;
                            const uint32_t d = tmem_base + (uint32_t)part * acc_cols;
                            for (int j = 0; j < run; ++j) {
                                const uint32_t a0 = a_0 + offset + (uint32_t)(part * (A_BYTES >> 4)), b0 = b_0 + offset, full = full_0 + 8u * stage, empty = empty_0 + 8u * stage;
                                const uint32_t a1 = a0 + a_step, a2 = a0 + 2 * a_step, a3 = a0 + 3 * a_step, b1 = b0 + b_step, b2 = b0 + 2 * b_step, b3 = b0 + 3 * b_step;
                                const uint32_t begun = kb + j == kb_begin ? 0u : 1u;
                                const bool last = part + 1 == subs;
                                advance();
                                const uint32_t next_full = full_0 + 8u * stage, next_phase = phase, this_phase = phase ^ (stage == 0 ? 1u : 0u);
                                if (elected && ok && (part > 0 || ready || (ok = patient_wait(full, this_phase, abort_flag)))) {
                                    if (part == 0) tc_fence_after();
                                    ready = mbar_test_wait(next_full, next_phase);
                                    mma<CG, KIND>(d, a0, a_hi, b0, b_hi, idesc, begun);
                                    mma<CG, KIND>(d, a1, a_hi, b1, b_hi, idesc, 1u);
                                    mma<CG, KIND>(d, a2, a_hi, b2, b_hi, idesc, 1u);
                                    mma<CG, KIND>(d, a3, a_hi, b3, b_hi, idesc, 1u);
                                    if (last) commit<CG>(empty);
                                    issued_any = true;
                                }
                            }
                            if (kb + run == kb_end && elected && ok) commit<CG>(acc_full_0 + 8u * part);
                        }
                        kb += run;
                    }
                }
            } else {
                int acc = 0;
                uint32_t acc_phase = 0;
                for (int tile = first_tile; tile < args.num_tiles; tile += tile_step) {
                    int in_segment = 0;
                    for (int kb = kb_begin; kb < kb_end; ++kb) {
                        if (in_segment == 0 && elected && ok) {
                            ok = patient_wait(acc_empty_0 + 8u * acc, acc_phase ^ 1u, abort_flag);
                            tc_fence_after();
                        }
                        const uint32_t d = tmem_base + (uint32_t)acc * acc_cols, small = d + (uint32_t)block_n;
                        uint32_t a[P][4], b[P][4];
#pragma unroll
                        for (int p = 0; p < P; ++p)
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                a[p][k] = a_0 + offset + (uint32_t)(p * (A_BYTES >> 4)) + a_step * k;
                                b[p][k] = b_0 + offset + (uint32_t)p * (b_plane >> 4) + b_step * k;
                            }
                        const uint32_t begun = in_segment != 0 ? 1u : 0u, full = full_0 + 8u * stage, empty = empty_0 + 8u * stage;
                        advance();
                        const uint32_t next_full = full_0 + 8u * stage, next_phase = phase, this_phase = phase ^ (stage == 0 ? 1u : 0u);
                        if (elected && ok && (ready || (ok = patient_wait(full, this_phase, abort_flag)))) {
                            tc_fence_after();
                            ready = mbar_test_wait(next_full, next_phase);
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const uint32_t more = k == 0 ? begun : 1u;
                                mma<CG, KIND>(d, a[0][k], a_hi, b[0][k], b_hi, idesc, more);
                                if constexpr (P == 3) {
                                    mma<CG, KIND>(small, a[2][k], a_hi, b[0][k], b_hi, idesc, more);
                                    mma<CG, KIND>(small, a[0][k], a_hi, b[2][k], b_hi, idesc, 1u);
                                    mma<CG, KIND>(small, a[1][k], a_hi, b[1][k], b_hi, idesc, 1u);
                                    mma<CG, KIND>(small, a[1][k], a_hi, b[0][k], b_hi, idesc, 1u);
                                    mma<CG, KIND>(small, a[0][k], a_hi, b[1][k], b_hi, idesc, 1u);
                                }
                            }
                            commit<CG>(empty);
                            issued_any = true;
                        }
                        ++in_segment;
                        if (kb + 1 == kb_end || (P == 3 && in_segment == args.seg_kb)) {
                            if (elected && ok) commit<CG>(acc_full_0 + 8u * acc);
                            if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
                            in_segment = 0;
                        }
                    }
                }
            }
            if (!ok) {
                give_up(abort_flag, args.dev_status, DEV_STATUS_TIMEOUT_MMA);
                if (issued_any) {  // let the MMAs already issued finish before tensor memory is released
                    if (CG == 2) tc_commit_pair(smem_u32(&bar_drain), (uint16_t)1);
                    else tc_commit(smem_u32(&bar_drain));
                    drain(smem_u32(&bar_drain), 0u, args.dev_status);
                }
            }
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- epilogue (warps 2..17)
        // The four warps of a quadrant of tensor-memory lanes (32 rows) take the chunks of 16 or 32 columns in turn; a gated tile's chunks
        // are pairs, of g and of u.  What a chunk takes is mostly latency (reading tensor memory 105 cycles, a copy's issue
        // 150, its buffer being read 230, the gate 400), so there are many warps.  The loop over chunks is rolled: a
        // short call runs its code once, and fetching it unrolled takes longer than the work.
        constexpr int PARTS = EPI_WARPS / 4;
        pdl_wait();
        pdl_launch_dependents();
        const int quad = warp & 3, part = (warp - 2) >> 2;
        const bool elected = elect_one();  // issues the warp's copies
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        const int chunk = EPI == EPI_STORE || (EPI == EPI_SCALE && args.out_bf16) ? 32 : 16;  // columns
        const int n_chunks = block_n / chunk / (EPI == EPI_GATED ? 2 : 1);  // chunks, or pairs of them
        const int segments = P == 3 ? (kb_end - kb_begin + args.seg_kb - 1) / args.seg_kb : 1;
        const int ew = warp - 2;
        const uint32_t slab = stage_base + (uint32_t)stages * stage_bytes + (uint32_t)(ew * SLAB);
        uint32_t z_phase = 0;
        int z_out = 0;  // a copy into the slab is on its way
        int acc = 0;
        uint32_t phases = 0;  // of the accumulators, a bit each
        bool ok = true;
        auto wait_acc = [&]() {
            const bool got = patient_wait(smem_u32(&bar_acc_full[acc]), phases >> acc & 1u, abort_flag, 1 + ((kb_end - kb_begin) >> 16));
            if (!__all_sync(0xffffffffu, got)) {
                if (lane == 0) give_up(abort_flag, args.dev_status, DEV_STATUS_TIMEOUT_EPILOGUE);
                return false;
            }
            phases ^= 1u << acc;
            tc_fence_after();
            return true;
        };
        auto release_acc = [&]() {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (CG == 2) arrive_relaxed(map_to_cta(smem_u32(&bar_acc_empty[acc]), 0u));
                else mbar_arrive(smem_u32(&bar_acc_empty[acc]));
            }
        };
        for (int tile = first_tile; ok && tile < args.num_tiles; tile += tile_step) {
            const Item it = item_at<SUBS>(args, tile);
            const int tn = it.tn;
            const int which = EPI == EPI_STORE && tn >= args.n_tiles ? 1 : 0;
            const int64_t m0 = (int64_t)it.tm * TILE_M + it.sub * (CG * ROWS) + (int)rank * ROWS;
            const int n0 = EPI == EPI_GATED ? tn * (block_n >> 1) : (tn - which * args.n_tiles) * block_n;
            float sum[P == 3 ? 2 : 1][16];  // P = 3: block_n is 128, a warp has two chunks of 16
            if constexpr (P == 3) {
                for (int segment = 0; segment < segments; ++segment) {
                    if (!(ok = wait_acc())) break;
                    const uint32_t at = tmem_base + lanes + (uint32_t)acc * acc_cols;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        uint32_t small[16], large[16];
                        ld_columns(at + (uint32_t)((part + PARTS * j) * 16 + block_n), small);
                        ld_columns(at + (uint32_t)((part + PARTS * j) * 16), large);
                        tc_ld_wait();
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            sum[j][i] = ((segment ? sum[j][i] : 0.f) + __uint_as_float(small[i])) + __uint_as_float(large[i]);
                    }
                    release_acc();
                    acc ^= 1;
                }
            } else if (args.splits > 1) {
                ok = wait_acc();
            } else {
                for (int u = 0; u < (SUBS == 1 ? 1 : it.subs); ++u) {
                    if (SUBS == 2) acc = u;
                    const int64_t row0 = m0 + u * (CG * ROWS) + quad * 32, row = row0 + lane;
                    const bool rows_live = row0 < args.M;
                    const float row_scale = EPI == EPI_SCALE && row < args.M ? load_global(args.a_scale + row) : 0.f;
                    // EPI_GRAD: g and u of a chunk's 32 rows and 16 columns, 4 KiB in one piece, on their way while the chunk before is worked on.
                    // (Loads into registers leave room for half as many bytes on their way: 4096 x 2048 x 8192 122 us.)
                    auto fetch = [&](int col) {
                        if (EPI != EPI_GRAD || !rows_live || col >= args.N) return;
                        const float* from = z_at(args, row0, col, 0);
                        const uint32_t bar = smem_u32(&bar_z[EPI == EPI_GRAD ? ew : 0]);
                        if (elected) {
                            mbar_arrive_expect_tx(bar, 4096u);
                            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(slab), "l"(from),
                                         "r"(4096u), "r"(bar) : "memory");
                        }
                        z_out = 1;
                    };
                    if (part < n_chunks) fetch(n0 + part * chunk);
                    if (!(ok = wait_acc())) break;
                    if (part >= n_chunks) release_acc();
                    const uint32_t at = tmem_base + lanes + (uint32_t)acc * acc_cols;
#pragma unroll 1
                    for (int ch = part; ch < n_chunks; ch += PARTS) {
                        const int col = n0 + ch * chunk;
                        if constexpr (EPI == EPI_GATED || EPI == EPI_GRAD) {
                            uint32_t first[2][8], second[2][8];
#pragma unroll
                            for (int j = 0; j < 2; ++j) {
                                ld_columns(at + (uint32_t)(ch * 16 + j * 8), first[j]);
                                if (EPI == EPI_GATED) ld_columns(at + (uint32_t)(block_n / 2 + ch * 16 + j * 8), second[j]);
                            }
                            tc_ld_wait();
                            if (ch + PARTS >= n_chunks) release_acc();
                            if (!rows_live || col >= args.N) continue;
                            float out[EPI == EPI_GATED ? 1 : 2][16];
                            if constexpr (EPI == EPI_GATED) {
#pragma unroll
                                for (int j = 0; j < 2; ++j) {
                                    float g[8], u[8], v[8];
#pragma unroll
                                    for (int i = 0; i < 8; ++i) { g[i] = __uint_as_float(first[j][i]); u[i] = __uint_as_float(second[j][i]); }
                                    if (args.z && col + 8 * j < args.N) {
                                        store_f32(z_at(args, row, col + 8 * j, 0), g, 8);
                                        store_f32(z_at(args, row, col + 8 * j, 1), u, 8);
                                    }
                                    gated<false>(args.gate, g, u, v);
#pragma unroll
                                    for (int i = 0; i < 8; ++i) out[0][8 * j + i] = v[i];
                                }
                            } else {
                                const bool got = bounded_wait(smem_u32(&bar_z[ew]), z_phase, abort_flag);
                                if (!__all_sync(0xffffffffu, got)) {
                                    if (lane == 0) give_up(abort_flag, args.dev_status, DEV_STATUS_TIMEOUT_EPILOGUE);
                                    ok = false;
                                    break;
                                }
                                z_phase ^= 1u;
                                z_out = 0;
                                float g[2][8], u[2][8];
#pragma unroll
                                for (int j = 0; j < 2; ++j)
#pragma unroll
                                    for (int i = 0; i < 8; i += 4) {
                                        const float4 x = tile::lds4(slab + (uint32_t)(j * 2048 + lane * 32 + i * 4)), y = tile::lds4(slab + (uint32_t)(j * 2048 + 1024 + lane * 32 + i * 4));
                                        g[j][i] = x.x; g[j][i + 1] = x.y; g[j][i + 2] = x.z; g[j][i + 3] = x.w;
                                        u[j][i] = y.x; u[j][i + 1] = y.y; u[j][i + 2] = y.z; u[j][i + 3] = y.w;
                                    }
                                // All have read it, and have their values, before the next copy overwrites it.  (Without the fence the
                                // compiler moved half of the reads behind the copy's issue, in one of the instances.)
                                fence_async_smem();
                                __syncwarp();
                                if (ch + PARTS < n_chunks) fetch(col + PARTS * 16);
#pragma unroll
                                for (int j = 0; j < 2; ++j) {
                                    float v[8], du[8];
#pragma unroll
                                    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(first[j][i]);
                                    gated_gradient<false>(args.gate, g[j], u[j], v, du);
#pragma unroll
                                    for (int i = 0; i < 8; ++i) { out[0][8 * j + i] = v[i]; out[EPI == EPI_GRAD ? 1 : 0][8 * j + i] = du[i]; }
                                }
                            }
                            if (row < args.M) {
                                __nv_bfloat16* to = static_cast<__nv_bfloat16*>(args.out[0]) + row * args.out_pitch + col;
                                store_bf16(to, out[0], args.N - col);
                                if (EPI == EPI_GRAD) store_bf16(to + args.out_plane, out[EPI == EPI_GRAD ? 1 : 0], args.N - col);
                            }
                        } else {
                            // rounded (and scaled) values of 32 rows through the slab, eight columns after eight
                            const bool bf16 = EPI == EPI_STORE || args.out_bf16;
                            uint32_t sums[4][8];
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                if (EPI == EPI_STORE || j * 8 < chunk) ld_columns(at + (uint32_t)(ch * chunk + j * 8), sums[j]);
                            if (elected) tma_store_wait_read<0>();
                            tc_ld_wait();
                            if (ch + PARTS >= n_chunks) release_acc();
                            if (!rows_live || col >= args.N) continue;
                            __syncwarp();
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                if (EPI == EPI_SCALE && j * 8 >= chunk) break;
                                float v[8];
                                if constexpr (EPI == EPI_SCALE) {
                                    float scale[8], bias[8];
                                    const int left = args.N - col - 8 * j;
                                    load_f32(args.b_scale + col + 8 * j, scale, left);
                                    if (args.bias) load_f32(args.bias + col + 8 * j, bias, left);
                                    else
#pragma unroll
                                        for (int i = 0; i < 8; ++i) bias[i] = 0.f;
                                    scaled(args, row_scale, sums[j], scale, bias, v);
                                } else {
#pragma unroll
                                    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(sums[j][i]);
                                }
                                if (bf16) {
                                    sts16(slab + piece<64>(lane, j), pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
                                } else {
#pragma unroll
                                    for (int i = 0; i < 2; ++i)
                                        sts16(slab + piece<64>(lane, 2 * j + i), __float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]),
                                              __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3]));
                                }
                            }
                            if (args.out_mapped) {
                                fence_async_smem();
                                __syncwarp();
                                const CUtensorMap* map_out = &maps.out[which];
                                const int r0 = (int)row0;
                                if (elected) {
                                    tma_store_2d(map_out, slab, col, r0);
                                    tma_store_commit();
                                }
                            } else {
                                // rows are no multiple of 16 bytes: a lane has a column of the chunk, row after row
                                __syncwarp();
                                const int rows = (int)min((int64_t)32, args.M - row0), c = lane & (chunk - 1), size = bf16 ? 2 : 4;
                                if (col + c < args.N) {
                                    const int64_t to = row0 * args.out_pitch + col + c;
#pragma unroll 4
                                    for (int r = lane / chunk; r < rows; r += 32 / chunk) {
                                        const uint32_t from = slab + piece<64>(r, c * size >> 4) + (uint32_t)(c * size & 15);
                                        if (bf16) {
                                            unsigned short b;
                                            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(b) : "r"(from));
                                            static_cast<unsigned short*>(args.out[which])[to + r * args.out_pitch] = b;
                                        } else {
                                            float f;
                                            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(f) : "r"(from));
                                            static_cast<float*>(args.out[which])[to + r * args.out_pitch] = f;
                                        }
                                    }
                                }
                            }
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                    if (SUBS == 1) acc ^= 1;
                }
            }
            if constexpr (P == 3) {
                if (ok && args.splits == 1) {
                    const int64_t row = m0 + quad * 32 + lane;
                    // Sixteen columns at a time, 32 bytes of each plane of a row: what stores cost goes by the rows that they touch.
                    uint32_t w0[16], w1[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) { w0[i] = __float_as_uint(sum[0][i]); w1[i] = __float_as_uint(sum[1][i]); }
                    if (EPI == EPI_GATED) {
                        finish<P, EPI, 16>(args, which, row, n0 + part * 16, w0, w1);
                    } else {
                        const bool across = EPI == EPI_STORE && args.out_pitch % 4;
#pragma unroll 1
                        for (int j = 0; j < 2; ++j) {
                            const int col = n0 + (part + PARTS * j) * 16;
                            if (across) store_across(static_cast<float*>(args.out[which]), args.out_pitch, row - lane, args.M, col, args.N, w0);
                            else finish<P, EPI, 16>(args, which, row, col, w0, w0);
#pragma unroll
                            for (int i = 0; i < 16; ++i) w0[i] = w1[i];
                        }
                    }
                }
            }
            if constexpr (CG == 1) {
                if (args.splits > 1) {
                    // Every CTA's MMAs have finished (or it has room of its own for the sums): each gets its columns of this slice's.
                    if (!args.parts_apart) cluster_arrive();
                    cluster_wait();
                    if (ok && m0 + quad * 32 < args.M) {
                        const Share share(block_n, args.splits, args.M, EPI == EPI_GATED);
                        const int columns = EPI == EPI_GATED ? block_n >> 1 : block_n;
#pragma unroll 1
                        for (int j = 0; part + PARTS * j < block_n / 16; ++j) {
                            const int ch = part + PARTS * j;
                            uint32_t v[16];
                            if constexpr (P == 3) {
#pragma unroll
                                for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(j == 0 ? sum[0][i] : sum[1][i]);
                            } else {
                                ld_columns(tmem_base + lanes + (uint32_t)ch * 16u, v);
                                tc_ld_wait();
                            }
#pragma unroll
                            for (int i = 0; i < 16; i += 8) {
                                const int plane = EPI == EPI_GATED && ch * 16 >= columns ? 1 : 0, col = ch * 16 + i - plane * columns;
                                const int owner = col / share.columns;
                                const uint32_t to = map_to_cta(parts_base + (uint32_t)(share.at((int)slice, plane, quad * 32 + lane) + col - owner * share.columns) * 4u,
                                                               (uint32_t)owner);
                                if (m0 + quad * 32 + lane >= args.M) continue;
                                sts16_cluster(to, &v[i]);
                                sts16_cluster(to + 16u, &v[i + 4]);
                            }
                        }
                    }
                }
            }
        }
        if (EPI == EPI_GRAD && P == 1 && z_out) drain(smem_u32(&bar_z[EPI == EPI_GRAD && P == 1 ? ew : 0]), z_phase, args.dev_status);  // after a time-out
        if (elected) tma_store_wait_all();
        __syncwarp();
    }

    if constexpr (CG == 1) {
        if (args.splits > 1) {
            if (warp < 2 || warp == B_WARP) {  // the epilogue has been through the first barrier
                if (!args.parts_apart) cluster_arrive();
                cluster_wait();
            }
            cluster_arrive();
            cluster_wait();  // every slice's sums are here; from now on nothing touches another CTA's memory
            // after a time-out in any CTA the sums are wrong, and the status word says so
            if (warp >= 2 && warp < B_WARP) {
                int tm, tn;
                tile_at(args, first_tile, &tm, &tn);
                const int which = EPI == EPI_STORE && tn >= args.n_tiles ? 1 : 0;
                const int64_t m0 = (int64_t)tm * ROWS;
                const int columns = EPI == EPI_GATED ? block_n >> 1 : block_n;
                const int n0 = EPI == EPI_GATED ? tn * columns : (tn - which * args.n_tiles) * block_n;
                const Share share(block_n, args.splits, args.M, EPI == EPI_GATED);
                const int groups = max(0, min(share.columns, columns - (int)slice * share.columns)) / 8;
                const int rows = (int)min((int64_t)ROWS, args.M - m0);
                const uint32_t plane = (uint32_t)(share.at(0, 1, 0) * 4), step = (uint32_t)(share.at(1, 0, 0) * 4);
                for (int item = (int)threadIdx.x - 64; item < rows * groups; item += 32 * EPI_WARPS) {
                    const int row = item / groups, own = (item - row * groups) * 8, col = (int)slice * share.columns + own;
                    const uint32_t at = parts_base + (uint32_t)(share.at(0, 0, row) + own) * 4u;
                    uint32_t first[8], second[8];
                    sum_parts<KIND>(at, step, args.splits, first);
                    if (EPI == EPI_GATED) sum_parts<KIND>(at + plane, step, args.splits, second);
                    finish<P, EPI, 8>(args, which, m0 + row, n0 + col, first, second);
                }
            }
        }
    }

    // ---------------------------------------------------------------- teardown
    tc_fence_before();
    __syncthreads();
    if (CG == 2) {  // nobody leaves while another may still signal its barriers
        cluster_arrive();
        cluster_wait();
    }
    if (warp == 1) {
        tc_fence_after();
        if (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
    }
}

// ---- host --------------------------------------------------------------------------------------------------

tfjsb_status encode(tfjsb_ctx* ctx, CUtensorMap* map, const Operand& o, Kind kind, int64_t rows, int64_t K, int box_rows, const char* what) {
    const int size = kind == KIND_BF16 ? 2 : 1, bk = 128 / size;
    cuuint64_t dims[3] = {(cuuint64_t)(o.mn ? rows : K), (cuuint64_t)(o.mn ? K : rows), (cuuint64_t)o.planes};
    const int64_t plane = o.planes > 1 ? o.plane : o.pitch * (o.mn ? K : rows);
    cuuint64_t strides[2] = {(cuuint64_t)(o.pitch * size), (cuuint64_t)(plane * size)};
    cuuint32_t box[3] = {(cuuint32_t)(o.mn ? 64 : bk), (cuuint32_t)(o.mn ? 64 : box_rows), 1u};
    cuuint32_t elem[3] = {1u, 1u, 1u};
    const CUresult r = ctx->encode_tiled(map, kind == KIND_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8, 3,
                                         const_cast<void*>(o.base), dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS)
        return fail(ctx, TFJSB_ERR_CUDA, std::string("cuTensorMapEncodeTiled failed for ") + what + " (CUresult " + std::to_string((int)r) + ")");
    return TFJSB_OK;
}

// A row-major result, stored in chunks of 32 rows of 64 bytes.
tfjsb_status encode_result(tfjsb_ctx* ctx, CUtensorMap* map, void* base, bool f32, int64_t columns, int64_t rows, int64_t pitch) {
    const int size = f32 ? 4 : 2;
    cuuint64_t dims[2] = {(cuuint64_t)columns, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)(pitch * size)};
    cuuint32_t box[2] = {(cuuint32_t)(64 / size), 32u}, elem[2] = {1u, 1u};
    const CUresult r = ctx->encode_tiled(map, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, dims, strides, box, elem,
                                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS)
        return fail(ctx, TFJSB_ERR_CUDA, "cuTensorMapEncodeTiled failed for the result (CUresult " + std::to_string((int)r) + ")");
    return TFJSB_OK;
}

template <int CG, int P, int KIND, int EPI, int SUBS, bool A_MN, bool B_MN>
cudaError_t launch(const Maps& maps, const Args& args, int grid, size_t smem, cudaStream_t s, int64_t* launches) {
    auto* kernel = &dense_kernel<CG, P, KIND, EPI, SUBS, A_MN, B_MN>;
    cudaError_t e = smem_attr_once(reinterpret_cast<const void*>(kernel), tile::SMEM_LIMIT - 2048);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    int n = 0;
    const int cluster = CG == 2 ? 2 : args.splits;
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
    e = cudaLaunchKernelEx(&cfg, kernel, maps, args);
    if (e == cudaSuccess) count_launch(launches);
    return e;
}

// The layouts that the layers' products come in: x or h with K contiguous times weights [K, N] (gated, stored), gradients with K
// contiguous times weights [N, K] (gradient, stored), activations across times gradients across (stored), 8-bit rows.
template <int CG, int P, int SUBS>
cudaError_t launch_any(const Product& p, const Maps& maps, int grid, size_t smem, cudaStream_t s, int64_t* launches) {
    const bool a = p.a.mn, b = p.b[0].mn;
    if constexpr (P == 1)
        if (p.kind == KIND_INT8 && !a && !b) return launch<CG, P, KIND_INT8, EPI_SCALE, SUBS, false, false>(maps, p.args, grid, smem, s, launches);
    if (p.kind == KIND_BF16) {
        if (p.epilogue == EPI_GATED && !a && b) return launch<CG, P, KIND_BF16, EPI_GATED, SUBS, false, true>(maps, p.args, grid, smem, s, launches);
        if (p.epilogue == EPI_GRAD && !a && !b) return launch<CG, P, KIND_BF16, EPI_GRAD, SUBS, false, false>(maps, p.args, grid, smem, s, launches);
        if (p.epilogue == EPI_STORE && !a && b) return launch<CG, P, KIND_BF16, EPI_STORE, SUBS, false, true>(maps, p.args, grid, smem, s, launches);
        if (p.epilogue == EPI_STORE && !a && !b) return launch<CG, P, KIND_BF16, EPI_STORE, SUBS, false, false>(maps, p.args, grid, smem, s, launches);
        if (p.epilogue == EPI_STORE && a && b) return launch<CG, P, KIND_BF16, EPI_STORE, SUBS, true, true>(maps, p.args, grid, smem, s, launches);
    }
    return cudaErrorInvalidValue;
}

// Which kernel: CTA pairs or single CTAs, columns of a tile, slices of K, parts of a tile's rows.
struct Shape { int cg, block_n, splits, subs; };

int64_t tiles_of(const Product& p, int cg, int block_n, int subs = 1) {
    const int64_t columns = p.epilogue == EPI_GATED ? block_n / 2 : block_n, rows = cg * ROWS * subs;
    return ((p.args.M + rows - 1) / rows) * ((p.args.N + columns - 1) / columns) * p.args.outputs;
}

// Estimated cycles, with constants fitted to 3600 measured times of products from 10 x 128 x 192 to 13248 x 256 x 2595 on every kernel shape (the shape
// with the least estimate takes 1 % longer than the best in the mean, 19 % at most):
//   - a k-block takes what its MMAs take, what an SM can fetch (48 to 63 bytes a cycle) or what issuing takes, whichever is longest; a pair
//     with two parts fetches three tiles for two, a pair half of B, single CTAs everything;
//   - the first k-block arrives, and the epilogue takes, so long; with one part a tile the epilogue runs beside the next tile's K
//     loop, with two it holds up the next tile (by more than itself: tensor memory is read while both parts' MMAs write it);
//   - slices cost a cluster barrier, the sums on their way to the CTAs that add them, and the adding; clusters of more CTAs, each with an SM of
//     its own in one group of SMs, also start later.
double cost(const Product& p, const Shape& c, int sm_count) {
    const Args& a = p.args;
    const int kb = (a.K + (p.kind == KIND_BF16 ? 63 : 127)) / (p.kind == KIND_BF16 ? 64 : 128) * a.passes, own_kb = (kb + c.splits - 1) / c.splits;
    const double rows = a.M < ROWS ? a.M : ROWS;
    auto k_block = [&](int subs) {
        const double rate = c.block_n == 256 ? (c.cg == 2 ? 48 : 50) : c.block_n == 64 ? 52.5 : 62.5;
        const double fetch = p.planes * 128. * (rows * subs + c.block_n / c.cg) / rate, mma = 1.63 * c.block_n * subs * (p.planes == 3 ? 6 : 1);
        const double longer = fetch > mma ? fetch : mma, issue = p.planes == 3 ? 975 : 450;
        return longer > issue ? longer : issue;
    };
    const double main = own_kb * k_block(c.subs), first = c.cg == 2 ? 3600 : 2200;
    const int columns = p.epilogue == EPI_GATED ? c.block_n / 2 : c.block_n;
    const double column = p.epilogue == EPI_STORE ? 25 : p.epilogue == EPI_SCALE ? 87 : p.epilogue == EPI_GRAD ? 101 : a.z ? 83 : 60;
    const double epilogue = columns / 4 * column * (p.planes == 3 ? 5 : 1);
    const int64_t tiles = tiles_of(p, c.cg, c.block_n, c.subs), slots = sm_count / c.cg;
    if (c.splits > 1) {
        const int64_t items = (int64_t)rows * ((columns / 8 + c.splits - 1) / c.splits), threads = 32 * EPI_WARPS;  // eight columns each
        return first + main + 1200 + 430 * c.splits + 0.25 * rows * c.block_n * (c.splits - 1) / c.splits + (double)((items + threads - 1) / threads) * 1800;
    }
    const int64_t rounds = tiles / slots, rest = tiles % slots;
    if (c.subs == 2) {
        const double whole = main + 3.7 * epilogue;
        return first + rounds * whole + (rest == 0 ? 0. : 2 * rest <= slots ? own_kb * k_block(1) + epilogue : whole) + epilogue;
    }
    const double step = main > epilogue ? main : epilogue;
    return first + main + epilogue + (rounds + (rest ? 1 : 0) - 1) * step;
}

// Clusters of that many CTAs, one to an SM, that are resident at once: less than the SMs over their number, which the GPU's groups of SMs
// do not divide.
int resident_clusters(int dev, int size) {
    constexpr int DEVICES = 64;
    static std::atomic<int> known[DEVICES][9];  // 0: not asked yet
    if (dev < DEVICES)
        if (const int n = known[dev][size].load(std::memory_order_relaxed)) return n;
    auto* kernel = &dense_kernel<1, 1, KIND_BF16, EPI_STORE, 1, false, false>;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(size * 64);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = tile::SMEM_LIMIT - 2048;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = size;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (smem_attr_once(reinterpret_cast<const void*>(kernel), tile::SMEM_LIMIT - 2048) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
        (void)cudaGetLastError();
        n = 96 / size;
    }
    if (dev < DEVICES) known[dev][size].store(n, std::memory_order_relaxed);
    return n;
}

Shape choose(const Product& p, int dev, int sm_count) {
    const char* forced = getenv("TFJSB_DENSE_SHAPE");  // for tests: "CTA group,columns,slices,parts", wherever the product allows it
    int f[4];
    const bool force = forced && sscanf(forced, "%d,%d,%d,%d", &f[0], &f[1], &f[2], &f[3]) == 4;
    Shape best = {1, 128, 1, 1};
    double least = -1;
    const int kb = (p.args.K + (p.kind == KIND_BF16 ? 63 : 127)) / (p.kind == KIND_BF16 ? 64 : 128) * p.args.passes;
    for (int cg = 1; cg <= 2; ++cg)
        for (int bn = 64; bn <= 256; bn *= 2) {
            if (p.planes == 3 && bn != 128) continue;                         // two accumulators of 128 columns, two stages
            if (bn == 64 && (cg == 2 || p.epilogue == EPI_GATED)) continue;   // boxes are 64 columns wide
            const int64_t tiles = tiles_of(p, cg, bn);
            for (int splits = 1; splits <= (cg == 1 ? 8 : 1); ++splits) {
                // at least four k-blocks a slice, none without any, one wave, and room for the sums
                const int each = (kb + splits - 1) / splits;
                if (splits > 1 && (each < 4 || each * (splits - 1) >= kb || tiles * splits > sm_count || tiles > resident_clusters(dev, splits) ||
                                   Share(bn, splits, p.args.M, p.epilogue == EPI_GATED).bytes(splits) > STAGES_AT_LEAST))
                    continue;
                for (int subs = 1; subs <= (cg == 2 && bn == 256 && p.planes == 1 ? 2 : 1); ++subs) {
                    const Shape c = {cg, bn, splits, subs};
                    if (force && f[0] == cg && f[1] == bn && f[2] == splits && f[3] == subs) return c;
                    const double cycles = cost(p, c, sm_count);
                    if (least < 0 || cycles < least) { least = cycles; best = c; }
                }
            }
        }
    return best;
}

}  // namespace

Ran& ran() {
    static thread_local Ran r;
    return r;
}

tfjsb_status run_product(tfjsb_ctx* ctx, Product& p, cudaStream_t s) {
    if (!ctx->encode_tiled) return fail(ctx, TFJSB_ERR_CUDA, "cuTensorMapEncodeTiled is not available");
    Args& a = p.args;
    const Shape c = choose(p, ctx->device, ctx->sm_count);
    const int bk = p.kind == KIND_BF16 ? 64 : 128;
    a.block_n = c.block_n;
    a.splits = c.splits;
    a.seg_kb = 2;  // 8 additions to an accumulator of large products
    a.num_kb = (a.K + bk - 1) / bk;
    a.kb_per_split = (a.num_kb * a.passes + c.splits - 1) / c.splits;
    a.m_tiles = (a.M + c.cg * ROWS * c.subs - 1) / (c.cg * ROWS * c.subs);
    const int columns = p.epilogue == EPI_GATED ? c.block_n / 2 : c.block_n;
    a.n_tiles = (a.N + columns - 1) / columns;
    const int64_t slots = ctx->sm_count / c.cg;
    int64_t tiles = tiles_of(p, c.cg, c.block_n, c.subs);
    if (tiles >= (1LL << 30)) return fail(ctx, TFJSB_ERR_UNSUPPORTED, "too many tiles");
    a.whole_tiles = (int)tiles;
    if (c.subs == 2 && 2 * (tiles % slots) <= slots) {  // a last round of few tiles: their parts as tiles of their own
        a.whole_tiles -= (int)(tiles % slots);
        tiles += tiles % slots;
    }
    a.num_tiles = (int)tiles;
    a.band = 8 / c.subs;
    // of a matrix of less rows than a tile only those are copied (a multiple of 8, the swizzle's period): the others' sums are not stored
    a.a_rows = !p.a.mn && a.M < ROWS ? (a.M + 7) / 8 * 8 : ROWS;
    a.dev_status = ctx->dev_status;
    const int own_n = c.block_n / c.cg;
    const int stage_bytes = p.planes * (c.subs * A_BYTES + own_n * 128);
    const int slabs = EPI_WARPS * (p.planes == 3 || p.epilogue == EPI_GATED || c.splits > 1 ? 0 : p.epilogue == EPI_GRAD ? SLAB_BYTES<1, EPI_GRAD> : SLAB_BYTES<1, EPI_STORE>);
    int room = tile::SMEM_LIMIT - 2048 - 1024 - slabs;
    // Room of their own for the slices' sums where it is small; otherwise they take that of the stages, once all MMAs have read them.
    const int parts = c.splits > 1 ? Share(c.block_n, c.splits, a.M, p.epilogue == EPI_GATED).bytes(c.splits) : 0;
    a.parts_apart = parts > 0 && parts <= stage_bytes && p.planes == 1;
    if (a.parts_apart) room -= parts;
    const int stages = room / stage_bytes;
    a.stages = stages < MAX_STAGES ? stages : MAX_STAGES;
    const size_t smem = 1024 + (size_t)a.stages * stage_bytes + slabs + (a.parts_apart ? parts : 0);
    Maps maps;
    tfjsb_status st;
    const int b_rows = p.epilogue == EPI_GATED ? c.block_n / 2 : own_n;
    if ((st = encode(ctx, &maps.a, p.a, p.kind, a.M, a.K, a.a_rows, "A")) != TFJSB_OK) return st;
    if ((st = encode(ctx, &maps.b[0], p.b[0], p.kind, a.N, a.K, b_rows, "B")) != TFJSB_OK) return st;
    maps.b[1] = maps.b[0];
    if (p.b[1].base && (st = encode(ctx, &maps.b[1], p.b[1], p.kind, a.N, a.K, b_rows, "B")) != TFJSB_OK) return st;
    if (p.planes == 1 && c.splits == 1) {
        const bool f32 = p.epilogue == EPI_SCALE && !a.out_bf16;
        a.out_mapped = (p.epilogue == EPI_STORE || p.epilogue == EPI_SCALE) && a.out_pitch * (f32 ? 4 : 2) % 16 == 0;
        for (int i = 0; i < a.outputs && a.out_mapped; ++i)
            if ((st = encode_result(ctx, &maps.out[i], a.out[i], f32, a.N, a.M, a.out_pitch)) != TFJSB_OK) return st;
    }
    const int grid = (int)(c.splits > 1 ? tiles * c.splits : (tiles < slots ? tiles : slots) * c.cg);
    const cudaError_t e = c.subs == 2                      ? launch_any<2, 1, 2>(p, maps, grid, smem, s, &ctx->launches)
                          : c.cg == 2 && p.planes == 1 ? launch_any<2, 1, 1>(p, maps, grid, smem, s, &ctx->launches)
                          : c.cg == 2                  ? launch_any<2, 3, 1>(p, maps, grid, smem, s, &ctx->launches)
                          : p.planes == 1              ? launch_any<1, 1, 1>(p, maps, grid, smem, s, &ctx->launches)
                                                       : launch_any<1, 3, 1>(p, maps, grid, smem, s, &ctx->launches);
    if (e != cudaSuccess) return cuda_fail(ctx, e, "dense product launch");
    Ran& r = ran();
    if (r.count < 8) r.product[r.count++] = {p.epilogue, c.cg, c.block_n, c.splits, c.subs};
    return TFJSB_OK;
}

}  // namespace dense
}  // namespace tfjsb

extern "C" tfjsb_status tfjsb_dense_kernels(tfjsb_ctx* ctx, char* text, int32_t text_len) {
    using namespace tfjsb;
    if (!ctx) return TFJSB_ERR_INVALID_ARG;
    if (!text || text_len < 1) return fail(ctx, TFJSB_ERR_INVALID_ARG, "text is null or has no room");
    const dense::Ran& r = dense::ran();
    std::string all;
    for (int i = 0; i < r.count; ++i) {
        const auto& k = r.product[i];
        const char* name = k.epilogue == dense::EPI_STORE ? "stored" : k.epilogue == dense::EPI_GATED ? "gated" : k.epilogue == dense::EPI_GRAD ? "gradient" : "scaled";
        all += std::string(i ? "; " : "") + name + " " + std::to_string(k.cg) + "," + std::to_string(k.block_n) + "," + std::to_string(k.splits) + "," +
               std::to_string(k.subs);
    }
    snprintf(text, (size_t)text_len, "%s", all.c_str());
    return TFJSB_OK;
}
