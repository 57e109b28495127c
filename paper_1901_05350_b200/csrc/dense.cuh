// Shared by the dense layers of transformer blocks: the tensor-core product with their epilogues (dense_tcgen05.cu), the gated
// feed-forward block (gated_ffn.cu) and the 8-bit dense layer (int8_dense.cu).
#pragma once

#include "common.cuh"

namespace tfjsb {
namespace dense {

// What an operand's planes are: one plane of bfloat16 or 8-bit values, or an fp32 matrix as three bfloat16 planes whose sum
// it is (8 + 8 + 8 significant bits, so the sum is exact).
enum Kind { KIND_BF16 = 0, KIND_INT8 = 1 };
// What becomes of the sums of a tile.
enum Epilogue {
    EPI_STORE,  // written as they are: bfloat16 (one plane) or fp32 (three)
    EPI_GATED,  // columns come in pairs (g, u) from two weights: h = gate(g) u, and (g, u) themselves where `z` is given
    EPI_GRAD,   // sums are dh: with g and u read from `z`, dg = dh u gate'(g) and du = dh gate(g)
    EPI_SCALE,  // 32-bit integers: act(sum a_scale[row] b_scale[column] + bias[column]) in bfloat16 or fp32
};

// A stored operand.  K-contiguous: [outer rows][K]; otherwise `mn`: [K][rows].  `pitch` in elements, a multiple of 16 bytes.
struct Operand {
    const void* base = nullptr;
    int64_t pitch = 0;   // between rows of memory
    int64_t plane = 0;   // between planes, in elements (any when there is one)
    int planes = 1;
    bool mn = false;
};

struct Args {
    int M = 0, N = 0, K = 0;      // of one pass; N: columns of one output (of h for EPI_GATED)
    int block_n = 0, stages = 0;
    int n_tiles = 0, m_tiles = 0, outputs = 1, num_tiles = 0, whole_tiles = 0, band = 8;
    int passes = 1, num_kb = 0, kb_per_split = 0, seg_kb = 0;
    int splits = 1;
    int parts_apart = 0;                   // the slices' sums have shared memory of their own
    int a_rows = 0;
    void* out[2] = {nullptr, nullptr};
    int64_t out_pitch = 0, out_plane = 0;  // elements
    int out_mapped = 0;                    // results leave through shared memory
    float* z = nullptr;                    // g and u in fp32, in blocks of 32 rows x 8 columns: see z_at
    int64_t z_pitch = 0;                   // columns, a multiple of 8
    int gate = 0;
    int out_bf16 = 1, act = 0;             // EPI_SCALE
    const float *a_scale = nullptr, *b_scale = nullptr, *bias = nullptr;
    // The kernel before in the stream, one of this chain, writes nothing of the operand (nor may it still be running with what it
    // waited for unfinished: kernels of a chain let the next one go after their own wait).
    int early_a = 0, early_b = 0;
    unsigned int* dev_status = nullptr;
};

// C = A B summed over `passes` pairs (plane group p of A with b[p]), or with `outputs` = 2 the products of A with the two
// plane groups of b[0]; EPI_GATED: A with b[0] and b[1].  Fill in args.{M, N, K, passes, outputs, out*, z*, gate, ...}.
struct Product {
    Kind kind = KIND_BF16;
    int planes = 1;
    Epilogue epilogue = EPI_STORE;
    Operand a, b[2];
    Args args;
};
tfjsb_status run_product(tfjsb_ctx* ctx, Product& p, cudaStream_t s);
// The kernels of the calling thread's products since its call began (tfjsb_dense_kernels).
struct Ran {
    struct { Epilogue epilogue; int cg, block_n, splits, subs; } product[8];
    int count = 0;
};
Ran& ran();

// Products of few rows (few_rows.cu).  h is fp32 [rows, N]; operands 16-byte aligned, of any sizes.  FEW_ROWS at most.
// bfloat16, whose weights the tensor cores take as they are stored: one or two rows.  Blocks of width x hidden, us of one row and of two, on
// CUDA cores | on tensor cores: 1024 x 4096 (24 MB, in L2) 11, 12 | 15, 15; 2048 x 8192 (100 MB, four sets of weights in turn) 34, 36 | 28, 28;
// 4096 x 16384 (402 MB) 83, 93 | 68, 68.  So where weights come from HBM the tensor cores are ahead already; the rule does not know that yet.
// fp32, whose weights would be split into planes first: one, eight rows 17, 38 | 64, 62; 70, 124 | 163, 171; 225, 368 | 584, 638.
constexpr int FEW_ROWS = 8;
constexpr int few_rows_ffn(bool f32) { return f32 ? FEW_ROWS : 2; }
tfjsb_status few_rows_gated(tfjsb_ctx* ctx, bool f32, const void* x, const void* w_gate, const void* w_up, int gate, float* h, int64_t rows, int64_t N,
                            int64_t K, cudaStream_t s);
tfjsb_status few_rows_down(tfjsb_ctx* ctx, bool f32, const float* h, const void* w, void* y, int64_t rows, int64_t N, int64_t K, cudaStream_t s);
// 8-bit products of rows that are quantised by the same kernel.  x_kind: 0 one row of 8-bit values [K rounded up to 16] with
// a_scale, 1 bfloat16, 2 fp32.  More than one row: M max(N, K) below 2^32.
constexpr int ROW_INT8_BYTES = 131072;  // of the largest K: the row's 8-bit values are in shared memory
tfjsb_status rows_int8(tfjsb_ctx* ctx, int x_kind, const void* x, const float* a_scale, const int8_t* bt, const float* b_scale, const float* bias, int act,
                      void* out, bool out_bf16, int64_t M, int64_t N, int64_t K, cudaStream_t s);

// The context's device is the current one while this lives: tensors say where they are, the caller's device may be another.
struct OnDevice {
    int before = -1;
    explicit OnDevice(const tfjsb_ctx* ctx) {
        int now = -1;
        if (cudaGetDevice(&now) == cudaSuccess && now != ctx->device && cudaSetDevice(ctx->device) == cudaSuccess) before = now;
    }
    ~OnDevice() {
        if (before >= 0) cudaSetDevice(before);
    }
    OnDevice(const OnDevice&) = delete;
};

}  // namespace dense
}  // namespace tfjsb
