// The gated feed-forward block, y = (gate(x Wg) * (x Wu)) Wd, and its gradients: argument checks, layout of the workspaces, and the
// order of the kernels.  The products are dense_tcgen05.cu's.
//
//   forward    [x Wg | x Wu] -> h (and z = (g, u) in fp32, where a gradient will be wanted);  y = h Wd
//   backward   dWd = h^T dy;  dh = dy Wd^T -> (dg, du);  dx = dg Wg^T + du Wu^T;  dWg = x^T dg, dWu = x^T du
//
// What is kept for the gradient is g and u in fp32: 8 bytes an element, written once and read once, which takes a fifth of the time of computing
// both again at a width of 4096 (4 T D F more operations), and spares their gradients two roundings.
#include <cuda_bf16.h>

#include "common.cuh"
#include "dense.cuh"
#include "dense_math.cuh"
#include "ptx_sm100.cuh"

namespace tfjsb {
namespace dense {
namespace {

// ---- copies into planes -----------------------------------------------------------------------------------
// Matrices [rows, columns] as P planes of bfloat16 with rows of a multiple of 16 bytes: an fp32 matrix in three parts, a bfloat16 one whose
// rows are not such a multiple as it is.  Several matrices in one launch; a thread has eight values of a row at a time, LAYOUT_STEPS times.
//
// Rows begin anywhere, so a thread loads the aligned 16-byte pieces that its eight values lie in and moves them into place (eight loads of one
// value each, which touch the same lines, took twice as long); the last pieces of a matrix, which may reach beyond its end, value by value.
struct LayoutItem {
    const void* src;
    __nv_bfloat16* dst;
    int64_t rows, columns, pitch, plane;
    int64_t first_block;
};
constexpr int LAYOUT_MAX = 5, LAYOUT_STEPS = 2, LAYOUT_PER_BLOCK = LAYOUT_STEPS * 2048;
struct LayoutArgs {
    LayoutItem item[LAYOUT_MAX];
    int count = 0;
    int64_t blocks = 0;
};

__device__ __forceinline__ uint4 ld16(const void* p) {
    uint4 v;
    asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
// Eight values of an item from `at` on (an index into the source), of which `left` are wanted; those beyond are anything.
template <bool F32>
__device__ __forceinline__ void source8(const LayoutItem& it, int64_t at, int left, float (&v)[8]) {
    constexpr int SIZE = F32 ? 4 : 2, PIECES = F32 ? 3 : 2;
    const char* p = static_cast<const char*>(it.src) + at * SIZE;
    const int shift = (int)(reinterpret_cast<uintptr_t>(p) & 15u) / SIZE;  // values
    const char* from = p - shift * SIZE;
    const int64_t there = it.rows * it.columns * SIZE - (from - static_cast<const char*>(it.src));  // bytes from there to the end
    if (there < 16 * PIECES) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] = 0.f;
            if (e < left) {
                if (F32) v[e] = load_global(reinterpret_cast<const float*>(p) + e);
                else v[e] = __uint_as_float((uint32_t)load_global(reinterpret_cast<const unsigned short*>(p) + e) << 16);
            }
        }
        return;
    }
    uint32_t w[4 * PIECES];
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        const uint4 q = ld16(from + 16 * j);
        w[4 * j] = q.x; w[4 * j + 1] = q.y; w[4 * j + 2] = q.z; w[4 * j + 3] = q.w;
    }
    const int words = F32 ? shift : shift >> 1;
    if (words & 1) {
#pragma unroll
        for (int i = 0; i + 1 < 4 * PIECES; ++i) w[i] = w[i + 1];
    }
    if (words & 2) {
#pragma unroll
        for (int i = 0; i + 2 < 4 * PIECES; ++i) w[i] = w[i + 2];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (F32) {
            v[e] = __uint_as_float(w[e]);
        } else {
            const uint32_t pair = (shift & 1) ? __funnelshift_r(w[e / 2], w[e / 2 + 1], 16) : w[e / 2];
            v[e] = __uint_as_float(e % 2 ? pair & 0xffff0000u : pair << 16);
        }
    }
}

template <bool F32>
__global__ void __launch_bounds__(256) layout_kernel(const __grid_constant__ LayoutArgs args) {
    ptx::pdl_wait();
    ptx::pdl_launch_dependents();
    int k = 0;
    while (k + 1 < args.count && (int64_t)blockIdx.x >= args.item[k + 1].first_block) ++k;
    const LayoutItem& it = args.item[k];
    float v[LAYOUT_STEPS][8];
    int64_t row[LAYOUT_STEPS];
    int col[LAYOUT_STEPS];
    const uint32_t per_row = (uint32_t)(it.pitch >> 3);
#pragma unroll
    for (int s = 0; s < LAYOUT_STEPS; ++s) {
        const int64_t eights = ((int64_t)blockIdx.x - it.first_block) * (LAYOUT_PER_BLOCK / 8) + s * 256 + threadIdx.x;
        row[s] = eights < (1LL << 31) ? (int64_t)((uint32_t)eights / per_row) : eights / per_row;
        col[s] = (int)(eights - row[s] * per_row) * 8;
        if (row[s] < it.rows) source8<F32>(it, row[s] * it.columns + col[s], (int)(it.columns - col[s]), v[s]);
    }
#pragma unroll
    for (int s = 0; s < LAYOUT_STEPS; ++s) {
        if (row[s] >= it.rows) continue;
        const int left = (int)(it.columns - col[s]);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[s][e] = e < left ? v[s][e] : 0.f;
        store_planes<F32 ? 3 : 1>(it.dst + row[s] * it.pitch + col[s], it.plane, v[s], 8);
    }
}

// ---- layout of the buffers ---------------------------------------------------------------------------------
constexpr int64_t up8(int64_t v) { return (v + 7) / 8 * 8; }
constexpr int64_t up16(int64_t v) { return (v + 15) / 16 * 16; }
constexpr int64_t MOST_BYTES = 1LL << 60;  // of a buffer: sums of a few of them, and addresses, stay within 64 bits

struct Sizes {
    int planes;            // 1 (bfloat16) or 3 (fp32)
    int64_t T, D, F, Do;
    int64_t fp;            // pitch of h, dg, du and z
    bool repack_x, repack_up, repack_down, repack_dy;  // operands that are copied: x; w_gate and w_up; w_down; dy
    int64_t x_bytes, w_bytes, wd_bytes, dy_bytes;      // of such a copy
    int64_t h_bytes, z_bytes, grad_bytes;              // grad: dg and du
    int64_t forward, backward;
};

tfjsb_status sizes_of(const tfjsb_ffn* f, Sizes* s, std::string* why) {
    if (!f) { *why = "ffn is null"; return TFJSB_ERR_INVALID_ARG; }
    if (f->dtype != TFJSB_DTYPE_F32 && f->dtype != TFJSB_DTYPE_BF16) { *why = "unknown dtype"; return TFJSB_ERR_INVALID_ARG; }
    if (f->gate < TFJSB_GATE_SILU || f->gate > TFJSB_GATE_RELU) { *why = "unknown gate"; return TFJSB_ERR_INVALID_ARG; }
    const int64_t most = 1LL << 30;
    if (f->tokens < 0 || f->tokens > most || f->width < 1 || f->width > most || f->hidden < 1 || f->hidden > most || f->out_width < 1 ||
        f->out_width > most) {
        *why = "sizes must be 1 to 2^30 (tokens 0 to 2^30)";
        return TFJSB_ERR_SHAPE;
    }
    const bool f32 = f->dtype == TFJSB_DTYPE_F32;
    s->planes = f32 ? 3 : 1;
    s->T = f->tokens; s->D = f->width; s->F = f->hidden; s->Do = f->out_width;
    s->fp = up16(s->F);  // rows of whole 32-byte sectors
    s->repack_x = f32 || s->D % 8;
    s->repack_up = f32 || s->F % 8;
    s->repack_down = s->repack_dy = f32 || s->Do % 8;
    // Every byte count below is worked out in 128 bits first: 2^30 tokens of 2^30 hidden values have more bytes than 64 bits hold, and a
    // count that wrapped around would let any workspace pass.
    const __int128 e = 2 * s->planes, T = s->T;
    const auto up = [](__int128 v) { return (v + 255) / 256 * 256; };
    const __int128 x_bytes = up(T * up8(s->D) * e), w_bytes = up(up8(s->F) * e * s->D), wd_bytes = up(up8(s->Do) * e * s->F), dy_bytes = up(T * up8(s->Do) * e);
    const __int128 h_bytes = up(T * s->fp * e), z_bytes = up((T + 31) / 32 * 32 * s->fp * 8), grad_bytes = up(T * s->fp * 2 * e);  // z: whole blocks of 32 rows
    const __int128 weights = (s->repack_x ? x_bytes : 0) + (s->repack_up ? 2 * w_bytes : 0) + (s->repack_down ? wd_bytes : 0);
    const __int128 few = T <= few_rows_ffn(f32) ? up(T * s->F * 4) : 0;
    const __int128 forward = weights + h_bytes > few ? weights + h_bytes : few, backward = weights + (s->repack_dy ? dy_bytes : 0) + grad_bytes;
    for (const __int128 bytes : {z_bytes, forward, backward, (__int128)s->D * s->F * e, (__int128)s->F * s->Do * e, T * s->D * e, T * s->Do * e})
        if (bytes > MOST_BYTES) {
            *why = "a buffer of the block would have more than 2^60 bytes";
            return TFJSB_ERR_SHAPE;
        }
    s->x_bytes = (int64_t)x_bytes;
    s->w_bytes = (int64_t)w_bytes;
    s->wd_bytes = (int64_t)wd_bytes;
    s->dy_bytes = (int64_t)dy_bytes;
    s->h_bytes = (int64_t)h_bytes;
    s->z_bytes = (int64_t)z_bytes;
    s->grad_bytes = (int64_t)grad_bytes;
    s->forward = (int64_t)forward;
    s->backward = (int64_t)backward;
    return TFJSB_OK;
}

// A workspace handed out piece by piece.
struct Arena {
    uint8_t* at;
    __nv_bfloat16* take(int64_t bytes) {
        uint8_t* p = at;
        at += bytes;
        return reinterpret_cast<__nv_bfloat16*>(p);
    }
};

// An operand [rows, columns] of the call: as it is, or its copy in the arena, with a layout item added.
Operand operand(LayoutArgs* layout, Arena* arena, bool copy, const void* src, int64_t rows, int64_t columns, int64_t bytes, int planes) {
    Operand o;
    o.base = src;
    o.pitch = columns;
    if (copy) {
        o.pitch = up8(columns);
        o.plane = rows * o.pitch;
        o.planes = planes;
        LayoutItem& it = layout->item[layout->count++];
        it = {src, arena->take(bytes), rows, columns, o.pitch, o.plane, layout->blocks};
        layout->blocks += (rows * o.pitch + LAYOUT_PER_BLOCK - 1) / LAYOUT_PER_BLOCK;
        o.base = it.dst;
    }
    return o;
}

tfjsb_status run_layout(tfjsb_ctx* ctx, const LayoutArgs& l, bool f32, cudaStream_t s) {
    if (l.count == 0 || l.blocks == 0) return TFJSB_OK;
    if (l.blocks >= (1LL << 31)) return fail(ctx, TFJSB_ERR_UNSUPPORTED, "operands too large to be copied");
    const cudaError_t e = f32 ? launch_k_serial(layout_kernel<true>, dim3((unsigned)l.blocks), dim3(256), 0, s, l)
                              : launch_k_serial(layout_kernel<false>, dim3((unsigned)l.blocks), dim3(256), 0, s, l);
    if (e != cudaSuccess) return cuda_fail(ctx, e, "operand layout launch");
    count_launch(&ctx->launches);
    return TFJSB_OK;
}

Operand stored(const void* base, int64_t pitch, int64_t plane, int planes) {
    Operand o;
    o.base = base;
    o.pitch = pitch;
    o.plane = plane;
    o.planes = planes;
    return o;
}
// The same memory with its rows as the other dimension of the product.
Operand across(Operand o, bool mn) {
    o.mn = mn;
    return o;
}

bool aligned16(const void* p) { return aligned(p, 16); }
struct Range { const void* p; int64_t bytes; const char* name; };
bool overlap(const Range& a, const Range& b) {
    if (!a.p || !b.p || a.bytes <= 0 || b.bytes <= 0) return false;
    const char *x = static_cast<const char*>(a.p), *y = static_cast<const char*>(b.p);
    return x < y + b.bytes && y < x + a.bytes;
}
// The first `outputs` ranges may overlap nothing; all are there (unless empty or optional) and aligned.
tfjsb_status check_ranges(tfjsb_ctx* ctx, const Range* r, int count, int outputs, unsigned optional) {
    for (int i = 0; i < count; ++i) {
        if (!r[i].p && r[i].bytes > 0 && !(optional >> i & 1)) return fail(ctx, TFJSB_ERR_INVALID_ARG, std::string(r[i].name) + " is null");
        if (r[i].bytes > 0 && !aligned16(r[i].p)) return fail(ctx, TFJSB_ERR_INVALID_ARG, std::string(r[i].name) + " is not 16-byte aligned");
    }
    for (int i = 0; i < outputs; ++i)
        for (int j = i + 1; j < count; ++j)
            if (overlap(r[i], r[j])) return fail(ctx, TFJSB_ERR_INVALID_ARG, std::string(r[i].name) + " overlaps " + r[j].name);
    return TFJSB_OK;
}

}  // namespace
}  // namespace dense
}  // namespace tfjsb

using namespace tfjsb;
using namespace tfjsb::dense;

extern "C" {

tfjsb_status tfjsb_gated_ffn_sizes(const tfjsb_ffn* ffn, int64_t* h_bytes, int64_t* z_bytes, int64_t* workspace_bytes, int64_t* backprop_workspace_bytes) {
    Sizes s;
    std::string why;
    const tfjsb_status st = sizes_of(ffn, &s, &why);
    if (st != TFJSB_OK) return st;
    if (h_bytes) *h_bytes = s.h_bytes;
    if (z_bytes) *z_bytes = s.z_bytes;
    if (workspace_bytes) *workspace_bytes = s.forward;
    if (backprop_workspace_bytes) *backprop_workspace_bytes = s.backward;
    return TFJSB_OK;
}

tfjsb_status tfjsb_gated_ffn(tfjsb_ctx* ctx, const tfjsb_ffn* ffn, const void* x, const void* w_gate, const void* w_up, const void* w_down, void* y,
                             void* h, void* z, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!ctx) return TFJSB_ERR_INVALID_ARG;
    const dense::OnDevice on(ctx);
    ran().count = 0;
    Sizes s;
    std::string why;
    tfjsb_status st = sizes_of(ffn, &s, &why);
    if (st != TFJSB_OK) return fail(ctx, st, why);
    if (!h != !z) return fail(ctx, TFJSB_ERR_INVALID_ARG, "h and z: both or neither");
    if (workspace_bytes < s.forward) return fail(ctx, TFJSB_ERR_INVALID_ARG, "the workspace needs " + std::to_string(s.forward) + " bytes");
    if (s.T == 0) return TFJSB_OK;
    const int64_t size = s.planes == 3 ? 4 : 2;
    const Range r[] = {{y, s.T * s.Do * size, "y"}, {h, s.h_bytes, "h"}, {z, s.z_bytes, "z"}, {workspace, s.forward, "workspace"},
                       {x, s.T * s.D * size, "x"}, {w_gate, s.D * s.F * size, "w_gate"}, {w_up, s.D * s.F * size, "w_up"},
                       {w_down, s.F * s.Do * size, "w_down"}};
    if ((st = check_ranges(ctx, r, 8, 4, 6u)) != TFJSB_OK) return st;
    const cudaStream_t stm = static_cast<cudaStream_t>(stream);
    if (!h && s.T <= few_rows_ffn(s.planes == 3)) {
        float* few = static_cast<float*>(workspace);
        if ((st = few_rows_gated(ctx, s.planes == 3, x, w_gate, w_up, ffn->gate, few, s.T, s.F, s.D, stm)) != TFJSB_OK) return st;
        return few_rows_down(ctx, s.planes == 3, few, w_down, y, s.T, s.Do, s.F, stm);
    }

    Arena arena{static_cast<uint8_t*>(workspace)};
    LayoutArgs layout;
    const Operand ox = operand(&layout, &arena, s.repack_x, x, s.T, s.D, s.x_bytes, s.planes);
    const Operand og = operand(&layout, &arena, s.repack_up, w_gate, s.D, s.F, s.w_bytes, s.planes);
    const Operand ou = operand(&layout, &arena, s.repack_up, w_up, s.D, s.F, s.w_bytes, s.planes);
    const Operand od = operand(&layout, &arena, s.repack_down, w_down, s.F, s.Do, s.wd_bytes, s.planes);
    if ((st = run_layout(ctx, layout, s.planes == 3, stm)) != TFJSB_OK) return st;
    void* hidden = h ? h : arena.take(s.h_bytes);

    Product up;
    up.planes = s.planes;
    up.epilogue = EPI_GATED;
    up.a = ox;
    up.b[0] = across(og, true);
    up.b[1] = across(ou, true);
    up.args.M = (int)s.T; up.args.N = (int)s.F; up.args.K = (int)s.D;
    up.args.out[0] = hidden;
    up.args.out_pitch = s.fp;
    up.args.out_plane = s.T * s.fp;
    up.args.z = static_cast<float*>(z);
    up.args.z_pitch = s.fp;
    up.args.gate = ffn->gate;
    if ((st = run_product(ctx, up, stm)) != TFJSB_OK) return st;

    Product down;
    down.planes = s.planes;
    down.a = stored(hidden, s.fp, s.T * s.fp, s.planes);
    down.b[0] = across(od, true);
    down.args.M = (int)s.T; down.args.N = (int)s.Do; down.args.K = (int)s.F;
    down.args.out[0] = y;
    down.args.out_pitch = s.Do;
    down.args.early_b = 1;  // the weights, or their copy, which was made before the product before
    return run_product(ctx, down, stm);
}

tfjsb_status tfjsb_gated_ffn_backprop(tfjsb_ctx* ctx, const tfjsb_ffn* ffn, const void* x, const void* w_gate, const void* w_up, const void* w_down,
                                      const void* h, const void* z, const void* dy, void* dx, void* dw_gate, void* dw_up, void* dw_down,
                                      void* workspace, int64_t workspace_bytes, void* stream) {
    if (!ctx) return TFJSB_ERR_INVALID_ARG;
    const dense::OnDevice on(ctx);
    ran().count = 0;
    Sizes s;
    std::string why;
    tfjsb_status st = sizes_of(ffn, &s, &why);
    if (st != TFJSB_OK) return fail(ctx, st, why);
    if (workspace_bytes < s.backward) return fail(ctx, TFJSB_ERR_INVALID_ARG, "the workspace needs " + std::to_string(s.backward) + " bytes");
    const int64_t size = s.planes == 3 ? 4 : 2;
    const Range r[] = {{dx, s.T * s.D * size, "dx"}, {dw_gate, s.D * s.F * size, "dw_gate"}, {dw_up, s.D * s.F * size, "dw_up"},
                       {dw_down, s.F * s.Do * size, "dw_down"}, {workspace, s.backward, "workspace"}, {x, s.T * s.D * size, "x"},
                       {w_gate, s.D * s.F * size, "w_gate"}, {w_up, s.D * s.F * size, "w_up"}, {w_down, s.F * s.Do * size, "w_down"},
                       {h, s.h_bytes, "h"}, {z, s.z_bytes, "z"}, {dy, s.T * s.Do * size, "dy"}};
    if ((st = check_ranges(ctx, r, 12, 5, 15u)) != TFJSB_OK) return st;
    const cudaStream_t stm = static_cast<cudaStream_t>(stream);
    if (s.T == 0) {  // sums of nothing
        for (int i = 1; i < 4; ++i) {
            if (!r[i].p) continue;
            const cudaError_t e = cudaMemsetAsync(const_cast<void*>(r[i].p), 0, (size_t)r[i].bytes, stm);
            if (e != cudaSuccess) return cuda_fail(ctx, e, "memset");
        }
        return TFJSB_OK;
    }
    const bool hidden_grads = dx || dw_gate || dw_up;
    if (!hidden_grads && !dw_down) return TFJSB_OK;

    Arena arena{static_cast<uint8_t*>(workspace)};
    LayoutArgs layout;
    Operand ox, og, ou, od;
    const Operand ody = operand(&layout, &arena, s.repack_dy, dy, s.T, s.Do, s.dy_bytes, s.planes);
    if (dw_gate || dw_up) ox = operand(&layout, &arena, s.repack_x, x, s.T, s.D, s.x_bytes, s.planes);
    if (dx) og = operand(&layout, &arena, s.repack_up, w_gate, s.D, s.F, s.w_bytes, s.planes);
    if (dx) ou = operand(&layout, &arena, s.repack_up, w_up, s.D, s.F, s.w_bytes, s.planes);
    if (hidden_grads) od = operand(&layout, &arena, s.repack_down, w_down, s.F, s.Do, s.wd_bytes, s.planes);
    if ((st = run_layout(ctx, layout, s.planes == 3, stm)) != TFJSB_OK) return st;
    const int64_t plane = s.T * s.fp;

    // The order leaves a kernel between those that write and read the same, so that each may start while the one before ends: the
    // gradients of g and u, that of w_down (of h and dy alone), those of x and of the other weights.
    __nv_bfloat16* grads = arena.take(s.grad_bytes);  // dg, then du: `planes` planes each
    if (hidden_grads) {
        Product dh;
        dh.planes = s.planes;
        dh.epilogue = EPI_GRAD;
        dh.a = ody;
        dh.b[0] = od;
        dh.args.M = (int)s.T; dh.args.N = (int)s.F; dh.args.K = (int)s.Do;
        dh.args.out[0] = grads;
        dh.args.out_pitch = s.fp;
        dh.args.out_plane = plane;
        dh.args.z = const_cast<float*>(static_cast<const float*>(z));
        dh.args.z_pitch = s.fp;
        dh.args.gate = ffn->gate;
        if ((st = run_product(ctx, dh, stm)) != TFJSB_OK) return st;
    }
    if (dw_down) {
        Product p;
        p.planes = s.planes;
        p.a = across(stored(h, s.fp, plane, s.planes), true);
        p.b[0] = across(ody, true);
        p.args.M = (int)s.F; p.args.N = (int)s.Do; p.args.K = (int)s.T;
        p.args.out[0] = dw_down;
        p.args.out_pitch = s.Do;
        p.args.early_a = p.args.early_b = hidden_grads;
        if ((st = run_product(ctx, p, stm)) != TFJSB_OK) return st;
    }
    if (dx) {
        Product p;
        p.planes = s.planes;
        p.a = stored(grads, s.fp, plane, 2 * s.planes);
        p.b[0] = og;
        p.b[1] = ou;
        p.args.passes = 2;
        p.args.M = (int)s.T; p.args.N = (int)s.D; p.args.K = (int)s.F;
        p.args.out[0] = dx;
        p.args.out_pitch = s.D;
        p.args.early_a = dw_down != nullptr;
        p.args.early_b = 1;
        if ((st = run_product(ctx, p, stm)) != TFJSB_OK) return st;
    }
    if (dw_gate || dw_up) {
        const int outputs = dw_gate && dw_up ? 2 : 1;
        Product p;
        p.planes = s.planes;
        p.a = across(ox, true);
        p.b[0] = across(stored(grads + (dw_gate ? 0 : s.planes * plane), s.fp, plane, outputs * s.planes), true);
        p.args.outputs = outputs;
        p.args.M = (int)s.D; p.args.N = (int)s.F; p.args.K = (int)s.T;
        p.args.out[0] = dw_gate ? dw_gate : dw_up;
        p.args.out[1] = dw_up;
        p.args.out_pitch = s.F;
        p.args.early_a = 1;
        p.args.early_b = dw_down || dx;
        if ((st = run_product(ctx, p, stm)) != TFJSB_OK) return st;
    }
    return TFJSB_OK;
}

}  // extern "C"
