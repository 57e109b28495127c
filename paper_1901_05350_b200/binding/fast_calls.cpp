// The op calls of the Python binding, marshalled in C++.
//
// A ctypes call with its argument structs, torch.empty and the stream lookup cost 12-16 us of host time, several times
// what the launch itself takes and more than most small ops run on the GPU; the same steps on the C++ side of torch take
// about 2 us.  Every function takes the context's handle as an integer and returns the output tensor, or None whenever an
// argument is not the plain case (contiguous fp32 CUDA tensors of rank 1..4, whole-number options): the caller then takes
// the ctypes path, which raises what there is to raise.  An error that the library reports is raised from here and the
// call is not repeated: a model run, or a call that packs or transposes an operand first, may have enqueued a part of it.
// The library is called through addresses that the caller hands over once, so both paths use one copy of it.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>

#include "tfjsb.h"

namespace {

#define FAST_CALLS(X)                                                                                                        \
    X(tfjsb_matmul) X(tfjsb_batch_matmul) X(tfjsb_conv2d) X(tfjsb_depthwise_conv2d) X(tfjsb_avg_pool) X(tfjsb_max_pool)       \
    X(tfjsb_binary) X(tfjsb_softmax) X(tfjsb_bias_act) X(tfjsb_conv2d_backprop_input) X(tfjsb_conv2d_backprop_filter)         \
    X(tfjsb_depthwise_conv2d_backprop_input) X(tfjsb_depthwise_conv2d_backprop_filter) X(tfjsb_act_backprop)                  \
    X(tfjsb_bias_backprop) X(tfjsb_run_model) X(tfjsb_model_layer_output_f32) X(tfjsb_model_layer_shape) X(tfjsb_window_out_shape)       \
    X(tfjsb_last_error) X(tfjsb_gated_ffn_sizes) X(tfjsb_gated_ffn) X(tfjsb_gated_ffn_backprop) X(tfjsb_dropout) X(tfjsb_dropout_backprop) X(tfjsb_dense_int8_workspace) X(tfjsb_dense_int8)
#define DECLARE(name) decltype(&::name) p_##name = nullptr;
FAST_CALLS(DECLARE)
#undef DECLARE
PyObject* error_type = nullptr;  // called with (status, message)

// An argument list read from left to right; `ok` turns false at the first argument that is not the plain case.
struct Args {
    PyObject* const* at;
    PyObject* const* end;
    bool ok;
    Args(PyObject* const* args, Py_ssize_t n, Py_ssize_t want) : at(args), end(args + n), ok(n == want) {}

    PyObject* next() { return ok ? *at++ : nullptr; }
    long long integer() {
        PyObject* o = next();
        if (!o || !PyLong_Check(o)) { ok = false; return 0; }  // bool is a PyLong
        int overflow = 0;
        const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
        if (overflow) ok = false;
        return v;
    }
    void* handle() {
        PyObject* o = next();
        if (!o || !PyLong_Check(o)) { ok = false; return nullptr; }
        void* p = PyLong_AsVoidPtr(o);
        if (!p) { PyErr_Clear(); ok = false; }
        return p;
    }
    void tensor(tfjsb_tensor* d) {
        PyObject* o = next();
        if (!o || !THPVariable_Check(o)) { ok = false; return; }
        const at::Tensor& t = THPVariable_Unpack(o);
        const int64_t rank = t.dim();
        if (rank < 1 || rank > 4 || !t.is_cuda() || t.scalar_type() != at::kFloat || !t.is_contiguous()) { ok = false; return; }
        d->data = const_cast<void*>(t.const_data_ptr());
        d->rank = (int32_t)rank;
        for (int64_t i = 0; i < rank; ++i) d->dims[i] = t.size(i);
    }
    // a tensor, or None
    const tfjsb_tensor* maybe(tfjsb_tensor* d) {
        if (!ok) return nullptr;
        if (*at == Py_None) { ++at; return nullptr; }
        tensor(d);
        return d;
    }
    // a tuple or list of `count` whole numbers (1..4 of them when count is 0); returns how many
    int integers(int64_t* v, int count) {
        PyObject* o = next();
        const bool tuple = o && PyTuple_Check(o);
        if (!tuple && !(o && PyList_Check(o))) { ok = false; return 0; }
        const Py_ssize_t n = tuple ? PyTuple_GET_SIZE(o) : PyList_GET_SIZE(o);
        if (count ? n != count : (n < 1 || n > 4)) { ok = false; return 0; }
        for (Py_ssize_t i = 0; i < n; ++i) {
            PyObject* e = tuple ? PyTuple_GET_ITEM(o, i) : PyList_GET_ITEM(o, i);
            if (!PyLong_Check(e)) { ok = false; return 0; }
            int overflow = 0;
            v[i] = PyLong_AsLongLongAndOverflow(e, &overflow);
            if (overflow) { ok = false; return 0; }
        }
        return (int)n;
    }
    void pair(int v[2]) {
        int64_t w[2] = {0, 0};
        integers(w, 2);
        for (int i = 0; i < 2; ++i) {
            v[i] = (int)w[i];
            if (v[i] != w[i]) ok = false;
        }
    }
};

// The output: the tensor that the caller passed, or a new one of the given shape.
struct Out {
    PyObject* given = nullptr;
    at::TensorBase made;
    tfjsb_tensor desc;

    bool take(Args& a) {  // the `out` argument; whether one was given
        if (!a.ok) return false;
        if (*a.at == Py_None) { ++a.at; return false; }
        given = *a.at;
        a.tensor(&desc);
        return true;
    }
    void make(Args& a, int device, const int64_t* dims, int rank) {
        for (int i = 0; i < rank; ++i)
            if (dims[i] < 0) a.ok = false;
        if (!a.ok || rank < 1 || rank > 4) { a.ok = false; return; }
        made = at::detail::empty_cuda(at::IntArrayRef(dims, rank), at::kFloat, at::Device(at::kCUDA, (at::DeviceIndex)device), std::nullopt);
        desc.data = const_cast<void*>(made.const_data_ptr());
        desc.rank = rank;
        for (int i = 0; i < rank; ++i) desc.dims[i] = dims[i];
    }
    PyObject* done(tfjsb_ctx* ctx, tfjsb_status st) {
        if (st != TFJSB_OK) {
            PyObject* error = PyObject_CallFunction(error_type, "is", (int)st, p_tfjsb_last_error(ctx));
            if (error) PyErr_SetObject(error_type, error);
            Py_XDECREF(error);
            return nullptr;
        }
        if (given) { Py_INCREF(given); return given; }
        return THPVariable_Wrap(std::move(made));
    }
};

void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

// The library call without the interpreter lock, as ctypes makes it.
template <typename F>
tfjsb_status unlocked(F f) {
    tfjsb_status st;
    Py_BEGIN_ALLOW_THREADS st = f();
    Py_END_ALLOW_THREADS return st;
}

// The Python entry point of an op with N arguments.  What is thrown in it (by an allocation, say), before the library is
// called, goes wrong again on the ctypes path, which reports it.
template <PyObject* (*OP)(Args&), int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    try {
        Args a(args, n, N);
        if (!a.ok) Py_RETURN_NONE;
        return OP(a);
    } catch (...) {
        if (PyErr_Occurred()) PyErr_Clear();
        Py_RETURN_NONE;
    }
}

PyObject* bind(PyObject*, PyObject* args) {  // {name: address}, the type of the errors
    PyObject *addresses, *type;
    if (!PyArg_ParseTuple(args, "O!O", &PyDict_Type, &addresses, &type)) return nullptr;
    Py_INCREF(type);
    Py_XSETREF(error_type, type);
#define TAKE(name)                                                                         \
    {                                                                                      \
        PyObject* o = PyDict_GetItemString(addresses, #name);                              \
        void* p = o ? PyLong_AsVoidPtr(o) : nullptr;                                       \
        if (!p) return PyErr_Format(PyExc_KeyError, "no address for " #name);              \
        std::memcpy(&p_##name, &p, sizeof p);                                              \
    }
    FAST_CALLS(TAKE)
#undef TAKE
    Py_RETURN_NONE;
}

// Every op begins with (handle, device, ...) and ends with `out`.
struct Head {
    tfjsb_ctx* ctx;
    int device;
    explicit Head(Args& a) : ctx(static_cast<tfjsb_ctx*>(a.handle())), device((int)a.integer()) {}
};

// matmul(ctx, device, a, b, transpose_a, transpose_b, out) and the rank-3 form
template <bool BATCH>
PyObject* matmul(Args& a) {
    const Head h(a);
    tfjsb_tensor ta, tb;
    Out out;
    a.tensor(&ta);
    a.tensor(&tb);
    const int x = a.integer() != 0, y = a.integer() != 0;
    constexpr int L = BATCH ? 1 : 0;
    const bool given = out.take(a);
    if (!a.ok || ta.rank != 2 + L || tb.rank != 2 + L) Py_RETURN_NONE;
    if (!given) {
        const int64_t d[3] = {BATCH ? ta.dims[0] : ta.dims[x], BATCH ? ta.dims[1 + x] : tb.dims[1 - y], BATCH ? tb.dims[2 - y] : 0};
        out.make(a, h.device, d, 2 + L);
    }
    if (!a.ok) Py_RETURN_NONE;
    void* s = stream();
    return out.done(h.ctx, unlocked([&] { return (BATCH ? p_tfjsb_batch_matmul : p_tfjsb_matmul)(h.ctx, &ta, &tb, x, y, &out.desc, s); }));
}

bool window_shape(const tfjsb_tensor& x, const int64_t size[2], const int strides[2], int pad, const int dilations[2], int64_t channels,
                  int64_t d[4]) {
    if (x.rank != 4 || size[0] != (int)size[0] || size[1] != (int)size[1]) return false;
    d[0] = x.dims[0];
    d[3] = channels;
    for (int i = 0; i < 2; ++i)
        if (p_tfjsb_window_out_shape(x.dims[1 + i], (int)size[i], strides[i], dilations[i], (tfjsb_pad)pad, &d[1 + i], nullptr, nullptr) != TFJSB_OK)
            return false;
    return true;
}

// conv2d(ctx, device, x, filter, strides, pad, dilations, bias, act, out) and the depthwise form
template <bool DEPTHWISE>
PyObject* conv2d(Args& a) {
    const Head h(a);
    tfjsb_tensor x, f, b;
    Out out;
    int st[2], dl[2];
    a.tensor(&x);
    a.tensor(&f);
    a.pair(st);
    const int pad = (int)a.integer();
    a.pair(dl);
    const tfjsb_tensor* bias = a.maybe(&b);
    const int act = (int)a.integer();
    const bool given = out.take(a);
    if (!a.ok || f.rank != 4) Py_RETURN_NONE;
    if (!given) {
        int64_t d[4];
        if (!window_shape(x, f.dims, st, pad, dl, DEPTHWISE ? f.dims[2] * f.dims[3] : f.dims[3], d)) Py_RETURN_NONE;
        out.make(a, h.device, d, 4);
    }
    if (!a.ok) Py_RETURN_NONE;
    void* s = stream();
    return out.done(h.ctx, unlocked([&] {
        return (DEPTHWISE ? p_tfjsb_depthwise_conv2d : p_tfjsb_conv2d)(h.ctx, &x, &f, st, (tfjsb_pad)pad, dl, bias, (tfjsb_act)act, &out.desc, s);
    }));
}

// avg_pool / max_pool(ctx, device, x, filter_size, strides, pad, out)
template <bool MAX>
PyObject* pool(Args& a) {
    const Head h(a);
    tfjsb_tensor x;
    Out out;
    int size[2], st[2];
    const int one[2] = {1, 1};
    a.tensor(&x);
    a.pair(size);
    a.pair(st);
    const int pad = (int)a.integer();
    const bool given = out.take(a);
    if (!a.ok || x.rank != 4) Py_RETURN_NONE;
    if (!given) {
        const int64_t w[2] = {size[0], size[1]};
        int64_t d[4];
        if (!window_shape(x, w, st, pad, one, x.dims[3], d)) Py_RETURN_NONE;
        out.make(a, h.device, d, 4);
    }
    if (!a.ok) Py_RETURN_NONE;
    void* s = stream();
    return out.done(h.ctx, unlocked([&] { return (MAX ? p_tfjsb_max_pool : p_tfjsb_avg_pool)(h.ctx, &x, size, st, (tfjsb_pad)pad, &out.desc, s); }));
}

// binary(ctx, device, op, a, b, out)
PyObject* binary(Args& a) {
    const Head h(a);
    tfjsb_tensor u, v;
    Out out;
    const int op = (int)a.integer();
    a.tensor(&u);
    a.tensor(&v);
    if (!out.take(a) && a.ok) out.make(a, h.device, u.dims, u.rank);
    if (!a.ok) Py_RETURN_NONE;
    void* s = stream();
    return out.done(h.ctx, unlocked([&] { return p_tfjsb_binary(h.ctx, (tfjsb_binary_op)op, &u, &v, &out.desc, s); }));
}

// softmax(ctx, device, logits, out)
PyObject* softmax(Args& a) {
    const Head h(a);
    tfjsb_tensor x;
    Out out;
    a.tensor(&x);
    if (!out.take(a) && a.ok) out.make(a, h.device, x.dims, x.rank);
    if (!a.ok) Py_RETURN_NONE;
    void* s = stream();
    return out.done(h.ctx, unlocked([&] { return p_tfjsb_softmax(h.ctx, &x, &out.desc, s); }));
}

// bias_act(ctx, device, x, bias, act, out)
PyObject* bias_act(Args& a) {
    const Head h(a);
    tfjsb_tensor x, b;
    Out out;
    a.tensor(&x);
    const tfjsb_tensor* bias = a.maybe(&b);
    const int act = (int)a.integer();
    if (!out.take(a) && a.ok) out.make(a, h.device, x.dims, x.rank);
    if (!a.ok) Py_RETURN_NONE;
    void* s = stream();
    return out.done(h.ctx, unlocked([&] { return p_tfjsb_bias_act(h.ctx, &x, bias, (tfjsb_act)act, &out.desc, s); }));
}

// conv_grad(ctx, device, which, shape of the result, first, second, strides, pad, dilations, out): which = 0 conv2d input
// (dy, filter), 1 conv2d filter (x, dy), 2 and 3 the depthwise pair
PyObject* conv_grad(Args& a) {
    const Head h(a);
    tfjsb_tensor u, v;
    Out out;
    int st[2], dl[2];
    int64_t d[4];
    const int which = (int)a.integer();
    const int rank = a.integers(d, 0);
    a.tensor(&u);
    a.tensor(&v);
    a.pair(st);
    const int pad = (int)a.integer();
    a.pair(dl);
    if (!out.take(a) && a.ok) out.make(a, h.device, d, rank);
    if (!a.ok) Py_RETURN_NONE;
    const auto call = which == 0   ? p_tfjsb_conv2d_backprop_input
                      : which == 1 ? p_tfjsb_conv2d_backprop_filter
                      : which == 2 ? p_tfjsb_depthwise_conv2d_backprop_input
                                   : p_tfjsb_depthwise_conv2d_backprop_filter;
    void* s = stream();
    return out.done(h.ctx, unlocked([&] { return call(h.ctx, &u, &v, st, (tfjsb_pad)pad, dl, &out.desc, s); }));
}

// act_backprop(ctx, device, y, dy, act, out)
PyObject* act_backprop(Args& a) {
    const Head h(a);
    tfjsb_tensor y, g;
    Out out;
    a.tensor(&y);
    a.tensor(&g);
    const int act = (int)a.integer();
    if (!out.take(a) && a.ok) out.make(a, h.device, y.dims, y.rank);
    if (!a.ok) Py_RETURN_NONE;
    void* s = stream();
    return out.done(h.ctx, unlocked([&] { return p_tfjsb_act_backprop(h.ctx, &y, &g, (tfjsb_act)act, &out.desc, s); }));
}

// bias_backprop(ctx, device, dz, out)
PyObject* bias_backprop(Args& a) {
    const Head h(a);
    tfjsb_tensor g;
    Out out;
    a.tensor(&g);
    if (!out.take(a) && a.ok) out.make(a, h.device, &g.dims[g.rank - 1], 1);
    if (!a.ok) Py_RETURN_NONE;
    void* s = stream();
    return out.done(h.ctx, unlocked([&] { return p_tfjsb_bias_backprop(h.ctx, &g, &out.desc, s); }));
}

// run_model(ctx, device, model, x, output shape, out)
PyObject* run_model(Args& a) {
    const Head h(a);
    auto* m = static_cast<tfjsb_model*>(a.handle());
    tfjsb_tensor x;
    Out out;
    int64_t d[4];
    a.tensor(&x);
    const int rank = a.integers(d, 0);
    if (!out.take(a) && a.ok) out.make(a, h.device, d, rank);
    if (!a.ok) Py_RETURN_NONE;
    void* s = stream();
    return out.done(h.ctx, unlocked([&] { return p_tfjsb_run_model(m, &x, &out.desc, s); }));
}

// layer_output_f32(ctx, device, model, layer)
PyObject* layer_output_f32(Args& a) {
    const Head h(a);
    auto* m = static_cast<tfjsb_model*>(a.handle());
    const int layer = (int)a.integer();
    Out out;
    int32_t rank = 0;
    int64_t d[4];
    if (!a.ok || p_tfjsb_model_layer_shape(m, layer, &rank, d) != TFJSB_OK) Py_RETURN_NONE;
    out.make(a, h.device, d, rank);
    if (!a.ok) Py_RETURN_NONE;
    void* s = stream();
    return out.done(h.ctx, unlocked([&] { return p_tfjsb_model_layer_output_f32(m, layer, static_cast<float*>(out.desc.data), s); }));
}

// ---- dense layers of transformer blocks: contiguous tensors of fp32 or bfloat16 on the context's device ----

// A tensor of such a call; `dtype` receives its tfjsb_dtype, or has to agree with it when it is not negative.
const at::Tensor* dense_tensor(Args& a, int device, int* dtype) {
    PyObject* o = a.next();
    if (!o || !THPVariable_Check(o)) { a.ok = false; return nullptr; }
    const at::Tensor& t = THPVariable_Unpack(o);
    const int is = t.scalar_type() == at::kFloat ? TFJSB_DTYPE_F32 : t.scalar_type() == at::kBFloat16 ? TFJSB_DTYPE_BF16 : -1;
    if (is < 0 || (*dtype >= 0 && *dtype != is) || !t.is_cuda() || t.get_device() != device || !t.is_contiguous()) { a.ok = false; return nullptr; }
    *dtype = is;
    return &t;
}
bool has_shape(const at::Tensor& t, int64_t rows, int64_t columns) { return t.dim() == 2 && t.size(0) == rows && t.size(1) == columns; }
at::TensorBase new_tensor(at::IntArrayRef shape, at::ScalarType type, int device) {
    return at::detail::empty_cuda(shape, type, at::Device(at::kCUDA, (at::DeviceIndex)device), std::nullopt);
}
at::ScalarType scalar_of(int dtype) { return dtype == TFJSB_DTYPE_F32 ? at::kFloat : at::kBFloat16; }

// The output of such a call: the tensor that the caller passed, which has to have the shape, or a new one.
struct DenseOut {
    PyObject* given = nullptr;
    at::TensorBase made;
    void* data = nullptr;
    void take(Args& a, int device, at::IntArrayRef shape, int* dtype) {
        if (!a.ok) return;
        if (*a.at == Py_None) {
            ++a.at;
            made = new_tensor(shape, scalar_of(*dtype), device);
            data = const_cast<void*>(made.const_data_ptr());
            return;
        }
        given = *a.at;
        const at::Tensor* t = dense_tensor(a, device, dtype);
        if (!t || t->sizes() != shape) { a.ok = false; return; }
        data = const_cast<void*>(t->const_data_ptr());
    }
    PyObject* done(tfjsb_ctx* ctx, tfjsb_status st) {
        Out o;
        o.given = given;
        o.made = std::move(made);
        return o.done(ctx, st);
    }
};

// x, w_gate, w_up, w_down and the gate of a gated feed-forward call.
struct FfnArgs {
    const at::Tensor* t[4];
    int dtype = -1;
    tfjsb_ffn f{};
    int64_t h_bytes = 0, z_bytes = 0, work_bytes = 0, grad_work_bytes = 0;
    int64_t y_shape[8];

    at::IntArrayRef y() const { return at::IntArrayRef(y_shape, t[0]->dim()); }
    bool take(Args& a, int device) {  // the tensors
        for (auto& p : t) {
            p = dense_tensor(a, device, &dtype);
            if (!p) return false;
        }
        return true;
    }
    bool shapes(int gate) {
        const at::Tensor& x = *t[0];
        if (x.dim() < 1 || x.dim() > 8 || t[1]->dim() != 2 || t[3]->dim() != 2) return false;
        const int64_t width = x.size(-1), hidden = t[1]->size(1), out_width = t[3]->size(1);
        if (width < 1 || !has_shape(*t[1], width, hidden) || !has_shape(*t[2], width, hidden) || !has_shape(*t[3], hidden, out_width)) return false;
        f = {x.numel() / width, width, hidden, out_width, dtype, gate};
        for (int64_t i = 0; i < x.dim(); ++i) y_shape[i] = x.size(i);
        y_shape[x.dim() - 1] = out_width;
        return f.tokens > 0 && p_tfjsb_gated_ffn_sizes(&f, &h_bytes, &z_bytes, &work_bytes, &grad_work_bytes) == TFJSB_OK;
    }
    const void* data(int i) const { return t[i]->const_data_ptr(); }
};
void* writable(const at::TensorBase& t) { return const_cast<void*>(t.const_data_ptr()); }

// gated_ffn(ctx, device, x, w_gate, w_up, w_down, gate, save, out): y, or (y, h, z)
PyObject* gated_ffn(Args& a) {
    const Head h(a);
    FfnArgs in;
    if (!in.take(a, h.device)) Py_RETURN_NONE;
    const int gate = (int)a.integer(), save = (int)a.integer();
    if (!a.ok || !in.shapes(gate)) Py_RETURN_NONE;
    DenseOut out;
    out.take(a, h.device, in.y(), &in.dtype);
    if (!a.ok) Py_RETURN_NONE;
    at::TensorBase kept[2];
    if (save) {
        kept[0] = new_tensor({in.h_bytes}, at::kByte, h.device);
        kept[1] = new_tensor({in.z_bytes}, at::kByte, h.device);
    }
    const at::TensorBase work = new_tensor({in.work_bytes}, at::kByte, h.device);
    void* s = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)h.device).stream();
    const tfjsb_status st = unlocked([&] {
        return p_tfjsb_gated_ffn(h.ctx, &in.f, in.data(0), in.data(1), in.data(2), in.data(3), out.data, save ? writable(kept[0]) : nullptr,
                                 save ? writable(kept[1]) : nullptr, writable(work), in.work_bytes, s);
    });
    PyObject* y = out.done(h.ctx, st);
    if (!y || !save) return y;
    PyObject* all = PyTuple_New(3);
    if (!all) { Py_DECREF(y); return nullptr; }
    PyTuple_SET_ITEM(all, 0, y);
    for (int i = 0; i < 2; ++i) PyTuple_SET_ITEM(all, 1 + i, THPVariable_Wrap(std::move(kept[i])));
    return all;
}

// gated_ffn_backprop(ctx, device, x, w_gate, w_up, w_down, h, z, dy, gate): the four gradients
PyObject* gated_ffn_backprop(Args& a) {
    const Head h(a);
    FfnArgs in;
    if (!in.take(a, h.device)) Py_RETURN_NONE;
    const at::Tensor* kept[2];
    for (auto& p : kept) {
        PyObject* o = a.next();
        if (!o || !THPVariable_Check(o)) Py_RETURN_NONE;
        p = &THPVariable_Unpack(o);
        if (p->scalar_type() != at::kByte || !p->is_cuda() || p->get_device() != h.device || !p->is_contiguous()) Py_RETURN_NONE;
    }
    const at::Tensor* dy = dense_tensor(a, h.device, &in.dtype);
    const int gate = (int)a.integer();
    if (!a.ok || !in.shapes(gate) || dy->sizes() != in.y() || kept[0]->numel() != in.h_bytes || kept[1]->numel() != in.z_bytes) Py_RETURN_NONE;
    at::TensorBase grads[4];
    for (int i = 0; i < 4; ++i) grads[i] = new_tensor(in.t[i]->sizes(), scalar_of(in.dtype), h.device);
    const at::TensorBase work = new_tensor({in.grad_work_bytes}, at::kByte, h.device);
    void* s = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)h.device).stream();
    const tfjsb_status st = unlocked([&] {
        return p_tfjsb_gated_ffn_backprop(h.ctx, &in.f, in.data(0), in.data(1), in.data(2), in.data(3), kept[0]->const_data_ptr(), kept[1]->const_data_ptr(),
                                          dy->const_data_ptr(), writable(grads[0]), writable(grads[1]), writable(grads[2]), writable(grads[3]),
                                          writable(work), in.grad_work_bytes, s);
    });
    if (st != TFJSB_OK) return Out().done(h.ctx, st);
    PyObject* all = PyTuple_New(4);
    if (!all) return nullptr;
    for (int i = 0; i < 4; ++i) PyTuple_SET_ITEM(all, i, THPVariable_Wrap(std::move(grads[i])));
    return all;
}

// dropout(ctx, device, x, rate, seed, offset, noise shape or None, residual or None, out); of the gradient without the residual
template <bool BACKPROP>
PyObject* dropout_of(Args& a) {
    const Head h(a);
    int dtype = -1;
    const at::Tensor* x = dense_tensor(a, h.device, &dtype);
    PyObject* rate = a.next();
    if (!x || !rate || !PyFloat_CheckExact(rate) || x->dim() < 1 || x->dim() > 4 || x->numel() == 0) Py_RETURN_NONE;
    uint64_t word[2];
    for (auto& w : word) {
        PyObject* o = a.next();
        if (!o || !PyLong_CheckExact(o)) Py_RETURN_NONE;
        w = PyLong_AsUnsignedLongLong(o);
        if (PyErr_Occurred()) { PyErr_Clear(); Py_RETURN_NONE; }
    }
    int64_t noise[4];
    const bool shared = a.ok && *a.at != Py_None;
    if (!shared) ++a.at;
    else if (a.integers(noise, (int)x->dim()) != x->dim()) Py_RETURN_NONE;
    if (!a.ok) Py_RETURN_NONE;
    const at::Tensor* residual = nullptr;
    if (BACKPROP) {}
    else if (*a.at == Py_None) ++a.at;
    else if (!(residual = dense_tensor(a, h.device, &dtype)) || residual->sizes() != x->sizes()) Py_RETURN_NONE;
    DenseOut out;
    out.take(a, h.device, x->sizes(), &dtype);
    if (!a.ok) Py_RETURN_NONE;
    void* s = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)h.device).stream();
    const double r = PyFloat_AS_DOUBLE(rate);
    return out.done(h.ctx, unlocked([&] {
        if (BACKPROP)
            return p_tfjsb_dropout_backprop(h.ctx, (tfjsb_dtype)dtype, x->const_data_ptr(), out.data, (int32_t)x->dim(), x->sizes().data(),
                                            shared ? noise : nullptr, r, word[0], word[1], s);
        return p_tfjsb_dropout(h.ctx, (tfjsb_dtype)dtype, x->const_data_ptr(), residual ? residual->const_data_ptr() : nullptr, out.data, (int32_t)x->dim(),
                               x->sizes().data(), shared ? noise : nullptr, r, word[0], word[1], s);
    }));
}

PyObject* dropout(Args& a) { return dropout_of<false>(a); }
PyObject* dropout_backprop(Args& a) { return dropout_of<true>(a); }

// dense_int8(ctx, device, x, bt, bt_scale, bias or None, act, out dtype (None: x's), out)
PyObject* dense_int8(Args& a) {
    const Head h(a);
    int dtype = -1, f32 = TFJSB_DTYPE_F32;
    const at::Tensor* x = dense_tensor(a, h.device, &dtype);
    PyObject* o = a.next();
    if (!x || x->dim() != 2 || !o || !THPVariable_Check(o)) Py_RETURN_NONE;
    const at::Tensor& bt = THPVariable_Unpack(o);
    const int64_t M = x->size(0), K = x->size(1);
    if (M < 1 || K < 1 || bt.scalar_type() != at::kChar || !bt.is_cuda() || bt.get_device() != h.device || !bt.is_contiguous() || bt.dim() != 2 ||
        bt.size(1) != (K + 15) / 16 * 16)
        Py_RETURN_NONE;
    const int64_t N = bt.size(0);
    const at::Tensor* scale = dense_tensor(a, h.device, &f32);
    if (!scale || scale->dim() != 1 || scale->size(0) != N || N < 1) Py_RETURN_NONE;
    const at::Tensor* bias = nullptr;
    if (*a.at == Py_None) ++a.at;
    else if (!(bias = dense_tensor(a, h.device, &f32)) || bias->dim() != 1 || bias->size(0) != N) Py_RETURN_NONE;
    const int act = (int)a.integer();
    if (!a.ok || a.next() != Py_None) Py_RETURN_NONE;
    int to = dtype;
    DenseOut out;
    if (*a.at != Py_None) to = -1;  // the dtype of the tensor that is given
    out.take(a, h.device, {M, N}, &to);
    const int64_t bytes = p_tfjsb_dense_int8_workspace(M, K);
    if (!a.ok || bytes < 1) Py_RETURN_NONE;
    const at::TensorBase work = new_tensor({bytes}, at::kByte, h.device);
    void* s = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)h.device).stream();
    return out.done(h.ctx, unlocked([&] {
        return p_tfjsb_dense_int8(h.ctx, (tfjsb_dtype)dtype, x->const_data_ptr(), static_cast<const int8_t*>(bt.const_data_ptr()),
                                  static_cast<const float*>(scale->const_data_ptr()), bias ? static_cast<const float*>(bias->const_data_ptr()) : nullptr,
                                  (tfjsb_act)act, out.data, (tfjsb_dtype)to, M, N, K, const_cast<void*>(work.const_data_ptr()), bytes, s);
    }));
}

#define METHOD(name, op, n) {name, (PyCFunction)(void (*)(void))(&entry<op, n>), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    METHOD("matmul", matmul<false>, 7),
    METHOD("batch_matmul", matmul<true>, 7),
    METHOD("conv2d", conv2d<false>, 10),
    METHOD("depthwise_conv2d", conv2d<true>, 10),
    METHOD("avg_pool", pool<false>, 7),
    METHOD("max_pool", pool<true>, 7),
    METHOD("binary", binary, 6),
    METHOD("softmax", softmax, 4),
    METHOD("bias_act", bias_act, 6),
    METHOD("conv_grad", conv_grad, 10),
    METHOD("act_backprop", act_backprop, 6),
    METHOD("bias_backprop", bias_backprop, 4),
    METHOD("run_model", run_model, 6),
    METHOD("layer_output_f32", layer_output_f32, 4),
    METHOD("gated_ffn", gated_ffn, 9),
    METHOD("gated_ffn_backprop", gated_ffn_backprop, 10),
    METHOD("dropout", dropout, 9),
    METHOD("dropout_backprop", dropout_backprop, 8),
    METHOD("dense_int8", dense_int8, 9),
    {nullptr, nullptr, 0, nullptr},
};
#undef METHOD
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fast_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" PyObject* PyInit__fast_calls() {
    PyObject* m = PyModule_Create(&module);
    if (m) {
        PyObject* names = PyList_New(0);
#define NAME(name)                                     \
    {                                                  \
        PyObject* s = PyUnicode_FromString(#name);     \
        PyList_Append(names, s);                       \
        Py_DECREF(s);                                  \
    }
        FAST_CALLS(NAME)
#undef NAME
        PyModule_AddObject(m, "CALLS", names);
    }
    return m;
}
