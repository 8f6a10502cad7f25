// The calls of the Python binding in native code: argument checks, output allocation and the C ABI call of
// include/terra.h in one go.  The small calls (one 8 x 8-window block on a regional grid) take the GPU a few microseconds; the same
// marshalling in Python and ctypes took 15 to 40 microseconds a call, this takes about 2.
//
// No function of the library is linked: binding.py hands over the entry points of the library that it loaded.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <vector>

#include "../../include/terra.h"

namespace {

decltype(&terra_swin_workspace_bytes) f_workspace = nullptr;
decltype(&terra_swin_attn_fwd) f_fwd = nullptr;
decltype(&terra_swin_attn_bwd) f_bwd = nullptr;
decltype(&terra_swin_attn_fwd_packed) f_fwd_packed = nullptr;
decltype(&terra_swin_attn_bwd_packed) f_bwd_packed = nullptr;
decltype(&terra_swin_attn_fwd_noalloc) f_fwd_noalloc = nullptr;
decltype(&terra_rms_norm_fwd) f_norm_fwd = nullptr;
decltype(&terra_rms_norm_fwd_e4m3) f_norm_fwd_e4m3 = nullptr;
decltype(&terra_rms_norm_workspace_bytes) f_norm_workspace = nullptr;
decltype(&terra_rms_norm_bwd) f_norm_bwd = nullptr;
decltype(&terra_linear_workspace_bytes) f_linear_workspace = nullptr;
decltype(&terra_linear_fwd) f_linear_fwd = nullptr;
decltype(&terra_linear_fwd_e4m3) f_linear_fwd_e4m3 = nullptr;
decltype(&terra_linear_bwd) f_linear_bwd = nullptr;
decltype(&terra_activation_bwd) f_activation_bwd = nullptr;
decltype(&terra_rotary) f_rotary = nullptr;
decltype(&terra_rotary_packed) f_rotary_packed = nullptr;
PyObject* on_status = nullptr;          // binding._check: raises the TerraError of a status

struct Failed {};                       // a Python error is set

// Other Python threads run while this one allocates or launches: both wait for the GPU at times (a new segment of the caching
// allocator, a full launch queue).
struct NoGil {
    PyThreadState* state = PyEval_SaveThread();
    ~NoGil() { PyEval_RestoreThread(state); }
};

// The descriptor is a ctypes structure; its bytes are read through the buffer protocol.
struct Desc {
    Py_buffer view{};
    const terra_swin_desc* d = nullptr;
    explicit Desc(PyObject* o) {
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE)) throw Failed{};
        if (view.len < (Py_ssize_t)sizeof(terra_swin_desc)) {
            PyBuffer_Release(&view);
            PyErr_SetString(PyExc_TypeError, "terra: the descriptor must be a terra_swin_desc");
            throw Failed{};
        }
        d = static_cast<const terra_swin_desc*>(view.buf);
    }
    ~Desc() { if (d) PyBuffer_Release(&view); }
    int64_t rows() const { return (int64_t)d->B * d->H * d->W * d->heads; }
    int64_t table() const { return (int64_t)(2 * d->window - 1) * (2 * d->window - 1) * d->heads; }
    at::ScalarType act() const { return d->dtype == TERRA_DTYPE_F16 ? at::kHalf : at::kBFloat16; }
};

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "terra: %s must be a tensor", name);
        throw Failed{};
    }
    return THPVariable_Unpack(o);
}

const char* dtype_name(at::ScalarType t) {
    switch (t) {
        case at::kBFloat16: return "torch.bfloat16";
        case at::kHalf: return "torch.float16";
        case at::kFloat: return "torch.float32";
        case at::kDouble: return "torch.float64";
        case at::kInt: return "torch.int32";
        case at::kFloat8_e4m3fn: return "torch.float8_e4m3fn";
        default: return c10::toString(t);
    }
}

void expect(const at::Tensor& t, at::ScalarType dtype, int64_t numel, const char* name) {
    if (t.scalar_type() == dtype && t.numel() == numel) return;
    PyErr_Format(PyExc_ValueError, "terra: %s must be %s with %lld elements, got %s x %lld", name, dtype_name(dtype), (long long)numel,
                 dtype_name(t.scalar_type()), (long long)t.numel());
    throw Failed{};
}

void* ptr(const at::Tensor& t) {
    if (!t.is_cuda()) {
        PyErr_SetString(PyExc_ValueError, "terra: tensors must be CUDA tensors (the library has no CPU path)");
        throw Failed{};
    }
    if (!t.is_contiguous()) {
        PyErr_SetString(PyExc_ValueError, "terra: tensors must be contiguous");
        throw Failed{};
    }
    // the library launches on the current device (its stream, SM count and built-in scratch are that device's)
    const int current = c10::cuda::current_device();
    if (t.device().index() != current) {
        PyErr_Format(PyExc_ValueError, "terra: tensor lives on cuda:%d but the current device is cuda:%d; make the tensors' device current "
                     "(torch.cuda.device(...)) around the call", (int)t.device().index(), current);
        throw Failed{};
    }
    return t.data_ptr();
}

void check(int status) {
    if (status == TERRA_OK) return;
    PyObject* r = PyObject_CallFunction(on_status, "i", status);
    Py_XDECREF(r);
    if (!PyErr_Occurred()) PyErr_Format(PyExc_RuntimeError, "terra status %d", status);
    throw Failed{};
}

void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

// The library call (its pointers are taken before: that may raise).
template <class F, class... A>
void launch(F f, A... args) {
    int status;
    {
        NoGil no_gil;
        status = f(args...);
    }
    check(status);
}

// The caller's tensor, or a new one.
at::Tensor output(PyObject* o, const char* name, at::ScalarType dtype, at::IntArrayRef shape, const at::Tensor& like) {
    if (o != Py_None) return tensor(o, name);
    NoGil no_gil;
    return at::detail::empty_cuda(shape, dtype, like.device(), std::nullopt);
}

// The caller's workspace, or a new one of the size the call wants (an undefined tensor where it wants none).
at::Tensor workspace(PyObject* o, const Desc& desc, bool backward, const at::Tensor& like, size_t& bytes) {
    at::Tensor t;
    if (o != Py_None) {
        t = tensor(o, "workspace");
    } else {
        size_t need = 0;
        check(f_workspace(desc.d, backward, &need));
        if (need) {
            NoGil no_gil;
            t = at::detail::empty_cuda({(int64_t)need}, at::kByte, like.device(), std::nullopt);
        }
    }
    bytes = t.defined() ? t.nbytes() : 0;
    return t;
}
void* opt_ptr(const at::Tensor& t) { return t.defined() ? ptr(t) : nullptr; }

PyObject* tuple(std::initializer_list<at::Tensor> ts) {
    PyObject* r = PyTuple_New((Py_ssize_t)ts.size());
    if (!r) throw Failed{};
    Py_ssize_t i = 0;
    for (const at::Tensor& t : ts) PyTuple_SET_ITEM(r, i++, THPVariable_Wrap(t));
    return r;
}

template <class F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F body) {
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "terra: %zd arguments, %zd wanted", n, want);
        return nullptr;
    }
    try {
        return body();
    } catch (const Failed&) {
        return nullptr;
    } catch (const c10::Error& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// desc, q, k, v, bias_table, o, lse, workspace -> (o, lse)
PyObject* fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 8, [&] {
        Desc d(a[0]);
        const at::Tensor &q = tensor(a[1], "q"), &k = tensor(a[2], "k"), &v = tensor(a[3], "v"), &b = tensor(a[4], "bias_table");
        const int64_t rows = d.rows(), all = rows * d.d->head_dim;
        expect(q, d.act(), all, "q"); expect(k, d.act(), all, "k"); expect(v, d.act(), all, "v");
        expect(b, at::kFloat, d.table(), "bias_table");
        void *pq = ptr(q), *pk = ptr(k), *pv = ptr(v), *pb = ptr(b);
        at::Tensor o = output(a[5], "o", d.act(), q.sizes(), q);
        at::Tensor lse = output(a[6], "lse", at::kFloat, {d.d->B, d.d->H, d.d->W, d.d->heads}, q);
        expect(o, d.act(), all, "o"); expect(lse, at::kFloat, rows, "lse");
        size_t bytes;
        at::Tensor ws = workspace(a[7], d, false, q, bytes);
        launch(f_fwd, d.d, pq, pk, pv, (const float*)pb, ptr(o), (float*)ptr(lse), opt_ptr(ws), bytes, stream());
        return tuple({o, lse});
    });
}

// desc, qkv, bias_table, o, lse, workspace -> (o, lse)
PyObject* fwd_packed(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 6, [&] {
        Desc d(a[0]);
        const at::Tensor &x = tensor(a[1], "qkv"), &b = tensor(a[2], "bias_table");
        const int64_t rows = d.rows(), all = rows * d.d->head_dim;
        expect(x, d.act(), 3 * all, "qkv");
        expect(b, at::kFloat, d.table(), "bias_table");
        void *px = ptr(x), *pb = ptr(b);
        at::Tensor o = output(a[3], "o", d.act(), {d.d->B, d.d->H, d.d->W, d.d->heads, d.d->head_dim}, x);
        at::Tensor lse = output(a[4], "lse", at::kFloat, {d.d->B, d.d->H, d.d->W, d.d->heads}, x);
        expect(o, d.act(), all, "o"); expect(lse, at::kFloat, rows, "lse");
        size_t bytes;
        at::Tensor ws = workspace(a[5], d, false, x, bytes);
        launch(f_fwd_packed, d.d, px, (const float*)pb, ptr(o), (float*)ptr(lse), opt_ptr(ws), bytes, stream());
        return tuple({o, lse});
    });
}

// desc, q, k, v, bias_table, o, lse -> (o, lse)
PyObject* fwd_noalloc(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 7, [&] {
        Desc d(a[0]);
        const at::Tensor &q = tensor(a[1], "q"), &k = tensor(a[2], "k"), &v = tensor(a[3], "v"), &b = tensor(a[4], "bias_table");
        const at::Tensor &o = tensor(a[5], "o"), &lse = tensor(a[6], "lse");
        const int64_t rows = d.rows(), all = rows * d.d->head_dim;
        expect(q, d.act(), all, "q"); expect(k, d.act(), all, "k"); expect(v, d.act(), all, "v"); expect(o, d.act(), all, "o");
        expect(b, at::kFloat, d.table(), "bias_table"); expect(lse, at::kFloat, rows, "lse");
        launch(f_fwd_noalloc, d.d, ptr(q), ptr(k), ptr(v), (const float*)ptr(b), ptr(o), (float*)ptr(lse), stream());
        return tuple({o, lse});
    });
}

// desc, q, k, v, bias_table, o, lse, d_o, dq, dk, dv, dbias, workspace -> (dq, dk, dv, dbias)
PyObject* bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 13, [&] {
        Desc d(a[0]);
        const at::Tensor &q = tensor(a[1], "q"), &k = tensor(a[2], "k"), &v = tensor(a[3], "v"), &b = tensor(a[4], "bias_table");
        const at::Tensor &o = tensor(a[5], "o"), &lse = tensor(a[6], "lse"), &g = tensor(a[7], "d_o");
        const int64_t rows = d.rows(), all = rows * d.d->head_dim;
        expect(q, d.act(), all, "q"); expect(k, d.act(), all, "k"); expect(v, d.act(), all, "v"); expect(o, d.act(), all, "o"); expect(g, d.act(), all, "d_o");
        expect(lse, at::kFloat, rows, "lse"); expect(b, at::kFloat, d.table(), "bias_table");
        void *pq = ptr(q), *pk = ptr(k), *pv = ptr(v), *pb = ptr(b), *po = ptr(o), *pl = ptr(lse), *pg = ptr(g);
        at::Tensor dq = output(a[8], "dq", d.act(), q.sizes(), q), dk = output(a[9], "dk", d.act(), q.sizes(), q), dv = output(a[10], "dv", d.act(), q.sizes(), q);
        at::Tensor db = output(a[11], "dbias", at::kFloat, b.sizes(), q);
        expect(dq, d.act(), all, "dq"); expect(dk, d.act(), all, "dk"); expect(dv, d.act(), all, "dv"); expect(db, at::kFloat, b.numel(), "dbias");
        size_t bytes;
        at::Tensor ws = workspace(a[12], d, true, q, bytes);
        launch(f_bwd, d.d, pq, pk, pv, (const float*)pb, po, (const float*)pl, pg, ptr(dq), ptr(dk), ptr(dv), (float*)ptr(db), opt_ptr(ws), bytes, stream());
        return tuple({dq, dk, dv, db});
    });
}

// desc, qkv, bias_table, o, lse, d_o, dqkv, dbias, workspace -> (dqkv, dbias)
PyObject* bwd_packed(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 9, [&] {
        Desc d(a[0]);
        const at::Tensor &x = tensor(a[1], "qkv"), &b = tensor(a[2], "bias_table"), &o = tensor(a[3], "o"), &lse = tensor(a[4], "lse"), &g = tensor(a[5], "d_o");
        const int64_t rows = d.rows(), all = rows * d.d->head_dim;
        expect(x, d.act(), 3 * all, "qkv"); expect(o, d.act(), all, "o"); expect(g, d.act(), all, "d_o");
        expect(lse, at::kFloat, rows, "lse"); expect(b, at::kFloat, d.table(), "bias_table");
        void *px = ptr(x), *pb = ptr(b), *po = ptr(o), *pl = ptr(lse), *pg = ptr(g);
        at::Tensor dx = output(a[6], "dqkv", d.act(), x.sizes(), x), db = output(a[7], "dbias", at::kFloat, b.sizes(), x);
        expect(dx, d.act(), 3 * all, "dqkv"); expect(db, at::kFloat, b.numel(), "dbias");
        size_t bytes;
        at::Tensor ws = workspace(a[8], d, true, x, bytes);
        launch(f_bwd_packed, d.d, px, (const float*)pb, po, (const float*)pl, pg, ptr(dx), (float*)ptr(db), opt_ptr(ws), bytes, stream());
        return tuple({dx, db});
    });
}

// ---- what stands around the attention ---------------------------------------------------------------------------
int dtype_code(at::ScalarType t, const char* name) {
    if (t == at::kBFloat16) return TERRA_DTYPE_BF16;
    if (t == at::kHalf) return TERRA_DTYPE_F16;
    PyErr_Format(PyExc_ValueError, "terra: %s must be torch.bfloat16 or torch.float16, got %s", name, dtype_name(t));
    throw Failed{};
}
at::Tensor optional(PyObject* o, const char* name, at::ScalarType dtype, int64_t numel) {
    if (o == Py_None) return at::Tensor();
    const at::Tensor& t = tensor(o, name);
    expect(t, dtype, numel, name);
    return t;
}
// an output: the caller's tensor, or a new one, of this type and size
at::Tensor result(PyObject* o, const char* name, at::ScalarType dtype, at::IntArrayRef shape, const at::Tensor& like) {
    at::Tensor t = output(o, name, dtype, shape, like);
    int64_t n = 1;
    for (int64_t d : shape) n *= d;
    expect(t, dtype, n, name);
    return t;
}
// the caller's workspace, or a new one of `need` bytes (an undefined tensor where none is wanted)
at::Tensor scratch(PyObject* o, size_t need, const at::Tensor& like, size_t& bytes) {
    at::Tensor t;
    if (o != Py_None) {
        t = tensor(o, "workspace");
    } else if (need) {
        NoGil no_gil;
        t = at::detail::empty_cuda({(int64_t)need}, at::kByte, like.device(), std::nullopt);
    }
    bytes = t.defined() ? t.nbytes() : 0;
    return t;
}
// rows of `last` values in t, whose last dimension they are
int64_t rows_of(const at::Tensor& t, int64_t last, const char* name) {
    if (t.dim() < 1 || last < 1 || t.size(-1) != last) {
        PyErr_Format(PyExc_ValueError, "terra: %s must have %lld values in its last dimension, got %lld", name, (long long)last,
                     t.dim() < 1 ? 0ll : (long long)t.size(-1));
        throw Failed{};
    }
    return t.numel() / last;
}
int as_int(PyObject* o) {
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw Failed{};
    return v > INT32_MAX || v < INT32_MIN ? -1 : (int)v;
}
float as_float(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1 && PyErr_Occurred()) throw Failed{};
    return (float)v;
}
PyObject* wrapped(const at::Tensor& t) {
    if (t.defined()) return THPVariable_Wrap(t);
    Py_RETURN_NONE;
}
PyObject* tuple_opt(std::initializer_list<at::Tensor> ts) {
    PyObject* r = PyTuple_New((Py_ssize_t)ts.size());
    if (!r) throw Failed{};
    Py_ssize_t i = 0;
    for (const at::Tensor& t : ts) PyTuple_SET_ITEM(r, i++, wrapped(t));
    return r;
}

terra_norm_desc norm_desc(const at::Tensor& x, const at::Tensor& weight, float eps) {
    const int64_t c = weight.numel();
    expect(weight, at::kFloat, c, "weight");
    terra_norm_desc d;
    d.rows = rows_of(x, c, "x");
    d.channels = c > INT32_MAX ? -1 : (int32_t)c;
    d.eps = eps;
    d.dtype = dtype_code(x.scalar_type(), "x");
    return d;
}

// x, weight, residual, eps, h, y, rstd -> (y, h, rstd)
PyObject* norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 7, [&] {
        const at::Tensor &x = tensor(a[0], "x"), &w = tensor(a[1], "weight");
        const terra_norm_desc d = norm_desc(x, w, as_float(a[3]));
        const at::Tensor r = optional(a[2], "residual", x.scalar_type(), x.numel());
        void *px = ptr(x), *pw = ptr(w), *pr = opt_ptr(r);
        at::Tensor h;
        if (r.defined() || a[4] != Py_None) h = result(a[4], "h", x.scalar_type(), x.sizes(), x);
        at::Tensor y = result(a[5], "y", x.scalar_type(), x.sizes(), x);
        at::Tensor rstd = result(a[6], "rstd", at::kFloat, {d.rows}, x);
        launch(f_norm_fwd, &d, px, pr, (const float*)pw, opt_ptr(h), ptr(y), (float*)ptr(rstd), stream());
        if (!h.defined() && ptr(y) != px) h = x;
        return tuple_opt({y, h, rstd});
    });
}

// x, weight, residual, eps, h, y, scale, rstd (written where it is given) -> (y, scale, h)
PyObject* norm_fwd_e4m3(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 8, [&] {
        const at::Tensor &x = tensor(a[0], "x"), &w = tensor(a[1], "weight");
        const terra_norm_desc d = norm_desc(x, w, as_float(a[3]));
        const at::Tensor r = optional(a[2], "residual", x.scalar_type(), x.numel());
        const at::Tensor rstd = optional(a[7], "rstd", at::kFloat, d.rows);
        void *px = ptr(x), *pw = ptr(w), *pr = opt_ptr(r), *ps = opt_ptr(rstd);
        at::Tensor h;
        if (r.defined() || a[4] != Py_None) h = result(a[4], "h", x.scalar_type(), x.sizes(), x);
        at::Tensor y = result(a[5], "y", at::kFloat8_e4m3fn, x.sizes(), x);
        at::Tensor scale = result(a[6], "scale", at::kFloat, {d.rows}, x);
        launch(f_norm_fwd_e4m3, &d, px, pr, (const float*)pw, opt_ptr(h), ptr(y), (float*)ptr(scale), (float*)ps, stream());
        return tuple({y, scale, h.defined() ? h : x});
    });
}

// h, weight, rstd, d_y, d_h, d_x, d_weight, workspace -> (d_x, d_weight)
PyObject* norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 8, [&] {
        const at::Tensor &h = tensor(a[0], "h"), &w = tensor(a[1], "weight"), &rstd = tensor(a[2], "rstd"), &g = tensor(a[3], "d_y");
        const terra_norm_desc d = norm_desc(h, w, 0.f);
        expect(rstd, at::kFloat, d.rows, "rstd");
        expect(g, h.scalar_type(), h.numel(), "d_y");
        const at::Tensor dh = optional(a[4], "d_h", h.scalar_type(), h.numel());
        void *ph = ptr(h), *pw = ptr(w), *ps = ptr(rstd), *pg = ptr(g), *pd = opt_ptr(dh);
        at::Tensor dx = result(a[5], "d_x", h.scalar_type(), h.sizes(), h), dw = result(a[6], "d_weight", at::kFloat, w.sizes(), h);
        size_t need = 0, bytes;
        check(f_norm_workspace(&d, &need));
        at::Tensor ws = scratch(a[7], need, h, bytes);
        launch(f_norm_bwd, &d, ph, (const float*)pw, (const float*)ps, pg, pd, ptr(dx), (float*)ptr(dw), opt_ptr(ws), bytes, stream());
        return tuple({dx, dw});
    });
}

terra_linear_desc linear_desc(const at::Tensor& x, const at::Tensor& w, int activation, int dtype) {
    if (w.dim() != 2) {
        PyErr_SetString(PyExc_ValueError, "terra: w must be [n_out, n_in]");
        throw Failed{};
    }
    terra_linear_desc d;
    d.rows = rows_of(x, w.size(1), "x");
    d.n_in = w.size(1) > INT32_MAX ? -1 : (int32_t)w.size(1);
    d.n_out = w.size(0) > INT32_MAX ? -1 : (int32_t)w.size(0);
    d.activation = activation;
    d.dtype = dtype;
    return d;
}
std::vector<int64_t> out_shape(const at::Tensor& x, int64_t last) {
    std::vector<int64_t> s = x.sizes().vec();
    s.back() = last;
    return s;
}

// x, w, bias, residual, activation, keep_z, y, z, workspace -> (y, z or None)
PyObject* linear_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 9, [&] {
        const at::Tensor &x = tensor(a[0], "x"), &w = tensor(a[1], "w");
        const terra_linear_desc d = linear_desc(x, w, as_int(a[4]), dtype_code(x.scalar_type(), "x"));
        const auto act = x.scalar_type();
        expect(w, act, w.numel(), "w");
        const at::Tensor b = optional(a[2], "bias", at::kFloat, d.n_out), r = optional(a[3], "residual", act, d.rows * d.n_out);
        void *px = ptr(x), *pw = ptr(w), *pb = opt_ptr(b), *pr = opt_ptr(r);
        const int keep = PyObject_IsTrue(a[5]);
        if (keep < 0) throw Failed{};
        const std::vector<int64_t> shape = out_shape(x, d.n_out);
        at::Tensor y = result(a[6], "y", act, shape, x), z;
        if (keep || a[7] != Py_None) z = result(a[7], "z", act, shape, x);
        size_t need = 0, bytes;
        check(f_linear_workspace(&d, TERRA_LINEAR_FWD, &need));
        at::Tensor ws = scratch(a[8], need, x, bytes);
        launch(f_linear_fwd, &d, px, pw, (const float*)pb, pr, ptr(y), opt_ptr(z), opt_ptr(ws), bytes, stream());
        return tuple_opt({y, z});
    });
}

// x8, x_scale, w8, w_scale, bias, residual, activation, dtype, y, workspace -> y
PyObject* linear_fwd_e4m3(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 10, [&] {
        const at::Tensor &x = tensor(a[0], "x"), &xs = tensor(a[1], "x_scale"), &w = tensor(a[2], "w"), &wsc = tensor(a[3], "w_scale");
        const terra_linear_desc d = linear_desc(x, w, as_int(a[6]), as_int(a[7]));
        expect(x, at::kFloat8_e4m3fn, x.numel(), "x");
        expect(w, at::kFloat8_e4m3fn, w.numel(), "w");
        expect(xs, at::kFloat, d.rows, "x_scale");
        expect(wsc, at::kFloat, d.n_out, "w_scale");
        const auto act = d.dtype == TERRA_DTYPE_F16 ? at::kHalf : at::kBFloat16;
        const at::Tensor b = optional(a[4], "bias", at::kFloat, d.n_out), r = optional(a[5], "residual", act, d.rows * d.n_out);
        void *px = ptr(x), *pxs = ptr(xs), *pw = ptr(w), *pws = ptr(wsc), *pb = opt_ptr(b), *pr = opt_ptr(r);
        at::Tensor y = result(a[8], "y", act, out_shape(x, d.n_out), x);
        size_t need = 0, bytes;
        check(f_linear_workspace(&d, TERRA_LINEAR_FWD_E4M3, &need));
        at::Tensor ws = scratch(a[9], need, x, bytes);
        launch(f_linear_fwd_e4m3, &d, px, (const float*)pxs, pw, (const float*)pws, (const float*)pb, pr, ptr(y), opt_ptr(ws), bytes, stream());
        return wrapped(y);
    });
}

// x, w, d_z, z_in, activation, need_dx, need_dw, need_dbias, d_x, d_w, d_bias, workspace -> (d_x, d_w, d_bias), None for what is not needed
PyObject* linear_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 12, [&] {
        const at::Tensor &x = tensor(a[0], "x"), &w = tensor(a[1], "w"), &g = tensor(a[2], "d_z");
        const auto act = x.scalar_type();
        const terra_linear_desc d = linear_desc(x, w, as_int(a[4]), dtype_code(act, "x"));
        expect(w, act, w.numel(), "w");
        expect(g, act, d.rows * d.n_out, "d_z");
        const at::Tensor z = optional(a[3], "z_in", act, x.numel());
        void *px = ptr(x), *pw = ptr(w), *pg = ptr(g), *pz = opt_ptr(z);
        bool needed[3];
        for (int i = 0; i < 3; ++i) {
            const int v = PyObject_IsTrue(a[5 + i]);
            if (v < 0) throw Failed{};
            needed[i] = v || a[8 + i] != Py_None;
        }
        at::Tensor dx, dw, db;
        if (needed[0]) dx = result(a[8], "d_x", act, x.sizes(), x);
        if (needed[1]) dw = result(a[9], "d_w", at::kFloat, w.sizes(), x);
        if (needed[2]) db = result(a[10], "d_bias", at::kFloat, {d.n_out}, x);
        size_t need = 0, bytes;
        check(f_linear_workspace(&d, TERRA_LINEAR_BWD, &need));
        at::Tensor ws = scratch(a[11], need, x, bytes);
        launch(f_linear_bwd, &d, px, pw, pg, pz, opt_ptr(dx), (float*)opt_ptr(dw), (float*)opt_ptr(db), opt_ptr(ws), bytes, stream());
        return tuple_opt({dx, dw, db});
    });
}

// z, d_y, activation, d_z -> d_z
PyObject* activation_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 4, [&] {
        const at::Tensor &z = tensor(a[0], "z"), &g = tensor(a[1], "d_y");
        const int dtype = dtype_code(z.scalar_type(), "z");
        expect(g, z.scalar_type(), z.numel(), "d_y");
        void *pz = ptr(z), *pg = ptr(g);
        at::Tensor d = result(a[3], "d_z", z.scalar_type(), z.sizes(), z);
        launch(f_activation_bwd, z.numel(), as_int(a[2]), dtype, pz, pg, ptr(d), stream());
        return wrapped(d);
    });
}

// inv_freq, row_pairs, layout, scale, inverse
terra_rotary_desc rotary_desc(PyObject* const* a, const at::Tensor& freq) {
    expect(freq, at::kDouble, freq.numel(), "inv_freq");
    terra_rotary_desc r;
    r.rot_dim = freq.numel() > 4096 ? -1 : (int32_t)(2 * freq.numel());
    r.row_pairs = as_int(a[1]);
    r.layout = as_int(a[2]);
    r.scale = as_float(a[3]);
    r.inverse = PyObject_IsTrue(a[4]);
    if (r.inverse < 0) throw Failed{};
    return r;
}

// desc, q, k, inv_freq, row_pairs, layout, scale, inverse, positions, q_out, k_out -> (q_out, k_out or None)
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 11, [&] {
        Desc d(a[0]);
        const at::Tensor &q = tensor(a[1], "q"), &freq = tensor(a[3], "inv_freq");
        const terra_rotary_desc r = rotary_desc(a + 3, freq);
        const int64_t tokens = (int64_t)d.d->B * d.d->H * d.d->W, all = d.rows() * d.d->head_dim;
        expect(q, d.act(), all, "q");
        const at::Tensor k = optional(a[2], "k", d.act(), all), pos = optional(a[8], "positions", at::kInt, 2 * tokens);
        void *pq = ptr(q), *pk = opt_ptr(k), *pf = ptr(freq), *pp = opt_ptr(pos);
        at::Tensor qo = result(a[9], "q_out", d.act(), q.sizes(), q), ko;
        if (k.defined()) ko = result(a[10], "k_out", d.act(), k.sizes(), q);
        launch(f_rotary, d.d, &r, (const double*)pf, (const int32_t*)pp, pq, pk, ptr(qo), opt_ptr(ko), stream());
        return tuple_opt({qo, ko});
    });
}

// desc, qkv, inv_freq, row_pairs, layout, scale, inverse, positions -> qkv
PyObject* rotary_packed(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 8, [&] {
        Desc d(a[0]);
        const at::Tensor &x = tensor(a[1], "qkv"), &freq = tensor(a[2], "inv_freq");
        const terra_rotary_desc r = rotary_desc(a + 2, freq);
        const int64_t tokens = (int64_t)d.d->B * d.d->H * d.d->W;
        expect(x, d.act(), 3 * d.rows() * d.d->head_dim, "qkv");
        const at::Tensor pos = optional(a[7], "positions", at::kInt, 2 * tokens);
        launch(f_rotary_packed, d.d, &r, (const double*)ptr(freq), (const int32_t*)opt_ptr(pos), ptr(x), stream());
        return wrapped(x);
    });
}

// The library's entry points (addresses, in this order) and the callable that raises for a status.
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 18, [&]() -> PyObject* {
        void* p[17];
        for (int i = 0; i < 17; ++i) {
            p[i] = PyLong_AsVoidPtr(a[i]);
            if (PyErr_Occurred()) throw Failed{};
        }
        f_workspace = (decltype(f_workspace))p[0];
        f_fwd = (decltype(f_fwd))p[1];
        f_bwd = (decltype(f_bwd))p[2];
        f_fwd_packed = (decltype(f_fwd_packed))p[3];
        f_bwd_packed = (decltype(f_bwd_packed))p[4];
        f_fwd_noalloc = (decltype(f_fwd_noalloc))p[5];
        f_norm_fwd = (decltype(f_norm_fwd))p[6];
        f_norm_fwd_e4m3 = (decltype(f_norm_fwd_e4m3))p[7];
        f_norm_workspace = (decltype(f_norm_workspace))p[8];
        f_norm_bwd = (decltype(f_norm_bwd))p[9];
        f_linear_workspace = (decltype(f_linear_workspace))p[10];
        f_linear_fwd = (decltype(f_linear_fwd))p[11];
        f_linear_fwd_e4m3 = (decltype(f_linear_fwd_e4m3))p[12];
        f_linear_bwd = (decltype(f_linear_bwd))p[13];
        f_activation_bwd = (decltype(f_activation_bwd))p[14];
        f_rotary = (decltype(f_rotary))p[15];
        f_rotary_packed = (decltype(f_rotary_packed))p[16];
        Py_INCREF(a[17]);
        Py_XDECREF(on_status);
        on_status = a[17];
        Py_RETURN_NONE;
    });
}

#define FN(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FN(bind), FN(fwd), FN(bwd), FN(fwd_packed), FN(bwd_packed), FN(fwd_noalloc), FN(norm_fwd),
                         FN(norm_fwd_e4m3), FN(norm_bwd), FN(linear_fwd), FN(linear_fwd_e4m3), FN(linear_bwd), FN(activation_bwd), FN(rotary), FN(rotary_packed), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host() { return PyModule_Create(&module); }
