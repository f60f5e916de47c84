// The host's side of the calls whose kernels take a few microseconds: a decode step's norm, routing and products, and the
// quantizers and products of a training step, which issues eight of them for the same experts. Argument checks, output tensors and the
// C ABI call in one step of native code; the binding's Python functions (which document them) pass their arguments on. In Python each output tensor costs 1.2 - 1.8 us, the checks 1 - 2 and the foreign call 1. us a call, so / here:
// norm 9.9 / 5.6, its gradient 15.1 / 9.0, sort 8.8 / 5.4, dispatch 7.1 / 3.9, combine 6.9 / 3.9, quantizing 9.2 / 5.2, a dense
// product 6.5 / 4.1, a product of 3 tokens 7.0 / 4.1, of 64 16.1 / 8.1, both operands of a tensor 13.7 / 7.7, grouped quantizing 10.1 /
// 6.0, a grouped product 7.7 / 4.7 (a launch alone is about 2).
// Errors: ValueError for a tensor that a call cannot take, TypeError for what is no tensor, the binding's error class for a status of
// the library.

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <math.h>

#include "../../include/ufp4.h"

namespace {

PyObject* g_error = nullptr;  // UFP4Error(status, call)

bool refuse(const char* what, const char* why) {
    PyErr_Format(PyExc_ValueError, "%s must be %s", what, why);
    return false;
}

bool check(int status, const char* call) {
    if (status == UFP4_OK) return true;
    PyObject* const e = PyObject_CallFunction(g_error, "is", status, call);
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    return false;
}

// A status of the library and the call that gave it.
struct Done {
    int status;
    const char* call;
};

// f(), which allocates and calls the library, without the interpreter's lock: a launch waits where the queue is full, an allocation where
// memory has to be freed first, and what the GPU waits for may be another Python thread's.
template <class F>
bool unlocked(F&& f) {
    Done done;
    {
        struct Lock {
            PyThreadState* const state = PyEval_SaveThread();
            ~Lock() { PyEval_RestoreThread(state); }  // also when f throws
        } lock;
        done = f();
    }
    return check(done.status, done.call);
}

bool arguments(Py_ssize_t have, Py_ssize_t want) {
    if (have == want) return true;
    PyErr_Format(PyExc_TypeError, "%zd arguments instead of %zd", have, want);
    return false;
}

const at::Tensor* tensor(PyObject* o, const char* what) {
    if (THPVariable_Check(o)) return &THPVariable_Unpack(o);
    PyErr_Format(PyExc_TypeError, "%s must be a tensor", what);
    return nullptr;
}

void* pointer(PyObject* o) { return PyLong_AsVoidPtr(o); }  // an error shows in PyErr_Occurred

// UFP4_OUT_* of a type, -1 for another.
int code_of(const at::Tensor& t) {
    const auto st = t.scalar_type();
    return st == at::kBFloat16 ? UFP4_OUT_BF16 : st == at::kFloat ? UFP4_OUT_F32 : -1;
}

// A 2-D row-major float32 or bfloat16 tensor on the GPU.
struct Rows {
    const at::Tensor* t = nullptr;
    int64_t rows = 0, cols = 0, ld = 0;
    int code = -1;
    void* data() const { return t->data_ptr(); }
};

bool rows_of(PyObject* o, const char* what, Rows& r) {
    r.t = tensor(o, what);
    if (!r.t) return false;
    const at::Tensor& t = *r.t;
    r.code = code_of(t);
    if (r.code < 0 || !t.is_cuda() || t.dim() != 2) return refuse(what, "a 2-D float32 or bfloat16 CUDA tensor");
    r.rows = t.size(0);
    r.cols = t.size(1);
    r.ld = r.cols;
    if (t.is_contiguous()) return true;
    if (t.numel() && r.cols > 1 && t.stride(1) != 1) return refuse(what, "row-major");
    if (r.rows > 1) {
        if (t.stride(0) < r.cols) return refuse(what, "of rows that do not overlap");
        r.ld = t.stride(0);
    }
    return true;
}

bool rows_like(PyObject* o, const char* what, const Rows& like, int64_t rows, int64_t cols, Rows& r) {
    if (!rows_of(o, what, r)) return false;
    if (r.code != like.code || r.t->device() != like.t->device()) return refuse(what, "of the input's type and device");
    if (r.rows != rows || r.cols != cols) {
        PyErr_Format(PyExc_ValueError, "%s must be of shape (%lld, %lld)", what, (long long)rows, (long long)cols);
        return false;
    }
    return true;
}

// The output: `o`, which `out` then holds, or for None a tensor that rows_new allocates.
bool rows_out(PyObject* o, const Rows& like, int64_t rows, int64_t cols, at::Tensor& out, Rows& r) {
    if (o != Py_None) {
        if (!rows_like(o, "out", like, rows, cols, r)) return false;
        out = *r.t;
        return true;
    }
    r.rows = rows;
    r.cols = r.ld = cols;
    r.code = like.code;
    return true;
}

void rows_new(const Rows& like, at::Tensor& out, Rows& r) {
    if (!out.defined()) out = at::empty({r.rows, r.cols}, like.t->options());
    r.t = &out;
}

at::Tensor floats(int64_t n, const at::Tensor& like) { return at::empty({n}, like.options().dtype(at::kFloat)); }

// The address of a contiguous tensor of n elements of type `type` (or, with bf16, bfloat16), null for None.
bool vector(PyObject* o, const char* what, at::ScalarType type, int64_t n, const at::Device& device, bool bf16, void*& p, int* code = nullptr) {
    p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor* const t = tensor(o, what);
    if (!t) return false;
    const auto st = t->scalar_type();
    if (!(st == type || (bf16 && st == at::kBFloat16)) || t->numel() != n || t->device() != device || !t->is_contiguous()) {
        PyErr_Format(PyExc_ValueError, "%s must be a contiguous %s%s tensor of %lld elements on the input's device", what,
                     type == at::kInt ? "int32" : "float32", bf16 ? " or bfloat16" : "", (long long)n);
        return false;
    }
    if (code) *code = code_of(*t);
    p = t->data_ptr();
    return true;
}

// gamma and beta, of one type.
bool weights(PyObject* gamma, PyObject* beta, int64_t cols, const at::Device& device, int& code, void*& g, void*& b) {
    int cg = -1, cb = -1;
    if (!vector(gamma, "gamma", at::kFloat, cols, device, true, g, &cg) || !vector(beta, "beta", at::kFloat, cols, device, true, b, &cb))
        return false;
    if (cg >= 0 && cb >= 0 && cg != cb) {
        PyErr_SetString(PyExc_ValueError, "gamma and beta must be of one type");
        return false;
    }
    code = cg >= 0 ? cg : cb >= 0 ? cb : UFP4_OUT_F32;
    return true;
}

// rows [tokens, k] of a sort and their weights.
struct Slots {
    int64_t tokens = 0, k = 0;
    void *rows = nullptr, *w = nullptr;
};

bool slots_of(PyObject* o, PyObject* w, const at::Device& device, Slots& s) {
    const at::Tensor* const t = tensor(o, "rows");
    if (!t) return false;
    if (t->scalar_type() != at::kInt || t->dim() != 2 || t->device() != device || !t->is_contiguous())
        return refuse("rows", "a contiguous int32 tensor [tokens, k] on the input's device");
    s.tokens = t->size(0);
    s.k = t->size(1);
    s.rows = t->data_ptr();
    if (w != Py_None && THPVariable_Check(w) && THPVariable_Unpack(w).sizes() != t->sizes()) return refuse("weights", "of the shape of rows");
    return vector(w, "weights", at::kFloat, s.tokens * s.k, device, false, s.w);
}

// offsets int64 [groups + 1]
bool offsets_of(PyObject* o, const at::Device& device, void*& p, int64_t& groups) {
    const at::Tensor* const t = tensor(o, "offsets");
    if (!t) return false;
    if (t->scalar_type() != at::kLong || t->dim() != 1 || t->device() != device || !t->is_contiguous())
        return refuse("offsets", "a contiguous int64 tensor [groups + 1] on the input's device");
    p = t->data_ptr();
    groups = t->numel() - 1;
    return true;
}

PyObject* pair(const at::Tensor& a, PyObject* b) {
    PyObject* const x = THPVariable_Wrap(a);
    PyObject* const r = x && b ? PyTuple_Pack(2, x, b) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(b);
    return r;
}

PyObject* triple(const at::Tensor& a, const at::Tensor& b, const at::Tensor& c) {  // an undefined tensor is None
    PyObject* const x = THPVariable_Wrap(a);
    PyObject* const y = THPVariable_Wrap(b);
    PyObject* const z = THPVariable_Wrap(c);
    PyObject* const r = x && y && z ? PyTuple_Pack(3, x, y, z) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    Py_XDECREF(z);
    return r;
}

#define CALL(name, count)                                                       \
    PyObject* name(PyObject*, PyObject* const* a, Py_ssize_t n_args) {          \
        HANDLE_TH_ERRORS                                                        \
        if (!arguments(n_args, count)) return nullptr;
#define END_CALL         \
    END_HANDLE_TH_ERRORS \
    }

// (x, gamma, beta, eps, out, stream) -> y, mean, rstd
CALL(layer_norm, 6)
    Rows x, y;
    if (!rows_of(a[0], "x", x)) return nullptr;
    void *g, *b;
    int wdt;
    if (!weights(a[1], a[2], x.cols, x.t->device(), wdt, g, b)) return nullptr;
    const double eps = PyFloat_AsDouble(a[3]);
    void* const stream = pointer(a[5]);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor out;
    if (!rows_out(a[4], x, x.rows, x.cols, out, y)) return nullptr;
    at::Tensor mean, rstd;
    if (!unlocked([&]() -> Done {
            rows_new(x, out, y);
            mean = floats(x.rows, *x.t);
            rstd = floats(x.rows, *x.t);
            if (x.cols == 0) {  // 0 / 0; the library has nothing to read and writes nothing
                mean.fill_(NAN);
                rstd.fill_(NAN);
            }
            return {ufp4_layer_norm(x.code, x.data(), x.rows, x.cols, x.ld, wdt, g, b, (float)eps, y.data(), y.ld, mean.data_ptr<float>(),
                                    rstd.data_ptr<float>(), stream), "ufp4_layer_norm"};
        }))
        return nullptr;
    return triple(out, mean, rstd);
END_CALL

// (dy, x, gamma, mean, rstd, weights, out, stream) -> dx, dgamma, dbeta
CALL(layer_norm_bwd, 8)
    Rows x, dy, dx;
    if (!rows_of(a[1], "x", x) || !rows_like(a[0], "dy", x, x.rows, x.cols, dy)) return nullptr;
    const at::Device device = x.t->device();
    void *g, *b, *mean, *rstd;
    int wdt;
    if (!weights(a[2], Py_None, x.cols, device, wdt, g, b) || !vector(a[3], "mean", at::kFloat, x.rows, device, false, mean) ||
        !vector(a[4], "rstd", at::kFloat, x.rows, device, false, rstd))
        return nullptr;
    const int some = PyObject_IsTrue(a[5]);
    void* const stream = pointer(a[7]);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor out, dgamma, dbeta, ws;
    if (!rows_out(a[6], x, x.rows, x.cols, out, dx)) return nullptr;
    if (!unlocked([&]() -> Done {
            size_t need = 0;
            rows_new(x, out, dx);
            if (some) {
                const int st = ufp4_layer_norm_bwd_workspace(x.code, x.rows, x.cols, &need);
                if (st != UFP4_OK) return {st, "ufp4_layer_norm_bwd_workspace"};
                dgamma = floats(x.cols, *x.t);
                dbeta = floats(x.cols, *x.t);
                ws = floats((int64_t)(need / 4), *x.t);
            }
            return {ufp4_layer_norm_bwd(x.code, dy.data(), dy.ld, x.data(), x.rows, x.cols, x.ld, wdt, g, static_cast<float*>(mean),
                                        static_cast<float*>(rstd), dx.data(), dx.ld, some ? dgamma.data_ptr<float>() : nullptr,
                                        some ? dbeta.data_ptr<float>() : nullptr, some ? ws.data_ptr() : nullptr, need, stream),
                    "ufp4_layer_norm_bwd"};
        }))
        return nullptr;
    return triple(out, dgamma, dbeta);
END_CALL

// (ids, experts, stream) -> offsets, rows, source
CALL(moe_sort, 3)
    const at::Tensor* const ids = tensor(a[0], "ids");
    if (!ids) return nullptr;
    const auto st = ids->scalar_type();
    if (!(st == at::kInt || st == at::kLong) || !ids->is_cuda() || ids->dim() != 2 || !ids->is_contiguous()) {
        refuse("ids", "a contiguous int32 or int64 CUDA tensor [tokens, k]");
        return nullptr;
    }
    const long long experts = PyLong_AsLongLong(a[1]);
    void* const stream = pointer(a[2]);
    if (PyErr_Occurred()) return nullptr;
    const int64_t tokens = ids->size(0), k = ids->size(1);
    const int32_t k32 = k > INT32_MAX ? INT32_MAX : (int32_t)k;
    const int32_t e32 = experts > INT32_MAX ? INT32_MAX : experts < 0 ? -1 : (int32_t)experts;
    at::Tensor offsets, rows, source, ws;
    if (!unlocked([&]() -> Done {
            size_t need = 0;
            const int bytes = ufp4_moe_sort_workspace(tokens, k32, e32, &need);
            if (bytes != UFP4_OK) return {bytes, "ufp4_moe_sort_workspace"};
            const auto ints = ids->options().dtype(at::kInt);
            offsets = at::empty({experts + 1}, ids->options().dtype(at::kLong));
            rows = at::empty({tokens, k}, ints);
            source = at::empty({tokens * k}, ints);
            if (need) ws = at::empty({(int64_t)(need / 4)}, ints);
            return {ufp4_moe_sort(ids->data_ptr(), st == at::kInt ? 32 : 64, tokens, k32, e32, offsets.data_ptr<int64_t>(),
                                  rows.data_ptr<int32_t>(), source.data_ptr<int32_t>(), need ? ws.data_ptr() : nullptr, need, stream),
                    "ufp4_moe_sort"};
        }))
        return nullptr;
    return triple(offsets, rows, source);
END_CALL

// (x, rows, offsets, weights, out, stream) -> y
CALL(moe_dispatch, 6)
    Rows x, y;
    if (!rows_of(a[0], "x", x)) return nullptr;
    const at::Device device = x.t->device();
    Slots s;
    void* offsets;
    int64_t experts;
    if (!slots_of(a[1], a[3], device, s) || !offsets_of(a[2], device, offsets, experts)) return nullptr;
    if (x.rows != s.tokens) {
        PyErr_Format(PyExc_ValueError, "x must hold %lld tokens", (long long)s.tokens);
        return nullptr;
    }
    void* const stream = pointer(a[5]);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor out;
    if (!rows_out(a[4], x, s.tokens * s.k, x.cols, out, y)) return nullptr;
    if (!unlocked([&]() -> Done {
            rows_new(x, out, y);
            return {ufp4_moe_dispatch(x.code, x.data(), x.rows, x.cols, x.ld, static_cast<int32_t*>(s.rows), (int32_t)s.k,
                                      static_cast<int64_t*>(offsets), (int32_t)experts, static_cast<float*>(s.w), y.data(), y.rows, y.ld,
                                      stream), "ufp4_moe_dispatch"};
        }))
        return nullptr;
    return THPVariable_Wrap(out);
END_CALL

// (y, rows, weights, out, stream) -> out
CALL(moe_combine, 5)
    Rows y, o;
    if (!rows_of(a[0], "y", y)) return nullptr;
    Slots s;
    if (!slots_of(a[1], a[2], y.t->device(), s)) return nullptr;
    void* const stream = pointer(a[4]);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor out;
    if (!rows_out(a[3], y, s.tokens, y.cols, out, o)) return nullptr;
    if (!unlocked([&]() -> Done {
            rows_new(y, out, o);
            return {ufp4_moe_combine(y.code, y.data(), y.rows, y.cols, y.ld, static_cast<int32_t*>(s.rows), s.tokens, (int32_t)s.k,
                                     static_cast<float*>(s.w), o.data(), o.ld, stream), "ufp4_moe_combine"};
        }))
        return nullptr;
    return THPVariable_Wrap(out);
END_CALL

// (dout, y, rows, offsets, weights, out, stream) -> dy, dweights
CALL(moe_combine_bwd, 7)
    Rows y, dout, dy;
    if (!rows_of(a[1], "y", y)) return nullptr;
    const at::Device device = y.t->device();
    Slots s;
    void* offsets;
    int64_t experts;
    if (!slots_of(a[2], a[4], device, s) || !rows_like(a[0], "dout", y, s.tokens, y.cols, dout) || !offsets_of(a[3], device, offsets, experts))
        return nullptr;
    void* const stream = pointer(a[6]);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor out;
    if (!rows_out(a[5], y, y.rows, y.cols, out, dy)) return nullptr;
    at::Tensor dw;
    if (!unlocked([&]() -> Done {
            rows_new(y, out, dy);
            dw = at::empty({s.tokens, s.k}, y.t->options().dtype(at::kFloat));
            return {ufp4_moe_combine_bwd(y.code, dout.data(), s.tokens, y.cols, dout.ld, y.data(), y.rows, y.ld, static_cast<int32_t*>(s.rows),
                                         (int32_t)s.k, static_cast<int64_t*>(offsets), (int32_t)experts, static_cast<float*>(s.w), dy.data(),
                                         dy.ld, dw.data_ptr<float>(), stream), "ufp4_moe_combine_bwd"};
        }))
        return nullptr;
    return pair(out, THPVariable_Wrap(dw));
END_CALL

// The bf16 input of a quantizer.
const at::Tensor* bf16_of(PyObject* o) {
    const at::Tensor* const t = tensor(o, "x");
    if (t && (t->scalar_type() != at::kBFloat16 || !t->is_cuda() || t->dim() != 2 || t->stride(1) != 1)) {
        refuse("x", "a 2-D row-major bf16 CUDA tensor");
        return nullptr;
    }
    return t;
}

ufp4_qtensor* operand_of(PyObject* o) {  // the address of a descriptor
    return static_cast<ufp4_qtensor*>(pointer(o));
}

// Buffers for a microscaled operand [rows, red], which `d` describes from then on.
Done new_operand(const at::Tensor& like, int64_t rows, int64_t red, ufp4_qtensor& d, at::Tensor& codes, at::Tensor& scales) {
    int64_t panels = 0, cld = 0, sld = 0;
    const Done done{ufp4_qtensor_bytes(UFP4_FMT_E2M1_MX32, rows, red, &panels, &cld, &sld, nullptr, nullptr), "ufp4_qtensor_bytes"};
    if (done.status != UFP4_OK) return done;
    const auto bytes = like.options().dtype(at::kByte);
    codes = at::empty({panels, cld}, bytes);
    scales = at::empty({panels, sld}, bytes);
    d = ufp4_qtensor{};
    d.codes = static_cast<uint8_t*>(codes.data_ptr());
    d.scales = scales.data_ptr();
    d.code_panel_ld = cld;
    d.scale_panel_ld = sld;
    d.panels = panels;
    d.rows = rows;
    d.red = red;
    d.format = UFP4_FMT_E2M1_MX32;
    return done;
}

// The shape of a product's output: [rows, cols] or, of groups > 0 matrices, [groups, rows, cols].
struct Shape {
    int64_t size[3];  // groups, 0 for the former
    at::IntArrayRef sizes() const { return {size + (size[0] ? 0 : 1), size_t(size[0] ? 3 : 2)}; }
};

// The output of a product, row-major float32 or bfloat16, matrices rows apart: `o`, which `out` then holds, or for None a tensor of type
// `code` that product_new allocates.
bool product_out(PyObject* o, const at::Tensor& like, const Shape& s, int code, at::Tensor& out) {
    const int64_t groups = s.size[0], rows = s.size[1], cols = s.size[2];
    if (o == Py_None) return code >= 0 || refuse("out_dtype", "float32 or bfloat16");
    const at::Tensor* const t = tensor(o, "out");
    if (!t) return false;
    if (t->sizes() != s.sizes() || t->stride(-1) != 1 || t->device() != like.device()) {
        if (groups)
            PyErr_Format(PyExc_ValueError, "out must be a row-major tensor of shape (%lld, %lld, %lld) on the input's device", (long long)groups,
                         (long long)rows, (long long)cols);
        else
            PyErr_Format(PyExc_ValueError, "out must be a row-major tensor of shape (%lld, %lld) on the input's device", (long long)rows,
                         (long long)cols);
        return false;
    }
    if (groups > 1 && t->stride(0) != rows * t->stride(1)) return refuse("out", "of groups that lie their rows apart");
    if (code_of(*t) < 0) return refuse("out", "float32 or bfloat16");
    out = *t;
    return true;
}

void product_new(const at::Tensor& like, const Shape& s, int code, at::Tensor& out) {
    if (!out.defined()) out = at::empty(s.sizes(), like.options().dtype(code == UFP4_OUT_BF16 ? at::kBFloat16 : at::kFloat));
}

// (x, transpose, rht, sign_mask, rounding, seed, stream_id, descriptor, fresh, stream) -> (codes, scales) of a fresh descriptor, or None
CALL(mxfp4_quantize, 10)
    const at::Tensor* const x = bf16_of(a[0]);
    if (!x) return nullptr;
    const int transpose = PyObject_IsTrue(a[1]), rht = PyObject_IsTrue(a[2]), fresh = PyObject_IsTrue(a[8]);
    const uint32_t mask = (uint32_t)PyLong_AsUnsignedLongMask(a[3]), id = (uint32_t)PyLong_AsUnsignedLongMask(a[6]);
    const int rounding = (int)PyLong_AsLong(a[4]);
    const uint64_t seed = PyLong_AsUnsignedLongLongMask(a[5]);
    ufp4_qtensor* const d = operand_of(a[7]);
    void* const stream = pointer(a[9]);
    if (PyErr_Occurred()) return nullptr;
    const int64_t rows = x->size(0), cols = x->size(1);
    at::Tensor codes, scales;
    if (!unlocked([&]() -> Done {
            if (fresh) {
                const Done made = new_operand(*x, transpose ? cols : rows, transpose ? rows : cols, *d, codes, scales);
                if (made.status != UFP4_OK) return made;
            }
            return {ufp4_mxfp4_quantize(x->data_ptr(), rows, cols, x->stride(0), transpose, rht, mask, rounding, seed, id, d, stream),
                    "ufp4_mxfp4_quantize"};
        }))
        return nullptr;
    if (!fresh) Py_RETURN_NONE;
    return pair(codes, THPVariable_Wrap(scales));
END_CALL

// (x, rht_rows, rht_cols, sign_mask_rows, sign_mask_cols, rounding, seed, stream_rows, stream_cols, descriptor of the rows, fresh,
// descriptor of the columns, fresh, stream) -> (codes, scales, codes, scales), None for those of a descriptor that is not fresh
CALL(mxfp4_quantize_dual, 14)
    const at::Tensor* const x = bf16_of(a[0]);
    if (!x) return nullptr;
    const int rht_r = PyObject_IsTrue(a[1]), rht_c = PyObject_IsTrue(a[2]), fresh_r = PyObject_IsTrue(a[10]), fresh_c = PyObject_IsTrue(a[12]);
    const uint32_t mask_r = (uint32_t)PyLong_AsUnsignedLongMask(a[3]), mask_c = (uint32_t)PyLong_AsUnsignedLongMask(a[4]);
    const int rounding = (int)PyLong_AsLong(a[5]);
    const uint64_t seed = PyLong_AsUnsignedLongLongMask(a[6]);
    const uint32_t id_r = (uint32_t)PyLong_AsUnsignedLongMask(a[7]), id_c = (uint32_t)PyLong_AsUnsignedLongMask(a[8]);
    ufp4_qtensor *const r = operand_of(a[9]), *const c = operand_of(a[11]);
    void* const stream = pointer(a[13]);
    if (PyErr_Occurred()) return nullptr;
    const int64_t rows = x->size(0), cols = x->size(1);
    at::Tensor codes_r, scales_r, codes_c, scales_c;
    if (!unlocked([&]() -> Done {
            Done made{UFP4_OK, nullptr};
            if (fresh_r) made = new_operand(*x, rows, cols, *r, codes_r, scales_r);
            if (made.status == UFP4_OK && fresh_c) made = new_operand(*x, cols, rows, *c, codes_c, scales_c);
            if (made.status != UFP4_OK) return made;
            return {ufp4_mxfp4_quantize_dual(x->data_ptr(), rows, cols, x->stride(0), rht_r, mask_r, id_r, rht_c, mask_c, id_c, rounding, seed,
                                             r, c, stream), "ufp4_mxfp4_quantize_dual"};
        }))
        return nullptr;
    PyObject* const t[4] = {THPVariable_Wrap(codes_r), THPVariable_Wrap(scales_r), THPVariable_Wrap(codes_c), THPVariable_Wrap(scales_c)};
    PyObject* const all = t[0] && t[1] && t[2] && t[3] ? PyTuple_Pack(4, t[0], t[1], t[2], t[3]) : nullptr;
    for (PyObject* o : t) Py_XDECREF(o);
    return all;
END_CALL

// (x, offsets, padded_total, transpose, rht, sign_mask, rounding, seed, stream_id, descriptor, fresh, stream) -> (codes, scales) of a
// fresh descriptor, or None
CALL(mxfp4_quantize_grouped, 12)
    const at::Tensor* const x = bf16_of(a[0]);
    void* offsets;
    int64_t groups;
    if (!x || !offsets_of(a[1], x->device(), offsets, groups)) return nullptr;
    const int64_t padded = PyLong_AsLongLong(a[2]);
    const int transpose = PyObject_IsTrue(a[3]), rht = PyObject_IsTrue(a[4]), fresh = PyObject_IsTrue(a[10]);
    const uint32_t mask = (uint32_t)PyLong_AsUnsignedLongMask(a[5]), id = (uint32_t)PyLong_AsUnsignedLongMask(a[8]);
    const int rounding = (int)PyLong_AsLong(a[6]);
    const uint64_t seed = PyLong_AsUnsignedLongLongMask(a[7]);
    ufp4_qtensor* const d = operand_of(a[9]);
    void* const stream = pointer(a[11]);
    if (PyErr_Occurred()) return nullptr;
    const int64_t rows = x->size(0), cols = x->size(1);
    at::Tensor codes, scales;
    if (!unlocked([&]() -> Done {
            if (fresh) {
                const Done made = new_operand(*x, transpose ? cols : padded, transpose ? padded : cols, *d, codes, scales);
                if (made.status != UFP4_OK) return made;
            }
            return {ufp4_mxfp4_quantize_grouped(x->data_ptr(), rows, cols, x->stride(0), transpose, static_cast<int64_t*>(offsets),
                                                (int32_t)groups, padded, rht, mask, rounding, seed, id, d, stream),
                    "ufp4_mxfp4_quantize_grouped"};
        }))
        return nullptr;
    if (!fresh) Py_RETURN_NONE;
    return pair(codes, THPVariable_Wrap(scales));
END_CALL

// (codes, descriptor, out, stream) -> out
CALL(mxfp4_dequantize, 4)
    const at::Tensor* const codes = tensor(a[0], "codes");
    const ufp4_qtensor* const d = operand_of(a[1]);
    void* const stream = pointer(a[3]);
    if (!codes || PyErr_Occurred()) return nullptr;
    at::Tensor out;
    if (a[2] != Py_None) {
        const at::Tensor* const t = tensor(a[2], "out");
        if (!t) return nullptr;
        if (t->scalar_type() != at::kBFloat16 || t->dim() != 2 || t->size(0) != d->rows || t->size(1) != d->red ||
            t->device() != codes->device() || t->stride(1) != 1) {
            PyErr_Format(PyExc_ValueError, "out must be a row-major bf16 tensor of shape (%lld, %lld) on the operand's device", (long long)d->rows,
                         (long long)d->red);
            return nullptr;
        }
        out = *t;
    }
    if (!unlocked([&]() -> Done {
            if (!out.defined()) out = at::empty({d->rows, d->red}, codes->options().dtype(at::kBFloat16));
            return {ufp4_mxfp4_dequantize(d, out.data_ptr(), out.stride(0), stream), "ufp4_mxfp4_dequantize"};
        }))
        return nullptr;
    return THPVariable_Wrap(out);
END_CALL

// (codes of A, descriptor of A, of B, out type, out, stream) -> out
template <int (*GEMM)(const ufp4_qtensor*, const ufp4_qtensor*, void*, int64_t, int, void*)>
PyObject* product(const char* name, PyObject* const* a, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    if (!arguments(n_args, 6)) return nullptr;
    const at::Tensor* const codes = tensor(a[0], "codes");
    const ufp4_qtensor *const x = operand_of(a[1]), *const w = operand_of(a[2]);
    const int code = (int)PyLong_AsLong(a[3]);
    void* const stream = pointer(a[5]);
    if (!codes || PyErr_Occurred()) return nullptr;
    at::Tensor out;
    const Shape shape{{0, x->rows, w->rows}};
    if (!product_out(a[4], *codes, shape, code, out)) return nullptr;
    if (!unlocked([&]() -> Done {
            product_new(*codes, shape, code, out);
            return {GEMM(x, w, out.data_ptr(), out.stride(0), code_of(out), stream), name};
        }))
        return nullptr;
    return THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}
#define PRODUCT(name) \
    PyObject* name(PyObject*, PyObject* const* a, Py_ssize_t n) { return product<ufp4_##name>("ufp4_" #name, a, n); }
PRODUCT(mxfp4_gemm_fwd_y)
PRODUCT(mxfp4_gemm_bwd_dx)
PRODUCT(mxfp4_gemm_bwd_dw)

// (codes of A, descriptor of A, of B, offsets, rows of the output, out type, out, stream) -> out. BY_GROUP: B holds the groups' rows one
// after the other (W), otherwise their columns (W transposed).
template <int (*GEMM)(const ufp4_qtensor*, const ufp4_qtensor*, const int64_t*, int32_t, int64_t, void*, int64_t, int, void*), bool BY_GROUP>
PyObject* product_rows(const char* name, PyObject* const* a, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    if (!arguments(n_args, 8)) return nullptr;
    const at::Tensor* const codes = tensor(a[0], "codes");
    void* offsets;
    int64_t groups;
    if (!codes || !offsets_of(a[3], codes->device(), offsets, groups)) return nullptr;
    const ufp4_qtensor *const x = operand_of(a[1]), *const w = operand_of(a[2]);
    const int64_t rows = PyLong_AsLongLong(a[4]);
    const int code = (int)PyLong_AsLong(a[5]);
    void* const stream = pointer(a[7]);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor out;
    if (groups < 1) return refuse("offsets", "of one group at least"), nullptr;
    const Shape shape{{0, rows, BY_GROUP ? w->rows / groups : w->rows}};
    if (!product_out(a[6], *codes, shape, code, out)) return nullptr;
    if (!unlocked([&]() -> Done {
            product_new(*codes, shape, code, out);
            return {GEMM(x, w, static_cast<int64_t*>(offsets), (int32_t)groups, rows, out.data_ptr(), out.stride(0), code_of(out), stream), name};
        }))
        return nullptr;
    return THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}
PyObject* mxfp4_gemm_fwd_y_grouped(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return product_rows<ufp4_mxfp4_gemm_fwd_y_grouped, true>("ufp4_mxfp4_gemm_fwd_y_grouped", a, n);
}
PyObject* mxfp4_gemm_bwd_dx_grouped(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return product_rows<ufp4_mxfp4_gemm_bwd_dx_grouped, false>("ufp4_mxfp4_gemm_bwd_dx_grouped", a, n);
}

// (codes of A, descriptor of A, of B, offsets, out type, out, stream) -> out [groups, rows of A, rows of B]
CALL(mxfp4_gemm_bwd_dw_grouped, 7)
    const at::Tensor* const codes = tensor(a[0], "codes");
    void* offsets;
    int64_t groups;
    if (!codes || !offsets_of(a[3], codes->device(), offsets, groups)) return nullptr;
    const ufp4_qtensor *const x = operand_of(a[1]), *const w = operand_of(a[2]);
    const int code = (int)PyLong_AsLong(a[4]);
    void* const stream = pointer(a[6]);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor out;
    if (groups < 1) return refuse("offsets", "of one group at least"), nullptr;
    const Shape shape{{groups, x->rows, w->rows}};
    if (!product_out(a[5], *codes, shape, code, out)) return nullptr;
    if (!unlocked([&]() -> Done {
            product_new(*codes, shape, code, out);
            return {ufp4_mxfp4_gemm_bwd_dw_grouped(x, w, static_cast<int64_t*>(offsets), (int32_t)groups, out.data_ptr(), out.stride(1),
                                                   code_of(out), stream), "ufp4_mxfp4_gemm_bwd_dw_grouped"};
        }))
        return nullptr;
    return THPVariable_Wrap(out);
END_CALL

// (x, descriptor of W, out type, out, most tokens of the one-launch product, stream) -> y
CALL(mxfp4_linear, 6)
    const at::Tensor* const x = bf16_of(a[0]);
    if (!x) return nullptr;
    const ufp4_qtensor* const w = operand_of(a[1]);
    const int code = (int)PyLong_AsLong(a[2]);
    const int64_t most = PyLong_AsLongLong(a[4]);
    void* const stream = pointer(a[5]);
    if (PyErr_Occurred()) return nullptr;
    const int64_t tokens = x->size(0), red = x->size(1);
    if (red != w->red) {
        PyErr_Format(PyExc_ValueError, "x must have %lld columns", (long long)w->red);
        return nullptr;
    }
    // a grouped W's rows or reduction are padded: as the few-token product, the two calls below must not multiply the padding
    if (w->layout != UFP4_LAYOUT_PLAIN) return check(UFP4_ERR_MISMATCH, "ufp4_mxfp4_linear"), nullptr;
    const Shape shape{{0, tokens, w->rows}};
    at::Tensor out;
    if (!product_out(a[3], *x, shape, code, out)) return nullptr;
    if (!unlocked([&]() -> Done {
            product_new(*x, shape, code, out);
            if (tokens <= most && w->rht_block == 0)
                return {ufp4_mxfp4_linear(x->data_ptr(), tokens, x->stride(0), w, out.data_ptr(), out.stride(0), code_of(out), stream),
                        "ufp4_mxfp4_linear"};
            ufp4_qtensor d;  // x as W was rotated
            at::Tensor codes, scales;
            Done done = new_operand(*x, tokens, red, d, codes, scales);
            if (done.status != UFP4_OK) return done;
            done = {ufp4_mxfp4_quantize(x->data_ptr(), tokens, red, x->stride(0), 0, w->rht_block != 0, w->rht_block ? w->sign_words[0] : 0,
                                        UFP4_ROUND_RTNE, 0, 0, &d, stream), "ufp4_mxfp4_quantize"};
            if (done.status != UFP4_OK) return done;
            return {ufp4_mxfp4_gemm_fwd_y(&d, w, out.data_ptr(), out.stride(0), code_of(out), stream), "ufp4_mxfp4_gemm_fwd_y"};
        }))
        return nullptr;
    return THPVariable_Wrap(out);
END_CALL

// (x or codes, codes): refuses two that are not on one GPU. A descriptor holds addresses, which the calls above cannot tell apart, so the
// binding asks this of an operand's tensor first.
CALL(on_one_gpu, 2)
    const at::Tensor* const x = tensor(a[0], "x");
    const at::Tensor* const codes = x ? tensor(a[1], "the operand's codes") : nullptr;
    if (!codes) return nullptr;
    if (!codes->is_cuda() || x->device() != codes->device()) {
        PyErr_Format(PyExc_ValueError, "the operand (%s) and the tensor or operand beside it (%s) must be on one CUDA device",
                     codes->device().str().c_str(), x->device().str().c_str());
        return nullptr;
    }
    Py_RETURN_NONE;
END_CALL

PyObject* set_error(PyObject*, PyObject* cls) {
    Py_INCREF(cls);
    Py_XDECREF(g_error);
    g_error = cls;
    Py_RETURN_NONE;
}

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {METHOD(layer_norm),   METHOD(layer_norm_bwd), METHOD(moe_sort),
                          METHOD(moe_dispatch), METHOD(moe_combine),    METHOD(moe_combine_bwd),
                          METHOD(mxfp4_quantize), METHOD(mxfp4_dequantize), METHOD(mxfp4_gemm_fwd_y),
                          METHOD(mxfp4_gemm_bwd_dx), METHOD(mxfp4_gemm_bwd_dw), METHOD(mxfp4_linear),
                          METHOD(mxfp4_quantize_dual), METHOD(mxfp4_quantize_grouped), METHOD(mxfp4_gemm_fwd_y_grouped),
                          METHOD(mxfp4_gemm_bwd_dx_grouped), METHOD(mxfp4_gemm_bwd_dw_grouped), METHOD(on_one_gpu),
                          {"set_error", set_error, METH_O, nullptr},    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_host", "Host side of the short calls of ufp4.py", -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host() { return PyModule_Create(&kModule); }
