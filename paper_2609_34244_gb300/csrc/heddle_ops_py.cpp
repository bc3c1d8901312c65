// heddle_ops_py.cpp -- the layer operators' calls from Python: torch tensors
// checked for shape, type and place, and packed into the C structs.
//
// A call of one token takes 3 to 8 us on the GPU; the same marshalling in
// Python, about 1 us a tensor, took longer (with the results' allocation: one
// row's product 13.3 us, now 9.6; norm with rotation 20.1, now 13.3; a small
// attention with its gradients 47, now 34).  Everything that the C side can
// check by itself is left to it.

#include <Python.h>

#include <cmath>
#include <stdexcept>
#include <string>

#include <ATen/core/Tensor.h>
#include <torch/csrc/autograd/python_variable.h>

#include "heddle.h"

namespace {

struct Refused : std::runtime_error {
    using std::runtime_error::runtime_error;
};
struct PythonError {};  // one is set

PyObject *error_class = nullptr, *current_stream = nullptr;  // HeddleError; device index -> address
PyObject *name_value = nullptr, *name_stream = nullptr;
enum Entry { kLinear, kLinearGrad, kFfn, kFfnGrad, kNorm, kNormGrad, kAttention, kAttentionGrad, kEntries };
const char* const kNames[kEntries] = {"heddle_linear",       "heddle_linear_backward",
                                      "heddle_gated_ffn",    "heddle_gated_ffn_backward",
                                      "heddle_qk_norm_rope", "heddle_qk_norm_rope_backward",
                                      "heddle_attention",    "heddle_attention_backward"};
void* functions[kEntries];
int32_t (*device_of)(const heddle_ctx*) = nullptr;

std::string text(at::IntArrayRef s) {
    std::string r = "(";
    for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
    return r + (s.size() == 1 ? ",)" : ")");
}

const at::Tensor& tensor(const char* what, PyObject* o) {
    if (!THPVariable_Check(o))
        throw Refused(std::string(what) + ": expected a CUDA tensor, got " + Py_TYPE(o)->tp_name);
    return THPVariable_Unpack(o);
}

[[noreturn]] void bad(const char* what, const at::Tensor& t, at::IntArrayRef shape, at::ScalarType type) {
    throw Refused(std::string(what) + ": expected a CUDA tensor " + text(shape) + " of " + c10::toString(type) +
                  " with a contiguous last axis, got " + text(t.sizes()) + " of " + c10::toString(t.scalar_type()) +
                  " on " + t.device().str());
}

bool fits(const at::Tensor& t, at::IntArrayRef shape, at::ScalarType type, int device) {
    return t.scalar_type() == type && t.sizes() == shape && t.is_cuda() && t.device().index() == device;
}

// A call's first tensor, which gives the element type and the device.
struct First {
    const at::Tensor& t;
    at::ScalarType type;
    int32_t code;
    int device;
    First(const char* what, PyObject* o, size_t axes) : t(tensor(what, o)), type(t.scalar_type()) {
        if (type == at::kBFloat16)
            code = HEDDLE_BF16;
        else if (type == at::kHalf)
            code = HEDDLE_FP16;
        else if (type == at::kFloat)
            code = HEDDLE_FP32;
        else
            throw Refused(std::string("unsupported element type ") + c10::toString(type) + " of " + what);
        if (t.sizes().size() != axes || !t.is_cuda())
            throw Refused(std::string(what) + ": expected a CUDA tensor of " + std::to_string(axes) + " axes, got " +
                          text(t.sizes()) + " on " + t.device().str());
        device = t.device().index();
    }
    int64_t operator[](int i) const { return t.sizes()[i]; }
};

at::IntArrayRef axes_of(const char* what, PyObject* o, size_t axes) {
    const at::Tensor& t = tensor(what, o);
    if (t.sizes().size() != axes)
        throw Refused(std::string(what) + ": expected " + std::to_string(axes) + " axes, got " + text(t.sizes()));
    return t.sizes();
}

// A [rows][cols] tensor and its row stride; none for None.
struct Mat {
    void* p = nullptr;
    int64_t ld = 0;
    Mat(const char* what, PyObject* o, int64_t rows, int64_t cols, at::ScalarType type, int device) {
        if (o == Py_None) return;
        const at::Tensor& t = tensor(what, o);
        const int64_t shape[2] = {rows, cols};
        if (!fits(t, shape, type, device) || (t.strides()[1] != 1 && cols > 1)) bad(what, t, shape, type);
        ld = t.strides()[0];
        if (ld < cols && rows <= 1) ld = cols;
        p = t.data_ptr();
    }
};

void* vec(const char* what, PyObject* o, int64_t n, at::ScalarType type, int device) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(what, o);
    const int64_t shape[1] = {n};
    if (!fits(t, shape, type, device) || (n > 1 && t.strides()[0] != 1)) bad(what, t, shape, type);
    return t.data_ptr();
}

// A [batch][tokens][heads][head_dim] tensor, or one without the batch axis.
heddle_heads heads(const char* what, PyObject* o, at::IntArrayRef shape, const First& f) {
    const at::Tensor& t = tensor(what, o);
    const size_t n = shape.size();
    if (!fits(t, shape, f.type, f.device) || (t.strides()[n - 1] != 1 && shape[n - 1] > 1)) bad(what, t, shape, f.type);
    const at::IntArrayRef s = t.strides();
    return {t.data_ptr(), n == 4 ? s[0] : 0, s[n - 3], s[n - 2]};
}

// The stride of two tensors of so many rows; a single row's means nothing.
int64_t same_stride(const char* what, const Mat& a, const Mat& b, int64_t rows) {
    if (rows <= 1) return a.ld < b.ld ? b.ld : a.ld;
    if (a.ld != b.ld) throw Refused(std::string(what) + " have different row strides");
    return a.ld;
}

int64_t integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw PythonError();
    return v;
}
int32_t integer32(PyObject* o) {
    const int64_t v = integer(o);
    if (v != (int32_t)v) {
        PyErr_SetString(PyExc_OverflowError, "an argument does not fit into 32 bits");
        throw PythonError();
    }
    return (int32_t)v;
}
float real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PythonError();
    return (float)v;
}
bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw PythonError();
    return v != 0;
}

// An address: None, an integer, or what an object holds as `attribute` or as
// its value.
void* address(PyObject* o, PyObject* attribute) {
    if (o == Py_None) return nullptr;
    PyObject* held = nullptr;
    if (!PyLong_Check(o)) {
        held = PyObject_GetAttr(o, attribute);
        if (!held && attribute != name_value) {
            PyErr_Clear();
            held = PyObject_GetAttr(o, name_value);
        }
        if (!held) throw PythonError();
        o = held;
    }
    void* p = o == Py_None ? nullptr : PyLong_AsVoidPtr(o);
    Py_XDECREF(held);
    if (!p && PyErr_Occurred()) throw PythonError();
    return p;
}

template <class Args>
PyObject* call(Entry entry, PyObject* ctx, const Args& a, int device, PyObject* stream) {
    if (!functions[entry]) throw Refused("the library's functions are not bound");
    heddle_ctx* c = static_cast<heddle_ctx*>(address(ctx, name_value));
    if (c && device_of(c) != device)  // kernels would run there on this device's addresses
        throw Refused("the context is of cuda:" + std::to_string(device_of(c)) + ", the tensors are on cuda:" +
                      std::to_string(device));
    void* st;
    if (stream == Py_None) {
        PyObject* index = PyLong_FromLong(device);
        PyObject* now = index ? PyObject_CallOneArg(current_stream, index) : nullptr;
        Py_XDECREF(index);
        if (!now) throw PythonError();
        st = PyLong_AsVoidPtr(now);
        Py_DECREF(now);
        if (!st && PyErr_Occurred()) throw PythonError();
    } else {
        st = address(stream, name_stream);
    }
    const auto f = reinterpret_cast<heddle_status (*)(heddle_ctx*, const Args*, void*)>(functions[entry]);
    PyThreadState* held = PyEval_SaveThread();
    const heddle_status r = f(c, &a, st);
    PyEval_RestoreThread(held);
    return PyLong_FromLong(r);
}

// What a call returns to Python: its status, or an error.
template <int N, class F>
PyObject* guarded(Py_ssize_t n, F f) {
    try {
        if (n != N) throw Refused("expected " + std::to_string(N) + " arguments");
        return f();
    } catch (const PythonError&) {
    } catch (const Refused& e) {
        PyObject* v = PyObject_CallFunction(error_class ? error_class : PyExc_RuntimeError, "is", (int)HEDDLE_E_ARG,
                                            e.what());
        if (v) {
            PyErr_SetObject((PyObject*)Py_TYPE(v), v);
            Py_DECREF(v);
        }
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown error");
    }
    return nullptr;
}

// (ctx, x, w, y, bias, residual, act, pre, stream)
PyObject* linear(PyObject*, PyObject* const* v, Py_ssize_t count) {
    return guarded<9>(count, [&] {
        const First x("x", v[1], 2);
        heddle_linear_args a{};
        a.m = x[0], a.n = axes_of("w", v[2], 2)[0], a.k = x[1];
        a.dtype = x.code, a.act = integer32(v[6]);
        const Mat mx("x", v[1], a.m, a.k, x.type, x.device), w("w", v[2], a.n, a.k, x.type, x.device),
            r("residual", v[5], a.m, a.n, x.type, x.device), y("y", v[3], a.m, a.n, x.type, x.device),
            pre("pre", v[7], a.m, a.n, at::kFloat, x.device);
        a.x = mx.p, a.ldx = mx.ld, a.w = w.p, a.ldw = w.ld;
        a.bias = vec("bias", v[4], a.n, x.type, x.device);
        a.residual = r.p, a.ldr = r.ld, a.y = y.p, a.ldy = y.ld;
        a.pre = static_cast<float*>(pre.p), a.ldp = pre.ld;
        return call(kLinear, v[0], a, x.device, v[8]);
    });
}

// (ctx, dy, x, w, act, pre, dx, dw, dbias, stream)
PyObject* linear_backward(PyObject*, PyObject* const* v, Py_ssize_t count) {
    return guarded<10>(count, [&] {
        const First x("x", v[2], 2);
        heddle_linear_grad_args a{};
        a.m = x[0], a.n = axes_of("w", v[3], 2)[0], a.k = x[1];
        a.dtype = x.code, a.act = integer32(v[4]);
        const Mat dy("dy", v[1], a.m, a.n, x.type, x.device), mx("x", v[2], a.m, a.k, x.type, x.device),
            w("w", v[3], a.n, a.k, x.type, x.device), pre("pre", v[5], a.m, a.n, at::kFloat, x.device),
            dx("dx", v[6], a.m, a.k, x.type, x.device), dw("dw", v[7], a.n, a.k, x.type, x.device);
        a.dy = dy.p, a.lddy = dy.ld, a.x = mx.p, a.ldx = mx.ld, a.w = w.p, a.ldw = w.ld;
        a.pre = static_cast<float*>(pre.p), a.ldp = pre.ld;
        a.dx = dx.p, a.lddx = dx.ld, a.dw = dw.p, a.lddw = dw.ld;
        a.dbias = vec("dbias", v[8], a.n, x.type, x.device);
        return call(kLinearGrad, v[0], a, x.device, v[9]);
    });
}

// (ctx, x, w_gate, w_up, y, act, gate, up, stream)
PyObject* gated_ffn(PyObject*, PyObject* const* v, Py_ssize_t count) {
    return guarded<9>(count, [&] {
        const First x("x", v[1], 2);
        heddle_gated_ffn_args a{};
        a.m = x[0], a.n = axes_of("w_gate", v[2], 2)[0], a.k = x[1];
        a.dtype = x.code, a.act = integer32(v[5]);
        const Mat gate("gate", v[6], a.m, a.n, at::kFloat, x.device), up("up", v[7], a.m, a.n, at::kFloat, x.device);
        a.lds = same_stride("gate and up", gate, up, a.m);
        a.gate = static_cast<float*>(gate.p), a.up = static_cast<float*>(up.p);
        const Mat mx("x", v[1], a.m, a.k, x.type, x.device), wg("w_gate", v[2], a.n, a.k, x.type, x.device),
            wu("w_up", v[3], a.n, a.k, x.type, x.device), y("y", v[4], a.m, a.n, x.type, x.device);
        a.x = mx.p, a.ldx = mx.ld, a.w_gate = wg.p, a.ldg = wg.ld, a.w_up = wu.p, a.ldu = wu.ld;
        a.y = y.p, a.ldy = y.ld;
        return call(kFfn, v[0], a, x.device, v[8]);
    });
}

// (ctx, dy, x, w_gate, w_up, gate, up, act, dx, dwg, dwu, stream)
PyObject* gated_ffn_backward(PyObject*, PyObject* const* v, Py_ssize_t count) {
    return guarded<12>(count, [&] {
        const First x("x", v[2], 2);
        heddle_gated_ffn_grad_args a{};
        a.m = x[0], a.n = axes_of("w_gate", v[3], 2)[0], a.k = x[1];
        a.dtype = x.code, a.act = integer32(v[7]);
        const Mat gate("gate", v[5], a.m, a.n, at::kFloat, x.device), up("up", v[6], a.m, a.n, at::kFloat, x.device);
        a.lds = same_stride("gate and up", gate, up, a.m);
        a.gate = static_cast<float*>(gate.p), a.up = static_cast<float*>(up.p);
        const Mat dwg("dwg", v[9], a.n, a.k, x.type, x.device), dwu("dwu", v[10], a.n, a.k, x.type, x.device);
        a.lddw = same_stride("dwg and dwu", dwg, dwu, a.n);
        a.dw_gate = dwg.p, a.dw_up = dwu.p;
        const Mat dy("dy", v[1], a.m, a.n, x.type, x.device), mx("x", v[2], a.m, a.k, x.type, x.device),
            wg("w_gate", v[3], a.n, a.k, x.type, x.device), wu("w_up", v[4], a.n, a.k, x.type, x.device),
            dx("dx", v[8], a.m, a.k, x.type, x.device);
        a.dy = dy.p, a.lddy = dy.ld, a.x = mx.p, a.ldx = mx.ld;
        a.w_gate = wg.p, a.ldg = wg.ld, a.w_up = wu.p, a.ldu = wu.ld, a.dx = dx.p, a.lddx = dx.ld;
        return call(kFfnGrad, v[0], a, x.device, v[11]);
    });
}

// v: q, k, wq, wk, q_out, k_out, positions, cos, sin, eps, interleaved; the
// gradient's call gives its outputs' gradients as q_out and k_out.
void norm_args(heddle_qk_norm_rope_args& a, const First& q, PyObject* const* v, int64_t (&keys)[3]) {
    const int64_t d = q[2];
    keys[0] = q[0], keys[1] = axes_of("k", v[1], 3)[1], keys[2] = d;
    a.tokens = q[0];
    if (q[1] > INT32_MAX || keys[1] > INT32_MAX || d > INT32_MAX) throw Refused("heads do not fit into 32 bits");
    a.q_heads = (int32_t)q[1], a.k_heads = (int32_t)keys[1], a.head_dim = (int32_t)d;
    a.dtype = q.code, a.interleaved = truth(v[10]), a.eps = real(v[9]);
    if (v[6] != Py_None) {
        const at::IntArrayRef angles = axes_of("cos", v[7], 2);
        if (angles[1] > INT32_MAX / 2) throw Refused("rot_dim does not fit into 32 bits");
        a.table_len = angles[0], a.rot_dim = (int32_t)(2 * angles[1]);
        a.positions = static_cast<const int32_t*>(vec("positions", v[6], q[0], at::kInt, q.device));
        const Mat c("cos", v[7], angles[0], angles[1], at::kFloat, q.device),
            s("sin", v[8], angles[0], angles[1], at::kFloat, q.device);
        if (v[8] == Py_None || !tensor("cos", v[7]).is_contiguous() || !tensor("sin", v[8]).is_contiguous())
            throw Refused("cos and sin are contiguous");
        a.cos = static_cast<const float*>(c.p), a.sin = static_cast<const float*>(s.p);
    }
    a.q = heads("q", v[0], q.t.sizes(), q), a.k = heads("k", v[1], keys, q);
    a.wq = vec("wq", v[2], d, q.type, q.device), a.wk = vec("wk", v[3], d, q.type, q.device);
    a.q_out = heads("q_out", v[4], q.t.sizes(), q), a.k_out = heads("k_out", v[5], keys, q);
}

// (ctx, q, k, wq, wk, q_out, k_out, positions, cos, sin, eps, interleaved, stream)
PyObject* qk_norm_rope(PyObject*, PyObject* const* v, Py_ssize_t count) {
    return guarded<13>(count, [&] {
        const First q("q", v[1], 3);
        heddle_qk_norm_rope_args a{};
        int64_t keys[3];
        norm_args(a, q, v + 1, keys);
        return call(kNorm, v[0], a, q.device, v[12]);
    });
}

// (ctx, q, k, wq, wk, dq_out, dk_out, positions, cos, sin, eps, interleaved, dq, dk, dwq, dwk, stream)
PyObject* qk_norm_rope_backward(PyObject*, PyObject* const* v, Py_ssize_t count) {
    return guarded<17>(count, [&] {
        const First q("q", v[1], 3);
        heddle_qk_norm_rope_grad_args a{};
        int64_t keys[3];
        norm_args(a.fwd, q, v + 1, keys);
        a.dq = heads("dq", v[12], q.t.sizes(), q), a.dk = heads("dk", v[13], keys, q);
        a.dwq = static_cast<float*>(vec("dwq", v[14], q[2], at::kFloat, q.device));
        a.dwk = static_cast<float*>(vec("dwk", v[15], q[2], at::kFloat, q.device));
        return call(kNormGrad, v[0], a, q.device, v[16]);
    });
}

// v: q, k, v, o, lse, q_lens, kv_lens, window, sinks, scale
void attention_args(heddle_attention_args& a, const First& q, PyObject* const* v, int64_t (&keys)[4]) {
    const at::IntArrayRef ks = axes_of("k", v[1], 4);
    const int64_t b = q[0], d = q[3];
    keys[0] = b, keys[1] = ks[1], keys[2] = ks[2], keys[3] = d;
    if (q[2] > INT32_MAX || keys[2] > INT32_MAX || d > INT32_MAX) throw Refused("heads do not fit into 32 bits");
    a.batch = b, a.q_len = q[1], a.kv_len = keys[1];
    a.q_heads = (int32_t)q[2], a.kv_heads = (int32_t)keys[2], a.head_dim = (int32_t)d, a.dtype = q.code;
    a.window = integer(v[7]), a.sinks = integer(v[8]);
    a.scale = v[9] == Py_None ? (float)std::pow((double)d, -0.5) : real(v[9]);
    if (v[4] != Py_None) {
        const at::Tensor& t = tensor("lse", v[4]);
        const int64_t shape[3] = {b, q[2], q[1]};
        if (!fits(t, shape, at::kFloat, q.device) || !t.is_contiguous()) bad("lse", t, shape, at::kFloat);
        a.lse = static_cast<float*>(t.data_ptr());
    }
    a.q = heads("q", v[0], q.t.sizes(), q), a.k = heads("k", v[1], keys, q), a.v = heads("v", v[2], keys, q);
    a.o = heads("o", v[3], q.t.sizes(), q);
    a.q_lens = static_cast<const int32_t*>(vec("q_lens", v[5], b, at::kInt, q.device));
    a.kv_lens = static_cast<const int32_t*>(vec("kv_lens", v[6], b, at::kInt, q.device));
}

// (ctx, q, k, v, o, lse, q_lens, kv_lens, window, sinks, scale, stream)
PyObject* attention(PyObject*, PyObject* const* v, Py_ssize_t count) {
    return guarded<12>(count, [&] {
        const First q("q", v[1], 4);
        heddle_attention_args a{};
        int64_t keys[4];
        attention_args(a, q, v + 1, keys);
        return call(kAttention, v[0], a, q.device, v[11]);
    });
}

// (ctx, q, k, v, o, lse, q_lens, kv_lens, window, sinks, scale, do, dq, dk, dv, stream)
PyObject* attention_backward(PyObject*, PyObject* const* v, Py_ssize_t count) {
    return guarded<16>(count, [&] {
        const First q("q", v[1], 4);
        heddle_attention_grad_args a{};
        int64_t keys[4];
        attention_args(a.fwd, q, v + 1, keys);
        a.d_o = heads("do", v[11], q.t.sizes(), q), a.dq = heads("dq", v[12], q.t.sizes(), q);
        a.dk = heads("dk", v[13], keys, q), a.dv = heads("dv", v[14], keys, q);
        return call(kAttentionGrad, v[0], a, q.device, v[15]);
    });
}

// (the functions' addresses by name, HeddleError, device index -> current stream)
PyObject* bind(PyObject*, PyObject* const* v, Py_ssize_t count) {
    return guarded<3>(count, [&] {
        void* found[kEntries + 1];
        for (int i = 0; i <= kEntries; ++i) {
            PyObject* p = PyMapping_GetItemString(v[0], i < kEntries ? kNames[i] : "heddle_device");
            if (!p) throw PythonError();
            found[i] = PyLong_AsVoidPtr(p);
            Py_DECREF(p);
            if (PyErr_Occurred()) throw PythonError();
        }
        for (int i = 0; i < kEntries; ++i) functions[i] = found[i];
        device_of = reinterpret_cast<int32_t (*)(const heddle_ctx*)>(found[kEntries]);
        Py_INCREF(v[1]), Py_INCREF(v[2]);
        Py_XSETREF(error_class, v[1]);
        Py_XSETREF(current_stream, v[2]);
        Py_INCREF(Py_None);
        return Py_None;
    });
}

#define METHOD(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(bind),
                         METHOD(linear),
                         METHOD(linear_backward),
                         METHOD(gated_ffn),
                         METHOD(gated_ffn_backward),
                         METHOD(qk_norm_rope),
                         METHOD(qk_norm_rope_backward),
                         METHOD(attention),
                         METHOD(attention_backward),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_heddle_ops", "Marshalling of the layer operators' calls.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__heddle_ops() {
    name_value = PyUnicode_InternFromString("value");
    name_stream = PyUnicode_InternFromString("cuda_stream");
    return name_value && name_stream ? PyModule_Create(&module) : nullptr;
}
