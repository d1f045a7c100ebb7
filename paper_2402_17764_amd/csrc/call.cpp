// The argument marshalling of binding.py's hot entry points, in C++: tensor checks, output allocation, the current HIP stream
// and the call through the C ABI.  A decode launch on a small layer takes the GPU four to five microseconds; done in Python
// (a dozen attribute reads, two torch calls and the ctypes conversion) the marshalling took six and a half of the 10.7 us
// that linear_fused on 1536 -> 4096 took per call; now the call takes 5.0, of which the launch itself is 4.3.
//
// binding.load() hands over the C ABI's function addresses (bind) -- the library stays whichever one it loaded -- and its
// BitnetError class.  The checks, their order and their messages are those of binding.py's own helpers.  The GIL is released
// around the call, as ctypes does.
#include <Python.h>

#include <algorithm>
#include <cmath>

#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "bitnet.h"

namespace {

struct Abi {
    decltype(&bitnet_quantize_acts) quantize_acts;
    decltype(&bitnet_rmsnorm_quantize) rmsnorm_quantize;
    decltype(&bitnet_swiglu_quantize) swiglu_quantize;
    decltype(&bitnet_linear) linear;
    decltype(&bitnet_linear_variant) linear_variant;
    decltype(&bitnet_linear_segmented) linear_segmented;
    decltype(&bitnet_linear_ws) linear_ws;
    decltype(&bitnet_linear_fused) linear_fused;
    decltype(&bitnet_linear_fused_segmented) linear_fused_segmented;
    decltype(&bitnet_rmsnorm_linear_fused) rmsnorm_linear_fused;
    decltype(&bitnet_rmsnorm_linear_fused_segmented) rmsnorm_linear_fused_segmented;
    decltype(&bitnet_swiglu_linear_fused) swiglu_linear_fused;
    decltype(&bitnet_ffn_gate_up_fused) ffn_gate_up_fused;
    decltype(&bitnet_rope_kv_append) rope_kv_append;
    decltype(&bitnet_attention_workspace) attention_workspace;
    decltype(&bitnet_attention_decode) attention_decode;
    decltype(&bitnet_attention_prefill) attention_prefill;
    decltype(&bitnet_norm_rope_kv_append) norm_rope_kv_append;
    decltype(&bitnet_attention_shared_workspace) attention_shared_workspace;
    decltype(&bitnet_attention_decode_shared) attention_decode_shared;
    decltype(&bitnet_attention_weights_workspace) attention_weights_workspace;
    decltype(&bitnet_attention_decode_weights) attention_decode_weights;
    decltype(&bitnet_attention_prefill_weights) attention_prefill_weights;
    decltype(&bitnet_kv_evict) kv_evict;
} abi;
PyObject* error_class = nullptr;

// A Python exception is set: unwinds to the entry point, which returns NULL.
struct Raised {};
template <typename... A>
[[noreturn]] void raise(PyObject* type, const char* fmt, A... a) {
    PyErr_Format(type, fmt, a...);
    throw Raised();
}

const char* dtype_name(at::ScalarType t) {
    switch (t) {
        case at::kFloat: return "torch.float32";
        case at::kDouble: return "torch.float64";
        case at::kHalf: return "torch.float16";
        case at::kBFloat16: return "torch.bfloat16";
        case at::kByte: return "torch.uint8";
        case at::kChar: return "torch.int8";
        case at::kShort: return "torch.int16";
        case at::kInt: return "torch.int32";
        case at::kLong: return "torch.int64";
        case at::kBool: return "torch.bool";
        default: return c10::toString(t);
    }
}

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) raise(PyExc_TypeError, "%s must be a CUDA/HIP tensor", name);
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda()) raise(PyExc_TypeError, "%s must be a CUDA/HIP tensor", name);
    if (!t.is_contiguous()) raise(PyExc_ValueError, "%s must be contiguous", name);
    return t;
}
const at::Tensor& tensor(PyObject* o, const char* name, at::ScalarType dt) {
    const at::Tensor& t = tensor(o, name);
    if (t.scalar_type() != dt) raise(PyExc_TypeError, "%s has dtype %s", name, dtype_name(t.scalar_type()));
    return t;
}
void two_d(const at::Tensor& t, const char* name) {
    if (t.dim() != 2) raise(PyExc_ValueError, "%s must be 2-D", name);
}
// a float matrix: fp32 or bf16, two dimensions
const at::Tensor& matrix(PyObject* o, const char* name, bitnet_dtype* dt) {
    const at::Tensor& t = tensor(o, name);
    if (t.scalar_type() == at::kFloat) *dt = BITNET_F32;
    else if (t.scalar_type() == at::kBFloat16) *dt = BITNET_BF16;
    else raise(PyExc_TypeError, "%s has dtype %s", name, dtype_name(t.scalar_type()));
    two_d(t, name);
    return t;
}
const at::Tensor& int8_matrix(PyObject* o, const char* name) {
    const at::Tensor& t = tensor(o, name, at::kChar);
    two_d(t, name);
    return t;
}

int64_t integer(PyObject* o) {
    PyObject* i = PyNumber_Index(o);
    if (!i) throw Raised();
    const unsigned long long v = PyLong_AsUnsignedLongLongMask(i);
    Py_DECREF(i);
    if (v == (unsigned long long)-1 && PyErr_Occurred()) throw Raised();
    return (int64_t)v;
}
float real(PyObject* o) {
    PyObject* f = PyNumber_Float(o);
    if (!f) throw Raised();
    const double v = PyFloat_AS_DOUBLE(f);
    Py_DECREF(f);
    return (float)v;
}
bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Raised();
    return v != 0;
}

at::ScalarType out_type(PyObject* code) {
    if (PyIndex_Check(code)) {
        switch (integer(code)) {
            case BITNET_F32: return at::kFloat;
            case BITNET_BF16: return at::kBFloat16;
            case BITNET_I32: return at::kInt;
            default: break;
        }
    }
    PyErr_SetObject(PyExc_KeyError, code);
    throw Raised();
}
// the caller's output tensor, or a new one on x's device
at::Tensor output(PyObject* given, const char* name, at::IntArrayRef shape, at::ScalarType dt, const at::Tensor& x) {
    if (given == Py_None) return at::empty(shape, at::TensorOptions().dtype(dt).device(x.device()));
    return tensor(given, name, dt);
}
const float* gain(PyObject* g, int64_t K, bool check_shape) {
    if (g == Py_None) return nullptr;
    const at::Tensor& t = tensor(g, "g", at::kFloat);
    if (check_shape && (t.dim() != 1 || t.size(0) != K)) raise(PyExc_ValueError, "g must have one entry per column");
    return static_cast<const float*>(t.const_data_ptr());
}
const float* floats(PyObject* o, const char* name) { return static_cast<const float*>(tensor(o, name, at::kFloat).const_data_ptr()); }
const float* per_block(PyObject* o, const char* name, int64_t N) {
    const at::Tensor& t = tensor(o, name, at::kFloat);
    if (t.numel() < (N + 15) / 16) raise(PyExc_ValueError, "%s needs one entry per 16-row block", name);
    return static_cast<const float*>(t.const_data_ptr());
}

void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

// other threads may run until it goes out of scope, however that happens
struct GilReleased {
    PyThreadState* state = PyEval_SaveThread();
    ~GilReleased() { PyEval_RestoreThread(state); }
};

template <typename F>
void call(const char* where, F&& f) {
    const bitnet_status st = [&] { GilReleased released; return f(); }();
    if (st == BITNET_OK) return;
    PyObject* e = PyObject_CallFunction(error_class, "is", (int)st, where);
    if (e) {
        PyErr_SetObject(error_class, e);
        Py_DECREF(e);
    }
    throw Raised();
}

// Every entry point: a fixed number of positional arguments; C++ exceptions become Python ones.
template <typename F>
PyObject* entry(Py_ssize_t n, Py_ssize_t want, F&& f) {
    HANDLE_TH_ERRORS
    if (!error_class) {
        PyErr_SetString(PyExc_RuntimeError, "bind() has not been called");
        return nullptr;
    }
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "%zd arguments expected", want);
        return nullptr;
    }
    try {
        return f();
    } catch (const Raised&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}
PyObject* pair(const at::Tensor& a, const at::Tensor& b) {
    PyObject* pa = THPVariable_Wrap(a);
    PyObject* pb = pa ? THPVariable_Wrap(b) : nullptr;
    PyObject* t = pb ? PyTuple_Pack(2, pa, pb) : nullptr;
    Py_XDECREF(pa);
    Py_XDECREF(pb);
    return t;
}

#define ENTRY(name_) PyObject* name_(PyObject*, PyObject* const* a, Py_ssize_t n)

ENTRY(quantize_acts) {      // x, xq, sx
    return entry(n, 3, [&] {
        bitnet_dtype dt;
        const at::Tensor& x = matrix(a[0], "x", &dt);
        const int64_t M = x.size(0), K = x.size(1);
        at::Tensor xq = output(a[1], "xq", {M, K}, at::kChar, x), sx = output(a[2], "sx", {M}, at::kFloat, x);
        const void* xp = x.const_data_ptr();
        int8_t* qp = static_cast<int8_t*>(xq.mutable_data_ptr());
        float* sp = static_cast<float*>(sx.mutable_data_ptr());
        void* st = stream();
        call("bitnet_quantize_acts", [&] { return abi.quantize_acts(xp, dt, M, K, qp, sp, st); });
        return pair(xq, sx);
    });
}

ENTRY(rmsnorm_quantize) {      // x, g, eps, xq, sx
    return entry(n, 5, [&] {
        bitnet_dtype dt;
        const at::Tensor& x = matrix(a[0], "x", &dt);
        const int64_t M = x.size(0), K = x.size(1);
        at::Tensor xq = output(a[3], "xq", {M, K}, at::kChar, x), sx = output(a[4], "sx", {M}, at::kFloat, x);
        const float* g = gain(a[1], K, true);
        const float eps = real(a[2]);
        const void* xp = x.const_data_ptr();
        int8_t* qp = static_cast<int8_t*>(xq.mutable_data_ptr());
        float* sp = static_cast<float*>(sx.mutable_data_ptr());
        void* st = stream();
        call("bitnet_rmsnorm_quantize", [&] { return abi.rmsnorm_quantize(xp, dt, g, eps, M, K, qp, sp, st); });
        return pair(xq, sx);
    });
}

ENTRY(swiglu_quantize) {      // gu, hq, sh
    return entry(n, 3, [&] {
        bitnet_dtype dt;
        const at::Tensor& gu = matrix(a[0], "gu", &dt);
        const int64_t M = gu.size(0);
        if (gu.size(1) % 2) raise(PyExc_ValueError, "gu must have an even number of columns");
        const int64_t F = gu.size(1) / 2;
        at::Tensor hq = output(a[1], "hq", {M, F}, at::kChar, gu), sh = output(a[2], "sh", {M}, at::kFloat, gu);
        const void* gp = gu.const_data_ptr();
        int8_t* qp = static_cast<int8_t*>(hq.mutable_data_ptr());
        float* sp = static_cast<float*>(sh.mutable_data_ptr());
        void* st = stream();
        call("bitnet_swiglu_quantize", [&] { return abi.swiglu_quantize(gp, dt, M, F, qp, sp, st); });
        return pair(hq, sh);
    });
}

// the product's operands that every linear entry point shares
struct Product {
    const at::Tensor& xq;
    int64_t M, K, N;
    at::Tensor y;
    const int8_t* xp;
    const float* sx;
    const void* packed;
    void* yp;
    bitnet_format f;
    bitnet_dtype yt;
    Product(PyObject* oxq, PyObject* osx, PyObject* opacked, PyObject* oN, PyObject* ofmt, PyObject* oyt, PyObject* oy)
        : xq(int8_matrix(oxq, "xq")), M(xq.size(0)), K(xq.size(1)), N(integer(oN)), y(output(oy, "y", {M, N}, out_type(oyt), xq)),
          xp(static_cast<const int8_t*>(xq.const_data_ptr())), sx(floats(osx, "sx")),
          packed(tensor(opacked, "packed").const_data_ptr()), yp(y.mutable_data_ptr()), f((bitnet_format)(int)integer(ofmt)),
          yt((bitnet_dtype)(int)integer(oyt)) {}
};

ENTRY(linear) {      // xq, sx, packed, gamma, N, fmt, y_dtype, y, kernel
    return entry(n, 9, [&] {
        Product p(a[0], a[1], a[2], a[4], a[5], a[6], a[7]);
        const float* gamma = floats(a[3], "gamma");
        const bitnet_kernel which = (bitnet_kernel)(int)integer(a[8]);
        void* st = stream();
        if (which == BITNET_KERNEL_AUTO)
            call("bitnet_linear", [&] { return abi.linear(p.xp, p.sx, p.packed, gamma, p.M, p.N, p.K, p.f, p.yp, p.yt, st); });
        else
            call("bitnet_linear_variant", [&] { return abi.linear_variant(p.xp, p.sx, p.packed, gamma, p.M, p.N, p.K, p.f, p.yp, p.yt, which, st); });
        return THPVariable_Wrap(p.y);
    });
}

ENTRY(linear_segmented) {      // xq, sx, packed, gamma_rb, N, fmt, y_dtype, y, kernel
    return entry(n, 9, [&] {
        Product p(a[0], a[1], a[2], a[4], a[5], a[6], a[7]);
        const float* gamma = per_block(a[3], "gamma_rb", p.N);
        const bitnet_kernel which = (bitnet_kernel)(int)integer(a[8]);
        void* st = stream();
        call("bitnet_linear_segmented", [&] { return abi.linear_segmented(p.xp, p.sx, p.packed, gamma, p.M, p.N, p.K, p.f, p.yp, p.yt, which, st); });
        return THPVariable_Wrap(p.y);
    });
}

ENTRY(linear_ws) {      // xq, sx, packed, gamma, N, fmt, y_dtype, y, kernel, workspace, gamma_per_block
    return entry(n, 11, [&] {
        Product p(a[0], a[1], a[2], a[4], a[5], a[6], a[7]);
        const float* gamma = floats(a[3], "gamma");
        const bitnet_kernel which = (bitnet_kernel)(int)integer(a[8]);
        void* ws = nullptr;
        size_t bytes = 0;
        if (a[9] != Py_None) {
            const at::Tensor& w = tensor(a[9], "workspace");
            ws = w.mutable_data_ptr();
            bytes = (size_t)w.numel() * w.element_size();
        }
        const int per = truth(a[10]) ? 1 : 0;
        void* st = stream();
        call("bitnet_linear_ws", [&] { return abi.linear_ws(p.xp, p.sx, p.packed, gamma, per, p.M, p.N, p.K, p.f, p.yp, p.yt, which, ws, bytes, st); });
        return THPVariable_Wrap(p.y);
    });
}

ENTRY(linear_fused) {      // x, packed, gamma, N, fmt, y_dtype, y, segmented
    return entry(n, 8, [&] {
        bitnet_dtype dt;
        const at::Tensor& x = matrix(a[0], "x", &dt);
        const int64_t M = x.size(0), K = x.size(1), N = integer(a[3]);
        at::Tensor y = output(a[6], "y", {M, N}, out_type(a[5]), x);
        const bool seg = truth(a[7]);
        const float* gamma = seg ? per_block(a[2], "gamma_rb", N) : floats(a[2], "gamma");
        const void *xp = x.const_data_ptr(), *w = tensor(a[1], "packed").const_data_ptr();
        const bitnet_format f = (bitnet_format)(int)integer(a[4]);
        const bitnet_dtype yt = (bitnet_dtype)(int)integer(a[5]);
        void *yp = y.mutable_data_ptr(), *st = stream();
        call(seg ? "bitnet_linear_fused_segmented" : "bitnet_linear_fused",
             [&] { return (seg ? abi.linear_fused_segmented : abi.linear_fused)(xp, dt, w, gamma, M, N, K, f, yp, yt, st); });
        return THPVariable_Wrap(y);
    });
}

ENTRY(rmsnorm_linear_fused) {      // x, g, eps, packed, gamma, N, fmt, y_dtype, y, segmented
    return entry(n, 10, [&] {
        bitnet_dtype dt;
        const at::Tensor& x = matrix(a[0], "x", &dt);
        const int64_t M = x.size(0), K = x.size(1), N = integer(a[5]);
        at::Tensor y = output(a[8], "y", {M, N}, out_type(a[7]), x);
        const float* g = gain(a[1], K, true);
        const float eps = real(a[2]);
        const bool seg = truth(a[9]);
        const float* gamma = seg ? per_block(a[4], "gamma", N) : floats(a[4], "gamma");
        const void *xp = x.const_data_ptr(), *w = tensor(a[3], "packed").const_data_ptr();
        const bitnet_format f = (bitnet_format)(int)integer(a[6]);
        const bitnet_dtype yt = (bitnet_dtype)(int)integer(a[7]);
        void *yp = y.mutable_data_ptr(), *st = stream();
        call(seg ? "bitnet_rmsnorm_linear_fused_segmented" : "bitnet_rmsnorm_linear_fused", [&] {
            return (seg ? abi.rmsnorm_linear_fused_segmented : abi.rmsnorm_linear_fused)(xp, dt, g, eps, w, gamma, M, N, K, f, yp, yt, st);
        });
        return THPVariable_Wrap(y);
    });
}

ENTRY(swiglu_linear_fused) {      // gu, packed, gamma, N, fmt, y_dtype, y
    return entry(n, 7, [&] {
        bitnet_dtype dt;
        const at::Tensor& gu = matrix(a[0], "gu", &dt);
        const int64_t M = gu.size(0), N = integer(a[3]);
        if (gu.size(1) % 2) raise(PyExc_ValueError, "gu must hold a gate and an up half");
        const int64_t F = gu.size(1) / 2;
        at::Tensor y = output(a[6], "y", {M, N}, out_type(a[5]), gu);
        const float* gamma = floats(a[2], "gamma");
        const void *gp = gu.const_data_ptr(), *w = tensor(a[1], "packed").const_data_ptr();
        const bitnet_format f = (bitnet_format)(int)integer(a[4]);
        const bitnet_dtype yt = (bitnet_dtype)(int)integer(a[5]);
        void *yp = y.mutable_data_ptr(), *st = stream();
        call("bitnet_swiglu_linear_fused", [&] { return abi.swiglu_linear_fused(gp, dt, w, gamma, M, N, F, f, yp, yt, st); });
        return THPVariable_Wrap(y);
    });
}

ENTRY(ffn_gate_up_fused) {      // x, packed, gamma, F, norm, g, eps, gamma_per_block, fmt, h_dtype, h
    return entry(n, 11, [&] {
        bitnet_dtype dt;
        const at::Tensor& x = matrix(a[0], "x", &dt);
        const int64_t M = x.size(0), K = x.size(1), F = integer(a[3]);
        at::Tensor h = output(a[10], "h", {M, F}, out_type(a[9]), x);
        const int norm = truth(a[4]) ? 1 : 0, per = truth(a[7]) ? 1 : 0;
        const float* g = gain(a[5], K, false);
        const float eps = real(a[6]);
        const float* gamma = floats(a[2], "gamma");
        const void *xp = x.const_data_ptr(), *w = tensor(a[1], "packed").const_data_ptr();
        const bitnet_format f = (bitnet_format)(int)integer(a[8]);
        const bitnet_dtype ht = (bitnet_dtype)(int)integer(a[9]);
        void *hp = h.mutable_data_ptr(), *st = stream();
        call("bitnet_ffn_gate_up_fused", [&] { return abi.ffn_gate_up_fused(xp, dt, norm, g, eps, w, gamma, per, M, F, K, f, hp, ht, st); });
        return THPVariable_Wrap(h);
    });
}

// The cache and its sequences as the C ABI takes them: k_cache [pages, kv heads, page tokens / 32, Dp / 8, 32, 8] and v_cache [pages, kv heads,
// page tokens / 32, 4, Dp, 8] (bf16), page_table [B, pages of a sequence] (int32, its rows may be strided), kv_len [B] and q_start [B + 1] or None (int32).
// Every tensor has to be on x's device, which is the current one while the call lasts.
struct Cache {
    const at::Tensor& x;
    c10::DeviceGuard on;
    bitnet_kv kv;
    const at::Tensor& here(PyObject* o, const char* name, at::ScalarType dt) const { return here(tensor(o, name, dt), name); }
    const at::Tensor& here(const at::Tensor& t, const char* name) const {
        if (t.device() != x.device()) raise(PyExc_ValueError, "%s is on another device", name);
        return t;
    }
    Cache(const at::Tensor& x_, int64_t head_dim, PyObject* ok, PyObject* ov, PyObject* otable, PyObject* olen, PyObject* ostart) : x(x_), on(x_.device()) {
        const at::Tensor &k = here(ok, "k_cache", at::kBFloat16), &v = here(ov, "v_cache", at::kBFloat16);
        const int64_t Dp = (head_dim + 7) / 8 * 8;
        if (k.dim() != 6 || k.size(3) != Dp / 8 || k.size(4) != 32 || k.size(5) != 8)
            raise(PyExc_ValueError, "k_cache must be [pages, kv heads, page tokens / 32, %lld, 32, 8] for heads of %lld", (long long)(Dp / 8), (long long)head_dim);
        if (v.dim() != 6 || v.size(0) != k.size(0) || v.size(1) != k.size(1) || v.size(2) != k.size(2) || v.size(3) != 4 || v.size(4) != Dp || v.size(5) != 8)
            raise(PyExc_ValueError, "v_cache must be [pages, kv heads, page tokens / 32, 4, %lld, 8], of the pages of k_cache", (long long)Dp);
        if (!THPVariable_Check(otable) || !THPVariable_Unpack(otable).is_cuda()) raise(PyExc_TypeError, "page_table must be a CUDA/HIP tensor");
        const at::Tensor& table = here(THPVariable_Unpack(otable), "page_table");
        if (table.scalar_type() != at::kInt) raise(PyExc_TypeError, "page_table has dtype %s", dtype_name(table.scalar_type()));
        two_d(table, "page_table");
        const int64_t B = table.size(0), pages = table.size(1);
        if ((pages > 1 && table.stride(1) != 1) || (B > 1 && table.stride(0) < pages)) raise(PyExc_ValueError, "page_table must have contiguous rows");
        const at::Tensor& len = here(olen, "kv_len", at::kInt);
        if (len.dim() != 1 || len.size(0) != B) raise(PyExc_ValueError, "kv_len must have one entry per row of page_table");
        const int32_t* start = nullptr;
        if (ostart != Py_None) {
            const at::Tensor& t = here(ostart, "q_start", at::kInt);
            if (t.dim() != 1 || t.size(0) != B + 1) raise(PyExc_ValueError, "q_start must have one entry more than page_table has rows");
            start = static_cast<const int32_t*>(t.const_data_ptr());
        }
        kv = {k.mutable_data_ptr(), v.mutable_data_ptr(), k.size(0), k.size(2) * 32, k.size(1), head_dim, B, static_cast<const int32_t*>(table.const_data_ptr()),
              B > 1 ? table.stride(0) : pages, pages, static_cast<const int32_t*>(len.const_data_ptr()), start};
    }
    at::Tensor output(PyObject* given, const char* name, at::IntArrayRef shape, at::ScalarType dt) const {
        if (given == Py_None) return at::empty(shape, at::TensorOptions().dtype(dt).device(x.device()));
        const at::Tensor& t = here(given, name, dt);
        if (t.sizes() != shape) raise(PyExc_ValueError, "%s has another shape than the result", name);
        return t;
    }
    void* stream() const { return c10::hip::getCurrentHIPStream(x.device().index()).stream(); }
    // `n` numbers of one dimension, or NULL for None where that is allowed
    template <typename T>
    const T* list(PyObject* o, const char* name, at::ScalarType dt, int64_t n, bool none) const {
        if (none && o == Py_None) return nullptr;
        const at::Tensor& t = here(o, name, dt);
        if (t.dim() != 1 || t.size(0) != n) raise(PyExc_ValueError, "%s must have %lld entries", name, (long long)n);
        return static_cast<const T*>(t.const_data_ptr());
    }
    // [sequences, kv heads, tokens]
    const at::Tensor& weights(PyObject* o, const char* name) const {
        const at::Tensor& t = here(o, name, at::kFloat);
        if (t.dim() != 3 || t.size(0) != kv.sequences || t.size(1) != kv.kv_heads)
            raise(PyExc_ValueError, "%s must be [%lld, %lld, tokens]", name, (long long)kv.sequences, (long long)kv.kv_heads);
        return t;
    }
    // the caller's scratch, or `bytes` of new one
    at::Tensor scratch(PyObject* given, size_t* bytes) const {
        if (given == Py_None) return at::empty({(int64_t)*bytes}, at::TensorOptions().dtype(at::kByte).device(x.device()));
        const at::Tensor& t = here(tensor(given, "workspace"), "workspace");
        *bytes = (size_t)t.numel() * t.element_size();
        return t;
    }
};

// What both appends take: the rows, their heads, the angles
struct Append {
    bitnet_dtype dt;
    const at::Tensor& qkv;
    int64_t T, heads, D, rotary = 0;
    Cache c;
    const float* freq = nullptr;
    static int64_t head_dim(const at::Tensor& qkv, PyObject* ok, int64_t heads) {
        const at::Tensor& k = tensor(ok, "k_cache");
        const int64_t kv_heads = k.dim() == 6 ? k.size(1) : 1;
        if (heads <= 0 || heads > qkv.size(1) || qkv.size(1) % (heads + 2 * kv_heads) != 0)
            raise(PyExc_ValueError, "qkv must have the columns of heads queries and two times kv heads keys and values");
        return qkv.size(1) / (heads + 2 * kv_heads);
    }
    Append(PyObject* oqkv, PyObject* ofreq, PyObject* ok, PyObject* ov, PyObject* otable, PyObject* olen, PyObject* oheads, PyObject* ostart)
        : qkv(matrix(oqkv, "qkv", &dt)), T(qkv.size(0)), heads(integer(oheads)), D(head_dim(qkv, ok, heads)), c(qkv, D, ok, ov, otable, olen, ostart) {
        if (ofreq == Py_None) return;
        const at::Tensor& f = c.here(ofreq, "inv_freq", at::kFloat);
        if (f.dim() != 1) raise(PyExc_ValueError, "inv_freq must be 1-D");
        freq = static_cast<const float*>(f.const_data_ptr());
        rotary = 2 * f.size(0);
    }
};

ENTRY(rope_kv_append) {      // qkv, inv_freq, k_cache, v_cache, page_table, kv_len, heads, q_start, pairs, q
    return entry(n, 10, [&] {
        Append p(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7]);
        const int pairs = truth(a[8]) ? 1 : 0;
        at::Tensor q = p.c.output(a[9], "q", {p.T, p.heads, p.D}, at::kBFloat16);
        const void* xp = p.qkv.const_data_ptr();
        void *qp = q.mutable_data_ptr(), *st = p.c.stream();
        call("bitnet_rope_kv_append", [&] { return abi.rope_kv_append(xp, p.dt, p.freq, p.rotary, pairs, &p.c.kv, p.T, p.heads, qp, st); });
        return THPVariable_Wrap(q);
    });
}

ENTRY(norm_rope_kv_append) {      // qkv, inv_freq, k_cache, v_cache, page_table, kv_len, heads, q_gain, k_gain, eps, q_start, pairs, norm, shift, q
    return entry(n, 15, [&] {
        Append p(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[10]);
        const float *qg = p.c.list<float>(a[7], "q_gain", at::kFloat, p.D, true), *kg = p.c.list<float>(a[8], "k_gain", at::kFloat, p.D, true);
        const float eps = real(a[9]);
        const int pairs = truth(a[11]) ? 1 : 0, norm = truth(a[12]) ? 1 : 0;
        const int32_t* shift = p.c.list<int32_t>(a[13], "shift", at::kInt, p.c.kv.sequences, true);
        at::Tensor q = p.c.output(a[14], "q", {p.T, p.heads, p.D}, at::kBFloat16);
        const void* xp = p.qkv.const_data_ptr();
        void *qp = q.mutable_data_ptr(), *st = p.c.stream();
        call("bitnet_norm_rope_kv_append",
             [&] { return abi.norm_rope_kv_append(xp, p.dt, norm, qg, kg, eps, p.freq, p.rotary, pairs, shift, &p.c.kv, p.T, p.heads, qp, st); });
        return THPVariable_Wrap(q);
    });
}

PyObject* attention(PyObject* const* a, bool prefill) {      // q, k_cache, v_cache, page_table, kv_len, q_start, scale, y_dtype, y, workspace
    const at::Tensor& q = tensor(a[0], "q", at::kBFloat16);
    if (q.dim() != 3) raise(PyExc_ValueError, "q must be 3-D");
    const int64_t T = q.size(0), heads = q.size(1), D = q.size(2);
    Cache c(q, D, a[1], a[2], a[3], a[4], a[5]);
    if (!prefill && T != c.kv.sequences) raise(PyExc_ValueError, "q must have one row per row of page_table");
    if (D <= 0) raise(PyExc_ValueError, "q has heads of no dims");
    const float scale = a[6] == Py_None ? (float)(1.0 / std::sqrt((double)D)) : real(a[6]);
    const at::ScalarType dt = out_type(a[7]);
    if (dt == at::kInt) raise(PyExc_ValueError, "y_dtype must be F32 or BF16");
    at::Tensor y = c.output(a[8], "y", {T, heads * D}, dt), ws;
    size_t bytes = 0;
    if (a[9] == Py_None) {
        call("bitnet_attention_workspace", [&] { return abi.attention_workspace(&c.kv, T, heads, prefill, &bytes); });
        if (bytes) ws = at::empty({(int64_t)bytes}, at::TensorOptions().dtype(at::kByte).device(q.device()));
    } else {
        ws = c.here(tensor(a[9], "workspace"), "workspace");
        bytes = (size_t)ws.numel() * ws.element_size();
    }
    void *wp = bytes ? ws.mutable_data_ptr() : nullptr, *yp = y.mutable_data_ptr(), *st = c.stream();
    const void* qp = q.const_data_ptr();
    const bitnet_dtype yt = dt == at::kFloat ? BITNET_F32 : BITNET_BF16;
    if (prefill) call("bitnet_attention_prefill", [&] { return abi.attention_prefill(qp, &c.kv, T, heads, scale, yp, yt, wp, bytes, st); });
    else call("bitnet_attention_decode", [&] { return abi.attention_decode(qp, &c.kv, heads, scale, yp, yt, wp, bytes, st); });
    return THPVariable_Wrap(y);
}
ENTRY(attention_decode) { return entry(n, 10, [&] { return attention(a, false); }); }
ENTRY(attention_prefill) { return entry(n, 10, [&] { return attention(a, true); }); }

// The rows of attention that is more than its output: q [T, heads, D], the cache, scale, the output
struct Rows {
    const at::Tensor& q;
    int64_t T, heads, D;
    Cache c;
    float scale;
    at::ScalarType dt;
    at::Tensor y;
    static const at::Tensor& checked(PyObject* o) {
        const at::Tensor& q = tensor(o, "q", at::kBFloat16);
        if (q.dim() != 3) raise(PyExc_ValueError, "q must be 3-D");
        return q;
    }
    Rows(PyObject* oq, PyObject* ok, PyObject* ov, PyObject* otable, PyObject* olen, PyObject* ostart, PyObject* oscale, PyObject* otype, PyObject* oy)
        : q(checked(oq)), T(q.size(0)), heads(q.size(1)), D(q.size(2)), c(q, D, ok, ov, otable, olen, ostart) {
        if (ostart == Py_None && T != c.kv.sequences) raise(PyExc_ValueError, "q must have one row per row of page_table");
        if (D <= 0) raise(PyExc_ValueError, "q has heads of no dims");
        scale = oscale == Py_None ? (float)(1.0 / std::sqrt((double)D)) : real(oscale);
        dt = out_type(otype);
        if (dt == at::kInt) raise(PyExc_ValueError, "y_dtype must be F32 or BF16");
        y = c.output(oy, "y", {T, heads * D}, dt);
    }
    bitnet_dtype type() const { return dt == at::kFloat ? BITNET_F32 : BITNET_BF16; }
};

ENTRY(attention_decode_shared) {      // q, k_cache, v_cache, page_table, kv_len, prefix_start, prefix_len, scale, y_dtype, y, workspace
    return entry(n, 11, [&] {
        Rows r(a[0], a[1], a[2], a[3], a[4], Py_None, a[7], a[8], a[9]);
        const at::Tensor& len = r.c.here(a[6], "prefix_len", at::kInt);
        if (len.dim() != 1) raise(PyExc_ValueError, "prefix_len must be 1-D");
        const int64_t groups = len.size(0);
        const int32_t* start = r.c.list<int32_t>(a[5], "prefix_start", at::kInt, groups + 1, false);
        size_t bytes = 0;
        if (a[10] == Py_None)
            call("bitnet_attention_shared_workspace", [&] { return abi.attention_shared_workspace(&r.c.kv, groups, r.heads, r.type(), &bytes); });
        at::Tensor ws = r.c.scratch(a[10], &bytes);
        const void* qp = r.q.const_data_ptr();
        const int32_t* lp = static_cast<const int32_t*>(len.const_data_ptr());
        void *wp = ws.mutable_data_ptr(), *yp = r.y.mutable_data_ptr(), *st = r.c.stream();
        call("bitnet_attention_decode_shared",
             [&] { return abi.attention_decode_shared(qp, &r.c.kv, start, lp, groups, r.heads, r.scale, yp, r.type(), wp, bytes, st); });
        return THPVariable_Wrap(r.y);
    });
}

PyObject* attention_weights(PyObject* const* a, bool prefill) {      // q, k_cache, v_cache, page_table, kv_len, q_start, weights, scale, y_dtype, y, workspace
    Rows r(a[0], a[1], a[2], a[3], a[4], a[5], a[7], a[8], a[9]);
    if (prefill && a[5] == Py_None) raise(PyExc_TypeError, "q_start must be a CUDA/HIP tensor");
    const at::Tensor& w = r.c.weights(a[6], "weights");
    size_t bytes = 0;
    if (a[10] == Py_None)
        call("bitnet_attention_weights_workspace", [&] { return abi.attention_weights_workspace(&r.c.kv, r.T, r.heads, prefill, r.type(), &bytes); });
    at::Tensor ws = r.c.scratch(a[10], &bytes);
    const void* qp = r.q.const_data_ptr();
    float* weights = static_cast<float*>(w.mutable_data_ptr());
    const int64_t stride = w.size(2);
    void *wp = ws.mutable_data_ptr(), *yp = r.y.mutable_data_ptr(), *st = r.c.stream();
    if (prefill)
        call("bitnet_attention_prefill_weights",
             [&] { return abi.attention_prefill_weights(qp, &r.c.kv, r.T, r.heads, r.scale, yp, r.type(), weights, stride, wp, bytes, st); });
    else
        call("bitnet_attention_decode_weights",
             [&] { return abi.attention_decode_weights(qp, &r.c.kv, r.heads, r.scale, yp, r.type(), weights, stride, wp, bytes, st); });
    return THPVariable_Wrap(r.y);
}
ENTRY(attention_decode_weights) { return entry(n, 11, [&] { return attention_weights(a, false); }); }
ENTRY(attention_prefill_weights) { return entry(n, 11, [&] { return attention_weights(a, true); }); }

ENTRY(kv_evict) {      // k_cache, v_cache, page_table, kv_len, weights, keep, recent, page_table_out, kv_len_out, weights_out, kept
    return entry(n, 11, [&] {
        const at::Tensor& k = tensor(a[0], "k_cache", at::kBFloat16);
        Cache c(k, k.dim() == 6 ? k.size(3) * 8 : 8, a[0], a[1], a[2], a[3], Py_None);
        const at::Tensor& w = c.weights(a[4], "weights");
        const int64_t keep = integer(a[5]), recent = integer(a[6]), B = c.kv.sequences;
        if (!THPVariable_Check(a[7]) || !THPVariable_Unpack(a[7]).is_cuda()) raise(PyExc_TypeError, "page_table_out must be a CUDA/HIP tensor");
        const at::Tensor& table = c.here(THPVariable_Unpack(a[7]), "page_table_out");
        if (table.scalar_type() != at::kInt) raise(PyExc_TypeError, "page_table_out has dtype %s", dtype_name(table.scalar_type()));
        two_d(table, "page_table_out");
        const int64_t pages = table.size(1);
        if (table.size(0) != B) raise(PyExc_ValueError, "page_table_out must have a row per row of page_table");
        if ((pages > 1 && table.stride(1) != 1) || (B > 1 && table.stride(0) < pages)) raise(PyExc_ValueError, "page_table_out must have contiguous rows");
        const int64_t most = std::min(keep, c.kv.max_pages * c.kv.page_tokens);
        if (keep <= 0 || pages * c.kv.page_tokens < most) raise(PyExc_ValueError, "page_table_out must have room for keep tokens, of which there is one at least");
        at::Tensor len = c.output(a[8], "kv_len_out", {B}, at::kInt);
        at::Tensor out = a[9] == Py_None ? at::empty({B, c.kv.kv_heads, pages * c.kv.page_tokens}, at::TensorOptions().dtype(at::kFloat).device(k.device()))
                                         : c.weights(a[9], "weights_out");
        at::Tensor kept = c.output(a[10], "kept", {B, c.kv.kv_heads, keep}, at::kInt);
        const float* wp = static_cast<const float*>(w.const_data_ptr());
        const int32_t* tp = static_cast<const int32_t*>(table.const_data_ptr());
        float* op = static_cast<float*>(out.mutable_data_ptr());
        int32_t *lp = static_cast<int32_t*>(len.mutable_data_ptr()), *kp = static_cast<int32_t*>(kept.mutable_data_ptr());
        void* st = c.stream();
        const int64_t stride = w.size(2), stride_out = out.size(2), table_stride = B > 1 ? table.stride(0) : pages;
        call("bitnet_kv_evict", [&] { return abi.kv_evict(&c.kv, wp, stride, keep, recent, tp, table_stride, op, stride_out, lp, kp, st); });
        PyObject* got = PyTuple_New(3);
        if (!got) throw Raised();
        PyTuple_SET_ITEM(got, 0, THPVariable_Wrap(len));
        PyTuple_SET_ITEM(got, 1, THPVariable_Wrap(out));
        PyTuple_SET_ITEM(got, 2, THPVariable_Wrap(kept));
        return got;
    });
}

// bind({name: address}, BitnetError)
PyObject* bind(PyObject*, PyObject* args) {
    PyObject *addresses, *cls;
    if (!PyArg_ParseTuple(args, "O!O", &PyDict_Type, &addresses, &cls)) return nullptr;
    Abi got;
#define TAKE(field_)                                                                                    \
    do {                                                                                                \
        PyObject* v = PyDict_GetItemString(addresses, "bitnet_" #field_);                               \
        void* p = v ? PyLong_AsVoidPtr(v) : nullptr;                                                    \
        if (!p) {                                                                                       \
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "no address for bitnet_" #field_); \
            return nullptr;                                                                             \
        }                                                                                               \
        got.field_ = reinterpret_cast<decltype(got.field_)>(p);                                         \
    } while (0)
    TAKE(quantize_acts); TAKE(rmsnorm_quantize); TAKE(swiglu_quantize); TAKE(linear); TAKE(linear_variant); TAKE(linear_segmented);
    TAKE(linear_ws); TAKE(linear_fused); TAKE(linear_fused_segmented); TAKE(rmsnorm_linear_fused);
    TAKE(rmsnorm_linear_fused_segmented); TAKE(swiglu_linear_fused); TAKE(ffn_gate_up_fused);
    TAKE(rope_kv_append); TAKE(attention_workspace); TAKE(attention_decode); TAKE(attention_prefill);
    TAKE(norm_rope_kv_append); TAKE(attention_shared_workspace); TAKE(attention_decode_shared); TAKE(attention_weights_workspace);
    TAKE(attention_decode_weights); TAKE(attention_prefill_weights); TAKE(kv_evict);
#undef TAKE
    abi = got;
    Py_INCREF(cls);
    Py_XDECREF(error_class);
    error_class = cls;
    Py_RETURN_NONE;
}

#define FAST(name_) {#name_, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name_)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    FAST(quantize_acts), FAST(rmsnorm_quantize), FAST(swiglu_quantize), FAST(linear), FAST(linear_segmented), FAST(linear_ws),
    FAST(linear_fused), FAST(rmsnorm_linear_fused), FAST(swiglu_linear_fused), FAST(ffn_gate_up_fused),
    FAST(rope_kv_append), FAST(attention_decode), FAST(attention_prefill),
    FAST(norm_rope_kv_append), FAST(attention_decode_shared), FAST(attention_decode_weights), FAST(attention_prefill_weights), FAST(kv_evict),
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__call() { return PyModule_Create(&module); }
