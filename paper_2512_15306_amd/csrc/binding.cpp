// Python module _binding: the calls of a training step without ctypes.  A call of llmq.py takes 11.4 us on the host in
// ctypes with three launches, of which the launches are 7.8: the checks of nine tensors and the conversion of thirteen arguments in
// Python are most of the rest.  Here they are reads of the tensors' fields.
//
// Every function takes the arguments of its namesake in llmq.py and returns the library's status, or None for whatever is not the
// plain case (a tensor subclass, another type, layout, device or size, a number out of range): the caller then takes the ctypes
// path, which does or refuses what it always has.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <limits>
#include <optional>
#include <utility>

#include "../../include/llmq.h"

namespace {

PyObject *g_get_device, *g_get_stream;          // torch._C functions

constexpr at::ScalarType kBf16 = at::kBFloat16, kF32 = at::kFloat, kU8 = at::kByte;

// The arguments of one call; ok turns false at the first one that is not the plain case.
struct Args {
    PyObject* const* a;
    bool ok;

    const at::Tensor* tensor(int i, at::ScalarType type) {
        if (!THPVariable_CheckExact(a[i])) { ok = false; return nullptr; }
        const at::Tensor& t = THPVariable_Unpack(a[i]);
        if (!t.is_cuda() || t.layout() != at::kStrided || t.scalar_type() != type || !t.is_contiguous()) { ok = false; return nullptr; }
        return &t;
    }
    // Device pointer of a tensor or NULL for None; numel: how many elements it has to have (-1: any)
    template <class T>
    T* ptr(int i, at::ScalarType type, int64_t numel = -1) {
        if (a[i] == Py_None) return nullptr;
        const at::Tensor* t = tensor(i, type);
        if (!t) return nullptr;
        if (numel >= 0 && t->numel() != numel) { ok = false; return nullptr; }
        return static_cast<T*>(t->data_ptr());
    }
    void* bf16(int i, int64_t numel = -1) { return ptr<void>(i, kBf16, numel); }
    float* f32(int i, int64_t numel = -1) { return ptr<float>(i, kF32, numel); }
    uint8_t* u8(int i, int64_t numel = -1) { return ptr<uint8_t>(i, kU8, numel); }
    uint8_t* some_u8(int i, int64_t numel) {                     // not None
        if (a[i] == Py_None) ok = false;
        return ok ? u8(i, numel) : nullptr;
    }
    void* some_bf16(int i, int64_t numel) {
        if (a[i] == Py_None) ok = false;
        return ok ? bf16(i, numel) : nullptr;
    }
    float* some_f32(int i, int64_t numel) {
        if (a[i] == Py_None) ok = false;
        return ok ? f32(i, numel) : nullptr;
    }
    // A workspace and its size
    void* workspace(int i, size_t& bytes) {
        const at::Tensor* t = tensor(i, kU8);
        if (!t) return nullptr;
        bytes = (size_t)t->numel();
        return t->data_ptr();
    }
    // [rows, cols] of a matrix
    bool dims(int i, at::ScalarType type, int64_t& rows, int64_t& cols) {
        const at::Tensor* t = tensor(i, type);
        if (!t || t->dim() != 2) { ok = false; return false; }
        rows = t->size(0);
        cols = t->size(1);
        return true;
    }
    int64_t i64(int i) {
        if (!PyLong_CheckExact(a[i])) { ok = false; return 0; }
        int over = 0;
        const long long v = PyLong_AsLongLongAndOverflow(a[i], &over);
        if (over) ok = false;
        return v;
    }
    int i32(int i) {
        const int64_t v = i64(i);
        if (v < std::numeric_limits<int>::min() || v > std::numeric_limits<int>::max()) ok = false;
        return (int)v;
    }
    int truth(int i) {
        if (!PyLong_Check(a[i])) { ok = false; return 0; }       // bool or int
        return PyObject_IsTrue(a[i]) == 1;
    }
};

// The current device's current stream
bool current_stream(void** stream) {
    PyObject* dev = PyObject_CallNoArgs(g_get_device);
    if (!dev) return false;
    PyObject* s = PyObject_CallOneArg(g_get_stream, dev);
    Py_DECREF(dev);
    if (!s) return false;
    *stream = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    return !PyErr_Occurred();
}

// N arguments read by `read` into a call, which `read` returns: a callable that takes the stream
template <class Read>
auto read_arguments(PyObject* const* args, Read read) -> std::optional<decltype(read(std::declval<Args&>()))> {
    Args a{args, true};
    try {
        auto call = read(a);
        if (a.ok) return call;
    } catch (...) {                                              // a tensor without storage, say
    }
    return std::nullopt;
}
template <class Read>
PyObject* run(PyObject* const* args, Py_ssize_t n, Py_ssize_t want, Read read) {
    if (n != want) Py_RETURN_NONE;
    const auto call = read_arguments(args, read);
    if (!call) Py_RETURN_NONE;
    void* stream = nullptr;
    if (!current_stream(&stream)) return nullptr;
    int status = 0;
    Py_BEGIN_ALLOW_THREADS                                       // (as ctypes does: a launch may wait for room in the queue)
    status = (*call)(stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

#define LLMQ_BINDING(name) PyObject* name(PyObject*, PyObject* const* args, Py_ssize_t n)

LLMQ_BINDING(linear_fwd) {
    return run(args, n, 11, [](Args& a) {
        size_t bytes = 0;
        void *X = a.bf16(0), *W = a.bf16(1);
        const int64_t M = a.i64(2), N = a.i64(3), K = a.i64(4);
        float *sx = a.f32(5), *sw = a.f32(6);
        void* Y = a.bf16(7);
        float* amax = a.f32(8);
        void* ws = a.workspace(9, bytes);
        const int flags = a.i32(10);
        return [=](void* s) { return llmq_fp8_linear_fwd(X, W, M, N, K, sx, sw, Y, amax, ws, bytes, flags, s); };
    });
}

LLMQ_BINDING(linear_dgrad) {
    return run(args, n, 12, [](Args& a) {
        size_t bytes = 0;
        void *dY = a.bf16(0), *W = a.bf16(1);
        const int64_t M = a.i64(2), N = a.i64(3), K = a.i64(4);
        float *sdy = a.f32(5), *sw = a.f32(6);
        const int fmt = a.i32(7);
        void* dX = a.bf16(8);
        float* amax = a.f32(9);
        void* ws = a.workspace(10, bytes);
        const int flags = a.i32(11);
        return [=](void* s) { return llmq_fp8_linear_dgrad(dY, W, M, N, K, sdy, sw, fmt, dX, amax, ws, bytes, flags, s); };
    });
}

LLMQ_BINDING(linear_wgrad) {
    return run(args, n, 12, [](Args& a) {
        size_t bytes = 0;
        void *dY = a.bf16(0), *X = a.bf16(1);
        const int64_t M = a.i64(2), N = a.i64(3), K = a.i64(4);
        float *sdy = a.f32(5), *sx = a.f32(6);
        const int fmt = a.i32(7);
        void* dW = a.bf16(8);
        const int accumulate = a.truth(9);
        void* ws = a.workspace(10, bytes);
        const int flags = a.i32(11);
        return [=](void* s) { return llmq_fp8_linear_wgrad(dY, X, M, N, K, sdy, sx, fmt, dW, accumulate, ws, bytes, flags, s); };
    });
}

LLMQ_BINDING(amax) {
    return run(args, n, 5, [](Args& a) {
        size_t bytes = 0;
        const at::Tensor* t = a.tensor(0, kBf16);
        const size_t count = t ? (size_t)t->numel() : 0;
        void* x = t ? t->data_ptr() : nullptr;
        const int fmt = a.i32(1);
        float *am = a.f32(2), *sc = a.f32(3);
        void* ws = a.workspace(4, bytes);
        return [=](void* s) { return llmq_amax(x, count, fmt, am, sc, ws, bytes, s); };
    });
}

template <bool SLABS>
PyObject* quantize(PyObject* const* args, Py_ssize_t n) {
    return run(args, n, 5, [](Args& a) {
        int64_t rows = 0, cols = 0;
        a.dims(0, kBf16, rows, cols);
        void* x = a.ok ? a.bf16(0) : nullptr;
        float* sc = a.f32(1);
        const int fmt = a.i32(2);
        uint8_t *q = a.some_u8(3, rows * cols), *qt = SLABS ? a.some_u8(4, rows * cols) : a.u8(4, rows * cols);
        return [=](void* s) { return SLABS ? llmq_quantize_fp8_slabs(x, rows, cols, sc, fmt, q, qt, s) : llmq_quantize_fp8(x, rows, cols, sc, fmt, q, qt, s); };
    });
}
LLMQ_BINDING(quantize_fp8) { return quantize<false>(args, n); }
LLMQ_BINDING(quantize_fp8_slabs) { return quantize<true>(args, n); }

LLMQ_BINDING(bf16_gemm_tn) {
    return run(args, n, 4, [](Args& a) {
        int64_t R = 0, T = 0, C = 0, T2 = 0, R2 = 0, C2 = 0;
        a.dims(0, kBf16, R, T);
        a.dims(1, kBf16, C, T2);
        a.dims(2, kBf16, R2, C2);
        if (T != T2 || R2 != R || C2 != C) a.ok = false;
        void *A = a.ok ? a.bf16(0) : nullptr, *B = a.ok ? a.bf16(1) : nullptr, *c = a.ok ? a.bf16(2) : nullptr;
        const int accumulate = a.truth(3);
        return [=](void* s) { return llmq_bf16_gemm_tn(A, B, R, C, T, c, accumulate, s); };
    });
}

// (M, I) of a gate + up tensor
void swiglu_dims(Args& a, int i, int64_t& M, int64_t& I) {
    if (a.dims(i, kBf16, M, I) && I % 2) a.ok = false;
    I /= 2;
}

LLMQ_BINDING(swiglu_fwd) {
    return run(args, n, 6, [](Args& a) {
        int64_t M = 0, I = 0;
        size_t bytes = 0;
        swiglu_dims(a, 0, M, I);
        void *gu = a.ok ? a.bf16(0) : nullptr, *h = a.some_bf16(1, M * I);
        const int fmt = a.i32(2);
        float *am = a.f32(3), *sc = a.f32(4);
        void* ws = a.workspace(5, bytes);
        return [=](void* s) { return llmq_swiglu_fwd(gu, M, I, h, fmt, am, sc, ws, bytes, s); };
    });
}

template <bool SLABS>
PyObject* swiglu_codes(PyObject* const* args, Py_ssize_t n) {
    return run(args, n, 6, [](Args& a) {
        int64_t M = 0, I = 0;
        swiglu_dims(a, 0, M, I);
        void* gu = a.ok ? a.bf16(0) : nullptr;
        float* sc = a.f32(1);
        const int fmt = a.i32(2);
        uint8_t *q = a.some_u8(3, M * I), *qt = SLABS ? a.some_u8(4, M * I) : a.u8(4, M * I);
        void* h = a.bf16(5, M * I);
        return [=](void* s) { return SLABS ? llmq_swiglu_fwd_fp8_slabs(gu, M, I, sc, fmt, q, qt, h, s) : llmq_swiglu_fwd_fp8(gu, M, I, sc, fmt, q, qt, h, s); };
    });
}
LLMQ_BINDING(swiglu_fwd_fp8) { return swiglu_codes<false>(args, n); }
LLMQ_BINDING(swiglu_fwd_fp8_slabs) { return swiglu_codes<true>(args, n); }

LLMQ_BINDING(swiglu_bwd) {
    return run(args, n, 7, [](Args& a) {
        int64_t M = 0, I = 0;
        size_t bytes = 0;
        swiglu_dims(a, 1, M, I);
        void *dh = a.some_bf16(0, M * I), *gu = a.ok ? a.bf16(1) : nullptr, *dgu = a.some_bf16(2, 2 * M * I);
        const int fmt = a.i32(3);
        float *am = a.f32(4), *sc = a.f32(5);
        void* ws = a.workspace(6, bytes);
        return [=](void* s) { return llmq_swiglu_bwd(dh, gu, M, I, dgu, fmt, am, sc, ws, bytes, s); };
    });
}

LLMQ_BINDING(rmsnorm_fwd) {
    return run(args, n, 11, [](Args& a) {
        int64_t M = 0, C = 0;
        size_t bytes = 0;
        a.dims(0, kBf16, M, C);
        void *res = a.ok ? a.bf16(0) : nullptr, *x = a.bf16(1, M * C), *w = a.some_bf16(2, C);
        if (!PyFloat_CheckExact(a.a[3])) a.ok = false;
        const float eps = a.ok ? (float)PyFloat_AS_DOUBLE(a.a[3]) : 0.0f;
        void *res_out = a.bf16(4, M * C), *y = a.some_bf16(5, M * C);
        float* rstd = a.some_f32(6, M);
        const int fmt = a.i32(7);
        float *am = a.f32(8), *sc = a.f32(9);
        void* ws = a.workspace(10, bytes);
        return [=](void* s) { return llmq_rmsnorm_fwd(res, x, w, M, C, eps, res_out, y, rstd, fmt, am, sc, ws, bytes, s); };
    });
}

template <bool SLABS>
PyObject* rmsnorm_codes(PyObject* const* args, Py_ssize_t n) {
    return run(args, n, 8, [](Args& a) {
        int64_t M = 0, C = 0;
        a.dims(0, kBf16, M, C);
        void *res = a.ok ? a.bf16(0) : nullptr, *w = a.some_bf16(1, C);
        float *rstd = a.some_f32(2, M), *sc = a.f32(3);
        const int fmt = a.i32(4);
        uint8_t *q = a.some_u8(5, M * C), *qt = SLABS ? a.some_u8(6, M * C) : a.u8(6, M * C);
        void* y = a.bf16(7, M * C);
        return [=](void* s) {
            return SLABS ? llmq_rmsnorm_apply_fp8_slabs(res, w, rstd, M, C, sc, fmt, q, qt, y, s) : llmq_rmsnorm_apply_fp8(res, w, rstd, M, C, sc, fmt, q, qt, y, s);
        };
    });
}
LLMQ_BINDING(rmsnorm_apply_fp8) { return rmsnorm_codes<false>(args, n); }
LLMQ_BINDING(rmsnorm_apply_fp8_slabs) { return rmsnorm_codes<true>(args, n); }

// Tensors of the current device only, whose stream the call takes
struct HereArgs : Args {
    int device;
    explicit HereArgs(const Args& args) : Args(args), device(-1) {
        PyObject* d = PyObject_CallNoArgs(g_get_device);
        if (d) { device = (int)PyLong_AsLong(d); Py_DECREF(d); }
        if (PyErr_Occurred()) { PyErr_Clear(); ok = false; }
    }
    const at::Tensor* here(int i, at::ScalarType type) {
        const at::Tensor* t = tensor(i, type);
        if (t && t->device().index() != device) { ok = false; return nullptr; }
        return t;
    }
    // (numel -1: any; required: not None)
    void* pointer(int i, at::ScalarType type, int64_t numel, bool required) {
        if (a[i] == Py_None) { if (required) ok = false; return nullptr; }
        const at::Tensor* t = here(i, type);
        if (t && numel >= 0 && t->numel() != numel) { ok = false; return nullptr; }
        return t ? t->data_ptr() : nullptr;
    }
    // A BF16 matrix [M, width] whose rows may lie apart
    void* rows(int i, int64_t M, int64_t width, bool required, int64_t& stride) {
        stride = 0;
        if (a[i] == Py_None) { if (required) ok = false; return nullptr; }
        if (!THPVariable_CheckExact(a[i])) { ok = false; return nullptr; }
        const at::Tensor& t = THPVariable_Unpack(a[i]);
        if (!t.is_cuda() || t.device().index() != device || t.layout() != at::kStrided || t.scalar_type() != kBf16 || t.dim() != 2 || t.size(0) != M || t.size(1) != width ||
            (width > 1 && t.stride(1) != 1) || (M > 1 && t.stride(0) < width)) { ok = false; return nullptr; }
        stride = M > 1 ? t.stride(0) : width;
        return t.data_ptr();
    }
    int64_t rows_of(int i) {
        if (!THPVariable_CheckExact(a[i]) || THPVariable_Unpack(a[i]).dim() != 2) { ok = false; return 0; }
        return THPVariable_Unpack(a[i]).size(0);
    }
    int64_t numel_of(int i) {
        if (a[i] == Py_None) return 0;
        if (!THPVariable_CheckExact(a[i])) { ok = false; return 0; }
        return THPVariable_Unpack(a[i]).numel();
    }
    uint8_t* codes(int i, int64_t numel, bool required) { return static_cast<uint8_t*>(pointer(i, kU8, numel, required)); }
};

LLMQ_BINDING(quantize_fp8_blocks) {
    return run(args, n, 7, [](Args& args_) {
        HereArgs a(args_);
        int64_t rows = 0, cols = 0;
        a.dims(0, kBf16, rows, cols);
        void* x = a.pointer(0, kBf16, -1, true);
        const int fmt = a.i32(1), block_rows = a.i32(2);
        uint8_t *q = a.codes(3, rows * cols, false), *s = a.codes(4, (int64_t)llmq_block_scales_bytes(rows, cols), false);
        uint8_t *qt = a.codes(5, rows * cols, false), *st = a.codes(6, (int64_t)llmq_block_scales_bytes(cols, rows), false);
        args_.ok = a.ok;
        return [=](void* stream) { return llmq_quantize_fp8_blocks(x, rows, cols, fmt, block_rows, q, s, qt, st, stream); };
    });
}

LLMQ_BINDING(fp8_gemm_blocks) {
    return run(args, n, 9, [](Args& args_) {
        HereArgs a(args_);
        int64_t R = 0, T = 0, C = 0, T2 = 0, R2 = 0, C2 = 0;
        a.dims(0, kU8, R, T);
        a.dims(3, kU8, C, T2);
        a.dims(6, kBf16, R2, C2);
        if (T != T2 || R2 != R || C2 != C) a.ok = false;
        uint8_t *A = a.codes(0, -1, true), *sA = a.codes(1, (int64_t)llmq_block_scales_bytes(R, T), true);
        const int fmt_a = a.i32(2), fmt_b = a.i32(5);
        uint8_t *B = a.codes(3, -1, true), *sB = a.codes(4, (int64_t)llmq_block_scales_bytes(C, T), true);
        void* c = a.pointer(6, kBf16, -1, true);
        const int accumulate = a.truth(7);
        float* amax = static_cast<float*>(a.pointer(8, kF32, 1, false));
        args_.ok = a.ok;
        return [=](void* stream) { return llmq_fp8_gemm_blocks(A, sA, fmt_a, B, sB, fmt_b, R, C, T, c, accumulate, amax, stream); };
    });
}

LLMQ_BINDING(fp8_gemm_blocks_swiglu_fwd) {
    return run(args, n, 9, [](Args& args_) {
        HereArgs a(args_);
        int64_t M = 0, T = 0, both = 0, T2 = 0, M2 = 0, I = 0;
        a.dims(0, kU8, M, T);
        a.dims(3, kU8, both, T2);
        a.dims(6, kBf16, M2, I);
        if (T != T2 || M2 != M || both != 2 * I) a.ok = false;
        uint8_t *A = a.codes(0, -1, true), *sA = a.codes(1, (int64_t)llmq_block_scales_bytes(M, T), true);
        const int fmt_a = a.i32(2), fmt_b = a.i32(5);
        uint8_t *W = a.codes(3, -1, true), *sW = a.codes(4, (int64_t)llmq_block_scales_bytes(both, T), true);
        void* h = a.pointer(6, kBf16, -1, true);
        int64_t M3 = M, both3 = both;
        if (a.ok && a.a[7] != Py_None) a.dims(7, kBf16, M3, both3);
        if (M3 != M || both3 != both) a.ok = false;
        void* gu = a.pointer(7, kBf16, -1, false);
        float* amax = static_cast<float*>(a.pointer(8, kF32, 1, false));
        args_.ok = a.ok;
        return [=](void* stream) { return llmq_fp8_gemm_blocks_swiglu_fwd(A, sA, fmt_a, W, sW, fmt_b, M, I, T, h, gu, amax, stream); };
    });
}

LLMQ_BINDING(fp8_gemm_blocks_swiglu_bwd) {
    return run(args, n, 10, [](Args& args_) {
        HereArgs a(args_);
        int64_t M = 0, T = 0, I = 0, T2 = 0, M2 = 0, both = 0, M3 = 0, both3 = 0;
        a.dims(0, kU8, M, T);
        a.dims(3, kU8, I, T2);
        a.dims(6, kBf16, M2, both);
        a.dims(7, kBf16, M3, both3);
        if (T != T2 || M2 != M || M3 != M || both != 2 * I || both3 != 2 * I) a.ok = false;
        uint8_t *A = a.codes(0, -1, true), *sA = a.codes(1, (int64_t)llmq_block_scales_bytes(M, T), true);
        const int fmt_a = a.i32(2), fmt_b = a.i32(5);
        uint8_t *B = a.codes(3, -1, true), *sB = a.codes(4, (int64_t)llmq_block_scales_bytes(I, T), true);
        void *gu = a.pointer(6, kBf16, -1, true), *dgu = a.pointer(7, kBf16, -1, true);
        int64_t M4 = M, I4 = I;
        if (a.ok && a.a[8] != Py_None) a.dims(8, kBf16, M4, I4);
        if (M4 != M || I4 != I) a.ok = false;
        void* h = a.pointer(8, kBf16, -1, false);
        float* amax = static_cast<float*>(a.pointer(9, kF32, 1, false));
        args_.ok = a.ok;
        return [=](void* stream) { return llmq_fp8_gemm_blocks_swiglu_bwd(A, sA, fmt_a, B, sB, fmt_b, gu, M, I, T, dgu, h, amax, stream); };
    });
}

LLMQ_BINDING(rmsnorm_fwd_fp8_blocks) {
    return run(args, n, 12, [](Args& args_) {
        HereArgs a(args_);
        int64_t M = 0, C = 0;
        a.dims(0, kBf16, M, C);
        void *res = a.pointer(0, kBf16, -1, true), *x = a.pointer(1, kBf16, M * C, false), *w = a.pointer(2, kBf16, C, true), *res_out = a.pointer(4, kBf16, M * C, false);
        if (!PyFloat_CheckExact(a.a[3])) a.ok = false;
        const float eps = a.ok ? (float)PyFloat_AS_DOUBLE(a.a[3]) : 0.0f;
        float* rstd = static_cast<float*>(a.pointer(5, kF32, M, true));
        const int fmt = a.i32(6);
        uint8_t *q = a.codes(7, M * C, false), *s = a.codes(8, (int64_t)llmq_block_scales_bytes(M, C), false);
        uint8_t *qt = a.codes(9, M * C, false), *st = a.codes(10, (int64_t)llmq_block_scales_bytes(C, M), false);
        void* y = a.pointer(11, kBf16, M * C, false);
        args_.ok = a.ok;
        return [=](void* stream) { return llmq_rmsnorm_fwd_fp8_blocks(res, x, w, M, C, eps, res_out, rstd, fmt, q, s, qt, st, y, stream); };
    });
}

LLMQ_BINDING(rmsnorm_bwd) {
    return run(args, n, 12, [](Args& args_) {
        HereArgs a(args_);
        int64_t M = 0, C = 0;
        a.dims(2, kBf16, M, C);
        void *dy = a.pointer(0, kBf16, M * C, true), *dres = a.pointer(1, kBf16, M * C, false), *res = a.pointer(2, kBf16, -1, true), *w = a.pointer(3, kBf16, C, true);
        float* rstd = static_cast<float*>(a.pointer(4, kF32, M, true));
        void* dx = a.pointer(5, kBf16, M * C, true);
        float* dw = static_cast<float*>(a.pointer(6, kF32, C, false));
        const int accumulate = a.truth(7), fmt = a.i32(8);
        float *am = static_cast<float*>(a.pointer(9, kF32, 1, false)), *sc = static_cast<float*>(a.pointer(10, kF32, 1, false));
        void* ws = a.pointer(11, kU8, -1, false);
        const size_t bytes = (size_t)a.numel_of(11);
        args_.ok = a.ok;
        return [=](void* s) { return llmq_rmsnorm_bwd(dy, dres, res, w, rstd, M, C, dx, dw, accumulate, fmt, am, sc, ws, bytes, s); };
    });
}

LLMQ_BINDING(qk_norm_rope_fwd) {
    return run(args, n, 13, [](Args& args_) {
        HereArgs a(args_);
        const int64_t M = a.rows_of(0);
        const int Hq = a.i32(1), Hkv = a.i32(2), D = a.i32(3), rot = (int)(2 * a.numel_of(8));
        int64_t xs = 0, qs = 0, ks = 0;
        void* x = a.rows(0, M, (int64_t)(Hq + 2 * (int64_t)Hkv) * D, true, xs);
        void *wq = a.pointer(4, kBf16, D, false), *wk = a.pointer(5, kBf16, D, false);
        if (!wq != !wk || !PyFloat_CheckExact(a.a[6])) a.ok = false;
        const float eps = a.ok ? (float)PyFloat_AS_DOUBLE(a.a[6]) : 0.0f;
        int64_t* positions = static_cast<int64_t*>(a.pointer(7, at::kLong, rot ? M : -1, false));
        double* freq = static_cast<double*>(a.pointer(8, at::kDouble, -1, false));
        const int interleaved = a.truth(9);
        void *q = a.rows(10, M, (int64_t)Hq * D, true, qs), *k = a.rows(11, M, (int64_t)Hkv * D, true, ks);
        float* rstd = static_cast<float*>(a.pointer(12, kF32, M * ((int64_t)Hq + Hkv), false));
        args_.ok = a.ok;
        return [=](void* s) { return llmq_qk_norm_rope_fwd(x, xs, M, Hq, Hkv, D, wq, wk, eps, positions, freq, rot, interleaved, q, qs, k, ks, rstd, s); };
    });
}

LLMQ_BINDING(qk_norm_rope_bwd) {
    return run(args, n, 21, [](Args& args_) {
        HereArgs a(args_);
        const int64_t M = a.rows_of(13);
        const int Hq = a.i32(4), Hkv = a.i32(5), D = a.i32(6), rot = (int)(2 * a.numel_of(11));
        const int64_t width = (int64_t)(Hq + 2 * (int64_t)Hkv) * D;
        int64_t qs = 0, ks = 0, vs = 0, xs = 0, dxs = 0;
        void *dq = a.rows(0, M, (int64_t)Hq * D, true, qs), *dk = a.rows(1, M, (int64_t)Hkv * D, true, ks), *dv = a.rows(2, M, (int64_t)Hkv * D, false, vs);
        void *x = a.rows(3, M, width, false, xs), *dx = a.rows(13, M, width, true, dxs);
        void *wq = a.pointer(7, kBf16, D, false), *wk = a.pointer(8, kBf16, D, false);
        if (!wq != !wk) a.ok = false;
        float* rstd = static_cast<float*>(a.pointer(9, kF32, M * ((int64_t)Hq + Hkv), false));
        int64_t* positions = static_cast<int64_t*>(a.pointer(10, at::kLong, rot ? M : -1, false));
        double* freq = static_cast<double*>(a.pointer(11, at::kDouble, -1, false));
        const int interleaved = a.truth(12);
        float *dwq = static_cast<float*>(a.pointer(14, kF32, D, false)), *dwk = static_cast<float*>(a.pointer(15, kF32, D, false));
        const int accumulate = a.truth(16), fmt = a.i32(17);
        float *amax = static_cast<float*>(a.pointer(18, kF32, 1, false)), *scale = static_cast<float*>(a.pointer(19, kF32, 1, false));
        void* ws = a.pointer(20, kU8, -1, false);
        const size_t bytes = ws ? (size_t)a.numel_of(20) : 0;
        args_.ok = a.ok;
        return [=](void* s) {
            return llmq_qk_norm_rope_bwd(dq, qs, dk, ks, dv, vs, x, xs, M, Hq, Hkv, D, wq, wk, rstd, positions, freq, rot, interleaved, dx, dxs, dwq, dwk, accumulate, fmt, amax, scale, ws,
                                         bytes, s);
        };
    });
}

LLMQ_BINDING(adamw_step) {
    return run(args, n, 4, [](Args& args_) {
        HereArgs a(args_);
        // (the plan's words and the numbers of the step, unless those are on the device, are read during the call)
        auto words = [&](int i, at::ScalarType type, int64_t numel) -> const at::Tensor* {
            if (!THPVariable_CheckExact(a.a[i])) { a.ok = false; return nullptr; }
            const at::Tensor& t = THPVariable_Unpack(a.a[i]);
            if (t.layout() != at::kStrided || t.scalar_type() != type || t.numel() != numel || !t.is_contiguous() || !(t.is_cpu() || t.is_cuda())) { a.ok = false; return nullptr; }
            return &t;
        };
        void* table = a.pointer(0, kU8, -1, true);
        const at::Tensor *info = words(1, at::kLong, 4), *hyper = words(2, at::kInt, LLMQ_ADAMW_HYPER_WORDS);
        if (info && !info->is_cpu()) a.ok = false;
        if (hyper && hyper->is_cuda() && hyper->device().index() != a.device) a.ok = false;
        const bool on_device = hyper && hyper->is_cuda();
        const int64_t* i = a.ok ? static_cast<const int64_t*>(info->data_ptr()) : nullptr;
        const void* h = a.ok ? hyper->data_ptr() : nullptr;
        float* scale = static_cast<float*>(a.pointer(3, kF32, 1, false));
        args_.ok = a.ok;
        return [=](void* s) { return llmq_adamw_step(table, i, on_device ? nullptr : static_cast<const uint32_t*>(h), on_device ? h : nullptr, scale, s); };
    });
}

#define LLMQ_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {LLMQ_METHOD(linear_fwd), LLMQ_METHOD(linear_dgrad), LLMQ_METHOD(linear_wgrad), LLMQ_METHOD(amax), LLMQ_METHOD(quantize_fp8),
                           LLMQ_METHOD(quantize_fp8_slabs), LLMQ_METHOD(bf16_gemm_tn), LLMQ_METHOD(swiglu_fwd), LLMQ_METHOD(swiglu_fwd_fp8),
                           LLMQ_METHOD(swiglu_fwd_fp8_slabs), LLMQ_METHOD(swiglu_bwd), LLMQ_METHOD(rmsnorm_fwd), LLMQ_METHOD(rmsnorm_apply_fp8),
                           LLMQ_METHOD(rmsnorm_apply_fp8_slabs), LLMQ_METHOD(quantize_fp8_blocks), LLMQ_METHOD(fp8_gemm_blocks), LLMQ_METHOD(fp8_gemm_blocks_swiglu_fwd), LLMQ_METHOD(fp8_gemm_blocks_swiglu_bwd), LLMQ_METHOD(rmsnorm_fwd_fp8_blocks), LLMQ_METHOD(rmsnorm_bwd), LLMQ_METHOD(qk_norm_rope_fwd), LLMQ_METHOD(qk_norm_rope_bwd), LLMQ_METHOD(adamw_step), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) {
    PyObject* c = PyImport_ImportModule("torch._C");
    if (!c) return nullptr;
    g_get_device = PyObject_GetAttrString(c, "_cuda_getDevice");
    g_get_stream = g_get_device ? PyObject_GetAttrString(c, "_cuda_getCurrentRawStream") : nullptr;
    Py_DECREF(c);
    if (!g_get_stream) {                                          // a PyTorch without GPUs
        PyErr_SetString(PyExc_ImportError, "torch._C has no device functions");
        return nullptr;
    }
    return PyModule_Create(&g_module);
}
