// Direct calls from Python into the C ABI, for the case every loop of a program is in: tensors that fit, and an output
// that exists.  Each function takes the arguments of the wrapper of the same name in binding.py, checks what that
// wrapper checks, reads pointers and strides off the tensors and calls the library on torch's current stream.
//
//   returns 0    launched
//   returns > 0  the library's status (nothing launched)
//   (the backward passes, which allocate what they return: a tuple of the status and the tensors)
//   returns -1   not a case for this path (another type, a tensor subclass or wrapper, a shape or stride that the
//                wrapper refuses): nothing was done, and the wrapper's own checks say what is wrong or go the long way
//
// Why it exists: with attribute reads, checks and a foreign call through ctypes a launch from Python took 6 - 8 us, twice
// what the GPU needs for a small layer (64 x 1024 x 1024 fused: 3.0 us).  Here it takes about 0.6 us.
//
// The library is loaded by binding.py, which hands over the entry points' addresses (bind); nothing is kept of a tensor
// after a call.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

namespace {

using Words = const uint32_t*;

struct EntryPoints {
    int (*pack_sign)(const float*, int64_t, int64_t, int64_t, uint32_t*, int64_t, void*);
    int (*xnor_gemm)(Words, int64_t, Words, int64_t, int32_t*, int64_t, int64_t, int64_t, int64_t, void*);
    int (*xnor_gemm_kernel)(Words, int64_t, Words, int64_t, int32_t*, int64_t, int64_t, int64_t, int64_t, int, void*);
    int (*bn_sign_pack)(const int32_t*, int64_t, int64_t, int64_t, const int32_t*, Words, uint32_t*, int64_t, void*);
    int (*xnor_gemm_bn_sign_pack)(Words, int64_t, Words, int64_t, int64_t, int64_t, int64_t, const int32_t*, Words, uint32_t*,
                                  int64_t, void*);
    int (*xnor_gemm_bn_sign_pack_kernel)(Words, int64_t, Words, int64_t, int64_t, int64_t, int64_t, const int32_t*, Words,
                                         uint32_t*, int64_t, int, void*);
    int (*sign_gemm_bn_sign_pack)(const float*, int64_t, Words, int64_t, int64_t, int64_t, int64_t, const int32_t*, Words, uint32_t*,
                                  int64_t, uint32_t*, int64_t, void*);
    int (*pack_bitplanes)(const uint8_t*, int64_t, int64_t, int64_t, uint32_t*, int64_t, void*);
    int (*bitplane_gemm)(Words, int64_t, Words, int64_t, int32_t*, int64_t, int64_t, int64_t, int64_t, void*);
    int (*bitplane_gemm_bn_sign_pack)(Words, int64_t, Words, int64_t, int64_t, int64_t, int64_t, const int32_t*, Words,
                                      uint32_t*, int64_t, void*);
    int (*conv_xnor)(Words, int64_t, int64_t, int64_t, int64_t, Words, int64_t, int64_t, int, int, int, int, int32_t*, int64_t,
                     void*);
    int (*conv_bn_sign_pack)(Words, int64_t, int64_t, int64_t, int64_t, Words, int64_t, int64_t, int, int, int, int,
                             const int32_t*, Words, uint32_t*, int64_t, void*);
    int (*conv_pool_bn_sign_pack)(Words, int64_t, int64_t, int64_t, int64_t, Words, int64_t, int64_t, int, int, int, int, int,
                                  const int32_t*, Words, uint32_t*, int64_t, void*);
    int (*conv_pool_windows_bn_sign_pack)(Words, int64_t, int64_t, int64_t, int64_t, Words, int64_t, int64_t, int, int, int, int, int,
                                          const int32_t*, Words, uint32_t*, int64_t, void*);
    int (*conv_im2col_pack)(Words, int64_t, int64_t, int64_t, int64_t, int, int, int, int, uint32_t*, int64_t, void*);
    int (*maxpool_bits)(Words, int64_t, int64_t, int64_t, int64_t, int, int, int, Words, uint32_t*, void*);
    int (*linear_bits)(int, const void*, int64_t, Words, int64_t, const float*, const float*, int, const void*, int64_t, void*,
                       int64_t, int64_t, int64_t, int64_t, void*);
    int (*gated_bits)(int, const void*, int64_t, Words, int64_t, const float*, const float*, int, void*, int64_t, int64_t, int64_t,
                      int64_t, void*);
    int (*norm_residual)(int, const void*, int64_t, const void*, int64_t, const void*, int64_t, int64_t, float, int, const float*,
                         const float*, int, const float*, const float*, float, void*, int64_t, void*, int64_t, int64_t, int64_t,
                         void*);
    int64_t (*linear_bits_backward_workspace)(int, int64_t, int64_t, int64_t, int);
    int64_t (*gated_bits_backward_workspace)(int, int64_t, int64_t, int64_t, int);
    int (*linear_bits_backward)(int, const void*, int64_t, const void*, int64_t, Words, int64_t, const float*, const float*, int, void*,
                                int64_t, void*, int64_t, float*, float*, int64_t, int64_t, int64_t, void*, int64_t, void*);
    int (*gated_bits_backward)(int, const void*, int64_t, const void*, int64_t, Words, int64_t, const float*, const float*, int, void*,
                               int64_t, void*, int64_t, float*, float*, int64_t, int64_t, int64_t, void*, int64_t, void*);
    int64_t (*norm_residual_backward_workspace)(int64_t, int64_t, int64_t);
    int (*norm_residual_backward)(int, const void*, int64_t, const void*, int64_t, const void*, int64_t, const void*, int64_t,
                                  const void*, int64_t, int64_t, float, int, const float*, const float*, int, const float*, float,
                                  void*, int64_t, void*, int64_t, void*, int64_t, float*, float*, float*, float*, int64_t, int64_t,
                                  void*, int64_t, void*);
};

EntryPoints entry{};
PyObject* raw_stream = nullptr;      // torch._C._cuda_getCurrentRawStream

int64_t words(int64_t n) { return (n + 31) / 32; }

// A plain torch.Tensor on the GPU with memory of its own, of the given type; null otherwise.
const at::Tensor* plain(PyObject* o, at::ScalarType type) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.scalar_type() != type || t.layout() != at::kStrided ||
        !t.unsafeGetTensorImpl()->has_storage())
        return nullptr;
    return &t;
}

// The wrappers' 2-D operand: unit stride along its rows.
struct Matrix {
    void* data = nullptr;
    int64_t rows = 0, cols = 0, ld = 0;
    const at::Tensor* t = nullptr;
    bool read(PyObject* o, at::ScalarType type) {
        t = plain(o, type);
        if (!t || t->dim() != 2) return false;
        rows = t->size(0);
        cols = t->size(1);
        if (cols > 1 && t->stride(1) != 1) return false;
        ld = rows > 1 ? t->stride(0) : std::max(t->stride(0), cols);
        data = t->data_ptr();
        return true;
    }
    template <typename T>
    T* as() const { return static_cast<T*>(data); }
    // The [r][c] elements a call reads or writes are there.  A leading dimension that is too short is left to the library,
    // which refuses it; too few rows, or a narrow slice of a wide buffer, it cannot see.
    bool holds(int64_t r, int64_t c) const { return r <= 0 || c <= 0 || ld < c || (rows >= r && cols >= c); }
};

// A packed map [B][H][W][words], contiguous.
struct Map {
    Words data = nullptr;
    int64_t B = 0, H = 0, W = 0, Cw = 0;
    bool read(PyObject* o, int64_t channels) {
        const at::Tensor* t = plain(o, at::kInt);
        if (!t || t->dim() != 4 || !t->is_contiguous()) return false;
        B = t->size(0);
        H = t->size(1);
        W = t->size(2);
        Cw = t->size(3);
        data = static_cast<Words>(t->data_ptr());
        return Cw == words(channels);
    }
};

// Contiguous int32 vector of n elements.
void* vector_of(PyObject* o, int64_t n) {
    const at::Tensor* t = plain(o, at::kInt);
    return t && t->numel() == n && t->is_contiguous() ? t->data_ptr() : nullptr;
}

bool integer(PyObject* o, int64_t& v) {
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    v = PyLong_AsLongLongAndOverflow(o, &overflow);
    return overflow == 0;
}

bool small_integer(PyObject* o, int& v) {
    int64_t w;
    if (!integer(o, w) || w < -1000000000 || w > 1000000000) return false;
    v = int(w);
    return true;
}

bool stream_of(const at::Tensor& t, void*& stream) {
    PyObject* index = PyLong_FromLong(t.get_device());
    if (!index) return false;
    PyObject* r = PyObject_CallOneArg(raw_stream, index);
    Py_DECREF(index);
    if (!r) return false;
    stream = PyLong_AsVoidPtr(r);
    Py_DECREF(r);
    return !PyErr_Occurred();
}

PyObject* long_way() { return PyLong_FromLong(-1); }

// Calls the library without the interpreter lock (a launch may wait for room in the stream's queue).
template <typename F>
PyObject* launch(const at::Tensor& out, F&& call) {
    void* stream;
    if (!stream_of(out, stream)) return nullptr;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = call(stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

// Every function below: no C++ exception may reach the interpreter; whatever a tensor throws is left to the wrapper.
template <PyObject* (*F)(PyObject* const*)>
PyObject* guarded(PyObject* const* a) noexcept {
    try {
        return F(a);
    } catch (...) {
        PyErr_Clear();
        return long_way();
    }
}

template <PyObject* (*F)(PyObject* const*), Py_ssize_t ARGS>
PyObject* entry_of(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != ARGS) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    return guarded<F>(a);
}

// (x, out)
PyObject* pack_sign(PyObject* const* a) {
    Matrix x, out;
    if (!x.read(a[0], at::kFloat) || !out.read(a[1], at::kInt) || !out.holds(x.rows, words(x.cols))) return long_way();
    return launch(*out.t, [&](void* s) { return entry.pack_sign(x.as<float>(), x.rows, x.cols, x.ld, out.as<uint32_t>(), out.ld, s); });
}

// (A, B, K, out, kernel)
PyObject* xnor_gemm(PyObject* const* a) {
    Matrix A, B, out;
    int64_t K;
    int kernel;
    if (!A.read(a[0], at::kInt) || !B.read(a[1], at::kInt) || !integer(a[2], K) || !out.read(a[3], at::kInt) ||
        !small_integer(a[4], kernel) || K < 0 || A.cols < words(K) || B.cols < words(K) || !out.holds(A.rows, B.rows))
        return long_way();
    return launch(*out.t, [&](void* s) {
        return kernel == 0 ? entry.xnor_gemm(A.as<uint32_t>(), A.ld, B.as<uint32_t>(), B.ld, out.as<int32_t>(), out.ld, A.rows,
                                             B.rows, K, s)
                           : entry.xnor_gemm_kernel(A.as<uint32_t>(), A.ld, B.as<uint32_t>(), B.ld, out.as<int32_t>(), out.ld,
                                                    A.rows, B.rows, K, kernel, s);
    });
}

// (C, thr, flip, out)
PyObject* bn_sign_pack(PyObject* const* a) {
    Matrix C, out;
    if (!C.read(a[0], at::kInt)) return long_way();
    const void* thr = vector_of(a[1], C.cols);
    const void* flip = vector_of(a[2], words(C.cols));
    if (!thr || !flip || !out.read(a[3], at::kInt) || !out.holds(C.rows, words(C.cols))) return long_way();
    return launch(*out.t, [&](void* s) {
        return entry.bn_sign_pack(C.as<int32_t>(), C.ld, C.rows, C.cols, static_cast<const int32_t*>(thr),
                                  static_cast<Words>(flip), out.as<uint32_t>(), out.ld, s);
    });
}

// (A, B, K, thr, flip, out, kernel)
PyObject* xnor_gemm_bn_sign_pack(PyObject* const* a) {
    Matrix A, B, out;
    int64_t K;
    int kernel;
    if (!A.read(a[0], at::kInt) || !B.read(a[1], at::kInt) || !integer(a[2], K) || K < 0 || A.cols < words(K) ||
        B.cols < words(K))
        return long_way();
    const void* thr = vector_of(a[3], B.rows);
    const void* flip = vector_of(a[4], words(B.rows));
    if (!thr || !flip || !out.read(a[5], at::kInt) || !small_integer(a[6], kernel) || !out.holds(A.rows, words(B.rows)))
        return long_way();
    return launch(*out.t, [&](void* s) {
        return kernel == 0
                   ? entry.xnor_gemm_bn_sign_pack(A.as<uint32_t>(), A.ld, B.as<uint32_t>(), B.ld, A.rows, B.rows, K,
                                                  static_cast<const int32_t*>(thr), static_cast<Words>(flip),
                                                  out.as<uint32_t>(), out.ld, s)
                   : entry.xnor_gemm_bn_sign_pack_kernel(A.as<uint32_t>(), A.ld, B.as<uint32_t>(), B.ld, A.rows, B.rows, K,
                                                         static_cast<const int32_t*>(thr), static_cast<Words>(flip),
                                                         out.as<uint32_t>(), out.ld, kernel, s);
    });
}

// (x, B, K, thr, flip, a_bits, out): every row of x is a row of a_bits, and K elements long
PyObject* sign_gemm_bn_sign_pack(PyObject* const* a) {
    Matrix x, B, bits, out;
    int64_t K;
    if (!x.read(a[0], at::kFloat) || !B.read(a[1], at::kInt) || !integer(a[2], K) || K <= 0 || x.cols != K || B.cols < words(K))
        return long_way();
    const void* thr = vector_of(a[3], B.rows);
    const void* flip = vector_of(a[4], words(B.rows));
    if (!thr || !flip || !bits.read(a[5], at::kInt) || bits.rows != x.rows || bits.cols < words(K) || !out.read(a[6], at::kInt) ||
        !out.holds(x.rows, words(B.rows)))
        return long_way();
    return launch(*out.t, [&](void* s) {
        return entry.sign_gemm_bn_sign_pack(x.as<float>(), x.ld, B.as<uint32_t>(), B.ld, x.rows, B.rows, K,
                                            static_cast<const int32_t*>(thr), static_cast<Words>(flip), bits.as<uint32_t>(), bits.ld,
                                            out.as<uint32_t>(), out.ld, s);
    });
}

// (x, out)
PyObject* pack_bitplanes(PyObject* const* a) {
    Matrix x, out;
    if (!x.read(a[0], at::kByte) || !out.read(a[1], at::kInt) || !out.holds(x.rows, 8 * words(x.cols))) return long_way();
    return launch(*out.t, [&](void* s) { return entry.pack_bitplanes(x.as<uint8_t>(), x.rows, x.cols, x.ld, out.as<uint32_t>(), out.ld, s); });
}

// The operands of a product on bit planes, where there is one.
bool planes_hold(const Matrix& X, const Matrix& B, int64_t K) {
    return X.holds(B.rows > 0 ? X.rows : 0, 8 * words(K)) && B.holds(X.rows > 0 ? B.rows : 0, words(K));
}

// (Xp, B, K, out)
PyObject* bitplane_gemm(PyObject* const* a) {
    Matrix X, B, out;
    int64_t K;
    if (!X.read(a[0], at::kInt) || !B.read(a[1], at::kInt) || !integer(a[2], K) || !out.read(a[3], at::kInt) ||
        !planes_hold(X, B, K) || !out.holds(X.rows, B.rows))
        return long_way();
    return launch(*out.t, [&](void* s) {
        return entry.bitplane_gemm(X.as<uint32_t>(), X.ld, B.as<uint32_t>(), B.ld, out.as<int32_t>(), out.ld, X.rows, B.rows, K, s);
    });
}

// (Xp, B, K, thr, flip, out)
PyObject* bitplane_gemm_bn_sign_pack(PyObject* const* a) {
    Matrix X, B, out;
    int64_t K;
    if (!X.read(a[0], at::kInt) || !B.read(a[1], at::kInt) || !integer(a[2], K) || !planes_hold(X, B, K)) return long_way();
    const void* thr = vector_of(a[3], B.rows);
    const void* flip = vector_of(a[4], words(B.rows));
    if (!thr || !flip || !out.read(a[5], at::kInt) || !out.holds(X.rows, words(B.rows))) return long_way();
    return launch(*out.t, [&](void* s) {
        return entry.bitplane_gemm_bn_sign_pack(X.as<uint32_t>(), X.ld, B.as<uint32_t>(), B.ld, X.rows, B.rows, K,
                                                static_cast<const int32_t*>(thr), static_cast<Words>(flip), out.as<uint32_t>(),
                                                out.ld, s);
    });
}

// Output pixels of a convolution; 0 for a geometry that the library refuses.
int64_t conv_pixels(const Map& x, int kh, int kw, int stride, int pad) {
    const int64_t dh = x.H + 2 * int64_t(pad) - kh, dw = x.W + 2 * int64_t(pad) - kw;
    return dh < 0 || dw < 0 ? 0 : x.B * (dh / stride + 1) * (dw / stride + 1);
}

struct Conv {
    Map x;
    Matrix w;
    int64_t Cin = 0, M = 0;
    int kh = 0, kw = 0, stride = 0, pad = 0;
    // (x_bits, Cin, w_bits, kh, kw, stride, pad)
    bool read(PyObject* const* a) {
        if (!integer(a[1], Cin) || Cin <= 0 || !x.read(a[0], Cin) || !w.read(a[2], at::kInt) || !small_integer(a[3], kh) ||
            !small_integer(a[4], kw) || !small_integer(a[5], stride) || !small_integer(a[6], pad) || stride < 1)
            return false;
        M = conv_pixels(x, kh, kw, stride, pad);
        // (a window whose bits do not fit 64 is the wrapper's and the library's to refuse)
        return kh > 0 && kw > 0 && Cin <= INT32_MAX && int64_t(kh) * kw <= INT32_MAX &&
               w.holds(M > 0 ? w.rows : 0, words(int64_t(kh) * kw * Cin));
    }
};

// (x_bits, Cin, w_bits, kh, kw, stride, pad, out)
PyObject* conv_xnor(PyObject* const* a) {
    Conv c;
    Matrix out;
    if (!c.read(a) || !out.read(a[7], at::kInt) || !out.holds(c.M, c.w.rows)) return long_way();
    return launch(*out.t, [&](void* s) {
        return entry.conv_xnor(c.x.data, c.x.B, c.x.H, c.x.W, c.Cin, c.w.as<uint32_t>(), c.w.ld, c.w.rows, c.kh, c.kw, c.stride,
                               c.pad, out.as<int32_t>(), out.ld, s);
    });
}

// (x_bits, Cin, w_bits, kh, kw, stride, pad, thr, flip, out)
PyObject* conv_bn_sign_pack(PyObject* const* a) {
    Conv c;
    Matrix out;
    if (!c.read(a)) return long_way();
    const void* thr = vector_of(a[7], c.w.rows);
    const void* flip = vector_of(a[8], words(c.w.rows));
    if (!thr || !flip || !out.read(a[9], at::kInt) || !out.holds(c.M, words(c.w.rows))) return long_way();
    return launch(*out.t, [&](void* s) {
        return entry.conv_bn_sign_pack(c.x.data, c.x.B, c.x.H, c.x.W, c.Cin, c.w.as<uint32_t>(), c.w.ld, c.w.rows, c.kh, c.kw,
                                       c.stride, c.pad, static_cast<const int32_t*>(thr), static_cast<Words>(flip),
                                       out.as<uint32_t>(), out.ld, s);
    });
}

// (x_bits, Cin, w_bits, kh, kw, stride, pad, thr, flip, out, pool)
template <auto EntryPoints::*POOLED>
PyObject* conv_pool_of(PyObject* const* a) {
    Conv c;
    Matrix out;
    int pool;
    if (!c.read(a) || !small_integer(a[10], pool) || pool < 1) return long_way();
    const void* thr = vector_of(a[7], c.w.rows);
    const void* flip = vector_of(a[8], words(c.w.rows));
    const int64_t dh = c.x.H + 2 * int64_t(c.pad) - c.kh, dw = c.x.W + 2 * int64_t(c.pad) - c.kw;
    if (!thr || !flip || !out.read(a[9], at::kInt) || dh < 0 || dw < 0) return long_way();
    const int64_t Ho = dh / c.stride + 1, Wo = dw / c.stride + 1;
    if (out.rows != c.x.B * (Ho / pool) * (Wo / pool) || out.cols != words(c.w.rows)) return long_way();
    return launch(*out.t, [&](void* s) {
        return (entry.*POOLED)(c.x.data, c.x.B, c.x.H, c.x.W, c.Cin, c.w.as<uint32_t>(), c.w.ld, c.w.rows, c.kh, c.kw,
                               c.stride, c.pad, pool, static_cast<const int32_t*>(thr), static_cast<Words>(flip),
                               out.as<uint32_t>(), out.ld, s);
    });
}
PyObject* conv_pool_bn_sign_pack(PyObject* const* a) { return conv_pool_of<&EntryPoints::conv_pool_bn_sign_pack>(a); }
PyObject* conv_pool_windows_bn_sign_pack(PyObject* const* a) {
    return conv_pool_of<&EntryPoints::conv_pool_windows_bn_sign_pack>(a);
}

// (x_bits, Cin, kh, kw, stride, pad, out)
PyObject* conv_im2col_pack(PyObject* const* a) {
    Map x;
    Matrix out;
    int64_t Cin;
    int kh, kw, stride, pad;
    if (!integer(a[1], Cin) || Cin <= 0 || !x.read(a[0], Cin) || !small_integer(a[2], kh) || !small_integer(a[3], kw) ||
        !small_integer(a[4], stride) || !small_integer(a[5], pad) || stride < 1 || !out.read(a[6], at::kInt) || kh < 1 || kw < 1 ||
        Cin > INT32_MAX || int64_t(kh) * kw > INT32_MAX ||
        !out.holds(conv_pixels(x, kh, kw, stride, pad), words(int64_t(kh) * kw * Cin)))
        return long_way();
    return launch(*out.t, [&](void* s) {
        return entry.conv_im2col_pack(x.data, x.B, x.H, x.W, Cin, kh, kw, stride, pad, out.as<uint32_t>(), out.ld, s);
    });
}

// (x_bits, C, flip or None, ph, pw, stride, out)
PyObject* maxpool_bits(PyObject* const* a) {
    Map x;
    int64_t C;
    int ph, pw, stride;
    if (!integer(a[1], C) || C <= 0 || !x.read(a[0], C) || !small_integer(a[3], ph) || !small_integer(a[4], pw) ||
        !small_integer(a[5], stride) || stride < 1 || x.H < ph || x.W < pw)
        return long_way();
    const void* flip = a[2] == Py_None ? nullptr : vector_of(a[2], x.Cw);
    const at::Tensor* out = plain(a[6], at::kInt);
    if ((a[2] != Py_None && !flip) || !out || !out->is_contiguous() ||
        out->numel() != x.B * ((x.H - ph) / stride + 1) * ((x.W - pw) / stride + 1) * x.Cw)
        return long_way();
    return launch(*out, [&](void* s) {
        return entry.maxpool_bits(x.data, x.B, x.H, x.W, C, ph, pw, stride, static_cast<Words>(flip),
                                  static_cast<uint32_t*>(out->data_ptr()), s);
    });
}

// ---- real activations, packed weights ----

// The bnn_type of a matrix of activations; -1 for another type.
int real_type(at::ScalarType t) { return t == at::kBFloat16 ? 0 : t == at::kHalf ? 1 : t == at::kFloat ? 2 : -1; }

// A matrix of activations; of the type and on the device of `like`, with its rows and cols given.
bool read_real(PyObject* o, Matrix& m, const at::Tensor* like, int64_t rows, int64_t cols) {
    if (!THPVariable_CheckExact(o)) return false;
    const at::ScalarType type = like ? like->scalar_type() : THPVariable_Unpack(o).scalar_type();
    if (real_type(type) < 0 || !m.read(o, type)) return false;
    return !like || (m.t->get_device() == like->get_device() && m.rows == rows && m.cols == cols);
}

// A contiguous float32 vector of n elements on the device of `like`, or None; false for anything else.
bool read_vector(PyObject* o, int64_t n, const at::Tensor& like, const float*& data) {
    data = nullptr;
    if (o == Py_None) return true;
    const at::Tensor* t = plain(o, at::kFloat);
    if (!t || t->dim() != 1 || t->size(0) != n || !t->is_contiguous() || t->get_device() != like.get_device()) return false;
    data = static_cast<const float*>(t->data_ptr());
    return true;
}

// x, its packed weights, their scale and bias: the arguments that both products begin with.
struct Weighted {
    Matrix x, w;
    const float *scale = nullptr, *bias = nullptr;
    int type = -1;
    bool read(PyObject* const* a) {
        if (!read_real(a[0], x, nullptr, 0, 0) || !w.read(a[1], at::kInt) || w.t->get_device() != x.t->get_device() ||
            w.cols < words(x.cols) || !read_vector(a[2], w.rows, *x.t, scale) || !read_vector(a[3], w.rows, *x.t, bias))
            return false;
        type = real_type(x.t->scalar_type());
        return true;
    }
};

// A caller's tensor is written: torch's count of that moves on, so that who kept the tensor can tell.
void count_write(const Matrix& m) {
    if (m.t && !m.t->is_inference()) m.t->unsafeGetTensorImpl()->bump_version();
}

// (x, w_bits, scale, bias, act, residual, out)
PyObject* linear_bits(PyObject* const* a) {
    Weighted p;
    Matrix residual, out;
    int act;
    if (!p.read(a) || !small_integer(a[4], act) || !read_real(a[6], out, p.x.t, p.x.rows, p.w.rows) ||
        (a[5] != Py_None && !read_real(a[5], residual, p.x.t, p.x.rows, p.w.rows)))
        return long_way();
    count_write(out);
    return launch(*out.t, [&](void* s) {
        return entry.linear_bits(p.type, p.x.data, p.x.ld, p.w.as<uint32_t>(), p.w.ld, p.scale, p.bias, act, residual.data,
                                 residual.ld, out.data, out.ld, p.x.rows, p.w.rows, p.x.cols, s);
    });
}

// (x, w_bits, scale, bias, act, out)
PyObject* gated_bits(PyObject* const* a) {
    Weighted p;
    Matrix out;
    int act;
    if (!p.read(a) || p.w.rows % 2 != 0 || !small_integer(a[4], act) || !read_real(a[5], out, p.x.t, p.x.rows, p.w.rows / 2))
        return long_way();
    count_write(out);
    return launch(*out.t, [&](void* s) {
        return entry.gated_bits(p.type, p.x.data, p.x.ld, p.w.as<uint32_t>(), p.w.ld, p.scale, p.bias, act, out.data, out.ld,
                                p.x.rows, p.w.rows / 2, p.x.cols, s);
    });
}

bool real_number(PyObject* o, float& v) {
    if (!PyFloat_CheckExact(o)) return false;
    v = static_cast<float>(PyFloat_AS_DOUBLE(o));
    return true;
}

// (y, x, gate, res_scale, post, post_gamma, post_beta, pre, pre_gamma, pre_beta, eps, rows_per_gate, out, out_n)
PyObject* norm_residual(PyObject* const* a) {
    Matrix y, x, gate, out, out_n;
    const float *post_gamma, *post_beta, *pre_gamma, *pre_beta;
    float res_scale, eps;
    int post, pre;
    int64_t rows_per_gate;
    if (!read_real(a[0], y, nullptr, 0, 0) || !real_number(a[3], res_scale) || !small_integer(a[4], post) ||
        !small_integer(a[7], pre) || !real_number(a[10], eps) || !integer(a[11], rows_per_gate) || rows_per_gate < 1)
        return long_way();
    const int64_t M = y.rows, D = y.cols;
    if ((a[1] != Py_None && !read_real(a[1], x, y.t, M, D)) ||
        (a[2] != Py_None && !read_real(a[2], gate, y.t, M / rows_per_gate + (M % rows_per_gate != 0), D)) ||
        !read_vector(a[5], D, *y.t, post_gamma) || !read_vector(a[6], D, *y.t, post_beta) || !read_vector(a[8], D, *y.t, pre_gamma) ||
        !read_vector(a[9], D, *y.t, pre_beta) || !read_real(a[12], out, y.t, M, D) || (pre == 0) != (a[13] == Py_None) ||
        (a[13] != Py_None && !read_real(a[13], out_n, y.t, M, D)))
        return long_way();
    count_write(out);
    count_write(out_n);
    return launch(*out.t, [&](void* s) {
        return entry.norm_residual(real_type(y.t->scalar_type()), y.data, y.ld, x.data, x.ld, gate.data, gate.ld, rows_per_gate,
                                   res_scale, post, post_gamma, post_beta, pre, pre_gamma, pre_beta, eps, out.data, out.ld,
                                   out_n.data, out_n.ld, M, D, s);
    });
}

// Backward passes: what they return is allocated here, and comes as (status, tensors or None ...).

bool truth(PyObject* o, bool& v) {
    if (!PyBool_Check(o)) return false;
    v = o == Py_True;
    return true;
}

at::Tensor empty_like(const at::Tensor& t, at::IntArrayRef size, at::ScalarType type) {
    return at::empty(size, t.options().dtype(type).requires_grad(false));
}

// The caller's workspace, or one that is made; false where the caller's is none or too small.
bool workspace_of(PyObject* o, int64_t size, const at::Tensor& like, at::Tensor& ws) {
    if (size < 0) return false;
    if (o == Py_None) {
        ws = empty_like(like, {size}, at::kByte);
        return true;
    }
    const at::Tensor* t = plain(o, at::kByte);
    if (!t || !t->is_contiguous() || t->get_device() != like.get_device() || t->numel() < size) return false;
    ws = *t;
    return true;
}

template <size_t N>
PyObject* results(int status, const at::Tensor (&t)[N]) {
    PyObject* r = PyTuple_New(N + 1);
    if (!r) return nullptr;
    PyObject* s = PyLong_FromLong(status);
    if (!s) {
        Py_DECREF(r);
        return nullptr;
    }
    PyTuple_SET_ITEM(r, 0, s);
    for (size_t i = 0; i < N; ++i) {
        PyObject* v = nullptr;
        if (t[i].defined()) {
            v = THPVariable_Wrap(t[i]);
        } else {
            v = Py_None;
            Py_INCREF(v);
        }
        if (!v) {
            Py_DECREF(r);
            return nullptr;
        }
        PyTuple_SET_ITEM(r, i + 1, v);
    }
    return r;
}

// Calls the library without the interpreter lock.
template <typename F>
bool run(const at::Tensor& t, int& status, F&& call) {
    void* stream;
    if (!stream_of(t, stream)) return false;
    Py_BEGIN_ALLOW_THREADS
    status = call(stream);
    Py_END_ALLOW_THREADS
    return true;
}

void* data_of(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

// (dy, x, w_bits, scale, bias, act, need_dx, need_dw, workspace) -> (status, dx, dw, dscale, dbias)
template <bool GATED>
PyObject* product_backward(PyObject* const* a) {
    Weighted p;
    Matrix dy;
    int act;
    bool need_dx, need_dw;
    if (!p.read(a + 1) || (GATED && p.w.rows % 2 != 0) || !small_integer(a[5], act) || !truth(a[6], need_dx) || !truth(a[7], need_dw))
        return long_way();
    const int64_t M = p.x.rows, K = p.x.cols, N = p.w.rows, cols = GATED ? N / 2 : N;
    if (!read_real(a[0], dy, p.x.t, M, cols)) return long_way();
    at::Tensor ws, out[4];
    const int64_t size = (GATED ? entry.gated_bits_backward_workspace : entry.linear_bits_backward_workspace)(p.type, M, cols, K, act);
    if (!workspace_of(a[8], size, *p.x.t, ws)) return long_way();
    const at::ScalarType type = p.x.t->scalar_type();
    if (need_dx) out[0] = empty_like(*p.x.t, {M, K}, type);
    if (need_dw) out[1] = empty_like(*p.x.t, {N, K}, type);
    if (p.scale) out[2] = empty_like(*p.x.t, {N}, at::kFloat);
    if (p.bias) out[3] = empty_like(*p.x.t, {N}, at::kFloat);
    int status;
    if (!run(*p.x.t, status, [&](void* s) {
            return (GATED ? entry.gated_bits_backward : entry.linear_bits_backward)(
                p.type, dy.data, dy.ld, p.x.data, p.x.ld, p.w.as<uint32_t>(), p.w.ld, p.scale, p.bias, act, data_of(out[0]), K,
                data_of(out[1]), K, static_cast<float*>(data_of(out[2])), static_cast<float*>(data_of(out[3])), M, cols, K,
                ws.data_ptr(), ws.numel(), s);
        }))
        return nullptr;
    return results(status, out);
}
PyObject* linear_bits_backward(PyObject* const* a) { return product_backward<false>(a); }
PyObject* gated_bits_backward(PyObject* const* a) { return product_backward<true>(a); }

// (dr, dn, y, r, gate, res_scale, post, post_gamma, post_beta, pre, pre_gamma, pre_beta, eps, rows_per_gate, need_dx, workspace)
//   -> (status, dx, dy, dgate, dpost_gamma, dpost_beta, dpre_gamma, dpre_beta)
PyObject* norm_residual_backward(PyObject* const* a) {
    Matrix dr, dn, y, r, gate;
    const float *post_gamma, *post_beta, *pre_gamma, *pre_beta;
    float res_scale, eps;
    int post, pre;
    int64_t R;
    bool need_dx;
    if (!read_real(a[2], y, nullptr, 0, 0) || !real_number(a[5], res_scale) || !small_integer(a[6], post) || !small_integer(a[9], pre) ||
        !real_number(a[12], eps) || !integer(a[13], R) || R < 1 || !truth(a[14], need_dx))
        return long_way();
    const int64_t M = y.rows, D = y.cols;
    auto optional = [&](PyObject* o, Matrix& m, int64_t rows) { return o == Py_None || read_real(o, m, y.t, rows, D); };
    if (!optional(a[0], dr, M) || !optional(a[1], dn, M) || !optional(a[3], r, M) || !optional(a[4], gate, M / R + (M % R != 0)) ||
        (pre == 0 ? a[1] != Py_None : a[1] == Py_None || a[3] == Py_None) || !read_vector(a[7], D, *y.t, post_gamma) ||
        !read_vector(a[8], D, *y.t, post_beta) || !read_vector(a[10], D, *y.t, pre_gamma) || !read_vector(a[11], D, *y.t, pre_beta))
        return long_way();
    at::Tensor ws, out[7];
    if (!workspace_of(a[15], entry.norm_residual_backward_workspace(M, D, R), *y.t, ws)) return long_way();
    const at::ScalarType type = y.t->scalar_type();
    if (need_dx) out[0] = empty_like(*y.t, {M, D}, type);
    out[1] = empty_like(*y.t, {M, D}, type);
    if (gate.t) out[2] = empty_like(*y.t, {gate.rows, D}, type);
    const float* const vectors[4] = {post_gamma, post_beta, pre_gamma, pre_beta};
    for (int i = 0; i < 4; ++i)
        if (vectors[i]) out[3 + i] = empty_like(*y.t, {D}, at::kFloat);
    int status;
    if (!run(*y.t, status, [&](void* s) {
            return entry.norm_residual_backward(
                real_type(type), dr.data, dr.ld, dn.data, dn.ld, y.data, y.ld, r.data, r.ld, gate.data, gate.ld, R, res_scale, post,
                post_gamma, post_beta, pre, pre_gamma, eps, data_of(out[0]), D, data_of(out[1]), D, data_of(out[2]), D,
                static_cast<float*>(data_of(out[3])), static_cast<float*>(data_of(out[4])), static_cast<float*>(data_of(out[5])),
                static_cast<float*>(data_of(out[6])), M, D, ws.data_ptr(), ws.numel(), s);
        }))
        return nullptr;
    return results(status, out);
}

// bind({"bnn_pack_sign": address, ...}, raw_stream)
PyObject* bind(PyObject*, PyObject* args) {
    PyObject *table, *stream;
    if (!PyArg_ParseTuple(args, "O!O", &PyDict_Type, &table, &stream)) return nullptr;
    EntryPoints e{};
    bool ok = true;
    auto set = [&](auto& fn, const char* name) {
        PyObject* v = PyDict_GetItemString(table, name);
        void* p = v ? PyLong_AsVoidPtr(v) : nullptr;
        if (!p) ok = false;
        fn = reinterpret_cast<std::decay_t<decltype(fn)>>(p);
    };
    set(e.pack_sign, "bnn_pack_sign");
    set(e.xnor_gemm, "bnn_xnor_gemm");
    set(e.xnor_gemm_kernel, "bnn_xnor_gemm_kernel");
    set(e.bn_sign_pack, "bnn_bn_sign_pack");
    set(e.xnor_gemm_bn_sign_pack, "bnn_xnor_gemm_bn_sign_pack");
    set(e.xnor_gemm_bn_sign_pack_kernel, "bnn_xnor_gemm_bn_sign_pack_kernel");
    set(e.sign_gemm_bn_sign_pack, "bnn_sign_gemm_bn_sign_pack");
    set(e.pack_bitplanes, "bnn_pack_bitplanes");
    set(e.bitplane_gemm, "bnn_bitplane_gemm");
    set(e.bitplane_gemm_bn_sign_pack, "bnn_bitplane_gemm_bn_sign_pack");
    set(e.conv_xnor, "bnn_conv_xnor");
    set(e.conv_bn_sign_pack, "bnn_conv_bn_sign_pack");
    set(e.conv_pool_bn_sign_pack, "bnn_conv_pool_bn_sign_pack");
    set(e.conv_pool_windows_bn_sign_pack, "bnn_conv_pool_windows_bn_sign_pack");
    set(e.conv_im2col_pack, "bnn_conv_im2col_pack");
    set(e.maxpool_bits, "bnn_maxpool_bits");
    set(e.linear_bits, "bnn_linear_bits");
    set(e.gated_bits, "bnn_gated_bits");
    set(e.norm_residual, "bnn_norm_residual");
    set(e.linear_bits_backward_workspace, "bnn_linear_bits_backward_workspace");
    set(e.gated_bits_backward_workspace, "bnn_gated_bits_backward_workspace");
    set(e.linear_bits_backward, "bnn_linear_bits_backward");
    set(e.gated_bits_backward, "bnn_gated_bits_backward");
    set(e.norm_residual_backward_workspace, "bnn_norm_residual_backward_workspace");
    set(e.norm_residual_backward, "bnn_norm_residual_backward");
    if (!ok || !PyCallable_Check(stream)) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an entry point or the stream function is missing");
        return nullptr;
    }
    entry = e;
    Py_INCREF(stream);
    Py_XDECREF(raw_stream);
    raw_stream = stream;
    Py_RETURN_NONE;
}

template <PyObject* (*F)(PyObject* const*), Py_ssize_t ARGS>
PyMethodDef fast(const char* name) {
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry_of<F, ARGS>)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    fast<pack_sign, 2>("pack_sign"),
    fast<xnor_gemm, 5>("xnor_gemm"),
    fast<bn_sign_pack, 4>("bn_sign_pack"),
    fast<xnor_gemm_bn_sign_pack, 7>("xnor_gemm_bn_sign_pack"),
    fast<sign_gemm_bn_sign_pack, 7>("sign_gemm_bn_sign_pack"),
    fast<pack_bitplanes, 2>("pack_bitplanes"),
    fast<bitplane_gemm, 4>("bitplane_gemm"),
    fast<bitplane_gemm_bn_sign_pack, 6>("bitplane_gemm_bn_sign_pack"),
    fast<conv_xnor, 8>("conv_xnor"),
    fast<conv_bn_sign_pack, 10>("conv_bn_sign_pack"),
    fast<conv_pool_bn_sign_pack, 11>("conv_pool_bn_sign_pack"),
    fast<conv_pool_windows_bn_sign_pack, 11>("conv_pool_windows_bn_sign_pack"),
    fast<conv_im2col_pack, 7>("conv_im2col_pack"),
    fast<maxpool_bits, 7>("maxpool_bits"),
    fast<linear_bits, 7>("linear_bits"),
    fast<gated_bits, 6>("gated_bits"),
    fast<norm_residual, 14>("norm_residual"),
    fast<linear_bits_backward, 9>("linear_bits_backward"),
    fast<gated_bits_backward, 9>("gated_bits_backward"),
    fast<norm_residual_backward, 16>("norm_residual_backward"),
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", "Direct calls of the bnn C ABI on torch tensors.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
