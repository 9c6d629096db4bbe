// Native argument marshalling of the serving operators: checks torch tensors and calls the C ABI (include/cake_serving.h).
// A decode step makes these calls hundreds of times for kernels of a few microseconds; the same checks in Python cost more than
// such a kernel.  Every output is given by the caller (paper_2608_12629_b200/serving.py allocates what its caller left out).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>

#include "../../../include/cake_serving.h"

namespace {

// A Python exception is set: unwinds to the entry point, which returns NULL.
struct Raised {};

[[noreturn]] void raise(PyObject* type, const char* format, const char* name, const char* more = "") {
    PyErr_Format(type, format, name, more);
    throw Raised();
}

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) raise(PyExc_TypeError, "%s must be a tensor%s", name);
    return THPVariable_Unpack(o);
}
const at::Tensor* maybe(PyObject* o, const char* name) { return o == Py_None ? nullptr : &tensor(o, name); }

long long integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised();
    return v;
}
int small(PyObject* o) {
    const long long v = integer(o);
    if (v < INT_MIN || v > INT_MAX) raise(PyExc_OverflowError, "%s%s", "integer argument out of range");
    return static_cast<int>(v);
}
float real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised();
    return static_cast<float>(v);
}

// The device that all of a call's tensors are on, made current for the call.
class Call {
public:
    Call(const at::Tensor& first) : index_(first.is_cuda() ? first.get_device() : -1) {
        if (index_ < 0) raise(PyExc_TypeError, "the operators take CUDA tensors%s%s", "");
        before_ = c10::cuda::current_device();
        if (before_ != index_) c10::cuda::set_device(index_);
    }
    ~Call() {
        if (before_ != index_) {
            try {
                c10::cuda::set_device(before_);
            } catch (...) {      // a destructor lets nothing out
            }
        }
    }
    void* at(const at::Tensor& t, const char* name) const {
        if (!t.is_cuda() || t.get_device() != index_) raise(PyExc_ValueError, "%s is not on the device of the other tensors%s", name);
        return t.data_ptr();
    }
    void* at(const at::Tensor* t, const char* name) const { return t ? at(*t, name) : nullptr; }
    // contiguous, of this type and shape
    void* dense(const at::Tensor& t, at::ScalarType type, c10::IntArrayRef shape, const char* name) const {
        if (t.scalar_type() != type || t.sizes() != shape || !t.is_contiguous())
            raise(PyExc_TypeError, "%s must be a contiguous tensor of the operator's type and shape%s", name);
        return at(t, name);
    }
    void* dense(const at::Tensor* t, at::ScalarType type, c10::IntArrayRef shape, const char* name) const {
        return t ? dense(*t, type, shape, name) : nullptr;
    }
    cake_stream_t stream(PyObject* given) const {
        if (given != Py_None) return reinterpret_cast<cake_stream_t>(PyLong_AsVoidPtr(given));
        return reinterpret_cast<cake_stream_t>(c10::cuda::getCurrentCUDAStream(index_).stream());
    }

private:
    c10::DeviceIndex index_, before_ = -1;
};

struct Matrix {
    long long rows, cols, stride;
};
// rows of any distance, contiguous each
Matrix rows_of(const at::Tensor& t, at::ScalarType type, const char* name) {
    if (t.scalar_type() != type || t.dim() != 2 || (t.stride(1) != 1 && t.size(1) > 1))
        raise(PyExc_TypeError, "%s must be a matrix of the operator's type with contiguous rows%s", name);
    return {t.size(0), t.size(1), t.size(0) > 1 ? t.stride(0) : t.size(1)};
}
struct Heads {
    long long tokens, heads, stride;
};
// [T, heads, D] bf16, heads contiguous and next to each other
Heads heads_of(const at::Tensor& t, int D, const char* name) {
    if (t.scalar_type() != at::kBFloat16 || t.dim() != 3 || t.size(2) != D || t.stride(2) != 1 || (t.stride(1) != D && t.size(1) > 1))
        raise(PyExc_TypeError, "%s must be a bf16 [T, heads, D] tensor with contiguous heads%s", name);
    return {t.size(0), t.size(1), t.size(0) > 1 ? t.stride(0) : t.size(1) * D};
}
const at::Tensor& scratch(PyObject* o) {
    const at::Tensor& t = tensor(o, "ws");
    if (t.scalar_type() != at::kByte || !t.is_contiguous()) raise(PyExc_TypeError, "%s must be a contiguous uint8 tensor%s", "ws");
    return t;
}

void check_count(Py_ssize_t n, Py_ssize_t want) {
    if (n != want) raise(PyExc_TypeError, "%s%s", "wrong number of arguments");
}

template <class F>
PyObject* guarded(F&& f) {
    try {
        return PyLong_FromLong(f());
    } catch (const Raised&) {
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}

const at::ScalarType kE4M3 = at::kFloat8_e4m3fn;

// (x, weight, residual, eps, group, out_residual, out_y, out_q, out_scale, stream, flags)
PyObject* rmsnorm_quant(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> int {
        check_count(n, 11);
        const at::Tensor& x = tensor(a[0], "x");
        const at::Tensor *w = maybe(a[1], "weight"), *r = maybe(a[2], "residual"), *out_r = maybe(a[5], "out_residual"),
                         *out_y = maybe(a[6], "out_y"), *out_q = maybe(a[7], "out_q"), *out_s = maybe(a[8], "out_scale");
        const Matrix m = rows_of(x, at::kBFloat16, "x");
        const Call call(x);
        long long r_stride = m.cols;
        if (r) {
            const Matrix mr = rows_of(*r, at::kBFloat16, "residual");
            if (mr.rows != m.rows || mr.cols != m.cols) raise(PyExc_ValueError, "%s must have x's shape%s", "residual");
            r_stride = mr.stride;
        }
        const int group = small(a[4]);
        const long long shape[2] = {m.rows, m.cols}, scales[2] = {m.rows, group == 0 ? 1 : (m.cols + 127) / 128};
        if (m.cols > INT_MAX) return CAKE_ERR_UNSUPPORTED;
        const long long wide[1] = {m.cols};
        const void* w_at = call.dense(w, at::kBFloat16, {reinterpret_cast<const int64_t*>(wide), 1}, "weight");
        const c10::IntArrayRef full(reinterpret_cast<const int64_t*>(shape), 2), per(reinterpret_cast<const int64_t*>(scales), 2);
        return cake_rmsnorm_quant(static_cast<const cake_bf16*>(call.at(x, "x")), m.stride, static_cast<const cake_bf16*>(call.at(r, "residual")), r_stride,
                                  static_cast<const cake_bf16*>(w_at), m.rows, static_cast<int>(m.cols), real(a[3]), group,
                                  static_cast<cake_bf16*>(call.dense(out_r, at::kBFloat16, full, "out_residual")),
                                  static_cast<cake_bf16*>(call.dense(out_y, at::kBFloat16, full, "out_y")),
                                  static_cast<cake_e4m3*>(call.dense(out_q, kE4M3, full, "out_q")),
                                  static_cast<float*>(call.dense(out_s, at::kFloat, per, "out_scale")), call.stream(a[9]),
                                  static_cast<unsigned>(small(a[10])));
    });
}

// (X, x_scale, W, w_scale, out, ws, stream)
PyObject* gemm_fp8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> int {
        check_count(n, 7);
        const at::Tensor &x = tensor(a[0], "X"), &xs = tensor(a[1], "x_scale"), &w = tensor(a[2], "W"), &ws = tensor(a[3], "w_scale"),
                         &out = tensor(a[4], "out"), &buf = scratch(a[5]);
        const Matrix mx = rows_of(x, kE4M3, "X"), mw = rows_of(w, kE4M3, "W");
        const Call call(x);
        if (mx.cols != mw.cols) raise(PyExc_ValueError, "X must be [M,K] and W [N,K]%s%s", "");
        const bool fp32 = out.scalar_type() == at::kFloat;
        const Matrix mo = rows_of(out, fp32 ? at::kFloat : at::kBFloat16, "out");
        if (mo.rows != mx.rows || mo.cols != mw.rows) raise(PyExc_TypeError, "%s must be a bf16 or fp32 [M,N] matrix%s", "out");
        if (mx.cols > INT_MAX || mw.rows > INT_MAX) return CAKE_ERR_SHAPE;
        const int64_t nk = (mx.cols + 127) / 128;
        const int64_t x_shape[2] = {mx.rows, nk}, w_shape[2] = {(mw.rows + 127) / 128, nk};
        const void* xs_at = call.dense(xs, at::kFloat, {x_shape, 2}, "x_scale");
        const void* ws_at = call.dense(ws, at::kFloat, {w_shape, 2}, "w_scale");
        return cake_gemm_fp8(static_cast<const cake_e4m3*>(call.at(x, "X")), mx.stride, static_cast<const float*>(xs_at),
                             static_cast<const cake_e4m3*>(call.at(w, "W")), mw.stride, static_cast<const float*>(ws_at), mx.rows,
                             static_cast<int>(mw.rows), static_cast<int>(mx.cols), call.at(out, "out"), mo.stride, call.at(buf, "ws"),
                             static_cast<size_t>(buf.numel()), call.stream(a[6]), fp32 ? CAKE_GEMM_OUT_FP32 : 0);
    });
}

const cake_paged_cache* cache_at(PyObject* o) {
    const void* p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) throw Raised();
    return static_cast<const cake_paged_cache*>(p);
}

// (cache address, cache's k, k, v, slots, positions, cos_sin, q, out_q, interleaved, ws, stream)
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> int {
        check_count(n, 12);
        const cake_paged_cache* cache = cache_at(a[0]);
        const Call call(tensor(a[1], "cache"));
        const at::Tensor &k = tensor(a[2], "k"), &v = tensor(a[3], "v"), &slots = tensor(a[4], "slots"), &buf = scratch(a[10]);
        const at::Tensor *pos = maybe(a[5], "positions"), *table = maybe(a[6], "cos_sin"), *q = maybe(a[7], "q"), *out = maybe(a[8], "out_q");
        const int D = cache->D;
        const Heads hk = heads_of(k, D, "k"), hv = heads_of(v, D, "v");
        if (hk.tokens != hv.tokens || hk.heads != hv.heads || hk.heads != cache->Hkv)
            raise(PyExc_ValueError, "k and v must be [T, Hkv, D] with the cache's Hkv%s%s", "");
        const int64_t T[1] = {hk.tokens};
        const void* slots_at = call.dense(slots, at::kLong, {T, 1}, "slots");
        const void *pos_at = nullptr, *table_at = nullptr;
        long long longest = 0, rot = 0;
        if (table) {
            if (!pos || table->dim() != 2) raise(PyExc_ValueError, "a rotation takes positions [T] and cos_sin [max_positions, rot]%s%s", "");
            longest = table->size(0), rot = table->size(1);
            table_at = call.dense(*table, at::kFloat, table->sizes(), "cos_sin");
            pos_at = call.dense(*pos, at::kInt, {T, 1}, "positions");
            if (rot > INT_MAX) return CAKE_ERR_SHAPE;
        }
        Heads hq = {0, 0, 0};
        void *q_at = nullptr, *out_at = nullptr;
        if (q) {
            hq = heads_of(*q, D, "q");
            if (hq.tokens != hk.tokens) raise(PyExc_ValueError, "%s must have k's tokens%s", "q");
            if (!out) raise(PyExc_TypeError, "%s must be given with q%s", "out_q");
            const int64_t shape[3] = {hq.tokens, hq.heads, D};
            q_at = call.at(*q, "q");
            out_at = call.dense(*out, at::kBFloat16, {shape, 3}, "out_q");
            if (hq.heads > INT_MAX) return CAKE_ERR_SHAPE;
        }
        const int turned = PyObject_IsTrue(a[9]);
        if (turned < 0) throw Raised();
        return cake_kv_append(cache, static_cast<const cake_bf16*>(call.at(k, "k")), hk.stride, static_cast<const cake_bf16*>(call.at(v, "v")), hv.stride,
                              static_cast<const cake_bf16*>(q_at), hq.stride, static_cast<int>(hq.heads), static_cast<cake_bf16*>(out_at),
                              static_cast<const long long*>(slots_at), rot ? static_cast<const int*>(pos_at) : nullptr,
                              rot ? static_cast<const float*>(table_at) : nullptr, longest, static_cast<int>(rot), hk.tokens, call.at(buf, "ws"),
                              static_cast<size_t>(buf.numel()), call.stream(a[11]), turned ? CAKE_APPEND_INTERLEAVED : 0);
    });
}

// (q, cache address, cache's k, page_table, seq_lens, scale, window, out, out_lse, ws, stream)
PyObject* paged_decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> int {
        check_count(n, 11);
        const at::Tensor &q = tensor(a[0], "q"), &table = tensor(a[3], "page_table"), &lens = tensor(a[4], "seq_lens"), &out = tensor(a[7], "out"),
                         &buf = scratch(a[9]);
        const at::Tensor* lse = maybe(a[8], "out_lse");
        const cake_paged_cache* cache = cache_at(a[1]);
        const int D = cache->D, Hkv = cache->Hkv;
        if (q.scalar_type() != at::kBFloat16 || q.dim() != 3 || q.size(2) != D || q.stride(2) != 1)
            raise(PyExc_TypeError, "%s must be a bf16 [B, Hq, D] tensor with contiguous rows%s", "q");
        const Call call(q);
        call.at(tensor(a[2], "cache"), "cache");
        if (table.scalar_type() != at::kInt || lens.scalar_type() != at::kInt) raise(PyExc_TypeError, "%s must be int32%s", "page_table and seq_lens");
        const int64_t td = table.dim(), ld = lens.dim();
        if ((td != 2 && td != 3) || (ld != 1 && ld != 2) || (table.size(-1) > 1 && table.stride(-1) != 1))
            raise(PyExc_TypeError, "page_table must be [B, max_pages] or [B, Hkv, max_pages] with contiguous rows, seq_lens [B] or [B, Hkv]%s%s", "");
        const int64_t B = q.size(0), Hq = q.size(1);
        if (table.size(0) != B || lens.size(0) != B || (td == 3 && table.size(1) != Hkv) || (ld == 2 && lens.size(1) != Hkv))
            raise(PyExc_ValueError, "page_table and seq_lens must have q's B (and the cache's Hkv where they are per head)%s%s", "");
        if (Hq > INT_MAX || table.size(-1) > INT_MAX) return CAKE_ERR_SHAPE;
        const int64_t out_shape[3] = {B, Hq, D};
        void* out_at = call.dense(out, at::kBFloat16, {out_shape, 3}, "out");
        void* lse_at = call.dense(lse, at::kFloat, {out_shape, 2}, "out_lse");
        return cake_paged_decode(static_cast<const cake_bf16*>(call.at(q, "q")), B > 1 ? q.stride(0) : 0, Hq > 1 ? q.stride(1) : 0, cache,
                                 static_cast<const int*>(call.at(table, "page_table")), table.stride(0), td == 3 ? table.stride(1) : 0,
                                 static_cast<int>(table.size(-1)), static_cast<const int*>(call.at(lens, "seq_lens")), lens.stride(0),
                                 ld == 2 ? lens.stride(1) : 0, B, static_cast<int>(Hq), real(a[5]), small(a[6]), static_cast<cake_bf16*>(out_at),
                                 static_cast<float*>(lse_at), call.at(buf, "ws"), static_cast<size_t>(buf.numel()), call.stream(a[10]));
    });
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name) {
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}
PyMethodDef methods[] = {method<rmsnorm_quant>("rmsnorm_quant"), method<gemm_fp8>("gemm_fp8"), method<kv_append>("kv_append"),
                         method<paged_decode>("paged_decode"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_serving", "Argument marshalling of the serving operators.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__serving() { return PyModule_Create(&module); }
