// Marshalling of torch tensors for the calls around the projection: shapes, types, strides and devices are looked at here, and the C
// entry point is called with what it wants.  The same through ctypes takes 3 to 5 us of host time a call, which is what a decode step's
// calls take on the GPU; here it is under 1 us.  Nothing is computed and nothing is kept between calls.
#include <Python.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cxxabi.h>
#include <limits.h>
#include <stdio.h>

#include <exception>

#include "../../include/gelo.h"

namespace {

// Raised as ValueError; `text` has been filled in
struct Refused { char text[400]; };

[[noreturn]] void refuse(const char* name, const char* wanted, const at::Tensor* t, int64_t rows, int64_t width, int device)
{
    Refused r;
    char is[160] = "no tensor";
    if (t) {
        int n = snprintf(is, sizeof is, "%s on %s of shape (", c10::toString(t->scalar_type()), t->device().str().c_str());
        for (int64_t i = 0; i < t->dim() && n > 0 && n < (int)sizeof is; ++i)
            n += snprintf(is + n, sizeof is - n, i ? ", %lld" : "%lld", (long long)t->size(i));
        if (n > 0 && n < (int)sizeof is) snprintf(is + n, sizeof is - n, ")");
    }
    if (width >= 0)
        snprintf(r.text, sizeof r.text, "%s must be %lld x %lld of %s on cuda:%d with contiguous rows, not %s", name, (long long)rows, (long long)width, wanted, device, is);
    else
        snprintf(r.text, sizeof r.text, "%s must hold %lld contiguous values of %s on cuda:%d, not %s", name, (long long)rows, wanted, device, is);
    throw r;
}

const at::Tensor& tensor(PyObject* o, const char* name)
{
    if (!THPVariable_Check(o)) refuse(name, "a type that the call takes", nullptr, 0, 0, 0);
    return THPVariable_Unpack(o);
}

int code_of(const at::Tensor& t, const char* name)
{
    switch (t.scalar_type()) {
        case at::kFloat: return GELO_F32;
        case at::kBFloat16: return GELO_BF16;
        case at::kHalf: return GELO_F16;
        default: break;
    }
    Refused r;
    snprintf(r.text, sizeof r.text, "unsupported dtype of %s: %s", name, c10::toString(t.scalar_type()));
    throw r;
}

struct Rows { void* at = nullptr; int ld = 0; };

// A matrix whose rows are contiguous and of one type; None where that is allowed
Rows rows_of(PyObject* o, const char* name, at::ScalarType type, int64_t rows, int64_t width, int device, bool optional = false)
{
    if (o == Py_None && optional) return {};
    const at::Tensor& t = tensor(o, name);
    if (t.scalar_type() != type || t.dim() != 2 || t.size(0) != rows || t.size(1) != width || !t.is_cuda() || t.get_device() != device ||
        (t.stride(1) != 1 && width > 1) || (rows > 1 && t.stride(0) > INT_MAX))
        refuse(name, c10::toString(type), &t, rows, width, device);
    return { t.data_ptr(), rows > 1 ? (int)t.stride(0) : (int)((width + 15) / 16 * 16) };      // (the stride of a single row is never used)
}

template <typename T>
T* values_of(PyObject* o, const char* name, at::ScalarType type, int64_t count, int device, bool optional = false)
{
    if (o == Py_None && optional) return nullptr;
    const at::Tensor& t = tensor(o, name);
    if (t.scalar_type() != type || t.numel() != count || !t.is_cuda() || t.get_device() != device || !t.is_contiguous())
        refuse(name, c10::toString(type), &t, count, -1, device);
    return static_cast<T*>(t.data_ptr());
}

void* address(PyObject* o)
{
    void* const p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) throw std::exception();
    return p;
}
void* stream_of(PyObject* o, int device)
{
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    if (PyLong_Check(o)) return address(o);
    PyObject* handle = PyObject_GetAttrString(o, "cuda_stream");
    if (!handle) throw std::exception();                      // (the Python error is set)
    void* const s = PyLong_AsVoidPtr(handle);
    Py_DECREF(handle);
    if (!s && PyErr_Occurred()) throw std::exception();
    return s;
}

template <typename T>
const T* struct_at(PyObject* o)                               // the address of a ctypes structure
{
    return o == Py_None ? nullptr : static_cast<const T*>(address(o));
}
int whole(PyObject* o)
{
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw std::exception();
    if (v < INT_MIN || v > INT_MAX) {
        Refused r;
        snprintf(r.text, sizeof r.text, "%ld is out of range", v);
        throw r;
    }
    return (int)v;
}
float number(PyObject* o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw std::exception();
    return (float)v;
}
gelo_ctx* context(PyObject* o) { return static_cast<gelo_ctx*>(address(o)); }

// Python's lock is let go of while the library launches, as ctypes does: a launch that waits for a full queue would hold up all threads, for good if what
// the queue waits for needs one of them.  Nothing of Python may be touched meanwhile; the caller's arguments keep the tensors alive.  (No destructor takes the
// lock back: where the interpreter is ending, that unwinds the thread.)
template <typename F>
int unlocked(F&& call)
{
    PyThreadState* const state = PyEval_SaveThread();
    const int status = call();                                // (throws nothing)
    PyEval_RestoreThread(state);
    return status;
}

template <typename F>
PyObject* guarded(Py_ssize_t given, Py_ssize_t wanted, F&& call)
{
    if (given != wanted) {
        PyErr_Format(PyExc_TypeError, "%zd arguments instead of %zd", given, wanted);
        return nullptr;
    }
    try {
        const int status = call();
        return PyErr_Occurred() ? nullptr : PyLong_FromLong(status);
    } catch (const Refused& r) {
        PyErr_SetString(PyExc_ValueError, r.text);
    } catch (const std::exception& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (const abi::__forced_unwind&) {
        throw;                                                // the thread is ending (see unlocked)
    } catch (...) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "unknown error");
    }
    return nullptr;
}

// (context, device, X, Y, weight, eps, residual, residual_out, codes, row_scale, stream)
PyObject* rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 11, [&] {
        const int device = whole(a[1]);
        const at::Tensor& x = tensor(a[2], "X");
        if (x.dim() != 2) refuse("X", "float, bfloat16 or half", &x, 0, 0, device);
        const int code = code_of(x, "X");
        const int64_t rows = x.size(0), d = x.size(1);
        if (rows > INT_MAX || d > INT_MAX) return (int)GELO_ERR_UNSUPPORTED;
        const at::ScalarType type = x.scalar_type();
        const Rows X = rows_of(a[2], "X", type, rows, d, device), Y = rows_of(a[3], "Y", type, rows, d, device, true);
        const void* w = values_of<void>(a[4], "weight", type, d, device, true);
        const Rows R = rows_of(a[6], "residual", type, rows, d, device, true), O = rows_of(a[7], "residual_out", type, rows, d, device, true);
        Rows C;
        if (a[8] != Py_None) {
            const at::ScalarType t = tensor(a[8], "codes").scalar_type();
            C = rows_of(a[8], "codes", t == at::kFloat8_e4m3fn ? t : at::kByte, rows, d, device);
        }
        float* const s = values_of<float>(a[9], "row_scale", at::kFloat, rows, device, true);
        gelo_ctx* const ctx = context(a[0]);
        const float eps = number(a[5]);
        void* const stream = stream_of(a[10], device);
        return unlocked([&] { return gelo_rms_norm(ctx, X.at, X.ld, R.at, R.ld, w, (int)rows, (int)d, eps, code, O.at, O.ld, Y.at, Y.ld, C.at, C.ld, s, stream); });
    });
}

// E4M3 codes: bytes, or torch's type for them
const void* codes_of(PyObject* o, const char* name, int64_t count, int device)
{
    const at::ScalarType t = tensor(o, name).scalar_type();
    return values_of<void>(o, name, t == at::kFloat8_e4m3fn ? t : at::kByte, count, device);
}

// (context, device, U8, u_scale, W8, w_scale, m, d, p, Yp, stream)
PyObject* project_e4m3_rows(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 11, [&] {
        const int device = whole(a[1]), m = whole(a[6]), d = whole(a[7]), p = whole(a[8]);
        const void* u = codes_of(a[2], "U8", (int64_t)m * d, device);
        const float* su = values_of<float>(a[3], "u_scale", at::kFloat, m, device);
        const void* w = codes_of(a[4], "W8", (int64_t)d * p, device);
        const at::Tensor& sw = tensor(a[5], "w_scale");                                // one value, or the pair that the quantiser leaves
        const float* scale = values_of<float>(a[5], "w_scale", at::kFloat, sw.numel() == 2 ? 2 : 1, device);
        void* y = values_of<void>(a[9], "Yp", at::kBFloat16, (int64_t)m * p, device);
        gelo_ctx* const ctx = context(a[0]);
        void* const stream = stream_of(a[10], device);
        return unlocked([&] { return gelo_project_e4m3_rows(ctx, u, su, w, scale, m, d, p, y, stream); });
    });
}

// (context, device, X, heads, pos, rope, Y, stream)
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 8, [&] {
        const int device = whole(a[1]), heads = whole(a[3]);
        const at::Tensor& x = tensor(a[2], "X");
        if (x.dim() != 2) refuse("X", "float, bfloat16 or half", &x, 0, 0, device);
        const int code = code_of(x, "X");
        const int64_t rows = x.size(0), width = x.size(1);
        if (rows > INT_MAX || width > INT_MAX) return (int)GELO_ERR_UNSUPPORTED;
        if (heads < 1 || width % heads) throw Refused{"the width of X must be a multiple of heads"};
        const Rows X = rows_of(a[2], "X", x.scalar_type(), rows, width, device);
        const Rows Y = a[6] == Py_None ? X : rows_of(a[6], "Y", x.scalar_type(), rows, width, device);
        const int* pos = values_of<int>(a[4], "pos", at::kInt, rows, device);
        gelo_ctx* const ctx = context(a[0]);
        const gelo_rope* const rope = struct_at<gelo_rope>(a[5]);
        void* const stream = stream_of(a[7], device);
        return unlocked([&] { return gelo_rotary(ctx, X.at, X.ld, (int)rows, heads, (int)(width / heads), pos, rope, code, Y.at, Y.ld, stream); });
    });
}

// (context, device, cache, K, V, pos, seq, rope, Q, Q_out, stream)
PyObject* append_kv(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 11, [&] {
        const int device = whole(a[1]);
        const gelo_kv_cache* cache = struct_at<gelo_kv_cache>(a[2]);
        if (!cache) return (int)GELO_ERR_INVALID;
        const at::Tensor& k = tensor(a[3], "K");
        const int code = code_of(k, "K");
        const at::ScalarType type = k.scalar_type();
        const int64_t rows = k.dim() ? k.size(0) : 0, width = (int64_t)cache->kv_heads * cache->head_dim;
        if (rows > INT_MAX) return (int)GELO_ERR_UNSUPPORTED;
        const Rows K = rows_of(a[3], "K", type, rows, width, device), V = rows_of(a[4], "V", type, rows, width, device);
        Rows Q, O;
        int heads = 0;
        if (a[8] != Py_None) {
            const at::Tensor& q = tensor(a[8], "Q");
            const int64_t wide = q.dim() == 2 ? q.size(1) : 0;
            if (wide < 1 || wide % cache->head_dim || wide > INT_MAX) throw Refused{"the width of Q must be a multiple of head_dim"};
            heads = (int)(wide / cache->head_dim);
            Q = rows_of(a[8], "Q", type, rows, wide, device);
            O = a[9] == Py_None ? Q : rows_of(a[9], "Q_out", type, rows, wide, device);
        } else if (a[9] != Py_None) {
            throw Refused{"Q_out without Q"};
        }
        const int* seq = values_of<int>(a[6], "seq", at::kInt, rows, device, true);
        const int* pos = values_of<int>(a[5], "pos", at::kInt, rows, device);
        gelo_ctx* const ctx = context(a[0]);
        const gelo_rope* const rope = struct_at<gelo_rope>(a[7]);
        void* const stream = stream_of(a[10], device);
        return unlocked([&] { return gelo_append_kv(ctx, cache, K.at, K.ld, V.at, V.ld, Q.at, Q.ld, heads, (int)rows, seq, pos, rope, code, O.at, O.ld, stream); });
    });
}

// (context, device, cache, Q, lengths, O, scale, window, lse, stream)
PyObject* paged_attention(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 10, [&] {
        const int device = whole(a[1]);
        const gelo_kv_cache* cache = struct_at<gelo_kv_cache>(a[2]);
        if (!cache) return (int)GELO_ERR_INVALID;
        const at::Tensor& q = tensor(a[3], "Q");
        const int code = code_of(q, "Q");
        const int64_t rows = cache->seqs, width = q.dim() == 2 ? q.size(1) : 0;
        if (width < 1 || width % cache->head_dim || width > INT_MAX) throw Refused{"the width of Q must be a multiple of head_dim"};
        const int heads = (int)(width / cache->head_dim);
        const Rows Q = rows_of(a[3], "Q", q.scalar_type(), rows, width, device), O = rows_of(a[5], "O", q.scalar_type(), rows, width, device);
        const int* lengths = values_of<int>(a[4], "lengths", at::kInt, rows, device);
        float* const lse = values_of<float>(a[8], "lse", at::kFloat, rows * heads, device, true);
        gelo_ctx* const ctx = context(a[0]);
        const float scale = number(a[6]);
        const int window = whole(a[7]);
        void* const stream = stream_of(a[9], device);
        return unlocked([&] { return gelo_paged_attention(ctx, cache, Q.at, Q.ld, heads, lengths, scale, window, code, O.at, O.ld, lse, stream); });
    });
}

PyMethodDef methods[] = {
    {"rms_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rms_norm)), METH_FASTCALL, nullptr},
    {"project_e4m3_rows", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(project_e4m3_rows)), METH_FASTCALL, nullptr},
    {"rotary", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rotary)), METH_FASTCALL, nullptr},
    {"append_kv", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(append_kv)), METH_FASTCALL, nullptr},
    {"paged_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_attention)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Marshalling of tensors for libgelo.so", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
