// The calls of binding.py whose launch takes the device no longer than Python takes to make it, as one native call each:
// arguments unpacked, outputs allocated by torch's allocator, the library's entry point called.  No arithmetic.
//
// A layer of one image (197 x 768 -> 768) is 3.5 us of device time.  Through ctypes a call took 8.6 us of host time: 2.5 in
// the library, 1.3 in the conversion of 15 arguments, 1.8 for the output tensor, the rest Python; four levels of a
// 3072 x 768 weight took 20.7, half of it views of the two allocations.
//
// Every function returns its result, or the entry point's status as an int when that is not ELSA_OK (binding.py raises).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cmath>
#include <initializer_list>
#include <string>

#include <ATen/ATen.h>
#include <ATen/EmptyTensor.h>
#include <c10/core/impl/DeviceGuardImplInterface.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "elsa.h"

namespace {

decltype(&elsa_nm_linear) g_linear;
decltype(&elsa_nm_linear_masked) g_linear_masked;
decltype(&elsa_nm_linear_i8) g_linear_i8;
decltype(&elsa_nm_linear_backward) g_backward;
decltype(&elsa_nm_compress) g_compress;
decltype(&elsa_nm_compress_levels) g_compress_levels;
decltype(&elsa_nm_values_bytes) g_values_bytes;
decltype(&elsa_nm_index_bytes) g_index_bytes;
decltype(&elsa_workspace_bytes) g_workspace_bytes;
decltype(&elsa_workspace_bytes_i8) g_workspace_bytes_i8;
decltype(&elsa_backward_workspace_bytes) g_backward_workspace_bytes;
decltype(&elsa_layer_norm) g_layer_norm;
decltype(&elsa_layer_norm_backward) g_layer_norm_backward;
decltype(&elsa_layer_norm_backward_workspace_bytes) g_layer_norm_backward_workspace_bytes;
decltype(&elsa_rotary) g_rotary;
decltype(&elsa_packed_attention) g_packed;
decltype(&elsa_packed_attention_backward) g_packed_backward;
decltype(&elsa_packed_attention_workspace_bytes) g_packed_workspace_bytes;

// What a conversion found wrong; the Python error is set.
struct Raised {};

const at::Tensor& tensor(PyObject* o)
{
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "tensor expected, got %s", Py_TYPE(o)->tp_name);
        throw Raised();
    }
    return THPVariable_Unpack(o);
}

void* pointer(const at::Tensor& t)
{
    if (!t.is_contiguous()) {
        PyErr_SetString(PyExc_ValueError, "contiguous tensor expected");
        throw Raised();
    }
    return t.data_ptr();
}

void* pointer(PyObject* o) { return o == Py_None ? nullptr : pointer(tensor(o)); }

int integer(PyObject* o)
{
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised();
    return (int)v;
}

void* handle(PyObject* o)
{
    if (o == Py_None) return nullptr;
    void* p = PyLong_AsVoidPtr(o);
    if (p == nullptr && PyErr_Occurred()) throw Raised();
    return p;
}

int64_t size_at(const at::Tensor& t, int64_t dim)
{
    if (dim >= t.dim()) {
        PyErr_SetString(PyExc_IndexError, "tensor has too few dimensions");
        throw Raised();
    }
    return t.size(dim);
}

// A tensor read as a matrix: a third dimension would be dropped without a word.
const at::Tensor& matrix(PyObject* o)
{
    const at::Tensor& t = tensor(o);
    if (t.dim() != 2) {
        PyErr_Format(t.dim() < 2 ? PyExc_IndexError : PyExc_ValueError, "tensor of two dimensions expected, got %d", (int)t.dim());
        throw Raised();
    }
    return t;
}

// A new tensor of this shape beside `like`.  On the current GPU straight from torch's current CUDA allocator (the one that
// torch.cuda.memory.change_current_allocator puts in place; c10::GetAllocator keeps the built-in one): by way of at::empty's dispatch
// eight outputs, four levels of a weight, were most of the call (3072 x 768 11.5 us with it, 9.4 without).  What at::empty
// does besides is left to it: another device, filled memory, and whatever takes part in a call on this thread beyond the ordinary
// (dispatch modes, functional transforms, tracing), which shows as a dispatch key included.
at::Tensor fresh(const at::Tensor& like, at::IntArrayRef shape, at::ScalarType type)
{
    const c10::Device device = like.device();
    const at::Context& context = at::globalContext();
    if (device.is_cuda() && c10::impl::getDeviceGuardImpl(c10::DeviceType::CUDA)->getDevice() == device &&
        (c10::impl::tls_local_dispatch_key_set().included_ - c10::default_included_set).empty() && !(context.deterministicAlgorithms() && context.deterministicFillUninitializedMemory()))
        return at::detail::empty_generic(shape, c10::cuda::CUDACachingAllocator::get(), c10::DispatchKeySet(c10::DispatchKey::CUDA), type, std::nullopt);
    return at::empty(shape, like.options().dtype(type));
}

// The given tensor, or a new one of this shape beside `like`.
at::Tensor given_or_new(PyObject* o, const at::Tensor& like, at::IntArrayRef shape, at::ScalarType type)
{
    return o != Py_None ? tensor(o) : fresh(like, shape, type);
}

// A workspace of at least `bytes`.
at::Tensor workspace(PyObject* o, const at::Tensor& like, size_t bytes)
{
    return given_or_new(o, like, {(int64_t)(bytes < 256 ? 256 : bytes)}, at::kByte);
}

PyObject* result_or_status(elsa_status st, const at::Tensor& t)
{
    return st == ELSA_OK ? THPVariable_Wrap(t) : PyLong_FromLong((long)st);
}

// C++ exceptions (torch's among them) become Python errors; n: the arguments expected.
template <typename F>
PyObject* guarded(Py_ssize_t got, Py_ssize_t n, F f)
{
    if (got != n) return PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", n, got);
    try {
        return f();
    } catch (const Raised&) {
        return nullptr;
    } catch (const c10::Error& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// The entry point without the interpreter's lock.
template <typename F>
elsa_status unlocked(F f)
{
    elsa_status st;
    Py_BEGIN_ALLOW_THREADS
    st = f();
    Py_END_ALLOW_THREADS
    return st;
}

// X, vals, idx, bias, out, in, N, M, dtype code, Y, workspace, dev_status, stream
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 13, [&] {
        const at::Tensor& X = tensor(a[0]);
        const int rows = (int)size_at(X, 0), out = integer(a[4]), in = integer(a[5]), N = integer(a[6]), M = integer(a[7]);
        const elsa_dtype code = (elsa_dtype)integer(a[8]);
        const at::Tensor Y = given_or_new(a[9], X, {rows, out}, X.scalar_type());
        const at::Tensor ws = workspace(a[10], X, a[10] == Py_None ? g_workspace_bytes(rows, in, out, N, M, code) : 0);
        void *x = pointer(X), *vals = pointer(a[1]), *idx = pointer(a[2]), *bias = pointer(a[3]), *y = pointer(Y), *w = pointer(ws),
             *status = pointer(a[11]), *stream = handle(a[12]);
        const size_t bytes = (size_t)ws.numel();
        return result_or_status(unlocked([&] {
            return g_linear(x, rows, vals, (const uint32_t*)idx, bias, out, in, N, M, code, y, w, bytes, (uint32_t*)status, stream);
        }), Y);
    });
}

// X, W, bias, N, M, dtype code, Y, workspace, dev_status, stream
PyObject* linear_masked(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 10, [&] {
        const at::Tensor &X = matrix(a[0]), &W = matrix(a[1]);
        const int rows = (int)size_at(X, 0), in = (int)size_at(X, 1), out = (int)size_at(W, 0), N = integer(a[3]), M = integer(a[4]);
        const elsa_dtype code = (elsa_dtype)integer(a[5]);
        const at::Tensor Y = given_or_new(a[6], X, {rows, out}, X.scalar_type());
        const at::Tensor ws = workspace(a[7], X, a[7] == Py_None ? g_workspace_bytes(rows, in, out, N, M, code) : 0);
        void *x = pointer(X), *wm = pointer(W), *bias = pointer(a[2]), *y = pointer(Y), *w = pointer(ws), *status = pointer(a[8]),
             *stream = handle(a[9]);
        const size_t bytes = (size_t)ws.numel();
        return result_or_status(unlocked([&] {
            return g_linear_masked(x, rows, wm, bias, out, in, N, M, code, y, w, bytes, (uint32_t*)status, stream);
        }), Y);
    });
}

// X, x_scale, vals, idx, w_scale, bias, out, in, N, M, dtype code of Y, dev_status, stream
PyObject* linear_i8(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 13, [&] {
        const at::Tensor& X = tensor(a[0]);
        const double x_scale = PyFloat_AsDouble(a[1]);
        if (x_scale == -1.0 && PyErr_Occurred()) throw Raised();
        const int rows = (int)size_at(X, 0), out = integer(a[6]), in = integer(a[7]), N = integer(a[8]), M = integer(a[9]), code = integer(a[10]);
        const at::Tensor Y = fresh(X, {rows, out}, code == ELSA_BF16 ? at::kBFloat16 : at::kHalf);
        const size_t need = g_workspace_bytes_i8(out, in, N, M);
        at::Tensor ws;
        if (need > 0) ws = workspace(Py_None, X, need);
        void *x = pointer(X), *vals = pointer(a[2]), *idx = pointer(a[3]), *scale = pointer(a[4]), *bias = pointer(a[5]), *y = pointer(Y),
             *w = need > 0 ? ws.data_ptr() : nullptr, *status = pointer(a[11]), *stream = handle(a[12]);
        return result_or_status(unlocked([&] {
            return g_linear_i8((const int8_t*)x, rows, (float)x_scale, (const int8_t*)vals, (const uint32_t*)idx, (const float*)scale, bias, out,
                               in, N, M, (elsa_dtype)code, y, w, need, (uint32_t*)status, stream);
        }), Y);
    });
}

// dY, X, vals, idx, out, in, N, M, dtype code, dX wanted, dW wanted, db wanted, workspace, dev_status, stream -> (dX, dW, db)
PyObject* linear_backward(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 15, [&]() -> PyObject* {
        const at::Tensor& dY = tensor(a[0]);
        const int rows = (int)size_at(dY, 0), out = integer(a[4]), in = integer(a[5]), N = integer(a[6]), M = integer(a[7]);
        const elsa_dtype code = (elsa_dtype)integer(a[8]);
        at::Tensor grad[3];
        const int64_t shape[3][2] = {{rows, in}, {out, in}, {out, 1}};
        void* g[3] = {nullptr, nullptr, nullptr};
        for (int i = 0; i < 3; ++i) {
            const int wanted = PyObject_IsTrue(a[9 + i]);
            if (wanted < 0) throw Raised();
            if (!wanted) continue;
            grad[i] = fresh(dY, at::IntArrayRef(shape[i], i == 2 ? 1 : 2), dY.scalar_type());
            g[i] = grad[i].data_ptr();
        }
        const at::Tensor ws = workspace(a[12], dY, a[12] == Py_None ? g_backward_workspace_bytes(rows, in, out, N, M, code) : 0);
        void *dy = pointer(dY), *x = pointer(a[1]), *vals = pointer(a[2]), *idx = pointer(a[3]), *w = pointer(ws), *status = pointer(a[13]),
             *stream = handle(a[14]);
        const size_t bytes = (size_t)ws.numel();
        const elsa_status st = unlocked([&] {
            return g_backward(dy, x, rows, vals, (const uint32_t*)idx, out, in, N, M, code, g[0], g[1], g[2], w, bytes, (uint32_t*)status, stream);
        });
        if (st != ELSA_OK) return PyLong_FromLong((long)st);
        PyObject* r = PyTuple_New(3);
        for (int i = 0; r != nullptr && i < 3; ++i) {
            PyObject* t = g[i] != nullptr ? THPVariable_Wrap(grad[i]) : Py_NewRef(Py_None);
            if (t == nullptr) { Py_DECREF(r); return nullptr; }
            PyTuple_SET_ITEM(r, i, t);
        }
        return r;
    });
}

// (vals, idx) of one level, idx None where there are no index words.
PyObject* packed_pair(const at::Tensor& vals, const at::Tensor& idx)
{
    PyObject* v = THPVariable_Wrap(vals);
    PyObject* i = v == nullptr ? nullptr : idx.defined() ? THPVariable_Wrap(idx) : Py_NewRef(Py_None);
    PyObject* r = i == nullptr ? nullptr : PyTuple_Pack(2, v, i);
    Py_XDECREF(v);
    Py_XDECREF(i);
    return r;
}

// W, N, M, dtype code, stream -> (vals, idx)
PyObject* compress(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 5, [&]() -> PyObject* {
        const at::Tensor& W = matrix(a[0]);
        const int out = (int)size_at(W, 0), in = (int)size_at(W, 1), N = integer(a[1]), M = integer(a[2]);
        const elsa_dtype code = (elsa_dtype)integer(a[3]);
        void *w = pointer(W), *stream = handle(a[4]);
        at::Tensor vals, idx;
        if (g_values_bytes(out, in, N, M, code) != 0) {            // otherwise the entry point says what is wrong
            vals = fresh(W, {out, (int64_t)(in / M) * N}, W.scalar_type());
            const int64_t words = (int64_t)(g_index_bytes(out, in, N, M) / 4);
            if (words > 0) idx = fresh(W, {out, words / out}, at::kInt);
        }
        void *v = vals.defined() ? vals.data_ptr() : nullptr, *i = idx.defined() ? idx.data_ptr() : nullptr;
        const elsa_status st = unlocked([&] { return g_compress(w, out, in, N, M, code, v, (uint32_t*)i, stream); });
        if (st != ELSA_OK) return PyLong_FromLong((long)st);
        return packed_pair(vals, idx);
    });
}

// W, list of N, M, dtype code, stream -> [(vals, idx), ...]; the levels are valid (binding.py checks)
PyObject* compress_levels(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 5, [&]() -> PyObject* {
        constexpr int kMost = 16;
        const at::Tensor& W = matrix(a[0]);
        const int64_t out = size_at(W, 0), in = size_at(W, 1);
        const int M = integer(a[2]);
        const elsa_dtype code = (elsa_dtype)integer(a[3]);
        if (!PyList_Check(a[1]) || PyList_GET_SIZE(a[1]) > kMost) {
            PyErr_Format(PyExc_ValueError, "a list of at most %d levels expected", kMost);
            throw Raised();
        }
        const int levels = (int)PyList_GET_SIZE(a[1]);
        int N[kMost];
        void* v[kMost];
        uint32_t* x[kMost];
        at::Tensor vals[kMost], idx[kMost];
        for (int l = 0; l < levels; ++l) {
            N[l] = integer(PyList_GET_ITEM(a[1], l));
            vals[l] = fresh(W, {out, in / M * N[l]}, W.scalar_type());
            const int64_t words = (int64_t)(g_index_bytes((int)out, (int)in, N[l], M) / 4);
            if (words > 0) idx[l] = fresh(W, {out, words / out}, at::kInt);
            v[l] = vals[l].data_ptr();
            x[l] = words > 0 ? (uint32_t*)idx[l].data_ptr() : nullptr;
        }
        void *w = pointer(W), *stream = handle(a[4]);
        const elsa_status st = unlocked([&] { return g_compress_levels(w, (int)out, (int)in, M, N, levels, code, v, x, stream); });
        if (st != ELSA_OK) return PyLong_FromLong((long)st);
        PyObject* r = PyList_New(levels);
        for (int l = 0; r != nullptr && l < levels; ++l) {
            PyObject* p = packed_pair(vals[l], idx[l]);
            if (p == nullptr) { Py_DECREF(r); return nullptr; }
            PyList_SET_ITEM(r, l, p);
        }
        return r;
    });
}

// ---- LayerNorm, rotary positions and packed attention: their calls are checked here, types first, then places, then shapes (a call
// of one image, 4 to 10 us of device time, took 9.6 to 20 us with the same checks in Python).

[[noreturn]] void raise(PyObject* type, const char* fmt, const char* a, const char* b)
{
    PyErr_Format(type, fmt, a, b);
    throw Raised();
}

elsa_dtype type_code(const at::Tensor& t)
{
    if (t.scalar_type() == at::kHalf) return ELSA_F16;
    if (t.scalar_type() == at::kBFloat16) return ELSA_BF16;
    raise(PyExc_TypeError, "fp16 or bf16 expected, got %s%s", c10::toString(t.scalar_type()), "");
}

// An argument that may be None.
const at::Tensor* maybe(PyObject* o) { return o == Py_None ? nullptr : &tensor(o); }

void same_type(const at::Tensor& like, std::initializer_list<const at::Tensor*> others)
{
    for (const at::Tensor* t : others)
        if (t != nullptr && t->scalar_type() != like.scalar_type())
            raise(PyExc_TypeError, "%s expected, got %s", c10::toString(like.scalar_type()), c10::toString(t->scalar_type()));
}

// The library launches on the current device: every tensor of a call has to be there.
void same_place(std::initializer_list<const at::Tensor*> all)
{
    const c10::impl::DeviceGuardImplInterface* cuda = nullptr;
    c10::Device here(c10::DeviceType::CPU);
    for (const at::Tensor* t : all) {
        if (t == nullptr) continue;
        if (!t->is_cuda()) raise(PyExc_ValueError, "CUDA tensor expected, got one on %s%s", t->device().str().c_str(), "");
        if (cuda == nullptr) {
            cuda = c10::impl::getDeviceGuardImpl(c10::DeviceType::CUDA);
            here = cuda->getDevice();
        }
        if (t->device() != here) raise(PyExc_ValueError, "tensor on %s, the current device is %s", t->device().str().c_str(), here.str().c_str());
    }
}

// "[4, 64]"; by hand, for a string stream of this module ends a process with the GPU's driver in it.
std::string text(at::IntArrayRef shape)
{
    std::string r = "[";
    for (size_t i = 0; i < shape.size(); ++i) r += (i > 0 ? ", " : "") + std::to_string((long long)shape[i]);
    return r + "]";
}

// Rows and columns as ints, which the entry points take; they say what else is too many.
void sizes_fit(const at::Tensor& t, const char* name)
{
    if (t.size(0) > 0x7fffffff || t.size(1) > 0x7fffffff) raise(PyExc_ValueError, "%s: shape %s does not fit an int", name, text(t.sizes()).c_str());
}

void shape_is(const at::Tensor* t, at::IntArrayRef want, const char* name)
{
    if (t != nullptr && t->sizes() != want)
        raise(PyExc_ValueError, "%s: shape %s", name, (text(want) + " expected, got " + text(t->sizes())).c_str());
}

void floats(const at::Tensor* t, at::IntArrayRef want, const char* name, bool needed)
{
    if (t == nullptr && !needed) return;
    if (t == nullptr || t->scalar_type() != at::kFloat || t->sizes() != want)
        raise(PyExc_ValueError, "%s: fp32 %s expected", name, text(want).c_str());
}

void* address(const at::Tensor* t) { return t == nullptr ? nullptr : pointer(*t); }

// The given stream's handle, or the current stream's.
void* stream_of(PyObject* o) { return o == Py_None ? (void*)c10::cuda::getCurrentCUDAStream().stream() : handle(o); }

// While it lives the given stream is torch's current one, so that what a call allocates belongs to the stream that it runs on: a block of
// another stream's could still be in use there, and would go back to it while this call runs.
struct OnStream {
    c10::cuda::OptionalCUDAStreamGuard guard;
    OnStream(PyObject* o, const at::Tensor& t)
    {
        if (o != Py_None) guard.reset_stream(c10::cuda::getStreamFromExternal((cudaStream_t)handle(o), t.device().index()));
    }
};

// A matrix whose rows are contiguous, such as the columns of one third of qkv: its address and the values between rows.
struct Rows {
    void* at;
    long long pitch;
};
Rows rows_of(const at::Tensor& t, const char* name)
{
    if (t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1)) raise(PyExc_ValueError, "%s: a matrix with contiguous rows expected%s", name, "");
    const long long width = (t.size(1) + 7) / 8 * 8;
    return {t.data_ptr(), t.size(0) > 1 || t.stride(0) > width ? t.stride(0) : width};
}

bool truth(PyObject* o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Raised();
    return v != 0;
}

double real(PyObject* o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised();
    return v;
}

// What is handed back for a tensor: the caller's own object where it gave one, None where there is none.
PyObject* handed(PyObject* given, const at::Tensor& t)
{
    return given != Py_None ? Py_NewRef(given) : t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None);
}

template <size_t kN>
PyObject* tuple_of(PyObject* const (&items)[kN])
{
    PyObject* r = PyTuple_New(kN);
    bool ok = r != nullptr;
    for (size_t i = 0; i < kN; ++i) {
        ok = ok && items[i] != nullptr;
        if (r != nullptr) PyTuple_SET_ITEM(r, i, items[i]);
        else Py_XDECREF(items[i]);
    }
    if (!ok) Py_CLEAR(r);
    return r;
}

// x, gain, bias, eps, residual, stats wanted, y, s, stats, stream -> (y, s, stats)
PyObject* layer_norm(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 10, [&]() -> PyObject* {
        const at::Tensor &x = matrix(a[0]), &gain = tensor(a[1]), &bias = tensor(a[2]);
        const at::Tensor *residual = maybe(a[4]), *y_in = maybe(a[6]), *s_in = maybe(a[7]), *stats_in = maybe(a[8]);
        const elsa_dtype code = type_code(x);
        same_type(x, {&gain, &bias, residual, y_in, s_in});
        same_place({&x, &gain, &bias, residual, y_in, s_in, stats_in});
        const OnStream on(a[9], x);
        const int64_t rows = x.size(0), dim = x.size(1);
        sizes_fit(x, "x");
        shape_is(&gain, {dim}, "gain");
        shape_is(&bias, {dim}, "bias");
        shape_is(residual, {rows, dim}, "residual");
        shape_is(y_in, {rows, dim}, "y");
        shape_is(s_in, {rows, dim}, "s");
        floats(stats_in, {rows, 2}, "stats", false);
        if (residual == nullptr && s_in != nullptr) raise(PyExc_ValueError, "s is written where there is a residual%s%s", "", "");
        at::Tensor y = y_in ? *y_in : fresh(x, {rows, dim}, x.scalar_type()), s, stats;
        if (residual != nullptr) s = s_in ? *s_in : fresh(x, {rows, dim}, x.scalar_type());
        if (stats_in != nullptr) stats = *stats_in;
        else if (truth(a[5])) stats = fresh(x, {rows, 2}, at::kFloat);
        void *xp = pointer(x), *rp = address(residual), *gp = pointer(gain), *bp = pointer(bias), *yp = pointer(y),
             *sp = s.defined() ? pointer(s) : nullptr, *tp = stats.defined() ? pointer(stats) : nullptr, *stream = stream_of(a[9]);
        const float eps = (float)real(a[3]);
        const elsa_status st = unlocked([&] { return g_layer_norm(xp, rp, gp, bp, (int)rows, (int)dim, eps, code, sp, yp, (float*)tp, stream); });
        if (st != ELSA_OK) return PyLong_FromLong((long)st);
        return tuple_of({handed(a[6], y), residual == nullptr ? Py_NewRef(a[0]) : handed(a[7], s), handed(a[8], stats)});
    });
}

// dy, s, gain, stats, ds, dx wanted, dgain wanted, dbias wanted, dx, workspace, stream -> (dx, dgain, dbias)
PyObject* layer_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 11, [&]() -> PyObject* {
        const at::Tensor &dy = matrix(a[0]), &s = tensor(a[1]), &gain = tensor(a[2]);
        const at::Tensor *stats = maybe(a[3]), *ds = maybe(a[4]), *dx_in = maybe(a[8]), *ws_in = maybe(a[9]);
        const elsa_dtype code = type_code(dy);
        same_type(dy, {&s, &gain, ds, dx_in});
        same_place({&dy, &s, &gain, stats, ds, dx_in, ws_in});
        const OnStream on(a[10], dy);
        const int64_t rows = dy.size(0), dim = dy.size(1);
        sizes_fit(dy, "dy");
        shape_is(&s, {rows, dim}, "s");
        shape_is(ds, {rows, dim}, "ds");
        shape_is(dx_in, {rows, dim}, "dx");
        shape_is(&gain, {dim}, "gain");
        floats(stats, {rows, 2}, "stats", true);
        const bool want[3] = {truth(a[5]), truth(a[6]), truth(a[7])};
        at::Tensor grad[3], ws;
        if (want[0]) grad[0] = dx_in ? *dx_in : fresh(dy, {rows, dim}, dy.scalar_type());
        for (int i = 1; i < 3; ++i)
            if (want[i]) grad[i] = fresh(dy, {dim}, dy.scalar_type());
        if (want[1] || want[2]) ws = workspace(a[9], dy, g_layer_norm_backward_workspace_bytes((int)rows, (int)dim));
        void* g[3];
        for (int i = 0; i < 3; ++i) g[i] = grad[i].defined() ? pointer(grad[i]) : nullptr;
        void *dyp = pointer(dy), *sp = pointer(s), *tp = pointer(*stats), *gp = pointer(gain), *dsp = address(ds),
             *w = ws.defined() ? pointer(ws) : nullptr, *stream = stream_of(a[10]);
        const size_t bytes = ws.defined() ? (size_t)ws.nbytes() : 0;
        const elsa_status st = unlocked([&] {
            return g_layer_norm_backward(dyp, sp, (const float*)tp, gp, dsp, (int)rows, (int)dim, code, g[0], g[1], g[2], w, bytes, stream);
        });
        if (st != ELSA_OK) return PyLong_FromLong((long)st);
        return tuple_of({handed(want[0] ? a[8] : Py_None, grad[0]), handed(Py_None, grad[1]), handed(Py_None, grad[2])});
    });
}

// x, positions, address of the plan, y, inverse, stream -> y
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 6, [&]() -> PyObject* {
        const at::Tensor &x = matrix(a[0]), &positions = tensor(a[1]);
        const at::Tensor* y_in = maybe(a[3]);
        const elsa_rotary_plan* plan = (const elsa_rotary_plan*)handle(a[2]);
        const elsa_dtype code = type_code(x);
        same_type(x, {y_in});
        if (positions.scalar_type() != at::kInt) raise(PyExc_TypeError, "positions: int32 expected, got %s%s", c10::toString(positions.scalar_type()), "");
        same_place({&x, &positions, y_in});
        const OnStream on(a[5], x);
        const int64_t rows = x.size(0), width = x.size(1);
        sizes_fit(x, "x");
        if (plan == nullptr || plan->head_dim <= 0 || width == 0 || width % plan->head_dim != 0) raise(PyExc_ValueError, "x: its columns are no heads of the plan's%s%s", "", "");
        shape_is(&positions, {rows, plan->axes}, "positions");
        shape_is(y_in, {rows, width}, "y");
        const at::Tensor y = y_in ? *y_in : fresh(x, {rows, width}, x.scalar_type());
        const Rows xr = rows_of(x, "x"), yr = rows_of(y, "y");
        void *pp = pointer(positions), *stream = stream_of(a[5]);
        const bool inverse = truth(a[4]);
        const elsa_status st = unlocked([&] {
            return g_rotary(xr.at, xr.pitch, (const int32_t*)pp, plan, (int)rows, (int)(width / plan->head_dim), inverse ? 1 : 0, code, yr.at, yr.pitch, stream);
        });
        return st == ELSA_OK ? handed(a[3], y) : PyLong_FromLong((long)st);
    });
}

// q, k, v and what is beside them in a packed call: plan buffer, rows, sequences, heads, kv_heads, causal, scale or None
struct Packed {
    elsa_packed_qkv in;
    elsa_dtype code;
    int64_t rows, wide, narrow;
    const at::Tensor *q, *plan;
    int sequences;
    bool full;
};

Packed packed_call(PyObject* const* a)
{
    Packed p;
    const at::Tensor &q = matrix(a[0]), &k = matrix(a[1]), &v = matrix(a[2]);
    p.q = &q;
    p.plan = &tensor(a[3]);
    p.rows = integer(a[4]);
    p.sequences = integer(a[5]);
    p.full = truth(a[6]);
    const int heads = integer(a[7]), kv_heads = integer(a[8]);
    p.code = type_code(q);
    same_type(q, {&k, &v});
    same_place({&q, &k, &v, p.plan});
    if (heads <= 0 || kv_heads <= 0 || q.size(1) % heads != 0) raise(PyExc_ValueError, "q: its columns are no heads of that number%s%s", "", "");
    sizes_fit(q, "q");
    const int64_t width = q.size(1) / heads;
    p.wide = q.size(1);
    p.narrow = width * kv_heads;
    shape_is(&q, {p.rows, p.wide}, "q");
    shape_is(&k, {p.rows, p.narrow}, "k");
    shape_is(&v, {p.rows, p.narrow}, "v");
    const Rows qr = rows_of(q, "q"), kr = rows_of(k, "k"), vr = rows_of(v, "v");
    p.in = {qr.at, kr.at, vr.at, qr.pitch, kr.pitch, vr.pitch, (int)p.rows, heads, kv_heads, (int)width, truth(a[9]) ? 1 : 0,
            a[10] == Py_None ? 1.0f / std::sqrt((float)width) : (float)real(a[10])};
    return p;
}

// Rows of no sequence are left as they are: where there may be some, an output of the call's own starts as zeros.
at::Tensor output(const Packed& p, const at::Tensor* given, at::IntArrayRef shape, at::ScalarType type)
{
    if (given != nullptr) return *given;
    return p.full ? fresh(*p.q, shape, type) : at::zeros(shape, p.q->options().dtype(type));
}

// the eleven of packed_call, a, lse wanted, lse, dev_status, stream -> (a, lse)
PyObject* packed_attention(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 16, [&]() -> PyObject* {
        const at::Tensor *a_in = maybe(a[11]), *lse_in = maybe(a[13]), *status = maybe(a[14]);
        const Packed p = packed_call(a);
        same_type(*p.q, {a_in});
        same_place({a_in, lse_in, status});
        shape_is(a_in, {p.rows, p.wide}, "a");
        floats(lse_in, {p.in.heads, p.rows}, "lse", false);
        const OnStream on(a[15], *p.q);
        const at::Tensor out = output(p, a_in, {p.rows, p.wide}, p.q->scalar_type());
        at::Tensor lse;
        if (lse_in != nullptr || truth(a[12])) lse = output(p, lse_in, {p.in.heads, p.rows}, at::kFloat);
        const Rows ar = rows_of(out, "a");
        void *plan = pointer(*p.plan), *lp = lse.defined() ? pointer(lse) : nullptr, *sp = address(status), *stream = stream_of(a[15]);
        const elsa_status st = unlocked([&] { return g_packed(&p.in, p.code, plan, p.sequences, ar.at, ar.pitch, (float*)lp, (uint32_t*)sp, stream); });
        if (st != ELSA_OK) return PyLong_FromLong((long)st);
        return tuple_of({handed(a[11], out), handed(a[13], lse)});
    });
}

// the eleven of packed_call, da, a, lse, dq, dk, dv, workspace, dev_status, stream -> (dq, dk, dv)
PyObject* packed_attention_backward(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 20, [&]() -> PyObject* {
        const at::Tensor &da = tensor(a[11]), &out = tensor(a[12]);
        const at::Tensor *lse = maybe(a[13]), *ws_in = maybe(a[17]), *status = maybe(a[18]);
        const at::Tensor* grad_in[3] = {maybe(a[14]), maybe(a[15]), maybe(a[16])};
        const Packed p = packed_call(a);
        same_type(*p.q, {&da, &out, grad_in[0], grad_in[1], grad_in[2]});
        same_place({&da, &out, lse, grad_in[0], grad_in[1], grad_in[2], ws_in, status});
        shape_is(&da, {p.rows, p.wide}, "da");
        shape_is(&out, {p.rows, p.wide}, "a");
        floats(lse, {p.in.heads, p.rows}, "lse", true);
        const OnStream on(a[19], *p.q);
        at::Tensor grad[3];
        Rows g[3];
        static const char* const names[3] = {"dq", "dk", "dv"};
        for (int i = 0; i < 3; ++i) {
            const int64_t width = i == 0 ? p.wide : p.narrow;
            shape_is(grad_in[i], {p.rows, width}, names[i]);
            grad[i] = output(p, grad_in[i], {p.rows, width}, p.q->scalar_type());
            g[i] = rows_of(grad[i], names[i]);
        }
        const at::Tensor ws = workspace(a[17], *p.q, g_packed_workspace_bytes((int)p.rows, p.in.heads));
        const Rows ar = rows_of(out, "a"), dr = rows_of(da, "da");
        void *plan = pointer(*p.plan), *lp = pointer(*lse), *w = pointer(ws), *sp = address(status), *stream = stream_of(a[19]);
        const size_t bytes = (size_t)ws.nbytes();
        const elsa_status st = unlocked([&] {
            return g_packed_backward(&p.in, p.code, plan, p.sequences, ar.at, ar.pitch, (const float*)lp, dr.at, dr.pitch, g[0].at, g[0].pitch, g[1].at, g[1].pitch,
                                     g[2].at, g[2].pitch, w, bytes, (uint32_t*)sp, stream);
        });
        if (st != ELSA_OK) return PyLong_FromLong((long)st);
        return tuple_of({handed(a[14], grad[0]), handed(a[15], grad[1]), handed(a[16], grad[2])});
    });
}

// bind({name: address of the entry point})
PyObject* bind(PyObject*, PyObject* table)
{
    auto take = [&](const char* name, auto& f) {
        PyObject* o = PyDict_Check(table) ? PyDict_GetItemString(table, name) : nullptr;
        void* p = o != nullptr ? PyLong_AsVoidPtr(o) : nullptr;
        if (p == nullptr && !PyErr_Occurred()) PyErr_Format(PyExc_KeyError, "no address of %s", name);
        f = reinterpret_cast<std::remove_reference_t<decltype(f)>>(p);
        return p != nullptr;
    };
    const bool ok = take("elsa_nm_linear", g_linear) && take("elsa_nm_linear_masked", g_linear_masked) && take("elsa_nm_linear_i8", g_linear_i8) &&
                    take("elsa_nm_linear_backward", g_backward) && take("elsa_nm_compress", g_compress) &&
                    take("elsa_nm_compress_levels", g_compress_levels) && take("elsa_nm_values_bytes", g_values_bytes) &&
                    take("elsa_nm_index_bytes", g_index_bytes) && take("elsa_workspace_bytes", g_workspace_bytes) &&
                    take("elsa_workspace_bytes_i8", g_workspace_bytes_i8) && take("elsa_backward_workspace_bytes", g_backward_workspace_bytes) &&
                    take("elsa_layer_norm", g_layer_norm) && take("elsa_layer_norm_backward", g_layer_norm_backward) &&
                    take("elsa_layer_norm_backward_workspace_bytes", g_layer_norm_backward_workspace_bytes) && take("elsa_rotary", g_rotary) &&
                    take("elsa_packed_attention", g_packed) && take("elsa_packed_attention_backward", g_packed_backward) &&
                    take("elsa_packed_attention_workspace_bytes", g_packed_workspace_bytes);
    if (!ok) return nullptr;
    Py_RETURN_NONE;
}

#define ELSA_FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&name)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {ELSA_FAST(linear), ELSA_FAST(linear_masked), ELSA_FAST(linear_i8), ELSA_FAST(linear_backward), ELSA_FAST(compress),
                           ELSA_FAST(compress_levels), ELSA_FAST(layer_norm), ELSA_FAST(layer_norm_backward), ELSA_FAST(rotary),
                           ELSA_FAST(packed_attention), ELSA_FAST(packed_attention_backward), {"bind", &bind, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_elsa_host", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

#ifndef ELSA_TORCH_VERSION
#define ELSA_TORCH_VERSION ""
#endif

// torch_version: the torch whose headers this was compiled against; binding.py refuses another.
PyMODINIT_FUNC PyInit__elsa_host()
{
    PyObject* m = PyModule_Create(&g_module);
    if (m != nullptr && PyModule_AddStringConstant(m, "torch_version", ELSA_TORCH_VERSION) != 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
