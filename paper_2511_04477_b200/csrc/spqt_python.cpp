// The per-token calls of binding.py as native functions: type and shape checks, output allocation, the current
// stream and the C-ABI call of include/spqt.h, without a Python-level step in between.  Argument marshalling
// only, like the ctypes path of the other calls.
//
// Why: a decode linear runs 4 to 10 us on the device, and marshalling it through Python and ctypes took 10 to
// 12 us per call (14 converted arguments, up to three torch.empty, one current_stream object, a checked
// data_ptr per tensor), so every small call was bound by the host.  In a stream of calls, before -> now: a
// 1024 x 4096 linear 13.7 -> 5.6 us, one index list and three 5120 x 5120 products 48.2 -> 22.9 us, the sixteen
// linears of four Llama-3-8B-shaped layers 175 -> 149 us (the device's own time in all three then; with later kernels 4.4, 15.8 and
// 115 us).
#include <Python.h>

#include <cmath>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/spqt.h"

namespace {

PyObject* g_error = nullptr;   // binding.SpqtError(status, where)

struct Names {
    PyObject *codes, *scale_zero, *records, *m, *n, *bits, *group, *cuda_stream, *desc, *device_index;
} g_names;

// Leaves a call with a Python exception set.
struct Raised {};

[[noreturn]] void raise(PyObject* type, const char* fmt, const char* name)
{
    PyErr_Format(type, fmt, name);
    throw Raised();
}

void need_args(Py_ssize_t got, Py_ssize_t want)
{
    if (got != want) raise(PyExc_TypeError, "%s", "wrong number of arguments");
}

// The CUDA tensor behind a Python object, of the given type, contiguous; borrowed from `o`.
const at::Tensor& tensor_of(PyObject* o, at::ScalarType dtype, const char* name, bool contiguous = true)
{
    if (!THPVariable_Check(o)) raise(PyExc_TypeError, "%s must be a CUDA tensor", name);
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda()) raise(PyExc_TypeError, "%s must be a CUDA tensor", name);
    if (t.scalar_type() != dtype) {
        PyErr_Format(PyExc_TypeError, "%s must be %s, got %s", name, c10::toString(dtype), c10::toString(t.scalar_type()));
        throw Raised();
    }
    if (contiguous && !t.is_contiguous()) raise(PyExc_ValueError, "%s must be contiguous", name);
    return t;
}

// A tensor attribute of a packed matrix: the object keeps it alive for the call.
const at::Tensor& tensor_attr(PyObject* p, PyObject* attr, at::ScalarType dtype, const char* name)
{
    PyObject* o = PyObject_GetAttr(p, attr);
    if (!o) throw Raised();
    Py_DECREF(o);
    return tensor_of(o, dtype, name);
}

// A whole number of 32 bits: one that has more is refused, not cut.
int in_int(int64_t v, const char* name)
{
    if (v > 0x7fffffffLL) raise(PyExc_ValueError, "%s is too large", name);
    return (int)v;
}

int int_of(PyObject* o, const char* name)
{
    int beyond = 0;
    const long v = PyLong_AsLongAndOverflow(o, &beyond);
    if (v == -1 && !beyond && PyErr_Occurred()) throw Raised();
    if (beyond || v != (int)v) raise(PyExc_ValueError, "%s does not fit 32 bits", name);
    return (int)v;
}

int int_attr(PyObject* p, PyObject* attr, const char* name)
{
    PyObject* o = PyObject_GetAttr(p, attr);
    if (!o) throw Raised();
    int v;
    try {
        v = int_of(o, name);
    } catch (const Raised&) {
        Py_DECREF(o);
        throw;
    }
    Py_DECREF(o);
    return v;
}

// Distance of two rows of a matrix; of one row, whose distance to the next may be anything, its length where that is too large.
int row_stride(const at::Tensor& t, const char* name)
{
    return in_int(t.size(0) == 1 && t.stride(0) > 0x7fffffffLL ? t.size(1) : t.stride(0), name);
}

float float_of(PyObject* o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised();
    return (float)v;
}

void* stream_of(PyObject* o)
{
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
    PyObject* s = PyObject_GetAttr(o, g_names.cuda_stream);
    if (!s) throw Raised();
    void* v = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    if (!v && PyErr_Occurred()) throw Raised();
    return v;
}

// A new tensor for a call on `stream` (an argument, which may be None).  Where that is not the current stream the memory is of
// its pool, as if it were: memory of the current stream's pool may still be in use there, and would be given away again while the
// call writes it.  The current stream, on which the caller may read the result, is made known as well.
at::Tensor empty(at::IntArrayRef shape, at::ScalarType dtype, const at::Tensor& like, PyObject* stream)
{
    if (stream != Py_None) {
        const auto current = c10::cuda::getCurrentCUDAStream(like.get_device());
        const auto other = static_cast<cudaStream_t>(stream_of(stream));
        if (other != current.stream()) {
            const c10::cuda::CUDAStreamGuard guard(c10::cuda::getStreamFromExternal(other, like.get_device()));
            at::Tensor t = at::detail::empty_cuda(shape, dtype, like.device(), std::nullopt);
            if (t.numel() > 0) c10::cuda::CUDACachingAllocator::recordStream(t.storage().data_ptr(), current);
            return t;
        }
    }
    return at::detail::empty_cuda(shape, dtype, like.device(), std::nullopt);
}

// The tensor an optional argument names, or a new one.
at::Tensor given_or_empty(PyObject* o, at::IntArrayRef shape, at::ScalarType dtype, const char* name, const at::Tensor& like, PyObject* stream)
{
    return o == Py_None ? empty(shape, dtype, like, stream) : tensor_of(o, dtype, name);
}

// A tensor argument as it goes back to the caller: the object that came in, or the new tensor.
PyObject* hand_back(PyObject* given, at::Tensor t)
{
    if (given != Py_None) {
        Py_INCREF(given);
        return given;
    }
    return THPVariable_Wrap(std::move(t));
}

// A tuple that takes over its items' references.
template <class... O>
PyObject* tuple_of(O... items)
{
    PyObject* const list[] = {items...};
    bool ok = true;
    for (PyObject* o : list) ok = ok && o;
    PyObject* t = ok ? PyTuple_New(sizeof...(items)) : nullptr;
    for (size_t i = 0; i < sizeof...(items); ++i) {
        if (t) PyTuple_SET_ITEM(t, (Py_ssize_t)i, list[i]);
        else Py_XDECREF(list[i]);
    }
    return t;
}

void check(spqt_status st, const char* where)
{
    if (st == SPQT_OK) return;
    PyObject* e = PyObject_CallFunction(g_error, "is", (int)st, where);
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    throw Raised();
}

struct Zigzag {
    const void *codes, *scale_zero;
    int m, n, bits, group;
    explicit Zigzag(PyObject* p)
        : codes(tensor_attr(p, g_names.codes, at::kByte, "codes").data_ptr()),
          scale_zero(tensor_attr(p, g_names.scale_zero, at::kHalf, "scale_zero").data_ptr()),
          m(int_attr(p, g_names.m, "m")), n(int_attr(p, g_names.n, "n")), bits(int_attr(p, g_names.bits, "bits")), group(int_attr(p, g_names.group, "group"))
    {
    }
};

// Runs the library call without the GIL (a launch can wait for room in the stream's queue): `f` raises nothing.
template <class F>
void call(const char* where, F f)
{
    spqt_status st;
    Py_BEGIN_ALLOW_THREADS
    st = f();
    Py_END_ALLOW_THREADS
    check(st, where);
}

template <class F>
PyObject* guarded(F f)
{
    HANDLE_TH_ERRORS
    try {
        return f();
    } catch (const Raised&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

using Args = PyObject* const*;

// (x, t, idx, count, stream) -> (idx, count)
PyObject* sparsify(PyObject*, Args a, Py_ssize_t na)
{
    return guarded([&]() -> PyObject* {
        need_args(na, 5);
        const at::Tensor& x = tensor_of(a[0], at::kHalf, "x");
        const float t = float_of(a[1]);
        const int n = in_int(x.numel(), "the number of entries");
        at::Tensor idx = given_or_empty(a[2], {n > 0 ? n : 1}, at::kInt, "idx", x, a[4]);
        at::Tensor count = given_or_empty(a[3], {1}, at::kInt, "count", x, a[4]);
        if (idx.numel() < n) raise(PyExc_ValueError, "%s", "idx must hold n entries");
        void* s = stream_of(a[4]);
        call("spqt_sparsify", [&] { return spqt_sparsify(x.data_ptr(), n, t, (int32_t*)idx.data_ptr(), (int32_t*)count.data_ptr(), s); });
        return tuple_of(hand_back(a[2], idx), hand_back(a[3], count));
    });
}

// (p, x, idx, count, workspace, y, stream) -> y
PyObject* sparse_gemv(PyObject*, Args a, Py_ssize_t na)
{
    return guarded([&]() -> PyObject* {
        need_args(na, 7);
        const Zigzag p(a[0]);
        const at::Tensor& x = tensor_of(a[1], at::kHalf, "x");
        at::Tensor y = given_or_empty(a[5], {p.m}, at::kHalf, "y", x, a[6]);
        if (x.numel() != p.n || y.numel() != p.m) raise(PyExc_ValueError, "%s", "x must have n entries and y m entries");
        const at::Tensor& idx = tensor_of(a[2], at::kInt, "idx");
        const at::Tensor& count = tensor_of(a[3], at::kInt, "count");
        const at::Tensor& ws = tensor_of(a[4], at::kByte, "workspace");
        void* s = stream_of(a[6]);
        call("spqt_sparse_gemv", [&] {
            return spqt_sparse_gemv(p.codes, p.scale_zero, p.m, p.n, p.bits, p.group, x.data_ptr(), (const int32_t*)idx.data_ptr(),
                                    (const int32_t*)count.data_ptr(), y.data_ptr(), ws.data_ptr(), (size_t)ws.numel(), s);
        });
        return hand_back(a[5], y);
    });
}

// (p, x, t, workspace, idx, count, y, stream) -> (y, idx, count)
PyObject* sparsify_gemv(PyObject*, Args a, Py_ssize_t na)
{
    return guarded([&]() -> PyObject* {
        need_args(na, 8);
        const Zigzag p(a[0]);
        const at::Tensor& x = tensor_of(a[1], at::kHalf, "x");
        const float t = float_of(a[2]);
        const at::Tensor& ws = tensor_of(a[3], at::kByte, "workspace");
        at::Tensor idx = given_or_empty(a[4], {p.n}, at::kInt, "idx", x, a[7]);
        at::Tensor count = given_or_empty(a[5], {1}, at::kInt, "count", x, a[7]);
        at::Tensor y = given_or_empty(a[6], {p.m}, at::kHalf, "y", x, a[7]);
        if (x.numel() != p.n || y.numel() != p.m || idx.numel() < p.n)
            raise(PyExc_ValueError, "%s", "x and idx must have n entries and y m entries");
        void* s = stream_of(a[7]);
        call("spqt_sparsify_gemv", [&] {
            return spqt_sparsify_gemv(p.codes, p.scale_zero, p.m, p.n, p.bits, p.group, x.data_ptr(), t, (int32_t*)idx.data_ptr(),
                                      (int32_t*)count.data_ptr(), y.data_ptr(), ws.data_ptr(), (size_t)ws.numel(), s);
        });
        return tuple_of(hand_back(a[6], y), hand_back(a[4], idx), hand_back(a[5], count));
    });
}

// (p, x, workspace, y, stream) -> y
PyObject* dense_gemv(PyObject*, Args a, Py_ssize_t na)
{
    return guarded([&]() -> PyObject* {
        need_args(na, 5);
        const Zigzag p(a[0]);
        const at::Tensor& x = tensor_of(a[1], at::kHalf, "x");
        at::Tensor y = given_or_empty(a[3], {p.m}, at::kHalf, "y", x, a[4]);
        if (x.numel() != p.n || y.numel() != p.m) raise(PyExc_ValueError, "%s", "x must have n entries and y m entries");
        const at::Tensor& ws = tensor_of(a[2], at::kByte, "workspace");
        void* s = stream_of(a[4]);
        call("spqt_dense_gemv", [&] {
            return spqt_dense_gemv(p.codes, p.scale_zero, p.m, p.n, p.bits, p.group, x.data_ptr(), y.data_ptr(), ws.data_ptr(),
                                   (size_t)ws.numel(), s);
        });
        return hand_back(a[3], y);
    });
}

// X [batch <= 8][n] with unit column stride, and Y [batch][m], given or new
at::Tensor batch_output(const Zigzag& p, PyObject* X_o, PyObject* Y_o, PyObject* stream)
{
    if (!THPVariable_Check(X_o)) raise(PyExc_TypeError, "%s", "X and Y must be CUDA float16 tensors");
    const at::Tensor& X = THPVariable_Unpack(X_o);
    if (X.dim() != 2 || X.stride(1) != 1 || X.size(1) != p.n || X.size(0) < 1 || X.size(0) > 8)
        raise(PyExc_ValueError, "%s", "X must be [batch <= 8][n] with unit column stride");
    if (X.scalar_type() != at::kHalf || !X.is_cuda()) raise(PyExc_TypeError, "%s", "X and Y must be CUDA float16 tensors");
    if (Y_o == Py_None) return empty({X.size(0), p.m}, at::kHalf, X, stream);
    if (!THPVariable_Check(Y_o)) raise(PyExc_TypeError, "%s", "X and Y must be CUDA float16 tensors");
    const at::Tensor& Y = THPVariable_Unpack(Y_o);
    if (Y.scalar_type() != at::kHalf || !Y.is_cuda()) raise(PyExc_TypeError, "%s", "X and Y must be CUDA float16 tensors");
    if (Y.dim() != 2 || Y.size(0) != X.size(0) || Y.size(1) != p.m || Y.stride(1) != 1)
        raise(PyExc_ValueError, "%s", "Y must be [batch][m] with unit column stride");
    return Y;
}

// (p, X, t, workspace, idx, count, Y, stream) -> (Y, idx, count)
PyObject* sparse_gemm_small(PyObject*, Args a, Py_ssize_t na)
{
    return guarded([&]() -> PyObject* {
        need_args(na, 8);
        const Zigzag p(a[0]);
        at::Tensor Y = batch_output(p, a[1], a[6], a[7]);
        const at::Tensor& X = THPVariable_Unpack(a[1]);
        const int ldx = row_stride(X, "the row stride of X"), ldy = row_stride(Y, "the row stride of Y");
        const float t = float_of(a[2]);
        const at::Tensor& ws = tensor_of(a[3], at::kByte, "workspace");
        at::Tensor idx = given_or_empty(a[4], {p.n}, at::kInt, "idx", X, a[7]);
        at::Tensor count = given_or_empty(a[5], {1}, at::kInt, "count", X, a[7]);
        void* s = stream_of(a[7]);
        call("spqt_sparse_gemm_small", [&] {
            return spqt_sparse_gemm_small(p.codes, p.scale_zero, p.m, p.n, p.bits, p.group, X.data_ptr(), ldx, (int)X.size(0), t,
                                          (int32_t*)idx.data_ptr(), (int32_t*)count.data_ptr(), Y.data_ptr(), ldy, ws.data_ptr(),
                                          (size_t)ws.numel(), s);
        });
        return tuple_of(hand_back(a[6], Y), hand_back(a[4], idx), hand_back(a[5], count));
    });
}

// (p, X, workspace, Y, stream) -> Y
PyObject* dense_gemm_small(PyObject*, Args a, Py_ssize_t na)
{
    return guarded([&]() -> PyObject* {
        need_args(na, 5);
        const Zigzag p(a[0]);
        at::Tensor Y = batch_output(p, a[1], a[3], a[4]);
        const at::Tensor& X = THPVariable_Unpack(a[1]);
        const int ldx = row_stride(X, "the row stride of X"), ldy = row_stride(Y, "the row stride of Y");
        const at::Tensor& ws = tensor_of(a[2], at::kByte, "workspace");
        void* s = stream_of(a[4]);
        call("spqt_dense_gemm_small", [&] {
            return spqt_dense_gemm_small(p.codes, p.scale_zero, p.m, p.n, p.bits, p.group, X.data_ptr(), ldx, (int)X.size(0),
                                         Y.data_ptr(), ldy, ws.data_ptr(), (size_t)ws.numel(), s);
        });
        return hand_back(a[3], Y);
    });
}

// list: (p, x, idx, count, workspace, y, stream, where) -> y; over all columns: without idx and count
template <bool LIST>
PyObject* kqw_gemv(PyObject*, Args a, Py_ssize_t na)
{
    return guarded([&]() -> PyObject* {
        need_args(na, LIST ? 8 : 6);
        PyObject* p = a[0];
        const Args rest = a + (LIST ? 4 : 2);   // workspace, y, stream, where
        const void* records = tensor_attr(p, g_names.records, at::kByte, "records").data_ptr();
        const int m = int_attr(p, g_names.m, "m"), n = int_attr(p, g_names.n, "n"), bits = int_attr(p, g_names.bits, "bits");
        const at::Tensor& x = tensor_of(a[1], at::kHalf, "x");
        at::Tensor y = given_or_empty(rest[1], {m}, at::kHalf, "y", x, rest[2]);
        const at::Tensor& ws = tensor_of(rest[0], at::kByte, "workspace");
        void* s = stream_of(rest[2]);
        const char* where = PyUnicode_AsUTF8(rest[3]);
        if (!where) throw Raised();
        if (LIST) {
            const at::Tensor& idx = tensor_of(a[2], at::kInt, "idx");
            const at::Tensor& count = tensor_of(a[3], at::kInt, "count");
            call(where, [&] {
                return spqt_kqw_sparse_gemv(records, m, n, bits, x.data_ptr(), (const int32_t*)idx.data_ptr(), (const int32_t*)count.data_ptr(),
                                            y.data_ptr(), ws.data_ptr(), (size_t)ws.numel(), s);
            });
        } else {
            call(where, [&] { return spqt_kqw_dense_gemv(records, m, n, bits, x.data_ptr(), y.data_ptr(), ws.data_ptr(), (size_t)ws.numel(), s); });
        }
        return hand_back(rest[1], y);
    });
}

constexpr auto kqw_sparse_gemv = kqw_gemv<true>;
constexpr auto kqw_dense_gemv = kqw_gemv<false>;

const at::Tensor& weights_of(PyObject* o)
{
    if (!THPVariable_Check(o)) raise(PyExc_TypeError, "%s", "W must be a CUDA float16 tensor");
    const at::Tensor& W = THPVariable_Unpack(o);
    if (W.dim() != 2 || W.stride(1) != 1) raise(PyExc_ValueError, "%s", "W must be 2-D with unit column stride");
    if (!W.is_cuda() || W.scalar_type() != at::kHalf) raise(PyExc_TypeError, "%s", "W must be a CUDA float16 tensor");
    return W;
}

// (W, bits, group, stream) -> (codes, scale_zero)
PyObject* pack(PyObject*, Args a, Py_ssize_t na)
{
    return guarded([&]() -> PyObject* {
        need_args(na, 4);
        const at::Tensor& W = weights_of(a[0]);
        const int m = in_int(W.size(0), "the number of rows"), n = in_int(W.size(1), "the number of columns"), ldw = row_stride(W, "the row stride of W");
        const int bits = int_of(a[1], "bits"), group = int_of(a[2], "group");
        size_t cb = 0, sb = 0;
        check(spqt_packed_sizes(m, n, bits, group, &cb, &sb, nullptr), "spqt_packed_sizes");
        at::Tensor codes = empty({(int64_t)cb}, at::kByte, W, a[3]), sz = empty({(int64_t)(sb / 2)}, at::kHalf, W, a[3]);
        void* s = stream_of(a[3]);
        call("spqt_pack", [&] { return spqt_pack(W.data_ptr(), m, n, ldw, bits, group, codes.data_ptr(), sz.data_ptr(), s); });
        return tuple_of(hand_back(Py_None, codes), hand_back(Py_None, sz));
    });
}

// (W, bits, stream, where) -> records
PyObject* kqw_pack(PyObject*, Args a, Py_ssize_t na)
{
    return guarded([&]() -> PyObject* {
        need_args(na, 4);
        const at::Tensor& W = weights_of(a[0]);
        const int m = in_int(W.size(0), "the number of rows"), n = in_int(W.size(1), "the number of columns"), ldw = row_stride(W, "the row stride of W");
        const int bits = int_of(a[1], "bits");
        const char* where = PyUnicode_AsUTF8(a[3]);
        if (!where) throw Raised();
        size_t rb = 0;
        check(spqt_kqw_packed_sizes(m, n, bits, &rb, nullptr), "spqt_kqw_packed_sizes");
        at::Tensor records = empty({(int64_t)rb}, at::kByte, W, a[2]);
        void* s = stream_of(a[2]);
        call(where, [&] { return spqt_kqw_pack(W.data_ptr(), m, n, ldw, bits, records.data_ptr(), s); });
        return hand_back(Py_None, records);
    });
}

// (handle, stream)
PyObject* host_step_launch(PyObject*, Args a, Py_ssize_t na)
{
    return guarded([&]() -> PyObject* {
        need_args(na, 2);
        void* step = a[0] == Py_None ? nullptr : PyLong_AsVoidPtr(a[0]);
        if (!step && PyErr_Occurred()) throw Raised();
        void* s = stream_of(a[1]);
        call("spqt_host_step_launch", [&] { return spqt_host_step_launch(step, s); });
        Py_RETURN_NONE;
    });
}

// ---- the 8-bit cache and what is asked of logits

// A KVCache object: the address of its spqt_kv_cache, the device of its buffers, which is the current one for the call.
struct Cache {
    const spqt_kv_cache* c;
    int device;
    c10::cuda::OptionalCUDAGuard guard;
    explicit Cache(PyObject* p) : c(nullptr), device(int_attr(p, g_names.device_index, "device_index"))
    {
        PyObject* o = PyObject_GetAttr(p, g_names.desc);
        if (!o) throw Raised();
        c = static_cast<const spqt_kv_cache*>(PyLong_AsVoidPtr(o));
        Py_DECREF(o);
        if (!c) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "not a KVCache");
            throw Raised();
        }
        guard.set_index((c10::DeviceIndex)device);
    }
    // a tensor of the cache's device
    const at::Tensor& tensor(PyObject* o, at::ScalarType dtype, const char* name, bool contiguous = true) const
    {
        const at::Tensor& t = tensor_of(o, dtype, name, contiguous);
        if (t.get_device() != device) raise(PyExc_ValueError, "%s must be on the cache's device", name);
        return t;
    }
    void* optional(PyObject* o, at::IntArrayRef shape, const char* name) const
    {
        if (o == Py_None) return nullptr;
        const at::Tensor& t = tensor(o, at::kInt, name);
        if (t.sizes() != shape) raise(PyExc_ValueError, "%s has another shape than the cache's", name);
        return t.data_ptr();
    }
    // [batch][tokens][heads][head_dim] whose heads lie side by side
    const at::Tensor& rows(PyObject* o, int64_t heads, const char* name, bool packed_heads = true) const
    {
        const at::Tensor& t = tensor(o, at::kHalf, name, false);
        if (t.dim() != 4 || t.size(0) != c->batch || t.size(1) < 1 || (heads > 0 && t.size(2) != heads) || t.size(3) != c->head_dim || t.stride(3) != 1 ||
            (packed_heads && t.size(2) > 1 && t.stride(2) != c->head_dim)) {
            PyErr_Format(PyExc_ValueError, packed_heads ? "%s must be [batch][tokens][heads][head_dim], the heads of a token side by side"
                                                        : "%s must be [batch][tokens][kv_heads][head_dim] with unit stride in a row", name);
            throw Raised();
        }
        return t;
    }
    void* stream(PyObject* o) const
    {
        if (o != Py_None) {
            PyObject* d = PyObject_GetAttr(o, g_names.device_index);
            if (d) {
                Py_DECREF(d);
                const int i = int_attr(o, g_names.device_index, "device_index");
                if (i != device) raise(PyExc_ValueError, "%s", "the stream is another device's");
            } else {
                PyErr_Clear();
            }
            return stream_of(o);
        }
        return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    }
};

int64_t batch_stride(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : 0; }
int64_t token_stride(const at::Tensor& t) { return t.size(1) > 1 ? t.stride(1) : 0; }

// (cache, k, v, workspace, counts, length_out, stream) -> the lengths
PyObject* kv_append(PyObject*, Args a, Py_ssize_t na)
{
    return guarded([&]() -> PyObject* {
        need_args(na, 7);
        const Cache p(a[0]);
        const at::Tensor &k = p.rows(a[1], p.c->kv_heads, "k"), &v = p.rows(a[2], p.c->kv_heads, "v");
        if (k.size(1) != v.size(1) || batch_stride(k) != batch_stride(v) || token_stride(k) != token_stride(v))
            raise(PyExc_ValueError, "%s", "k and v must have the same shape and strides");
        const at::Tensor& ws = p.tensor(a[3], at::kByte, "workspace");
        const void* counts = p.optional(a[4], {p.c->batch}, "counts");
        void* out = p.optional(a[5], {p.c->batch, p.c->kv_heads}, "length_out");
        const int tokens = in_int(k.size(1), "the number of tokens");
        void* s = p.stream(a[6]);
        call("spqt_kv_append", [&] {
            return spqt_kv_append(p.c, k.data_ptr(), v.data_ptr(), tokens, batch_stride(k), token_stride(k),
                                  static_cast<const int32_t*>(counts), static_cast<int32_t*>(out), ws.data_ptr(), (size_t)ws.numel(), s);
        });
        Py_RETURN_NONE;
    });
}

// (cache, k, v, workspace, length, stream)
PyObject* kv_read(PyObject*, Args a, Py_ssize_t na)
{
    return guarded([&]() -> PyObject* {
        need_args(na, 6);
        const Cache p(a[0]);
        const at::Tensor &k = p.rows(a[1], p.c->kv_heads, "k", false), &v = p.rows(a[2], p.c->kv_heads, "v", false);
        if (k.size(1) != v.size(1) || k.strides() != v.strides()) raise(PyExc_ValueError, "%s", "k and v must have the same shape and strides");
        const at::Tensor& ws = p.tensor(a[3], at::kByte, "workspace");
        const void* length = p.optional(a[4], {p.c->batch, p.c->kv_heads}, "length");
        const int tokens = in_int(k.size(1), "the number of tokens");
        void* s = p.stream(a[5]);
        call("spqt_kv_read", [&] {
            return spqt_kv_read(p.c, static_cast<const int32_t*>(length), k.data_ptr(), v.data_ptr(), tokens, batch_stride(k), token_stride(k),
                                k.size(2) > 1 ? k.stride(2) : 0, ws.data_ptr(), (size_t)ws.numel(), s);
        });
        Py_RETURN_NONE;
    });
}

// (cache, q, workspace, scale or None, accumulate, out, stream) -> out
PyObject* kv_attention(PyObject*, Args a, Py_ssize_t na)
{
    return guarded([&]() -> PyObject* {
        need_args(na, 7);
        const Cache p(a[0]);
        const at::Tensor& q = p.rows(a[1], 0, "q");
        const at::Tensor& ws = p.tensor(a[2], at::kByte, "workspace");
        const float scale = a[3] == Py_None ? (float)(1.0 / std::sqrt((double)p.c->head_dim)) : float_of(a[3]);
        const int accumulate = PyObject_IsTrue(a[4]);
        if (accumulate < 0) throw Raised();
        const int heads = in_int(q.size(2), "the number of heads"), queries = in_int(q.size(1), "the number of queries");
        at::Tensor out;
        if (a[5] == Py_None) {
            out = empty(q.sizes(), at::kHalf, q, a[6]);
        } else {
            out = p.rows(a[5], q.size(2), "out");
            if (out.size(1) != q.size(1)) raise(PyExc_ValueError, "%s", "out must have the shape of q");
        }
        void* s = p.stream(a[6]);
        call("spqt_kv_attention", [&] {
            return spqt_kv_attention(p.c, q.data_ptr(), batch_stride(q), token_stride(q), heads, queries, scale, accumulate, out.data_ptr(),
                                     batch_stride(out), token_stride(out), ws.data_ptr(), (size_t)ws.numel(), s);
        });
        return hand_back(a[5], out);
    });
}

// (cache, keep, first, recent, workspace, table_out, length_out, stream)
PyObject* kv_evict(PyObject*, Args a, Py_ssize_t na)
{
    return guarded([&]() -> PyObject* {
        need_args(na, 8);
        const Cache p(a[0]);
        const int keep = int_of(a[1], "keep"), first = int_of(a[2], "first"), recent = int_of(a[3], "recent");
        const at::Tensor& ws = p.tensor(a[4], at::kByte, "workspace");
        void* table = p.optional(a[5], {p.c->batch, p.c->kv_heads, p.c->table_width}, "table_out");
        void* length = p.optional(a[6], {p.c->batch, p.c->kv_heads}, "length_out");
        void* s = p.stream(a[7]);
        call("spqt_kv_evict", [&] {
            return spqt_kv_evict(p.c, keep, first, recent, static_cast<int32_t*>(table), static_cast<int32_t*>(length), ws.data_ptr(), (size_t)ws.numel(), s);
        });
        Py_RETURN_NONE;
    });
}

// (logits, tokens or None, top, entropy, stream) -> (logprob or None, entropy or None, top_logprob, top_index)
PyObject* token_logprobs(PyObject*, Args a, Py_ssize_t na)
{
    return guarded([&]() -> PyObject* {
        need_args(na, 5);
        if (!THPVariable_Check(a[0])) raise(PyExc_TypeError, "%s must be a CUDA tensor", "logits");
        const at::Tensor& x = THPVariable_Unpack(a[0]);
        if (!x.is_cuda()) raise(PyExc_TypeError, "%s must be a CUDA tensor", "logits");
        const at::ScalarType t = x.scalar_type();
        if (t != at::kHalf && t != at::kBFloat16 && t != at::kFloat) raise(PyExc_TypeError, "%s must be float16, bfloat16 or float32", "logits");
        if (x.dim() != 2 || (x.size(1) > 1 && x.stride(1) != 1)) raise(PyExc_ValueError, "%s", "logits must be [rows][vocab] with unit column stride");
        const c10::cuda::OptionalCUDAGuard guard(x.device());
        const int rows = in_int(x.size(0), "the number of rows"), vocab = in_int(x.size(1), "the vocabulary");
        const int top = int_of(a[2], "top");
        if (top < 0) raise(PyExc_ValueError, "%s", "top must not be negative");
        const int wants_entropy = PyObject_IsTrue(a[3]);
        if (wants_entropy < 0) throw Raised();
        const int32_t* tokens = nullptr;
        const bool wants_logprob = a[1] != Py_None;
        at::Tensor logprob, entropy;
        if (wants_logprob) {
            const at::Tensor& k = tensor_of(a[1], at::kInt, "tokens");
            if (k.dim() != 1 || k.size(0) != rows || k.get_device() != x.get_device()) raise(PyExc_ValueError, "%s", "tokens must be [rows] on the device of logits");
            tokens = static_cast<const int32_t*>(k.data_ptr());
            logprob = empty({rows}, at::kFloat, x, a[4]);
        }
        if (wants_entropy) entropy = empty({rows}, at::kFloat, x, a[4]);
        at::Tensor best = empty({rows, top}, at::kFloat, x, a[4]), index = empty({rows, top}, at::kInt, x, a[4]);
        void* s = a[4] == Py_None ? c10::cuda::getCurrentCUDAStream(x.get_device()).stream() : stream_of(a[4]);
        call("spqt_token_logprobs", [&] {
            return spqt_token_logprobs(x.data_ptr(), t == at::kHalf ? SPQT_LOGITS_FP16 : t == at::kBFloat16 ? SPQT_LOGITS_BF16 : SPQT_LOGITS_FP32,
                                       rows, vocab, rows > 1 ? x.stride(0) : vocab, tokens, top,
                                       wants_logprob ? static_cast<float*>(logprob.data_ptr()) : nullptr, wants_entropy ? static_cast<float*>(entropy.data_ptr()) : nullptr,
                                       top > 0 ? static_cast<float*>(best.data_ptr()) : nullptr, top > 0 ? static_cast<int32_t*>(index.data_ptr()) : nullptr, s);
        });
        auto wrapped = [](bool there, at::Tensor& v) {
            if (there) return THPVariable_Wrap(std::move(v));
            Py_INCREF(Py_None);
            return Py_None;
        };
        return tuple_of(wrapped(wants_logprob, logprob), wrapped(wants_entropy, entropy), THPVariable_Wrap(std::move(best)), THPVariable_Wrap(std::move(index)));
    });
}

PyObject* set_error(PyObject*, PyObject* cls)
{
    Py_INCREF(cls);
    Py_XSETREF(g_error, cls);
    Py_RETURN_NONE;
}

#define SPQT_METHOD(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {
    SPQT_METHOD(sparsify), SPQT_METHOD(sparse_gemv), SPQT_METHOD(sparsify_gemv), SPQT_METHOD(dense_gemv),
    SPQT_METHOD(sparse_gemm_small), SPQT_METHOD(dense_gemm_small), SPQT_METHOD(kqw_sparse_gemv), SPQT_METHOD(kqw_dense_gemv), SPQT_METHOD(pack),
    SPQT_METHOD(kqw_pack), SPQT_METHOD(host_step_launch), SPQT_METHOD(kv_append), SPQT_METHOD(kv_read), SPQT_METHOD(kv_attention),
    SPQT_METHOD(kv_evict), SPQT_METHOD(token_logprobs),
    {"set_error", set_error, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void)
{
    g_names = {PyUnicode_InternFromString("codes"), PyUnicode_InternFromString("scale_zero"), PyUnicode_InternFromString("records"),
               PyUnicode_InternFromString("m"), PyUnicode_InternFromString("n"), PyUnicode_InternFromString("bits"),
               PyUnicode_InternFromString("group"), PyUnicode_InternFromString("cuda_stream"), PyUnicode_InternFromString("desc"),
               PyUnicode_InternFromString("device_index")};
    return PyModule_Create(&g_module);
}
