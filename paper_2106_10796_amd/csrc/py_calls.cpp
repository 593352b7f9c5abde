// The calls that a program makes per tensor or per step, with the binding's argument checks in native code.
//
// A call on a small tensor is bound by the host: of 4.0 us for a step of a plan on 64 k elements the runtime's launch
// takes 2.4, and marshalling a list of 16 streams in Python took 10 of the 15.7 us of a small decode-and-sum and update.
//
// Every function takes the arguments of the binding's function of the same name, then the binding's `_stream`, which is
// asked for the stream once the arguments are known to be good.  It returns the library's status, or -1 and does nothing
// where an argument is anything but plainly good: the binding's own checks then say what is wrong, or convert it.
#include <Python.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/detail/CUDAHooksInterface.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <cmath>
#include <cstring>

#include "cdsgd.h"
#include "cdsgd_block.h"
#include "cdsgd_ops.h"

namespace {

struct Library {
    decltype(&cdsgd_quantize_pack) quantize_pack;
    decltype(&cdsgd_decode_sum) decode_sum;
    decltype(&cdsgd_decode_sum_sparse) decode_sum_sparse;
    decltype(&cdsgd_update) update;
    decltype(&cdsgd_sparse_encode) sparse_encode;
    decltype(&cdsgd_sparse_words) sparse_words;
    decltype(&cdsgd_sparse_segments) sparse_segments;
    decltype(&cdsgd_step_fused) step_fused;
    decltype(&cdsgd_step_fused_range) step_fused_range;
    decltype(&cdsgd_step_fused_static) step_fused_static;
    decltype(&cdsgd_grad_norm_compute) grad_norm_compute;
    decltype(&cdsgd_adamw_step) adamw_step;
    decltype(&cdsgd_adamw_grad_norm) adamw_grad_norm;
    decltype(&cdsgd_adamw_read_states) adamw_read_states;
    decltype(&cdsgd_mxfp4_quantize) mxfp4_quantize;
    decltype(&cdsgd_mxfp4_dequantize) mxfp4_dequantize;
    decltype(&cdsgd_mxfp4_matmul) mxfp4_matmul;
    decltype(&cdsgd_mxint8_quantize) mxint8_quantize;
    decltype(&cdsgd_mxint8_dequantize) mxint8_dequantize;
    decltype(&cdsgd_gated_forward) gated_forward;
    decltype(&cdsgd_gated_backward) gated_backward;
    decltype(&cdsgd_block_norm_forward) block_norm_forward;
    decltype(&cdsgd_block_norm_backward) block_norm_backward;
    decltype(&cdsgd_attention_forward) attention_forward;
    decltype(&cdsgd_attention_backward) attention_backward;
} lib;

struct NotPlain {};  // leave it to the binding

size_t packed_words(size_t n) { return (n + 15) / 16; }

// A dense contiguous tensor on the GPU, not of a subclass, with `n` elements (kAny: any number).
constexpr size_t kAny = (size_t)-1;
void *buffer(PyObject *o, at::ScalarType type, size_t n, size_t *numel = nullptr)
{
    if (!THPVariable_CheckExact(o)) throw NotPlain();
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.scalar_type() != type || !t.is_cuda() || !t.is_contiguous()) throw NotPlain();
    const size_t have = (size_t)t.numel();
    if (n != kAny && have != n) throw NotPlain();
    if (numel) *numel = have;
    return t.data_ptr();
}

float *floats(PyObject *o, size_t n, size_t *numel = nullptr) { return static_cast<float *>(buffer(o, at::kFloat, n, numel)); }
float *floats_or_null(PyObject *o, size_t n) { return o == Py_None ? nullptr : floats(o, n); }
uint32_t *words(PyObject *o, size_t n) { return static_cast<uint32_t *>(buffer(o, at::kInt, n)); }

double real(PyObject *o)
{
    if (PyFloat_CheckExact(o)) return PyFloat_AS_DOUBLE(o);
    throw NotPlain();
}

float number(PyObject *o) { return (float)real(o); }

long whole(PyObject *o)
{
    if (!PyLong_CheckExact(o)) throw NotPlain();
    int over = 0;
    const long v = PyLong_AsLongAndOverflow(o, &over);
    if (over) throw NotPlain();
    return v;
}

int small(PyObject *o)
{
    const long v = whole(o);
    if (v < INT_MIN || v > INT_MAX) throw NotPlain();
    return (int)v;
}

template <typename T>
T *address(PyObject *o)
{
    if (!PyLong_CheckExact(o)) throw NotPlain();
    void *p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) {
        PyErr_Clear();
        throw NotPlain();
    }
    return static_cast<T *>(p);
}

struct Raised {};  // a Python error is set

void *stream_of(PyObject *lookup)
{
    PyObject *s = PyObject_CallNoArgs(lookup);
    if (!s) throw Raised();
    void *p = PyLong_Check(s) ? PyLong_AsVoidPtr(s) : nullptr;
    const bool bad = !PyLong_Check(s) || (!p && PyErr_Occurred());
    Py_DECREF(s);
    if (bad) {
        PyErr_Clear();
        throw NotPlain();
    }
    return p;
}

// `call` does what a function does with its arguments; the lock is given up inside it, around the library's part.
template <typename Call>
PyObject *guarded(Py_ssize_t have, Py_ssize_t want, Call call)
{
    int status = -1;
    if (have == want && lib.update && !at::impl::torch_function_mode_enabled()) {
        try {
            status = call();
        } catch (const Raised &) {
            return nullptr;
        } catch (...) {
            status = -1;  // (a tensor without storage, a layout without strides: the binding says what it is)
        }
    }
    return PyLong_FromLong(status);
}

template <typename Call>
int unlocked(Call call)
{
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = call();
    Py_END_ALLOW_THREADS
    return status;
}

PyObject *quantize_pack(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 5, [&] {
        size_t count;
        const float *grad = floats(a[0], kAny, &count);
        float *residual = floats(a[1], count);
        uint32_t *packed = words(a[2], packed_words(count));
        const float t = number(a[3]);
        void *s = stream_of(a[4]);
        return unlocked([&] { return lib.quantize_pack(grad, residual, packed, count, t, s); });
    });
}

PyObject *decode(PyObject *const *a, Py_ssize_t n, bool sparse)
{
    return guarded(n, 4, [&] {
        if (!PyList_CheckExact(a[0]) && !PyTuple_CheckExact(a[0])) throw NotPlain();
        const Py_ssize_t workers = PySequence_Fast_GET_SIZE(a[0]);
        if (workers < 1 || workers > CDSGD_MAX_WORKERS) throw NotPlain();
        size_t count;
        float *agg = floats(a[1], kAny, &count);
        const size_t each = sparse ? lib.sparse_words(count) : packed_words(count);
        const uint32_t *streams[CDSGD_MAX_WORKERS];
        for (Py_ssize_t j = 0; j < workers; ++j) streams[j] = words(PySequence_Fast_GET_ITEM(a[0], j), each);
        const float t = number(a[2]);
        void *s = stream_of(a[3]);
        const auto f = sparse ? lib.decode_sum_sparse : lib.decode_sum;
        return unlocked([&] { return f(streams, (int)workers, agg, count, t, s); });
    });
}

PyObject *decode_sum(PyObject *, PyObject *const *a, Py_ssize_t n) { return decode(a, n, false); }
PyObject *decode_sum_sparse(PyObject *, PyObject *const *a, Py_ssize_t n) { return decode(a, n, true); }

PyObject *update(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 8, [&] {
        size_t count;
        float *w_global = floats(a[0], kAny, &count);
        float *w_local = floats_or_null(a[1], count);
        const float *grad = floats_or_null(a[2], count);
        const float *agg = floats_or_null(a[3], count);
        const float lr_local = number(a[4]), lr_global = number(a[5]);
        const int workers = small(a[6]);
        void *s = stream_of(a[7]);
        return unlocked([&] { return lib.update(w_global, w_local, grad, agg, count, lr_local, lr_global, workers, s); });
    });
}

PyObject *sparse_encode(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 5, [&] {
        const long count = whole(a[1]);
        if (count < 1) throw NotPlain();
        const uint32_t *packed = words(a[0], packed_words((size_t)count));
        uint32_t *sparse = words(a[2], lib.sparse_words((size_t)count));
        uint32_t *counts = a[3] == Py_None ? nullptr : words(a[3], lib.sparse_segments((size_t)count));
        void *s = stream_of(a[4]);
        return unlocked([&] { return lib.sparse_encode(packed, (size_t)count, sparse, counts, s); });
    });
}

PyObject *step(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 7, [&] {
        cdsgd_plan *plan = address<cdsgd_plan>(a[0]);
        const long i = whole(a[1]);
        const int k = small(a[2]);
        const float t = number(a[3]), lr_local = number(a[4]), lr_global = number(a[5]);
        void *s = stream_of(a[6]);
        return unlocked([&] { return lib.step_fused(plan, i, k, t, lr_local, lr_global, s); });
    });
}

PyObject *step_range(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 9, [&] {
        cdsgd_plan *plan = address<cdsgd_plan>(a[0]);
        const int first = small(a[1]), count = small(a[2]);
        const long i = whole(a[3]);
        const int k = small(a[4]);
        const float t = number(a[5]), lr_local = number(a[6]), lr_global = number(a[7]);
        void *s = stream_of(a[8]);
        return unlocked([&] { return lib.step_fused_range(plan, first, count, i, k, t, lr_local, lr_global, s); });
    });
}

PyObject *step_static(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 12, [&] {
        const cdsgd_tensor *tensors = address<const cdsgd_tensor>(a[0]);
        const int num_tensors = small(a[1]);
        const uint32_t *const *const *peers = address<const uint32_t *const *const>(a[2]);
        const int workers = small(a[3]), self = small(a[4]), dtype = small(a[5]);
        const long i = whole(a[6]);
        const int k = small(a[7]);
        const float t = number(a[8]), lr_local = number(a[9]), lr_global = number(a[10]);
        void *s = stream_of(a[11]);
        return unlocked([&] {
            return lib.step_fused_static(tensors, num_tensors, peers, workers, self, dtype, i, k, t, lr_local, lr_global, s);
        });
    });
}

// A handle's address (not 0: a handle that has been destroyed).
template <typename T>
T *handle(PyObject *o)
{
    T *p = address<T>(o);
    if (!p) throw NotPlain();
    return p;
}

template <typename Handle, typename Call>
PyObject *norm_of(PyObject *const *a, Py_ssize_t n, Call f)
{
    return guarded(n, 5, [&] {
        Handle *h = handle<Handle>(a[0]);
        float *out = floats(a[1], 2);
        const double scale = real(a[2]), max_norm = real(a[3]);
        void *s = stream_of(a[4]);
        return unlocked([&] { return (lib.*f)(h, scale, max_norm, out, s); });
    });
}

PyObject *grad_norm_compute(PyObject *, PyObject *const *a, Py_ssize_t n) { return norm_of<cdsgd_grad_norm>(a, n, &Library::grad_norm_compute); }
PyObject *adamw_grad_norm(PyObject *, PyObject *const *a, Py_ssize_t n) { return norm_of<cdsgd_adamw_plan>(a, n, &Library::adamw_grad_norm); }

PyObject *adamw_step(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 10, [&] {
        cdsgd_adamw_plan *plan = handle<cdsgd_adamw_plan>(a[0]);
        const long i = whole(a[1]);
        const double lr = real(a[2]), beta1 = real(a[3]), beta2 = real(a[4]), eps = real(a[5]), scale = real(a[6]);
        if (!PyLong_CheckExact(a[7])) throw NotPlain();
        const uint64_t seed = PyLong_AsUnsignedLongLongMask(a[7]);
        const float *clip = floats_or_null(a[8], 2);
        void *s = stream_of(a[9]);
        return unlocked([&] { return lib.adamw_step(plan, i, lr, beta1, beta2, eps, scale, seed, clip, s); });
    });
}

PyObject *adamw_read_states(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 2, [&] {
        cdsgd_adamw_plan *plan = handle<cdsgd_adamw_plan>(a[0]);
        void *s = stream_of(a[1]);
        return unlocked([&] { return lib.adamw_read_states(plan, s); });
    });
}

// A matrix in MXFP4, as the binding's class of that name holds it.
struct Mx {
    uint8_t *codes = nullptr, *scales = nullptr;
    size_t rows = 0, cols = 0;
};

Mx mx(PyObject *o, bool written = false)
{
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) throw NotPlain();
    // (copies of the caller's tensors are read alone)
    const char *kind = Py_TYPE(o)->tp_name;
    if (std::strcmp(kind, "Mxfp4") != 0 && (written || std::strcmp(kind, "_Mxfp4Copy") != 0)) throw NotPlain();
    const long rows = whole(PyTuple_GET_ITEM(o, 2)), cols = whole(PyTuple_GET_ITEM(o, 3));
    if (rows < 1 || cols < 1 || rows > INT_MAX || cols > INT_MAX) throw NotPlain();
    const size_t groups = ((size_t)cols + 127) / 128;
    Mx q;
    q.rows = (size_t)rows;
    q.cols = (size_t)cols;
    q.codes = static_cast<uint8_t *>(buffer(PyTuple_GET_ITEM(o, 0), at::kByte, q.rows * 64 * groups));
    q.scales = static_cast<uint8_t *>(buffer(PyTuple_GET_ITEM(o, 1), at::kByte, q.rows * 4 * groups));
    return q;
}

// A matrix of ordinary numbers whose rows are contiguous and do not overlap.
struct Matrix {
    void *p;
    int dtype;
    size_t rows, cols, ld;
};

Matrix matrix(PyObject *o)
{
    if (!THPVariable_CheckExact(o)) throw NotPlain();
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.dim() != 2) throw NotPlain();
    Matrix m;
    switch (t.scalar_type()) {
    case at::kFloat: m.dtype = CDSGD_GRAD_F32; break;
    case at::kBFloat16: m.dtype = CDSGD_GRAD_BF16; break;
    case at::kHalf: m.dtype = CDSGD_GRAD_F16; break;
    default: throw NotPlain();
    }
    const int64_t rows = t.size(0), cols = t.size(1), row = t.stride(0);
    if (rows < 1 || cols < 1 || (cols > 1 && t.stride(1) != 1) || (rows > 1 && row < cols)) throw NotPlain();
    m.p = t.data_ptr();
    m.rows = (size_t)rows;
    m.cols = (size_t)cols;
    m.ld = (size_t)(rows > 1 ? row : cols);
    return m;
}

PyObject *mxfp4_quantize(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 4, [&] {
        const Matrix x = matrix(a[0]);
        const Mx row = a[1] == Py_None ? Mx() : mx(a[1], true), col = a[2] == Py_None ? Mx() : mx(a[2], true);
        if ((row.codes && (row.rows != x.rows || row.cols != x.cols)) || (col.codes && (col.rows != x.cols || col.cols != x.rows))) throw NotPlain();
        void *s = stream_of(a[3]);
        return unlocked([&] { return lib.mxfp4_quantize(x.p, x.dtype, x.rows, x.cols, x.ld, row.codes, row.scales, col.codes, col.scales, s); });
    });
}

PyObject *mxfp4_dequantize(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 3, [&] {
        const Mx q = mx(a[0]);
        const Matrix out = matrix(a[1]);
        if (out.rows != q.rows || out.cols != q.cols) throw NotPlain();
        void *s = stream_of(a[2]);
        return unlocked([&] { return lib.mxfp4_dequantize(q.codes, q.scales, q.rows, q.cols, out.p, out.dtype, out.ld, s); });
    });
}

PyObject *mxfp4_matmul(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 6, [&] {
        const Mx x = mx(a[0]), y = mx(a[1]);
        const Matrix out = matrix(a[2]);
        if (x.cols != y.cols || out.rows != x.rows || out.cols != y.rows) throw NotPlain();
        size_t room = 0;
        void *workspace = a[3] == Py_None ? nullptr : buffer(a[3], at::kByte, kAny, &room);
        if (a[4] != Py_False && a[4] != Py_True) throw NotPlain();
        const int add = a[4] == Py_True;
        void *s = stream_of(a[5]);
        return unlocked([&] {
            return lib.mxfp4_matmul(x.codes, x.scales, y.codes, y.scales, x.rows, y.rows, x.cols, out.p, out.dtype, out.ld, add, workspace, room, s);
        });
    });
}

// ---- include/cdsgd_block.h: as above, and every tensor is on the current device ----------------------------------------------------

void on_this_device(PyObject *o)
{
    if (o == Py_None) return;
    if (THPVariable_Unpack(o).get_device() != at::detail::getCUDAHooks().getCurrentDevice()) throw NotPlain();
}

Matrix matrix_here(PyObject *o)
{
    const Matrix m = matrix(o);
    on_this_device(o);
    return m;
}

// A matrix like another, of its type or of `dtype`; None where that is allowed.
Matrix like(PyObject *o, const Matrix &x, int dtype, bool or_none = false)
{
    if (or_none && o == Py_None) return {nullptr, dtype, x.rows, x.cols, 0};
    const Matrix m = matrix_here(o);
    if (m.dtype != dtype || m.rows != x.rows || m.cols != x.cols) throw NotPlain();
    return m;
}

void *buffer_here(PyObject *o, at::ScalarType type, size_t n, size_t *numel = nullptr)
{
    if (o == Py_None) {
        if (numel) *numel = 0;
        return nullptr;
    }
    void *p = buffer(o, type, n, numel);
    on_this_device(o);
    return p;
}
float *floats_here(PyObject *o, size_t n) { return static_cast<float *>(buffer_here(o, at::kFloat, n)); }

// A matrix in 8 bits, as the binding's class of that name holds it.
struct Mx8 {
    int8_t *codes = nullptr;
    uint8_t *scales = nullptr;
    size_t rows = 0, cols = 0;
};

bool is_mx8(PyObject *o) { return PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 4 && std::strcmp(Py_TYPE(o)->tp_name, "Mxint8") == 0; }

Mx8 mx8(PyObject *o)
{
    if (!is_mx8(o)) throw NotPlain();
    const long rows = whole(PyTuple_GET_ITEM(o, 2)), cols = whole(PyTuple_GET_ITEM(o, 3));
    if (rows < 1 || cols < 1 || rows > INT_MAX || cols > INT_MAX) throw NotPlain();
    const size_t groups = ((size_t)cols + 31) / 32;
    Mx8 q;
    q.rows = (size_t)rows;
    q.cols = (size_t)cols;
    q.codes = static_cast<int8_t *>(buffer(PyTuple_GET_ITEM(o, 0), at::kChar, q.rows * 32 * groups));
    q.scales = static_cast<uint8_t *>(buffer(PyTuple_GET_ITEM(o, 1), at::kByte, q.rows * groups));
    on_this_device(PyTuple_GET_ITEM(o, 0));
    on_this_device(PyTuple_GET_ITEM(o, 1));
    return q;
}

Mx8 mx8_like(PyObject *o, const Matrix &x)
{
    if (o == Py_None) return Mx8();
    const Mx8 q = mx8(o);
    if (q.rows != x.rows || q.cols != x.cols) throw NotPlain();
    return q;
}

cdsgd_held held(PyObject *o, const Matrix &x, int dtype)
{
    if (is_mx8(o)) {
        const Mx8 q = mx8_like(o, x);
        return {nullptr, 0, q.codes, q.scales};
    }
    const Matrix m = like(o, x, dtype);
    return {m.p, m.ld, nullptr, nullptr};
}

PyObject *mxint8_quantize(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 3, [&] {
        const Matrix x = matrix_here(a[0]);
        const Mx8 q = mx8(a[1]);
        if (q.rows != x.rows || q.cols != x.cols) throw NotPlain();
        void *s = stream_of(a[2]);
        return unlocked([&] { return lib.mxint8_quantize(x.p, x.dtype, x.rows, x.cols, x.ld, q.codes, q.scales, s); });
    });
}

PyObject *mxint8_dequantize(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 3, [&] {
        const Mx8 q = mx8(a[0]);
        const Matrix out = matrix_here(a[1]);
        if (out.rows != q.rows || out.cols != q.cols) throw NotPlain();
        void *s = stream_of(a[2]);
        return unlocked([&] { return lib.mxint8_dequantize(q.codes, q.scales, q.rows, q.cols, out.p, out.dtype, out.ld, s); });
    });
}

PyObject *gated_forward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 7, [&] {
        const Matrix x = matrix_here(a[0]), u = like(a[1], x, x.dtype), y = like(a[2], x, x.dtype);
        const Mx8 a8 = mx8_like(a[3], x), u8 = mx8_like(a[4], x);
        const int act = small(a[5]);
        void *s = stream_of(a[6]);
        return unlocked([&] {
            return lib.gated_forward(act, x.dtype, x.rows, x.cols, x.p, x.ld, u.p, u.ld, y.p, y.ld, a8.codes, a8.scales, u8.codes, u8.scales, s);
        });
    });
}

PyObject *gated_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 7, [&] {
        const Matrix dy = matrix_here(a[0]);
        const cdsgd_held x = held(a[1], dy, dy.dtype), u = held(a[2], dy, dy.dtype);
        const Matrix da = like(a[3], dy, dy.dtype), du = like(a[4], dy, dy.dtype);
        const int act = small(a[5]);
        void *s = stream_of(a[6]);
        return unlocked([&] { return lib.gated_backward(act, dy.dtype, dy.rows, dy.cols, dy.p, dy.ld, &x, &u, da.p, da.ld, du.p, du.ld, s); });
    });
}

// The norm at that address, for that matrix and stream type; `device` is that of its weights.
cdsgd_block_norm norm_of_rows(PyObject *at, PyObject *device, const Matrix &y, int stream, bool block)
{
    cdsgd_block_norm n = *handle<const cdsgd_block_norm>(at);
    if (n.cols != y.cols || small(device) != at::detail::getCUDAHooks().getCurrentDevice()) throw NotPlain();
    n.dtype = y.dtype;
    n.stream_dtype = stream;
    n.rows = y.rows;
    if (!block) n.block_weight = n.gate = nullptr;
    return n;
}

PyObject *block_norm_forward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 10, [&] {
        const Matrix y = matrix_here(a[3]), h = matrix_here(a[2]);
        if (h.rows != y.rows || h.cols != y.cols) throw NotPlain();
        const cdsgd_block_norm norm = norm_of_rows(a[0], a[1], y, h.dtype, a[5] != Py_None);
        float *rstd = floats_here(a[4], 2 * y.rows);
        const Matrix b = like(a[5], y, y.dtype, true), out = like(a[6], y, h.dtype, true);
        const Mx8 h8 = mx8_like(a[7], y), b8 = mx8_like(a[8], y);
        void *s = stream_of(a[9]);
        return unlocked([&] {
            return lib.block_norm_forward(&norm, h.p, h.ld, b.p, b.ld, out.p, out.ld, y.p, y.ld, rstd, h8.codes, h8.scales, b8.codes, b8.scales, s);
        });
    });
}

PyObject *block_norm_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 14, [&] {
        const Matrix dy = matrix_here(a[2]), dh = matrix_here(a[5]);
        if (dh.rows != dy.rows || dh.cols != dy.cols) throw NotPlain();
        const bool block = a[9] != Py_None;
        const cdsgd_block_norm norm = norm_of_rows(a[0], a[1], dy, dh.dtype, block);
        const cdsgd_held h = held(a[3], dy, dh.dtype), none = {nullptr, 0, nullptr, nullptr}, b = block ? held(a[9], dy, dy.dtype) : none;
        const float *rstd = floats_here(a[4], 2 * dy.rows);
        float *dw = floats_here(a[6], dy.cols);
        size_t room = 0;
        void *workspace = buffer_here(a[7], at::kByte, kAny, &room);
        const Matrix dt = like(a[8], dy, dh.dtype, true), db = like(a[10], dy, dy.dtype, true);
        float *dw_b = floats_here(a[11], dy.cols), *dgate = floats_here(a[12], dy.cols);
        void *s = stream_of(a[13]);
        return unlocked([&] {
            return lib.block_norm_backward(&norm, dy.p, dy.ld, dt.p, dt.ld, &h, &b, rstd, dh.p, dh.ld, db.p, db.ld, dw, dw_b, dgate, workspace, room, s);
        });
    });
}

// [tokens, heads, dim] with a token's heads in a row.
struct Heads {
    void *p;
    int dtype;
    size_t tokens, heads, dim, ld;
};

Heads heads(PyObject *o)
{
    if (!THPVariable_CheckExact(o)) throw NotPlain();
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.dim() != 3) throw NotPlain();
    Heads x;
    if (t.scalar_type() == at::kBFloat16) x.dtype = CDSGD_GRAD_BF16;
    else if (t.scalar_type() == at::kHalf) x.dtype = CDSGD_GRAD_F16;
    else throw NotPlain();
    const int64_t n = t.size(0), h = t.size(1), d = t.size(2), ld = n > 1 ? t.stride(0) : h * d;
    if (n < 1 || h < 1 || d < 1 || h > INT_MAX || d > INT_MAX || (d > 1 && t.stride(2) != 1) || (h > 1 && t.stride(1) != d) || ld < h * d) throw NotPlain();
    on_this_device(o);
    x.p = t.data_ptr();
    x.tokens = (size_t)n;
    x.heads = (size_t)h;
    x.dim = (size_t)d;
    x.ld = (size_t)ld;
    return x;
}

Heads heads_like(PyObject *o, const Heads &x)
{
    const Heads y = heads(o);
    if (y.dtype != x.dtype || y.tokens != x.tokens || y.heads != x.heads || y.dim != x.dim) throw NotPlain();
    return y;
}

cdsgd_attention batch_of(const Heads &q, const Heads &k, PyObject *starts, PyObject *starts_k, PyObject *causal, PyObject *scale)
{
    if (q.dtype != k.dtype || q.dim != k.dim || (causal != Py_True && causal != Py_False)) throw NotPlain();
    cdsgd_attention b = {};
    b.dtype = q.dtype;
    b.causal = causal == Py_True;
    b.tokens_q = q.tokens;
    b.tokens_k = k.tokens;
    b.num_seqs = 1;
    b.heads = (int)q.heads;
    b.kv_heads = (int)k.heads;
    b.dim = (int)q.dim;
    b.scale = scale == Py_None ? 1.0 / std::sqrt((double)q.dim) : real(scale);
    if (starts == Py_None) {
        if (starts_k != Py_None) throw NotPlain();
        return b;
    }
    size_t count = 0;
    b.starts_q = static_cast<const int32_t *>(buffer_here(starts, at::kInt, kAny, &count));
    if (count < 2 || THPVariable_Unpack(starts).dim() != 1) throw NotPlain();
    if (starts_k != Py_None && THPVariable_CheckExact(starts_k) && THPVariable_Unpack(starts_k).dim() != 1) throw NotPlain();
    b.num_seqs = count - 1;
    b.starts_k = static_cast<const int32_t *>(buffer_here(starts_k, at::kInt, count));
    return b;
}

PyObject *attention_forward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 11, [&] {
        const Heads q = heads(a[0]), k = heads(a[1]), v = heads_like(a[2], k), out = heads_like(a[3], q);
        float *lse = floats_here(a[4], q.tokens * q.heads);
        const cdsgd_attention b = batch_of(q, k, a[5], a[6], a[7], a[8]);
        size_t room = 0;
        void *workspace = buffer_here(a[9], at::kByte, kAny, &room);
        void *s = stream_of(a[10]);
        return unlocked([&] { return lib.attention_forward(&b, q.p, q.ld, k.p, k.ld, v.p, v.ld, out.p, out.ld, lse, workspace, room, s); });
    });
}

PyObject *attention_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 15, [&] {
        const Heads q = heads(a[1]), k = heads(a[2]), v = heads_like(a[3], k), dout = heads_like(a[0], q), out = heads_like(a[4], q);
        const float *lse = floats_here(a[5], q.tokens * q.heads);
        const Heads dq = heads_like(a[6], q), dk = heads_like(a[7], k), dv = heads_like(a[8], k);
        const cdsgd_attention b = batch_of(q, k, a[9], a[10], a[11], a[12]);
        size_t room = 0;
        void *workspace = buffer_here(a[13], at::kByte, kAny, &room);
        void *s = stream_of(a[14]);
        return unlocked([&] {
            return lib.attention_backward(&b, dout.p, dout.ld, q.p, q.ld, k.p, k.ld, v.p, v.ld, out.p, out.ld, lse, dq.p, dq.ld, dk.p, dk.ld, dv.p, dv.ld,
                                          workspace, room, s);
        });
    });
}

// bind(addresses of the library's functions, in the order of `Library`)
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    void *p[sizeof(Library) / sizeof(void *)];
    if (n != (Py_ssize_t)(sizeof(p) / sizeof(p[0]))) {
        PyErr_SetString(PyExc_TypeError, "bind takes an address for each of the library's functions");
        return nullptr;
    }
    for (Py_ssize_t i = 0; i < n; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an address is 0");
            return nullptr;
        }
    }
    static_assert(sizeof(Library) == sizeof(p), "nothing but function pointers");
    __builtin_memcpy(&lib, p, sizeof(p));
    Py_RETURN_NONE;
}

template <typename F>
PyMethodDef method(const char *name, F f)
{
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method("bind", bind), method("quantize_pack", quantize_pack), method("decode_sum", decode_sum),
                         method("decode_sum_sparse", decode_sum_sparse), method("update", update),
                         method("sparse_encode", sparse_encode), method("step", step), method("step_range", step_range),
                         method("step_static", step_static),
                         method("grad_norm_compute", grad_norm_compute), method("adamw_step", adamw_step),
                         method("adamw_grad_norm", adamw_grad_norm), method("adamw_read_states", adamw_read_states),
                         method("mxfp4_quantize", mxfp4_quantize), method("mxfp4_dequantize", mxfp4_dequantize),
                         method("mxfp4_matmul", mxfp4_matmul), method("mxint8_quantize", mxint8_quantize),
                         method("mxint8_dequantize", mxint8_dequantize), method("gated_forward", gated_forward),
                         method("gated_backward", gated_backward), method("block_norm_forward", block_norm_forward),
                         method("block_norm_backward", block_norm_backward), method("attention_forward", attention_forward),
                         method("attention_backward", attention_backward), {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

#ifndef CDSGD_BUILD_ID_HEX
#define CDSGD_BUILD_ID_HEX "0000000000000000"
#endif
#ifndef CDSGD_CALLS_LIBRARY
#define CDSGD_CALLS_LIBRARY ""
#define CDSGD_CALLS_TORCH ""
#define CDSGD_CALLS_SOABI ""
#endif

// The identity of what the module was built from; the marker makes it findable in the file.
extern "C" __attribute__((used, visibility("default"))) const char cdsgd_calls_id[] = "CDSGD_BUILD_ID=" CDSGD_BUILD_ID_HEX;

// made_for: the library (its identity), the torch and the Python that the module may be used with.
PyMODINIT_FUNC PyInit__calls(void)
{
    PyObject *m = PyModule_Create(&module);
    if (!m) return nullptr;
    PyObject *made_for = Py_BuildValue("(sss)", CDSGD_CALLS_LIBRARY, CDSGD_CALLS_TORCH, CDSGD_CALLS_SOABI);
    if (!made_for || PyModule_AddObject(m, "made_for", made_for) != 0) {
        Py_XDECREF(made_for);
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
