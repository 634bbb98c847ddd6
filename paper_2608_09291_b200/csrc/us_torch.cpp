// The per-call half of the Python front end (binding.py): takes the caller's torch tensors apart, makes the
// output, finds the stream and calls the C ABI, in native code. Torch tensors are used only as device memory.
//
// A decode-sized product takes 3 to 5 us on the GPU. Marshalling the call in Python took 9.3 us (an output tensor
// 2.5, the current stream 2.2, ctypes with the launch 3.1, the rest argument handling), so every product up to
// about 8 us of GPU time was bound by it; the calls below leave 0.6 us around the launch's own 1.8.
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>

#include <optional>

#include "../../include/unionsparse.h"

namespace {

PyObject* g_error = nullptr;   // binding.UsError

PyObject* fail(us_status s, const char* where)
{
    if (!g_error) return PyErr_Format(PyExc_RuntimeError, "%s: status %d", where, (int)s);
    PyObject* e = PyObject_CallFunction(g_error, "is", (int)s, where);
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    return nullptr;
}

// A tensor argument; nullptr with an error set if it is none.
const at::Tensor* tensor(PyObject* o, const char* name)
{
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s must be a torch.Tensor, not %s", name, Py_TYPE(o)->tp_name);
        return nullptr;
    }
    return &THPVariable_Unpack(o);
}

// Optional tensor argument: None gives a null pointer.
bool pointer(PyObject* o, const char* name, void** out)
{
    *out = nullptr;
    if (o == Py_None) return true;
    const at::Tensor* t = tensor(o, name);
    if (!t) return false;
    *out = t->data_ptr();
    return true;
}

bool stream_of(PyObject* o, const at::Tensor& on, void** out)
{
    if (o != Py_None) {
        *out = PyLong_AsVoidPtr(o);
        return !PyErr_Occurred();
    }
    if (!on.is_cuda()) {
        PyErr_SetString(PyExc_ValueError, "expected a tensor on a CUDA device");
        return false;
    }
    *out = c10::cuda::getCurrentCUDAStream(on.device().index()).stream();
    return true;
}

bool is_f16_rows(const at::Tensor& t) { return t.scalar_type() == at::kHalf && t.dim() == 2 && t.stride(1) == 1; }

// The caller's output tensor, or a new one on the device of `on`.
at::Tensor new_output(const at::Tensor& on, int64_t N, int64_t M, at::ScalarType type)
{
    const int64_t shape[2] = {N, M};
    if (on.is_cuda()) return at::detail::empty_cuda(shape, type, on.device(), std::nullopt);
    return at::empty(shape, on.options().dtype(type));
}

// spmm(handle, M, X, N, x_scale, out, stream) -> the output tensor
PyObject* spmm(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 7) return PyErr_Format(PyExc_TypeError, "spmm takes 7 arguments");
    HANDLE_TH_ERRORS
    void *h = nullptr, *xs = nullptr, *st = nullptr;
    if (a[0] != Py_None) h = PyLong_AsVoidPtr(a[0]);
    const int64_t M = PyLong_AsLongLong(a[1]);
    const int64_t N = PyLong_AsLongLong(a[3]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor* X = tensor(a[2], "X");
    if (!X || !pointer(a[4], "x_scale", &xs) || !stream_of(a[6], *X, &st)) return nullptr;
    if (N < 1 || N > 64) return fail(US_ERR_INVALID_ARG, "us_spmm");
    at::Tensor fresh;
    const at::Tensor* out = nullptr;
    if (a[5] != Py_None) {
        out = tensor(a[5], "out");
        if (!out) return nullptr;
    } else {
        fresh = new_output(*X, N, M, xs ? at::kHalf : at::kInt);
    }
    us_status s;
    void* y = out ? out->data_ptr() : fresh.data_ptr();
    Py_BEGIN_ALLOW_THREADS
    s = us_spmm(static_cast<us_handle*>(h), X->data_ptr(), (int32_t)N, xs, y, st);
    Py_END_ALLOW_THREADS
    if (s != US_OK) return fail(s, "us_spmm");
    if (out) {
        Py_INCREF(a[5]);
        return a[5];
    }
    return THPVariable_Wrap(std::move(fresh));
    END_HANDLE_TH_ERRORS
}

// spmm_requant(handle, M, K, X16, N, x_amax, out, y_amax, m0, m1, stream) -> the output tensor
PyObject* spmm_requant(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 11) return PyErr_Format(PyExc_TypeError, "spmm_requant takes 11 arguments");
    HANDLE_TH_ERRORS
    void *h = nullptr, *xa = nullptr, *ya = nullptr, *st = nullptr;
    if (a[0] != Py_None) h = PyLong_AsVoidPtr(a[0]);
    const int64_t M = PyLong_AsLongLong(a[1]), K = PyLong_AsLongLong(a[2]), N = PyLong_AsLongLong(a[4]);
    const int64_t m0 = PyLong_AsLongLong(a[8]), m1 = PyLong_AsLongLong(a[9]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor* X = tensor(a[3], "X16");
    if (!X || !pointer(a[5], "x_amax", &xa) || !pointer(a[7], "y_amax", &ya) || !stream_of(a[10], *X, &st)) return nullptr;
    if (!is_f16_rows(*X) || X->size(1) != K)
        return PyErr_Format(PyExc_AssertionError, "X16 must be a float16 (N, K) tensor with unit column stride");
    if (N < 1 || N > 64) return fail(US_ERR_INVALID_ARG, "us_spmm_requant");
    at::Tensor fresh;
    const at::Tensor* out = nullptr;
    if (a[6] != Py_None) {
        out = tensor(a[6], "out");
        if (!out) return nullptr;
    } else {
        fresh = new_output(*X, N, M, at::kHalf);
    }
    us_status s;
    void* y = out ? out->data_ptr() : fresh.data_ptr();
    const int64_t ldx = X->stride(0);
    Py_BEGIN_ALLOW_THREADS
    s = us_spmm_requant(static_cast<us_handle*>(h), X->data_ptr(), ldx, xa, (int32_t)N, y, ya, m0, m1, st);
    Py_END_ALLOW_THREADS
    if (s != US_OK) return fail(s, "us_spmm_requant");
    if (out) {
        Py_INCREF(a[6]);
        return a[6];
    }
    return THPVariable_Wrap(std::move(fresh));
    END_HANDLE_TH_ERRORS
}

// absmax_f16(X16, amax, stream)
PyObject* absmax_f16(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 3) return PyErr_Format(PyExc_TypeError, "absmax_f16 takes 3 arguments");
    HANDLE_TH_ERRORS
    void *am = nullptr, *st = nullptr;
    const at::Tensor* X = tensor(a[0], "X16");
    if (!X || !pointer(a[1], "amax", &am) || !stream_of(a[2], *X, &st)) return nullptr;
    if (!is_f16_rows(*X)) return PyErr_Format(PyExc_AssertionError, "X16 must be a float16 (N, K) tensor with unit column stride");
    const int64_t N = X->size(0);
    if (N < 1 || N > 64) return fail(US_ERR_INVALID_ARG, "us_absmax_f16");
    us_status s;
    Py_BEGIN_ALLOW_THREADS
    s = us_absmax_f16(X->data_ptr(), X->stride(0), (int32_t)N, X->size(1), am, st);
    Py_END_ALLOW_THREADS
    if (s != US_OK) return fail(s, "us_absmax_f16");
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// ---- MX4 ----

// What a call runs on: the device of its first tensor made current, and the stream. A stream that the caller names becomes the current
// one for the call, so that scratch and results come from its memory.
struct Place {
    std::optional<c10::cuda::CUDAGuard> device;
    std::optional<c10::cuda::CUDAStreamGuard> guard;
    void* stream = nullptr;
    bool enter(PyObject* st, const at::Tensor& on)
    {
        if (!on.is_cuda()) {
            PyErr_SetString(PyExc_ValueError, "expected a tensor on a CUDA device");
            return false;
        }
        device.emplace(on.device());
        if (!stream_of(st, on, &stream)) return false;
        if (stream != (void*)c10::cuda::getCurrentCUDAStream(on.device().index()).stream())
            guard.emplace(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(stream), on.device().index()));
        return true;
    }
};

int type_of(at::ScalarType t) { return t == at::kHalf ? US_F16 : t == at::kBFloat16 ? US_BF16 : t == at::kFloat ? US_F32 : -1; }

// Rows of a float type with unit column stride.
bool is_rows(const at::Tensor& t)
{
    return t.dim() == 2 && type_of(t.scalar_type()) >= 0 && (t.stride(1) == 1 || t.size(1) <= 1) && t.size(1) >= 1 &&
           (t.size(0) <= 1 || t.stride(0) >= t.size(1));
}
bool is_byte_rows(const at::Tensor& t, int64_t cols)
{
    return t.dim() == 2 && t.scalar_type() == at::kByte && t.size(1) == cols && (t.stride(1) == 1 || cols == 1) && (t.size(0) <= 1 || t.stride(0) >= cols);
}
// The tiles of a matrix: its bytes, on the device of `on`.
bool is_mx(const at::Tensor& t, int64_t rows, int64_t K, const at::Tensor& on)
{
    return t.scalar_type() == at::kByte && t.is_contiguous() && t.device() == on.device() && us_mx4_bytes(rows, K) >= 0 && t.numel() == us_mx4_bytes(rows, K);
}
PyObject* bad(const char* text)
{
    PyErr_SetString(PyExc_ValueError, text);
    return nullptr;
}
// The type asked for: None gives `otherwise`.
bool dtype_of(PyObject* o, at::ScalarType otherwise, at::ScalarType* out)
{
    *out = otherwise;
    if (o == Py_None) return true;
    if (!THPDtype_Check(o)) {
        PyErr_SetString(PyExc_TypeError, "dtype must be a torch.dtype");
        return false;
    }
    *out = reinterpret_cast<THPDtype*>(o)->scalar_type;
    if (type_of(*out) < 0) {
        PyErr_SetString(PyExc_ValueError, "dtype must be float16, bfloat16 or float32");
        return false;
    }
    return true;
}
// The caller's (rows, cols) output, or a new one of the type asked for.
const at::Tensor* rows_out(PyObject* o, PyObject* dtype, at::ScalarType otherwise, const at::Tensor& on, int64_t rows, int64_t cols, at::Tensor* fresh)
{
    at::ScalarType type;
    if (!dtype_of(dtype, otherwise, &type)) return nullptr;
    if (o == Py_None) {
        *fresh = new_output(on, rows, cols, type);
        return fresh;
    }
    const at::Tensor* t = tensor(o, "out");
    if (!t) return nullptr;
    if (!is_rows(*t) || t->size(0) != rows || t->size(1) != cols || t->device() != on.device() || (dtype != Py_None && t->scalar_type() != type)) {
        PyErr_Format(PyExc_ValueError, "out must be a (%lld, %lld) float tensor with unit column stride on the inputs' device", (long long)rows, (long long)cols);
        return nullptr;
    }
    return t;
}
int64_t row_stride(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }
PyObject* give(PyObject* o, at::Tensor&& fresh)
{
    if (o == Py_None) return THPVariable_Wrap(std::move(fresh));
    Py_INCREF(o);
    return o;
}

// mx4_quantize(X, mx, stream) -> (the tiles, rows, K)
PyObject* mx4_quantize(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 3) return PyErr_Format(PyExc_TypeError, "mx4_quantize takes 3 arguments");
    HANDLE_TH_ERRORS
    const at::Tensor* X = tensor(a[0], "X");
    if (!X) return nullptr;
    if (!is_rows(*X)) return bad("X must be a float16, bfloat16 or float32 (rows, K) tensor with unit column stride");
    const int64_t rows = X->size(0), K = X->size(1);
    Place at_;
    if (!at_.enter(a[2], *X)) return nullptr;
    at::Tensor fresh;
    const at::Tensor* mx = &fresh;
    if (a[1] == Py_None) {
        const int64_t bytes = us_mx4_bytes(rows, K);
        if (bytes < 0) return fail(US_ERR_INVALID_ARG, "us_mx4_quantize");
        fresh = at::detail::empty_cuda({bytes}, at::kByte, X->device(), std::nullopt);
    } else {
        mx = tensor(a[1], "out");
        if (!mx) return nullptr;
        if (!is_mx(*mx, rows, K, *X)) return bad("out does not hold a matrix of X's shape on X's device");
    }
    us_status s;
    Py_BEGIN_ALLOW_THREADS
    s = us_mx4_quantize(X->data_ptr(), type_of(X->scalar_type()), row_stride(*X), rows, K, mx->data_ptr(), at_.stream);
    Py_END_ALLOW_THREADS
    if (s != US_OK) return fail(s, "us_mx4_quantize");
    PyObject* tiles = give(a[1], std::move(fresh));
    return tiles ? Py_BuildValue("NLL", tiles, (long long)rows, (long long)K) : nullptr;
    END_HANDLE_TH_ERRORS
}

// mx4_dequantize(mx, rows, K, dtype, out, stream) -> the values
PyObject* mx4_dequantize(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 6) return PyErr_Format(PyExc_TypeError, "mx4_dequantize takes 6 arguments");
    HANDLE_TH_ERRORS
    const at::Tensor* mx = tensor(a[0], "data");
    const int64_t rows = PyLong_AsLongLong(a[1]), K = PyLong_AsLongLong(a[2]);
    if (!mx || PyErr_Occurred()) return nullptr;
    Place at_;
    if (!at_.enter(a[5], *mx)) return nullptr;
    if (!is_mx(*mx, rows, K, *mx)) return bad("data does not hold a matrix of this shape");
    at::Tensor fresh;
    const at::Tensor* out = rows_out(a[4], a[3], at::kFloat, *mx, rows, K, &fresh);
    if (!out) return nullptr;
    us_status s;
    Py_BEGIN_ALLOW_THREADS
    s = us_mx4_dequantize(mx->data_ptr(), rows, K, out->data_ptr(), type_of(out->scalar_type()), row_stride(*out), at_.stream);
    Py_END_ALLOW_THREADS
    if (s != US_OK) return fail(s, "us_mx4_dequantize");
    return give(a[4], std::move(fresh));
    END_HANDLE_TH_ERRORS
}

// mx4_pack(codes, scales, K, stream) -> the tiles
PyObject* mx4_pack(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 4) return PyErr_Format(PyExc_TypeError, "mx4_pack takes 4 arguments");
    HANDLE_TH_ERRORS
    const at::Tensor *codes = tensor(a[0], "codes"), *scales = codes ? tensor(a[1], "scales") : nullptr;
    const int64_t K = PyLong_AsLongLong(a[2]);
    if (!scales || PyErr_Occurred()) return nullptr;
    if (K < 1 || K > (1ll << 30) || !is_byte_rows(*codes, (K + 1) / 2) || !is_byte_rows(*scales, (K + 31) / 32) || codes->size(0) != scales->size(0) ||
        codes->device() != scales->device())
        return bad("codes and scales must be uint8 (rows, ceil(K/2)) and (rows, ceil(K/32)) tensors with unit column stride on one device");
    const int64_t rows = codes->size(0), bytes = us_mx4_bytes(rows, K);
    if (bytes < 0) return fail(US_ERR_INVALID_ARG, "us_mx4_pack");
    Place at_;
    if (!at_.enter(a[3], *codes)) return nullptr;
    at::Tensor mx = at::detail::empty_cuda({bytes}, at::kByte, codes->device(), std::nullopt);
    us_status s;
    Py_BEGIN_ALLOW_THREADS
    s = us_mx4_pack(codes->data_ptr(), row_stride(*codes), scales->data_ptr(), row_stride(*scales), rows, K, mx.data_ptr(), at_.stream);
    Py_END_ALLOW_THREADS
    if (s != US_OK) return fail(s, "us_mx4_pack");
    return THPVariable_Wrap(std::move(mx));
    END_HANDLE_TH_ERRORS
}

// mx4_unpack(mx, rows, K, stream) -> (codes, scales)
PyObject* mx4_unpack(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 4) return PyErr_Format(PyExc_TypeError, "mx4_unpack takes 4 arguments");
    HANDLE_TH_ERRORS
    const at::Tensor* mx = tensor(a[0], "data");
    const int64_t rows = PyLong_AsLongLong(a[1]), K = PyLong_AsLongLong(a[2]);
    if (!mx || PyErr_Occurred()) return nullptr;
    Place at_;
    if (!at_.enter(a[3], *mx)) return nullptr;
    if (!is_mx(*mx, rows, K, *mx)) return bad("data does not hold a matrix of this shape");
    at::Tensor codes = new_output(*mx, rows, (K + 1) / 2, at::kByte), scales = new_output(*mx, rows, (K + 31) / 32, at::kByte);
    us_status s;
    Py_BEGIN_ALLOW_THREADS
    s = us_mx4_unpack(mx->data_ptr(), rows, K, codes.data_ptr(), (K + 1) / 2, scales.data_ptr(), (K + 31) / 32, at_.stream);
    Py_END_ALLOW_THREADS
    if (s != US_OK) return fail(s, "us_mx4_unpack");
    PyObject *c = THPVariable_Wrap(std::move(codes)), *sc = THPVariable_Wrap(std::move(scales));
    return Py_BuildValue("NN", c, sc);
    END_HANDLE_TH_ERRORS
}

// mx4_linear(X, rows, w, M, K, out, dtype, stable, stream) -> the product; rows >= 0: X holds the tiles of that many rows
PyObject* mx4_linear(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 9) return PyErr_Format(PyExc_TypeError, "mx4_linear takes 9 arguments");
    HANDLE_TH_ERRORS
    const at::Tensor *X = tensor(a[0], "X"), *w = X ? tensor(a[2], "w") : nullptr;
    const int64_t rows = PyLong_AsLongLong(a[1]), M = PyLong_AsLongLong(a[3]), K = PyLong_AsLongLong(a[4]);
    if (!w || PyErr_Occurred()) return nullptr;
    Place at_;
    if (!at_.enter(a[8], *X)) return nullptr;
    if (!is_mx(*w, M, K, *X)) return bad("w does not hold a matrix of this shape on X's device");
    if (rows >= 0 ? !is_mx(*X, rows, K, *X) : (!is_rows(*X) || X->size(1) != K))
        return bad("X must be a float16, bfloat16 or float32 (N, K) tensor with unit column stride, K as the weight's");
    const int64_t N = rows >= 0 ? rows : X->size(0);
    at::Tensor fresh, scratch;
    const at::Tensor* out = rows_out(a[5], a[6], rows >= 0 ? at::kHalf : X->scalar_type(), *X, N, M, &fresh);
    if (!out) return nullptr;
    const uint32_t flags = a[7] == Py_True ? US_MX4_W_STABLE : 0u;
    const int yt = type_of(out->scalar_type());
    const int64_t ldy = row_stride(*out);
    void* y = out->data_ptr();
    us_status s;
    if (rows >= 0) {
        Py_BEGIN_ALLOW_THREADS
        s = us_mx4_matmul(X->data_ptr(), N, w->data_ptr(), M, K, y, yt, ldy, flags, at_.stream);
        Py_END_ALLOW_THREADS
    } else {
        const int64_t bytes = us_mx4_linear_scratch(N, M, K);
        if (bytes > 0) scratch = at::detail::empty_cuda({bytes}, at::kByte, X->device(), std::nullopt);
        Py_BEGIN_ALLOW_THREADS
        s = us_mx4_linear(X->data_ptr(), type_of(X->scalar_type()), row_stride(*X), N, w->data_ptr(), M, K, y, yt, ldy,
                          bytes > 0 ? scratch.data_ptr() : nullptr, bytes, flags, at_.stream);
        Py_END_ALLOW_THREADS
    }
    if (s != US_OK) return fail(s, "us_mx4_linear");
    return give(a[5], std::move(fresh));
    END_HANDLE_TH_ERRORS
}

// ---- the 8-bit cache ----

bool is_ints(const at::Tensor& t, const at::Tensor& on) { return t.scalar_type() == at::kInt && t.device() == on.device(); }

// A batch of sequences from (block_table, lengths, cu_tokens); N: the call's rows, or -1 where it has none.
bool take_seqs(PyObject* table, PyObject* lengths, PyObject* cu, int64_t N, const at::Tensor& on, us_kv_seqs* q)
{
    const at::Tensor *t = tensor(table, "block_table"), *l = t ? tensor(lengths, "lengths") : nullptr;
    if (!l) return false;
    if (t->dim() != 2 || !is_ints(*t, on) || (t->stride(1) != 1 && t->size(1) > 1) || (t->size(0) > 1 && t->stride(0) < t->size(1)) || t->size(0) >= (1ll << 31) ||
        t->size(1) >= (1ll << 31)) {
        PyErr_SetString(PyExc_ValueError, "block_table must be an int32 (sequences, width) tensor with unit column stride on the cache's device");
        return false;
    }
    if (l->dim() != 1 || !is_ints(*l, on) || l->size(0) != t->size(0) || !l->is_contiguous()) {
        PyErr_SetString(PyExc_ValueError, "lengths must be a contiguous int32 tensor with an entry for each row of block_table, on the cache's device");
        return false;
    }
    *q = us_kv_seqs{};
    q->block_table = static_cast<const int32_t*>(t->data_ptr());
    q->table_stride = row_stride(*t);
    q->lengths = static_cast<const int32_t*>(l->data_ptr());
    q->n_seqs = (int32_t)t->size(0);
    q->table_width = (int32_t)t->size(1);
    if (cu == Py_None) {
        if (N >= 0 && N != t->size(0)) {
            PyErr_SetString(PyExc_ValueError, "without cu_tokens there is one row for each sequence");
            return false;
        }
        return true;
    }
    const at::Tensor* c = tensor(cu, "cu_tokens");
    if (!c) return false;
    if (c->dim() != 1 || !is_ints(*c, on) || c->size(0) != t->size(0) + 1 || !c->is_contiguous()) {
        PyErr_SetString(PyExc_ValueError, "cu_tokens must be a contiguous int32 tensor with one entry more than block_table has rows, on the cache's device");
        return false;
    }
    q->cu_tokens = static_cast<const int32_t*>(c->data_ptr());
    return true;
}
// (N, heads, D) rows of a float type, any token and head strides that do not overlap.
bool is_heads(const at::Tensor& t, int64_t D, const at::Tensor& on)
{
    return t.dim() == 3 && type_of(t.scalar_type()) >= 0 && t.size(2) == D && t.stride(2) == 1 && t.device() == on.device() &&
           (t.size(0) <= 1 || t.stride(0) >= D) && (t.size(1) <= 1 || t.stride(1) >= D);
}
int64_t token_stride(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : 0; }
int64_t head_stride(const at::Tensor& t) { return t.size(1) > 1 ? t.stride(1) : 0; }

// kv_append(handle, pool, k, v, table, lengths, cu, stream)
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 8) return PyErr_Format(PyExc_TypeError, "kv_append takes 8 arguments");
    HANDLE_TH_ERRORS
    void* h = a[0] == Py_None ? nullptr : PyLong_AsVoidPtr(a[0]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor *pool = tensor(a[1], "pool"), *k = pool ? tensor(a[2], "k") : nullptr, *v = k ? tensor(a[3], "v") : nullptr;
    if (!v) return nullptr;
    if (!h) return fail(US_ERR_INVALID_ARG, "us_kv_append");
    Place at_;
    if (!at_.enter(a[7], *pool)) return nullptr;
    if (!is_heads(*k, pool->size(3), *pool) || !is_heads(*v, pool->size(3), *pool) || k->size(1) != pool->size(1) || v->size(1) != pool->size(1) ||
        k->size(0) != v->size(0) || k->scalar_type() != v->scalar_type())
        return bad("k and v must be (N, n_kv_heads, head_dim) tensors of one type (float16, bfloat16 or float32) with unit last stride on the cache's device");
    us_kv_seqs q;
    if (!take_seqs(a[4], a[5], a[6], k->size(0), *pool, &q)) return nullptr;
    us_status s;
    Py_BEGIN_ALLOW_THREADS
    s = us_kv_append(static_cast<us_kv*>(h), &q, k->size(0), k->data_ptr(), v->data_ptr(), type_of(k->scalar_type()), token_stride(*k), head_stride(*k),
                     token_stride(*v), head_stride(*v), at_.stream);
    Py_END_ALLOW_THREADS
    if (s != US_OK) return fail(s, "us_kv_append");
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// kv_read(handle, pool, table, lengths, tokens, dtype, stream) -> (K, V)
PyObject* kv_read(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 7) return PyErr_Format(PyExc_TypeError, "kv_read takes 7 arguments");
    HANDLE_TH_ERRORS
    void* h = a[0] == Py_None ? nullptr : PyLong_AsVoidPtr(a[0]);
    const int64_t tokens = PyLong_AsLongLong(a[4]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor* pool = tensor(a[1], "pool");
    if (!pool) return nullptr;
    if (!h || tokens < 0) return fail(US_ERR_INVALID_ARG, "us_kv_read");
    at::ScalarType type;
    if (!dtype_of(a[5], at::kFloat, &type)) return nullptr;
    Place at_;
    if (!at_.enter(a[6], *pool)) return nullptr;
    us_kv_seqs q;
    if (!take_seqs(a[2], a[3], Py_None, -1, *pool, &q)) return nullptr;
    if (tokens > (int64_t)q.table_width * pool->size(2)) return fail(US_ERR_INVALID_ARG, "us_kv_read");
    const int64_t shape[4] = {q.n_seqs, tokens, pool->size(1), pool->size(3)};
    at::Tensor K = at::detail::empty_cuda(shape, type, pool->device(), std::nullopt), V = at::detail::empty_cuda(shape, type, pool->device(), std::nullopt);
    us_status s;
    Py_BEGIN_ALLOW_THREADS
    s = us_kv_read(static_cast<us_kv*>(h), &q, tokens, K.data_ptr(), V.data_ptr(), type_of(type), at_.stream);
    Py_END_ALLOW_THREADS
    if (s != US_OK) return fail(s, "us_kv_read");
    PyObject *k = THPVariable_Wrap(std::move(K)), *v = THPVariable_Wrap(std::move(V));
    return Py_BuildValue("NN", k, v);
    END_HANDLE_TH_ERRORS
}

// kv_attention(handle, pool, q, table, lengths, cu, scale, causal, window, out, lse, stream) -> out
PyObject* kv_attention(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 12) return PyErr_Format(PyExc_TypeError, "kv_attention takes 12 arguments");
    HANDLE_TH_ERRORS
    void* h = a[0] == Py_None ? nullptr : PyLong_AsVoidPtr(a[0]);
    const double scale = PyFloat_AsDouble(a[6]);
    const int causal = PyObject_IsTrue(a[7]);
    const int64_t window = PyLong_AsLongLong(a[8]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor *pool = tensor(a[1], "pool"), *Q = pool ? tensor(a[2], "q") : nullptr;
    if (!Q) return nullptr;
    if (!h) return fail(US_ERR_INVALID_ARG, "us_kv_attention");
    Place at_;
    if (!at_.enter(a[11], *pool)) return nullptr;
    if (!is_heads(*Q, pool->size(3), *pool) || Q->scalar_type() == at::kFloat || Q->size(1) < 1 || Q->size(1) % pool->size(1) || Q->size(1) >= (1ll << 31))
        return bad("q must be a float16 or bfloat16 (N, n_heads, head_dim) tensor, n_heads a multiple of n_kv_heads, with unit last stride on the cache's device");
    if (window < 0 || window > 0x7FFFFFFF) return bad("window must be 0 (none) or a number of tokens");
    const int64_t N = Q->size(0), H = Q->size(1), D = Q->size(2);
    us_kv_seqs q;
    if (!take_seqs(a[3], a[4], a[5], N, *pool, &q)) return nullptr;
    at::Tensor fresh, scratch;
    const at::Tensor* out = &fresh;
    if (a[9] == Py_None) {
        const int64_t shape[3] = {N, H, D};
        fresh = at::detail::empty_cuda(shape, Q->scalar_type(), pool->device(), std::nullopt);
    } else {
        out = tensor(a[9], "out");
        if (!out) return nullptr;
        if (!is_heads(*out, D, *pool) || out->scalar_type() != Q->scalar_type() || out->size(0) != N || out->size(1) != H)
            return bad("out must be a tensor of q's shape and type with unit last stride on the cache's device");
    }
    void* lse = nullptr;
    if (a[10] != Py_None) {
        const at::Tensor* l = tensor(a[10], "lse");
        if (!l) return nullptr;
        if (l->dim() != 2 || l->scalar_type() != at::kFloat || l->size(0) != N || l->size(1) != H || !l->is_contiguous() || l->device() != pool->device())
            return bad("lse must be a contiguous float32 (N, n_heads) tensor on the cache's device");
        lse = l->data_ptr();
    }
    const int64_t bytes = us_kv_attention_scratch(static_cast<us_kv*>(h), &q, N, (int32_t)H);
    if (bytes < 0) return fail(US_ERR_INVALID_ARG, "us_kv_attention");
    if (bytes > 0) scratch = at::detail::empty_cuda({bytes}, at::kByte, pool->device(), std::nullopt);
    us_status s;
    Py_BEGIN_ALLOW_THREADS
    s = us_kv_attention(static_cast<us_kv*>(h), &q, N, Q->data_ptr(), type_of(Q->scalar_type()), (int32_t)H, token_stride(*Q), head_stride(*Q), (float)scale,
                        causal, (int32_t)window, out->data_ptr(), token_stride(*out), head_stride(*out), static_cast<float*>(lse),
                        bytes > 0 ? scratch.data_ptr() : nullptr, bytes, at_.stream);
    Py_END_ALLOW_THREADS
    if (s != US_OK) return fail(s, "us_kv_attention");
    return give(a[9], std::move(fresh));
    END_HANDLE_TH_ERRORS
}

PyObject* set_error(PyObject*, PyObject* cls)
{
    Py_XDECREF(g_error);
    Py_INCREF(cls);
    g_error = cls;
    Py_RETURN_NONE;
}

template <class F>
PyCFunction fast(F* f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef methods[] = {
    {"spmm", fast(spmm), METH_FASTCALL, nullptr},
    {"spmm_requant", fast(spmm_requant), METH_FASTCALL, nullptr},
    {"absmax_f16", fast(absmax_f16), METH_FASTCALL, nullptr},
    {"mx4_quantize", fast(mx4_quantize), METH_FASTCALL, nullptr},
    {"mx4_dequantize", fast(mx4_dequantize), METH_FASTCALL, nullptr},
    {"mx4_pack", fast(mx4_pack), METH_FASTCALL, nullptr},
    {"mx4_unpack", fast(mx4_unpack), METH_FASTCALL, nullptr},
    {"mx4_linear", fast(mx4_linear), METH_FASTCALL, nullptr},
    {"kv_append", fast(kv_append), METH_FASTCALL, nullptr},
    {"kv_read", fast(kv_read), METH_FASTCALL, nullptr},
    {"kv_attention", fast(kv_attention), METH_FASTCALL, nullptr},
    {"set_error", set_error, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_us_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__us_torch() { return PyModule_Create(&module); }
