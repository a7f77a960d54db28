// Argument marshalling of the calls that a decoder makes per layer and token (residual + norm + quantizer, cache
// append, read, attention): the functions of the same names in binding.py pass their arguments here.  The work
// of such a call takes the device 3 us or so, and the checks, allocations and the foreign call took 12 to 14 us in Python
// (one token of 4096: 12.1 us there, 5.6 us here).  Nothing is computed or kept here.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <cmath>
#include <initializer_list>
#include <string>

#include "w4a8.h"

namespace {

PyObject *g_status_error, *g_memory_error;     // W4A8Error(status, what); torch's exception of a full device

struct Refusal {                   // a Python exception to be
    PyObject *type;
    std::string text;
};
struct Raised {};                  // one that is set already
[[noreturn]] void wrong_type(const std::string &t) { throw Refusal{PyExc_TypeError, t}; }
[[noreturn]] void wrong_value(const std::string &t) { throw Refusal{PyExc_ValueError, t}; }

const at::Tensor &tensor(PyObject *o, const char *what)
{
    if (!THPVariable_Check(o)) wrong_type(std::string(what) + ": expected a tensor");
    return THPVariable_Unpack(o);
}
const at::Tensor &of_type(PyObject *o, at::ScalarType type, const char *what)
{
    const at::Tensor &t = tensor(o, what);
    if (!t.is_cuda() || t.scalar_type() != type || !t.is_contiguous())
        wrong_type(std::string(what) + ": expected a contiguous CUDA tensor of " + c10::toString(type));
    return t;
}
const at::Tensor *maybe(PyObject *o, at::ScalarType type, const char *what)
{
    return o == Py_None ? nullptr : &of_type(o, type, what);
}
const at::Tensor &of_16_bits(PyObject *o, const char *what, bool contiguous = true)
{
    const at::Tensor &t = tensor(o, what);
    if (!t.is_cuda() || (t.scalar_type() != at::kHalf && t.scalar_type() != at::kBFloat16) || (contiguous && !t.is_contiguous()))
        wrong_type(std::string(what) + ": expected a CUDA tensor of float16 or bfloat16" + (contiguous ? ", contiguous" : ""));
    return t;
}
int dtype_of(const at::Tensor &t)
{
    return t.scalar_type() == at::kHalf ? W4A8_F16 : t.scalar_type() == at::kBFloat16 ? W4A8_BF16 : W4A8_F32;
}
at::ScalarType scalar_type(PyObject *o, const char *what)
{
    if (!THPDtype_Check(o)) wrong_type(std::string(what) + ": expected a torch dtype");
    return reinterpret_cast<THPDtype *>(o)->scalar_type;
}
void shaped(const at::Tensor &t, at::IntArrayRef shape, const char *what)
{
    if (t.sizes() == shape) return;
    std::string s = std::string(what) + ": expected shape (";
    for (size_t i = 0; i < shape.size(); ++i) s += (i ? ", " : "") + std::to_string(shape[i]);
    s += "), got (";
    for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
    wrong_value(s + ")");
}
int number(int64_t v, const char *what)
{
    if (v < INT_MIN || v > INT_MAX) wrong_value(std::string(what) + ": out of range");
    return (int)v;
}
int integer(PyObject *o, const char *what)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised();
    return number(v, what);
}
float real(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised();
    return (float)v;
}
// The stream of the current device, on which all the tensors live: the library launches there.
void *stream_of(const char *call, std::initializer_list<const at::Tensor *> tensors)
{
    const auto at = c10::cuda::current_device();
    for (const at::Tensor *t : tensors)
        if (t && t->get_device() != at)
            wrong_value(std::string(call) + ": tensor on " + t->device().str() + ", current device is cuda:" + std::to_string((int)at));
    return c10::cuda::getCurrentCUDAStream(at).stream();
}
// An uninitialised tensor straight from the device's allocator: through the dispatcher each takes 0.3 us longer.
at::Tensor fresh(at::IntArrayRef shape, at::ScalarType type, const at::Tensor &beside)
{
    return at::Tensor(at::detail::empty_cuda(shape, type, beside.device(), std::nullopt));
}
void *at_or_null(const at::Tensor *t) { return t ? t->data_ptr() : nullptr; }
void check(w4a8_status status, const char *what)
{
    if (status == W4A8_OK) return;
    PyObject *e = PyObject_CallFunction(g_status_error, "is", (int)status, what);
    if (e) {
        PyErr_SetObject(g_status_error, e);
        Py_DECREF(e);
    }
    throw Raised();
}
PyObject *own(PyObject *given, const at::Tensor &t)
{
    if (given != Py_None) {
        Py_INCREF(given);
        return given;
    }
    PyObject *o = THPVariable_Wrap(t);
    if (!o) throw Raised();
    return o;
}
// A tuple that takes over its parts.
template <int N>
PyObject *tuple(PyObject *(&parts)[N])
{
    PyObject *t = PyTuple_New(N);
    if (!t) throw Raised();
    for (int i = 0; i < N; ++i) PyTuple_SET_ITEM(t, i, parts[i]);
    return t;
}

template <class F>
PyObject *guarded(F &&body)
{
    try {
        return body();
    } catch (const Raised &) {
    } catch (const Refusal &r) {
        PyErr_SetString(r.type, r.text.c_str());
    } catch (const c10::OutOfMemoryError &e) {
        PyErr_SetString(g_memory_error, e.what_without_backtrace());
    } catch (const c10::Error &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}
bool counted(const char *what, Py_ssize_t n, Py_ssize_t want)
{
    if (n != want) PyErr_Format(PyExc_TypeError, "%s: expected %zd arguments, got %zd", what, want, n);
    return n == want;
}

// What the cache calls share.
struct Batch {
    const at::Tensor &cache, &table, &lens, &space;
    const at::Tensor *cu;
    int num_pages, page_size, max_pages, batch;
    Batch(const char *call, PyObject *cache_, PyObject *table_, PyObject *lens_, PyObject *cu_, PyObject *space_, int64_t heads, int64_t D)
        : cache(of_type(cache_, at::kByte, "cache")), table(of_type(table_, at::kInt, "page_table")), lens(of_type(lens_, at::kInt, "kv_lens")),
          space(of_type(space_, at::kByte, "workspace")), cu(maybe(cu_, at::kInt, "cu_rows"))
    {
        if (table.dim() != 2) wrong_value("page_table: expected [batch, max_pages]");
        if (cache.dim() != 2) wrong_value("cache: expected [num_pages, page_bytes]");
        batch = number(table.size(0), "page_table");
        max_pages = number(table.size(1), "page_table");
        shaped(lens, {table.size(0)}, "kv_lens");
        if (cu) shaped(*cu, {table.size(0) + 1}, "cu_rows");
        num_pages = number(cache.size(0), "cache");
        const int64_t bytes = cache.size(1), slot = heads * (D + 8);          // bytes of a token, all heads
        if (slot <= 0 || bytes % slot || bytes / slot > INT_MAX || heads > INT_MAX || D > INT_MAX ||
            (size_t)bytes != w4a8_kv_page_bytes((int)(bytes / slot), (int)heads, (int)D))
            wrong_value(std::string(call) + ": pages of " + std::to_string(bytes) + " bytes do not hold " + std::to_string(heads) + " heads of " +
                        std::to_string(D));
        page_size = (int)(bytes / slot);
    }
    const int32_t *table_at() const { return static_cast<const int32_t *>(table.data_ptr()); }
    const int32_t *lens_at() const { return static_cast<const int32_t *>(lens.data_ptr()); }
    const int32_t *cu_at() const { return static_cast<const int32_t *>(at_or_null(cu)); }
};

// [rows, heads, D] whose rows may be slices of wider ones: the row stride in elements.
int64_t row_stride(const at::Tensor &t, const char *what)
{
    if (t.dim() != 3 || t.stride(2) != 1 || (t.size(1) > 1 && t.stride(1) != t.size(2)))
        wrong_type(std::string(what) + ": expected [rows, heads, D] with contiguous heads");
    // the stride of a dimension of one row has no meaning
    return t.size(0) > 1 ? t.stride(0) : t.size(1) * t.size(2);
}

// X, residual, norm_weight, norm_bias, kind, eps, residual_out, Xq, tok_scale
PyObject *add_norm_quantize_act(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (!counted("add_norm_quantize_act", n, 9)) return nullptr;
    return guarded([&] {
        const at::Tensor &X = of_16_bits(v[0], "X");
        const at::Tensor &any = tensor(v[1], "residual");
        const at::ScalarType type = any.scalar_type();
        if (type != at::kHalf && type != at::kBFloat16 && type != at::kFloat) wrong_type("residual: expected float16, bfloat16 or float32");
        const at::Tensor &residual = of_type(v[1], type, "residual"), &weight = of_type(v[2], at::kFloat, "norm_weight");
        const at::Tensor *bias = maybe(v[3], at::kFloat, "norm_bias");
        if (X.dim() != 2) wrong_value("X: expected [M, K]");
        const int64_t M = X.size(0), K = X.size(1);
        shaped(residual, X.sizes(), "residual");
        shaped(weight, {K}, "norm_weight");
        if (bias) shaped(*bias, {K}, "norm_bias");
        const int kind = integer(v[4], "kind");
        const float eps = real(v[5]);
        const at::Tensor sum = v[6] == Py_None ? fresh({M, K}, residual.scalar_type(), residual) : of_type(v[6], type, "residual_out");
        const at::Tensor q = v[7] == Py_None ? fresh({M, K}, at::kChar, X) : of_type(v[7], at::kChar, "Xq");
        const at::Tensor tok = v[8] == Py_None ? fresh({M}, at::kFloat, X) : of_type(v[8], at::kFloat, "tok_scale");
        shaped(sum, X.sizes(), "residual_out");
        shaped(q, X.sizes(), "Xq");
        shaped(tok, {M}, "tok_scale");
        void *st = stream_of("add_norm_quantize_act", {&X, &residual, &weight, bias, &sum, &q, &tok});
        const int m = number(M, "X"), k = number(K, "X");
        w4a8_status status;
        Py_BEGIN_ALLOW_THREADS
        status = w4a8_add_norm_quantize_act(X.data_ptr(), dtype_of(X), residual.data_ptr(), dtype_of(residual), sum.data_ptr(),
                                            static_cast<const float *>(weight.data_ptr()), static_cast<const float *>(at_or_null(bias)), kind,
                                            eps, m, k, static_cast<int8_t *>(q.data_ptr()), static_cast<float *>(tok.data_ptr()), st);
        Py_END_ALLOW_THREADS
        check(status, "w4a8_add_norm_quantize_act");
        PyObject *out[3] = {own(v[7], q), own(v[8], tok), own(v[6], sum)};
        return tuple(out);
    });
}

// K, V, cache, page_table, kv_lens, workspace, cu_rows
PyObject *kv_append(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (!counted("kv_append", n, 7)) return nullptr;
    return guarded([&] {
        const at::Tensor &K = of_16_bits(v[0], "K", false), &V = of_16_bits(v[1], "V", false);
        const int64_t ks = row_stride(K, "K"), vs = row_stride(V, "V");
        if (K.scalar_type() != V.scalar_type()) wrong_type("V: expected the type of K");
        shaped(V, K.sizes(), "V");
        const Batch b("kv_append", v[2], v[3], v[4], v[6], v[5], K.size(1), K.size(2));
        void *st = stream_of("kv_append", {&b.cache, &b.table, &b.lens, b.cu, &b.space, &K, &V});
        const int rows = number(K.size(0), "K");
        w4a8_status status;
        Py_BEGIN_ALLOW_THREADS
        status = w4a8_kv_append(K.data_ptr(), V.data_ptr(), dtype_of(K), ks, vs, b.cache.data_ptr(), b.num_pages, b.page_size, (int)K.size(1),
                                (int)K.size(2), b.table_at(), b.max_pages, b.lens_at(), b.cu_at(), b.batch, rows, b.space.data_ptr(),
                                b.space.numel(), st);
        Py_END_ALLOW_THREADS
        check(status, "w4a8_kv_append");
        Py_RETURN_NONE;
    });
}

// cache, page_table, kv_lens, rows, kv_heads, head_dim, workspace, cu_rows, dtype, K, V
PyObject *kv_read(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (!counted("kv_read", n, 11)) return nullptr;
    return guarded([&] {
        const int rows = integer(v[3], "rows"), heads = integer(v[4], "kv_heads"), D = integer(v[5], "head_dim");
        const Batch b("kv_read", v[0], v[1], v[2], v[7], v[6], heads, D);
        const at::ScalarType type = scalar_type(v[8], "dtype");
        if (type != at::kHalf && type != at::kBFloat16) wrong_type("dtype: expected float16 or bfloat16");
        if (rows < 0) wrong_value("rows: negative");
        auto space = [&](PyObject *given, const char *what) {
            return given == Py_None ? fresh({rows, heads, D}, type, b.cache) : of_16_bits(given, what);
        };
        const at::Tensor K = space(v[9], "K"), V = space(v[10], "V");
        if (K.scalar_type() != V.scalar_type()) wrong_type("out: expected two tensors of one type");
        shaped(K, {rows, heads, D}, "out");
        shaped(V, {rows, heads, D}, "out");
        void *st = stream_of("kv_read", {&b.cache, &b.table, &b.lens, b.cu, &b.space, &K, &V});
        w4a8_status status;
        Py_BEGIN_ALLOW_THREADS
        status = w4a8_kv_read(b.cache.data_ptr(), b.num_pages, b.page_size, heads, D, b.table_at(), b.max_pages, b.lens_at(), b.cu_at(), b.batch,
                              rows, K.data_ptr(), V.data_ptr(), dtype_of(K), b.space.data_ptr(), b.space.numel(), st);
        Py_END_ALLOW_THREADS
        check(status, "w4a8_kv_read");
        PyObject *out[2] = {own(v[9], K), own(v[10], V)};
        return tuple(out);
    });
}

// Q, cache, page_table, kv_lens, kv_heads, workspace, cu_rows, scale, causal, window, dtype, out, lse
PyObject *kv_attention(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (!counted("kv_attention", n, 13)) return nullptr;
    return guarded([&] {
        const at::Tensor &Q = of_16_bits(v[0], "Q", false);
        const int64_t stride = row_stride(Q, "Q"), D = Q.size(2);
        const int heads = integer(v[4], "kv_heads");
        const Batch b("kv_attention", v[1], v[2], v[3], v[6], v[5], heads, D);
        const float scale = v[7] == Py_None ? (float)std::pow((double)D, -0.5) : real(v[7]);
        const int causal = PyObject_IsTrue(v[8]), window = integer(v[9], "window");
        if (causal < 0) throw Raised();
        const at::ScalarType type = scalar_type(v[10], "dtype");
        if (v[11] == Py_None && type != at::kHalf && type != at::kBFloat16) wrong_type("dtype: expected float16 or bfloat16");
        if (v[11] != Py_None) shaped(tensor(v[11], "out"), Q.sizes(), "out");
        const at::Tensor O = v[11] == Py_None ? fresh(Q.sizes(), type, Q) : of_16_bits(v[11], "out");
        const at::Tensor *lse = maybe(v[12], at::kFloat, "lse");
        if (lse) shaped(*lse, {Q.size(0), Q.size(1)}, "lse");
        void *st = stream_of("kv_attention", {&b.cache, &b.table, &b.lens, b.cu, &b.space, &Q, &O, lse});
        const int rows = number(Q.size(0), "Q"), q_heads = number(Q.size(1), "Q");
        w4a8_status status;
        Py_BEGIN_ALLOW_THREADS
        status = w4a8_kv_attention(Q.data_ptr(), dtype_of(Q), stride, b.cache.data_ptr(), b.num_pages, b.page_size, heads, (int)D, b.table_at(),
                                   b.max_pages, b.lens_at(), b.cu_at(), b.batch, rows, q_heads, scale, causal, window, O.data_ptr(),
                                   dtype_of(O), static_cast<float *>(at_or_null(lse)), b.space.data_ptr(), b.space.numel(), st);
        Py_END_ALLOW_THREADS
        check(status, "w4a8_kv_attention");
        return own(v[11], O);
    });
}

PyObject *set_errors(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (!counted("set_errors", n, 2)) return nullptr;
    Py_INCREF(v[0]);
    Py_XSETREF(g_status_error, v[0]);
    Py_INCREF(v[1]);
    Py_XSETREF(g_memory_error, v[1]);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"add_norm_quantize_act", (PyCFunction)(void (*)(void))add_norm_quantize_act, METH_FASTCALL, nullptr},
    {"kv_append", (PyCFunction)(void (*)(void))kv_append, METH_FASTCALL, nullptr},
    {"kv_read", (PyCFunction)(void (*)(void))kv_read, METH_FASTCALL, nullptr},
    {"kv_attention", (PyCFunction)(void (*)(void))kv_attention, METH_FASTCALL, nullptr},
    {"set_errors", (PyCFunction)(void (*)(void))set_errors, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls()
{
    PyObject *m = PyModule_Create(&module_def);
    if (m && PyModule_AddStringConstant(m, "built_for", W4A8_BUILT_FOR) != 0) Py_CLEAR(m);
    return m;
}
