// Argument marshalling of the calls that a decoder makes per layer and token (residual + norm + quantizer, cache
// append, read, attention, rotary positions, accepted paths) and of a step's plan: the functions of the same names in binding.py pass their arguments here.  The work
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

// What the three attention calls share: their arguments in the places of `v` that they name.
struct Attention {
    const at::Tensor &Q;
    const int64_t stride, D;
    const int heads;
    const Batch b;
    const float scale;
    at::Tensor O;
    const at::Tensor *lse;
    void *st;
    int rows, q_heads;
    Attention(const char *call, PyObject *Q_, PyObject *cache, PyObject *table, PyObject *lens, PyObject *heads_, PyObject *space, PyObject *cu,
              PyObject *scale_, PyObject *dtype, PyObject *out, PyObject *lse_, const at::Tensor *mask = nullptr)
        : Q(of_16_bits(Q_, "Q", false)), stride(row_stride(Q, "Q")), D(Q.size(2)), heads(integer(heads_, "kv_heads")),
          b(call, cache, table, lens, cu, space, heads, D), scale(scale_ == Py_None ? (float)std::pow((double)D, -0.5) : real(scale_))
    {
        const at::ScalarType type = scalar_type(dtype, "dtype");
        if (out == Py_None && type != at::kHalf && type != at::kBFloat16) wrong_type("dtype: expected float16 or bfloat16");
        if (out != Py_None) shaped(tensor(out, "out"), Q.sizes(), "out");
        O = out == Py_None ? fresh(Q.sizes(), type, Q) : of_16_bits(out, "out");
        lse = maybe(lse_, at::kFloat, "lse");
        if (lse) shaped(*lse, {Q.size(0), Q.size(1)}, "lse");
        st = stream_of(call, {&b.cache, &b.table, &b.lens, b.cu, &b.space, &Q, &O, lse, mask});
        rows = number(Q.size(0), "Q");
        q_heads = number(Q.size(1), "Q");
    }
    float *lse_at() const { return static_cast<float *>(at_or_null(lse)); }
};

// Q, cache, page_table, kv_lens, kv_heads, workspace, window, sinks, cu_rows, scale, causal, dtype, out, lse
PyObject *kv_attention_sinks(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (!counted("kv_attention_sinks", n, 14)) return nullptr;
    return guarded([&] {
        const int window = integer(v[6], "window"), sinks = integer(v[7], "sinks"), causal = PyObject_IsTrue(v[10]);
        if (causal < 0) throw Raised();
        const Attention a("kv_attention_sinks", v[0], v[1], v[2], v[3], v[4], v[5], v[8], v[9], v[11], v[12], v[13]);
        const Batch &b = a.b;
        w4a8_status status;
        Py_BEGIN_ALLOW_THREADS
        status = w4a8_kv_attention_sinks(a.Q.data_ptr(), dtype_of(a.Q), a.stride, b.cache.data_ptr(), b.num_pages, b.page_size, a.heads, (int)a.D,
                                         b.table_at(), b.max_pages, b.lens_at(), b.cu_at(), b.batch, a.rows, a.q_heads, a.scale, causal, window,
                                         sinks, a.O.data_ptr(), dtype_of(a.O), a.lse_at(), b.space.data_ptr(), b.space.numel(), a.st);
        Py_END_ALLOW_THREADS
        check(status, "w4a8_kv_attention_sinks");
        return own(v[12], a.O);
    });
}

// Q, cache, page_table, kv_lens, kv_heads, workspace, tree_mask, cu_rows, scale, window, sinks, dtype, out, lse
PyObject *kv_attention_tree(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (!counted("kv_attention_tree", n, 14)) return nullptr;
    return guarded([&] {
        const at::Tensor &mask = of_type(v[6], at::kInt, "tree_mask");
        if (mask.dim() != 2) wrong_value("tree_mask: expected [rows, words]");
        const int window = integer(v[9], "window"), sinks = integer(v[10], "sinks"), words = number(mask.size(1), "tree_mask");
        const Attention a("kv_attention_tree", v[0], v[1], v[2], v[3], v[4], v[5], v[7], v[8], v[11], v[12], v[13], &mask);
        shaped(mask, {a.Q.size(0), mask.size(1)}, "tree_mask");
        const Batch &b = a.b;
        w4a8_status status;
        Py_BEGIN_ALLOW_THREADS
        status = w4a8_kv_attention_tree(a.Q.data_ptr(), dtype_of(a.Q), a.stride, b.cache.data_ptr(), b.num_pages, b.page_size, a.heads, (int)a.D,
                                        b.table_at(), b.max_pages, b.lens_at(), b.cu_at(), b.batch, a.rows, a.q_heads, a.scale,
                                        static_cast<const uint32_t *>(mask.data_ptr()), words, window, sinks, a.O.data_ptr(), dtype_of(a.O),
                                        a.lse_at(), b.space.data_ptr(), b.space.numel(), a.st);
        Py_END_ALLOW_THREADS
        check(status, "w4a8_kv_attention_tree");
        return own(v[12], a.O);
    });
}

// cache, page_table, kv_lens, accepted, accept_lens, kv_heads, head_dim, workspace, cu_rows, out, kept
PyObject *kv_accept(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (!counted("kv_accept", n, 11)) return nullptr;
    return guarded([&] {
        const int heads = integer(v[5], "kv_heads"), D = integer(v[6], "head_dim");
        const Batch b("kv_accept", v[0], v[1], v[2], v[8], v[7], heads, D);
        const at::Tensor &accepted = of_type(v[3], at::kInt, "accepted"), &lens = of_type(v[4], at::kInt, "accept_lens");
        if (accepted.dim() != 2 || accepted.size(0) != b.batch) wrong_value("accepted: expected [batch, max_accept]");
        const at::Tensor *kept = maybe(v[10], at::kInt, "kept");
        shaped(lens, {b.batch}, "accept_lens");
        if (kept) shaped(*kept, {b.batch}, "kept");
        const at::Tensor out = v[9] == Py_None ? fresh({b.batch}, at::kInt, b.lens) : of_type(v[9], at::kInt, "out");
        shaped(out, {b.batch}, "out");
        void *st = stream_of("kv_accept", {&b.cache, &b.table, &b.lens, b.cu, &b.space, &accepted, &lens, kept, &out});
        // (no row of the call is read here: with cu_rows any number of them will do)
        const int most = number(accepted.size(1), "accepted"), rows = b.cu ? INT_MAX / heads : b.batch;
        w4a8_status status;
        Py_BEGIN_ALLOW_THREADS
        status = w4a8_kv_accept_ex(b.cache.data_ptr(), b.num_pages, b.page_size, heads, D, b.table_at(), b.max_pages, b.lens_at(), b.cu_at(), b.batch, rows,
                                   static_cast<const int32_t *>(accepted.data_ptr()), most, static_cast<const int32_t *>(lens.data_ptr()),
                                   static_cast<const int32_t *>(at_or_null(kept)), static_cast<int32_t *>(out.data_ptr()), b.space.data_ptr(),
                                   b.space.numel(), st);
        Py_END_ALLOW_THREADS
        check(status, "w4a8_kv_accept");
        return own(v[9], out);
    });
}

// Q, K, V, positions, inv_freq, cache, slots, workspace, pair_axis, interleaved, out
PyObject *rope_kv_append(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (!counted("rope_kv_append", n, 11)) return nullptr;
    return guarded([&] {
        const at::Tensor &Q = of_16_bits(v[0], "Q", false), &K = of_16_bits(v[1], "K", false), &V = of_16_bits(v[2], "V", false);
        const int64_t qs = row_stride(Q, "Q"), ks = row_stride(K, "K"), vs = row_stride(V, "V"), rows = Q.size(0), D = Q.size(2), heads = K.size(1);
        if (K.scalar_type() != Q.scalar_type() || V.scalar_type() != Q.scalar_type()) wrong_type("Q, K, V: expected one type");
        shaped(K, {rows, heads, D}, "K");
        shaped(V, K.sizes(), "V");
        const at::Tensor &positions = of_type(v[3], at::kInt, "positions"), &freq = of_type(v[4], at::kFloat, "inv_freq");
        if (positions.dim() != 1 && positions.dim() != 2) wrong_value("positions: expected [rows] or [axes, rows]");
        const int64_t axes = positions.dim() == 2 ? positions.size(0) : 1;
        if (positions.size(-1) != rows) wrong_value("positions: expected [rows] or [axes, rows]");
        if (freq.dim() != 1) wrong_value("inv_freq: expected [rotary_dim / 2]");
        const at::Tensor &cache = of_type(v[5], at::kByte, "cache"), &slots = of_type(v[6], at::kLong, "slots"), &space = of_type(v[7], at::kByte, "workspace");
        const at::Tensor *axis = maybe(v[8], at::kInt, "pair_axis");
        const int interleaved = PyObject_IsTrue(v[9]);
        if (interleaved < 0) throw Raised();
        if (axis) shaped(*axis, freq.sizes(), "pair_axis");
        shaped(slots, {rows}, "slots");
        if (cache.dim() != 2) wrong_value("cache: expected [num_pages, page_bytes]");
        const int64_t bytes = cache.size(1), token = heads * (D + 8);
        if (token <= 0 || bytes % token || bytes / token > INT_MAX || heads > INT_MAX || D > INT_MAX ||
            (size_t)bytes != w4a8_kv_page_bytes((int)(bytes / token), (int)heads, (int)D))
            wrong_value("rope_kv_append: pages of " + std::to_string(bytes) + " bytes do not hold " + std::to_string(heads) + " heads of " + std::to_string(D));
        if (v[10] != Py_None) shaped(tensor(v[10], "out"), Q.sizes(), "out");
        const at::Tensor out = v[10] == Py_None ? fresh(Q.sizes(), Q.scalar_type(), Q) : of_16_bits(v[10], "out", false);
        if (out.scalar_type() != Q.scalar_type()) wrong_type("out: expected the type of Q");
        const int64_t os = row_stride(out, "out");
        void *st = stream_of("rope_kv_append", {&Q, &K, &V, &positions, &freq, &cache, &slots, &space, axis, &out});
        const int r = number(rows, "Q"), q_heads = number(Q.size(1), "Q"), rotary = number(2 * freq.size(0), "inv_freq"), pages = number(cache.size(0), "cache"),
                  n_axes = number(axes, "positions");
        w4a8_status status;
        Py_BEGIN_ALLOW_THREADS
        status = w4a8_rope_kv_append(Q.data_ptr(), K.data_ptr(), V.data_ptr(), dtype_of(Q), qs, ks, vs, static_cast<const int32_t *>(positions.data_ptr()), n_axes,
                                     static_cast<const int32_t *>(at_or_null(axis)), static_cast<const float *>(freq.data_ptr()), rotary, interleaved,
                                     out.data_ptr(), os, cache.data_ptr(), pages, (int)(bytes / token), (int)heads, (int)D,
                                     static_cast<const int64_t *>(slots.data_ptr()), r, q_heads, space.data_ptr(), space.numel(), st);
        Py_END_ALLOW_THREADS
        check(status, "w4a8_rope_kv_append");
        return own(v[10], out);
    });
}

// held, kv_lens, add, page_table, free_pages, free_count, page_size, rows, workspace, kv_lens_out, cu_rows, positions, slots, free_count_out
PyObject *kv_plan(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (!counted("kv_plan", n, 14)) return nullptr;
    return guarded([&] {
        const at::Tensor *held = maybe(v[0], at::kInt, "held");
        const at::Tensor &lens = of_type(v[1], at::kInt, "kv_lens"), &add = of_type(v[2], at::kInt, "add"), &table = of_type(v[3], at::kInt, "page_table"),
                         &pages = of_type(v[4], at::kInt, "free_pages"), &count = of_type(v[5], at::kInt, "free_count"),
                         &space = of_type(v[8], at::kByte, "workspace");
        const int page_size = integer(v[6], "page_size"), rows = integer(v[7], "rows");
        if (rows < 0) wrong_value("rows: negative");
        if (table.dim() != 2) wrong_value("page_table: expected [batch, max_pages]");
        const int batch = number(table.size(0), "page_table"), max_pages = number(table.size(1), "page_table");
        shaped(lens, {batch}, "kv_lens");
        shaped(add, {batch}, "add");
        if (held) shaped(*held, {batch}, "held");
        if (pages.dim() != 1) wrong_value("free_pages: expected [num_pages]");
        const int num_pages = number(pages.size(0), "free_pages");
        shaped(count, {1}, "free_count");
        auto space_of = [&](PyObject *given, int64_t size, at::ScalarType type, const char *what) {
            const at::Tensor t = given == Py_None ? fresh({size}, type, lens) : of_type(given, type, what);
            shaped(t, {size}, what);
            return t;
        };
        const at::Tensor new_lens = space_of(v[9], batch, at::kInt, "kv_lens_out"), cu = space_of(v[10], (int64_t)batch + 1, at::kInt, "cu_rows"),
                         pos = space_of(v[11], rows, at::kInt, "positions"), slots = space_of(v[12], rows, at::kLong, "slots"),
                         left = space_of(v[13], 1, at::kInt, "free_count_out");
        void *st = stream_of("kv_plan", {held, &lens, &add, &table, &pages, &count, &space, &new_lens, &cu, &pos, &slots, &left});
        auto ints = [](const at::Tensor &t) { return static_cast<int32_t *>(t.data_ptr()); };
        w4a8_status status;
        Py_BEGIN_ALLOW_THREADS
        status = w4a8_kv_plan(held ? ints(*held) : nullptr, ints(lens), ints(add), batch, ints(table), max_pages, page_size, ints(pages), num_pages,
                              ints(count), ints(left), ints(new_lens), ints(cu), ints(pos), static_cast<int64_t *>(slots.data_ptr()), rows,
                              space.data_ptr(), space.numel(), st);
        Py_END_ALLOW_THREADS
        check(status, "w4a8_kv_plan");
        PyObject *out[5] = {own(v[9], new_lens), own(v[10], cu), own(v[11], pos), own(v[12], slots), own(v[13], left)};
        return tuple(out);
    });
}

// Q, cache, page_table, kv_lens, kv_heads, workspace, cu_rows, scale, causal, window, dtype, out, lse
PyObject *kv_attention(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (!counted("kv_attention", n, 13)) return nullptr;
    return guarded([&] {
        const int causal = PyObject_IsTrue(v[8]), window = integer(v[9], "window");
        if (causal < 0) throw Raised();
        const Attention a("kv_attention", v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7], v[10], v[11], v[12]);
        const Batch &b = a.b;
        w4a8_status status;
        Py_BEGIN_ALLOW_THREADS
        status = w4a8_kv_attention(a.Q.data_ptr(), dtype_of(a.Q), a.stride, b.cache.data_ptr(), b.num_pages, b.page_size, a.heads, (int)a.D, b.table_at(),
                                   b.max_pages, b.lens_at(), b.cu_at(), b.batch, a.rows, a.q_heads, a.scale, causal, window, a.O.data_ptr(),
                                   dtype_of(a.O), a.lse_at(), b.space.data_ptr(), b.space.numel(), a.st);
        Py_END_ALLOW_THREADS
        check(status, "w4a8_kv_attention");
        return own(v[11], a.O);
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
    {"kv_attention_sinks", (PyCFunction)(void (*)(void))kv_attention_sinks, METH_FASTCALL, nullptr},
    {"kv_attention_tree", (PyCFunction)(void (*)(void))kv_attention_tree, METH_FASTCALL, nullptr},
    {"kv_accept", (PyCFunction)(void (*)(void))kv_accept, METH_FASTCALL, nullptr},
    {"kv_plan", (PyCFunction)(void (*)(void))kv_plan, METH_FASTCALL, nullptr},
    {"rope_kv_append", (PyCFunction)(void (*)(void))rope_kv_append, METH_FASTCALL, nullptr},
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
