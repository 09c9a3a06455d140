// torch_calls.cpp -- the calls of operators.py that run once or more in every step of a caller's model: they check tensors, allocate the
// results and call the C ABI, in a Python extension because the same through ctypes takes longer than the kernels of a few tokens
// (norm of 4 rows 14 us a call, 3 of them on the GPU).  Host code only; nothing is computed here.
//
// Arguments are those of the functions in operators.py, with the stream's address behind.  ValueError for what is checked here; a
// code of the library's other than QSR_OK goes to the function that setup() was given, which raises.
#include <ATen/EmptyTensor.h>
#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <c10/core/Allocator.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "qsr.h"

namespace {

PyObject *g_check, *g_norm, *g_logprobs, *g_layer, *g_scan;    // _check(code, function), and the types of results

struct Bad { const char *what; };
void need(bool ok, const char *what)
{
    if (!ok) throw Bad{what};
}

const at::Tensor &tensor(PyObject *o, const char *what)
{
    need(THPVariable_Check(o), what);
    return THPVariable_Unpack(o);
}
const at::Tensor *maybe(PyObject *o, const char *what) { return o == Py_None ? nullptr : &tensor(o, what); }

// No graph is recorded here: a tensor that asks for a gradient is not taken as one that does not
void unrecorded(std::initializer_list<const at::Tensor *> ts)
{
    if (!at::GradMode::is_enabled()) return;
    for (const at::Tensor *t : ts)
        need(t == nullptr || !t->requires_grad(),
             "a tensor requires a gradient, and no graph is recorded here: call with detached tensors or under torch.no_grad(), and the backward function by hand");
}

// A tensor that was written in place has a new version (tensors of inference mode have none), by which graphs that kept it find out
void written(const at::Tensor &t)
{
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

int type_of(const at::Tensor &t, const char *what)
{
    const at::ScalarType s = t.scalar_type();
    need(s == at::kFloat || s == at::kBFloat16, what);
    return s == at::kFloat ? QSR_TYPE_F32 : QSR_TYPE_BF16;
}

// Elements from row to row of a tensor [..., d] whose rows are dense and evenly spaced
int64_t row_stride(const at::Tensor &t, const char *what)
{
    if (t.is_contiguous()) return t.size(-1);
    need(t.size(-1) == 1 || t.stride(-1) == 1, what);
    int64_t stride = -1, expect = 0;
    for (int64_t i = t.dim() - 2; i >= 0; --i) {
        if (t.size(i) == 1) continue;
        if (stride < 0) stride = t.stride(i);
        else need(t.stride(i) == expect, what);
        expect = t.stride(i) * t.size(i);
    }
    return stride < 0 ? t.size(-1) : stride;
}

// a row argument that goes with the rows x
int64_t like(const at::Tensor &t, const at::Tensor &x, const char *what)
{
    need(t.scalar_type() == x.scalar_type() && t.sizes() == x.sizes() && t.device() == x.device(), what);
    return row_stride(t, what);
}

// float32 numbers, `each` (0: one, without a dimension of its own) for each row of x
const float *numbers(const at::Tensor &t, const at::Tensor &x, int64_t each, const char *what)
{
    const int64_t lead = x.dim() - 1;
    bool ok = t.scalar_type() == at::kFloat && t.is_contiguous() && t.device() == x.device() && t.dim() == lead + (each ? 1 : 0);
    for (int64_t i = 0; ok && i < lead; ++i) ok = t.size(i) == x.size(i);
    need(ok && (!each || t.size(lead) == each), what);
    return (const float *)t.const_data_ptr();
}

// A new tensor on x's device, which is the current one (operators.py), from the allocator that x's memory is from: 0.3 us, where at::empty's
// way through the dispatcher makes it 0.7, with up to ten of them in a call and its backward pass.  Memory from elsewhere has none.
// Dispatch modes do not see it, and torch's deterministic algorithms do not fill it: the library writes all of a result.
at::Tensor fresh(const at::Tensor &x, c10::IntArrayRef size, at::ScalarType type)
{
    c10::Allocator *const allocator = x.storage().unsafeGetStorageImpl()->allocator();
    if (allocator != nullptr) {
        at::Tensor t = at::detail::empty_generic(size, allocator, c10::DispatchKeySet(c10::DispatchKey::CUDA), type, std::nullopt);
        if (t.device() == x.device()) return t;
    }
    return at::empty(size, x.options().dtype(type));
}
at::Tensor new_bytes(const at::Tensor &x, size_t n) { return n ? fresh(x, {(int64_t)n}, at::kByte) : at::Tensor(); }
at::Tensor new_like(const at::Tensor &x, at::ScalarType type) { return fresh(x, x.sizes(), type); }
at::Tensor new_rows(const at::Tensor &x, at::ScalarType type, int64_t each = 0)
{
    c10::SmallVector<int64_t, 6> s(x.sizes().begin(), x.sizes().end() - 1);
    if (each) s.push_back(each);
    return fresh(x, s, type);
}

// Workers, rows of each, and the stride of their weights
void workers(const at::Tensor &x, const at::Tensor &w, int32_t &K, int64_t &rows, int64_t &stride)
{
    need(x.dim() >= 1 && (w.dim() == 1 || w.dim() == 2) && w.size(-1) == x.size(-1) && w.scalar_type() == at::kFloat &&
             (w.size(-1) == 1 || w.stride(-1) == 1) && w.device() == x.device(), "weight: float32 [d] or [K][d], dense, on the rows' device");
    need(w.dim() == 1 || (x.dim() >= 2 && x.size(0) == w.size(0)), "weight [K][d] goes with rows [K][...][d]");
    const int64_t k = w.dim() == 2 ? w.size(0) : 1;
    need(k >= 1 && k <= 65535 && x.size(-1) >= 1, "1 to 65535 workers and at least one element");
    K = (int32_t)k;
    rows = x.numel() / (k * x.size(-1));
    stride = w.dim() == 2 ? w.stride(0) : 0;
}

struct Failed {};
void check(int rc, const char *function)
{
    if (rc == QSR_OK) return;
    PyObject *r = PyObject_CallFunction(g_check, "is", rc, function);
    Py_XDECREF(r);
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, function);
    throw Failed{};
}

// items, whose references are taken over, as one of the named tuples
PyObject *result(PyObject *type, std::initializer_list<PyObject *> items)
{
    PyObject *t = PyTuple_New((Py_ssize_t)items.size());
    Py_ssize_t i = 0;
    for (PyObject *o : items) PyTuple_SET_ITEM(t, i++, o);
    if (type == nullptr) return t;
    PyObject *args = PyTuple_Pack(1, t), *r = PyTuple_Type.tp_new((PyTypeObject *)type, args, nullptr);
    Py_DECREF(args);
    Py_DECREF(t);
    return r;
}
PyObject *none() { Py_INCREF(Py_None); return Py_None; }
PyObject *wrap(at::Tensor t) { return t.defined() ? THPVariable_Wrap(std::move(t)) : none(); }
void *stream_of(PyObject *o) { return PyLong_AsVoidPtr(o); }

template <typename F> PyObject *guarded(Py_ssize_t n, Py_ssize_t want, F f)
{
    HANDLE_TH_ERRORS
    try {
        need(n == want, "number of arguments");
        return f();
    } catch (const Bad &b) {
        PyErr_SetString(PyExc_ValueError, b.what);
    } catch (const Failed &) {
    }
    return nullptr;
    END_HANDLE_TH_ERRORS
}

// x, weight, residual, eps, fp8, sum_out, stream
PyObject *rmsnorm(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return guarded(n, 7, [&] {
        const at::Tensor &x = tensor(o[0], "x"), &w = tensor(o[1], "weight");
        const at::Tensor *res = maybe(o[2], "residual"), *out = maybe(o[5], "sum_out");
        const bool fp8 = o[4] == Py_True;
        unrecorded({&x, &w, res, out});
        qsr_rmsnorm_args a{};
        a.type = type_of(x, "x: float32 or bfloat16");
        a.y_type = fp8 ? QSR_TYPE_E4M3 : a.type;
        workers(x, w, a.K, a.rows, a.weight_stride);
        a.d = a.y_stride = x.size(-1);
        a.eps = PyFloat_AsDouble(o[3]);
        if (PyErr_Occurred()) throw Failed{};
        a.x = x.const_data_ptr();
        a.weight = (const float *)w.const_data_ptr();
        a.x_stride = row_stride(x, "x: rows with one stride, their elements side by side");
        if (res) { a.residual = res->const_data_ptr(); a.residual_stride = like(*res, x, "residual: as x"); }
        at::Tensor sum = out ? *out : res ? new_like(x, x.scalar_type()) : at::Tensor();
        if (sum.defined()) { a.sum = sum.mutable_data_ptr(); a.sum_stride = like(sum, x, "sum_out: as x"); }
        at::Tensor y = new_like(x, fp8 ? at::kFloat8_e4m3fn : x.scalar_type()), rstd = new_rows(x, at::kFloat), scale;
        if (fp8) { scale = new_rows(x, at::kFloat); a.scale = (float *)scale.mutable_data_ptr(); }
        a.y = y.mutable_data_ptr();
        a.rstd = (float *)rstd.mutable_data_ptr();
        check(qsr_rmsnorm(&a, stream_of(o[6])), "qsr_rmsnorm");
        if (out) written(*out);
        PyObject *s;
        if (sum.defined() && !out) s = wrap(std::move(sum));
        else { s = out ? o[5] : o[0]; Py_INCREF(s); }
        return result(g_norm, {wrap(std::move(y)), s, wrap(std::move(rstd)), wrap(std::move(scale))});
    });
}

// y_grad, sum, weight, rstd, residual_grad, stream
PyObject *rmsnorm_backward(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return guarded(n, 6, [&] {
        const at::Tensor &dy = tensor(o[0], "y_grad"), &h = tensor(o[1], "sum"), &w = tensor(o[2], "weight"), &rstd = tensor(o[3], "rstd");
        const at::Tensor *res = maybe(o[4], "residual_grad");
        unrecorded({&dy, &h, &w, &rstd, res});
        qsr_rmsnorm_backward_args a{};
        a.type = type_of(h, "sum: float32 or bfloat16");
        workers(h, w, a.K, a.rows, a.weight_stride);
        a.d = a.x_grad_stride = h.size(-1);
        a.y_grad = dy.const_data_ptr();
        a.y_grad_stride = like(dy, h, "y_grad: as sum");
        a.sum = h.const_data_ptr();
        a.sum_stride = row_stride(h, "sum: rows with one stride, their elements side by side");
        a.weight = (const float *)w.const_data_ptr();
        a.rstd = numbers(rstd, h, 0, "rstd: contiguous float32, one for each row");
        if (res) { a.residual_grad = res->const_data_ptr(); a.residual_grad_stride = like(*res, h, "residual_grad: as sum"); }
        size_t bytes = 0;
        check(qsr_rmsnorm_workspace_bytes(a.K, a.rows, a.d, a.type, &bytes), "qsr_rmsnorm_workspace_bytes");
        at::Tensor ws, dx = new_like(h, h.scalar_type()), dw = new_like(w, at::kFloat);
        ws = new_bytes(h, bytes);
        a.x_grad = dx.mutable_data_ptr();
        a.weight_grad = (float *)dw.mutable_data_ptr();
        check(qsr_rmsnorm_backward(&a, bytes ? ws.mutable_data_ptr() : nullptr, bytes, stream_of(o[5])), "qsr_rmsnorm_backward");
        return result(nullptr, {wrap(std::move(dx)), wrap(std::move(dw))});
    });
}

// x, weight, bias, residual, eps, fp8, sum_out, stream
PyObject *layernorm(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return guarded(n, 8, [&] {
        const at::Tensor &x = tensor(o[0], "x"), &w = tensor(o[1], "weight");
        const at::Tensor *b = maybe(o[2], "bias"), *res = maybe(o[3], "residual"), *out = maybe(o[6], "sum_out");
        const bool fp8 = o[5] == Py_True;
        unrecorded({&x, &w, b, res, out});
        qsr_layernorm_args a{};
        a.type = type_of(x, "x: float32 or bfloat16");
        a.y_type = fp8 ? QSR_TYPE_E4M3 : a.type;
        workers(x, w, a.K, a.rows, a.weight_stride);
        a.d = a.y_stride = x.size(-1);
        a.eps = PyFloat_AsDouble(o[4]);
        if (PyErr_Occurred()) throw Failed{};
        a.x = x.const_data_ptr();
        a.weight = (const float *)w.const_data_ptr();
        a.x_stride = row_stride(x, "x: rows with one stride, their elements side by side");
        if (b) {
            int32_t K;
            int64_t rows;
            need(b->sizes() == w.sizes(), "bias: as weight");
            workers(x, *b, K, rows, a.bias_stride);
            a.bias = (const float *)b->const_data_ptr();
        }
        if (res) { a.residual = res->const_data_ptr(); a.residual_stride = like(*res, x, "residual: as x"); }
        at::Tensor sum = out ? *out : res ? new_like(x, x.scalar_type()) : at::Tensor();
        if (sum.defined()) { a.sum = sum.mutable_data_ptr(); a.sum_stride = like(sum, x, "sum_out: as x"); }
        at::Tensor y = new_like(x, fp8 ? at::kFloat8_e4m3fn : x.scalar_type()), mean = new_rows(x, at::kFloat), rstd = new_rows(x, at::kFloat), scale;
        if (fp8) { scale = new_rows(x, at::kFloat); a.scale = (float *)scale.mutable_data_ptr(); }
        a.y = y.mutable_data_ptr();
        a.mean = (float *)mean.mutable_data_ptr();
        a.rstd = (float *)rstd.mutable_data_ptr();
        check(qsr_layernorm(&a, stream_of(o[7])), "qsr_layernorm");
        if (out) written(*out);
        PyObject *s;
        if (sum.defined() && !out) s = wrap(std::move(sum));
        else { s = out ? o[6] : o[0]; Py_INCREF(s); }
        return result(g_layer, {wrap(std::move(y)), s, wrap(std::move(mean)), wrap(std::move(rstd)), wrap(std::move(scale))});
    });
}

// y_grad, sum, weight, mean, rstd, residual_grad, bias, stream
PyObject *layernorm_backward(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return guarded(n, 8, [&] {
        const at::Tensor &dy = tensor(o[0], "y_grad"), &h = tensor(o[1], "sum"), &w = tensor(o[2], "weight"), &mean = tensor(o[3], "mean"),
                         &rstd = tensor(o[4], "rstd");
        const at::Tensor *res = maybe(o[5], "residual_grad");
        unrecorded({&dy, &h, &w, &mean, &rstd, res});
        qsr_layernorm_backward_args a{};
        a.type = type_of(h, "sum: float32 or bfloat16");
        workers(h, w, a.K, a.rows, a.weight_stride);
        a.d = a.x_grad_stride = h.size(-1);
        a.y_grad = dy.const_data_ptr();
        a.y_grad_stride = like(dy, h, "y_grad: as sum");
        a.sum = h.const_data_ptr();
        a.sum_stride = row_stride(h, "sum: rows with one stride, their elements side by side");
        a.weight = (const float *)w.const_data_ptr();
        a.mean = numbers(mean, h, 0, "mean: contiguous float32, one for each row");
        a.rstd = numbers(rstd, h, 0, "rstd: contiguous float32, one for each row");
        if (res) { a.residual_grad = res->const_data_ptr(); a.residual_grad_stride = like(*res, h, "residual_grad: as sum"); }
        size_t bytes = 0;
        check(qsr_layernorm_workspace_bytes(a.K, a.rows, a.d, a.type, &bytes), "qsr_layernorm_workspace_bytes");
        at::Tensor ws, dx = new_like(h, h.scalar_type()), dw = new_like(w, at::kFloat), db;
        if (o[6] == Py_True) { db = new_like(w, at::kFloat); a.bias_grad = (float *)db.mutable_data_ptr(); }
        ws = new_bytes(h, bytes);
        a.x_grad = dx.mutable_data_ptr();
        a.weight_grad = (float *)dw.mutable_data_ptr();
        check(qsr_layernorm_backward(&a, bytes ? ws.mutable_data_ptr() : nullptr, bytes, stream_of(o[7])), "qsr_layernorm_backward");
        return result(nullptr, {wrap(std::move(dx)), wrap(std::move(dw)), wrap(std::move(db))});
    });
}

// A table [V][d] or [K][V][d] for tokens: workers, tokens of each, and the table's strides
void table_ok(const at::Tensor &t, const at::Tensor &tok, int32_t &K, int64_t &each, int64_t &stride, int64_t &worker, const char *what)
{
    need((t.dim() == 2 || t.dim() == 3) && t.size(-1) >= 1 && t.size(-2) >= 1 && (t.size(-1) == 1 || t.stride(-1) == 1) &&
             (t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16), what);
    need(tok.scalar_type() == at::kLong && tok.is_contiguous() && tok.device() == t.device(), "tokens: contiguous int64, on the table's device");
    need(t.dim() == 2 || (tok.dim() >= 1 && tok.size(0) == t.size(0)), "a table [K][V][d] goes with tokens [K][...]");
    const int64_t k = t.dim() == 3 ? t.size(0) : 1;
    need(k >= 1 && k <= 65535, "1 to 65535 workers");
    K = (int32_t)k;
    each = tok.numel() / k;
    stride = t.size(-2) > 1 ? t.stride(-2) : t.size(-1);
    worker = k > 1 ? t.stride(0) : 0;
}

// tokens, table, scale, type (-1: the table's), stream
PyObject *embedding(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return guarded(n, 5, [&] {
        const at::Tensor &tok = tensor(o[0], "tokens"), &table = tensor(o[1], "table");
        unrecorded({&table});
        qsr_embedding_args a{};
        table_ok(table, tok, a.K, a.tokens_each, a.table_stride, a.worker_stride, "table: float32 or bfloat16 [V][d] or [K][V][d], rows dense");
        a.type = type_of(table, "table");
        a.scale = PyFloat_AsDouble(o[2]);
        const long type = PyLong_AsLong(o[3]);
        if (PyErr_Occurred()) throw Failed{};
        a.y_type = type < 0 ? a.type : (int32_t)type;
        a.vocab = table.size(-2);
        a.d = a.y_stride = table.size(-1);
        c10::SmallVector<int64_t, 6> shape(tok.sizes().begin(), tok.sizes().end());
        shape.push_back(a.d);
        at::Tensor y = fresh(table, shape, a.y_type == QSR_TYPE_F32 ? at::kFloat : at::kBFloat16);
        a.table = table.const_data_ptr();
        a.tokens = (const int64_t *)tok.const_data_ptr();
        a.y = y.mutable_data_ptr();
        check(qsr_embedding(&a, stream_of(o[4])), "qsr_embedding");
        return wrap(std::move(y));
    });
}

// y_grad, tokens, table, scale, out, accumulate, stream
PyObject *embedding_backward(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return guarded(n, 7, [&] {
        const at::Tensor &dy = tensor(o[0], "y_grad"), &tok = tensor(o[1], "tokens"), &table = tensor(o[2], "table");
        const at::Tensor *out = maybe(o[4], "out");
        unrecorded({&dy, out});
        qsr_embedding_backward_args a{};
        int64_t ignored;
        table_ok(table, tok, a.K, a.tokens_each, ignored, ignored, "table: float32 or bfloat16 [V][d] or [K][V][d], rows dense");
        a.vocab = table.size(-2);
        a.d = table.size(-1);
        a.accumulate = o[5] == Py_True;
        a.scale = PyFloat_AsDouble(o[3]);
        if (PyErr_Occurred()) throw Failed{};
        need(!a.accumulate || out != nullptr, "accumulate: a tensor `out` to add to");
        a.type = type_of(dy, "y_grad: float32 or bfloat16");
        bool ok = dy.dim() == tok.dim() + 1 && dy.size(-1) == a.d && dy.device() == table.device();
        for (int64_t i = 0; ok && i < tok.dim(); ++i) ok = dy.size(i) == tok.size(i);
        need(ok, "y_grad: [tokens' shape][d], on the table's device");
        a.y_grad_stride = row_stride(dy, "y_grad: rows with one stride, their elements side by side");
        at::Tensor grad = out ? *out : new_like(table, table.scalar_type());
        need(grad.sizes() == table.sizes() && grad.device() == table.device(), "out: shaped as table, on its device");
        int32_t K;
        int64_t each;
        table_ok(grad, tok, K, each, a.grad_stride, a.worker_stride, "out: float32 or bfloat16, rows dense");
        a.grad_type = type_of(grad, "out");
        size_t bytes = 0;
        check(qsr_embedding_workspace_bytes(a.K, a.tokens_each, a.vocab, a.d, a.type, &bytes), "qsr_embedding_workspace_bytes");
        at::Tensor ws;
        ws = new_bytes(table, bytes);
        a.y_grad = dy.const_data_ptr();
        a.tokens = (const int64_t *)tok.const_data_ptr();
        a.grad = grad.mutable_data_ptr();
        check(qsr_embedding_backward(&a, bytes ? ws.mutable_data_ptr() : nullptr, bytes, stream_of(o[6])), "qsr_embedding_backward");
        if (out) { written(*out); Py_INCREF(o[4]); return o[4]; }
        return wrap(std::move(grad));
    });
}

// Elements from sequence to sequence and from step to step of a tensor [..., T, d] on x's device
void scan_strides(const at::Tensor &t, const at::Tensor &x, int64_t &batch, int64_t &step, const char *what)
{
    need(t.scalar_type() == x.scalar_type() && t.sizes() == x.sizes() && t.device() == x.device() && (t.size(-1) == 1 || t.stride(-1) == 1), what);
    step = t.size(-2) > 1 ? t.stride(-2) : t.size(-1);
    batch = -1;
    int64_t expect = 0;
    for (int64_t i = t.dim() - 3; i >= 0; --i) {
        if (t.size(i) == 1) continue;
        if (batch < 0) batch = t.stride(i);
        else need(t.stride(i) == expect, what);
        expect = t.stride(i) * t.size(i);
    }
    if (batch < 0) batch = t.size(-1);
}

// float32 [..., d] for sequences x [..., T, d]
const float *scan_state(const at::Tensor &t, const at::Tensor &x, const char *what)
{
    bool ok = t.scalar_type() == at::kFloat && t.is_contiguous() && t.device() == x.device() && t.dim() == x.dim() - 1 && t.size(-1) == x.size(-1);
    for (int64_t i = 0; ok && i < x.dim() - 2; ++i) ok = t.size(i) == x.size(i);
    need(ok, what);
    return (const float *)t.const_data_ptr();
}
at::Tensor new_state(const at::Tensor &x, int64_t each = -1)
{
    c10::SmallVector<int64_t, 6> s(x.sizes().begin(), x.sizes().end() - 2);
    if (each >= 0) s.push_back(each);
    s.push_back(x.size(-1));
    return fresh(x, s, at::kFloat);
}

// what both passes have
template <typename Args>
void scan_common(Args &a, const at::Tensor &x, const at::Tensor &gate, const at::Tensor *reset, const at::Tensor *lengths)
{
    a.type = type_of(x, "x: float32 or bfloat16");
    need(x.dim() >= 2 && x.size(-1) >= 1, "x: [..., T, d]");
    a.steps = x.size(-2);
    a.d = x.size(-1);
    a.batch = 1;
    for (int64_t i = 0; i < x.dim() - 2; ++i) a.batch *= x.size(i);
    scan_strides(x, x, a.x_batch_stride, a.x_stride, "x: sequences with one stride, a step's channels side by side");
    scan_strides(gate, x, a.gate_batch_stride, a.gate_stride, "gate: as x");
    a.x = x.const_data_ptr();
    a.gate = gate.const_data_ptr();
    if (reset) {
        bool ok = (reset->scalar_type() == at::kBool || reset->scalar_type() == at::kByte) && reset->is_contiguous() && reset->device() == x.device() &&
                  reset->dim() == x.dim() - 1;
        for (int64_t i = 0; ok && i < x.dim() - 1; ++i) ok = reset->size(i) == x.size(i);
        need(ok, "reset: contiguous bool [..., T]");
        a.reset = (const uint8_t *)reset->const_data_ptr();
    }
    if (lengths) {
        bool ok = lengths->scalar_type() == at::kLong && lengths->is_contiguous() && lengths->device() == x.device() && lengths->dim() == x.dim() - 2;
        for (int64_t i = 0; ok && i < x.dim() - 2; ++i) ok = lengths->size(i) == x.size(i);
        need(ok, "lengths: contiguous int64, one for each sequence");
        a.lengths = (const int64_t *)lengths->const_data_ptr();
    }
}
at::Tensor scan_workspace(const at::Tensor &x, int64_t batch, int64_t steps, int64_t d, int32_t type, size_t &bytes)
{
    check(qsr_gated_scan_workspace_bytes(batch, steps, d, type, &bytes), "qsr_gated_scan_workspace_bytes");
    return new_bytes(x, bytes);
}

// x, gate, initial, reset, lengths, input, keep, state_out, stream
PyObject *gated_scan(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return guarded(n, 9, [&] {
        const at::Tensor &x = tensor(o[0], "x"), &gate = tensor(o[1], "gate");
        const at::Tensor *initial = maybe(o[2], "initial"), *reset = maybe(o[3], "reset"), *lengths = maybe(o[4], "lengths"), *out = maybe(o[7], "state_out");
        unrecorded({&x, &gate, initial, out});
        qsr_gated_scan_args a{};
        scan_common(a, x, gate, reset, lengths);
        a.input = (int32_t)PyLong_AsLong(o[5]);
        if (PyErr_Occurred()) throw Failed{};
        if (initial) a.initial = scan_state(*initial, x, "initial: contiguous float32 [..., d]");
        at::Tensor last = out ? *out : new_state(x), h = new_like(x, x.scalar_type()), states;
        scan_state(last, x, "state_out: contiguous float32 [..., d]");
        a.last = (float *)last.mutable_data_ptr();
        a.h = h.mutable_data_ptr();
        a.h_stride = a.d;
        a.h_batch_stride = a.steps > 0 ? a.steps * a.d : a.d;
        if (o[6] == Py_True) {
            states = new_state(x, (a.steps + QSR_SCAN_STEPS - 1) / QSR_SCAN_STEPS);
            a.states = (float *)states.mutable_data_ptr();
        }
        size_t bytes = 0;
        at::Tensor ws = scan_workspace(x, a.batch, a.steps, a.d, a.type, bytes);
        check(qsr_gated_scan(&a, bytes ? ws.mutable_data_ptr() : nullptr, bytes, stream_of(o[8])), "qsr_gated_scan");
        PyObject *l;
        if (out) { written(*out); l = o[7]; Py_INCREF(l); }
        else l = wrap(std::move(last));
        return result(g_scan, {wrap(std::move(h)), l, wrap(std::move(states))});
    });
}

// h_grad, x, gate, states, reset, lengths, last_grad, input, stream
PyObject *gated_scan_backward(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return guarded(n, 9, [&] {
        const at::Tensor &dh = tensor(o[0], "h_grad"), &x = tensor(o[1], "x"), &gate = tensor(o[2], "gate"), &states = tensor(o[3], "states: those of gated_scan(keep=True)");
        const at::Tensor *reset = maybe(o[4], "reset"), *lengths = maybe(o[5], "lengths"), *end = maybe(o[6], "last_grad");
        unrecorded({&dh, &x, &gate, &states, end});
        qsr_gated_scan_backward_args a{};
        scan_common(a, x, gate, reset, lengths);
        a.input = (int32_t)PyLong_AsLong(o[7]);
        if (PyErr_Occurred()) throw Failed{};
        scan_strides(dh, x, a.h_grad_batch_stride, a.h_grad_stride, "h_grad: as x");
        a.h_grad = dh.const_data_ptr();
        bool ok = states.scalar_type() == at::kFloat && states.is_contiguous() && states.device() == x.device() && states.dim() == x.dim() &&
                  states.size(-1) == a.d && states.size(-2) == (a.steps + QSR_SCAN_STEPS - 1) / QSR_SCAN_STEPS;
        for (int64_t i = 0; ok && i < x.dim() - 2; ++i) ok = states.size(i) == x.size(i);
        need(ok, "states: those of gated_scan(keep=True)");
        a.states = (const float *)states.const_data_ptr();
        if (end) a.last_grad = scan_state(*end, x, "last_grad: contiguous float32 [..., d]");
        at::Tensor dx = new_like(x, x.scalar_type()), dgate = new_like(x, x.scalar_type()), first = new_state(x);
        a.x_grad = dx.mutable_data_ptr();
        a.gate_grad = dgate.mutable_data_ptr();
        a.initial_grad = (float *)first.mutable_data_ptr();
        a.x_grad_stride = a.gate_grad_stride = a.d;
        a.x_grad_batch_stride = a.gate_grad_batch_stride = a.steps > 0 ? a.steps * a.d : a.d;
        size_t bytes = 0;
        at::Tensor ws = scan_workspace(x, a.batch, a.steps, a.d, a.type, bytes);
        check(qsr_gated_scan_backward(&a, bytes ? ws.mutable_data_ptr() : nullptr, bytes, stream_of(o[8])), "qsr_gated_scan_backward");
        return result(nullptr, {wrap(std::move(dx)), wrap(std::move(dgate)), wrap(std::move(first))});
    });
}

void tokens_ok(const at::Tensor &x, const at::Tensor &t)
{
    need(x.dim() >= 1 && x.size(-1) >= 1, "logits: [..., V]");
    bool ok = t.scalar_type() == at::kLong && t.is_contiguous() && t.device() == x.device() && t.dim() == x.dim() - 1;
    for (int64_t i = 0; ok && i < t.dim(); ++i) ok = t.size(i) == x.size(i);
    need(ok, "tokens: contiguous int64, one for each row of logits");
}

// logits, tokens, top, temperature, stream
PyObject *token_logprobs(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return guarded(n, 5, [&] {
        const at::Tensor &x = tensor(o[0], "logits"), &tok = tensor(o[1], "tokens");
        unrecorded({&x});
        qsr_token_logprobs_args a{};
        a.type = type_of(x, "logits: float32 or bfloat16");
        tokens_ok(x, tok);
        const long top = PyLong_AsLong(o[2]);
        a.temperature = PyFloat_AsDouble(o[3]);
        if (PyErr_Occurred()) throw Failed{};
        need(top >= -1 && top <= 1 << 30, "top");
        a.top = (int32_t)top;
        a.vocab = x.size(-1);
        a.rows = x.numel() / a.vocab;
        a.stride = row_stride(x, "logits: rows with one stride, their elements side by side");
        a.logits = x.const_data_ptr();
        a.tokens = (const int64_t *)tok.const_data_ptr();
        size_t bytes = 0;
        check(qsr_token_logprobs_workspace_bytes(a.rows, a.vocab, a.type, a.top, &bytes), "qsr_token_logprobs_workspace_bytes");
        at::Tensor logp = new_rows(x, at::kFloat), entropy = new_rows(x, at::kFloat), lse = new_rows(x, at::kFloat),
                   stats = new_rows(x, at::kFloat, 2), top_logp, top_id, ws;
        a.logp = (float *)logp.mutable_data_ptr();
        a.entropy = (float *)entropy.mutable_data_ptr();
        a.lse = (float *)lse.mutable_data_ptr();
        a.stats = (float *)stats.mutable_data_ptr();
        if (top > 0) {
            top_logp = new_rows(x, at::kFloat, top);
            top_id = new_rows(x, at::kInt, top);
            a.top_logp = (float *)top_logp.mutable_data_ptr();
            a.top_id = (int32_t *)top_id.mutable_data_ptr();
        }
        ws = new_bytes(x, bytes);
        check(qsr_token_logprobs(&a, bytes ? ws.mutable_data_ptr() : nullptr, bytes, stream_of(o[4])), "qsr_token_logprobs");
        return result(g_logprobs, {wrap(std::move(logp)), wrap(std::move(entropy)), wrap(std::move(lse)), wrap(std::move(stats)),
                                   wrap(std::move(top_logp)), wrap(std::move(top_id))});
    });
}

// logits, tokens, stats, entropy, logp_grad, entropy_grad, temperature, out, stream
PyObject *token_logprobs_backward(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return guarded(n, 9, [&] {
        const at::Tensor &x = tensor(o[0], "logits"), &tok = tensor(o[1], "tokens");
        const at::Tensor *ga = maybe(o[4], "logp_grad"), *gb = maybe(o[5], "entropy_grad"), *out = maybe(o[7], "out");
        const at::Tensor &stats = tensor(o[2], "stats"), &entropy = tensor(o[3], "entropy");
        unrecorded({&x, &stats, &entropy, ga, gb, out});
        qsr_token_logprobs_backward_args a{};
        a.type = type_of(x, "logits: float32 or bfloat16");
        tokens_ok(x, tok);
        a.temperature = PyFloat_AsDouble(o[6]);
        if (PyErr_Occurred()) throw Failed{};
        a.vocab = x.size(-1);
        a.rows = x.numel() / a.vocab;
        a.stride = row_stride(x, "logits: rows with one stride, their elements side by side");
        a.logits = x.const_data_ptr();
        a.tokens = (const int64_t *)tok.const_data_ptr();
        a.stats = numbers(stats, x, 2, "stats: contiguous float32 [..., 2]");
        a.entropy = numbers(entropy, x, 0, "entropy: contiguous float32, one for each row");
        if (ga) a.logp_grad = numbers(*ga, x, 0, "logp_grad: contiguous float32, one for each row");
        if (gb) a.entropy_grad = numbers(*gb, x, 0, "entropy_grad: contiguous float32, one for each row");
        at::Tensor grad = out ? *out : new_like(x, x.scalar_type());
        a.grad = grad.mutable_data_ptr();
        a.grad_stride = like(grad, x, "out: as logits");
        check(qsr_token_logprobs_backward(&a, stream_of(o[8])), "qsr_token_logprobs_backward");
        if (out) { written(*out); Py_INCREF(o[7]); return o[7]; }
        return wrap(std::move(grad));
    });
}

// handle, t, eta, stream, a tuple of the tensors that it writes
PyObject *adamw_step(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return guarded(n, 5, [&] {
        need(PyTuple_Check(o[4]), "a tuple of tensors");
        qsr_adamw *const a = (qsr_adamw *)PyLong_AsVoidPtr(o[0]);
        const long long t = PyLong_AsLongLong(o[1]);
        const double eta = PyFloat_AsDouble(o[2]);
        if (PyErr_Occurred()) throw Failed{};
        check(qsr_adamw_step(a, t, eta, stream_of(o[3])), "qsr_adamw_step");
        for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(o[4]); ++i) written(tensor(PyTuple_GET_ITEM(o[4], i), "a tuple of tensors"));
        return none();
    });
}

// check, RMSNorm, TokenLogprobs, LayerNorm, GatedScan
PyObject *setup(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return guarded(n, 5, [&] {
        bool ok = PyCallable_Check(o[0]);
        for (int i = 1; ok && i < 5; ++i) ok = PyType_Check(o[i]) && PyType_IsSubtype((PyTypeObject *)o[i], &PyTuple_Type);
        need(ok, "a function and four types of tuples");
        for (int i = 0; i < 5; ++i) Py_INCREF(o[i]);
        g_check = o[0]; g_norm = o[1]; g_logprobs = o[2]; g_layer = o[3]; g_scan = o[4];
        return none();
    });
}

PyMethodDef methods[] = {
    {"setup", (PyCFunction)(void *)setup, METH_FASTCALL, nullptr},
    {"rmsnorm", (PyCFunction)(void *)rmsnorm, METH_FASTCALL, nullptr},
    {"rmsnorm_backward", (PyCFunction)(void *)rmsnorm_backward, METH_FASTCALL, nullptr},
    {"layernorm", (PyCFunction)(void *)layernorm, METH_FASTCALL, nullptr},
    {"layernorm_backward", (PyCFunction)(void *)layernorm_backward, METH_FASTCALL, nullptr},
    {"embedding", (PyCFunction)(void *)embedding, METH_FASTCALL, nullptr},
    {"embedding_backward", (PyCFunction)(void *)embedding_backward, METH_FASTCALL, nullptr},
    {"gated_scan", (PyCFunction)(void *)gated_scan, METH_FASTCALL, nullptr},
    {"gated_scan_backward", (PyCFunction)(void *)gated_scan_backward, METH_FASTCALL, nullptr},
    {"token_logprobs", (PyCFunction)(void *)token_logprobs, METH_FASTCALL, nullptr},
    {"token_logprobs_backward", (PyCFunction)(void *)token_logprobs_backward, METH_FASTCALL, nullptr},
    {"adamw_step", (PyCFunction)(void *)adamw_step, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void) { return PyModule_Create(&module); }
