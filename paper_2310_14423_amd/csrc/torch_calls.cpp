// torch_calls.cpp -- the calls of operators.py that run once or more in every step of a caller's model: they check tensors, allocate the
// results and call the C ABI, in a Python extension because the same through ctypes takes longer than the kernels of a few tokens
// (norm of 4 rows 14 us a call, 3 of them on the GPU).  Host code only; nothing is computed here.
//
// Arguments are those of the functions in operators.py, with the stream's address behind.  ValueError for what is checked here; a
// code of the library's other than QSR_OK goes to the function that setup() was given, which raises.
#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "qsr.h"

namespace {

PyObject *g_check, *g_norm, *g_logprobs;       // _check(code, function), and the types of results

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

at::Tensor new_like(const at::Tensor &x, at::ScalarType type) { return at::empty(x.sizes(), x.options().dtype(type)); }
at::Tensor new_rows(const at::Tensor &x, at::ScalarType type, int64_t each = 0)
{
    c10::SmallVector<int64_t, 6> s(x.sizes().begin(), x.sizes().end() - 1);
    if (each) s.push_back(each);
    return at::empty(s, x.options().dtype(type));
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
        if (bytes) ws = at::empty({(int64_t)bytes}, h.options().dtype(at::kByte));
        a.x_grad = dx.mutable_data_ptr();
        a.weight_grad = (float *)dw.mutable_data_ptr();
        check(qsr_rmsnorm_backward(&a, bytes ? ws.mutable_data_ptr() : nullptr, bytes, stream_of(o[5])), "qsr_rmsnorm_backward");
        return result(nullptr, {wrap(std::move(dx)), wrap(std::move(dw))});
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
        if (bytes) ws = at::empty({(int64_t)bytes}, x.options().dtype(at::kByte));
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

// check, RMSNorm, TokenLogprobs
PyObject *setup(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    return guarded(n, 3, [&] {
        need(PyCallable_Check(o[0]) && PyType_Check(o[1]) && PyType_IsSubtype((PyTypeObject *)o[1], &PyTuple_Type) && PyType_Check(o[2]) &&
                 PyType_IsSubtype((PyTypeObject *)o[2], &PyTuple_Type), "a function and two types of tuples");
        for (int i = 0; i < 3; ++i) Py_INCREF(o[i]);
        g_check = o[0]; g_norm = o[1]; g_logprobs = o[2];
        return none();
    });
}

PyMethodDef methods[] = {
    {"setup", (PyCFunction)(void *)setup, METH_FASTCALL, nullptr},
    {"rmsnorm", (PyCFunction)(void *)rmsnorm, METH_FASTCALL, nullptr},
    {"rmsnorm_backward", (PyCFunction)(void *)rmsnorm_backward, METH_FASTCALL, nullptr},
    {"token_logprobs", (PyCFunction)(void *)token_logprobs, METH_FASTCALL, nullptr},
    {"token_logprobs_backward", (PyCFunction)(void *)token_logprobs_backward, METH_FASTCALL, nullptr},
    {"adamw_step", (PyCFunction)(void *)adamw_step, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void) { return PyModule_Create(&module); }
