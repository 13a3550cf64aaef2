// What embedding.py, norm.py, muon.py, dropout.py and linear.py do for a call - check tensors, make outputs and workspaces, take addresses
// and the stream, call, and leave a node for autograd - on the tensors' C++ objects.  A call on few rows is bound by the
// host: of 13 us for the features of one node, and of 130 us for a step of ten small matrices, the kernels were 4 and 20.
// Tensors that a call does not take as they are (other types, devices or strides, wrong arguments) are left to the Python
// code (by returning NotImplemented), which copies them or knows the error.
#include <ATen/ATen.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <vector>

#include "pcsr_train.h"

namespace {

using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

struct Library {
    decltype(&pcsr_embed) embed;
    decltype(&pcsr_embed_workspace) embed_workspace;
    decltype(&pcsr_embed_backward) embed_backward;
    decltype(&pcsr_norm) norm;
    decltype(&pcsr_norm_workspace) norm_workspace;
    decltype(&pcsr_norm_backward) norm_backward;
    decltype(&pcsr_orthogonalize) orthogonalize;
    decltype(&pcsr_ortho_workspace) ortho_workspace;
    decltype(&pcsr_dropout) dropout;
    decltype(&pcsr_linear) linear;
    decltype(&pcsr_linear_workspace) linear_workspace;
    decltype(&pcsr_linear_backward) linear_backward;
} lib;
bool ready = false;
PyObject *error_type = PyExc_RuntimeError; // what a call of the library that returned an error raises, given the code and the call's name

// Throws that, through autograd's threads too: as torch hands on what Python code raised.
void ok(int rc, const char *where)
{
    if (rc == PCSR_OK) return;
    pybind11::gil_scoped_acquire locked;
    PyObject *e = PyObject_CallFunction(error_type, "is", rc, where);
    if (e) PyErr_SetObject(error_type, e);
    Py_XDECREF(e);
    python_error raised;
    raised.persist();
    throw std::move(raised);
}

int type_of(const at::Tensor &t)
{
    switch (t.scalar_type()) {
    case at::kFloat: return PCSR_F32;
    case at::kBFloat16: return PCSR_BF16;
    case at::kHalf: return PCSR_F16;
    default: return -1;
    }
}
// on the current device, plain memory (numbers as they are stored), without a forward-mode tangent
bool here(const at::Tensor &t)
{
    return t.is_cuda() && t.layout() == at::kStrided && t.device().index() == c10::hip::current_device() && !t.is_neg() && !t._fw_grad(0).defined();
}
void *stream() { return c10::hip::getCurrentHIPStream().stream(); }
at::Tensor bytes(int64_t n, const at::Tensor &like) { return at::empty({n}, like.options().dtype(at::kByte)); }
bool records(const at::Tensor &t) { return t.defined() && t.requires_grad(); }

// distance of the rows of a matrix whose numbers lie one behind the other; -1 otherwise
int64_t distance(const at::Tensor &t)
{
    const int64_t n = t.size(0), d = t.size(1), s = t.stride(0);
    if (t.numel() == 0) return d;
    if ((t.stride(1) != 1 && d > 1) || (s < d && n > 1)) return -1;
    return s > d && n > 1 ? s : d; // (of one row it means nothing)
}

// Gradients of a backward pass that is recorded itself are marked as having none.
variable_list once(variable_list grads)
{
    if (!at::GradMode::is_enabled()) return grads;
    return torch::autograd::DelayedError("this gradient cannot be differentiated",
                                         (int64_t)grads.size())(std::move(grads));
}

// ------------------------------------------------------------------ embedding
at::Tensor embed_forward(const at::Tensor &ids, const at::Tensor &table, double scale)
{
    auto shape = ids.sizes().vec();
    shape.push_back(table.size(1));
    at::Tensor out = at::empty(shape, table.options().requires_grad(false));
    ok(lib.embed(ids.numel(), table.size(0), table.size(1), type_of(table), ids.const_data_ptr(), ids.scalar_type() == at::kLong,
                 table.const_data_ptr(), distance(table), (float)scale, out.data_ptr(), stream()), "pcsr_embed");
    return out;
}

struct Embed : torch::autograd::Function<Embed> {
    static at::Tensor forward(AutogradContext *ctx, const at::Tensor &ids, const at::Tensor &table, double scale)
    {
        ctx->save_for_backward({ids});
        ctx->saved_data["scale"] = scale;
        ctx->saved_data["rows"] = table.size(0);
        return embed_forward(ids, table, scale);
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        const at::Tensor ids = ctx->get_saved_variables()[0];
        const int64_t n = ids.numel(), d = grads[0].size(-1), rows = ctx->saved_data["rows"].toInt();
        at::Tensor g = grads[0].detach().resolve_neg().reshape({n, d});
        if (distance(g) < 0) g = g.contiguous();
        at::Tensor out = at::empty({rows, d}, g.options()), ws = bytes(lib.embed_workspace(n, rows, d), g);
        ok(lib.embed_backward(n, rows, d, type_of(g), ids.const_data_ptr(), ids.scalar_type() == at::kLong, g.const_data_ptr(), distance(g),
                              (float)ctx->saved_data["scale"].toDouble(), out.data_ptr(), ws.data_ptr(), stream()), "pcsr_embed_backward");
        return once({at::Tensor(), out, at::Tensor()});
    }
};

// embed(ids, table, scale)
PyObject *embed(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 3 || !ready || !THPVariable_Check(args[0]) || !THPVariable_Check(args[1]) || !PyFloat_Check(args[2])) Py_RETURN_NOTIMPLEMENTED;
    const at::Tensor &ids = THPVariable_Unpack(args[0]), &table = THPVariable_Unpack(args[1]);
    if (!here(ids) || !here(table) || (ids.scalar_type() != at::kLong && ids.scalar_type() != at::kInt) || !ids.is_contiguous() || table.dim() != 2 ||
        type_of(table) < 0 || table.size(1) < 1 || distance(table) < 0)
        Py_RETURN_NOTIMPLEMENTED;
    const double scale = PyFloat_AS_DOUBLE(args[2]);
    at::Tensor out;
    {
        pybind11::gil_scoped_release unlocked;
        out = at::GradMode::is_enabled() && table.requires_grad() ? Embed::apply(ids, table, scale) : embed_forward(ids, table, scale);
    }
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// ------------------------------------------------------------------ group norm
struct NormCall {
    at::Tensor x; // (rows, channels)
    pcsr_norm_t a;
};
NormCall norm_call(const at::Tensor &X, const at::Tensor &weight, const at::Tensor &bias, const at::Tensor &offsets, const at::Tensor &stats,
                   int64_t groups, double eps, int64_t act)
{
    NormCall c;
    c.x = X.dim() == 2 ? X : X.reshape({-1, X.size(-1)});
    const int64_t graphs = offsets.defined() ? offsets.numel() - 1 : X.dim() == 2 ? 1 : X.size(0);
    const at::Tensor &p = weight.defined() ? weight : bias;
    auto ptr = [](const at::Tensor &t) -> const void * { return t.defined() ? t.const_data_ptr() : nullptr; };
    c.a = {c.x.size(0), c.x.size(1), groups, graphs, ptr(offsets), offsets.defined() && offsets.scalar_type() == at::kLong, type_of(X),
           p.defined() ? type_of(p) : PCSR_F32, (int32_t)act, c.x.const_data_ptr(), distance(c.x), ptr(weight), ptr(bias), (float)eps,
           stats.defined() ? stats.mutable_data_ptr<float>() : nullptr, nullptr};
    if (stats.defined()) c.a.rstd = c.a.mean + graphs * groups;
    return c;
}
at::Tensor norm_forward(const at::Tensor &X, const at::Tensor &weight, const at::Tensor &bias, const at::Tensor &offsets, int64_t groups, double eps,
                        int64_t act, at::Tensor *stats)
{
    const int64_t graphs = offsets.defined() ? offsets.numel() - 1 : X.dim() == 2 ? 1 : X.size(0);
    *stats = at::empty({2, graphs, groups}, X.options().dtype(at::kFloat).requires_grad(false));
    at::Tensor y = at::empty(X.sizes(), X.options().requires_grad(false));
    const NormCall c = norm_call(X, weight, bias, offsets, *stats, groups, eps, act);
    const int64_t need = lib.norm_workspace(&c.a, 0);
    at::Tensor ws;
    if (need) ws = bytes(need, X);
    ok(lib.norm(&c.a, y.data_ptr(), need ? ws.data_ptr() : nullptr, stream()), "pcsr_norm");
    return y;
}

struct Norm : torch::autograd::Function<Norm> {
    static at::Tensor forward(AutogradContext *ctx, const at::Tensor &X, const std::optional<at::Tensor> &weight, const std::optional<at::Tensor> &bias,
                              const std::optional<at::Tensor> &offsets, int64_t groups, double eps, int64_t act)
    {
        auto of = [](const std::optional<at::Tensor> &t) { return t.has_value() ? *t : at::Tensor(); };
        at::Tensor stats, y = norm_forward(X, of(weight), of(bias), of(offsets), groups, eps, act, &stats);
        ctx->save_for_backward({X, of(weight), of(bias), of(offsets), stats});
        ctx->saved_data["groups"] = groups;
        ctx->saved_data["eps"] = eps;
        ctx->saved_data["act"] = act;
        return y;
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        const variable_list saved = ctx->get_saved_variables();
        const at::Tensor X = saved[0].detach();
        auto plain = [](const at::Tensor &t) { return t.defined() ? t.detach() : t; };
        const NormCall c = norm_call(X, plain(saved[1]), plain(saved[2]), saved[3], saved[4], ctx->saved_data["groups"].toInt(),
                                     ctx->saved_data["eps"].toDouble(), ctx->saved_data["act"].toInt());
        at::Tensor g = grads[0].detach().resolve_neg().reshape({c.x.size(0), c.x.size(1)});
        if (distance(g) < 0) g = g.contiguous();
        at::Tensor dx, dw, db, ws; // (tensors that are not there are not counted)
        if (ctx->needs_input_grad(0)) dx = at::empty(X.sizes(), X.options());
        if (saved[1].defined() && ctx->needs_input_grad(1)) dw = at::empty(saved[1].sizes(), saved[1].options().requires_grad(false));
        if (saved[2].defined() && ctx->needs_input_grad(saved[1].defined() ? 2 : 1)) db = at::empty(saved[2].sizes(), saved[2].options().requires_grad(false));
        const int64_t need = lib.norm_workspace(&c.a, 1);
        if (need) ws = bytes(need, X);
        auto ptr = [](const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; };
        ok(lib.norm_backward(&c.a, g.const_data_ptr(), distance(g), ptr(dx), ptr(dw), ptr(db), ptr(ws), stream()), "pcsr_norm_backward");
        return once({dx, dw, db, at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor()});
    }
};

// group_norm(X, groups, weight or None, bias or None, offsets or None, eps, activation's number)
PyObject *group_norm(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 7 || !ready || !THPVariable_Check(args[0]) || !PyLong_CheckExact(args[1]) || !PyFloat_Check(args[5]) || !PyLong_Check(args[6]))
        Py_RETURN_NOTIMPLEMENTED;
    at::Tensor more[3]; // weight, bias, offsets
    for (int k = 0; k < 3; ++k) {
        if (args[2 + k] == Py_None) continue;
        if (!THPVariable_Check(args[2 + k])) Py_RETURN_NOTIMPLEMENTED;
        more[k] = THPVariable_Unpack(args[2 + k]);
        if (!here(more[k]) || more[k].dim() != 1 || !more[k].is_contiguous()) Py_RETURN_NOTIMPLEMENTED;
    }
    const at::Tensor &X = THPVariable_Unpack(args[0]), &w = more[0], &b = more[1], &offsets = more[2];
    const int64_t groups = PyLong_AsLongLong(args[1]), act = PyLong_AsLongLong(args[6]);
    const double eps = PyFloat_AS_DOUBLE(args[5]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        Py_RETURN_NOTIMPLEMENTED;
    }
    if (!here(X) || X.dim() < 2 || type_of(X) < 0 || X.numel() == 0 || (X.dim() == 2 ? distance(X) < 0 : !X.is_contiguous())) Py_RETURN_NOTIMPLEMENTED;
    const int64_t C = X.size(-1);
    if (groups < 1 || C % groups || !(eps >= 0.0) || act < PCSR_ACT_NONE || act > PCSR_ACT_GELU) Py_RETURN_NOTIMPLEMENTED;
    for (const at::Tensor *p : {&w, &b})
        if (p->defined() && (p->numel() != C || (p->scalar_type() != at::kFloat && p->scalar_type() != X.scalar_type()))) Py_RETURN_NOTIMPLEMENTED;
    if (w.defined() && b.defined() && w.scalar_type() != b.scalar_type()) Py_RETURN_NOTIMPLEMENTED;
    if (offsets.defined() && (X.dim() != 2 || offsets.numel() < 2 || (offsets.scalar_type() != at::kLong && offsets.scalar_type() != at::kInt)))
        Py_RETURN_NOTIMPLEMENTED;
    if (C / groups > (type_of(X) == PCSR_F32 ? 2048 : 4096)) Py_RETURN_NOTIMPLEMENTED;
    at::Tensor out, stats;
    {
        pybind11::gil_scoped_release unlocked;
        auto maybe = [](const at::Tensor &t) { return t.defined() ? std::optional<at::Tensor>(t) : std::nullopt; };
        if (at::GradMode::is_enabled() && (records(X) || records(w) || records(b)))
            out = Norm::apply(X, maybe(w), maybe(b), maybe(offsets), groups, eps, act);
        else
            out = norm_forward(X, w, b, offsets, groups, eps, act, &stats);
    }
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// ------------------------------------------------------------------ orthogonalised updates
// update(weights, momenta, lr, steps, address of coefficients, nesterov, momentum, keep): matrices of one type in lists; their gradients
// are what .grad holds.  The library's code, or NotImplemented where one of them is not taken as it is (nothing was done then).
PyObject *update(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 8 || !ready || !PyList_Check(args[0]) || !PyList_Check(args[1])) Py_RETURN_NOTIMPLEMENTED;
    const Py_ssize_t count = PyList_GET_SIZE(args[0]);
    if (PyList_GET_SIZE(args[1]) != count || count == 0) Py_RETURN_NOTIMPLEMENTED;
    pcsr_ortho_t how = {};
    how.steps = (int32_t)PyLong_AsLong(args[3]);
    how.coefficients = static_cast<const double *>(PyLong_AsVoidPtr(args[4]));
    how.update = 1;
    how.nesterov = PyObject_IsTrue(args[5]);
    how.momentum = (float)PyFloat_AsDouble(args[6]);
    how.keep = (float)PyFloat_AsDouble(args[7]);
    const double lr = PyFloat_AsDouble(args[2]);
    if (PyErr_Occurred()) return nullptr;
    std::vector<pcsr_matrix_t> m((size_t)count);
    at::Tensor first;
    for (Py_ssize_t k = 0; k < count; ++k) {
        PyObject *pw = PyList_GET_ITEM(args[0], k), *pb = PyList_GET_ITEM(args[1], k);
        if (!THPVariable_Check(pw) || !THPVariable_Check(pb)) Py_RETURN_NOTIMPLEMENTED;
        const at::Tensor &w = THPVariable_Unpack(pw), &b = THPVariable_Unpack(pb);
        if (k == 0) {
            first = w;
            how.type = type_of(w);
        }
        const at::Tensor &g = w.grad();
        if (!g.defined() || !here(w) || !here(g) || !here(b) || type_of(w) != how.type || type_of(w) < 0 || type_of(g) != how.type || b.scalar_type() != at::kFloat ||
            w.dim() != 2 || w.sizes() != g.sizes() || w.sizes() != b.sizes() || w.numel() == 0)
            Py_RETURN_NOTIMPLEMENTED;
        const int64_t wl = distance(w), gl = distance(g), bl = distance(b);
        const double rate = lr * std::sqrt(std::max(1.0, (double)w.size(0) / (double)w.size(1)));
        if (wl < 0 || gl < 0 || bl < 0) Py_RETURN_NOTIMPLEMENTED;
        m[(size_t)k] = {g.const_data_ptr(), b.mutable_data_ptr<float>(), w.mutable_data_ptr(), w.size(0), w.size(1), gl, bl, wl, (float)rate, 0};
    }
    int rc;
    {
        pybind11::gil_scoped_release unlocked;
        const int64_t need = lib.ortho_workspace(m.data(), count, &how);
        at::Tensor ws;
        if (need) ws = bytes(need, first);
        rc = lib.orthogonalize(m.data(), count, &how, need ? ws.data_ptr() : nullptr, stream());
    }
    for (Py_ssize_t k = 0; k < count; ++k) {
        const at::Tensor &w = THPVariable_Unpack(PyList_GET_ITEM(args[0], k));
        if (!w.is_inference()) w.unsafeGetTensorImpl()->bump_version();
    }
    return PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// orthogonalize(G, steps, address of coefficients)
PyObject *orthogonalize(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 3 || !ready || !THPVariable_Check(args[0])) Py_RETURN_NOTIMPLEMENTED;
    const at::Tensor &G = THPVariable_Unpack(args[0]);
    if (!here(G) || type_of(G) < 0 || (G.dim() != 2 && G.dim() != 3) || G.numel() == 0 || !G.is_contiguous()) Py_RETURN_NOTIMPLEMENTED;
    pcsr_ortho_t how = {};
    how.type = type_of(G);
    how.steps = (int32_t)PyLong_AsLong(args[1]);
    how.coefficients = static_cast<const double *>(PyLong_AsVoidPtr(args[2]));
    if (PyErr_Occurred()) return nullptr;
    const int64_t count = G.dim() == 3 ? G.size(0) : 1, rows = G.size(-2), cols = G.size(-1), size = rows * cols * (int64_t)G.element_size();
    at::Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release unlocked;
        out = at::empty(G.sizes(), G.options().requires_grad(false));
        std::vector<pcsr_matrix_t> m((size_t)count);
        for (int64_t k = 0; k < count; ++k)
            m[(size_t)k] = {static_cast<const char *>(G.const_data_ptr()) + k * size, nullptr, static_cast<char *>(out.mutable_data_ptr()) + k * size, rows, cols,
                            cols, 0, cols, 0.0f, 0};
        const int64_t need = lib.ortho_workspace(m.data(), count, &how);
        at::Tensor ws;
        if (need) ws = bytes(need, G);
        rc = lib.orthogonalize(m.data(), count, &how, need ? ws.data_ptr() : nullptr, stream());
    }
    if (rc != PCSR_OK) return PyLong_FromLong(rc);
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// ------------------------------------------------------------------ dropout and linear layers
struct DropCall {
    double p = 0.0;
    int64_t seed = 0, offset = 0;
    at::Tensor state; // in their place

    // from a call's arguments; false: Python's to look at
    bool take(PyObject *prob, PyObject *s, PyObject *o, const at::Tensor &X)
    {
        if (!PyFloat_Check(prob)) return false;
        p = PyFloat_AS_DOUBLE(prob);
        if (!(p >= 0.0 && p <= 1.0)) return false;
        if (THPVariable_Check(s)) {
            state = THPVariable_Unpack(s);
            return here(state) && state.device() == X.device() && state.scalar_type() == at::kLong && state.dim() == 1 && state.numel() == 2 && state.is_contiguous();
        }
        return word(s, seed) && word(o, offset);
    }
    static bool word(PyObject *v, int64_t &to)
    {
        if (!PyLong_CheckExact(v)) return false;
        int over = 0;
        to = PyLong_AsLongLongAndOverflow(v, &over);
        if (!over) return true;
        if (over < 0) return false;
        to = (int64_t)PyLong_AsUnsignedLongLong(v);
        if (!PyErr_Occurred()) return true;
        PyErr_Clear();
        return false;
    }
    // where a call that reads its seed on the GPU writes what it read, for the backward pass
    at::Tensor used() const { return state.defined() && p > 0.0 ? at::empty({2}, state.options().requires_grad(false)) : at::Tensor(); }
    pcsr_drop_t to_library(const at::Tensor &used) const
    {
        return {p, (uint64_t)seed, (uint64_t)offset, state.defined() ? state.const_data_ptr<int64_t>() : nullptr,
                used.defined() ? used.mutable_data_ptr<int64_t>() : nullptr};
    }
    std::vector<int64_t> numbers() const
    {
        int64_t bits;
        memcpy(&bits, &p, 8);
        return {bits, seed, offset};
    }
    static DropCall of(const std::vector<int64_t> &n, const at::Tensor &used)
    {
        DropCall d;
        memcpy(&d.p, &n[0], 8);
        d.seed = n[1], d.offset = n[2], d.state = used;
        return d;
    }
};
at::Tensor rows(const at::Tensor &t) { return t.dim() == 2 ? t : t.reshape({-1, t.size(-1)}); }
// whether the library takes the rows as they lie
bool whole(const at::Tensor &t) { return t.dim() == 2 ? distance(t) >= 0 : t.is_contiguous(); }
std::optional<at::Tensor> maybe(const at::Tensor &t) { return t.defined() ? std::optional<at::Tensor>(t) : std::nullopt; }
at::Tensor of(const std::optional<at::Tensor> &t) { return t.has_value() ? *t : at::Tensor(); }
at::Tensor gradient_rows(const at::Tensor &grad, int64_t n, int64_t d)
{
    if (grad.dim() == 2 && !grad.is_neg() && distance(grad) >= 0) return grad;
    const at::Tensor g = grad.detach().resolve_neg().reshape({n, d});
    return distance(g) < 0 ? g.contiguous() : g;
}
const void *address(const at::Tensor &t) { return t.defined() ? t.const_data_ptr() : nullptr; }

at::Tensor dropout_forward(const at::Tensor &X, const at::Tensor &R, const DropCall &d, const at::Tensor &used)
{
    at::Tensor out = at::empty(X.sizes(), X.options().requires_grad(false));
    const at::Tensor x = rows(X), r = R.defined() ? rows(R) : R;
    const pcsr_drop_t how = d.to_library(used);
    ok(lib.dropout(x.size(0), x.size(1), type_of(X), x.const_data_ptr(), distance(x), address(r), r.defined() ? distance(r) : 0, &how, out.data_ptr(), stream()),
       "pcsr_dropout");
    return out;
}

struct Dropout : torch::autograd::Function<Dropout> {
    static at::Tensor forward(AutogradContext *ctx, const at::Tensor &X, const std::optional<at::Tensor> &R, const std::optional<at::Tensor> &state,
                              const std::vector<int64_t> &numbers)
    {
        const DropCall d = DropCall::of(numbers, of(state));
        const at::Tensor used = d.used();
        ctx->save_for_backward({used});
        ctx->saved_data["how"] = numbers;
        ctx->saved_data["residual"] = R.has_value();
        return dropout_forward(X, of(R), d, used);
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        const DropCall d = DropCall::of(ctx->saved_data["how"].toIntVector(), ctx->get_saved_variables()[0]);
        at::Tensor dx;
        if (ctx->needs_input_grad(0)) {
            const at::Tensor &dy = grads[0];
            const int64_t C = dy.size(-1);
            dx = dropout_forward(gradient_rows(dy, dy.numel() / C, C), at::Tensor(), d, at::Tensor()).view(dy.sizes());
        }
        const bool both = ctx->saved_data["residual"].toBool() && ctx->needs_input_grad(1);
        return once({dx, both ? grads[0] : at::Tensor(), at::Tensor(), at::Tensor()});
    }
};

// dropout(X, p, seed or tensor, offset, residual or None)
PyObject *dropout(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 5 || !ready || !THPVariable_Check(args[0]) || (args[4] != Py_None && !THPVariable_Check(args[4]))) Py_RETURN_NOTIMPLEMENTED;
    const at::Tensor &X = THPVariable_Unpack(args[0]);
    at::Tensor R;
    if (args[4] != Py_None) R = THPVariable_Unpack(args[4]);
    DropCall d;
    if (!here(X) || X.dim() < 1 || type_of(X) < 0 || X.numel() == 0 || !whole(X) || !d.take(args[1], args[2], args[3], X)) Py_RETURN_NOTIMPLEMENTED;
    if (R.defined() && (!here(R) || R.scalar_type() != X.scalar_type() || R.sizes() != X.sizes() || !whole(R))) Py_RETURN_NOTIMPLEMENTED;
    at::Tensor out;
    {
        pybind11::gil_scoped_release unlocked;
        out = at::GradMode::is_enabled() && (records(X) || records(R)) ? Dropout::apply(X, maybe(R), maybe(d.state), d.numbers())
                                                                      : dropout_forward(X, R, d, at::Tensor());
    }
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

pcsr_linear_t linear_call(const at::Tensor &x, const at::Tensor &W, const at::Tensor &b, const at::Tensor &r, int64_t bias_type, int64_t act, const pcsr_drop_t &how)
{
    return {x.size(0), x.size(1), W.size(0), type_of(x), (int32_t)bias_type, (int32_t)act, 0, x.const_data_ptr(), W.const_data_ptr(), address(b), address(r),
            distance(x), distance(W), r.defined() ? distance(r) : 0, how};
}
at::Tensor linear_forward(const at::Tensor &X, const at::Tensor &W, const at::Tensor &b, const at::Tensor &R, int64_t act, const DropCall &d, const at::Tensor &used,
                          at::Tensor *slope)
{
    auto shape = X.sizes().vec();
    shape.back() = W.size(0);
    const auto options = X.options().requires_grad(false);
    at::Tensor out = at::empty(shape, options), ws;
    const at::Tensor x = rows(X);
    if (slope && act != PCSR_ACT_NONE)
        *slope = at::empty({x.size(0), W.size(0)}, options.dtype(X.scalar_type() == at::kFloat ? at::kFloat : at::kShort));
    const pcsr_linear_t a = linear_call(x, W, b, R.defined() ? rows(R) : R, type_of(b.defined() ? b : X), act, d.to_library(used));
    const int64_t need = lib.linear_workspace(&a, 0);
    if (need) ws = bytes(need, X);
    ok(lib.linear(&a, out.data_ptr(), slope && slope->defined() ? slope->data_ptr() : nullptr, need ? ws.data_ptr() : nullptr, stream()), "pcsr_linear");
    return out;
}

struct Linear : torch::autograd::Function<Linear> {
    static at::Tensor forward(AutogradContext *ctx, const at::Tensor &X, const at::Tensor &W, const std::optional<at::Tensor> &b, const std::optional<at::Tensor> &R,
                              const std::optional<at::Tensor> &state, int64_t act, const std::vector<int64_t> &numbers)
    {
        const DropCall d = DropCall::of(numbers, of(state));
        const at::Tensor used = d.used();
        at::Tensor slope;
        const bool keep = records(X) || records(W) || (b.has_value() && records(*b));
        at::Tensor out = linear_forward(X, W, of(b), of(R), act, d, used, keep ? &slope : nullptr);
        ctx->save_for_backward({X, W, slope, used});
        std::vector<int64_t> how = numbers;
        how.insert(how.end(), {act, b.has_value() ? type_of(*b) : -1, R.has_value()});
        ctx->saved_data["how"] = std::move(how);
        return out;
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        const variable_list saved = ctx->get_saved_variables();
        const std::vector<int64_t> how = ctx->saved_data["how"].toIntVector();
        const DropCall d = DropCall::of(how, saved[3]);
        const at::Tensor X = saved[0].dim() == 2 ? saved[0] : saved[0].detach(), &W = saved[1];
        const int64_t act = how[3], bias = how[4];
        size_t at = 2; // (tensors that are not there are not counted)
        const bool need_b = bias >= 0 && ctx->needs_input_grad(at++), need_r = how[5] && ctx->needs_input_grad(at++);
        at::Tensor dx, dw, db;
        if (ctx->needs_input_grad(0)) dx = at::empty(X.sizes(), X.options());
        if (ctx->needs_input_grad(1)) dw = at::empty(W.sizes(), X.options());
        if (need_b) db = at::empty({W.size(0)}, X.options().dtype(bias == PCSR_F32 ? at::kFloat : X.scalar_type()));
        if (dx.defined() || dw.defined() || db.defined()) {
            const at::Tensor x = rows(X), g = gradient_rows(grads[0], x.size(0), W.size(0));
            const pcsr_linear_t a = linear_call(x, W, at::Tensor(), at::Tensor(), bias < 0 ? type_of(X) : bias, act, d.to_library(at::Tensor()));
            const at::Tensor ws = bytes(lib.linear_workspace(&a, 1), X);
            auto ptr = [](const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; };
            ok(lib.linear_backward(&a, address(saved[2]), g.const_data_ptr(), distance(g), ptr(dx), ptr(dw), ptr(db), ws.data_ptr(), stream()), "pcsr_linear_backward");
        }
        return once({dx, dw, db, need_r ? grads[0] : at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor()});
    }
};

// linear(X, weight, bias or None, activation's number, residual or None, p, seed or tensor, offset)
PyObject *linear(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 8 || !ready || !THPVariable_Check(args[0]) || !THPVariable_Check(args[1]) || !PyLong_Check(args[3])) Py_RETURN_NOTIMPLEMENTED;
    const at::Tensor &X = THPVariable_Unpack(args[0]), &W = THPVariable_Unpack(args[1]);
    at::Tensor b, R;
    for (const int k : {2, 4}) {
        if (args[k] == Py_None) continue;
        if (!THPVariable_Check(args[k])) Py_RETURN_NOTIMPLEMENTED;
        (k == 2 ? b : R) = THPVariable_Unpack(args[k]);
    }
    const int64_t act = PyLong_AsLongLong(args[3]);
    DropCall d;
    if (!here(X) || X.dim() < 1 || type_of(X) < 0 || X.numel() == 0 || !whole(X) || !d.take(args[5], args[6], args[7], X)) Py_RETURN_NOTIMPLEMENTED;
    if (!here(W) || W.dim() != 2 || W.scalar_type() != X.scalar_type() || W.size(0) < 1 || W.size(1) != X.size(-1) || distance(W) < 0) Py_RETURN_NOTIMPLEMENTED;
    if (b.defined() && (!here(b) || b.dim() != 1 || b.numel() != W.size(0) || !b.is_contiguous() || (b.scalar_type() != at::kFloat && b.scalar_type() != X.scalar_type())))
        Py_RETURN_NOTIMPLEMENTED;
    if (R.defined() && (!here(R) || R.scalar_type() != X.scalar_type() || R.dim() != X.dim() || R.size(-1) != W.size(0) ||
                        R.sizes().slice(0, (size_t)R.dim() - 1) != X.sizes().slice(0, (size_t)X.dim() - 1) || !whole(R)))
        Py_RETURN_NOTIMPLEMENTED;
    at::Tensor out;
    {
        pybind11::gil_scoped_release unlocked;
        if (at::GradMode::is_enabled() && (records(X) || records(W) || records(b) || records(R)))
            out = Linear::apply(X, W, maybe(b), maybe(R), maybe(d.state), act, d.numbers());
        else
            out = linear_forward(X, W, b, R, act, d, at::Tensor(), nullptr);
    }
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// init(addresses of the library's functions, in the order of Library)
PyObject *init(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    constexpr Py_ssize_t N = sizeof(Library) / sizeof(void *);
    if (n != N) {
        PyErr_SetString(PyExc_TypeError, "init takes an address for each function of the library");
        return nullptr;
    }
    void *at[N];
    for (Py_ssize_t k = 0; k < N; ++k) {
        at[k] = PyLong_AsVoidPtr(args[k]);
        if (PyErr_Occurred()) return nullptr;
    }
    static_assert(sizeof(at) == sizeof(lib), "one address for each function");
    memcpy(static_cast<void *>(&lib), at, sizeof(lib));
    ready = true;
    Py_RETURN_NONE;
}

// raises(exception type)
PyObject *raises(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 1 || !PyExceptionClass_Check(args[0])) {
        PyErr_SetString(PyExc_TypeError, "raises takes the type of an exception");
        return nullptr;
    }
    Py_INCREF(args[0]);
    error_type = args[0];
    Py_RETURN_NONE;
}

template <PyObject *(*F)(PyObject *, PyObject *const *, Py_ssize_t)> PyMethodDef method(const char *name)
{
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(F)), METH_FASTCALL, nullptr};
}
PyMethodDef methods[] = {method<embed>("embed"),   method<group_norm>("group_norm"), method<orthogonalize>("orthogonalize"),
                         method<update>("update"), method<dropout>("dropout"),       method<linear>("linear"),
                         method<init>("init"),     method<raises>("raises"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pcsr_train", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

PyMODINIT_FUNC PyInit__pcsr_train(void)
{
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", PCSR_TORCH_VERSION) < 0) Py_CLEAR(m);
    return m;
}
