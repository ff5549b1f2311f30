// The binding's fast way into libsphattn.so: checks, outputs, workspace and launch of a call in one step, as a CPython
// extension on torch's C++ headers.  No arithmetic, no kernels.
//
// The smallest calls are bound by what the host does before the launch, and a training step's two halves run on two threads
// that wake each other, where the interpreter runs at half its speed.  In Python, with ctypes, a forward call took 8.8 us of host
// time, 3.8 with this, of which the launch is 3 (1 x 256 x 64 in fp32 8.7 -> 6.4 us a call), a backward call 22 and 11 (a training step of 8
// heads on 2 of 1500 x 64 with counts 137 -> 89).
//
// A function here does a call only if everything about it is as it has to be: exactly torch's tensor type, with storage, the
// shapes, element types and device that the entry point's header states, contiguous, no function or dispatch mode in force.  For anything
// else, and for whatever throws on the way (no memory for an output), it returns None, having launched nothing, and the binding's Python does the call and finds out what is wrong.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/python_variable.h>

#include <array>
#include <climits>
#include <exception>
#include <optional>
#include <stdexcept>
#include <string>
#include <vector>

#include "../../include/sphattn_train.h"

namespace {

struct EntryPoints {
    decltype(&sphattn_cross_fwd) cross = nullptr;
    decltype(&sphattn_cross_splitkv_fwd) cross_cut = nullptr;
    decltype(&sphattn_cross_splitkv_workspace_bytes) cross_bytes = nullptr;
    decltype(&sphattn_grn_bwd) bwd = nullptr;
    decltype(&sphattn_grn_bwd_split) bwd_cut = nullptr;
    decltype(&sphattn_bwd_workspace_bytes) bwd_bytes = nullptr;
    decltype(&sphattn_fp8_grn_fwd) fp8 = nullptr;
    decltype(&sphattn_embed_fwd) embed = nullptr;
    decltype(&sphattn_embed_bwd_workspace_bytes) embed_bwd_bytes = nullptr;
    decltype(&sphattn_embed_bwd) embed_bwd = nullptr;
    decltype(&sphattn_vocab_loss_workspace_bytes) loss_bytes = nullptr;
    decltype(&sphattn_vocab_loss_fwd) loss = nullptr;
    decltype(&sphattn_vocab_loss_bwd_workspace_bytes) loss_bwd_bytes = nullptr;
    decltype(&sphattn_vocab_loss_bwd) loss_bwd = nullptr;
    decltype(&sphattn_clip_grads_workspace_bytes) clip_bytes = nullptr;
    decltype(&sphattn_clip_grads) clip = nullptr;
    decltype(&sphattn_strerror) text = nullptr;
} entry;
PyObject* raise_on = nullptr;                      // the binding's function that raises for an error code

// The interpreter's lock is given back while torch allocates and the library launches.
struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};

// Workspace sizes by shape and device (and by the function asked): the library's choice of slices takes a few microseconds.  Per thread,
// one shape per place.
class SizeTable {
public:
    template <typename Ask>
    size_t get(const std::array<int64_t, 9>& key, Ask ask)
    {
        uint64_t h = 0;
        for (const int64_t k : key) h = (h ^ (uint64_t)k) * 0x9e3779b97f4a7c15ull;
        Place& place = places_[h >> 59];
        if (!place.known || place.key != key) place = Place{key, ask(), true};
        return place.bytes;
    }
private:
    struct Place { std::array<int64_t, 9> key; size_t bytes; bool known = false; };
    Place places_[32];
};
thread_local SizeTable sizes;

const at::Tensor* tensor(PyObject* o)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.defined() && t.has_storage() ? &t : nullptr;
}

bool fits(const at::Tensor& t, at::IntArrayRef shape, at::ScalarType type, at::Device device)
{
    return t.scalar_type() == type && t.device() == device && t.layout() == at::kStrided && t.sizes() == shape && t.is_contiguous();
}

bool is_e4m3(const at::Tensor& t) { return t.scalar_type() == at::kFloat8_e4m3fn || t.scalar_type() == at::kByte; }

void* data(const at::Tensor& t) { return t.data_ptr(); }
void* data(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }

// Q [B,H,Nq,d]; K, V [B,H_kv,Nk,d]
struct Shape {
    int64_t B, H, Nq, d, H_kv, Nk;
    bool read(const at::Tensor& Q, const at::Tensor& K, bool same_n, bool same_h)
    {
        if (Q.dim() != 4 || K.dim() != 4 || !Q.is_cuda()) return false;
        B = Q.size(0), H = Q.size(1), Nq = Q.size(2), d = Q.size(3), H_kv = K.size(1), Nk = K.size(2);
        const int64_t most = INT_MAX;
        return K.size(0) == B && K.size(3) == d && H_kv > 0 && H % H_kv == 0 && (!same_n || Nk == Nq) && (!same_h || H_kv == H) &&
               B <= most && H <= most && Nq <= most && Nk <= most && d <= most;
    }
};

void* stream_of(const at::Tensor& t) { return c10::hip::getCurrentHIPStream(t.get_device()).stream(); }

at::Tensor workspace(size_t bytes, const at::Tensor& like)
{
    if (bytes == 0) return {};
    try {
        return at::empty({(int64_t)bytes}, like.options().dtype(at::kByte));
    } catch (const c10::OutOfMemoryError&) {
        return {};                                 // the uncut launches need none
    }
}

// An optional tensor argument: `there` and its tensor, or false for something that is neither None nor a tensor.
bool optional(PyObject* o, const at::Tensor*& t)
{
    t = nullptr;
    return o == Py_None || (t = tensor(o)) != nullptr;
}

PyObject* wrapped(at::Tensor&& t)
{
    try {
        return THPVariable_Wrap(std::move(t));
    } catch (const std::exception& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

PyObject* raised(int rc)
{
    PyObject* none = PyObject_CallFunction(raise_on, "i", rc);
    if (none != nullptr) {                         // (it always raises)
        Py_DECREF(none);
        PyErr_SetString(PyExc_RuntimeError, "sphattn error");
    }
    return nullptr;
}

bool arguments(Py_ssize_t n, Py_ssize_t want)
{
    if (n == want) return true;
    PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", want, n);
    return false;
}

// (A dispatch mode makes its own tensors for what is allocated here: Python checks those as it does a caller's.)
bool ready() { return entry.cross != nullptr && !at::impl::torch_function_mode_enabled() && !c10::impl::TorchDispatchModeTLS::any_modes_set(); }

// forward(Q, K, V, mult, Z, code, same_n, same_h, want_z) -> O, with want_z (O, Z)
PyObject* forward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arguments(n, 9)) return nullptr;
    const at::Tensor *Q = tensor(args[0]), *K = tensor(args[1]), *V = tensor(args[2]), *mult, *Z;
    const long code = PyLong_AsLong(args[5]);
    if (code == -1 && PyErr_Occurred()) return nullptr;
    if (!Q || !K || !V || !optional(args[3], mult) || !optional(args[4], Z) || !ready()) Py_RETURN_NONE;
    at::Tensor O, own_z;
    int rc = 0;
    try {
        Shape s;
        if (!s.read(*Q, *K, args[6] == Py_True, args[7] == Py_True)) Py_RETURN_NONE;
        const at::Device device = Q->device();
        const at::ScalarType vo = code == SPHATTN_F32 ? at::kFloat : code == SPHATTN_F16 ? at::kHalf : at::kBFloat16;
        if (code == SPHATTN_FP8QK_BF16V) {
            if (!is_e4m3(*Q) || !is_e4m3(*K)) Py_RETURN_NONE;
        } else if ((code != SPHATTN_F32 && code != SPHATTN_F16 && code != SPHATTN_BF16) || Q->scalar_type() != vo || K->scalar_type() != vo) {
            Py_RETURN_NONE;
        }
        const int64_t kv[4] = {s.B, s.H_kv, s.Nk, s.d}, counts[2] = {s.B, s.Nk}, rows[3] = {s.B, s.H, s.Nq};
        if (!Q->is_contiguous() || Q->layout() != at::kStrided || !fits(*K, kv, K->scalar_type(), device) || !fits(*V, kv, vo, device) ||
            (mult && !fits(*mult, counts, at::kFloat, device)) || (Z && !fits(*Z, rows, at::kFloat, device)))
            Py_RETURN_NONE;
        const Unlocked unlocked;
        O = Q->scalar_type() == vo ? at::empty_like(*Q) : at::empty(Q->sizes(), Q->options().dtype(vo));
        if (args[8] == Py_True) {
            own_z = at::empty(rows, Q->options().dtype(at::kFloat));
            Z = &own_z;
        }
        const size_t bytes = sizes.get({(int64_t)entry.cross_bytes, Q->get_device(), s.B, s.H, s.H_kv, s.Nq, s.Nk, s.d, code}, [&] {
            return entry.cross_bytes((int)s.B, (int)s.H, (int)s.H_kv, (int)s.Nq, (int)s.Nk, (int)s.d, (int)code);
        });
        const at::Tensor ws = workspace(bytes, *Q);
        auto launch = [&](auto call, auto... rest) {
            return call(data(*Q), data(*K), data(*V), (const float*)data(mult), data(O), (float*)data(Z), (int)s.B, (int)s.H, (int)s.H_kv, (int)s.Nq,
                        (int)s.Nk, (int)s.d, (int)code, rest..., stream_of(*Q));
        };
        rc = ws.defined() ? launch(entry.cross_cut, data(ws), bytes) : launch(entry.cross);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if (rc != 0) return raised(rc);
    if (!own_z.defined()) return wrapped(std::move(O));
    PyObject *o = wrapped(std::move(O)), *z = o ? wrapped(std::move(own_z)) : nullptr;
    PyObject* both = z ? PyTuple_Pack(2, o, z) : nullptr;
    Py_XDECREF(o);
    Py_XDECREF(z);
    return both;
}

// backward(Q, K, V, mult, O, dO, Z, code, same_h) -> (dQ, dK, dV)
PyObject* backward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arguments(n, 9)) return nullptr;
    const at::Tensor *Q = tensor(args[0]), *K = tensor(args[1]), *V = tensor(args[2]), *O = tensor(args[4]), *dO = tensor(args[5]), *Z = tensor(args[6]), *mult;
    const long code = PyLong_AsLong(args[7]);
    if (code == -1 && PyErr_Occurred()) return nullptr;
    if (!Q || !K || !V || !O || !dO || !Z || !optional(args[3], mult) || (code != SPHATTN_BF16 && code != SPHATTN_F16) || !ready()) Py_RETURN_NONE;
    at::Tensor d[3];
    int rc = 0;
    try {
        Shape s;
        if (!s.read(*Q, *K, true, args[8] == Py_True)) Py_RETURN_NONE;
        const at::Device device = Q->device();
        const at::ScalarType t16 = code == SPHATTN_F16 ? at::kHalf : at::kBFloat16;
        const int64_t q[4] = {s.B, s.H, s.Nq, s.d}, kv[4] = {s.B, s.H_kv, s.Nk, s.d}, counts[2] = {s.B, s.Nk}, rows[3] = {s.B, s.H, s.Nq};
        if (!fits(*Q, q, t16, device) || !fits(*K, kv, t16, device) || !fits(*V, kv, t16, device) || !fits(*O, q, t16, device) || !fits(*dO, q, t16, device) ||
            !fits(*Z, rows, at::kFloat, device) || (mult && !fits(*mult, counts, at::kFloat, device)))
            Py_RETURN_NONE;
        const Unlocked unlocked;
        d[0] = at::empty_like(*Q);
        d[1] = at::empty_like(*K);
        d[2] = at::empty_like(*V);
        if (!fits(d[0], q, t16, device) || !fits(d[1], kv, t16, device) || !fits(d[2], kv, t16, device)) throw 0;
        const at::Tensor delta = at::empty({2, s.B, s.H, s.Nq}, Q->options().dtype(at::kFloat));
        const size_t bytes = sizes.get({(int64_t)entry.bwd_bytes, Q->get_device(), s.B, s.H, s.H_kv, s.Nq, s.Nk, s.d, code}, [&] {
            return entry.bwd_bytes((int)s.B, (int)s.H, (int)s.H_kv, (int)s.Nq, (int)s.d, (int)code);
        });
        const at::Tensor ws = workspace(bytes, *Q);
        auto launch = [&](auto call, auto... rest) {
            return call(data(*Q), data(*K), data(*V), (const float*)data(mult), data(*O), data(*dO), (const float*)data(*Z), data(d[0]), data(d[1]), data(d[2]),
                        (float*)data(delta), (int)s.B, (int)s.H, (int)s.H_kv, (int)s.Nq, (int)s.d, (int)code, rest..., stream_of(*Q));
        };
        rc = ws.defined() ? launch(entry.bwd_cut, data(ws), bytes) : launch(entry.bwd);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if (rc != 0) return raised(rc);
    PyObject* out = PyTuple_New(3);
    for (int i = 0; out != nullptr && i < 3; ++i) {
        PyObject* o = wrapped(std::move(d[i]));
        if (o == nullptr) Py_CLEAR(out);
        else PyTuple_SET_ITEM(out, i, o);
    }
    return out;
}

// fp8_forward(Q, K, V, mult, workspace) -> O
PyObject* fp8_forward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arguments(n, 5)) return nullptr;
    const at::Tensor *Q = tensor(args[0]), *K = tensor(args[1]), *V = tensor(args[2]), *ws = tensor(args[4]), *mult;
    if (!Q || !K || !V || !ws || !optional(args[3], mult) || !ready()) Py_RETURN_NONE;
    at::Tensor O;
    int rc = 0;
    try {
        Shape s;
        if (!s.read(*Q, *K, true, false) || !is_e4m3(*Q) || !is_e4m3(*K) || !is_e4m3(*V)) Py_RETURN_NONE;
        const at::Device device = Q->device();
        const int64_t kv[4] = {s.B, s.H_kv, s.Nk, s.d}, counts[2] = {s.B, s.Nk};
        if (!Q->is_contiguous() || Q->layout() != at::kStrided || !fits(*K, kv, K->scalar_type(), device) || !fits(*V, kv, V->scalar_type(), device) ||
            (mult && !fits(*mult, counts, at::kFloat, device)) || ws->dim() != 1 || !fits(*ws, ws->sizes(), ws->scalar_type(), device))
            Py_RETURN_NONE;
        const Unlocked unlocked;
        O = at::empty(Q->sizes(), Q->options().dtype(at::kBFloat16));
        rc = entry.fp8(data(*Q), data(*K), data(*V), (const float*)data(mult), data(O), data(*ws), ws->nbytes(), (int)s.B, (int)s.H, (int)s.H_kv,
                       (int)s.Nq, (int)s.d, stream_of(*Q));
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if (rc != 0) return raised(rc);
    return wrapped(std::move(O));
}

// ---- sphattn_train.h -------------------------------------------------------------------------------
//
// The differentiable calls are autograd nodes of their own here: a backward pass's worker thread then neither waits for the
// interpreter nor runs it.  A lookup of 8192 rows of 19999 x 1024 with its gradient took 105 us through Python (kernels 38) and takes 52, a
// lookup of one row 9.9 and 5.0, clipping twelve tensors 26.8 and 10.8 (kernels 10).

int code_of(const at::Tensor& t)
{
    return t.scalar_type() == at::kFloat ? SPHATTN_F32 : t.scalar_type() == at::kBFloat16 ? SPHATTN_BF16 : t.scalar_type() == at::kHalf ? SPHATTN_F16 : -1;
}

bool plain(const at::Tensor& t, at::Device device) { return t.device() == device && t.layout() == at::kStrided && t.is_contiguous(); }

bool are_ids(const at::Tensor& t, at::Device device) { return (t.scalar_type() == at::kLong || t.scalar_type() == at::kInt) && plain(t, device); }

at::Tensor bytes_of(size_t n, const at::Tensor& like) { return at::empty({(int64_t)n}, like.options().dtype(at::kByte)); }

at::Tensor floats(at::IntArrayRef shape, const at::Tensor& like) { return at::empty(shape, like.options().dtype(at::kFloat)); }

// In a backward pass, where no Python is at hand to raise the binding's own error.
void throw_on(int rc)
{
    if (rc != 0) throw std::runtime_error("sphattn error " + std::to_string(rc) + ": " + entry.text(rc));
}

// Gradients that a second derivative is asked of say that they have none.
torch::autograd::variable_list once(torch::autograd::variable_list grads)
{
    if (!at::GradMode::is_enabled()) return grads;
    std::vector<size_t> at;
    torch::autograd::variable_list there;
    for (size_t i = 0; i < grads.size(); ++i)
        if (grads[i].defined()) {
            at.push_back(i);
            there.push_back(grads[i].detach().requires_grad_());
        }
    const auto error = std::make_shared<torch::autograd::DelayedError>("this gradient of sphattn has no derivative", (int64_t)there.size());
    torch::autograd::variable_list marked = (*error)(std::move(there));
    for (size_t i = 0; i < at.size(); ++i) grads[at[i]] = marked[i];
    return grads;
}

at::Tensor embed(const at::Tensor& tokens, const at::Tensor& table, const at::Tensor* mult, double scale, int& rc)
{
    std::vector<int64_t> shape = tokens.sizes().vec();
    shape.push_back(table.size(1));
    at::Tensor O = at::empty(shape, table.options());
    rc = entry.embed(data(tokens), (int)tokens.element_size(), data(table), (const float*)data(mult), data(O), (int)tokens.numel(), (int)table.size(0),
                     (int)table.size(1), (float)scale, code_of(table), stream_of(table));
    return O;
}

at::Tensor embed_gradient(const at::Tensor& tokens, const at::Tensor& dO, int64_t V, const at::Tensor* mult, double scale, int& rc)
{
    const int T = (int)tokens.numel(), D = (int)dO.size(-1);
    at::Tensor dtable = at::empty({V, D}, dO.options());
    const size_t bytes = entry.embed_bwd_bytes(T, (int)V, D);
    const at::Tensor ws = bytes_of(bytes, dO);
    rc = entry.embed_bwd(data(tokens), (int)tokens.element_size(), (const float*)data(mult), data(dO), data(dtable), T, (int)V, D, (float)scale, code_of(dO),
                         data(ws), bytes, stream_of(dO));
    return dtable;
}

struct TokenEmbedding : torch::autograd::Function<TokenEmbedding> {
    static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& tokens, const at::Tensor& table, const std::optional<at::Tensor>& mult, double scale,
                              int* rc)
    {
        at::Tensor O = embed(tokens, table, mult ? &*mult : nullptr, scale, *rc);
        ctx->save_for_backward({tokens, mult.value_or(at::Tensor())});
        ctx->saved_data["V"] = table.size(0);
        ctx->saved_data["scale"] = scale;
        return O;
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        const auto saved = ctx->get_saved_variables();
        int rc = 0;
        at::Tensor dtable;
        {
            const at::NoGradGuard off;
            dtable = embed_gradient(saved[0], grads[0].contiguous(), ctx->saved_data["V"].toInt(), saved[1].defined() ? &saved[1] : nullptr,
                                    ctx->saved_data["scale"].toDouble(), rc);
        }
        throw_on(rc);
        return once({at::Tensor(), dtable, at::Tensor(), at::Tensor(), at::Tensor()});
    }
};

// What the embedding's calls have to be like: tokens of any shape if `any`, else [T].
bool embed_fits(const at::Tensor& tokens, const at::Tensor& like, const at::Tensor* mult, bool any)
{
    const at::Device device = like.device();
    return like.is_cuda() && plain(like, device) && code_of(like) >= 0 && (any || tokens.dim() == 1) && are_ids(tokens, device) && tokens.numel() <= INT_MAX &&
           (!mult || fits(*mult, tokens.sizes(), at::kFloat, device));
}

// embed_forward(tokens, table, mult, scale, differentiable) -> O
PyObject* embed_forward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arguments(n, 5)) return nullptr;
    const at::Tensor *tokens = tensor(args[0]), *table = tensor(args[1]), *mult;
    const double scale = PyFloat_AsDouble(args[3]);
    if (scale == -1.0 && PyErr_Occurred()) return nullptr;
    if (!tokens || !table || !optional(args[2], mult) || !ready()) Py_RETURN_NONE;
    at::Tensor O;
    int rc = 0;
    try {
        const bool differentiable = args[4] == Py_True;
        if (table->dim() != 2 || table->size(0) > INT_MAX || table->size(1) > INT_MAX || !embed_fits(*tokens, *table, mult, differentiable)) Py_RETURN_NONE;
        const Unlocked unlocked;
        O = differentiable ? TokenEmbedding::apply(*tokens, *table, mult ? std::optional<at::Tensor>(*mult) : std::nullopt, scale, &rc) : embed(*tokens, *table, mult, scale, rc);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    return rc != 0 ? raised(rc) : wrapped(std::move(O));
}

// embed_backward(tokens, dO, V, mult, scale) -> dtable
PyObject* embed_backward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arguments(n, 5)) return nullptr;
    const at::Tensor *tokens = tensor(args[0]), *dO = tensor(args[1]), *mult;
    const long long V = PyLong_AsLongLong(args[2]);
    const double scale = PyFloat_AsDouble(args[4]);
    if (PyErr_Occurred()) return nullptr;
    if (!tokens || !dO || !optional(args[3], mult) || !ready()) Py_RETURN_NONE;
    at::Tensor dtable;
    int rc = 0;
    try {
        if (dO->dim() != 2 || dO->size(0) != tokens->numel() || dO->size(1) > INT_MAX || V < 1 || V > INT_MAX || !embed_fits(*tokens, *dO, mult, false)) Py_RETURN_NONE;
        const Unlocked unlocked;
        dtable = embed_gradient(*tokens, *dO, V, mult, scale, rc);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    return rc != 0 ? raised(rc) : wrapped(std::move(dtable));
}

struct Head { int T, V, D, code; };
Head head_of(const at::Tensor& targets, const at::Tensor& W) { return Head{(int)targets.numel(), (int)W.size(0), (int)W.size(1), code_of(W)}; }

struct Losses { at::Tensor losses, lse, mean; };

Losses loss(const at::Tensor& X, const at::Tensor& W, const at::Tensor& targets, double scale, int reduction, bool all_rows, int& rc)
{
    const Head h = head_of(targets, W);
    Losses out{floats(targets.sizes(), X), floats(targets.sizes(), X), reduction ? floats({}, X) : at::Tensor()};
    const size_t bytes = entry.loss_bytes(h.T, h.V, h.D, h.code);
    const at::Tensor ws = bytes_of(bytes, X);
    rc = entry.loss(data(X), data(W), data(targets), (int)targets.element_size(), (float*)data(out.losses), (float*)data(out.lse),
                    reduction ? (float*)data(out.mean) : nullptr, h.T, h.V, h.D, (float)scale, reduction, all_rows, h.code, data(ws), bytes, stream_of(X));
    return out;
}

std::array<at::Tensor, 2> loss_gradients(const at::Tensor& X, const at::Tensor& W, const at::Tensor& targets, const at::Tensor& lse, const at::Tensor& dloss,
                                         double scale, int reduction, bool want_dX, bool want_dW, int& rc)
{
    const Head h = head_of(targets, W);
    std::array<at::Tensor, 2> d;
    if (want_dX) d[0] = at::empty_like(X);
    if (want_dW) d[1] = at::empty_like(W);
    const size_t bytes = entry.loss_bwd_bytes(h.T, h.V, h.D, h.code);
    const at::Tensor ws = bytes_of(bytes, X);
    rc = entry.loss_bwd(data(X), data(W), data(targets), (int)targets.element_size(), (const float*)data(lse), (const float*)data(dloss),
                        want_dX ? data(d[0]) : nullptr, want_dW ? data(d[1]) : nullptr, h.T, h.V, h.D, (float)scale, reduction, h.code, data(ws), bytes,
                        stream_of(X));
    return d;
}

struct VocabCrossEntropy : torch::autograd::Function<VocabCrossEntropy> {
    static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& X, const at::Tensor& W, const at::Tensor& targets, double scale,
                              int64_t reduction, int* rc)
    {
        Losses out = loss(X, W, targets, scale, (int)reduction, false, *rc);
        ctx->save_for_backward({X, W, targets, out.lse});
        ctx->saved_data["scale"] = scale;
        ctx->saved_data["reduction"] = reduction;
        return reduction ? out.mean : out.losses;
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        const auto saved = ctx->get_saved_variables();
        int rc = 0;
        std::array<at::Tensor, 2> d;
        {
            const at::NoGradGuard off;
            d = loss_gradients(saved[0], saved[1], saved[2], saved[3], grads[0].contiguous(), ctx->saved_data["scale"].toDouble(),
                               (int)ctx->saved_data["reduction"].toInt(), ctx->needs_input_grad(0), ctx->needs_input_grad(1), rc);
        }
        throw_on(rc);
        return once({d[0], d[1], at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor()});
    }
};

// X [..., D] (rows of any shape if `any`, else [T,D]), W [V,D], targets [...]
bool head_fits(const at::Tensor& X, const at::Tensor& W, const at::Tensor& targets, bool any)
{
    if (!X.is_cuda() || W.dim() != 2 || X.dim() < 1 || (!any && X.dim() != 2)) return false;
    const at::Device device = X.device();
    return code_of(X) >= 0 && W.scalar_type() == X.scalar_type() && plain(X, device) && plain(W, device) && are_ids(targets, device) &&
           X.sizes().slice(0, X.dim() - 1) == targets.sizes() && X.size(-1) == W.size(1) && W.size(0) <= INT_MAX && W.size(1) <= INT_MAX &&
           targets.numel() <= INT_MAX;
}

PyObject* tuple_of(std::initializer_list<at::Tensor*> tensors)
{
    PyObject* out = PyTuple_New((Py_ssize_t)tensors.size());
    Py_ssize_t i = 0;
    for (at::Tensor* t : tensors) {
        if (out == nullptr) break;
        PyObject* o = Py_None;
        if (t->defined()) o = wrapped(std::move(*t));
        else Py_INCREF(o);
        if (o == nullptr) Py_CLEAR(out);
        else PyTuple_SET_ITEM(out, i++, o);
    }
    return out;
}

// loss_forward(X, W, targets, scale, reduction, all_rows, differentiable) -> (losses, lse[, mean]), or if differentiable what vocab_cross_entropy returns
PyObject* loss_forward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arguments(n, 7)) return nullptr;
    const at::Tensor *X = tensor(args[0]), *W = tensor(args[1]), *targets = tensor(args[2]);
    const double scale = PyFloat_AsDouble(args[3]);
    const long reduction = PyLong_AsLong(args[4]);
    if (PyErr_Occurred()) return nullptr;
    if (!X || !W || !targets || !ready()) Py_RETURN_NONE;
    const bool differentiable = args[6] == Py_True;
    Losses out;
    int rc = 0;
    try {
        if (!head_fits(*X, *W, *targets, differentiable)) Py_RETURN_NONE;
        const Unlocked unlocked;
        if (differentiable) out.losses = VocabCrossEntropy::apply(*X, *W, *targets, scale, (int64_t)reduction, &rc);
        else out = loss(*X, *W, *targets, scale, (int)reduction, args[5] == Py_True, rc);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if (rc != 0) return raised(rc);
    if (differentiable) return wrapped(std::move(out.losses));
    return reduction ? tuple_of({&out.losses, &out.lse, &out.mean}) : tuple_of({&out.losses, &out.lse});
}

// loss_backward(X, W, targets, lse, dloss, scale, reduction, want_dX, want_dW) -> (dX, dW)
PyObject* loss_backward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arguments(n, 9)) return nullptr;
    const at::Tensor *X = tensor(args[0]), *W = tensor(args[1]), *targets = tensor(args[2]), *lse = tensor(args[3]), *dloss = tensor(args[4]);
    const double scale = PyFloat_AsDouble(args[5]);
    const long reduction = PyLong_AsLong(args[6]);
    if (PyErr_Occurred()) return nullptr;
    if (!X || !W || !targets || !lse || !dloss || !ready()) Py_RETURN_NONE;
    std::array<at::Tensor, 2> d;
    int rc = 0;
    try {
        if (!head_fits(*X, *W, *targets, false) || !fits(*lse, targets->sizes(), at::kFloat, X->device()) ||
            !fits(*dloss, reduction ? at::IntArrayRef() : targets->sizes(), at::kFloat, X->device()))
            Py_RETURN_NONE;
        const Unlocked unlocked;
        d = loss_gradients(*X, *W, *targets, *lse, *dloss, scale, (int)reduction, args[7] == Py_True, args[8] == Py_True, rc);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    return rc != 0 ? raised(rc) : tuple_of({&d[0], &d[1]});
}

// clip(grads, out, max_norm) -> norm: two lists, or one twice
PyObject* clip(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arguments(n, 3)) return nullptr;
    const double max_norm = PyFloat_AsDouble(args[2]);
    if (PyErr_Occurred()) return nullptr;
    if (!PyList_CheckExact(args[0]) || !PyList_CheckExact(args[1]) || !ready()) Py_RETURN_NONE;
    const Py_ssize_t count = PyList_GET_SIZE(args[0]);
    if (count == 0 || count > INT_MAX || PyList_GET_SIZE(args[1]) != count || !(max_norm >= 0)) Py_RETURN_NONE;
    at::Tensor norm;
    int rc = 0;
    try {
        std::vector<const void*> in(count);
        std::vector<void*> out(count);
        std::vector<long long> size(count);
        std::vector<int> type(count);
        std::vector<const at::Tensor*> written(count);
        const at::Tensor* first = nullptr;
        for (Py_ssize_t i = 0; i < count; ++i) {
            const at::Tensor *g = tensor(PyList_GET_ITEM(args[0], i)), *o = tensor(PyList_GET_ITEM(args[1], i));
            if (!g || !o || !g->is_cuda() || g->layout() != at::kStrided || code_of(*g) < 0 || !g->is_non_overlapping_and_dense()) Py_RETURN_NONE;
            if (!first) first = g;
            if (g->device() != first->device() || (o != g && (o->scalar_type() != g->scalar_type() || o->device() != g->device() || o->layout() != at::kStrided ||
                                                              o->sizes() != g->sizes() || o->strides() != g->strides())))
                Py_RETURN_NONE;
            written[i] = o;
            in[i] = data(*g), out[i] = data(*o), size[i] = g->numel(), type[i] = code_of(*g);
        }
        const Unlocked unlocked;
        norm = floats({}, *first);
        const size_t bytes = entry.clip_bytes((int)count);
        const at::Tensor ws = bytes_of(bytes, *first);
        rc = entry.clip(in.data(), out.data(), size.data(), type.data(), (int)count, (float)max_norm, (float*)data(norm), data(ws), bytes, stream_of(*first));
        // autograd is told, as by torch's own operations in place: what it has saved of these tensors is no longer there
        if (rc == 0)
            for (const at::Tensor* o : written)
                if (!o->is_inference()) o->unsafeGetTensorImpl()->bump_version();
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    return rc != 0 ? raised(rc) : wrapped(std::move(norm));
}

// bind(raise_on, addresses of the entry points in the order of EntryPoints)
PyObject* bind(PyObject*, PyObject* args)
{
    constexpr Py_ssize_t COUNT = 17;
    unsigned long long a[COUNT];
    if (!arguments(PyTuple_GET_SIZE(args), COUNT + 1)) return nullptr;
    for (Py_ssize_t i = 0; i < COUNT; ++i) {
        a[i] = PyLong_AsUnsignedLongLong(PyTuple_GET_ITEM(args, i + 1));
        if (PyErr_Occurred()) return nullptr;
    }
    PyObject* handler = PyTuple_GET_ITEM(args, 0);
    Py_INCREF(handler);
    Py_XDECREF(raise_on);
    raise_on = handler;
    auto set = [&, i = 0](auto&... to) mutable { ((to = (std::decay_t<decltype(to)>)a[i++]), ...); };
    set(entry.cross, entry.cross_cut, entry.cross_bytes, entry.bwd, entry.bwd_cut, entry.bwd_bytes, entry.fp8, entry.embed, entry.embed_bwd_bytes,
        entry.embed_bwd, entry.loss_bytes, entry.loss, entry.loss_bwd_bytes, entry.loss_bwd, entry.clip_bytes, entry.clip, entry.text);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"forward", (PyCFunction)(void*)forward, METH_FASTCALL, nullptr},
                         {"backward", (PyCFunction)(void*)backward, METH_FASTCALL, nullptr},
                         {"fp8_forward", (PyCFunction)(void*)fp8_forward, METH_FASTCALL, nullptr},
                         {"embed_forward", (PyCFunction)(void*)embed_forward, METH_FASTCALL, nullptr},
                         {"embed_backward", (PyCFunction)(void*)embed_backward, METH_FASTCALL, nullptr},
                         {"loss_forward", (PyCFunction)(void*)loss_forward, METH_FASTCALL, nullptr},
                         {"loss_backward", (PyCFunction)(void*)loss_backward, METH_FASTCALL, nullptr},
                         {"clip", (PyCFunction)(void*)clip, METH_FASTCALL, nullptr},
                         {"bind", bind, METH_VARARGS, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Checks, outputs, workspace and launch of a call (see marshal.cpp).", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal()
{
    PyObject* m = PyModule_Create(&module);
    // the torch whose headers this was compiled with (its tensors' layout), for the binding to compare
    if (m != nullptr && PyModule_AddStringConstant(m, "built_for", MARSHAL_TORCH) != 0) Py_CLEAR(m);
    return m;
}
