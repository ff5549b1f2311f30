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

#include "../../include/sphattn_layer.h"
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
    decltype(&sphattn_vocab_distill_workspace_bytes) distill_bytes = nullptr;
    decltype(&sphattn_vocab_distill_fwd) distill = nullptr;
    decltype(&sphattn_vocab_distill_bwd_workspace_bytes) distill_bwd_bytes = nullptr;
    decltype(&sphattn_vocab_distill_bwd) distill_bwd = nullptr;
    decltype(&sphattn_head_norm_rotary_fwd) heads = nullptr;
    decltype(&sphattn_head_norm_rotary_bwd_workspace_bytes) heads_bwd_bytes = nullptr;
    decltype(&sphattn_head_norm_rotary_bwd) heads_bwd = nullptr;
    decltype(&sphattn_gated_ffn_workspace_bytes) ffn_bytes = nullptr;
    decltype(&sphattn_gated_ffn_fwd) ffn = nullptr;
    decltype(&sphattn_gated_ffn_bwd_workspace_bytes) ffn_bwd_bytes = nullptr;
    decltype(&sphattn_gated_ffn_bwd) ffn_bwd = nullptr;
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

// ---- distillation -------------------------------------------------------------------------------------

struct Distilled { at::Tensor losses, lse, kept, mean; };

Distilled distill(const at::Tensor& X, const at::Tensor& W, const at::Tensor& ids, const at::Tensor& teacher, double scale, double tau, int reduction, bool keep, int& rc)
{
    const int K = (int)ids.size(-1), V = (int)W.size(0), D = (int)W.size(1), T = (int)(X.numel() / D);
    const at::IntArrayRef rows = X.sizes().slice(0, X.dim() - 1);
    Distilled out{floats(rows, X), floats(rows, X), keep ? floats(ids.sizes(), X) : at::Tensor(), reduction ? floats({}, X) : at::Tensor()};
    const size_t bytes = entry.distill_bytes(T, V, D, K, code_of(W));
    const at::Tensor ws = bytes_of(bytes, X);
    rc = entry.distill(data(X), data(W), data(ids), (int)ids.element_size(), (const float*)data(teacher), (float*)data(out.losses), (float*)data(out.lse),
                       keep ? (float*)data(out.kept) : nullptr, reduction ? (float*)data(out.mean) : nullptr, T, V, D, K, (float)scale, (float)tau, reduction,
                       code_of(W), data(ws), bytes, stream_of(X));
    return out;
}

struct VocabDistillation : torch::autograd::Function<VocabDistillation> {
    static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& X, const at::Tensor& W, const at::Tensor& ids, const at::Tensor& teacher,
                              double scale, double tau, int64_t reduction, int* rc)
    {
        Distilled out = distill(X, W, ids, teacher, scale, tau, (int)reduction, true, *rc);
        ctx->save_for_backward({X, W, ids, teacher, out.lse, out.kept});
        ctx->saved_data["scale"] = scale;
        ctx->saved_data["tau"] = tau;
        ctx->saved_data["reduction"] = reduction;
        return reduction ? out.mean : out.losses;
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        const auto saved = ctx->get_saved_variables();
        const at::Tensor &X = saved[0], &W = saved[1], &ids = saved[2];
        int rc = 0;
        at::Tensor dX, dW;
        {
            const at::NoGradGuard off;
            const at::Tensor dloss = grads[0].contiguous();
            const int K = (int)ids.size(-1), V = (int)W.size(0), D = (int)W.size(1), T = (int)(X.numel() / D);
            if (ctx->needs_input_grad(0)) dX = at::empty_like(X);
            if (ctx->needs_input_grad(1)) dW = at::empty_like(W);
            const size_t bytes = entry.distill_bwd_bytes(T, V, D, K, code_of(W));
            const at::Tensor ws = bytes_of(bytes, X);
            rc = entry.distill_bwd(data(X), data(W), data(ids), (int)ids.element_size(), (const float*)data(saved[3]), (const float*)data(saved[4]),
                                   (const float*)data(saved[5]), (const float*)data(dloss), dX.defined() ? data(dX) : nullptr, dW.defined() ? data(dW) : nullptr,
                                   T, V, D, K, (float)ctx->saved_data["scale"].toDouble(), (float)ctx->saved_data["tau"].toDouble(),
                                   (int)ctx->saved_data["reduction"].toInt(), code_of(W), data(ws), bytes, stream_of(X));
        }
        throw_on(rc);
        return once({dX, dW, at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor()});
    }
};

// distill_forward(X, W, ids, teacher, scale, tau, reduction, keep, differentiable) -> (losses, lse[, kept][, mean]), or if differentiable what
// vocab_distillation returns
PyObject* distill_forward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arguments(n, 9)) return nullptr;
    const at::Tensor *X = tensor(args[0]), *W = tensor(args[1]), *ids = tensor(args[2]), *teacher = tensor(args[3]);
    const double scale = PyFloat_AsDouble(args[4]), tau = PyFloat_AsDouble(args[5]);
    const long reduction = PyLong_AsLong(args[6]);
    if (PyErr_Occurred()) return nullptr;
    if (!X || !W || !ids || !teacher || !ready()) Py_RETURN_NONE;
    const bool differentiable = args[8] == Py_True, keep = args[7] == Py_True;
    Distilled out;
    int rc = 0;
    try {
        if (!X->is_cuda() || W->dim() != 2 || X->dim() < 1 || ids->dim() != X->dim() || (!differentiable && X->dim() != 2) || code_of(*X) < 0) Py_RETURN_NONE;
        const at::Device device = X->device();
        if (W->scalar_type() != X->scalar_type() || !plain(*X, device) || !plain(*W, device) || !are_ids(*ids, device) ||
            !fits(*teacher, ids->sizes(), at::kFloat, device) || X->sizes().slice(0, X->dim() - 1) != ids->sizes().slice(0, X->dim() - 1) ||
            X->size(-1) != W->size(1) || W->size(0) < 1 || W->size(0) > INT_MAX || W->size(1) < 1 || W->size(1) > INT_MAX || ids->size(-1) < 1 ||
            ids->size(-1) > INT_MAX || X->numel() / W->size(1) > INT_MAX)
            Py_RETURN_NONE;
        const Unlocked unlocked;
        if (differentiable) out.losses = VocabDistillation::apply(*X, *W, *ids, *teacher, scale, tau, (int64_t)reduction, &rc);
        else out = distill(*X, *W, *ids, *teacher, scale, tau, (int)reduction, keep, rc);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if (rc != 0) return raised(rc);
    if (differentiable) return wrapped(std::move(out.losses));
    if (keep) return reduction ? tuple_of({&out.losses, &out.lse, &out.kept, &out.mean}) : tuple_of({&out.losses, &out.lse, &out.kept});
    return reduction ? tuple_of({&out.losses, &out.lse, &out.mean}) : tuple_of({&out.losses, &out.lse});
}

// ---- sphattn_layer.h -------------------------------------------------------------------------------

// How a call of head_norm_rotary is rotated and normalised, and its sizes.
struct HeadsHow {
    int axes = 0, sections[3] = {0, 0, 0}, interleaved = 0, norm = 1;   // axes 0: nothing is rotated
    float eps = 0.f;
};

sphattn_heads by_token(const at::Tensor& t) { return sphattn_heads{data(t), t.stride(0), t.stride(1), t.stride(2)}; }
sphattn_heads by_head(const at::Tensor& t) { return sphattn_heads{data(t), t.stride(0), t.stride(2), t.stride(1)}; }

sphattn_rotary rotary_of(const HeadsHow& how, const at::Tensor* positions, const at::Tensor* inv_freq, int64_t B)
{
    sphattn_rotary r{};
    if (!how.axes) return r;
    r.positions = data(positions), r.id_bytes = (int)positions->element_size(), r.axes = how.axes, r.interleaved = how.interleaved;
    r.axis = positions->dim() == 3 ? positions->stride(0) : 0;
    r.batch = positions->dim() > 1 && positions->size(-2) > 1 ? positions->stride(-2) : 0;
    r.inv_freq = (const float*)data(inv_freq);
    for (int i = 0; i < 3; ++i) r.sections[i] = how.sections[i];
    return r;
}

void rotate_heads(const at::Tensor& Xq, const at::Tensor* Xk, const at::Tensor* wq, const at::Tensor* wk, const at::Tensor* positions, const at::Tensor* inv_freq,
                  const HeadsHow& how, at::Tensor& Q, at::Tensor& K, int& rc)
{
    const int64_t B = Xq.size(0), N = Xq.size(1), Hq = Xq.size(2), d = Xq.size(3), Hk = Xk ? Xk->size(2) : 0;
    if (!Q.defined()) Q = at::empty({B, Hq, N, d}, Xq.options());
    if (Xk && !K.defined()) K = at::empty({B, Hk, N, d}, Xq.options());
    const sphattn_heads xq = by_token(Xq), q = by_head(Q);
    sphattn_heads xk{}, k{};
    if (Xk) xk = by_token(*Xk), k = by_head(K);
    const sphattn_rotary r = rotary_of(how, positions, inv_freq, B);
    rc = entry.heads(&xq, Xk ? &xk : nullptr, data(wq), data(wk), &q, Xk ? &k : nullptr, &r, (int)B, (int)N, (int)Hq, (int)Hk, (int)d, how.norm, how.eps,
                     code_of(Xq), stream_of(Xq));
}

// Rows of neighbouring elements, anywhere
bool rows_fit(const at::Tensor& t, at::IntArrayRef shape, at::ScalarType type, at::Device device)
{
    return t.scalar_type() == type && t.device() == device && t.layout() == at::kStrided && t.sizes() == shape && t.stride(3) == 1;
}

struct HeadNormRotary : torch::autograd::Function<HeadNormRotary> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const at::Tensor& Xq, const at::Tensor& Xk, const at::Tensor& wq,
                                                  const at::Tensor& wk, const std::optional<at::Tensor>& positions, const std::optional<at::Tensor>& inv_freq,
                                                  const HeadsHow* how, int* rc)
    {
        at::Tensor Q, K;
        rotate_heads(Xq, &Xk, &wq, &wk, positions ? &*positions : nullptr, inv_freq ? &*inv_freq : nullptr, *how, Q, K, *rc);
        ctx->save_for_backward({Xq, Xk, wq, wk, positions.value_or(at::Tensor()), inv_freq.value_or(at::Tensor())});
        ctx->saved_data["how"] = std::vector<int64_t>{how->axes, how->sections[0], how->sections[1], how->sections[2], how->interleaved, how->norm};
        ctx->saved_data["eps"] = (double)how->eps;
        return {Q, K};
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        const auto saved = ctx->get_saved_variables();
        const at::Tensor &Xq = saved[0], &Xk = saved[1];
        at::Tensor d[4];
        int rc = 0;
        {
            const at::NoGradGuard off;
            const auto list = ctx->saved_data["how"].toIntVector();
            HeadsHow how;
            how.axes = (int)list[0], how.interleaved = (int)list[4], how.norm = (int)list[5], how.eps = (float)ctx->saved_data["eps"].toDouble();
            for (int i = 0; i < 3; ++i) how.sections[i] = (int)list[1 + i];
            for (int i = 0; i < 2; ++i)
                if (grads[i].stride(3) != 1) grads[i] = grads[i].contiguous();
            sphattn_heads view[2];
            for (int i = 0; i < 4; ++i) {
                if (!ctx->needs_input_grad(i)) continue;
                d[i] = at::empty(saved[i].sizes(), saved[i].options());
                if (i < 2) view[i] = by_token(d[i]);
            }
            const sphattn_heads xq = by_token(Xq), xk = by_token(Xk), q = by_head(grads[0]), k = by_head(grads[1]);
            const sphattn_rotary r = rotary_of(how, &saved[4], &saved[5], Xq.size(0));
            const bool sums = d[2].defined() || d[3].defined();
            const size_t bytes = sums ? entry.heads_bwd_bytes((int)Xq.size(3)) : 0;
            const at::Tensor ws = sums ? bytes_of(bytes, Xq) : at::Tensor();
            rc = entry.heads_bwd(&xq, &xk, data(saved[2]), data(saved[3]), &q, &k, d[0].defined() ? &view[0] : nullptr, d[1].defined() ? &view[1] : nullptr,
                                 d[2].defined() ? data(d[2]) : nullptr, d[3].defined() ? data(d[3]) : nullptr, &r, (int)Xq.size(0), (int)Xq.size(1), (int)Xq.size(2),
                                 (int)Xk.size(2), (int)Xq.size(3), how.norm, how.eps, code_of(Xq), sums ? data(ws) : nullptr, bytes, stream_of(Xq));
        }
        throw_on(rc);
        return once({d[0], d[1], d[2], d[3], at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor()});
    }
};

// heads_forward(Xq, Xk, wq, wk, positions, inv_freq, sections, interleaved, norm, eps, Q, K, differentiable) -> (Q, K)
PyObject* heads_forward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arguments(n, 13)) return nullptr;
    const at::Tensor *Xq = tensor(args[0]), *Xk, *wq, *wk, *positions, *inv_freq, *given_q, *given_k;
    const double eps = PyFloat_AsDouble(args[9]);
    if (PyErr_Occurred()) return nullptr;
    if (!Xq || !optional(args[1], Xk) || !optional(args[2], wq) || !optional(args[3], wk) || !optional(args[4], positions) || !optional(args[5], inv_freq) ||
        !optional(args[10], given_q) || !optional(args[11], given_k) || !ready() || !(eps >= 0))
        Py_RETURN_NONE;
    HeadsHow how;
    how.interleaved = args[7] == Py_True, how.norm = args[8] == Py_True, how.eps = (float)eps;
    const bool differentiable = args[12] == Py_True;
    Py_ssize_t listed = -1;                        // sections
    if (args[6] != Py_None) {
        if (!PyList_CheckExact(args[6]) || (listed = PyList_GET_SIZE(args[6])) < 1 || listed > 3) Py_RETURN_NONE;
        for (Py_ssize_t i = 0; i < listed; ++i) {
            PyObject* x = PyList_GET_ITEM(args[6], i);
            const long v = PyLong_CheckExact(x) ? PyLong_AsLong(x) : -1;
            PyErr_Clear();
            if (v < 0 || v > 1 << 20) Py_RETURN_NONE;
            how.sections[i] = (int)v;
        }
    }
    at::Tensor Q, K;
    int rc = 0;
    try {
        if (!Xq->is_cuda() || Xq->dim() != 4 || code_of(*Xq) < 0 || (Xk && Xk->dim() != 4) || (!Xk && (wk || given_k))) Py_RETURN_NONE;
        const at::Device device = Xq->device();
        const at::ScalarType type = Xq->scalar_type();
        const int64_t B = Xq->size(0), N = Xq->size(1), Hq = Xq->size(2), d = Xq->size(3), Hk = Xk ? Xk->size(2) : 0, most = INT_MAX;
        if (B > most || N > most || Hq > most || Hk > most || d < 1 || d > most || (Xk && Hk < 1)) Py_RETURN_NONE;
        const int64_t xq[4] = {B, N, Hq, d}, xk[4] = {B, N, Hk, d}, q[4] = {B, Hq, N, d}, k[4] = {B, Hk, N, d}, w[1] = {d}, f[1] = {d / 2};
        if (!rows_fit(*Xq, xq, type, device) || (Xk && !rows_fit(*Xk, xk, type, device)) || (wq && !fits(*wq, w, type, device)) || (wk && !fits(*wk, w, type, device)) ||
            (given_q && !rows_fit(*given_q, q, type, device)) || (given_k && !rows_fit(*given_k, k, type, device)))
            Py_RETURN_NONE;
        if (positions) {
            const at::Tensor& p = *positions;
            if ((p.scalar_type() != at::kLong && p.scalar_type() != at::kInt) || p.device() != device || p.layout() != at::kStrided || p.dim() < 1 || p.dim() > 3 ||
                p.size(-1) != N || (N > 1 && p.stride(-1) != 1) || (p.dim() > 1 && p.size(-2) != B && p.size(-2) != 1) || !inv_freq ||
                !fits(*inv_freq, f, at::kFloat, device))
                Py_RETURN_NONE;
            how.axes = p.dim() == 3 ? (int)p.size(0) : 1;
            if (how.axes < 1 || how.axes > 3 || (listed < 0 ? how.axes > 1 : listed != how.axes)) Py_RETURN_NONE;
            if (listed < 0) how.sections[0] = (int)(d / 2);
            if (how.sections[0] + how.sections[1] + how.sections[2] != d / 2) Py_RETURN_NONE;
        } else if (inv_freq || listed >= 0) {
            Py_RETURN_NONE;
        }
        if (differentiable && (!Xk || !wq || !wk)) Py_RETURN_NONE;
        const Unlocked unlocked;
        if (differentiable) {
            auto out = HeadNormRotary::apply(*Xq, *Xk, *wq, *wk, positions ? std::optional<at::Tensor>(*positions) : std::nullopt,
                                             inv_freq ? std::optional<at::Tensor>(*inv_freq) : std::nullopt, (const HeadsHow*)&how, &rc);
            Q = out[0], K = out[1];
        } else {
            if (given_q) Q = *given_q;
            if (given_k) K = *given_k;
            rotate_heads(*Xq, Xk, wq, wk, positions, inv_freq, how, Q, K, rc);
            if (rc == 0)                           // (autograd is told, as by torch's own operations in place)
                for (const at::Tensor* o : {given_q, given_k})
                    if (o && !o->is_inference()) o->unsafeGetTensorImpl()->bump_version();
        }
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    return rc != 0 ? raised(rc) : tuple_of({&Q, &K});
}

at::Tensor gated(const at::Tensor& X, const at::Tensor& Wg, const at::Tensor& Wu, int gate, int& rc)
{
    const int F = (int)Wg.size(0), D = (int)Wg.size(1), T = (int)(X.numel() / D);
    std::vector<int64_t> shape = X.sizes().vec();
    shape.back() = F;
    at::Tensor H = at::empty(shape, X.options());
    const size_t bytes = entry.ffn_bytes(T, D, F, code_of(X));
    const at::Tensor ws = bytes ? bytes_of(bytes, X) : at::Tensor();
    rc = entry.ffn(data(X), data(Wg), data(Wu), data(H), T, D, F, gate, code_of(X), bytes ? data(ws) : nullptr, bytes, stream_of(X));
    return H;
}

struct GatedFeedForward : torch::autograd::Function<GatedFeedForward> {
    static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& X, const at::Tensor& Wg, const at::Tensor& Wu, int64_t gate, int* rc)
    {
        at::Tensor H = gated(X, Wg, Wu, (int)gate, *rc);
        ctx->save_for_backward({X, Wg, Wu});
        ctx->saved_data["gate"] = gate;
        return H;
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        const auto saved = ctx->get_saved_variables();
        const at::Tensor &X = saved[0], &Wg = saved[1];
        at::Tensor d[3];
        int rc = 0;
        {
            const at::NoGradGuard off;
            const at::Tensor dH = grads[0].contiguous();
            const int F = (int)Wg.size(0), D = (int)Wg.size(1), T = (int)(X.numel() / D);
            for (int i = 0; i < 3; ++i)
                if (ctx->needs_input_grad(i)) d[i] = at::empty_like(saved[i]);
            const size_t bytes = entry.ffn_bwd_bytes(T, D, F, code_of(X));
            const at::Tensor ws = bytes_of(bytes, X);
            auto or_null = [](const at::Tensor& t) { return t.defined() ? data(t) : nullptr; };
            rc = entry.ffn_bwd(data(X), data(Wg), data(saved[2]), data(dH), or_null(d[0]), or_null(d[1]), or_null(d[2]), T, D, F, (int)ctx->saved_data["gate"].toInt(),
                               code_of(X), data(ws), bytes, stream_of(X));
        }
        throw_on(rc);
        return once({d[0], d[1], d[2], at::Tensor(), at::Tensor()});
    }
};

// ffn_forward(X, Wg, Wu, gate, differentiable) -> H
PyObject* ffn_forward(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (!arguments(n, 5)) return nullptr;
    const at::Tensor *X = tensor(args[0]), *Wg = tensor(args[1]), *Wu = tensor(args[2]);
    const long gate = PyLong_AsLong(args[3]);
    if (PyErr_Occurred()) return nullptr;
    if (!X || !Wg || !Wu || !ready()) Py_RETURN_NONE;
    at::Tensor H;
    int rc = 0;
    try {
        const bool differentiable = args[4] == Py_True;
        if (!X->is_cuda() || code_of(*X) < 0 || X->dim() < 1 || (!differentiable && X->dim() != 2) || Wg->dim() != 2) Py_RETURN_NONE;
        const at::Device device = X->device();
        if (!plain(*X, device) || !fits(*Wg, Wg->sizes(), X->scalar_type(), device) || !fits(*Wu, Wg->sizes(), X->scalar_type(), device) ||
            X->size(-1) != Wg->size(1) || Wg->size(1) < 1 || Wg->size(1) > INT_MAX || Wg->size(0) < 1 || Wg->size(0) > INT_MAX || X->numel() / Wg->size(1) > INT_MAX)
            Py_RETURN_NONE;
        const Unlocked unlocked;
        H = differentiable ? GatedFeedForward::apply(*X, *Wg, *Wu, (int64_t)gate, &rc) : gated(*X, *Wg, *Wu, (int)gate, rc);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    return rc != 0 ? raised(rc) : wrapped(std::move(H));
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
    constexpr Py_ssize_t COUNT = 28;
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
        entry.embed_bwd, entry.loss_bytes, entry.loss, entry.loss_bwd_bytes, entry.loss_bwd, entry.clip_bytes, entry.clip,
        entry.distill_bytes, entry.distill, entry.distill_bwd_bytes, entry.distill_bwd, entry.heads, entry.heads_bwd_bytes, entry.heads_bwd, entry.ffn_bytes,
        entry.ffn, entry.ffn_bwd_bytes, entry.ffn_bwd, entry.text);
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
                         {"distill_forward", (PyCFunction)(void*)distill_forward, METH_FASTCALL, nullptr},
                         {"heads_forward", (PyCFunction)(void*)heads_forward, METH_FASTCALL, nullptr},
                         {"ffn_forward", (PyCFunction)(void*)ffn_forward, METH_FASTCALL, nullptr},
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
