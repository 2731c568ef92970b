// The module _bqhost's half for the operators around the optimizer step, in the manner
// of bq_host.cpp.
//
// bq.py, nn.py and optim.py describe each call completely and stay the reference for it.
// The functions here do the same for the ordinary case -- plain GPU tensors of the right
// types and sizes on the current device and stream, all checks passing -- and return None
// for anything else, whereupon the Python code runs as if they did not exist.  Nothing is
// remembered between calls.
//
// Why: a training pass through a small layer norm took 180 us of host time, of which the
// backward pass's Python in the engine's thread was 100; the gradients of the ResNet-50
// list (161 tensors) 260 us to collect.
#include "bq_host.h"

#include <cstring>
#include <optional>
#include <unordered_set>
#include <vector>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/TracerMode.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/forward_grad.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/python_variable.h>

#include "bq.h"

namespace {

using namespace bq_host;

// Entry points of the libbq.so that bq.py loaded (addresses passed to bind).
struct Library {
    decltype(&bq_layer_norm_forward) norm_forward;
    decltype(&bq_layer_norm_workspace_bytes) norm_workspace;
    decltype(&bq_layer_norm_backward) norm_backward;
    decltype(&bq_embedding_forward) lookup;
    decltype(&bq_embedding_workspace_bytes) lookup_workspace;
    decltype(&bq_embedding_backward) lookup_backward;
    decltype(&bq_stable_embedding_forward) stable;
    decltype(&bq_stable_embedding_workspace_bytes) stable_workspace;
    decltype(&bq_stable_embedding_backward) stable_backward;
    decltype(&bq_grad_norm_workspace_bytes) clip_workspace;
    decltype(&bq_grad_norm) grad_norm;
    decltype(&bq_clip_grad_norm) clip;
} lib;
constexpr int kEntries = 12;

// Calls that only the Python code goes through: Python modes, torch.func's transforms,
// and what it refuses: tracing, and tensors with a forward-mode tangent (of which there are
// some only while a dual level is entered: asking each of a list's 161 gradients instead
// took 6 us).
bool modes()
{
    return at::tracer::impl::is_dispatch_enabled() ||
           c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::PreDispatch) ||
           c10::impl::TorchDispatchModeTLS::any_modes_set() ||
           at::impl::PythonTorchFunctionTLS::stack_len() != 0 ||
           c10::impl::tls_local_dispatch_key_set().included_.has(
               c10::DispatchKey::FuncTorchDynamicLayerFrontMode) ||
           torch::autograd::ForwardADLevel::try_get_by_idx(0) != nullptr;
}

// Runs f without the interpreter lock, which the functions below hold when Python calls
// them; the engine calls the backward passes without it.
template <class F>
auto unlocked(F f)
{
    struct Lock {
        PyThreadState *save = PyEval_SaveThread();
        ~Lock() { PyEval_RestoreThread(save); }
    } lock;
    return f();
}

// The tensor that f computes, without the interpreter lock.  An exception of Python code
// that it ran (hooks on the tensors that it saved; checkpointing ends a recomputation by
// one) is the call's, which is not made again.
template <class F>
PyObject *computed(F f)
{
    try {
        return THPVariable_Wrap(unlocked(f));
    } catch (python_error &e) {
        e.restore();
    } catch (pybind11::error_already_set &e) {
        e.restore();
    }
    return PyErr_Occurred() ? nullptr : none();
}

void succeed(bq_status s, const char *what)
{
    TORCH_CHECK(s == BQ_OK, what, " failed (status ", static_cast<int>(s), ")");
}

bq_dtype dtype_of(at::ScalarType t)
{
    need(t == at::kFloat || t == at::kHalf || t == at::kBFloat16);
    return t == at::kFloat ? BQ_F32 : t == at::kHalf ? BQ_F16 : BQ_BF16;
}

// Whether the tensor's elements are there: its storage may have been emptied (sharded
// training does so), and a null parameter stands for ones or zeros in the C calls.
bool in_memory(const at::Tensor &t) { return t.numel() == 0 || t.storage().data() != nullptr; }

// A dense tensor with memory of its own on the device.
const at::Tensor &dense(const at::Tensor &t, int device)
{
    need(t.is_cuda() && t.layout() == at::kStrided && t.get_device() == device &&
         t.has_storage() && in_memory(t) && !t.is_neg() && !t.is_conj());
    return t;
}

const at::Tensor &tensor(PyObject *o, int device)
{
    need(THPVariable_CheckExact(o));
    return dense(THPVariable_Unpack(o), device);
}

// An optional parameter vector of n elements (an undefined tensor for None).
at::Tensor vector(PyObject *o, int64_t n, at::ScalarType type, int device)
{
    if (o == Py_None)
        return at::Tensor();
    const at::Tensor &t = tensor(o, device);
    need(t.scalar_type() == type && t.numel() == n && t.is_contiguous());
    return t;
}

double real(PyObject *o)
{
    const double d = PyFloat_AsDouble(o);
    if (d == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        throw NotHandled{};
    }
    return d;
}

bool truth(PyObject *o)
{
    need(o == Py_True || o == Py_False);
    return o == Py_True;
}

hipStream_t current(const at::Tensor &t)
{
    return c10::hip::getCurrentHIPStream(t.device().index()).stream();
}

void *data(const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }

bool wants_grad(std::initializer_list<const at::Tensor *> tensors)
{
    if (!at::GradMode::is_enabled())
        return false;
    for (const at::Tensor *t : tensors)
        if (t->defined() && t->requires_grad())
            return true;
    return false;
}

using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

// A parameter as an argument of an autograd function: one that is left out is no tensor
// (an undefined tensor may not be an input), and has no edge in the graph.
using Param = std::optional<at::Tensor>;
Param param(const at::Tensor &t) { return t.defined() ? Param(t) : std::nullopt; }
at::Tensor given(const Param &p) { return p.has_value() ? *p : at::Tensor(); }

// Whether the gradients of a weight and a bias are wanted, whose edges begin at `edge`.
void wanted(AutogradContext *ctx, size_t edge, bool weight, bool &need_w, bool &need_b)
{
    const bool bias = ctx->saved_data["bias"].toBool();
    need_w = weight && ctx->needs_input_grad(edge);
    need_b = bias && ctx->needs_input_grad(edge + weight);
}

// What comes into a backward pass, as values in memory.
at::Tensor incoming(const at::Tensor &dy)
{
    TORCH_CHECK_NOT_IMPLEMENTED(!dy._fw_grad(/*level=*/0).defined(),
                                "libbq's kernels have no forward-mode derivatives");
    return dy.resolve_neg();
}

// A tensor that the forward pass saved.  Hooks on saved tensors (as of
// torch.autograd.graph.saved_tensors_hooks) may hand back another one than they were
// given, and its memory may be gone: what the kernels read through its address is checked
// again.
at::Tensor checked(const at::Tensor &t, at::IntArrayRef sizes, at::ScalarType type,
                   at::Device device)
{
    TORCH_CHECK(t.layout() == at::kStrided && t.device() == device && t.scalar_type() == type &&
                    t.sizes() == sizes,
                "a saved tensor came back on another device, or of another type or shape");
    TORCH_CHECK(in_memory(t), "a saved tensor has no memory any more");
    return t.resolve_neg();
}

// The same packed; an undefined tensor as it is.
at::Tensor saved_as(const at::Tensor &t, at::IntArrayRef sizes, at::ScalarType type,
                    at::Device device)
{
    return t.defined() ? checked(t, sizes, type, device).contiguous() : t;
}

// Saved token ids.
at::Tensor saved_ids(const at::Tensor &t, at::IntArrayRef sizes, at::Device device)
{
    return saved_as(t, sizes, t.scalar_type() == at::kInt ? at::kInt : at::kLong, device);
}

// Gradients of first order: as Python's once_differentiable, a second derivative raises.
variable_list once(variable_list grads)
{
    if (!at::GradMode::is_enabled())
        return grads;
    variable_list outs;
    for (at::Tensor &g : grads)
        if (g.defined())
            outs.push_back(g.detach().set_requires_grad(true));
    if (outs.empty())
        return grads;
    torch::autograd::DelayedError error(
        "trying to differentiate twice a function that was marked with @once_differentiable",
        static_cast<int64_t>(outs.size()));
    outs = error.apply(std::move(outs));
    size_t i = 0;
    for (at::Tensor &g : grads)
        if (g.defined())
            g = outs[i++];
    return grads;
}

// ---------------------------------------------------------------------------
// layer norm
// ---------------------------------------------------------------------------

struct Rows {
    int64_t rows, cols, stride;
};
bool packed_rows(const at::Tensor &t)
{
    return t.is_contiguous() || (t.dim() == 2 && (t.stride(1) == 1 || t.size(1) == 1));
}
Rows rows_of(const at::Tensor &t)
{
    const int64_t cols = t.size(-1);
    if (t.is_contiguous())
        return {t.numel() / cols, cols, cols};
    return {t.size(0), cols, t.stride(0)};
}

at::Tensor norm_forward(const at::Tensor &x, const at::Tensor &w, const at::Tensor &b, double eps,
                        at::Tensor *mean, at::Tensor *rstd)
{
    const Rows r = rows_of(x);
    const at::ScalarType pt = w.defined() ? w.scalar_type() : b.defined() ? b.scalar_type()
                                                                          : x.scalar_type();
    at::Tensor y = at::empty(x.sizes(), x.options());
    if (mean) {
        *mean = at::empty({r.rows}, x.options().dtype(at::kFloat));
        *rstd = at::empty({r.rows}, x.options().dtype(at::kFloat));
    }
    const bq_dtype xt = dtype_of(x.scalar_type()), wt = dtype_of(pt);
    const hipStream_t stream = current(x);
    succeed(lib.norm_forward(xt, wt, data(x), r.rows, r.cols, r.stride, data(w), data(b),
                             static_cast<float>(eps), data(y),
                             static_cast<float *>(mean ? data(*mean) : nullptr),
                             static_cast<float *>(rstd ? data(*rstd) : nullptr), stream),
            "bq_layer_norm_forward");
    return y;
}

struct LayerNorm : torch::autograd::Function<LayerNorm> {
    static at::Tensor forward(AutogradContext *ctx, const at::Tensor &x, const Param &weight,
                              const Param &bias, double eps)
    {
        const at::Tensor w = given(weight), b = given(bias);
        at::Tensor mean, rstd;
        at::Tensor y = norm_forward(x, w, b, eps, &mean, &rstd);
        ctx->save_for_backward({x, w, mean, rstd});
        ctx->saved_data["bias"] = b.defined();
        ctx->saved_data["param"] = static_cast<int64_t>(
            w.defined() ? w.scalar_type() : b.defined() ? b.scalar_type() : x.scalar_type());
        return y;
    }

    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        const variable_list saved = ctx->get_saved_variables();
        const bool need_x = ctx->needs_input_grad(0);
        bool need_w, need_b;
        wanted(ctx, 1, saved[1].defined(), need_w, need_b);
        at::Tensor dy = incoming(grads[0]);
        const at::DeviceGuard guard(dy.device());
        if (!packed_rows(dy))
            dy = dy.contiguous();
        const auto pt = static_cast<at::ScalarType>(ctx->saved_data["param"].toInt());
        const Rows g = rows_of(dy);
        at::Tensor x = checked(saved[0], dy.sizes(), dy.scalar_type(), dy.device());
        if (!packed_rows(x))
            x = x.contiguous();
        const at::Tensor w = saved_as(saved[1], {g.cols}, pt, dy.device());
        const at::Tensor mean = saved_as(saved[2], {g.rows}, at::kFloat, dy.device());
        const at::Tensor rstd = saved_as(saved[3], {g.rows}, at::kFloat, dy.device());
        const Rows r = rows_of(x);
        at::Tensor dx, dw, db, ws;
        if (need_x)
            dx = at::empty(x.sizes(), x.options());
        if (need_w || need_b) {
            if (need_w)
                dw = at::empty({r.cols}, x.options().dtype(pt));
            if (need_b)
                db = at::empty({r.cols}, x.options().dtype(pt));
            ws = at::empty({lib.norm_workspace(r.rows, r.cols)}, x.options().dtype(at::kByte));
        }
        succeed(lib.norm_backward(dtype_of(x.scalar_type()), dtype_of(pt), data(dy), g.stride,
                                  data(x), r.stride, r.rows, r.cols, data(w),
                                  static_cast<const float *>(data(mean)),
                                  static_cast<const float *>(data(rstd)), data(dx), data(dw),
                                  data(db), data(ws), current(x)),
                "bq_layer_norm_backward");
        return once({dx, dw, db, at::Tensor()});
    }
};

// layer_norm(x, weight, bias, eps, with gradients) -> y or None
PyObject *layer_norm(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return handled([&]() -> PyObject * {
        need(nargs == 5);
        if (modes() || !plain({args[0], args[1], args[2]}))
            return none();
        const int device = c10::hip::current_device();
        const at::Tensor &x = tensor(args[0], device);
        need(x.dim() > 0 && x.numel() > 0 && packed_rows(x));
        dtype_of(x.scalar_type());
        const int64_t cols = x.size(-1);
        PyObject *const given = args[1] != Py_None ? args[1] : args[2];
        const at::ScalarType pt =
            given == Py_None ? x.scalar_type() : THPVariable_Unpack(given).scalar_type();
        need(pt == at::kFloat || pt == x.scalar_type());
        const at::Tensor w = vector(args[1], cols, pt, device);
        const at::Tensor b = vector(args[2], cols, pt, device);
        const double eps = real(args[3]);
        const bool grads = truth(args[4]) && wants_grad({&x, &w, &b});
        return computed([&] {
            return grads ? LayerNorm::apply(x, param(w), param(b), eps)
                         : norm_forward(x, w, b, eps, nullptr, nullptr);
        });
    });
}

// ---------------------------------------------------------------------------
// embedding, stable embedding
// ---------------------------------------------------------------------------

std::vector<int64_t> output_sizes(const at::Tensor &ids, const at::Tensor &w)
{
    std::vector<int64_t> sizes = ids.sizes().vec();
    sizes.push_back(w.size(1));
    return sizes;
}

int32_t id_bits(const at::Tensor &ids) { return ids.scalar_type() == at::kLong ? 64 : 32; }

at::Tensor lookup_forward(const at::Tensor &ids, const at::Tensor &w, double scale,
                          at::ScalarType out)
{
    at::Tensor y = at::empty(output_sizes(ids, w), w.options().dtype(out));
    succeed(lib.lookup(dtype_of(w.scalar_type()), dtype_of(out), data(w), w.size(0), w.size(1),
                       data(ids), id_bits(ids), ids.numel(), static_cast<float>(scale), data(y),
                       current(w)),
            "bq_embedding_forward");
    return y;
}

struct Embedding : torch::autograd::Function<Embedding> {
    static at::Tensor forward(AutogradContext *ctx, const at::Tensor &ids, const at::Tensor &w,
                              int64_t padding, double scale, int64_t out)
    {
        at::Tensor y = lookup_forward(ids, w, scale, static_cast<at::ScalarType>(out));
        ctx->save_for_backward({ids});
        ctx->saved_data["num"] = w.size(0);
        ctx->saved_data["dtype"] = static_cast<int64_t>(w.scalar_type());
        ctx->saved_data["padding"] = padding;
        ctx->saved_data["scale"] = scale;
        return y;
    }

    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        const at::Tensor dy = incoming(grads[0]).contiguous();
        const at::DeviceGuard guard(dy.device());
        const at::Tensor ids = saved_ids(ctx->get_saved_variables()[0],
                                         dy.sizes().slice(0, dy.dim() - 1), dy.device());
        const int64_t num = ctx->saved_data["num"].toInt(), dim = dy.size(-1);
        const auto type = static_cast<at::ScalarType>(ctx->saved_data["dtype"].toInt());
        const auto scale = static_cast<float>(ctx->saved_data["scale"].toDouble());
        at::Tensor dw = at::empty({num, dim}, dy.options().dtype(type));
        at::Tensor ws = at::empty({lib.lookup_workspace(ids.numel(), num, dim)},
                                  dy.options().dtype(at::kByte));
        succeed(lib.lookup_backward(dtype_of(type), dtype_of(dy.scalar_type()), data(dy), data(ids),
                                    id_bits(ids), ids.numel(), num, dim,
                                    ctx->saved_data["padding"].toInt(), scale, data(dw), data(ws),
                                    current(dy)),
                "bq_embedding_backward");
        return once({at::Tensor(), dw, at::Tensor(), at::Tensor(), at::Tensor()});
    }
};

// The table, the ids, the padding row and the result's type of a lookup.
struct Lookup {
    at::Tensor w, ids;
    int64_t padding;
    at::ScalarType out;
};
Lookup lookup_of(PyObject *ids, PyObject *weight, PyObject *padding, PyObject *out, int device)
{
    Lookup l;
    l.w = tensor(weight, device);
    l.ids = tensor(ids, device);
    dtype_of(l.w.scalar_type());
    need(l.w.dim() == 2 && l.w.is_contiguous() && l.w.numel() > 0 && l.ids.is_contiguous() &&
         l.ids.numel() > 0 && (l.ids.scalar_type() == at::kLong || l.ids.scalar_type() == at::kInt));
    l.padding = -1;
    if (padding != Py_None) {
        const int64_t p = whole(padding), num = l.w.size(0);
        need(p >= -num && p < num);
        l.padding = p < 0 ? p + num : p;
    }
    l.out = l.w.scalar_type();
    if (out != Py_None) {
        need(THPDtype_Check(out));
        l.out = reinterpret_cast<THPDtype *>(out)->scalar_type;
        dtype_of(l.out);
        need(l.w.scalar_type() == at::kFloat || l.w.scalar_type() == l.out);
    }
    return l;
}

// embedding(ids, weight, padding, scale, out dtype, with gradients) -> y or None
PyObject *embedding(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return handled([&]() -> PyObject * {
        need(nargs == 6);
        if (modes() || !plain({args[0], args[1]}))
            return none();
        const Lookup l = lookup_of(args[0], args[1], args[2], args[4], c10::hip::current_device());
        const double scale = real(args[3]);
        const bool grads = truth(args[5]) && wants_grad({&l.w});
        return computed([&] {
            return grads ? Embedding::apply(l.ids, l.w, l.padding, scale,
                                            static_cast<int64_t>(l.out))
                         : lookup_forward(l.ids, l.w, scale, l.out);
        });
    });
}

at::Tensor stable_forward(const at::Tensor &ids, const at::Tensor &w, const at::Tensor &nw,
                          const at::Tensor &nb, double eps, at::ScalarType out)
{
    at::Tensor y = at::empty(output_sizes(ids, w), w.options().dtype(out));
    succeed(lib.stable(dtype_of(w.scalar_type()), dtype_of(out), data(w), w.size(0), w.size(1),
                       data(ids), id_bits(ids), ids.numel(), data(nw), data(nb),
                       static_cast<float>(eps), data(y), current(w)),
            "bq_stable_embedding_forward");
    return y;
}

struct StableEmbedding : torch::autograd::Function<StableEmbedding> {
    static at::Tensor forward(AutogradContext *ctx, const at::Tensor &ids, const at::Tensor &w,
                              const Param &weight, const Param &bias, double eps,
                              int64_t padding, int64_t out)
    {
        const at::Tensor nw = given(weight), nb = given(bias);
        at::Tensor y = stable_forward(ids, w, nw, nb, eps, static_cast<at::ScalarType>(out));
        ctx->save_for_backward({ids, w, nw});
        ctx->saved_data["num"] = w.size(0);
        ctx->saved_data["dtype"] = static_cast<int64_t>(w.scalar_type());
        ctx->saved_data["bias"] = nb.defined();
        ctx->saved_data["eps"] = eps;
        ctx->saved_data["padding"] = padding;
        return y;
    }

    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        const variable_list saved = ctx->get_saved_variables();
        const at::Tensor dy = incoming(grads[0]).contiguous();
        const at::DeviceGuard guard(dy.device());
        const int64_t num = ctx->saved_data["num"].toInt(), dim = dy.size(-1);
        const auto type = static_cast<at::ScalarType>(ctx->saved_data["dtype"].toInt());
        const at::Tensor ids =
            saved_ids(saved[0], dy.sizes().slice(0, dy.dim() - 1), dy.device());
        const at::Tensor w = saved_as(saved[1], {num, dim}, type, dy.device());
        const at::Tensor nw = saved_as(saved[2], {dim}, type, dy.device());
        const bool need_w = ctx->needs_input_grad(1);
        bool need_nw, need_nb;
        wanted(ctx, 2, nw.defined(), need_nw, need_nb);
        at::Tensor dw = at::empty({num, dim}, w.options()), dnw, dnb;
        if (need_nw)
            dnw = at::empty({dim}, w.options());
        if (need_nb)
            dnb = at::empty({dim}, w.options());
        at::Tensor ws = at::empty({lib.stable_workspace(ids.numel(), num, dim)},
                                  w.options().dtype(at::kByte));
        succeed(lib.stable_backward(
                    dtype_of(w.scalar_type()), dtype_of(dy.scalar_type()), data(dy), data(ids),
                    id_bits(ids), ids.numel(), data(w), num, dim,
                    ctx->saved_data["padding"].toInt(), data(nw),
                    static_cast<float>(ctx->saved_data["eps"].toDouble()), data(dw), data(dnw),
                    data(dnb), data(ws), current(w)),
                "bq_stable_embedding_backward");
        if (!need_w)
            dw = at::Tensor();
        return once({at::Tensor(), dw, dnw, dnb, at::Tensor(), at::Tensor(), at::Tensor()});
    }
};

// stable_embedding(ids, weight, norm weight, norm bias, eps, padding, out dtype, with
// gradients) -> y or None
PyObject *stable_embedding(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return handled([&]() -> PyObject * {
        need(nargs == 8);
        if (modes() || !plain({args[0], args[1], args[2], args[3]}))
            return none();
        const int device = c10::hip::current_device();
        const Lookup l = lookup_of(args[0], args[1], args[5], args[6], device);
        const at::Tensor nw = vector(args[2], l.w.size(1), l.w.scalar_type(), device);
        const at::Tensor nb = vector(args[3], l.w.size(1), l.w.scalar_type(), device);
        const double eps = real(args[4]);
        const bool grads = truth(args[7]) && wants_grad({&l.w, &nw, &nb});
        return computed([&] {
            return grads ? StableEmbedding::apply(l.ids, l.w, param(nw), param(nb), eps, l.padding,
                                                  static_cast<int64_t>(l.out))
                         : stable_forward(l.ids, l.w, nw, nb, eps, l.out);
        });
    });
}

// ---------------------------------------------------------------------------
// gradient norm and clipping
// ---------------------------------------------------------------------------

// Whether the tensor's elements fill one range of memory, in any order.
bool one_range(const at::Tensor &t) { return t.is_contiguous() || t.is_non_overlapping_and_dense(); }

// clip(list of parameters, max norm or None, kind) -> the norm of their gradients (clipped
// in place unless max norm is None), the status of a C call that failed (which must not be
// made again: some of its launches may have run), or None
PyObject *clip(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return handled([&]() -> PyObject * {
        need(nargs == 3 && PyList_CheckExact(args[0]));
        if (modes())
            return none();
        const bool clips = args[1] != Py_None;
        const double max_norm = clips ? real(args[1]) : 0.0;
        const auto kind = static_cast<bq_norm>(whole(args[2]));
        const int device = c10::hip::current_device();
        const Py_ssize_t n = PyList_GET_SIZE(args[0]);
        std::vector<bq_grad> list;
        std::vector<at::Tensor> grads;
        std::unordered_set<const void *> seen;
        list.reserve(n);
        grads.reserve(n);
        seen.reserve(n);
        for (Py_ssize_t i = 0; i < n; ++i) {
            PyObject *const o = PyList_GET_ITEM(args[0], i);
            if (!THPVariable_CheckExact(o))
                return none();
            const at::Tensor &g = THPVariable_Unpack(o).grad();
            if (!g.defined() || !seen.insert(g.unsafeGetTensorImpl()).second)
                continue;
            PyObject *const go = THPVariable_Wrap(g);  // its class (as in _bqhost)
            need(go != nullptr);
            const bool exact = THPVariable_CheckExact(go);
            Py_DECREF(go);
            if (!exact)
                return none();
            dense(g, device);
            // (two gradients in the same place: Python refuses to clip them)
            need(one_range(g) && (g.numel() == 0 || !clips || seen.insert(g.data_ptr()).second));
            list.push_back({g.data_ptr(), g.numel(), dtype_of(g.scalar_type())});
            grads.push_back(g);
        }
        need(!list.empty() && list.size() <= INT32_MAX);
        const int32_t count = static_cast<int32_t>(list.size());
        at::Tensor norm = at::empty({}, grads[0].options().dtype(at::kFloat));
        at::Tensor ws = at::empty({lib.clip_workspace(count)}, grads[0].options().dtype(at::kByte));
        const hipStream_t stream = current(norm);
        float *const out = static_cast<float *>(norm.data_ptr());
        const bq_status status = unlocked([&] {
            return clips ? lib.clip(list.data(), count, kind, max_norm, ws.data_ptr(), out, stream)
                         : lib.grad_norm(list.data(), count, kind, ws.data_ptr(), out, stream);
        });
        // (a call that failed on the GPU's side may have scaled some of them)
        if (clips && (status == BQ_OK || status == BQ_ERR_HIP))
            for (const at::Tensor &g : grads)
                if (!g.is_inference())
                    g.unsafeGetTensorImpl()->bump_version();
        return status == BQ_OK ? THPVariable_Wrap(norm) : PyLong_FromLong(status);
    });
}

// bind_ops(addresses): the addresses of lib's entry points, in its order.
PyObject *bind_ops(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 1 || !PyTuple_CheckExact(args[0]) || PyTuple_GET_SIZE(args[0]) != kEntries) {
        PyErr_Format(PyExc_TypeError, "bind_ops takes a tuple of %d addresses", kEntries);
        return nullptr;
    }
    static_assert(sizeof(Library) == kEntries * sizeof(void *), "one pointer each");
    void *p[kEntries];
    for (int i = 0; i < kEntries; ++i) {
        p[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(args[0], i));
        if (!p[i]) {
            if (!PyErr_Occurred())
                PyErr_SetString(PyExc_ValueError, "null address");
            return nullptr;
        }
    }
    std::memcpy(&lib, p, sizeof(lib));
    return none();
}

}  // namespace

PyMethodDef bq_ops_methods[] = {
    {"bind_ops", reinterpret_cast<PyCFunction>(bind_ops), METH_FASTCALL, nullptr},
    {"layer_norm", reinterpret_cast<PyCFunction>(layer_norm), METH_FASTCALL, nullptr},
    {"embedding", reinterpret_cast<PyCFunction>(embedding), METH_FASTCALL, nullptr},
    {"stable_embedding", reinterpret_cast<PyCFunction>(stable_embedding), METH_FASTCALL, nullptr},
    {"clip", reinterpret_cast<PyCFunction>(clip), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
