// The usual calls of the operators around a model's blocks and at the ends of its backward pass, from Python to the library and back
// through autograd without the interpreter in between: packed CUDA tensors of plain types, no tracing, no transforms. Where a call is not
// of that kind its function returns None, and the caller's own path takes it, with its checks, copies and errors. The library is reached
// through addresses that bind() is given, the same that ctypes has.
//
// What it is for: a training pass of rms_norm over a few rows takes the host 125 us through Python functions and ctypes, where its kernels
// take 10.
#include <Python.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>
#include <ATen/ATen.h>

#include <memory>
#include <optional>
#include <stdexcept>
#include <string>
#include <vector>

#include "../../include/compams.h"

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

struct Entries {
    decltype(&compams_rms_norm_forward) rms_norm_forward;
    decltype(&compams_rms_norm_backward) rms_norm_backward;
    decltype(&compams_rms_norm_workspace_bytes) rms_norm_workspace_bytes;
    decltype(&compams_head_forward) head_forward;
    decltype(&compams_head_backward) head_backward;
    decltype(&compams_head_workspace_bytes) head_workspace_bytes;
    decltype(&compams_collect_workers) collect_workers;
    decltype(&compams_collect_workers_workspace_bytes) collect_workers_workspace_bytes;
    decltype(&compams_error_string) error_string;
    decltype(&compams_last_cuda_error) last_cuda_error;
} entry = {};

// What the library refuses or fails at: the binding's own error in Python, where it comes from a backward pass a RuntimeError.
struct LibraryError : std::runtime_error {
    using std::runtime_error::runtime_error;
};
PyObject* library_error = nullptr;

void check(int rc, const char* what) {
    if (rc == COMPAMS_OK) return;
    const std::string cuda = entry.last_cuda_error();
    throw LibraryError(std::string(what) + " failed: " + entry.error_string(rc) + " (" + std::to_string(rc) + ")" +
                             (cuda.empty() ? "" : " [" + cuda + "]"));
}

int type_of(const Tensor& t) {
    switch (t.scalar_type()) {
        case at::kFloat: return COMPAMS_F32;
        case at::kBFloat16: return COMPAMS_BF16;
        case at::kHalf: return COMPAMS_F16;
        default: return -1;
    }
}

// A tensor as the operators' usual calls have it: of torch's own kind, in CUDA memory, packed.
bool usual(const Tensor& t) {
    using c10::DispatchKey;
    const auto keys = t.key_set();
    return t.is_cuda() && t.layout() == c10::kStrided && t.is_contiguous() && !keys.has(DispatchKey::Python) && !keys.has(DispatchKey::Negative) &&
           !keys.has(DispatchKey::Conjugate) && !keys.has(DispatchKey::ZeroTensor) && !keys.has(DispatchKey::FuncTorchBatched) &&
           !keys.has(DispatchKey::FuncTorchGradWrapper) && !keys.has(DispatchKey::Functionalize);
}
// Whether nobody looks on: no tracer, no dispatch mode, no transform. (Forward-mode levels are the caller's question.)
bool alone() {
    return !torch::jit::tracer::isTracing() && !c10::impl::TorchDispatchModeTLS::any_modes_set() &&
           !c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::FuncTorchDynamicLayerFrontMode) &&
           !c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::Python);
}
// An activation [n, ..., h] with elements.
bool activation(const Tensor& x) { return usual(x) && type_of(x) >= 0 && x.dim() >= 2 && x.numel() > 0 && x.size(0) <= 65535; }
// A parameter [h] or [n, h] with packed columns; undefined: not given.
bool parameter(const Tensor& w, const Tensor& x) {
    if (!w.defined()) return true;
    const auto keys = w.key_set();
    return w.is_cuda() && w.scalar_type() == at::kFloat && w.layout() == c10::kStrided && w.device() == x.device() &&
           (w.dim() == 1 || (w.dim() == 2 && w.size(0) == x.size(0))) && w.size(-1) == x.size(-1) && w.stride(-1) == 1 && !keys.has(c10::DispatchKey::Python) &&
           !keys.has(c10::DispatchKey::Negative) && !keys.has(c10::DispatchKey::FuncTorchBatched) &&
           !keys.has(c10::DispatchKey::FuncTorchGradWrapper);
}
const float* data(const Tensor& w) { return w.defined() ? static_cast<const float*>(w.const_data_ptr()) : nullptr; }
int64_t stride(const Tensor& w) { return w.defined() && w.dim() == 2 ? w.stride(0) : 0; }
void* out(const Tensor& t) { return t.defined() ? t.mutable_data_ptr() : nullptr; }

void* stream_of(const Tensor& t) { return c10::cuda::getCurrentCUDAStream(t.device().index()).stream(); }
Tensor bytes(const Tensor& like, size_t count) { return at::empty({(int64_t)count}, like.options().dtype(at::kByte).requires_grad(false)); }
Tensor floats(const Tensor& like, at::IntArrayRef shape) { return at::empty(shape, like.options().dtype(at::kFloat).requires_grad(false)); }
Tensor packed_like(const Tensor& t) { return at::empty(t.sizes(), t.options().requires_grad(false)); }

// A backward pass of gradients with forward-mode tangents would lose them.
void no_tangents(const variable_list& grads) {
    for (const Tensor& g : grads)
        if (g.defined() && g._fw_grad(0).defined()) throw LibraryError("forward-mode derivatives of a backward pass are not offered");
}
// The gradients of a backward pass, which is not differentiable itself: said where someone tries, as the Python functions do.
variable_list once(variable_list grads) {
    if (!at::GradMode::is_enabled()) return grads;
    bool any = false;
    for (auto& g : grads) {
        any = any || g.defined();
        if (g.defined()) g = g.detach().requires_grad_();
    }
    if (!any) return grads;
    const auto error = std::make_shared<torch::autograd::DelayedError>(
        "trying to differentiate twice a function that was marked with @once_differentiable", (int64_t)grads.size());
    return error->apply(std::move(grads));
}

// Saved tensors come as a hook unpacks them (torch.autograd.graph.saved_tensors_hooks): the same values, but perhaps not as they lay.
Tensor packed(const Tensor& t) { return t.defined() ? t.resolve_neg().contiguous() : t; }
Tensor packed_columns(const Tensor& t) { return t.defined() && (t.is_neg() || t.stride(-1) != 1) ? packed(t) : t; }

struct Shape {
    int32_t n;
    int64_t rows, h;
};
Shape shape_of(const Tensor& x) {
    const int64_t n = x.size(0), h = x.size(-1);
    return {(int32_t)n, x.numel() / (n * h), h};
}

// ---- root-mean-square norms ------------------------------------------------------------------------------------------------

void norm_forward(const Tensor& y, const Tensor& s, const Tensor& stats, const Tensor& x, const Tensor& residual, const Tensor& weight,
                  const Tensor& gate, const Tensor& next, double scale, double eps) {
    const Shape z = shape_of(x);
    const c10::DeviceGuard guard(x.device());
    check(entry.rms_norm_forward(out(y), out(s), (float*)out(stats), x.const_data_ptr(), residual.defined() ? residual.const_data_ptr() : nullptr,
                                 type_of(x), residual.defined() ? type_of(residual) : 0, z.n, z.rows, z.h, z.rows * z.h, z.h, z.rows * z.h, z.h,
                                 data(weight), stride(weight), data(gate), stride(gate), data(next), stride(next), scale, (float)eps, stream_of(x)),
          "compams_rms_norm_forward");
}
// [dx, dresidual, dweight, dgate, dnext], those that are wanted. dy and ds may be undefined, not both.
variable_list norm_backward(Tensor dy, Tensor ds, const Tensor& x, const Tensor& s, const Tensor& stats, const Tensor (&p)[3], const bool (&wanted)[5],
                            double scale) {
    const Shape z = shape_of(x);
    const c10::DeviceGuard guard(x.device());
    // (a packed tensor may be the negative of what lies in memory)
    dy = dy.defined() ? dy.resolve_neg().contiguous() : at::zeros(x.sizes(), x.options().requires_grad(false));
    if (ds.defined()) ds = ds.resolve_neg().contiguous();
    variable_list got(5);
    if (wanted[0]) got[0] = packed_like(x);
    if (wanted[1]) got[1] = packed_like(s);
    bool apart = false, sums = false;
    for (const Tensor& w : p) apart = apart || (w.defined() && w.dim() == 2);
    for (int k = 0; k < 3; ++k)
        if (wanted[2 + k]) {
            got[2 + k] = apart ? floats(x, {z.n, z.h}) : floats(x, {z.h});
            sums = true;
        }
    size_t need = 0;
    Tensor work;
    if (sums) {
        check(entry.rms_norm_workspace_bytes(&need, z.n, z.rows, z.h), "compams_rms_norm_workspace_bytes");
        work = bytes(x, need);
    }
    check(entry.rms_norm_backward(out(got[0]), out(got[1]), (float*)out(got[2]), (float*)out(got[3]), (float*)out(got[4]), apart ? 0 : 1,
                                  dy.const_data_ptr(), ds.defined() ? ds.const_data_ptr() : nullptr, x.const_data_ptr(),
                                  s.defined() ? s.const_data_ptr() : nullptr, (const float*)stats.const_data_ptr(), type_of(x),
                                  s.defined() ? type_of(s) : 0, z.n, z.rows, z.h, z.rows * z.h, z.h, z.rows * z.h, z.h, z.rows * z.h, z.h, data(p[0]),
                                  stride(p[0]), data(p[1]), stride(p[1]), data(p[2]), stride(p[2]), scale, out(work), need, stream_of(x)),
          "compams_rms_norm_backward");
    return got;
}

// A parameter as autograd takes one that may not be given; it numbers the edges of those that are.
using Given = std::optional<Tensor>;
Given given(const Tensor& w) { return w.defined() ? Given(w) : Given(); }
Tensor tensor(const Given& w) { return w ? *w : Tensor(); }

struct RmsNorm : torch::autograd::Function<RmsNorm> {
    static Tensor forward(AutogradContext* ctx, const Tensor& x, const Given& maybe, double eps) {
        const Tensor weight = tensor(maybe);
        const Shape z = shape_of(x);
        const Tensor y = packed_like(x), stats = floats(x, {z.n * z.rows, 2});
        norm_forward(y, {}, stats, x, {}, weight, {}, {}, 1.0, eps);
        ctx->save_for_backward({x, weight, stats});
        return y;
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        no_tangents(grads);
        const variable_list saved = ctx->get_saved_variables();
        const Tensor parameters[3] = {packed_columns(saved[1]), Tensor(), Tensor()};
        const bool wanted[5] = {ctx->needs_input_grad(0), false, saved[1].defined() && ctx->needs_input_grad(1), false, false};
        const variable_list got = norm_backward(grads[0], {}, packed(saved[0]), {}, packed(saved[2]), parameters, wanted, 1.0);
        return once({got[0], got[2], Tensor()});
    }
};

struct GatedNorm : torch::autograd::Function<GatedNorm> {
    static variable_list forward(AutogradContext* ctx, const Tensor& x, const Tensor& residual, const Given& maybe_weight, const Given& maybe_gate,
                                 const Given& maybe_next, double scale, double eps) {
        const Tensor weight = tensor(maybe_weight), gate = tensor(maybe_gate), next = tensor(maybe_next);
        const Shape z = shape_of(x);
        const Tensor y = packed_like(x), s = packed_like(residual), stats = floats(x, {z.n * z.rows, 2});
        norm_forward(y, s, stats, x, residual, weight, gate, next, scale, eps);
        ctx->set_materialize_grads(false);
        ctx->save_for_backward({x, s, stats, weight, gate, next});
        ctx->saved_data["scale"] = scale;
        return {y, s};
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        if (!grads[0].defined() && !grads[1].defined()) return variable_list(7);
        no_tangents(grads);
        const variable_list saved = ctx->get_saved_variables();
        const Tensor parameters[3] = {packed_columns(saved[3]), packed_columns(saved[4]), packed_columns(saved[5])};
        bool wanted[5] = {ctx->needs_input_grad(0), ctx->needs_input_grad(1), false, false, false};
        for (int k = 0, edge = 2; k < 3; ++k) wanted[2 + k] = parameters[k].defined() && ctx->needs_input_grad(edge++);
        const variable_list got = norm_backward(grads[0], grads[1], packed(saved[0]), packed(saved[1]), packed(saved[2]), parameters, wanted,
                                                ctx->saved_data["scale"].toDouble());
        return once({got[0], got[1], got[2], got[3], got[4], Tensor(), Tensor()});
    }
};

// ---- the head --------------------------------------------------------------------------------------------------------------

struct HeadCall {
    Shape z;
    int64_t vocab, weight_worker, weight_row;
    int x_copied, weight_copied;
};
bool multiple_of_16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
HeadCall head_call(const Tensor& x, const Tensor& weight) {
    HeadCall c = {shape_of(x), weight.size(-2), 0, weight.stride(-2), 1, 1};
    c.weight_worker = weight.dim() == 3 && c.z.n > 1 ? weight.stride(0) : 0;
    const int type = type_of(x), weight_type = type_of(weight);
    const bool whole = c.z.h % 8 == 0, rows = c.z.n * c.z.rows > 1;
    if (type == COMPAMS_BF16 || (type == COMPAMS_F16 && weight_type == COMPAMS_F16)) c.x_copied = !(multiple_of_16(x.const_data_ptr()) && (whole || !rows));
    if (type == weight_type && type != COMPAMS_F32)
        c.weight_copied = !(multiple_of_16(weight.const_data_ptr()) && (c.vocab == 1 || (c.weight_row % 8 == 0 && c.weight_row >= c.z.h)) &&
                            (c.weight_worker == 0 || c.weight_worker % 8 == 0));
    return c;
}
Tensor head_workspace(const HeadCall& c, const Tensor& x, const Tensor& weight, int wanted, size_t& need) {
    check(entry.head_workspace_bytes(&need, c.z.n, c.z.rows, c.z.h, c.vocab, type_of(x), type_of(weight), c.weight_worker == 0, c.x_copied,
                                     c.weight_copied, wanted),
          "compams_head_workspace_bytes");
    return bytes(x, need);
}
void head_forward(const Tensor& loss, const Tensor& lse, const Tensor& x, const Tensor& weight, const Tensor& target, int reduction, int64_t ignored) {
    const c10::DeviceGuard guard(x.device());
    const HeadCall c = head_call(x, weight);
    size_t need = 0;
    const Tensor work = head_workspace(c, x, weight, 0, need);
    check(entry.head_forward((float*)out(loss), (float*)out(lse), x.const_data_ptr(), type_of(x), weight.const_data_ptr(), type_of(weight),
                             (const int64_t*)target.const_data_ptr(), c.z.n, c.z.rows, c.z.h, c.vocab, c.z.rows * c.z.h, c.z.h, c.weight_worker,
                             c.weight_row, ignored, reduction, out(work), need, stream_of(x)),
          "compams_head_forward");
}
Tensor loss_for(const Tensor& x, const Tensor& target, int reduction) { return reduction ? floats(x, {x.size(0)}) : floats(x, target.sizes()); }

struct Head : torch::autograd::Function<Head> {
    static Tensor forward(AutogradContext* ctx, const Tensor& x, const Tensor& weight, const Tensor& target, int64_t reduction, int64_t ignored) {
        const Tensor loss = loss_for(x, target, (int)reduction), lse = floats(x, {target.numel() + x.size(0)});
        head_forward(loss, lse, x, weight, target, (int)reduction, ignored);
        ctx->save_for_backward({x, weight, target, lse});
        ctx->saved_data["reduction"] = reduction;
        ctx->saved_data["ignored"] = ignored;
        return loss;
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        no_tangents(grads);
        const variable_list saved = ctx->get_saved_variables();
        const Tensor x = packed(saved[0]), weight = packed_columns(saved[1]), target = packed(saved[2]), lse = packed(saved[3]);
        const c10::DeviceGuard guard(x.device());
        const int reduction = (int)ctx->saved_data["reduction"].toInt();
        const HeadCall c = head_call(x, weight);
        Tensor dx, dweight, g = grads[0].resolve_neg();
        if (!reduction) g = g.reshape({c.z.n, c.z.rows});
        if (ctx->needs_input_grad(0)) dx = packed_like(x);
        if (ctx->needs_input_grad(1)) dweight = at::empty(weight.sizes(), weight.options().requires_grad(false));
        if (dx.defined() || dweight.defined()) {
            size_t need = 0;
            const Tensor work = head_workspace(c, x, weight, (dx.defined() ? 1 : 0) | (dweight.defined() ? 2 : 0), need);
            check(entry.head_backward(out(dx), out(dweight), weight.dim() == 2 ? 1 : 0, (const float*)g.const_data_ptr(), g.stride(0),
                                      reduction ? 0 : g.stride(1), x.const_data_ptr(), type_of(x), weight.const_data_ptr(), type_of(weight),
                                      (const int64_t*)target.const_data_ptr(), (const float*)lse.const_data_ptr(), c.z.n, c.z.rows, c.z.h,
                                      c.vocab, c.z.rows * c.z.h, c.z.h, c.weight_worker, c.weight_row, ctx->saved_data["ignored"].toInt(), reduction,
                                      out(work), need, stream_of(x)),
                  "compams_head_backward");
        }
        return once({dx, dweight, Tensor(), Tensor(), Tensor()});
    }
};

// ---- Python ----------------------------------------------------------------------------------------------------------------

#define NOT_USUAL Py_RETURN_NONE
#define BEGIN_CALL HANDLE_TH_ERRORS try {
#define END_CALL                                      \
    }                                                 \
    catch (const LibraryError& e) {                   \
        PyErr_SetString(library_error, e.what());     \
        return nullptr;                               \
    }                                                 \
    END_HANDLE_TH_ERRORS

bool tensor_of(PyObject* o, Tensor& t) {  // None: undefined
    if (o == Py_None) return true;
    if (!THPVariable_Check(o)) return false;
    t = THPVariable_Unpack(o);
    return true;
}
bool wants(std::initializer_list<const Tensor*> tensors) {
    if (!at::GradMode::is_enabled()) return false;
    for (const Tensor* t : tensors)
        if (t->defined() && t->requires_grad()) return true;
    return false;
}
bool number_of(PyObject* o, double& v) {
    if (!PyFloat_CheckExact(o)) return false;
    v = PyFloat_AS_DOUBLE(o);
    return true;
}

PyObject* rms_norm(PyObject*, PyObject* const* args, Py_ssize_t count) {
    BEGIN_CALL
    Tensor x, weight;
    double eps;
    if (count != 3 || !tensor_of(args[0], x) || !x.defined() || !tensor_of(args[1], weight) || !number_of(args[2], eps) || !(eps >= 0.0) || !alone() ||
        !activation(x) || !parameter(weight, x))
        NOT_USUAL;
    if (wants({&x, &weight})) return THPVariable_Wrap(RmsNorm::apply(x, given(weight), eps));
    const Tensor y = packed_like(x);
    norm_forward(y, {}, {}, x, {}, weight, {}, {}, 1.0, eps);
    return THPVariable_Wrap(y);
    END_CALL
}

PyObject* pair(const Tensor& a, const Tensor& b) {
    PyObject *first = THPVariable_Wrap(a), *second = THPVariable_Wrap(b), *both = PyTuple_Pack(2, first, second);
    Py_DECREF(first);
    Py_DECREF(second);
    return both;
}

PyObject* gated_add_rms_norm(PyObject*, PyObject* const* args, Py_ssize_t count) {
    BEGIN_CALL
    Tensor x, residual, weight, gate, next;
    double scale, eps;
    if (count != 7 || !tensor_of(args[0], x) || !x.defined() || !tensor_of(args[1], residual) || !residual.defined() || !tensor_of(args[2], weight) ||
        !tensor_of(args[3], gate) || !tensor_of(args[4], next) || !number_of(args[5], scale) || !number_of(args[6], eps) || !(eps >= 0.0) || !alone() ||
        !activation(x) || !usual(residual) || residual.device() != x.device() || residual.sizes() != x.sizes() ||
        (residual.scalar_type() != x.scalar_type() && residual.scalar_type() != at::kFloat) || !parameter(weight, x) || !parameter(gate, x) ||
        !parameter(next, x))
        NOT_USUAL;
    int64_t dims = 0;
    for (const Tensor* w : {&weight, &gate, &next})
        if (w->defined()) {
            if (dims && w->dim() != dims) NOT_USUAL;
            dims = w->dim();
        }
    if (wants({&x, &residual, &weight, &gate, &next})) {
        const variable_list got = GatedNorm::apply(x, residual, given(weight), given(gate), given(next), scale, eps);
        return pair(got[0], got[1]);
    }
    const Tensor y = packed_like(x), s = packed_like(residual);
    norm_forward(y, s, {}, x, residual, weight, gate, next, scale, eps);
    return pair(y, s);
    END_CALL
}

PyObject* linear_cross_entropy(PyObject*, PyObject* const* args, Py_ssize_t count) {
    BEGIN_CALL
    Tensor x, weight, target;
    if (count != 5 || !tensor_of(args[0], x) || !x.defined() || !tensor_of(args[1], weight) || !weight.defined() || !tensor_of(args[2], target) ||
        !target.defined() || !PyLong_CheckExact(args[3]) || !PyLong_CheckExact(args[4]) || !alone() || !activation(x))
        NOT_USUAL;
    const long reduction = PyLong_AsLong(args[3]);
    int overflow = 0;
    const long long ignored = PyLong_AsLongLongAndOverflow(args[4], &overflow);
    const auto keys = weight.key_set();
    if (reduction < 0 || reduction > 2 || overflow || !weight.is_cuda() || weight.layout() != c10::kStrided || weight.device() != x.device() ||
        (weight.scalar_type() != x.scalar_type() && weight.scalar_type() != at::kFloat) || (weight.dim() != 2 && weight.dim() != 3) ||
        weight.size(-1) != x.size(-1) || weight.size(-2) < 1 || (weight.dim() == 3 && weight.size(0) != x.size(0)) || weight.stride(-1) != 1 ||
        keys.has(c10::DispatchKey::Python) || keys.has(c10::DispatchKey::Negative) || keys.has(c10::DispatchKey::FuncTorchBatched) ||
        keys.has(c10::DispatchKey::FuncTorchGradWrapper) || !usual(target) || target.scalar_type() != at::kLong || target.device() != x.device() ||
        target.dim() != x.dim() - 1 || target.sizes() != x.sizes().slice(0, x.dim() - 1))
        NOT_USUAL;
    if (wants({&x, &weight})) return THPVariable_Wrap(Head::apply(x, weight, target, (int64_t)reduction, (int64_t)ignored));
    const Tensor loss = loss_for(x, target, (int)reduction), lse = floats(x, {target.numel() + x.size(0)});
    head_forward(loss, lse, x, weight, target, (int)reduction, ignored);
    return THPVariable_Wrap(loss);
    END_CALL
}

// (list of gradients, out or None, max_norm, eps)
PyObject* collect_gradients(PyObject*, PyObject* const* args, Py_ssize_t count) {
    BEGIN_CALL
    Tensor G;
    double max_norm, eps;
    if (count != 4 || !PyList_CheckExact(args[0]) || !PyList_GET_SIZE(args[0]) || !tensor_of(args[1], G) || !number_of(args[2], max_norm) ||
        !number_of(args[3], eps) || !(max_norm >= 0.0) || !(eps >= 0.0) || !alone())
        NOT_USUAL;
    const Py_ssize_t many = PyList_GET_SIZE(args[0]);
    std::vector<const void*> addresses(many);
    std::vector<int64_t> sizes(many), ends(many + 1);
    std::vector<int32_t> types(many);
    int64_t n = 0;
    c10::Device device(c10::kCPU);
    for (Py_ssize_t k = 0; k < many; ++k) {
        PyObject* o = PyList_GET_ITEM(args[0], k);
        if (!THPVariable_Check(o)) NOT_USUAL;
        const Tensor& g = THPVariable_Unpack(o);
        types[k] = type_of(g);
        if (!usual(g) || types[k] < 0 || g.dim() < 1 || g.numel() < 1) NOT_USUAL;
        if (k == 0) {
            n = g.size(0);
            device = g.device();
        }
        if (g.size(0) != n || n > 65535 || g.device() != device) NOT_USUAL;
        addresses[k] = g.const_data_ptr();
        sizes[k] = g.numel() / n;
        ends[k + 1] = ends[k] + sizes[k];
    }
    const auto options = at::TensorOptions().dtype(at::kFloat).device(device);
    if (G.defined()) {
        if (!usual(G) || G.scalar_type() != at::kFloat || G.device() != device || G.dim() != 2 || G.size(0) != n || G.size(1) != ends[many] || G.requires_grad())
            NOT_USUAL;
        const char* lo = (const char*)G.const_data_ptr();
        for (Py_ssize_t k = 0; k < many; ++k) {
            const char* g = (const char*)addresses[k];
            if (g < lo + G.nbytes() && lo < g + n * sizes[k] * (types[k] == 0 ? 4 : 2)) NOT_USUAL;  // a gradient that lies in G: refused there
        }
        if (!G.is_inference()) G.unsafeGetTensorImpl()->bump_version();
    } else {
        G = at::empty({n, ends[many]}, options);
    }
    const c10::DeviceGuard guard(device);
    const Tensor norms = at::empty({n}, options);
    size_t need = 0;
    check(entry.collect_workers_workspace_bytes(&need, (int32_t)n, (int32_t)many), "compams_collect_workers_workspace_bytes");
    const Tensor work = bytes(G, need);
    check(entry.collect_workers((float*)out(G), ends[many], (float*)out(norms), addresses.data(), sizes.data(), types.data(), ends.data(), (int32_t)many,
                                (int32_t)n, max_norm, eps, out(work), need, stream_of(G)),
          "compams_collect_workers");
    return pair(G, norms);
    END_CALL
}

// bind(addresses in the order of Entries, the error's class)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t count) {
    static_assert(sizeof(Entries) == 10 * sizeof(void*), "the order of the addresses");
    if (count != 11) {
        PyErr_SetString(PyExc_TypeError, "ten addresses and an error");
        return nullptr;
    }
    void* addresses[10];
    for (int k = 0; k < 10; ++k) {
        addresses[k] = PyLong_AsVoidPtr(args[k]);
        if (!addresses[k]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an address is null");
            return nullptr;
        }
    }
    memcpy(&entry, addresses, sizeof(entry));
    Py_INCREF(args[10]);
    Py_XDECREF(library_error);
    library_error = args[10];
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"bind", (PyCFunction)(void*)bind, METH_FASTCALL, nullptr},
                         {"rms_norm", (PyCFunction)(void*)rms_norm, METH_FASTCALL, nullptr},
                         {"gated_add_rms_norm", (PyCFunction)(void*)gated_add_rms_norm, METH_FASTCALL, nullptr},
                         {"linear_cross_entropy", (PyCFunction)(void*)linear_cross_entropy, METH_FASTCALL, nullptr},
                         {"collect_gradients", (PyCFunction)(void*)collect_gradients, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_ops", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_ops(void) { return PyModule_Create(&module); }
