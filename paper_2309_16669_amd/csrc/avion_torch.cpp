// The autograd front end's calls as native functions: what paper_2309_16669_amd/autograd.py does in
// Python for every call -- checks, allocations, one entry point of the C ABI, the autograd node -- without
// the interpreter.  A forward and backward pass of layer_norm spent 140 us there (the kernels take 86), a
// caption's forward 18 us (kernel 6); the node's backward also no longer takes the interpreter lock on
// autograd's thread.  Nothing is computed here.
//
// Each function takes plain calls only (see `plain`): exact torch tensors on the GPU in the expected
// formats and shapes, with no transform, mode, tracer or tangent in force.  For anything else it returns
// None, and the caller goes through the Python classes, which raise or behave as they always did.  Errors
// of the library are raised as the binding's AvionError.
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>
#include <torch/csrc/utils/pybind.h>
#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>

#include "avion_attn.h"

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

// AvionError of the binding, also from autograd's own threads
void check(int rc)
{
    if (rc == AVION_OK) return;
    pybind11::gil_scoped_acquire gil;
    try {
        pybind11::module_::import("paper_2309_16669_amd").attr("_check")(rc);
    } catch (pybind11::error_already_set& e) {
        e.restore();
    }
    python_error err;
    err.persist();
    throw err;
}

unsigned format_flag(const Tensor& t) { return t.scalar_type() == at::kHalf ? AVION_FLAG_F16 : 0u; }
bool element_format(const Tensor& t) { return t.scalar_type() == at::kHalf || t.scalar_type() == at::kBFloat16; }

// nothing that would have to see or replace the tensors' operations is in force on this thread
bool plain_thread()
{
    return !c10::impl::TorchDispatchModeTLS::any_modes_set() && !at::impl::torch_function_mode_enabled() &&
           !torch::jit::tracer::isTracing() &&
           !c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::FuncTorchDynamicLayerFrontMode);
}

// an exact torch.Tensor or Parameter with data on the GPU, without a tangent
bool plain(PyObject* obj, const Tensor** out)
{
    if (!THPVariable_CheckExact(obj)) return false;
    const Tensor& t = THPVariable_Unpack(obj);
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || t.is_conj() || t.is_neg() || t.numel() == 0 ||
        t._fw_grad(0).defined())
        return false;
    *out = &t;
    return true;
}
bool parameter(PyObject* obj, int64_t width, const Tensor& like, const Tensor** out)
{
    return plain(obj, out) && (*out)->scalar_type() == at::kFloat && (*out)->dim() == 1 && (*out)->size(0) == width &&
           (*out)->device() == like.device();
}

// The binding's checks (`_require`) before an address is taken.  A saved tensor is whatever the unpack hook of
// torch.autograd.graph.saved_tensors_hooks returned: other strides, another format, on the host, shorter.  The
// incoming gradient has the shape, format and device of the forward's output (autograd checks that).
void require(const Tensor& t, const char* name, at::IntArrayRef shape, at::ScalarType dtype, const Tensor& grad)
{
    TORCH_CHECK_VALUE(t.defined() && t.layout() == at::kStrided && t.is_cuda() && t.device() == grad.device(), name,
                      " must live on the GPU of the gradient");
    TORCH_CHECK_VALUE(t.scalar_type() == dtype, name, " must be ", dtype, ", got ", t.scalar_type());
    TORCH_CHECK_VALUE(t.is_contiguous(), name, " must be contiguous");
    TORCH_CHECK_VALUE(t.sizes() == shape, name, " must have shape ", shape, ", got ", t.sizes());
}

// Runs a call without the interpreter lock, as torch's own functions and ctypes do: an allocation that goes to the
// driver or a launch that waits for room in the queue stops this thread only.  The caller's frame holds the arguments.
template <typename F>
pybind11::object without_lock(F call)
{
    Tensor out;
    {
        pybind11::gil_scoped_release release;
        out = call();
    }
    return pybind11::cast(out);
}

// whether a node has to be recorded; without one a call is its allocations and its launch (a caption's forward
// 7.5 -> 6.7 us, of which the kernel runs 5.5)
bool records(std::initializer_list<const Tensor*> inputs)
{
    if (!at::GradMode::is_enabled()) return false;
    for (const Tensor* t : inputs)
        if (t->requires_grad()) return true;
    return false;
}

Tensor workspace(size_t bytes, const Tensor& like) { return at::empty({(int64_t)bytes}, like.options().dtype(at::kByte)); }

// ------------------------------------------------------------------------------------- attention
struct Shape {
    int B, H, N, d;
};
Shape shape_of(const Tensor& q, bool packed)
{
    return {(int)q.size(0), (int)q.size(packed ? 3 : 2), (int)q.size(1), (int)q.size(packed ? 4 : 3)};
}
bool fits_int(const Tensor& t)
{
    for (int64_t s : t.sizes())
        if (s > INT32_MAX) return false;
    return true;
}

// o and lse of one forward; k and v are undefined for a packed q
void attention_fwd(const Tensor& q, const Tensor& k, const Tensor& v, Tensor& o, Tensor& lse, double scale, bool causal)
{
    const bool packed = !k.defined();
    const Shape s = shape_of(q, packed);
    o = at::empty({s.B, s.N, s.H, s.d}, q.options());
    lse = at::empty({s.B, s.H, s.N}, q.options().dtype(at::kFloat));
    const unsigned flags = format_flag(q) | (causal ? AVION_FLAG_CAUSAL : 0u) | (packed ? AVION_FLAG_QKVPACKED : 0u);
    check(avion_attn_fwd_ex(q.data_ptr(), packed ? nullptr : k.data_ptr(), packed ? nullptr : v.data_ptr(), o.data_ptr(),
                            lse.data_ptr<float>(), s.B, s.H, s.N, s.d, (float)scale, flags, stream()));
}
// gradients of q, k, v (of q alone when it is packed)
variable_list attention_bwd(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& o, const Tensor& lse,
                            const Tensor& grad, double scale, bool causal)
{
    const bool packed = !k.defined();
    const Tensor dO = grad.contiguous();
    const Shape s = shape_of(dO, false);
    const at::ScalarType dt = dO.scalar_type();
    if (packed) {
        require(q, "qkv", {s.B, s.N, 3, s.H, s.d}, dt, dO);
    } else {
        require(q, "q", dO.sizes(), dt, dO);
        require(k, "k", dO.sizes(), dt, dO);
        require(v, "v", dO.sizes(), dt, dO);
    }
    require(o, "o", dO.sizes(), dt, dO);
    require(lse, "lse", {s.B, s.H, s.N}, at::kFloat, dO);
    variable_list g{at::empty_like(q)};
    if (!packed) {
        g.push_back(at::empty_like(k));
        g.push_back(at::empty_like(v));
    }
    const size_t need = avion_attn_bwd_workspace_bytes(s.B, s.H, s.N, s.d);
    const Tensor ws = workspace(need, q);
    const unsigned flags = format_flag(q) | (causal ? AVION_FLAG_CAUSAL : 0u) | (packed ? AVION_FLAG_QKVPACKED : 0u);
    check(avion_attn_bwd_ex(q.data_ptr(), packed ? nullptr : k.data_ptr(), packed ? nullptr : v.data_ptr(), o.data_ptr(),
                            lse.data_ptr<float>(), dO.data_ptr(), g[0].data_ptr(), packed ? nullptr : g[1].data_ptr(),
                            packed ? nullptr : g[2].data_ptr(), s.B, s.H, s.N, s.d, (float)scale, flags, ws.data_ptr(), need,
                            stream()));
    return g;
}

struct Attention : torch::autograd::Function<Attention> {
    static Tensor forward(AutogradContext* ctx, const Tensor& q_, const Tensor& k_, const Tensor& v_, double scale, bool causal)
    {
        const Tensor q = q_.contiguous(), k = k_.contiguous(), v = v_.contiguous();
        Tensor o, lse;
        attention_fwd(q, k, v, o, lse, scale, causal);
        ctx->save_for_backward({q, k, v, o, lse});
        ctx->saved_data["scale"] = scale;
        ctx->saved_data["causal"] = causal;
        return o;
    }
    static variable_list backward(AutogradContext* ctx, variable_list grad)
    {
        const variable_list s = ctx->get_saved_variables();
        variable_list g = attention_bwd(s[0], s[1], s[2], s[3], s[4], grad[0], ctx->saved_data["scale"].toDouble(),
                                        ctx->saved_data["causal"].toBool());
        g.resize(5);
        return g;
    }
};
struct AttentionPacked : torch::autograd::Function<AttentionPacked> {
    static Tensor forward(AutogradContext* ctx, const Tensor& qkv_, double scale, bool causal)
    {
        const Tensor qkv = qkv_.contiguous();
        Tensor o, lse;
        attention_fwd(qkv, Tensor(), Tensor(), o, lse, scale, causal);
        ctx->save_for_backward({qkv, o, lse});
        ctx->saved_data["scale"] = scale;
        ctx->saved_data["causal"] = causal;
        return o;
    }
    static variable_list backward(AutogradContext* ctx, variable_list grad)
    {
        const variable_list s = ctx->get_saved_variables();
        variable_list g = attention_bwd(s[0], Tensor(), Tensor(), s[1], s[2], grad[0], ctx->saved_data["scale"].toDouble(),
                                        ctx->saved_data["causal"].toBool());
        g.resize(3);
        return g;
    }
};

pybind11::object attention(pybind11::handle q_, pybind11::handle k_, pybind11::handle v_, double scale, bool causal)
{
    HANDLE_TH_ERRORS
    const Tensor *q, *k, *v;
    if (!plain(q_.ptr(), &q) || !plain(k_.ptr(), &k) || !plain(v_.ptr(), &v) || !plain_thread()) return pybind11::none();
    if (q->dim() != 4 || !element_format(*q) || !fits_int(*q)) return pybind11::none();
    for (const Tensor* t : {k, v})
        if (t->scalar_type() != q->scalar_type() || t->sizes() != q->sizes() || t->device() != q->device()) return pybind11::none();
    return without_lock([&] {
        if (records({q, k, v})) return Attention::apply(*q, *k, *v, scale, causal);
        Tensor o, lse;
        attention_fwd(q->contiguous(), k->contiguous(), v->contiguous(), o, lse, scale, causal);
        return o;
    });
    END_HANDLE_TH_ERRORS_PYBIND
}
pybind11::object attention_qkvpacked(pybind11::handle qkv_, double scale, bool causal)
{
    HANDLE_TH_ERRORS
    const Tensor* qkv;
    if (!plain(qkv_.ptr(), &qkv) || !plain_thread()) return pybind11::none();
    if (qkv->dim() != 5 || qkv->size(2) != 3 || !element_format(*qkv) || !fits_int(*qkv)) return pybind11::none();
    return without_lock([&] {
        if (records({qkv})) return AttentionPacked::apply(*qkv, scale, causal);
        Tensor o, lse;
        attention_fwd(qkv->contiguous(), Tensor(), Tensor(), o, lse, scale, causal);
        return o;
    });
    END_HANDLE_TH_ERRORS_PYBIND
}

// -------------------------------------------------------------------------- layer normalisation
struct LayerNorm : torch::autograd::Function<LayerNorm> {
    static Tensor forward(AutogradContext* ctx, const Tensor& x_, const Tensor& gamma, const Tensor& beta, double eps)
    {
        const int64_t D = x_.size(-1);
        const Tensor x = x_.contiguous().view({-1, D});
        const int64_t M = x.size(0);
        const Tensor y = at::empty(x_.sizes(), x.options());
        const Tensor mean = at::empty({M}, gamma.options()), rstd = at::empty({M}, gamma.options());
        check(avion_layernorm_fwd(x.data_ptr(), gamma.contiguous().data_ptr<float>(), beta.contiguous().data_ptr<float>(),
                                  y.data_ptr(), mean.data_ptr<float>(), rstd.data_ptr<float>(), M, (int)D, (float)eps,
                                  format_flag(x), stream()));
        ctx->save_for_backward({x, gamma, mean, rstd});  // the input and two floats per token; not y
        ctx->saved_data["shape"] = x_.sizes().vec();
        return y;
    }
    static variable_list backward(AutogradContext* ctx, variable_list grad)
    {
        const variable_list s = ctx->get_saved_variables();
        const Tensor &x = s[0], gamma = s[1].contiguous(), dy = grad[0].contiguous();
        const int64_t D = dy.size(-1), M = dy.numel() / D;
        require(x, "x", {M, D}, dy.scalar_type(), dy);
        require(gamma, "gamma", {D}, at::kFloat, dy);
        require(s[2], "mean", {M}, at::kFloat, dy);
        require(s[3], "rstd", {M}, at::kFloat, dy);
        const Tensor dx = at::empty_like(x), dgamma = at::empty_like(gamma), dbeta = at::empty_like(gamma);
        const size_t need = avion_layernorm_bwd_workspace_bytes(M, (int)D);
        const Tensor ws = workspace(need, x);
        check(avion_layernorm_bwd(x.data_ptr(), gamma.data_ptr<float>(), s[2].data_ptr<float>(), s[3].data_ptr<float>(),
                                  dy.data_ptr(), dx.data_ptr(), dgamma.data_ptr<float>(), dbeta.data_ptr<float>(), M, (int)D,
                                  format_flag(x), ws.data_ptr(), need, stream()));
        return {dx.view(ctx->saved_data["shape"].toIntVector()), dgamma, dbeta, Tensor()};
    }
};
pybind11::object layer_norm(pybind11::handle x_, pybind11::handle gamma_, pybind11::handle beta_, double eps)
{
    HANDLE_TH_ERRORS
    const Tensor *x, *gamma, *beta;
    if (!plain(x_.ptr(), &x) || !plain_thread()) return pybind11::none();
    if (x->dim() < 1 || !element_format(*x) || x->size(-1) > INT32_MAX) return pybind11::none();
    if (!parameter(gamma_.ptr(), x->size(-1), *x, &gamma) || !parameter(beta_.ptr(), x->size(-1), *x, &beta))
        return pybind11::none();
    return without_lock([&] { return LayerNorm::apply(*x, *gamma, *beta, eps); });
    END_HANDLE_TH_ERRORS_PYBIND
}

// ---------------------------------------------------------------------------------- bias + GELU
Tensor gelu_fwd(const Tensor& x, const Tensor& bias, at::IntArrayRef shape)
{
    const Tensor y = at::empty(shape, x.options());
    check(avion_bias_gelu_fwd(x.data_ptr(), bias.contiguous().data_ptr<float>(), y.data_ptr(), x.size(0), (int)x.size(1),
                              format_flag(x), stream()));
    return y;
}
void gelu_bwd(const Tensor& x, const Tensor& bias_, const Tensor& dy, Tensor& dx, Tensor& dbias)
{
    const Tensor bias = bias_.contiguous();
    dx = at::empty_like(x);
    dbias = at::empty_like(bias);
    const size_t need = avion_bias_gelu_bwd_workspace_bytes(x.size(0), (int)x.size(1));
    const Tensor ws = workspace(need, x);
    check(avion_bias_gelu_bwd(x.data_ptr(), bias.data_ptr<float>(), dy.data_ptr(), dx.data_ptr(), dbias.data_ptr<float>(),
                              x.size(0), (int)x.size(1), format_flag(x), ws.data_ptr(), need, stream()));
}

// d.sum(0); torch's where the rows are no multiple of 16 bytes, and where the sum is to be differentiated itself
// (create_graph, a tangent): it is linear in d
Tensor column_sum(const Tensor& d)
{
    const int64_t M = d.size(0), F = d.size(1);
    const size_t need = F <= INT32_MAX ? avion_column_sum_workspace_bytes(M, (int)F) : 0;
    if (need == 0 || !element_format(d) || reinterpret_cast<uintptr_t>(d.data_ptr()) % 16 != 0 || records({&d}) ||
        d._fw_grad(0).defined())
        return d.sum(0);
    const Tensor sum = at::empty({F}, d.options());
    check(avion_column_sum(d.data_ptr(), sum.data_ptr(), M, (int)F, format_flag(d), workspace(need, d).data_ptr(), need, stream()));
    return sum;
}

struct BiasGelu : torch::autograd::Function<BiasGelu> {
    static Tensor forward(AutogradContext* ctx, const Tensor& x_, const Tensor& bias)
    {
        const Tensor x = x_.contiguous().view({-1, x_.size(-1)});
        const Tensor y = gelu_fwd(x, bias, x_.sizes());
        ctx->save_for_backward({x, bias});  // the pre-activation only; the derivative is rebuilt from it
        ctx->saved_data["shape"] = x_.sizes().vec();
        return y;
    }
    static variable_list backward(AutogradContext* ctx, variable_list grad)
    {
        const variable_list s = ctx->get_saved_variables();
        const Tensor dy = grad[0].contiguous();
        const int64_t F = dy.size(-1);
        require(s[0], "x", {dy.numel() / F, F}, dy.scalar_type(), dy);
        require(s[1].contiguous(), "bias", {F}, at::kFloat, dy);
        Tensor dx, dbias;
        gelu_bwd(s[0], s[1], dy, dx, dbias);
        return {dx.view(ctx->saved_data["shape"].toIntVector()), dbias};
    }
};
// linear(GELU(x + bias), weight, out_bias) that keeps x only: the activation's output is rebuilt by the
// backward pass, beside dx, for the weight gradient.  The matrix products are torch's.
struct BiasGeluLinear : torch::autograd::Function<BiasGeluLinear> {
    static Tensor forward(AutogradContext* ctx, const Tensor& x_, const Tensor& bias, const Tensor& weight,
                          const std::optional<Tensor>& out_bias)
    {
        const Tensor x = x_.contiguous().view({-1, x_.size(-1)});
        const Tensor y = gelu_fwd(x, bias, x.sizes());
        const Tensor out = out_bias ? at::addmm(*out_bias, y, weight.t()) : at::matmul(y, weight.t());
        ctx->save_for_backward({x, bias, weight});
        ctx->saved_data["shape"] = x_.sizes().vec();
        ctx->saved_data["format"] = x.scalar_type();
        ctx->saved_data["has_out_bias"] = out_bias.has_value();
        std::vector<int64_t> shape = x_.sizes().vec();
        shape.back() = weight.size(0);
        return out.view(shape);
    }
    static variable_list backward(AutogradContext* ctx, variable_list grad)
    {
        const variable_list s = ctx->get_saved_variables();
        const Tensor &x = s[0], &bias = s[1], &weight = s[2];
        const std::vector<int64_t> shape = ctx->saved_data["shape"].toIntVector();
        const int64_t F = shape.back(), M = grad[0].numel() / grad[0].size(-1);
        require(x, "x", {M, F}, ctx->saved_data["format"].toScalarType(), grad[0]);
        require(bias.contiguous(), "bias", {F}, at::kFloat, grad[0]);
        const Tensor d2 = grad[0].contiguous().view({M, weight.size(0)});
        // variable_data: the product's storage without its node (create_graph) or tangent, which are not those of the
        // gradient of x that the kernel writes into it
        const Tensor dy = at::matmul(d2, weight).variable_data();
        require(dy, "dy", {M, F}, x.scalar_type(), grad[0]);  // under autocast a product comes in autocast's format
        // the gradient of x takes dy's place; y is rebuilt beside it, not kept
        const Tensor b = bias.contiguous(), y = at::empty_like(x), dbias = at::empty_like(b);
        const size_t need = avion_bias_gelu_bwd_workspace_bytes(M, (int)F);
        check(avion_bias_gelu_bwd_y(x.data_ptr(), b.data_ptr<float>(), dy.data_ptr(), dy.data_ptr(), y.data_ptr(),
                                    dbias.data_ptr<float>(), M, (int)F, format_flag(x), workspace(need, x).data_ptr(), need, stream()));
        return {dy.view(shape), dbias, at::matmul(d2.t(), y),
                ctx->saved_data["has_out_bias"].toBool() ? column_sum(d2) : Tensor()};
    }
};
bool gelu_args(pybind11::handle x_, pybind11::handle bias_, const Tensor** x, const Tensor** bias)
{
    return plain(x_.ptr(), x) && plain_thread() && (*x)->dim() >= 1 && element_format(**x) && (*x)->size(-1) <= INT32_MAX &&
           parameter(bias_.ptr(), (*x)->size(-1), **x, bias);
}
pybind11::object bias_gelu(pybind11::handle x_, pybind11::handle bias_)
{
    HANDLE_TH_ERRORS
    const Tensor *x, *bias;
    if (!gelu_args(x_, bias_, &x, &bias)) return pybind11::none();
    return without_lock([&] { return BiasGelu::apply(*x, *bias); });
    END_HANDLE_TH_ERRORS_PYBIND
}
pybind11::object bias_gelu_linear(pybind11::handle x_, pybind11::handle bias_, pybind11::handle weight_, pybind11::handle out_)
{
    HANDLE_TH_ERRORS
    const Tensor *x, *bias, *weight, *out = nullptr;
    if (!gelu_args(x_, bias_, &x, &bias) || !plain(weight_.ptr(), &weight)) return pybind11::none();
    if (weight->dim() != 2 || weight->size(1) != x->size(-1) || weight->scalar_type() != x->scalar_type() ||
        weight->device() != x->device())
        return pybind11::none();
    if (!out_.is_none()) {
        if (!plain(out_.ptr(), &out) || out->dim() != 1 || out->size(0) != weight->size(0) ||
            out->scalar_type() != x->scalar_type() || out->device() != x->device())
            return pybind11::none();
    }
    return without_lock([&] { return BiasGeluLinear::apply(*x, *bias, *weight, out ? std::optional<Tensor>(*out) : std::nullopt); });
    END_HANDLE_TH_ERRORS_PYBIND
}

// --------------------------------------------------------- token table, RMS normalisation, 8-bit path
// These run on the device of their tensors, whatever the current one is.
unsigned wide_flag(const Tensor& t) { return t.scalar_type() == at::kFloat ? AVION_FLAG_WIDE_F32 : 0u; }
void* data_of(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
// Contiguous and at a multiple of 16 bytes, as the C entries ask: a piece of a larger tensor (a gradient that comes out of a
// concatenation) may begin at any element, and its place is not the caller's to choose.
Tensor dense(const Tensor& t)
{
    const Tensor c = t.contiguous();
    return reinterpret_cast<uintptr_t>(c.data_ptr()) % 16 == 0 ? c : c.clone();
}

// As without_lock, for a call with several outputs
template <typename F>
pybind11::object many_without_lock(F call)
{
    variable_list out;
    {
        pybind11::gil_scoped_release release;
        out = call();
    }
    pybind11::tuple t(out.size());
    for (size_t i = 0; i < out.size(); ++i) t[i] = pybind11::cast(out[i]);
    return std::move(t);
}

// The node of a gradient that a kernel has written: it leads to the tensors that the gradient depends on, and says that the way
// back through it does not exist.  Without it a second derivative would silently miss this operator's part.
struct NoSecondDerivative : torch::autograd::Node {
    const char* what;
    explicit NoSecondDerivative(const char* operation) : what(operation) {}
    variable_list apply(variable_list&&) override { TORCH_CHECK(false, what, " has no second derivative"); }
};
// where the backward itself is recorded (create_graph)
void depends_on(const Tensor& gradient, const char* what, std::initializer_list<Tensor> inputs)
{
    if (!gradient.defined() || !at::GradMode::is_enabled()) return;
    std::shared_ptr<NoSecondDerivative> node;
    for (const Tensor& t : inputs) {
        if (!t.defined() || !t.requires_grad()) continue;
        if (!node) node = std::shared_ptr<NoSecondDerivative>(new NoSecondDerivative(what), torch::autograd::deleteNode);
        node->add_next_edge(torch::autograd::impl::gradient_edge(t));
    }
    if (node) torch::autograd::set_history(gradient, node);
}

unsigned embedding_flags(const Tensor& tokens, const Tensor& table, at::ScalarType out)
{
    return (out == at::kHalf ? AVION_FLAG_F16 : 0u) | wide_flag(table) | (tokens.scalar_type() == at::kInt ? AVION_FLAG_TOKENS_I32 : 0u);
}
Tensor embedding_fwd(const Tensor& tokens, const Tensor& weight_, double scale, at::ScalarType out)
{
    const Tensor t = tokens.contiguous(), weight = dense(weight_);
    std::vector<int64_t> shape = tokens.sizes().vec();
    shape.push_back(weight.size(1));
    const Tensor y = at::empty(shape, weight.options().dtype(out));
    check(avion_embedding_fwd(t.data_ptr(), weight.data_ptr(), y.data_ptr(), t.numel(), weight.size(0), (int)weight.size(1), (float)scale,
                              embedding_flags(t, weight, out), stream()));
    return y;
}
struct Embedding : torch::autograd::Function<Embedding> {
    static Tensor forward(AutogradContext* ctx, const Tensor& weight, const Tensor& tokens, double scale, bool f16)
    {
        const c10::DeviceGuard guard(weight.device());
        ctx->save_for_backward({tokens});
        ctx->saved_data["scale"] = scale;
        ctx->saved_data["shape"] = weight.sizes().vec();
        ctx->saved_data["format"] = weight.scalar_type();
        ctx->saved_data["tokens"] = tokens.scalar_type();
        return embedding_fwd(tokens, weight, scale, f16 ? at::kHalf : at::kBFloat16);
    }
    static variable_list backward(AutogradContext* ctx, variable_list grad)
    {
        const c10::DeviceGuard guard(grad[0].device());
        const Tensor dy = dense(grad[0]), tokens = ctx->get_saved_variables()[0].contiguous();
        const std::vector<int64_t> shape = ctx->saved_data["shape"].toIntVector();
        const int64_t V = shape[0], D = shape[1], n = dy.numel() / D;
        require(tokens, "tokens", dy.sizes().slice(0, dy.dim() - 1), ctx->saved_data["tokens"].toScalarType(), dy);
        const Tensor dweight = at::empty(shape, dy.options().dtype(ctx->saved_data["format"].toScalarType()));
        const size_t need = avion_embedding_bwd_workspace_bytes(n, V, (int)D);
        const Tensor ws = workspace(need, dy);
        check(avion_embedding_bwd(tokens.data_ptr(), dy.data_ptr(), dweight.data_ptr(), n, V, (int)D,
                                  (float)ctx->saved_data["scale"].toDouble(), embedding_flags(tokens, dweight, dy.scalar_type()),
                                  ws.data_ptr(), need, stream()));
        depends_on(dweight, "embedding", {grad[0]});
        return {dweight, Tensor(), Tensor(), Tensor()};
    }
};
pybind11::object embedding(pybind11::handle tokens_, pybind11::handle weight_, double scale, bool f16, bool bf16)
{
    HANDLE_TH_ERRORS
    const Tensor *tokens, *weight;
    if (!plain(tokens_.ptr(), &tokens) || !plain(weight_.ptr(), &weight) || !plain_thread() || f16 == bf16) return pybind11::none();
    const at::ScalarType out = f16 ? at::kHalf : at::kBFloat16;
    if (weight->dim() != 2 || weight->size(1) > INT32_MAX || tokens->device() != weight->device() ||
        (weight->scalar_type() != at::kFloat && weight->scalar_type() != out) ||
        (tokens->scalar_type() != at::kLong && tokens->scalar_type() != at::kInt))
        return pybind11::none();
    return without_lock([&] {
        if (records({weight})) return Embedding::apply(*weight, *tokens, scale, f16);
        const c10::DeviceGuard guard(weight->device());
        return embedding_fwd(*tokens, *weight, scale, out);
    });
    END_HANDLE_TH_ERRORS_PYBIND
}

// residual undefined: the norm of x itself.  {y, h (undefined then), rstd (where a backward follows)}
struct RmsOut {
    Tensor y, h, rstd, x;
};
RmsOut rms_fwd(const Tensor& x_, const Tensor& residual, const Tensor& weight, double eps, bool keep)
{
    RmsOut r;
    r.x = dense(x_);
    const int64_t D = r.x.size(-1), M = r.x.numel() / D;
    const Tensor res = residual.defined() ? dense(residual) : Tensor();
    r.y = at::empty(r.x.sizes(), r.x.options());
    if (res.defined()) r.h = at::empty(res.sizes(), res.options());
    if (keep) r.rstd = at::empty({M}, weight.options());
    check(avion_rmsnorm_fwd(r.x.data_ptr(), data_of(res), dense(weight).data_ptr<float>(), r.y.data_ptr(), data_of(r.h),
                            static_cast<float*>(data_of(r.rstd)), M, (int)D, (float)eps,
                            format_flag(r.x) | (res.defined() ? wide_flag(res) : 0u), stream()));
    return r;
}
// {dx, dresidual, dweight}; where the stream has the format of y, dx is the gradient of both.  vary: h depends on what is
// differentiated
variable_list rms_bwd(const Tensor& h_, const Tensor& weight_, const Tensor& rstd, const Tensor& dy_, const Tensor& dh_, at::ScalarType format,
                      bool want_dx, bool want_dr, const char* what, bool vary)
{
    const Tensor& given = dy_.defined() ? dy_ : dh_;
    const c10::DeviceGuard guard(given.device());
    const Tensor dh = dh_.defined() ? dense(dh_) : Tensor();
    const Tensor dy = dy_.defined() ? dense(dy_) : at::zeros(given.sizes(), given.options().dtype(format));
    const int64_t D = given.size(-1), M = given.numel() / D;
    require(h_, "h", given.sizes(), dh.defined() ? dh.scalar_type() : h_.scalar_type(), given);
    const Tensor h = dense(h_), weight = dense(weight_);
    TORCH_CHECK_VALUE(h.scalar_type() == format || h.scalar_type() == at::kFloat, "h must be ", format, " or float, got ", h.scalar_type());
    require(weight, "weight", {D}, at::kFloat, given);
    require(rstd, "rstd", {M}, at::kFloat, given);
    const bool wide = h.scalar_type() == at::kFloat;
    Tensor dx, dr;
    if (want_dx || !wide) dx = at::empty_like(dy);
    if (want_dr && wide) dr = at::empty_like(h);
    const Tensor dweight = at::empty({D}, weight.options());
    const size_t need = avion_rmsnorm_bwd_workspace_bytes(M, (int)D);
    const Tensor ws = workspace(need, h);
    check(avion_rmsnorm_bwd(h.data_ptr(), weight.data_ptr<float>(), rstd.data_ptr<float>(), dy.data_ptr(), data_of(dh), data_of(dx),
                            static_cast<float*>(data_of(dr)), dweight.data_ptr<float>(), M, (int)D, format_flag(dy) | wide_flag(h),
                            ws.data_ptr(), need, stream()));
    depends_on(dx, what, {dy_, dh_, h_, weight_});
    if (wide) depends_on(dr, what, {dy_, dh_, h_, weight_});
    depends_on(dweight, what, {dy_, vary ? h_ : Tensor()});
    return {dx, wide ? dr : dx, dweight};
}
struct RmsNorm : torch::autograd::Function<RmsNorm> {
    static Tensor forward(AutogradContext* ctx, const Tensor& x, const Tensor& weight, double eps)
    {
        const c10::DeviceGuard guard(x.device());
        const RmsOut r = rms_fwd(x, Tensor(), weight, eps, true);
        ctx->save_for_backward({r.x, weight, r.rstd});  // the input and one float per token
        return r.y;
    }
    static variable_list backward(AutogradContext* ctx, variable_list grad)
    {
        const variable_list s = ctx->get_saved_variables();
        require(s[0], "x", grad[0].sizes(), grad[0].scalar_type(), grad[0]);
        variable_list g = rms_bwd(s[0], s[1], s[2], grad[0], Tensor(), grad[0].scalar_type(), true, false, "rms_norm", true);
        return {g[0], g[2], Tensor()};
    }
};
struct AddRmsNorm : torch::autograd::Function<AddRmsNorm> {
    static variable_list forward(AutogradContext* ctx, const Tensor& x, const Tensor& residual, const Tensor& weight, double eps)
    {
        const c10::DeviceGuard guard(x.device());
        const RmsOut r = rms_fwd(x, residual, weight, eps, true);
        ctx->set_materialize_grads(false);
        ctx->save_for_backward({r.h, weight, r.rstd});  // the residual stream, kept anyway, and one float per token; not y
        ctx->saved_data["format"] = x.scalar_type();
        ctx->saved_data["vary"] = x.requires_grad() || residual.requires_grad();
        return {r.y, r.h};
    }
    static variable_list backward(AutogradContext* ctx, variable_list grad)
    {
        if (!grad[0].defined() && !grad[1].defined()) return {Tensor(), Tensor(), Tensor(), Tensor()};
        const variable_list s = ctx->get_saved_variables();
        variable_list g = rms_bwd(s[0], s[1], s[2], grad[0], grad[1], ctx->saved_data["format"].toScalarType(),
                                  ctx->needs_input_grad(0), ctx->needs_input_grad(1), "add_rms_norm", ctx->saved_data["vary"].toBool());
        g.resize(4);
        return g;
    }
};
// x, weight and (where there is one) residual of a norm in the expected formats and shapes
bool rms_args(pybind11::handle x_, pybind11::handle residual_, pybind11::handle weight_, const Tensor** x, const Tensor** residual,
              const Tensor** weight)
{
    if (!plain(x_.ptr(), x) || !plain_thread()) return false;
    if ((*x)->dim() < 1 || !element_format(**x) || (*x)->size(-1) > INT32_MAX || !parameter(weight_.ptr(), (*x)->size(-1), **x, weight))
        return false;
    if (!residual) return true;
    if (!plain(residual_.ptr(), residual)) return false;
    const Tensor& r = **residual;
    return r.sizes() == (*x)->sizes() && r.device() == (*x)->device() &&
           (r.scalar_type() == (*x)->scalar_type() || r.scalar_type() == at::kFloat);
}
pybind11::object rms_norm(pybind11::handle x_, pybind11::handle weight_, double eps)
{
    HANDLE_TH_ERRORS
    const Tensor *x, *weight;
    if (!rms_args(x_, x_, weight_, &x, nullptr, &weight)) return pybind11::none();
    return without_lock([&] {
        if (records({x, weight})) return RmsNorm::apply(dense(*x), *weight, eps);
        const c10::DeviceGuard guard(x->device());
        return rms_fwd(*x, Tensor(), *weight, eps, false).y;
    });
    END_HANDLE_TH_ERRORS_PYBIND
}
pybind11::object add_rms_norm(pybind11::handle x_, pybind11::handle residual_, pybind11::handle weight_, double eps)
{
    HANDLE_TH_ERRORS
    const Tensor *x, *residual, *weight;
    if (!rms_args(x_, residual_, weight_, &x, &residual, &weight)) return pybind11::none();
    return many_without_lock([&]() -> variable_list {
        if (records({x, residual, weight})) return AddRmsNorm::apply(*x, *residual, *weight, eps);
        const c10::DeviceGuard guard(x->device());
        const RmsOut r = rms_fwd(*x, *residual, *weight, eps, false);
        return {r.y, r.h};
    });
    END_HANDLE_TH_ERRORS_PYBIND
}

// ---- 8 bits: no backward; the caller has made sure that nothing records
variable_list rms_fp8(const Tensor& x_, const Tensor& residual, const Tensor& weight, double eps)
{
    const c10::DeviceGuard guard(x_.device());
    const Tensor x = dense(x_), res = residual.defined() ? dense(residual) : Tensor();
    const int64_t D = x.size(-1), M = x.numel() / D;
    const Tensor y8 = at::empty(x.sizes(), x.options().dtype(at::kFloat8_e4m3fn));
    const Tensor scale = at::empty(x.sizes().slice(0, x.dim() - 1), weight.options());
    const Tensor h = res.defined() ? at::empty(res.sizes(), res.options()) : Tensor();
    check(avion_rmsnorm_fwd_fp8(x.data_ptr(), data_of(res), dense(weight).data_ptr<float>(), y8.data_ptr(), scale.data_ptr<float>(),
                                data_of(h), M, (int)D, (float)eps, format_flag(x) | (res.defined() ? wide_flag(res) : 0u), stream()));
    if (h.defined()) return {y8, scale, h};
    return {y8, scale};
}
pybind11::object rms_norm_fp8(pybind11::handle x_, pybind11::handle weight_, double eps)
{
    HANDLE_TH_ERRORS
    const Tensor *x, *weight;
    if (!rms_args(x_, x_, weight_, &x, nullptr, &weight) || records({x, weight})) return pybind11::none();
    return many_without_lock([&] { return rms_fp8(*x, Tensor(), *weight, eps); });
    END_HANDLE_TH_ERRORS_PYBIND
}
pybind11::object add_rms_norm_fp8(pybind11::handle x_, pybind11::handle residual_, pybind11::handle weight_, double eps)
{
    HANDLE_TH_ERRORS
    const Tensor *x, *residual, *weight;
    if (!rms_args(x_, residual_, weight_, &x, &residual, &weight) || records({x, residual, weight})) return pybind11::none();
    return many_without_lock([&] { return rms_fp8(*x, *residual, *weight, eps); });
    END_HANDLE_TH_ERRORS_PYBIND
}
pybind11::object quantize_rows(pybind11::handle x_)
{
    HANDLE_TH_ERRORS
    const Tensor* x;
    if (!plain(x_.ptr(), &x) || !plain_thread() || x->dim() < 1 || !element_format(*x) || x->size(-1) > INT32_MAX || records({x}))
        return pybind11::none();
    return many_without_lock([&]() -> variable_list {
        const c10::DeviceGuard guard(x->device());
        const Tensor in = dense(*x);
        const int64_t D = in.size(-1);
        const Tensor x8 = at::empty(in.sizes(), in.options().dtype(at::kFloat8_e4m3fn));
        const Tensor scale = at::empty(in.sizes().slice(0, in.dim() - 1), in.options().dtype(at::kFloat));
        check(avion_quantize_rows(in.data_ptr(), x8.data_ptr(), scale.data_ptr<float>(), in.numel() / D, (int)D, format_flag(in), stream()));
        return {x8, scale};
    });
    END_HANDLE_TH_ERRORS_PYBIND
}
pybind11::object linear_fp8(pybind11::handle x8_, pybind11::handle xs_, pybind11::handle w8_, pybind11::handle ws_, pybind11::handle bias_,
                            bool f16, bool bf16)
{
    HANDLE_TH_ERRORS
    const Tensor *x8, *xs, *w8, *ws, *bias = nullptr;
    if (!plain(x8_.ptr(), &x8) || !plain(xs_.ptr(), &xs) || !plain(w8_.ptr(), &w8) || !plain_thread() || f16 == bf16)
        return pybind11::none();
    if (x8->dim() < 1 || w8->dim() != 2 || x8->scalar_type() != at::kFloat8_e4m3fn || w8->scalar_type() != at::kFloat8_e4m3fn ||
        w8->size(1) != x8->size(-1) || w8->device() != x8->device() || !fits_int(*w8) || xs->scalar_type() != at::kFloat ||
        xs->device() != x8->device() || xs->sizes() != x8->sizes().slice(0, x8->dim() - 1))
        return pybind11::none();
    if (!parameter(ws_.ptr(), w8->size(0), *x8, &ws) || (!bias_.is_none() && !parameter(bias_.ptr(), w8->size(0), *x8, &bias)))
        return pybind11::none();
    if (records({xs, ws}) || (bias && records({bias}))) return pybind11::none();
    return without_lock([&] {
        const c10::DeviceGuard guard(x8->device());
        const Tensor x = dense(*x8), s = xs->contiguous(), w = dense(*w8), sw = dense(*ws);
        const Tensor b = bias ? dense(*bias) : Tensor();
        const int64_t K = x.size(-1), N = w.size(0);
        std::vector<int64_t> shape = x.sizes().vec();
        shape.back() = N;
        const Tensor y = at::empty(shape, x.options().dtype(f16 ? at::kHalf : at::kBFloat16));
        check(avion_linear_fp8(x.data_ptr(), s.data_ptr<float>(), w.data_ptr(), sw.data_ptr<float>(), static_cast<float*>(data_of(b)),
                               y.data_ptr(), x.numel() / K, (int)N, (int)K, f16 ? AVION_FLAG_F16 : 0u, stream()));
        return y;
    });
    END_HANDLE_TH_ERRORS_PYBIND
}

}  // namespace

PYBIND11_MODULE(_avion_torch, m)
{
    m.doc() = "native calls of the autograd front end (csrc/avion_torch.cpp); each returns None for a call it does not take";
    m.def("attention", &attention);
    m.def("attention_qkvpacked", &attention_qkvpacked);
    m.def("layer_norm", &layer_norm);
    m.def("bias_gelu", &bias_gelu);
    m.def("bias_gelu_linear", &bias_gelu_linear);
    m.def("embedding", &embedding);
    m.def("rms_norm", &rms_norm);
    m.def("add_rms_norm", &add_rms_norm);
    m.def("rms_norm_fp8", &rms_norm_fp8);
    m.def("add_rms_norm_fp8", &add_rms_norm_fp8);
    m.def("quantize_rows", &quantize_rows);
    m.def("linear_fp8", &linear_fp8);
}
