// The sequence-model operators of include/sig_sequence.h for torch: argument checks and marshalling, and their autograd
// nodes.  As in sig_torch.cpp all arithmetic stays behind the C ABI.
#include "sig_torch.h"

#include <torch/csrc/autograd/functions/basic_ops.h>

#include "sig_sequence.h"

namespace {

using namespace sig_torch;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

[[noreturn]] void refuse(const std::string &what) { throw std::invalid_argument(what); }

void check(int rc, const char *where)
{
    if (rc != SIG_OK) throw Failure{rc, where};
}

// the same on a thread of the autograd engine
void check_in_backward(int rc, const char *where)
{
    if (rc != SIG_OK) rethrow_in_python(Failure{rc, where});
}

int type_of(const at::Tensor &t, const char *name)
{
    if (t.is_cuda()) {
        if (t.scalar_type() == at::kFloat) return SIG_F32;
        if (t.scalar_type() == at::kBFloat16) return SIG_BF16;
        if (t.scalar_type() == at::kHalf) return SIG_F16;
    }
    refuse(std::string(name) + " must be a float32, bfloat16 or float16 tensor on the GPU");
}

void same_place(const at::Tensor &t, const at::Tensor &as, const char *name)
{
    if (t.device() != as.device()) refuse(std::string(name) + " must be on the same GPU as the other tensors");
}

void same_type(const at::Tensor &t, const at::Tensor &as, const char *name)
{
    if (t.scalar_type() != as.scalar_type()) refuse(std::string(name) + " must have the type of the other operands");
    same_place(t, as, name);
}

// values of an axis next to each other
at::Tensor unit_rows(const at::Tensor &t) { return t.dim() > 0 && t.size(-1) > 1 && t.stride(-1) != 1 ? t.contiguous() : t; }

const void *data(const at::Tensor &t) { return t.defined() ? t.const_data_ptr() : nullptr; }
void *own_data(const at::Tensor &t) { return t.defined() ? t.mutable_data_ptr() : nullptr; }
const float *floats(const at::Tensor &t) { return t.defined() ? t.const_data_ptr<float>() : nullptr; }
float *own_floats(const at::Tensor &t) { return t.defined() ? t.mutable_data_ptr<float>() : nullptr; }

bool tracked(std::initializer_list<const at::Tensor *> inputs)
{
    bool any = false;
    for (const at::Tensor *t : inputs) {
        if (!t->defined()) continue;
        TORCH_CHECK_NOT_IMPLEMENTED(!t->_fw_grad(0).defined(), "libsig's operators have no forward-mode derivative");
        any = any || t->requires_grad();
    }
    return any && at::GradMode::is_enabled();
}

// An input that may be missing, on its way through a custom function, which takes no undefined tensors
using Maybe = std::optional<at::Tensor>;
Maybe maybe(const at::Tensor &t) { return t.defined() ? Maybe(t) : Maybe(); }
at::Tensor given(const Maybe &t) { return t ? *t : at::Tensor(); }

// Gradients of a backward pass that may itself be differentiated (with respect to any of `from`): that is an error, not a zero
variable_list first_order_only(variable_list grads, const variable_list &from, const variable_list &upstream)
{
    if (!at::GradMode::is_enabled()) return grads;
    torch::autograd::edge_list edges;
    for (const variable_list *list : {&from, &upstream})
        for (const at::Tensor &t : *list)
            if (t.defined() && t.requires_grad()) edges.push_back(torch::autograd::impl::gradient_edge(t));
    const auto error = std::make_shared<torch::autograd::Error>("libsig's operators have no second derivative", std::move(edges));
    for (const at::Tensor &g : grads)
        if (g.defined()) torch::autograd::set_history(g, error);
    return grads;
}

// ---------------------------------------------------------------- layer norm
// rows of a tensor [..., width]: how many, and how far apart (a tensor whose rows are not evenly spaced is copied)
struct Rows {
    at::Tensor t;
    int64_t count, width, stride;

    explicit Rows(const at::Tensor &from) : t(unit_rows(from)), count(1), width(from.size(-1)), stride(from.size(-1))
    {
        bool even = true, first = true;
        int64_t next = 0;
        for (int64_t i = t.dim() - 2; i >= 0; --i) {
            count *= t.size(i);
            if (t.size(i) == 1) continue;
            if (first) stride = t.stride(i);
            else even = even && t.stride(i) == next;
            next = t.stride(i) * t.size(i);
            first = false;
        }
        if (!even) {
            t = t.contiguous();
            stride = width;
        }
    }
};

struct NormWeights {
    at::Tensor weight, bias;
    int type;

    NormWeights(const at::Tensor &x, const at::Tensor &w, const at::Tensor &b) : type(SIG_F32)
    {
        for (const auto &[t, name] : {std::pair<const at::Tensor &, const char *>{w, "weight"}, {b, "bias"}}) {
            if (!t.defined()) continue;
            if (t.dim() != 1 || t.size(0) != x.size(-1)) refuse(std::string(name) + " must have one value for each value of a row");
            if (t.scalar_type() != at::kFloat && t.scalar_type() != x.scalar_type()) refuse(std::string(name) + " must be float32 or have the type of x");
            same_place(t, x, name);
        }
        if (w.defined() && b.defined() && w.scalar_type() != b.scalar_type()) refuse("weight and bias must have the same type");
        if (w.defined()) weight = w.contiguous();
        if (b.defined()) bias = b.contiguous();
        if (w.defined() || b.defined()) type = type_of(w.defined() ? w : b, "weight");
    }
};

at::Tensor layer_norm(const at::Tensor &x, const at::Tensor &weight, const at::Tensor &bias, double eps, at::Tensor *stats)
{
    const int type = type_of(x, "x");
    if (x.dim() < 1) refuse("x must have an axis to normalise");
    const NormWeights w(x, weight, bias);
    const Rows rows(x);
    at::Tensor y = at::empty(x.sizes(), x.options().memory_format(at::MemoryFormat::Contiguous));
    if (stats) *stats = at::empty({rows.count, 2}, x.options().dtype(at::kFloat));
    check(sig_layer_norm(default_ctx, data(rows.t), rows.stride, rows.count, rows.width, type, data(w.weight), data(w.bias), w.type, eps,
                         own_data(y), stats ? own_floats(*stats) : nullptr, current_stream()), "sig_layer_norm");
    return y;
}

struct LayerNorm : torch::autograd::Function<LayerNorm> {
    static at::Tensor forward(AutogradContext *ctx, const at::Tensor &x, const Maybe &weight_, const Maybe &bias_, double eps)
    {
        at::AutoDispatchBelowADInplaceOrView below_autograd;
        const at::Tensor weight = given(weight_), bias = given(bias_);
        at::Tensor stats;
        const at::Tensor y = layer_norm(x, weight, bias, eps, &stats);
        ctx->save_for_backward({x, weight, stats});
        ctx->saved_data["weight_type"] = (int64_t)(weight.defined() ? weight.scalar_type() : bias.defined() ? bias.scalar_type() : at::kFloat);
        ctx->saved_data["bias"] = bias.defined();
        return y;
    }

    static variable_list backward(AutogradContext *ctx, const variable_list &grads)
    {
        const variable_list saved = ctx->get_saved_variables();
        const at::Tensor &x = saved[0], &weight = saved[1], &stats = saved[2];
        const auto weight_type = (at::ScalarType)ctx->saved_data["weight_type"].toInt();
        variable_list out(4);
        {
            at::AutoDispatchBelowADInplaceOrView below_autograd;
            const Rows rows(x), g(grads[0]);
            const at::Tensor w = weight.defined() ? weight.contiguous() : weight;
            if (ctx->needs_input_grad(0)) out[0] = at::empty(x.sizes(), x.options().memory_format(at::MemoryFormat::Contiguous));
            if (weight.defined() && ctx->needs_input_grad(1)) out[1] = at::empty({rows.width}, x.options().dtype(weight_type));
            // (an edge for each tensor that was given)
            if (ctx->saved_data["bias"].toBool() && ctx->needs_input_grad(weight.defined() ? 2 : 1)) out[2] = at::empty({rows.width}, x.options().dtype(weight_type));
            const int kind = weight_type == at::kFloat ? SIG_F32 : weight_type == at::kBFloat16 ? SIG_BF16 : SIG_F16;
            check_in_backward(sig_layer_norm_backward(default_ctx, data(rows.t), rows.stride, rows.count, rows.width, type_of(x, "x"), data(w), kind,
                                                      floats(stats), data(g.t), g.stride, own_data(out[0]), own_data(out[1]), own_data(out[2]),
                                                      current_stream()), "sig_layer_norm_backward");
        }
        return first_order_only(std::move(out), saved, grads);
    }
};

at::Tensor differentiable_layer_norm(const at::Tensor &x, const at::Tensor &weight, const at::Tensor &bias, double eps)
{
    if (tracked({&x, &weight, &bias})) return LayerNorm::apply(x, maybe(weight), maybe(bias), eps);
    at::AutoDispatchBelowADInplaceOrView below_autograd;
    return layer_norm(x, weight, bias, eps, nullptr);
}

// ---------------------------------------------------------------- rotary positions
// first and last byte that a tensor's values take
std::pair<const char *, const char *> span_of(const at::Tensor &t)
{
    int64_t low = 0, high = 0;
    for (int64_t i = 0; i < t.dim(); ++i) (t.stride(i) < 0 ? low : high) += (t.size(i) - 1) * t.stride(i);
    const char *at = (const char *)t.const_data_ptr();
    return {at + low * t.element_size(), at + (high + 1) * t.element_size()};
}

struct RotaryPlace {
    at::Tensor positions, frequencies;
    int type;
    int64_t strides[2];

    RotaryPlace(const at::Tensor &x, const at::Tensor &p, const at::Tensor &f)
    {
        if (x.dim() != 4) refuse("x must have four dimensions: batch, length, heads, components");
        same_place(p, x, "positions");
        same_place(f, x, "frequencies");
        if (f.dim() != 1 || f.scalar_type() != at::kDouble) refuse("frequencies must be a float64 vector, one for each pair that is turned");
        if (2 * f.size(0) > x.size(3)) refuse("there are more frequencies than pairs of components");
        switch (p.scalar_type()) {
        case at::kInt: type = SIG_POSITION_I32; break;
        case at::kLong: type = SIG_POSITION_I64; break;
        case at::kFloat: type = SIG_POSITION_F32; break;
        case at::kDouble: type = SIG_POSITION_F64; break;
        default: refuse("positions must be int32, int64, float32 or float64");
        }
        if (p.dim() < 1 || p.dim() > 2 || p.size(-1) != x.size(1) || (p.dim() == 2 && p.size(0) != x.size(0) && p.size(0) != 1))
            refuse("positions must be [length] or [batch, length]");
        positions = p;
        frequencies = f.contiguous();
        strides[0] = p.dim() == 2 && p.size(0) > 1 ? p.stride(0) : 0;
        strides[1] = p.stride(-1);
    }
};

int turn(const at::Tensor &x, const at::Tensor &y, const RotaryPlace &at, bool interleaved, double scale, bool inverse)
{
    return sig_rotary(default_ctx, data(x), x.strides().data(), own_data(y), y.strides().data(), type_of(x, "x"), x.size(0), x.size(1), x.size(2),
                      x.size(3), 2 * at.frequencies.size(0), data(at.positions), at.type, at.strides, at.frequencies.const_data_ptr<double>(),
                      interleaved, scale, inverse, current_stream());
}

at::Tensor rotary(const at::Tensor &from, const at::Tensor &positions, const at::Tensor &frequencies, bool interleaved, double scale, const at::Tensor &out)
{
    type_of(from, "x");
    const RotaryPlace place(from, positions, frequencies);
    const at::Tensor x = unit_rows(from);
    at::Tensor y = out;
    if (out.defined()) {
        same_type(out, from, "out");
        if (out.sizes() != from.sizes()) refuse("out must have the shape of x");
        if (out.size(3) > 1 && out.stride(3) != 1) refuse("the last axis of out must be contiguous");
        // (a value that is written twice, or read after it was: wrong in a way that depends on the order)
        if (out.numel() > 0) {
            at::assert_no_internal_overlap(out);
            const bool same = out.const_data_ptr() == x.const_data_ptr() && out.strides() == x.strides();
            const auto a = span_of(x), b = span_of(out);
            if (!same && a.first < b.second && b.first < a.second) refuse("out must be x itself or lie apart from it");
        }
    } else {
        y = at::empty(x.sizes(), x.options().memory_format(at::MemoryFormat::Contiguous));
    }
    check(turn(x, y, place, interleaved, scale, false), "sig_rotary");
    if (out.defined()) out.unsafeGetTensorImpl()->bump_version();
    return y;
}

struct Rotary : torch::autograd::Function<Rotary> {
    static at::Tensor forward(AutogradContext *ctx, const at::Tensor &x, const at::Tensor &positions, const at::Tensor &frequencies, bool interleaved,
                              double scale)
    {
        at::AutoDispatchBelowADInplaceOrView below_autograd;
        const at::Tensor y = rotary(x, positions, frequencies, interleaved, scale, at::Tensor());
        ctx->save_for_backward({positions, frequencies});
        ctx->saved_data["interleaved"] = interleaved;
        ctx->saved_data["scale"] = scale;
        return y;
    }

    static variable_list backward(AutogradContext *ctx, const variable_list &grads)
    {
        const variable_list saved = ctx->get_saved_variables();
        variable_list out(5);
        {
            at::AutoDispatchBelowADInplaceOrView below_autograd;
            const at::Tensor g = unit_rows(grads[0]);
            out[0] = at::empty(g.sizes(), g.options().memory_format(at::MemoryFormat::Contiguous));
            check_in_backward(turn(g, out[0], RotaryPlace(g, saved[0], saved[1]), ctx->saved_data["interleaved"].toBool(),
                                   ctx->saved_data["scale"].toDouble(), true), "sig_rotary");
        }
        return first_order_only(std::move(out), saved, grads);
    }
};

at::Tensor differentiable_rotary(const at::Tensor &x, const at::Tensor &positions, const at::Tensor &frequencies, bool interleaved, double scale)
{
    if (at::GradMode::is_enabled() && (positions.requires_grad() || frequencies.requires_grad()))
        refuse("rotary has no gradient with respect to positions or frequencies");
    if (tracked({&x, &positions, &frequencies})) return Rotary::apply(x, positions, frequencies, interleaved, scale);
    at::AutoDispatchBelowADInplaceOrView below_autograd;
    return rotary(x, positions, frequencies, interleaved, scale, at::Tensor());
}

// ---------------------------------------------------------------- linear attention
struct Attention {
    at::Tensor q, k, v, log_decay, state, lengths;
    sig_attention_t shape;

    // q, k, v: [batch, length, heads, .]
    Attention(const at::Tensor &q_, const at::Tensor &k_, const at::Tensor &v_, const at::Tensor &decay, const at::Tensor &state_,
              const at::Tensor &lengths_, double scale)
    {
        const int type = type_of(q_, "q");
        same_type(k_, q_, "k");
        same_type(v_, q_, "v");
        const int64_t B = q_.size(0), T = q_.size(1), H = q_.size(2), K = q_.size(3), G = k_.size(2), V = v_.size(3);
        if (k_.size(0) != B || k_.size(1) != T || k_.size(3) != K) refuse("k must have the batch, length and components of q");
        if (v_.size(0) != B || v_.size(1) != T || v_.size(2) != G) refuse("v must have the batch, length and heads of k");
        if (G < 1 || H < 1 || H % G) refuse("the heads of q must be a multiple of the heads of k and v");
        if (std::max({H, K, V}) > INT32_MAX) refuse("too many heads or components");
        same_place(decay, q_, "log_decay");
        if (decay.dim() != 1 || decay.size(0) != H || decay.scalar_type() != at::kFloat) refuse("log_decay must be float32, one value for each head of q");
        if (state_.defined()) {
            same_place(state_, q_, "state");
            if (state_.scalar_type() != at::kFloat || state_.sizes() != at::IntArrayRef({B, H, K, V}))
                refuse("state must be float32 [batch, heads, components of k, components of v]");
            state = state_.contiguous();
        }
        if (lengths_.defined()) {
            same_place(lengths_, q_, "lengths");
            if (lengths_.dim() != 1 || lengths_.size(0) != B || (lengths_.scalar_type() != at::kLong && lengths_.scalar_type() != at::kInt))
                refuse("lengths must be int64 or int32, one for each batch element");
            lengths = lengths_.to(at::kLong).contiguous();
        }
        q = unit_rows(q_);
        k = unit_rows(k_);
        v = unit_rows(v_);
        log_decay = decay.contiguous();
        shape = {B, T, (int32_t)H, (int32_t)G, (int32_t)K, (int32_t)V, type, (float)scale, {}, {}, {}};
        for (int i = 0; i < 3; ++i) {
            shape.q_strides[i] = q.stride(i);
            shape.k_strides[i] = k.stride(i);
            shape.v_strides[i] = v.stride(i);
        }
    }

    at::Tensor new_out() const { return at::empty({shape.B, shape.T, shape.heads, shape.value_dim}, q.options().memory_format(at::MemoryFormat::Contiguous)); }
    at::Tensor new_state() const { return at::empty({shape.B, shape.heads, shape.key_dim, shape.value_dim}, log_decay.options()); }

    int forward(const at::Tensor &out, const at::Tensor &state_out) const
    {
        return sig_linear_attention(default_ctx, &shape, data(q), data(k), data(v), floats(log_decay), floats(state),
                                    lengths.defined() ? lengths.const_data_ptr<int64_t>() : nullptr, own_data(out), own_floats(state_out),
                                    current_stream());
    }
};

void four_dimensions(const at::Tensor &t, const char *name)
{
    if (t.dim() != 4) refuse(std::string(name) + " must have four dimensions: batch, length, heads, components");
}

// the output, and the final state if it is asked for
variable_list linear_attention(const Attention &a, bool return_state)
{
    variable_list out{a.new_out()};
    if (return_state) out.push_back(a.new_state());
    check(a.forward(out[0], return_state ? out[1] : at::Tensor()), "sig_linear_attention");
    return out;
}

struct LinearAttention : torch::autograd::Function<LinearAttention> {
    static variable_list forward(AutogradContext *ctx, const at::Tensor &q, const at::Tensor &k, const at::Tensor &v, const Maybe &state_,
                                 const at::Tensor &log_decay, const Maybe &lengths_, double scale, bool return_state)
    {
        at::AutoDispatchBelowADInplaceOrView below_autograd;
        const at::Tensor state = given(state_), lengths = given(lengths_);
        variable_list out = linear_attention(Attention(q, k, v, log_decay, state, lengths, scale), return_state);
        ctx->save_for_backward({q, k, v, state, log_decay, lengths});
        ctx->saved_data["scale"] = scale;
        ctx->set_materialize_grads(false);
        return out;
    }

    static variable_list backward(AutogradContext *ctx, const variable_list &grads)
    {
        const variable_list saved = ctx->get_saved_variables();
        variable_list out(8);
        {
            at::AutoDispatchBelowADInplaceOrView below_autograd;
            const Attention a(saved[0], saved[1], saved[2], saved[4], saved[3], saved[5], ctx->saved_data["scale"].toDouble());
            const at::Tensor g = grads[0].defined() ? grads[0].contiguous() : at::zeros({a.shape.B, a.shape.T, a.shape.heads, a.shape.value_dim}, a.q.options());
            const at::Tensor g_state = grads.size() > 1 && grads[1].defined() ? grads[1].contiguous() : at::Tensor();
            for (int i = 0; i < 3; ++i) out[i] = at::empty(saved[i].sizes(), saved[i].options().memory_format(at::MemoryFormat::Contiguous));
            if (saved[3].defined() && ctx->needs_input_grad(3)) out[3] = a.new_state();
            check_in_backward(sig_linear_attention_backward(default_ctx, &a.shape, data(a.q), data(a.k), data(a.v), floats(a.log_decay), floats(a.state),
                                                            a.lengths.defined() ? a.lengths.const_data_ptr<int64_t>() : nullptr, data(g), floats(g_state),
                                                            own_data(out[0]), own_data(out[1]), own_data(out[2]), own_floats(out[3]), current_stream()),
                              "sig_linear_attention_backward");
        }
        return first_order_only(std::move(out), saved, grads);
    }
};

// o_t of one token of every batch element: q [B, H, K], k [B, G, K], v [B, G, V]; the state is updated in place, or written to `next`
at::Tensor step(const at::Tensor &q, const at::Tensor &k, const at::Tensor &v, const at::Tensor &log_decay, const at::Tensor &state, double scale,
                const at::Tensor &next)
{
    for (const at::Tensor *t : {&q, &k, &v})
        if (t->dim() != 3) refuse("q, k and v of a token must have three dimensions: batch, heads, components");
    const Attention a(q.unsqueeze(1), k.unsqueeze(1), v.unsqueeze(1), log_decay, state, at::Tensor(), scale);
    const at::Tensor &to = next.defined() ? next : state;
    if (next.defined()) {
        same_type(next, state, "out_state");
        if (next.sizes() != state.sizes()) refuse("out_state must have the shape of state");
    }
    if (!to.is_contiguous()) refuse("the state that is written must be contiguous");
    if (to.numel() > 0) {
        const auto x = span_of(a.state), y = span_of(to);
        if (x.first != y.first && x.first < y.second && y.first < x.second) refuse("out_state must be state itself or lie apart from it");
    }
    const at::Tensor o = a.new_out();
    check(a.forward(o, to), "sig_linear_attention");
    to.unsafeGetTensorImpl()->bump_version();
    return o.squeeze(1);
}

// ---------------------------------------------------------------- Python
bool optional_tensor_arg(PyObject *o, at::Tensor *t)
{
    if (o == Py_None) return true;
    const at::Tensor *p = tensor_arg(o);
    if (p) *t = *p;
    return p != nullptr;
}

bool double_arg(PyObject *o, double *value)
{
    *value = PyFloat_AsDouble(o);
    return *value != -1.0 || !PyErr_Occurred();
}

bool flag_arg(PyObject *o, bool *value)
{
    const int truth = PyObject_IsTrue(o);
    *value = truth > 0;
    return truth >= 0;
}

PyObject *wrap(variable_list out)
{
    if (out.size() == 1) return THPVariable_Wrap(std::move(out[0]));
    PyObject *pair = PyTuple_New((Py_ssize_t)out.size());
    for (size_t i = 0; pair && i < out.size(); ++i) {
        PyObject *t = THPVariable_Wrap(std::move(out[i]));
        if (!t) {
            Py_DECREF(pair);
            return nullptr;
        }
        PyTuple_SET_ITEM(pair, (Py_ssize_t)i, t);
    }
    return pair;
}

// (x, weight, bias, eps)
template <bool DIFFERENTIABLE>
PyObject *py_layer_norm(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (!arity(n, 4)) return nullptr;
    const at::Tensor *x = tensor_arg(args[0]);
    at::Tensor weight, bias;
    double eps;
    if (!x || !optional_tensor_arg(args[1], &weight) || !optional_tensor_arg(args[2], &bias) || !double_arg(args[3], &eps)) return nullptr;
    return guarded([&] {
        at::Tensor y = unlocked([&] {
            if (DIFFERENTIABLE) return differentiable_layer_norm(*x, weight, bias, eps);
            at::AutoDispatchBelowADInplaceOrView below_autograd;
            return layer_norm(*x, weight, bias, eps, nullptr);
        });
        return THPVariable_Wrap(std::move(y));
    });
}

// (x, positions, frequencies, interleaved, scale[, out])
template <bool DIFFERENTIABLE>
PyObject *py_rotary(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (!arity(n, DIFFERENTIABLE ? 5 : 6)) return nullptr;
    const at::Tensor *x = tensor_arg(args[0]), *p = x ? tensor_arg(args[1]) : nullptr, *f = p ? tensor_arg(args[2]) : nullptr;
    at::Tensor out;
    bool interleaved;
    double scale;
    if (!f || !flag_arg(args[3], &interleaved) || !double_arg(args[4], &scale) || (n > 5 && !optional_tensor_arg(args[5], &out))) return nullptr;
    return guarded([&] {
        at::Tensor y = unlocked([&] {
            if (DIFFERENTIABLE) return differentiable_rotary(*x, *p, *f, interleaved, scale);
            at::AutoDispatchBelowADInplaceOrView below_autograd;
            return rotary(*x, *p, *f, interleaved, scale, out);
        });
        return THPVariable_Wrap(std::move(y));
    });
}

// None: one over the square root of the components of k
bool scale_arg(PyObject *o, const at::Tensor &q, double *scale)
{
    if (o != Py_None) return double_arg(o, scale);
    *scale = q.dim() > 0 && q.size(-1) > 0 ? 1.0 / std::sqrt((double)q.size(-1)) : 1.0;
    return true;
}

// (q, k, v, log_decay, state, lengths, scale, return_state)
template <bool DIFFERENTIABLE>
PyObject *py_linear_attention(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (!arity(n, 8)) return nullptr;
    const at::Tensor *t[4];
    for (int i = 0; i < 4; ++i)
        if (!(t[i] = tensor_arg(args[i]))) return nullptr;
    at::Tensor state, lengths;
    double scale;
    bool return_state;
    if (!optional_tensor_arg(args[4], &state) || !optional_tensor_arg(args[5], &lengths) || !scale_arg(args[6], *t[0], &scale) ||
        !flag_arg(args[7], &return_state))
        return nullptr;
    return guarded([&] {
        variable_list out = unlocked([&] {
            const char *names[] = {"q", "k", "v"};
            for (int i = 0; i < 3; ++i) four_dimensions(*t[i], names[i]);
            if (DIFFERENTIABLE) {
                if (at::GradMode::is_enabled() && t[3]->requires_grad()) refuse("linear_attention has no gradient with respect to log_decay");
                if (tracked({t[0], t[1], t[2], &state, t[3]}))
                    return LinearAttention::apply(*t[0], *t[1], *t[2], maybe(state), *t[3], maybe(lengths), scale, return_state);
            }
            at::AutoDispatchBelowADInplaceOrView below_autograd;
            return linear_attention(Attention(*t[0], *t[1], *t[2], *t[3], state, lengths, scale), return_state);
        });
        return wrap(std::move(out));
    });
}

// (q, k, v, log_decay, state, scale, out_state)
PyObject *py_linear_attention_step(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (!arity(n, 7)) return nullptr;
    const at::Tensor *t[5];
    for (int i = 0; i < 5; ++i)
        if (!(t[i] = tensor_arg(args[i]))) return nullptr;
    double scale;
    at::Tensor next;
    if (!scale_arg(args[5], *t[0], &scale) || !optional_tensor_arg(args[6], &next)) return nullptr;
    return guarded([&] {
        at::Tensor o = unlocked([&] {
            at::AutoDispatchBelowADInplaceOrView below_autograd;
            return step(*t[0], *t[1], *t[2], *t[3], *t[4], scale, next);
        });
        return THPVariable_Wrap(std::move(o));
    });
}

}  // namespace

PyMethodDef sig_torch::sequence_methods[] = {
    {"layer_norm", FASTCALL(py_layer_norm<false>), "layer_norm(x, weight, bias, eps)"},
    {"autograd_layer_norm", FASTCALL(py_layer_norm<true>), "layer_norm(x, weight, bias, eps) with a gradient"},
    {"rotary", FASTCALL(py_rotary<false>), "rotary(x, positions, frequencies, interleaved, scale, out)"},
    {"autograd_rotary", FASTCALL(py_rotary<true>), "rotary(x, positions, frequencies, interleaved, scale) with a gradient"},
    {"linear_attention", FASTCALL(py_linear_attention<false>), "linear_attention(q, k, v, log_decay, state, lengths, scale, return_state)"},
    {"autograd_linear_attention", FASTCALL(py_linear_attention<true>),
     "linear_attention(q, k, v, log_decay, state, lengths, scale, return_state) with a gradient"},
    {"linear_attention_step", FASTCALL(py_linear_attention_step), "linear_attention_step(q, k, v, log_decay, state, scale, out_state)"},
    {nullptr, nullptr, 0, nullptr}};
