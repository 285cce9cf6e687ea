// The sequence operators of include/snn_seq.h on torch tensors, and as autograd functions:
// argument checks, outputs, workspaces and streams.  The Python functions that users call
// (sequence.py, autograd.py) document them and pass their arguments on.
//
// Host code in C++ because the smallest calls are bound by it: a step of one token takes 4 to
// 10 us on the GPU, and what stood here in Python before took 10 to 15 us per call and, in a
// backward, which runs on a thread of its own, 45 to 120 us.
#include <ATen/Functions.h>
#include <ATen/TracerMode.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/utils/pybind.h>

#include "snn_seq.h"

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;
using Optional = std::optional<Tensor>;

Tensor or_none(const Optional& a) { return a.has_value() ? *a : Tensor(); }

[[noreturn]] void refuse(const std::string& what) { throw py::value_error(what); }

struct StatusError : std::runtime_error {
    StatusError(const char* f, snn_status s) : std::runtime_error(std::string(f) + ": " + snn_status_str(s)), fn(f), status(s) {}
    const char* fn;
    snn_status status;
};

void check(const char* fn, snn_status st) {
    if (st != SNN_OK) throw StatusError(fn, st);
}

// -- Arguments -----------------------------------------------------------------------------

int io_of(const Tensor& x) {
    if (!x.is_cuda()) refuse("tensors must be on the GPU");
    if (x.dim() != 3 || (x.scalar_type() != at::kFloat && x.scalar_type() != at::kBFloat16))
        refuse("data must be a float32 or bfloat16 tensor [T, B, F]");
    return x.scalar_type() == at::kFloat ? SNN_IO_F32 : SNN_IO_BF16;
}

// Whether the axes behind the second are contiguous.
bool has_rows(const Tensor& a) {
    int64_t n = 1;
    for (int64_t d = a.dim() - 1; d >= 2; --d) {
        if (a.size(d) != 1 && a.stride(d) != n) return false;
        n *= a.size(d);
    }
    return true;
}
Tensor rows(const Tensor& a) { return a.is_contiguous() || has_rows(a) ? a : a.contiguous(); }

// An output shaped like the rows of `a`, in its order of steps and sequences.  Where rows of `a`
// overlap that order may put an axis inside the rows: then dense and time-major.
Tensor rows_like(const Tensor& a) {
    Tensor out = at::empty_like(a);
    return out.is_contiguous() || has_rows(out) ? out : at::empty(a.sizes(), a.options());
}

void check_tensor(const char* name, const Tensor& a, const Tensor& x, at::IntArrayRef shape, at::ScalarType dtype,
                  bool dense) {
    if (!a.defined() || a.scalar_type() != dtype || a.sizes() != shape || a.device() != x.device() ||
        (dense && !a.is_contiguous()))
        refuse(c10::str(name, " must be a ", dense ? "contiguous " : "", dtype, " tensor of shape ", shape, " on ",
                        x.device()));
}

// `a` as [T, B, X] data that goes with x.
Tensor data(const char* name, const Tensor& a, const Tensor& x, at::IntArrayRef shape) {
    check_tensor(name, a, x, shape, x.scalar_type(), false);
    return rows(a);
}
Tensor data_or_none(const char* name, const Tensor& a, const Tensor& x, at::IntArrayRef shape) {
    return a.defined() ? data(name, a, x, shape) : a;
}

void* address(const Tensor& a) { return a.defined() ? a.data_ptr() : nullptr; }
float* floats(const Tensor& a) { return static_cast<float*>(address(a)); }

// The address of a parameter, a state or lengths; NULL without one.
template <typename T = float>
T* dense(const char* name, const Tensor& a, const Tensor& x, at::IntArrayRef shape, at::ScalarType dtype = at::kFloat) {
    if (!a.defined()) return nullptr;
    check_tensor(name, a, x, shape, dtype, true);
    return static_cast<T*>(a.data_ptr());
}

// An snn_seq, or NULL without a tensor.
struct Seq {
    snn_seq s;
    explicit Seq(const Tensor& a) : s{address(a), a.defined() ? a.stride(0) : 0, a.defined() ? a.stride(1) : 0} {}
    operator const snn_seq*() const { return s.data == nullptr ? nullptr : &s; }
};

void* stream_of(const Tensor& x) { return c10::hip::getCurrentHIPStream(x.get_device()).stream(); }

Tensor bytes(size_t n, const Tensor& x) {
    return n == 0 ? Tensor() : at::empty({int64_t(n)}, x.options().dtype(at::kByte));
}

Tensor like(const Tensor& a) { return a.defined() ? rows_like(a) : a; }

// A parameter's gradient: the kernels write it whole, unless there is nothing to do.
Tensor param_like(const Tensor& p, bool empty) {
    return !p.defined() ? p : empty ? at::zeros_like(p) : at::empty_like(p);
}

// No steps: the state out is the state in.
void hand_over(const Tensor& out, const Tensor& given) {
    if (!out.defined() || out.is_same(given)) return;
    if (given.defined()) out.copy_(given);
    else out.zero_();
}

// A caller's tensor has been written: a graph that saved it is to notice.
void written(const Tensor& a) {
    if (a.defined() && !a.is_inference()) a.unsafeGetTensorImpl()->bump_version();
}

// -- Convolution ---------------------------------------------------------------------------

struct ConvCall {
    int64_t T, B, F, W;
    Tensor x;
    snn_conv_cfg cfg;
    float *weight, *bias;
    void* state;
    int32_t* lengths;
    ConvCall(const Tensor& x_, const Tensor& w, const Tensor& b, int64_t act, const Tensor& st, const Tensor& ln) {
        const int io = io_of(x_);
        if (!w.defined() || w.dim() != 2 || (act != SNN_ACT_NONE && act != SNN_ACT_SILU))
            refuse("weight must be [F, W], act None or 'silu'");
        x = rows(x_);
        T = x.size(0), B = x.size(1), F = x.size(2), W = w.size(1);
        cfg = {io, int32_t(std::min<int64_t>(W, INT32_MAX)), int32_t(act)};
        weight = dense("weight", w, x, {F, W});
        bias = dense("bias", b, x, {F});
        state = state_like("state", st);
        lengths = dense<int32_t>("lengths", ln, x, {B}, at::kInt);
        size_t bytes;
        check("snn_conv_workspace_bytes", snn_conv_workspace_bytes(&cfg, T, B, F, &bytes));
    }
    void* state_like(const char* name, const Tensor& a) const {
        return dense<void>(name, a, x, {W - 1, B, F}, x.scalar_type());
    }
    bool empty() const { return T == 0 || B == 0 || F == 0; }
};

Tensor conv_forward(const Tensor& x, const Tensor& weight, const Tensor& bias, int64_t act, const Tensor& state,
                    const Tensor& state_out, const Tensor& lengths) {
    const ConvCall c(x, weight, bias, act, state, lengths);
    const c10::DeviceGuard guard(x.device());
    void* out = c.state_like("state_out", state_out);
    Tensor y = rows_like(c.x);
    if (c.empty()) hand_over(state_out, state);
    else
        check("snn_conv_forward", snn_conv_forward(&c.cfg, c.T, c.B, c.F, Seq(c.x), c.weight, c.bias, c.state, c.lengths,
                                                   Seq(y), out, stream_of(x)));
    written(state_out);
    return y;
}

variable_list conv_backward(const Tensor& x, const Tensor& weight, const Tensor& bias, const Tensor& grad_y, int64_t act,
                            const Tensor& state, const Tensor& lengths, const Tensor& grad_state_out) {
    const ConvCall c(x, weight, bias, act, state, lengths);
    const c10::DeviceGuard guard(x.device());
    const Tensor gy = data("grad_y", grad_y, c.x, {c.T, c.B, c.F});
    const void* g_out = c.state_like("grad_state_out", grad_state_out);
    Tensor gx = rows_like(c.x), gw = param_like(weight, c.empty()), gb = param_like(bias, c.empty()), gs = like(state);
    if (c.empty()) {
        hand_over(gs, grad_state_out);
    } else {
        size_t n;
        check("snn_conv_workspace_bytes", snn_conv_workspace_bytes(&c.cfg, c.T, c.B, c.F, &n));
        const Tensor ws = bytes(n, x);
        check("snn_conv_backward",
              snn_conv_backward(&c.cfg, c.T, c.B, c.F, Seq(c.x), c.weight, c.bias, c.state, c.lengths, Seq(gy), g_out,
                                Seq(gx), floats(gw), floats(gb), address(gs), address(ws), stream_of(x)));
    }
    return {gx, gw, gb, gs};
}

// -- Scan ----------------------------------------------------------------------------------

struct ScanCall {
    int64_t T, B, F, G, S;
    Tensor x, dt, Bm, Cm;
    snn_scan_cfg cfg;
    float *A, *D, *dt_bias, *h_in;
    int32_t* lengths;
    size_t saved, forward_ws, backward_ws;
    ScanCall(const Tensor& x_, const Tensor& dt_, const Tensor& A_, const Tensor& Bm_, const Tensor& Cm_, const Tensor& D_,
             const Tensor& dt_bias_, bool softplus, const Tensor& h, const Tensor& ln) {
        const int io = io_of(x_);
        if (!A_.defined() || !Bm_.defined() || Bm_.dim() != 4 || A_.dim() != 2)
            refuse("A must be [F, S], Bm and Cm [T, B, G, S]");
        x = rows(x_);
        T = x.size(0), B = x.size(1), F = x.size(2), G = Bm_.size(2), S = Bm_.size(3);
        dt = data("dt", dt_, x, {T, B, F});
        Bm = data("Bm", Bm_, x, {T, B, G, S});
        Cm = data("Cm", Cm_, x, {T, B, G, S});
        A = dense("A", A_, x, {F, S});
        D = dense("D", D_, x, {F});
        dt_bias = dense("dt_bias", dt_bias_, x, {F});
        h_in = dense("h_in", h, x, {B, F, S});
        lengths = dense<int32_t>("lengths", ln, x, {B}, at::kInt);
        cfg = {io, int32_t(std::min<int64_t>(S, INT32_MAX)), int32_t(std::min<int64_t>(G, INT32_MAX)), softplus};
        check("snn_scan_saved_bytes", snn_scan_saved_bytes(&cfg, T, B, F, &saved));
        check("snn_scan_workspace_bytes", snn_scan_workspace_bytes(&cfg, T, B, F, &forward_ws, &backward_ws));
    }
    bool empty() const { return T == 0 || B == 0 || F == 0; }
};

variable_list scan_forward(const Tensor& x, const Tensor& dt, const Tensor& A, const Tensor& Bm, const Tensor& Cm,
                           const Tensor& D, const Tensor& dt_bias, bool softplus, const Tensor& h_in, const Tensor& h_out,
                           const Tensor& lengths, bool train) {
    const ScanCall c(x, dt, A, Bm, Cm, D, dt_bias, softplus, h_in, lengths);
    const c10::DeviceGuard guard(x.device());
    float* out = dense("h_out", h_out, c.x, {c.B, c.F, c.S});
    if (train && out != nullptr && out == c.h_in) refuse("the backward reads h_in: h_out must be another tensor");
    Tensor y = rows_like(c.x), saved;
    if (train) saved = at::empty({int64_t(c.saved)}, x.options().dtype(at::kByte));
    if (c.empty()) {
        hand_over(h_out, h_in);
    } else {
        const Tensor ws = bytes(c.forward_ws, x);
        check("snn_scan_forward",
              snn_scan_forward(&c.cfg, c.T, c.B, c.F, Seq(c.x), Seq(c.dt), c.A, Seq(c.Bm), Seq(c.Cm), c.D, c.dt_bias, c.h_in,
                               c.lengths, Seq(y), out, address(saved), address(ws), stream_of(x)));
    }
    written(h_out);
    return {y, saved};
}

variable_list scan_backward(const Tensor& x, const Tensor& dt, const Tensor& A, const Tensor& Bm, const Tensor& Cm,
                            const Tensor& D, const Tensor& dt_bias, const Tensor& saved, const Tensor& grad_y, bool softplus,
                            const Tensor& h_in, const Tensor& lengths, const Tensor& grad_h_out) {
    const ScanCall c(x, dt, A, Bm, Cm, D, dt_bias, softplus, h_in, lengths);
    const c10::DeviceGuard guard(x.device());
    if (!saved.defined()) refuse("saved must be what scan_forward(train=True) returned for these arguments");
    check_tensor("saved", saved, c.x, {int64_t(c.saved)}, at::kByte, true);
    const Tensor gy = data("grad_y", grad_y, c.x, {c.T, c.B, c.F});
    const float* g_out = dense("grad_h_out", grad_h_out, c.x, {c.B, c.F, c.S});
    const bool none = c.empty();
    Tensor gx = rows_like(c.x), gdt = rows_like(c.x), gB = rows_like(c.Bm), gC = rows_like(c.Cm);
    Tensor gA = param_like(A, none), gD = param_like(D, none), gbias = param_like(dt_bias, none), gh = like(h_in);
    if (none) {
        gB.zero_();
        gC.zero_();
        hand_over(gh, grad_h_out);
    } else {
        const Tensor ws = bytes(c.backward_ws, x);
        check("snn_scan_backward",
              snn_scan_backward(&c.cfg, c.T, c.B, c.F, Seq(c.x), Seq(c.dt), c.A, Seq(c.Bm), Seq(c.Cm), c.D, c.dt_bias, c.h_in,
                                c.lengths, address(saved), Seq(gy), g_out, Seq(gx), Seq(gdt), floats(gA), Seq(gB), Seq(gC),
                                floats(gD), floats(gbias), floats(gh), address(ws), stream_of(x)));
    }
    return {gx, gdt, gA, gB, gC, gD, gbias, gh};
}

// -- Norm ----------------------------------------------------------------------------------

struct NormCall {
    int64_t T, B, F;
    Tensor y, r, z;
    snn_norm_cfg cfg;
    float *w_post, *scale, *w_pre;
    int32_t* lengths;
    size_t ws;
    NormCall(const Tensor& y_, const Tensor& r_, const Tensor& z_, const Tensor& post, const Tensor& s, const Tensor& pre,
             double eps, const Tensor& ln) {
        cfg = {io_of(y_), float(eps)};
        y = rows(y_);
        T = y.size(0), B = y.size(1), F = y.size(2);
        r = data_or_none("r", r_, y, {T, B, F});
        z = data_or_none("z", z_, y, {T, B, F});
        w_post = dense("w_post", post, y, {F});
        scale = dense("scale", s, y, {F});
        w_pre = dense("w_pre", pre, y, {F});
        lengths = dense<int32_t>("lengths", ln, y, {B}, at::kInt);
        check("snn_norm_workspace_bytes", snn_norm_workspace_bytes(&cfg, T, B, F, &ws));
    }
    bool empty() const { return T == 0 || B == 0 || F == 0; }
};

variable_list norm_forward(const Tensor& y, const Tensor& r, const Tensor& z, const Tensor& w_post, const Tensor& scale,
                           const Tensor& w_pre, double eps, const Tensor& lengths, bool train) {
    const NormCall c(y, r, z, w_post, scale, w_pre, eps, lengths);
    const c10::DeviceGuard guard(y.device());
    Tensor r_new = rows_like(c.y), u, rstd;
    if (w_pre.defined()) u = rows_like(c.y);
    if (train) rstd = at::empty({2, c.T, c.B}, y.options().dtype(at::kFloat));
    if (!c.empty())
        check("snn_norm_forward",
              snn_norm_forward(&c.cfg, c.T, c.B, c.F, Seq(c.y), Seq(c.z), Seq(c.r), c.w_post, c.scale, c.w_pre, c.lengths,
                               Seq(r_new), Seq(u), floats(rstd), stream_of(y)));
    return {r_new, u, rstd};
}

variable_list norm_backward(const Tensor& y, const Tensor& r, const Tensor& z, const Tensor& w_post, const Tensor& scale,
                            const Tensor& w_pre, const Tensor& rstd, const Tensor& grad_r_new, const Tensor& grad_u,
                            double eps, const Tensor& lengths) {
    const NormCall c(y, r, z, w_post, scale, w_pre, eps, lengths);
    const c10::DeviceGuard guard(y.device());
    const float* k = dense("rstd", rstd, c.y, {2, c.T, c.B});
    const Tensor g1 = data_or_none("grad_r_new", grad_r_new, c.y, {c.T, c.B, c.F});
    const Tensor g2 = data_or_none("grad_u", grad_u, c.y, {c.T, c.B, c.F});
    const bool none = c.empty();
    Tensor gy = like(c.y), gr = like(c.r), gz = like(c.z);
    Tensor g_post = param_like(w_post, none), g_scale = param_like(scale, none), g_pre = param_like(w_pre, none);
    if (!none) {
        const Tensor ws = bytes(c.ws, y);
        check("snn_norm_backward",
              snn_norm_backward(&c.cfg, c.T, c.B, c.F, Seq(c.y), Seq(c.z), Seq(c.r), c.w_post, c.scale, c.w_pre, c.lengths, k,
                                Seq(g1), Seq(g2), Seq(gy), Seq(gz), Seq(gr), floats(g_post), floats(g_scale), floats(g_pre),
                                address(ws), stream_of(y)));
    }
    return {gy, gr, gz, g_post, g_scale, g_pre};
}

// -- Autograd ------------------------------------------------------------------------------

// The gradients have none of their own: under create_graph a second backward through them
// raises an error instead of taking them for constants.
variable_list once(variable_list grads, size_t others) {
    if (at::GradMode::is_enabled()) {
        variable_list in;
        for (const Tensor& g : grads)
            if (g.defined()) in.push_back(g.detach().requires_grad_(true));
        auto node = std::make_shared<torch::autograd::DelayedError>(
            "the sequence operators' gradients cannot be differentiated again", int64_t(in.size()));
        const variable_list out = (*node)(std::move(in));
        size_t i = 0;
        for (Tensor& g : grads)
            if (g.defined()) g = out[i++];
    }
    grads.resize(grads.size() + others);     // none for the arguments that are no tensors of data
    return grads;
}

// Whether autograd has to hear of a call: a gradient is wanted, or an input has a forward-mode
// tangent, which the functions below have no rule for and refuse.
bool differentiated(std::initializer_list<Tensor> all) {
    const bool grad = at::GradMode::is_enabled();
    return std::any_of(all.begin(), all.end(), [grad](const Tensor& a) {
        return a.defined() && ((grad && a.requires_grad()) || a._fw_grad(/*level=*/0).defined());
    });
}

Tensor zeros_if_none(const Tensor& g, const Tensor& x) { return g.defined() ? g : at::zeros_like(x); }
Tensor contiguous(const Tensor& g) { return g.defined() ? g.contiguous() : g; }

struct Conv : torch::autograd::Function<Conv> {
    static variable_list forward(AutogradContext* ctx, const Tensor& x, const Tensor& weight, const Optional& bias,
                                 const Optional& state, const Optional& lengths, int64_t act, bool want_state) {
        const Tensor b = or_none(bias), s = or_none(state), ln = or_none(lengths);
        Tensor out;
        if (want_state) out = at::empty({weight.size(1) - 1, x.size(1), x.size(2)}, x.options());
        const Tensor y = conv_forward(x, weight, b, act, s, out, ln);
        ctx->save_for_backward({x, weight, b, s, ln});
        ctx->saved_data["act"] = act;
        ctx->set_materialize_grads(false);
        return want_state ? variable_list{y, out} : variable_list{y};
    }
    static variable_list backward(AutogradContext* ctx, variable_list g) {
        const auto v = ctx->get_saved_variables();
        return once(conv_backward(v[0], v[1], v[2], zeros_if_none(g[0], v[0]), ctx->saved_data["act"].toInt(), v[3], v[4],
                                  g.size() > 1 ? contiguous(g[1]) : Tensor()), 3);
    }
};

variable_list causal_conv(const Tensor& x, const Tensor& weight, const Optional& bias, int64_t act, const Optional& state,
                          const Optional& lengths, bool want_state) {
    io_of(x);
    if (!weight.defined() || weight.dim() != 2 || weight.size(1) < 1) refuse("weight must be [F, W], act None or 'silu'");
    if (differentiated({x, weight, or_none(bias), or_none(state)}))
        return Conv::apply(x, weight, bias, state, lengths, act, want_state);
    Tensor out;
    if (want_state) out = at::empty({weight.size(1) - 1, x.size(1), x.size(2)}, x.options());
    const Tensor y = conv_forward(x, weight, or_none(bias), act, or_none(state), out, or_none(lengths));
    return want_state ? variable_list{y, out} : variable_list{y};
}

struct Scan : torch::autograd::Function<Scan> {
    static variable_list forward(AutogradContext* ctx, const Tensor& x, const Tensor& dt, const Tensor& A, const Tensor& Bm,
                                 const Tensor& Cm, const Optional& D, const Optional& dt_bias, const Optional& h_in,
                                 const Optional& lengths, bool softplus, bool want_state) {
        const Tensor d = or_none(D), b = or_none(dt_bias), h = or_none(h_in), ln = or_none(lengths);
        Tensor out;
        if (want_state) out = at::empty({x.size(1), A.size(0), A.size(1)}, x.options().dtype(at::kFloat));
        const variable_list r = scan_forward(x, dt, A, Bm, Cm, d, b, softplus, h, out, ln, true);
        ctx->save_for_backward({x, dt, A, Bm, Cm, d, b, h, ln, r[1]});
        ctx->saved_data["softplus"] = softplus;
        ctx->set_materialize_grads(false);
        return want_state ? variable_list{r[0], out} : variable_list{r[0]};
    }
    static variable_list backward(AutogradContext* ctx, variable_list g) {
        const auto v = ctx->get_saved_variables();
        return once(scan_backward(v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[9], zeros_if_none(g[0], v[0]),
                                  ctx->saved_data["softplus"].toBool(), v[7], v[8],
                                  g.size() > 1 ? contiguous(g[1]) : Tensor()), 3);
    }
};

variable_list selective_scan(const Tensor& x, const Tensor& dt, const Tensor& A, const Tensor& Bm, const Tensor& Cm,
                             const Optional& D, const Optional& dt_bias, bool softplus, const Optional& h_in,
                             const Optional& lengths, bool want_state) {
    io_of(x);
    if (!dt.defined() || !A.defined() || A.dim() != 2 || !Bm.defined() || !Cm.defined())
        refuse("dt must be [T, B, F], A [F, S], Bm and Cm [T, B, G, S]");
    if (differentiated({x, dt, A, Bm, Cm, or_none(D), or_none(dt_bias), or_none(h_in)}))
        return Scan::apply(x, dt, A, Bm, Cm, D, dt_bias, h_in, lengths, softplus, want_state);
    Tensor out;
    if (want_state) out = at::empty({x.size(1), A.size(0), A.size(1)}, x.options().dtype(at::kFloat));
    const Tensor y = scan_forward(x, dt, A, Bm, Cm, or_none(D), or_none(dt_bias), softplus, or_none(h_in), out,
                                  or_none(lengths), false)[0];
    return want_state ? variable_list{y, out} : variable_list{y};
}

struct Norm : torch::autograd::Function<Norm> {
    static variable_list forward(AutogradContext* ctx, const Tensor& y, const Optional& r, const Optional& z,
                                 const Optional& w_post, const Optional& scale, const Optional& w_pre,
                                 const Optional& lengths, double eps) {
        const Tensor rr = or_none(r), zz = or_none(z), post = or_none(w_post), s = or_none(scale), pre = or_none(w_pre),
                     ln = or_none(lengths);
        const variable_list out = norm_forward(y, rr, zz, post, s, pre, eps, ln, true);
        ctx->save_for_backward({y, rr, zz, post, s, pre, out[2], ln});
        ctx->saved_data["eps"] = eps;
        ctx->set_materialize_grads(false);
        return pre.defined() ? variable_list{out[0], out[1]} : variable_list{out[0]};
    }
    static variable_list backward(AutogradContext* ctx, variable_list g) {
        const auto v = ctx->get_saved_variables();
        return once(norm_backward(v[0], v[1], v[2], v[3], v[4], v[5], v[6], g[0], g.size() > 1 ? g[1] : Tensor(),
                                  ctx->saved_data["eps"].toDouble(), v[7]), 2);
    }
};

variable_list block_norm(const Tensor& y, const Optional& r, const Optional& z, const Optional& w_post,
                         const Optional& scale, const Optional& w_pre, const Optional& lengths, double eps) {
    if (differentiated({y, or_none(r), or_none(z), or_none(w_post), or_none(scale), or_none(w_pre)}))
        return Norm::apply(y, r, z, w_post, scale, w_pre, lengths, eps);
    return norm_forward(y, or_none(r), or_none(z), or_none(w_post), or_none(scale), or_none(w_pre), eps, or_none(lengths),
                        false);
}

// Python's None as a tensor that is not defined, and the other way round: the casters do the latter.
template <typename A>
struct FromPython {
    using type = A;
    static A pass(A a) { return a; }
};
template <>
struct FromPython<const Tensor&> {
    using type = const Optional&;
    static Tensor pass(const Optional& a) { return or_none(a); }
};

// A list goes back as a tuple.
inline py::object to_python(const Tensor& a) { return py::cast(a); }
inline py::object to_python(const variable_list& all) {
    py::tuple out(all.size());
    for (size_t i = 0; i < all.size(); ++i) out[i] = py::cast(all[i]);
    return out;
}

template <typename R, typename... A>
auto bound(R (*fn)(A...)) {
    return [fn](typename FromPython<A>::type... a) {
        R out;
        {
            const py::gil_scoped_release free;
            // a trace would record where the outputs are allocated and not what fills them
            if (at::tracer::impl::is_dispatch_enabled())
                throw std::runtime_error("the sequence operators cannot be traced by torch.jit.trace");
            out = fn(FromPython<A>::pass(a)...);
        }
        return to_python(out);
    };
}

}  // namespace

PYBIND11_MODULE(_sequence, m) {
    py::register_local_exception_translator([](std::exception_ptr p) {
        try {
            if (p) std::rethrow_exception(p);
        } catch (const StatusError& e) {
            const py::object type = py::module_::import("paper_2408_00280_amd.native").attr("SnnError");
            const py::object error = type(e.fn, int(e.status), snn_status_str(e.status));
            PyErr_SetObject(type.ptr(), error.ptr());
        }
    });
    m.def("conv_forward", bound(conv_forward));
    m.def("conv_backward", bound(conv_backward));
    m.def("scan_forward", bound(scan_forward));
    m.def("scan_backward", bound(scan_backward));
    m.def("norm_forward", bound(norm_forward));
    m.def("norm_backward", bound(norm_backward));
    m.def("causal_conv", bound(causal_conv));
    m.def("selective_scan", bound(selective_scan));
    m.def("block_norm", bound(block_norm));
}
