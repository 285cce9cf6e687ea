// The C ABI declared in include/snn_seq.h: argument checks, workspaces and dispatch.
#include "seq_host.h"

using namespace snnlif;

namespace {

bool empty(int64_t T, int64_t B, int64_t F) { return T == 0 || B == 0 || F == 0; }

hipStream_t stream_of(void* s) { return static_cast<hipStream_t>(s); }

template <typename T>
T* carve(void* base, int64_t& at, int64_t bytes) {
    T* p = reinterpret_cast<T*>(static_cast<char*>(base) + at);
    at += piece(bytes);
    return p;
}

// Workspace: NULL only where its size is 0.  Pieces of it start on boundaries of their own.
snn_status check_workspace(const void* ws, int64_t bytes) { return bytes == 0 ? optional(ws, 16) : need(ws, 16); }

snn_status check_conv(const snn_conv_cfg* c, int64_t T, int64_t B, int64_t F) {
    const snn_status st = check_conv_cfg(c);
    if (st != SNN_OK) return st;
    if (check_seq_shape(T, B, F) != SNN_OK) return SNN_E_SHAPE;
    if (empty(T, B, F)) return SNN_OK;
    for (bool backward : {false, true}) {
        const ConvPlan p = conv_plan(c, T, B, F, backward);
        if (p.lanes * B * p.chunks > kMaxThreads - kBlock) return SNN_E_SHAPE;
    }
    return SNN_OK;
}

// With the plan, where there is anything to do.
snn_status check_scan(const snn_scan_cfg* c, int64_t T, int64_t B, int64_t F, ScanPlan& p) {
    const snn_status st = check_scan_cfg(c);
    if (st != SNN_OK) return st;
    if (check_seq_shape(T, B, F) != SNN_OK) return SNN_E_SHAPE;
    if (F % c->groups != 0) return SNN_E_SHAPE;
    if (empty(T, B, F)) return SNN_OK;
    p = scan_plan(c, T, B, F);
    if (p.tiles * c->groups > kMaxBlocks / B || F > kMaxN / B) return SNN_E_SHAPE;
    return T * B * c->groups <= kMaxBlocks && F * c->states <= kMaxSpan / B ? SNN_OK : SNN_E_SHAPE;
}

snn_status check_norm(const snn_norm_cfg* c, int64_t T, int64_t B, int64_t F) {
    const snn_status st = check_norm_cfg(c);
    if (st != SNN_OK) return st;
    if (check_seq_shape(T, B, F) != SNN_OK) return SNN_E_SHAPE;
    return SNN_OK;
}

ScanArgs scan_args(const snn_scan_cfg* c, const ScanPlan& plan, int64_t T, int64_t B, int64_t F, const snn_seq* x, const snn_seq* dt,
                   const float* A, const snn_seq* Bm, const snn_seq* Cm, const float* D, const float* dt_bias,
                   const float* h_in, const int32_t* lengths) {
    ScanArgs a = {};
    a.T = T;
    a.B = B;
    a.F = F;
    a.S = c->states;
    a.G = c->groups;
    a.softplus = c->softplus;
    a.x = rows(x);
    a.dt = rows(dt);
    a.Bm = rows(Bm);
    a.Cm = rows(Cm);
    a.A = A;
    a.D = D;
    a.dt_bias = dt_bias;
    a.h_in = h_in;
    a.lengths = lengths;
    a.plan = plan;
    a.layer = scan_grid(a.plan, B, a.G, 1).x;
    return a;
}

snn_status check_scan_inputs(const snn_scan_cfg* c, int64_t T, int64_t B, int64_t F, const snn_seq* x,
                             const snn_seq* dt, const float* A, const snn_seq* Bm, const snn_seq* Cm,
                             const float* D, const float* dt_bias, const float* h_in, const int32_t* lengths) {
    const int64_t gs = int64_t(c->groups) * c->states;
    return first_error({check_in(x, T, B, F, c->io), check_in(dt, T, B, F, c->io), need(A),
                        check_in(Bm, T, B, gs, c->io), check_in(Cm, T, B, gs, c->io), optional(D), optional(dt_bias),
                        optional(h_in), optional(lengths)});
}

NormArgs norm_args(const snn_norm_cfg* c, int64_t T, int64_t B, int64_t F, const snn_seq* y, const snn_seq* z,
                   const snn_seq* r, const float* w_post, const float* scale, const float* w_pre,
                   const int32_t* lengths, bool backward) {
    NormArgs a = {};
    a.T = T;
    a.B = B;
    a.F = F;
    a.eps = c->eps;
    a.y = rows(y);
    a.z = rows(z);
    a.r = rows(r);
    a.w_post = w_post;
    a.scale = scale;
    a.w_pre = w_pre;
    a.lengths = lengths;
    a.groups = norm_groups(T, B, F, backward);
    return a;
}

snn_status in_or_null(const snn_seq* s, int64_t T, int64_t B, int64_t F, int io) {
    return s == nullptr ? SNN_OK : check_in(s, T, B, F, io);
}

}  // namespace

extern "C" {

snn_status snn_conv_forward(const snn_conv_cfg* cfg, int64_t T, int64_t B, int64_t F, const snn_seq* x,
                            const float* weight, const float* bias, const void* state_in, const int32_t* lengths,
                            const snn_seq* y, void* state_out, void* stream) {
    snn_status st = check_conv(cfg, T, B, F);
    if (st != SNN_OK || empty(T, B, F)) return st;
    const int io = cfg->io;
    const uintptr_t e = uintptr_t(elem_bytes(io));
    st = first_error({check_in(x, T, B, F, io), check_out(y, T, B, F, io), need(weight), optional(bias),
                      optional(state_in, e), optional(state_out, e), optional(lengths)});
    if (st != SNN_OK) return st;
    ConvArgs a = {};
    a.T = T;
    a.B = B;
    a.F = F;
    a.x = rows(x);
    a.y = rows(y);
    a.weight = weight;
    a.bias = bias;
    a.state_in = state_in;
    a.lengths = lengths;
    a.state_out = state_out;
    a.plan = conv_plan(cfg, T, B, F, false);
    return conv_forward_entry(cfg, a, stream_of(stream));
}

snn_status snn_conv_workspace_bytes(const snn_conv_cfg* cfg, int64_t T, int64_t B, int64_t F, size_t* bytes) {
    const snn_status st = check_conv(cfg, T, B, F);
    if (st != SNN_OK) return st;
    if (bytes == nullptr) return SNN_E_NULL;
    *bytes = empty(T, B, F) ? 0 : size_t(conv_workspace(cfg, T, B, F));
    return SNN_OK;
}

snn_status snn_conv_backward(const snn_conv_cfg* cfg, int64_t T, int64_t B, int64_t F, const snn_seq* x,
                             const float* weight, const float* bias, const void* state_in, const int32_t* lengths,
                             const snn_seq* grad_y, const void* grad_state_out, const snn_seq* grad_x,
                             float* grad_weight, float* grad_bias, void* grad_state_in, void* workspace, void* stream) {
    snn_status st = check_conv(cfg, T, B, F);
    if (st != SNN_OK || empty(T, B, F)) return st;
    const int io = cfg->io;
    const uintptr_t e = uintptr_t(elem_bytes(io));
    st = first_error({check_in(x, T, B, F, io), check_in(grad_y, T, B, F, io), check_out(grad_x, T, B, F, io),
                      need(weight), need(grad_weight), need(workspace, 16), optional(bias), optional(grad_bias),
                      optional(state_in, e), optional(grad_state_out, e), optional(grad_state_in, e),
                      optional(lengths)});
    if (st != SNN_OK) return st;
    ConvArgs a = {};
    a.T = T;
    a.B = B;
    a.F = F;
    a.x = rows(x);
    a.gy = rows(grad_y);
    a.gx = rows(grad_x);
    a.weight = weight;
    a.bias = bias;
    a.state_in = state_in;
    a.lengths = lengths;
    a.gstate_out = grad_state_out;
    a.gstate_in = grad_state_in;
    a.part = static_cast<float*>(workspace);
    a.plan = conv_plan(cfg, T, B, F, true);
    st = conv_backward_entry(cfg, a, stream_of(stream));
    if (st != SNN_OK) return st;
    const ReduceOut out = {{grad_weight, grad_bias, nullptr}, {F * cfg->width, F, 0}};
    return reduce_entry(a.part, a.plan.chunks * B, conv_partial(cfg, F), out, stream_of(stream));
}

snn_status snn_scan_saved_bytes(const snn_scan_cfg* cfg, int64_t T, int64_t B, int64_t F, size_t* bytes) {
    ScanPlan plan;
    const snn_status st = check_scan(cfg, T, B, F, plan);
    if (st != SNN_OK) return st;
    if (bytes == nullptr) return SNN_E_NULL;
    *bytes = empty(T, B, F) ? 0 : size_t(scan_saved(cfg, plan, T, B, F));
    return SNN_OK;
}

snn_status snn_scan_workspace_bytes(const snn_scan_cfg* cfg, int64_t T, int64_t B, int64_t F, size_t* forward_bytes,
                                    size_t* backward_bytes) {
    ScanPlan plan;
    const snn_status st = check_scan(cfg, T, B, F, plan);
    if (st != SNN_OK) return st;
    if (forward_bytes == nullptr || backward_bytes == nullptr) return SNN_E_NULL;
    *forward_bytes = empty(T, B, F) ? 0 : size_t(scan_forward_workspace(cfg, plan, B, F));
    *backward_bytes = empty(T, B, F) ? 0 : size_t(scan_backward_workspace(cfg, plan, T, B, F));
    return SNN_OK;
}

snn_status snn_scan_forward(const snn_scan_cfg* cfg, int64_t T, int64_t B, int64_t F, const snn_seq* x,
                            const snn_seq* dt, const float* A, const snn_seq* Bm, const snn_seq* Cm, const float* D,
                            const float* dt_bias, const float* h_in, const int32_t* lengths, const snn_seq* y,
                            float* h_out, void* saved, void* workspace, void* stream) {
    ScanPlan plan;
    snn_status st = check_scan(cfg, T, B, F, plan);
    if (st != SNN_OK || empty(T, B, F)) return st;
    st = first_error({check_scan_inputs(cfg, T, B, F, x, dt, A, Bm, Cm, D, dt_bias, h_in, lengths),
                      check_out(y, T, B, F, cfg->io), optional(h_out), optional(saved),
                      check_workspace(workspace, scan_forward_workspace(cfg, plan, B, F))});
    if (st != SNN_OK) return st;
    ScanArgs a = scan_args(cfg, plan, T, B, F, x, dt, A, Bm, Cm, D, dt_bias, h_in, lengths);
    a.y = rows(y);
    a.h_out = h_out;
    a.saved = static_cast<float*>(saved);
    a.walk = scan_walks(a.plan, h_in, h_out);
    if (a.plan.segments > 1) {
        int64_t at = 0;
        a.part_h = carve<float>(workspace, at, scan_part_h(cfg, a.plan, B, F));
        a.part_d = carve<float>(workspace, at, scan_part_d(a.plan, B, F));
        if ((st = scan_split_entry(cfg->io, false, a, stream_of(stream))) != SNN_OK) return st;
    }
    return scan_forward_entry(cfg->io, a, stream_of(stream));
}

snn_status snn_scan_backward(const snn_scan_cfg* cfg, int64_t T, int64_t B, int64_t F, const snn_seq* x,
                             const snn_seq* dt, const float* A, const snn_seq* Bm, const snn_seq* Cm, const float* D,
                             const float* dt_bias, const float* h_in, const int32_t* lengths, const void* saved,
                             const snn_seq* grad_y, const float* grad_h_out, const snn_seq* grad_x,
                             const snn_seq* grad_dt, float* grad_A, const snn_seq* grad_Bm, const snn_seq* grad_Cm,
                             float* grad_D, float* grad_dt_bias, float* grad_h_in, void* workspace, void* stream) {
    ScanPlan plan;
    snn_status st = check_scan(cfg, T, B, F, plan);
    if (st != SNN_OK || empty(T, B, F)) return st;
    const int io = cfg->io;
    const int64_t gs = int64_t(cfg->groups) * cfg->states;
    st = first_error({check_scan_inputs(cfg, T, B, F, x, dt, A, Bm, Cm, D, dt_bias, h_in, lengths),
                      scan_saved(cfg, plan, T, B, F) > 0 ? need(saved) : optional(saved), check_in(grad_y, T, B, F, io),
                      optional(grad_h_out), check_out(grad_x, T, B, F, io), check_out(grad_dt, T, B, F, io),
                      need(grad_A), check_out(grad_Bm, T, B, gs, io), check_out(grad_Cm, T, B, gs, io),
                      optional(grad_D), optional(grad_dt_bias), optional(grad_h_in),
                      check_workspace(workspace, scan_backward_workspace(cfg, plan, T, B, F))});
    if (st != SNN_OK) return st;
    ScanArgs a = scan_args(cfg, plan, T, B, F, x, dt, A, Bm, Cm, D, dt_bias, h_in, lengths);
    a.saved = static_cast<float*>(const_cast<void*>(saved));
    a.gy = rows(grad_y);
    a.gh_out = grad_h_out;
    a.gx = rows(grad_x);
    a.gdt = rows(grad_dt);
    a.gA = grad_A;
    a.gB = rows(grad_Bm);
    a.gC = rows(grad_Cm);
    a.gD = grad_D;
    a.gdt_bias = grad_dt_bias;
    a.gh_in = grad_h_in;
    a.walk = scan_walks(a.plan, grad_h_out, grad_h_in);
    int64_t at = 0;
    a.part_h = carve<float>(workspace, at, scan_part_h(cfg, a.plan, B, F));
    a.part_d = carve<float>(workspace, at, scan_part_d(a.plan, B, F));
    a.part_bc = carve<float>(workspace, at, scan_partial_bc(cfg, a.plan, T, B));
    a.part_f = carve<float>(workspace, at, a.plan.segments * B * scan_partial_values(F, cfg->states) * 4);
    if (a.plan.segments > 1 && (st = scan_split_entry(io, true, a, stream_of(stream))) != SNN_OK) return st;
    return scan_backward_entry(io, a, stream_of(stream));
}

snn_status snn_norm_forward(const snn_norm_cfg* cfg, int64_t T, int64_t B, int64_t F, const snn_seq* y,
                            const snn_seq* z, const snn_seq* r, const float* w_post, const float* scale,
                            const float* w_pre, const int32_t* lengths, const snn_seq* r_new, const snn_seq* u,
                            float* rstd, void* stream) {
    snn_status st = check_norm(cfg, T, B, F);
    if (st != SNN_OK || empty(T, B, F)) return st;
    const int io = cfg->io;
    st = first_error({check_in(y, T, B, F, io), in_or_null(z, T, B, F, io), in_or_null(r, T, B, F, io),
                      optional(w_post), optional(scale), optional(w_pre), optional(lengths),
                      check_out(r_new, T, B, F, io), w_pre != nullptr ? check_out(u, T, B, F, io) : SNN_OK,
                      optional(rstd)});
    if (st != SNN_OK) return st;
    NormArgs a = norm_args(cfg, T, B, F, y, z, r, w_post, scale, w_pre, lengths, false);
    a.r_new = rows(r_new);
    a.u = rows(u);
    a.rstd = rstd;
    return norm_forward_entry(io, a, stream_of(stream));
}

snn_status snn_norm_workspace_bytes(const snn_norm_cfg* cfg, int64_t T, int64_t B, int64_t F, size_t* bytes) {
    const snn_status st = check_norm(cfg, T, B, F);
    if (st != SNN_OK) return st;
    if (bytes == nullptr) return SNN_E_NULL;
    *bytes = empty(T, B, F) ? 0 : size_t(norm_workspace(T, B, F));
    return SNN_OK;
}

snn_status snn_norm_backward(const snn_norm_cfg* cfg, int64_t T, int64_t B, int64_t F, const snn_seq* y,
                             const snn_seq* z, const snn_seq* r, const float* w_post, const float* scale,
                             const float* w_pre, const int32_t* lengths, const float* rstd, const snn_seq* grad_r_new,
                             const snn_seq* grad_u, const snn_seq* grad_y, const snn_seq* grad_z,
                             const snn_seq* grad_r, float* grad_w_post, float* grad_scale, float* grad_w_pre,
                             void* workspace, void* stream) {
    snn_status st = check_norm(cfg, T, B, F);
    if (st != SNN_OK || empty(T, B, F)) return st;
    const int io = cfg->io;
    st = first_error({check_in(y, T, B, F, io), in_or_null(z, T, B, F, io), in_or_null(r, T, B, F, io),
                      optional(w_post), optional(scale), optional(w_pre), optional(lengths),
                      w_post != nullptr || w_pre != nullptr ? need(rstd) : SNN_OK, in_or_null(grad_r_new, T, B, F, io),
                      in_or_null(grad_u, T, B, F, io), check_out(grad_y, T, B, F, io),
                      z != nullptr ? check_out(grad_z, T, B, F, io) : SNN_OK,
                      r != nullptr ? check_out(grad_r, T, B, F, io) : SNN_OK,
                      w_post != nullptr ? need(grad_w_post) : SNN_OK, scale != nullptr ? need(grad_scale) : SNN_OK,
                      w_pre != nullptr ? need(grad_w_pre) : SNN_OK, need(workspace, 16)});
    if (st != SNN_OK) return st;
    NormArgs a = norm_args(cfg, T, B, F, y, z, r, w_post, scale, w_pre, lengths, true);
    a.rstd_in = rstd;
    a.gr_new = rows(grad_r_new);
    a.gu = rows(grad_u);
    a.gy = rows(grad_y);
    a.gz = rows(grad_z);
    a.gr = rows(grad_r);
    a.gw_post = w_post != nullptr ? grad_w_post : nullptr;
    a.gscale = scale != nullptr ? grad_scale : nullptr;
    a.gw_pre = w_pre != nullptr ? grad_w_pre : nullptr;
    a.part = static_cast<float*>(workspace);
    return norm_backward_entry(io, a, stream_of(stream));
}

}  // extern "C"
