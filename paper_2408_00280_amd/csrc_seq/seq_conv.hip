// Short causal convolution along time, forward and backward.
//
// A lane owns V neighbouring features (8 or 16 bytes of a row) of one sequence and walks a chunk
// of its steps with the last W-1 inputs in registers, so each input is read once, but for
// W-1 rows at a chunk's start.  The backward walks W-1 steps past its chunk: dL/dx[s] needs
// dL/du of steps s to s+W-1, whose activation it recomputes from x.  Sums over steps for the
// filter's gradient stay in registers per chunk and are then added up by a second kernel.
// The next rows are loaded while these are computed.  Bound by memory.
#include "seq_device.h"

namespace snnlif {
namespace {

struct ConvLane {
    int64_t f, b, c;
    bool vec;    // whole vector, or one feature of those left over
};

template <int V>
__device__ __forceinline__ ConvLane conv_lane(const ConvArgs& a, bool& any) {
    const int64_t i = int64_t(blockIdx.x) * kBlock + threadIdx.x, n = a.plan.lanes, nv = a.F / V;
    any = i < n * a.B * a.plan.chunks;
    const int64_t q = i / n, j = i - q * n;
    ConvLane l;
    l.vec = j < nv;
    l.f = l.vec ? j * V : nv * V + (j - nv);
    l.c = q / a.B;
    l.b = q - l.c * a.B;
    return l;
}

// Input row t (t >= -(W-1)) of features f .. f+V-1: x, the state before step 0, or 0.
template <int IO, int W, int V>
__device__ __forceinline__ void conv_input(const ConvArgs& a, int64_t t, int64_t b, int64_t f, float (&v)[V]) {
    if (t >= 0) return load_vec<IO, V>(at<IO>(a.x, t, b, f), v);
    if (a.state_in != nullptr) {
        const Rows st = {a.state_in, a.B * a.F, a.F};
        return load_vec<IO, V>(at<IO>(st, t + (W - 1), b, f), v);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = 0.0f;
}

template <int W, int V>
__device__ __forceinline__ void load_filter(const ConvArgs& a, int64_t f, float (&w)[V][W], float (&bias)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
        bias[j] = a.bias != nullptr ? a.bias[f + j] : 0.0f;
#pragma unroll
        for (int k = 0; k < W; ++k) w[j][k] = a.weight[(f + j) * W + k];
    }
}

// The last W-1 inputs of a sequence of `len` steps.  All are read before the first is
// written, so that the state may be updated in place.
template <int IO, int W, int V>
__device__ void conv_state(const ConvArgs& a, int64_t len, int64_t b, int64_t f) {
    float v[W][V];
#pragma unroll
    for (int i = 0; i < W - 1; ++i) conv_input<IO, W, V>(a, len - (W - 1) + i, b, f, v[i]);
#pragma unroll
    for (int i = 0; i < W - 1; ++i)
        IoVec<IO, V>::store(a.state_out, (i * a.B + b) * a.F + f, v[i]);
}

__host__ __device__ bool conv_state_later(const ConvArgs& a) {
    return a.plan.chunks > 1 && a.state_out == a.state_in;
}

// A lane's column of a [T][B][F] tensor, V features wide.
template <int IO, int V>
struct WideColumn {
    static constexpr int kBytes = IO == SNN_IO_F32 ? 4 : 2;
    char* p;         // row 0
    int64_t step;    // bytes
    __device__ WideColumn(const Rows& r, const ConvLane& l)
        : p(static_cast<char*>(at_out<IO>(r, 0, l.b, l.f))), step(r.t * kBytes) {}
    __device__ auto load(int64_t t) const { return IoVec<IO, V>::load(p + t * step, 0); }
    __device__ void store(int64_t t, const float (&v)[V]) const { IoVec<IO, V>::store(p + t * step, 0, v); }
};

// Rows t .. t+U-1 below `stop`, without a branch per row where all of them are.
template <int U, typename Col, typename Raw>
__device__ __forceinline__ void load_rows_ahead(const Col& c, int64_t t, int64_t stop, Raw (&raw)[U]) {
    if (t + U <= stop) {
#pragma unroll
        for (int k = 0; k < U; ++k) raw[k] = c.load(t + k);
    } else {
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (t + k < stop) raw[k] = c.load(t + k);
    }
}

template <int IO, int W, int ACT, int V>
__device__ void conv_forward_walk(const ConvArgs& a, const ConvLane& l) {
    constexpr int U = conv_rows(false);     // rows in flight
    float w[V][W], bias[V], hist[W][V];
    load_filter<W, V>(a, l.f, w, bias);
    const int64_t len = steps_of(a.lengths, l.b, a.T), t0 = l.c * a.plan.steps;
    const int64_t end = min(a.T, t0 + a.plan.steps), stop = min(end, len);
    const WideColumn<IO, V> cx(a.x, l), cy(a.y, l);
    if (t0 < stop) {
#pragma unroll
        for (int i = 0; i < W - 1; ++i) conv_input<IO, W, V>(a, t0 - (W - 1) + i, l.b, l.f, hist[i]);
    }
    typename IoVec<IO, V>::raw raw[U], ahead[U];
    const auto row = [&](int64_t t, const typename IoVec<IO, V>::raw& x) {
        float u[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            hist[W - 1][j] = IoVec<IO, V>::get(x, j);
            u[j] = bias[j];
#pragma unroll
            for (int i = 0; i < W; ++i) u[j] = fmaf(w[j][i], hist[i][j], u[j]);
#pragma unroll
            for (int i = 0; i < W - 1; ++i) hist[i][j] = hist[i + 1][j];
            if (ACT == SNN_ACT_SILU) u[j] *= sigmoid(u[j]);
        }
        cy.store(t, u);
    };
    load_rows_ahead<U>(cx, t0, stop, ahead);
    for (int64_t t = t0; t < stop; t += U) {
#pragma unroll
        for (int k = 0; k < U; ++k) raw[k] = ahead[k];
        load_rows_ahead<U>(cx, t + U, stop, ahead);
        if (t + U <= stop) {
#pragma unroll
            for (int k = 0; k < U; ++k) row(t + k, raw[k]);
        } else {
#pragma unroll
            for (int k = 0; k < U; ++k)
                if (t + k < stop) row(t + k, raw[k]);
        }
    }
    float zero[V] = {};
    for (int64_t t = max(t0, stop); t < end; ++t) IoVec<IO, V>::store(at_out<IO>(a.y, t, l.b, l.f), 0, zero);
    // The chunk with the sequence's last step leaves the state.  In place that is safe for one
    // chunk only, whose lane alone reads and writes its features' state.
    const bool own = t0 < max(len, int64_t(1)) && len <= end;
    if (a.state_out != nullptr && own && !conv_state_later(a)) conv_state<IO, W, V>(a, len, l.b, l.f);
}

template <int IO, int W, int ACT>
__global__ __launch_bounds__(kBlock) void conv_forward_kernel(ConvArgs a) {
    constexpr int V = conv_vec(IO, false);
    bool any;
    const ConvLane l = conv_lane<V>(a, any);
    if (!any) return;
    if (l.vec) conv_forward_walk<IO, W, ACT, V>(a, l);
    else conv_forward_walk<IO, W, ACT, 1>(a, l);
}

// The state in place behind several chunks, once all of them have read the one before.
template <int IO, int W>
__global__ __launch_bounds__(kBlock) void conv_state_kernel(ConvArgs a) {
    constexpr int V = conv_vec(IO, false);
    bool any;
    const ConvLane l = conv_lane<V>(a, any);
    if (!any || l.c != 0) return;
    const int64_t len = steps_of(a.lengths, l.b, a.T);
    if (l.vec) conv_state<IO, W, V>(a, len, l.b, l.f);
    else conv_state<IO, W, 1>(a, len, l.b, l.f);
}

template <int IO, int W, int ACT, int V>
__device__ void conv_backward_walk(const ConvArgs& a, const ConvLane& l) {
    constexpr int U = conv_rows(true);
    float w[V][W], bias[V], hist[W][V], gu[W][V], gw[V][W], gb[V];
    load_filter<W, V>(a, l.f, w, bias);
    const int64_t len = steps_of(a.lengths, l.b, a.T), t0 = l.c * a.plan.steps;
    const int64_t end = min(a.T, t0 + a.plan.steps), stop = min(end, len);
    const Rows gso = {a.gstate_out, a.B * a.F, a.F}, gsi = {a.gstate_in, a.B * a.F, a.F};
#pragma unroll
    for (int j = 0; j < V; ++j) {
        gb[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < W; ++i) gw[j][i] = gu[i][j] = 0.0f;
    }
    // dL/dx[s] from gu[i] = dL/du[s + i], and the state's gradient where input s is part of it
    const auto grad_x = [&](float (&g)[V]) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            g[j] = 0.0f;
#pragma unroll
            for (int i = 0; i < W; ++i) g[j] = fmaf(w[j][W - 1 - i], gu[i][j], g[j]);
        }
    };
    const auto emit = [&](int64_t s) {
        float g[V];
        grad_x(g);
        const int64_t i = s - (len - (W - 1));
        if (a.gstate_out != nullptr && i >= 0 && i < W - 1) {
            float e[V];
            load_vec<IO, V>(at<IO>(gso, i, l.b, l.f), e);
#pragma unroll
            for (int j = 0; j < V; ++j) g[j] += e[j];
        }
        if (s >= 0) IoVec<IO, V>::store(at_out<IO>(a.gx, s, l.b, l.f), 0, g);
        else if (a.gstate_in != nullptr) IoVec<IO, V>::store(at_out<IO>(gsi, s + (W - 1), l.b, l.f), 0, g);
    };
    const auto push = [&](const float (&g)[V]) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
#pragma unroll
            for (int i = 0; i < W - 1; ++i) gu[i][j] = gu[i + 1][j];
            gu[W - 1][j] = g[j];
        }
    };
    if (t0 < len || t0 == 0) {
        const int64_t past = min(len, end + (W - 1));   // steps whose dL/du this chunk needs
#pragma unroll
        for (int i = 0; i < W - 1; ++i) conv_input<IO, W, V>(a, t0 - (W - 1) + i, l.b, l.f, hist[i]);
        typename IoVec<IO, V>::raw xr[U], gr[U], xa[U], ga[U];
        const WideColumn<IO, V> cx(a.x, l), cgy(a.gy, l), cgx(a.gx, l);
        // inner rows: every step of the batch is the chunk's own, and so is the input W-1 steps
        // before, which is part of no state
        const auto row = [&](auto inner, int64_t t, const typename IoVec<IO, V>::raw& x, const typename IoVec<IO, V>::raw& gy) {
            float g[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                hist[W - 1][j] = IoVec<IO, V>::get(x, j);
                float u = bias[j];
#pragma unroll
                for (int i = 0; i < W; ++i) u = fmaf(w[j][i], hist[i][j], u);
                g[j] = IoVec<IO, V>::get(gy, j);
                if (ACT == SNN_ACT_SILU) g[j] *= silu_slope(u, sigmoid(u));
                if (inner.value || t < stop) {       // steps past the chunk are another's
                    gb[j] += g[j];
#pragma unroll
                    for (int i = 0; i < W; ++i) gw[j][i] = fmaf(g[j], hist[i][j], gw[j][i]);
                }
#pragma unroll
                for (int i = 0; i < W - 1; ++i) hist[i][j] = hist[i + 1][j];
            }
            push(g);
            const int64_t s = t - (W - 1);
            if constexpr (inner.value) {
                float gx[V];
                grad_x(gx);
                cgx.store(s, gx);
            } else {
                if (s >= t0 || t0 == 0) emit(s);
            }
        };
        load_rows_ahead<U>(cx, t0, past, xa);
        load_rows_ahead<U>(cgy, t0, past, ga);
        for (int64_t t = t0; t < past; t += U) {
#pragma unroll
            for (int k = 0; k < U; ++k) {
                xr[k] = xa[k];
                gr[k] = ga[k];
            }
            load_rows_ahead<U>(cx, t + U, past, xa);
            load_rows_ahead<U>(cgy, t + U, past, ga);
            if (t >= t0 + (W - 1) && t + U <= stop) {
#pragma unroll
                for (int k = 0; k < U; ++k) row(std::true_type{}, t + k, xr[k], gr[k]);
            } else {
#pragma unroll
                for (int k = 0; k < U; ++k)
                    if (t + k < past) row(std::false_type{}, t + k, xr[k], gr[k]);
            }
        }
        // the steps after the sequence's last have no gradient
        const float zero[V] = {};
        for (int64_t t = max(past, t0); t < stop + (W - 1); ++t) {
            push(zero);
            const int64_t s = t - (W - 1);
            if (s >= t0 || t0 == 0) emit(s);
        }
    }
    const float zero[V] = {};
    for (int64_t t = max(t0, stop); t < end; ++t) IoVec<IO, V>::store(at_out<IO>(a.gx, t, l.b, l.f), 0, zero);
    float* part = a.part + (l.c * a.B + l.b) * (a.F * (W + 1));
#pragma unroll
    for (int j = 0; j < V; ++j) {
#pragma unroll
        for (int i = 0; i < W; ++i) part[(l.f + j) * W + i] = gw[j][i];
        part[a.F * W + l.f + j] = gb[j];
    }
}

template <int IO, int W, int ACT>
__global__ __launch_bounds__(kBlock) void conv_backward_kernel(ConvArgs a) {
    constexpr int V = conv_vec(IO, true);
    bool any;
    const ConvLane l = conv_lane<V>(a, any);
    if (!any) return;
    if (l.vec) conv_backward_walk<IO, W, ACT, V>(a, l);
    else conv_backward_walk<IO, W, ACT, 1>(a, l);
}

template <int IO, int W>
snn_status conv_forward_w(int act, const ConvArgs& a, hipStream_t s) {
    const dim3 grid = grid_for(a.plan.lanes * a.B * a.plan.chunks);
    const snn_status st = act == SNN_ACT_SILU ? launch(conv_forward_kernel<IO, W, SNN_ACT_SILU>, grid, s, a)
                                              : launch(conv_forward_kernel<IO, W, SNN_ACT_NONE>, grid, s, a);
    if (st != SNN_OK || a.state_out == nullptr || W == 1 || !conv_state_later(a)) return st;
    return launch(conv_state_kernel<IO, W>, grid_for(a.plan.lanes * a.B), s, a);
}

template <int IO, int W>
snn_status conv_backward_w(int act, const ConvArgs& a, hipStream_t s) {
    const dim3 grid = grid_for(a.plan.lanes * a.B * a.plan.chunks);
    return act == SNN_ACT_SILU ? launch(conv_backward_kernel<IO, W, SNN_ACT_SILU>, grid, s, a)
                               : launch(conv_backward_kernel<IO, W, SNN_ACT_NONE>, grid, s, a);
}

template <int W = 1, typename F>
snn_status with_width(int w, F f) {
    if constexpr (W < kMaxTaps) {
        if (w != W) return with_width<W + 1>(w, f);
    }
    return f(IntC<W>{});
}

}  // namespace

snn_status conv_forward_entry(const snn_conv_cfg* c, const ConvArgs& a, hipStream_t s) {
    return with_width(c->width, [&](auto w) {
        return c->io == SNN_IO_F32 ? conv_forward_w<SNN_IO_F32, decltype(w)::value>(c->act, a, s)
                                   : conv_forward_w<SNN_IO_BF16, decltype(w)::value>(c->act, a, s);
    });
}

snn_status conv_backward_entry(const snn_conv_cfg* c, const ConvArgs& a, hipStream_t s) {
    return with_width(c->width, [&](auto w) {
        return c->io == SNN_IO_F32 ? conv_backward_w<SNN_IO_F32, decltype(w)::value>(c->act, a, s)
                                   : conv_backward_w<SNN_IO_BF16, decltype(w)::value>(c->act, a, s);
    });
}

}  // namespace snnlif
