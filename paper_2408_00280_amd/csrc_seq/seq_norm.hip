// A block's gate, norm and scaled residual with the next block's norm, forward and backward,
// and the sums of partial results over workgroups.
//
// Rows of up to 8192 features are read once: a lane holds 8 of a row's features (16 bytes of
// bf16, two pieces of 16 bytes of fp32) and their parameters, a workgroup's lanes one row, and
// the workgroup walks rows with the next one's loads in flight.  A row costs two sums over the
// workgroup per direction, and more than one workgroup per CU hides them.  Longer rows are
// walked in pieces and read again for each sum.  Bound by memory.
#include "seq_device.h"

namespace snnlif {
namespace {

// -- Rows in registers ---------------------------------------------------------------------

// The features of a row that a lane holds: N pieces of V, of which the last may be cut off by
// the row's end.
template <int IO>
struct Lane8 {
    static constexpr int V = IO == SNN_IO_F32 ? 4 : 8, N = kNormLane / V;
    using raw = typename IoVec<IO, V>::raw;
    struct Raw {
        raw v[N];
    };
    int f[N], n[N];     // first feature and how many
    __device__ explicit Lane8(int64_t F, int first = 0) {
#pragma unroll
        for (int c = 0; c < N; ++c) {
            f[c] = first + int(c * blockDim.x + threadIdx.x) * V;
            n[c] = max(0, min(V, int(F) - f[c]));
        }
    }
    __device__ void load(const Rows& r, int64_t t, int64_t b, Raw& out) const {
#pragma unroll
        for (int c = 0; c < N; ++c) {
            if (n[c] == V) {
                out.v[c] = IoVec<IO, V>::load(at<IO>(r, t, b, f[c]), 0);
            } else {
                uint32_t w[4] = {};
#pragma unroll
                for (int j = 0; j < V - 1; ++j) {
                    if (j < n[c]) {
                        if constexpr (IO == SNN_IO_F32) w[j] = __float_as_uint(load1<IO>(at<IO>(r, t, b, f[c] + j)));
                        else w[j >> 1] |= (__float_as_uint(load1<IO>(at<IO>(r, t, b, f[c] + j))) >> 16) << (16 * (j & 1));
                    }
                }
                const u32x4_t u = {w[0], w[1], w[2], w[3]};
                out.v[c] = __builtin_bit_cast(raw, u);
            }
        }
    }
    __device__ void load(const Rows& r, int64_t t, int64_t b, float (&v)[kNormLane]) const {
        Raw raw;
        load(r, t, b, raw);
        get(raw, v);
    }
    __device__ void get(const Raw& r, float (&v)[kNormLane]) const {
#pragma unroll
        for (int i = 0; i < kNormLane; ++i) v[i] = IoVec<IO, V>::get(r.v[i / V], i % V);
    }
    __device__ void store(const Rows& r, int64_t t, int64_t b, const float (&v)[kNormLane]) const {
#pragma unroll
        for (int c = 0; c < N; ++c) {
            if (n[c] == V) {
                float p[V];
#pragma unroll
                for (int j = 0; j < V; ++j) p[j] = v[c * V + j];
                IoVec<IO, V>::store(at_out<IO>(r, t, b, f[c]), 0, p);
            } else {
#pragma unroll
                for (int j = 0; j < V - 1; ++j)
                    if (j < n[c]) store1<IO>(at_out<IO>(r, t, b, f[c] + j), v[c * V + j]);
            }
        }
    }
    // Parameters: `other` where there are none, 0 behind the row's end.
    __device__ void params(const float* p, float other, float (&v)[kNormLane]) const {
#pragma unroll
        for (int c = 0; c < N; ++c) {
            if (p != nullptr && n[c] == V) {
#pragma unroll
                for (int j = 0; j < V; j += 4) {
                    typedef f32x4_t vec __attribute__((aligned(4)));
                    const f32x4_t w = *reinterpret_cast<const vec*>(p + f[c] + j);
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[c * V + j + i] = w[i];
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) v[c * V + j] = j < n[c] ? (p != nullptr ? p[f[c] + j] : other) : 0.0f;
            }
        }
    }
    // p += x y, of partial sums that this workgroup alone holds.
    __device__ void add(float* p, const float (&x)[kNormLane], const float (&y)[kNormLane]) const {
        float v[kNormLane];
        params(p, 0.0f, v);
#pragma unroll
        for (int i = 0; i < kNormLane; ++i) v[i] = fmaf(x[i], y[i], v[i]);
        put(p, v);
    }
    __device__ void put(float* p, const float (&v)[kNormLane]) const {
#pragma unroll
        for (int i = 0; i < kNormLane; ++i)
            if (i % V < n[i / V]) p[f[i / V] + i % V] = v[i];
    }
};

// Sum over the workgroup, in every lane.  Consecutive sums use the two slots in turn, so that
// one barrier each is enough.
struct RowSum {
    float (*lds)[16];
    int slot = 0;
    __device__ float operator()(float v) {
        v = wave_sum(v);
        const int waves = blockDim.x / kWave;
        if (waves == 1) return v;
        if ((threadIdx.x & (kWave - 1)) == 0) lds[slot][threadIdx.x / kWave] = v;
        lds_barrier();
        float s = 0.0f;
        for (int w = 0; w < waves; ++w) s += lds[slot][w];
        slot ^= 1;
        return s;
    }
};

template <int IO, int MAXT>
__global__ __launch_bounds__(MAXT) void norm_forward_kernel(NormArgs a) {
    __shared__ float lds[2][16];
    using L = Lane8<IO>;
    const L lane(a.F);
    RowSum sum{lds};
    float w_post[kNormLane], scale[kNormLane], w_pre[kNormLane];
    lane.params(a.w_post, 1.0f, w_post);
    lane.params(a.scale, 1.0f, scale);
    lane.params(a.w_pre, 0.0f, w_pre);
    const float mean = 1.0f / float(a.F);
    const int rows = int(a.T * a.B), B = int(a.B);
    typename L::Raw y, z, r;
    const auto fetch = [&](int i) {
        if (i >= rows) return;
        const int t = i / B, b = i - t * B;
        if (t >= steps_of(a.lengths, b, a.T)) return;
        lane.load(a.y, t, b, y);
        if (a.z.p != nullptr) lane.load(a.z, t, b, z);
        if (a.r.p != nullptr) lane.load(a.r, t, b, r);
    };
    fetch(blockIdx.x);
    for (int i = blockIdx.x; i < rows; i += int(a.groups)) {
        const int t = i / B, b = i - t * B;
        float g[kNormLane], v[kNormLane];
        if (t >= steps_of(a.lengths, b, a.T)) {
            fetch(i + int(a.groups));
#pragma unroll
            for (int j = 0; j < kNormLane; ++j) g[j] = 0.0f;
            lane.store(a.r_new, t, b, g);
            if (a.w_pre != nullptr) lane.store(a.u, t, b, g);
            continue;
        }
        lane.get(y, g);
        if (a.z.p != nullptr) {
            lane.get(z, v);
#pragma unroll
            for (int j = 0; j < kNormLane; ++j) g[j] *= v[j] * sigmoid(v[j]);
        }
        if (a.r.p != nullptr) {
            lane.get(r, v);
        } else {
#pragma unroll
            for (int j = 0; j < kNormLane; ++j) v[j] = 0.0f;
        }
        fetch(i + int(a.groups));
        float k1 = 1.0f, k2 = 0.0f, s = 0.0f;
        if (a.w_post != nullptr) {
#pragma unroll
            for (int j = 0; j < kNormLane; ++j) s = fmaf(g[j], g[j], s);
            k1 = 1.0f / sqrtf(fmaf(sum(s), mean, a.eps));
            s = 0.0f;
        }
#pragma unroll
        for (int j = 0; j < kNormLane; ++j) {
            v[j] = fmaf(scale[j], g[j] * k1 * w_post[j], v[j]);
            s = fmaf(v[j], v[j], s);
        }
        lane.store(a.r_new, t, b, v);
        if (a.w_pre != nullptr) {
            k2 = 1.0f / sqrtf(fmaf(sum(s), mean, a.eps));
#pragma unroll
            for (int j = 0; j < kNormLane; ++j) v[j] *= k2 * w_pre[j];
            lane.store(a.u, t, b, v);
        }
        if (a.rstd != nullptr && threadIdx.x == 0) {
            a.rstd[i] = k1;
            a.rstd[rows + i] = k2;
        }
    }
}

template <int IO, int MAXT>
__global__ __launch_bounds__(MAXT) void norm_backward_kernel(NormArgs a) {
    __shared__ float lds[2][16];
    using L = Lane8<IO>;
    const L lane(a.F);
    RowSum sum{lds};
    float w_post[kNormLane], scale[kNormLane], w_pre[kNormLane];
    float g_post[kNormLane], g_scale[kNormLane], g_pre[kNormLane];
    lane.params(a.w_post, 1.0f, w_post);
    lane.params(a.scale, 1.0f, scale);
    lane.params(a.w_pre, 0.0f, w_pre);
    // 16 waves of one workgroup have no registers for the next row's loads and the sums: those
    // are in LDS then, each lane's own, and some 90 registers are spilled all the same
    // (x[1024][8][8192] bf16: 290 us, 383 with the sums and loads among them)
    constexpr bool kAhead = MAXT < 1024;
    __shared__ f32x4_t sums[kAhead ? 1 : 6][kAhead ? 1 : MAXT];
    const auto open = [&](int k, float (&g)[kNormLane]) {
        if (kAhead) return;
        const f32x4_t x = sums[2 * k][threadIdx.x], y = sums[2 * k + 1][threadIdx.x];
#pragma unroll
        for (int j = 0; j < kNormLane; ++j) g[j] = j < 4 ? x[j & 3] : y[j & 3];
    };
    const auto close = [&](int k, const float (&g)[kNormLane]) {
        if (kAhead) return;
        sums[2 * k][threadIdx.x] = {g[0], g[1], g[2], g[3]};
        sums[2 * k + 1][threadIdx.x] = {g[4], g[5], g[6], g[7]};
    };
#pragma unroll
    for (int j = 0; j < kNormLane; ++j) g_post[j] = g_scale[j] = g_pre[j] = 0.0f;
    close(0, g_post);
    close(1, g_scale);
    close(2, g_pre);
    const float mean = 1.0f / float(a.F);
    const int rows = int(a.T * a.B), B = int(a.B);
    const bool pre = a.w_pre != nullptr && a.gu.p != nullptr;
    struct Row {
        typename L::Raw y, z, r, gr, gu;
        float k1, k2;
    } row;
    const auto fetch = [&](int i) {
        if (i >= rows) return;
        const int t = i / B, b = i - t * B;
        if (t >= steps_of(a.lengths, b, a.T)) return;
        lane.load(a.y, t, b, row.y);
        if (a.z.p != nullptr) lane.load(a.z, t, b, row.z);
        if (a.gr_new.p != nullptr) lane.load(a.gr_new, t, b, row.gr);
        if (pre) {
            if (a.r.p != nullptr) lane.load(a.r, t, b, row.r);
            lane.load(a.gu, t, b, row.gu);
            row.k2 = a.rstd_in[rows + i];
        }
        if (a.w_post != nullptr) row.k1 = a.rstd_in[i];
    };
    if (kAhead) fetch(blockIdx.x);
    for (int i = blockIdx.x; i < rows; i += int(a.groups)) {
        const int t = i / B, b = i - t * B;
        if (t >= steps_of(a.lengths, b, a.T)) {
            if (kAhead) fetch(i + int(a.groups));
            const float zero[kNormLane] = {};
            lane.store(a.gy, t, b, zero);
            if (a.z.p != nullptr) lane.store(a.gz, t, b, zero);
            if (a.r.p != nullptr) lane.store(a.gr, t, b, zero);
            continue;
        }
        if (!kAhead) fetch(i);
        const Row now = row;
        if (kAhead) fetch(i + int(a.groups));
        const float k1 = a.w_post != nullptr ? now.k1 : 1.0f, k2 = pre ? now.k2 : 0.0f;
        float y[kNormLane], z[kNormLane], gn[kNormLane], gr[kNormLane], s = 0.0f;
        lane.get(now.y, y);
        if (a.z.p != nullptr) lane.get(now.z, z);
#pragma unroll
        for (int j = 0; j < kNormLane; ++j) gn[j] = y[j] * k1;
        if (a.z.p != nullptr) {
#pragma unroll
            for (int j = 0; j < kNormLane; ++j) gn[j] *= z[j] * sigmoid(z[j]);
        }
        if (a.gr_new.p != nullptr) {
            lane.get(now.gr, gr);
        } else {
#pragma unroll
            for (int j = 0; j < kNormLane; ++j) gr[j] = 0.0f;
        }
        if (pre) {
            float rn[kNormLane], gu[kNormLane];
            lane.get(now.gu, gu);
            if (a.r.p != nullptr) {
                lane.get(now.r, rn);
            } else {
#pragma unroll
                for (int j = 0; j < kNormLane; ++j) rn[j] = 0.0f;
            }
#pragma unroll
            for (int j = 0; j < kNormLane; ++j) rn[j] = k2 * fmaf(scale[j], gn[j] * w_post[j], rn[j]);
            open(2, g_pre);
#pragma unroll
            for (int j = 0; j < kNormLane; ++j) {
                g_pre[j] = fmaf(gu[j], rn[j], g_pre[j]);
                gu[j] *= w_pre[j];
                s = fmaf(gu[j], rn[j], s);
            }
            close(2, g_pre);
            const float m = sum(s) * mean;
#pragma unroll
            for (int j = 0; j < kNormLane; ++j) gr[j] = fmaf(k2, fmaf(-m, rn[j], gu[j]), gr[j]);
            s = 0.0f;
        }
        if (a.r.p != nullptr) lane.store(a.gr, t, b, gr);
        open(1, g_scale);
#pragma unroll
        for (int j = 0; j < kNormLane; ++j) {
            g_scale[j] = fmaf(gr[j], gn[j] * w_post[j], g_scale[j]);
            gr[j] *= scale[j];                                     // dL/dn
        }
        close(1, g_scale);
        open(0, g_post);
#pragma unroll
        for (int j = 0; j < kNormLane; ++j) {
            g_post[j] = fmaf(gr[j], gn[j], g_post[j]);
            gr[j] *= w_post[j];
        }
        close(0, g_post);
        if (a.w_post != nullptr) {
#pragma unroll
            for (int j = 0; j < kNormLane; ++j) s = fmaf(gr[j], gn[j], s);
            const float m = sum(s) * mean;
#pragma unroll
            for (int j = 0; j < kNormLane; ++j) gr[j] = k1 * fmaf(-m, gn[j], gr[j]);   // dL/dg
        }
        if (a.z.p != nullptr) {
#pragma unroll
            for (int j = 0; j < kNormLane; ++j) {
                const float q = sigmoid(z[j]);
                y[j] *= gr[j] * silu_slope(z[j], q);
                gr[j] *= z[j] * q;
            }
            lane.store(a.gz, t, b, y);
        }
        lane.store(a.gy, t, b, gr);
    }
    float* part = a.part + int64_t(blockIdx.x) * 3 * a.F;
    open(0, g_post);
    lane.put(part, g_post);
    open(1, g_scale);
    lane.put(part + a.F, g_scale);
    open(2, g_pre);
    lane.put(part + 2 * a.F, g_pre);
}

// -- Longer rows: in pieces of 8192 features, read again for each sum (from the L2, as a rule) --

constexpr int kLongLanes = kNormRegs / kNormLane;

template <int IO>
struct LongRow {
    using L = Lane8<IO>;
    const NormArgs& a;
    int t, b;
    __device__ void gated(const L& lane, float (&g)[kNormLane]) const {
        lane.load(a.y, t, b, g);
        if (a.z.p == nullptr) return;
        float z[kNormLane];
        lane.load(a.z, t, b, z);
#pragma unroll
        for (int j = 0; j < kNormLane; ++j) g[j] *= z[j] * sigmoid(z[j]);
    }
    // r' from g, which becomes g k1 w_post.
    __device__ void residual(const L& lane, float k1, float (&g)[kNormLane], float (&r)[kNormLane]) const {
        float w[kNormLane];
        lane.params(a.w_post, 1.0f, w);
#pragma unroll
        for (int j = 0; j < kNormLane; ++j) {
            g[j] *= k1 * w[j];
            r[j] = 0.0f;
        }
        if (a.r.p != nullptr) lane.load(a.r, t, b, r);
        lane.params(a.scale, 1.0f, w);
#pragma unroll
        for (int j = 0; j < kNormLane; ++j) r[j] = fmaf(w[j], g[j], r[j]);
    }
};

template <int IO>
__global__ __launch_bounds__(kLongLanes) void norm_long_forward_kernel(NormArgs a) {
    __shared__ float lds[2][16];
    using L = Lane8<IO>;
    RowSum sum{lds};
    const int F = int(a.F), rows = int(a.T * a.B), B = int(a.B);
    const float mean = 1.0f / float(a.F);
    for (int i = blockIdx.x; i < rows; i += int(a.groups)) {
        const LongRow<IO> row = {a, i / B, i % B};
        float g[kNormLane], r[kNormLane], w[kNormLane], k1 = 1.0f, k2 = 0.0f, s = 0.0f;
        const bool in = row.t < steps_of(a.lengths, row.b, a.T);
        if (in && a.w_post != nullptr) {
            for (int f = 0; f < F; f += kNormRegs) {
                row.gated(L(F, f), g);
#pragma unroll
                for (int j = 0; j < kNormLane; ++j) s = fmaf(g[j], g[j], s);
            }
            k1 = 1.0f / sqrtf(fmaf(sum(s), mean, a.eps));
        }
        if (in && a.w_pre != nullptr) {
            s = 0.0f;
            for (int f = 0; f < F; f += kNormRegs) {
                const L lane(F, f);
                row.gated(lane, g);
                row.residual(lane, k1, g, r);
#pragma unroll
                for (int j = 0; j < kNormLane; ++j) s = fmaf(r[j], r[j], s);
            }
            k2 = 1.0f / sqrtf(fmaf(sum(s), mean, a.eps));
        }
        for (int f = 0; f < F; f += kNormRegs) {
            const L lane(F, f);
            if (in) {
                row.gated(lane, g);
                row.residual(lane, k1, g, r);
            } else {
#pragma unroll
                for (int j = 0; j < kNormLane; ++j) r[j] = 0.0f;
            }
            lane.store(a.r_new, row.t, row.b, r);
            if (a.w_pre != nullptr) {
                lane.params(a.w_pre, 0.0f, w);
#pragma unroll
                for (int j = 0; j < kNormLane; ++j) r[j] *= k2 * w[j];
                lane.store(a.u, row.t, row.b, r);
            }
        }
        if (in && a.rstd != nullptr && threadIdx.x == 0) {
            a.rstd[i] = k1;
            a.rstd[rows + i] = k2;
        }
    }
}

template <int IO>
__global__ __launch_bounds__(kLongLanes) void norm_long_backward_kernel(NormArgs a) {
    __shared__ float lds[2][16];
    using L = Lane8<IO>;
    RowSum sum{lds};
    const int F = int(a.F), rows = int(a.T * a.B), B = int(a.B);
    const float mean = 1.0f / float(a.F);
    const bool pre = a.w_pre != nullptr && a.gu.p != nullptr;
    float* part = a.part + int64_t(blockIdx.x) * 3 * a.F;      // w_post, scale, w_pre
    const float zero[kNormLane] = {};
    for (int k = 0; k < 3; ++k)
        for (int f = 0; f < F; f += kNormRegs) L(F, f).put(part + k * a.F, zero);
    for (int i = blockIdx.x; i < rows; i += int(a.groups)) {
        const LongRow<IO> row = {a, i / B, i % B};
        const int t = row.t, b = row.b;
        if (t >= steps_of(a.lengths, b, a.T)) {
            for (int f = 0; f < F; f += kNormRegs) {
                const L lane(F, f);
                lane.store(a.gy, t, b, zero);
                if (a.z.p != nullptr) lane.store(a.gz, t, b, zero);
                if (a.r.p != nullptr) lane.store(a.gr, t, b, zero);
            }
            continue;
        }
        const float k1 = a.w_post != nullptr ? a.rstd_in[i] : 1.0f, k2 = pre ? a.rstd_in[rows + i] : 0.0f;
        float n[kNormLane], rn[kNormLane], gu[kNormLane], w[kNormLane], m2 = 0.0f, m1 = 0.0f, s = 0.0f;
        if (pre) {
            for (int f = 0; f < F; f += kNormRegs) {
                const L lane(F, f);
                row.gated(lane, n);
                row.residual(lane, k1, n, rn);
                lane.load(a.gu, t, b, gu);
                lane.params(a.w_pre, 0.0f, w);
#pragma unroll
                for (int j = 0; j < kNormLane; ++j) s = fmaf(gu[j] * w[j], rn[j] * k2, s);
            }
            m2 = sum(s) * mean;
        }
        // dL/dr', and n and r' k2 beside it
        const auto grad_r = [&](const L& lane, float (&gr)[kNormLane]) {
            row.gated(lane, n);
            row.residual(lane, k1, n, rn);
#pragma unroll
            for (int j = 0; j < kNormLane; ++j) gr[j] = 0.0f;
            if (a.gr_new.p != nullptr) lane.load(a.gr_new, t, b, gr);
            if (!pre) return;
            lane.load(a.gu, t, b, gu);
            lane.params(a.w_pre, 0.0f, w);
#pragma unroll
            for (int j = 0; j < kNormLane; ++j) {
                rn[j] *= k2;
                gr[j] = fmaf(k2, fmaf(-m2, rn[j], gu[j] * w[j]), gr[j]);
            }
        };
        float gr[kNormLane];
        if (a.w_post != nullptr) {
            s = 0.0f;
            for (int f = 0; f < F; f += kNormRegs) {
                const L lane(F, f);
                grad_r(lane, gr);
                lane.params(a.scale, 1.0f, w);
#pragma unroll
                for (int j = 0; j < kNormLane; ++j) s = fmaf(gr[j] * w[j], n[j], s);   // n = g k1 w_post
            }
            m1 = sum(s) * mean;
        }
        for (int f = 0; f < F; f += kNormRegs) {
            const L lane(F, f);
            grad_r(lane, gr);
            if (a.r.p != nullptr) lane.store(a.gr, t, b, gr);
            if (pre) lane.add(part + 2 * a.F, gu, rn);
            lane.add(part + a.F, gr, n);
            lane.params(a.scale, 1.0f, w);
            float y[kNormLane], z[kNormLane], gn[kNormLane];
            lane.load(a.y, t, b, y);
            if (a.z.p != nullptr) lane.load(a.z, t, b, z);
#pragma unroll
            for (int j = 0; j < kNormLane; ++j) {
                gr[j] *= w[j];                                     // dL/dn
                gn[j] = y[j] * k1 * (a.z.p != nullptr ? z[j] * sigmoid(z[j]) : 1.0f);
            }
            if (a.w_post != nullptr) {
                lane.add(part, gr, gn);
                lane.params(a.w_post, 1.0f, w);
#pragma unroll
                for (int j = 0; j < kNormLane; ++j) gr[j] = k1 * fmaf(-m1, gn[j], gr[j] * w[j]);   // dL/dg
            }
            if (a.z.p != nullptr) {
#pragma unroll
                for (int j = 0; j < kNormLane; ++j) {
                    const float q = sigmoid(z[j]);
                    y[j] *= gr[j] * silu_slope(z[j], q);
                    gr[j] *= z[j] * q;
                }
                lane.store(a.gz, t, b, y);
            }
            lane.store(a.gy, t, b, gr);
        }
    }
}

template <int V>
__global__ __launch_bounds__(1024) void reduce_kernel(const float* part, int64_t P, int64_t stride, ReduceOut out) {
    __shared__ float lds[1024];
    reduce_partials<V>(part, P, stride, out, blockIdx.x, lds);
}

}  // namespace

snn_status reduce_entry(const float* part, int64_t P, int64_t stride, const ReduceOut& out, hipStream_t s) {
    const int64_t n = out.n[0] + out.n[1] + out.n[2];
    // Many partial results of few values: 16 values per workgroup, so that more CUs read them
    // (4096 of 120 values: 9 us to 16; of 405, 11 to 18; 3200 of 1536, 11 to 12; 2048 of 2040, 9 to
    // 10; 4096 of 4080 the other way, 10 to 9).
    if (P >= 256 && n <= 32 * kWave) return launch_blk(reduce_kernel<16>, grid_for(n, 16), 1024, s, part, P, stride, out);
    const int waves = P >= 16 ? 16 : P >= 4 ? 4 : 1;
    return launch_blk(reduce_kernel<kWave>, grid_for(n, kWave), waves * kWave, s, part, P, stride, out);
}

template <int IO>
static snn_status norm_forward_io(const NormArgs& a, hipStream_t s) {
    const dim3 grid{unsigned(a.groups)};
    if (a.F > kNormRegs) return launch_blk(norm_long_forward_kernel<IO>, grid, kLongLanes, s, a);
    const int n = norm_lanes(a.F);
    return n > 512 ? launch_blk(norm_forward_kernel<IO, 1024>, grid, n, s, a)
                   : launch_blk(norm_forward_kernel<IO, 512>, grid, n, s, a);
}

template <int IO>
static snn_status norm_backward_io(const NormArgs& a, hipStream_t s) {
    const dim3 grid{unsigned(a.groups)};
    if (a.F > kNormRegs) return launch_blk(norm_long_backward_kernel<IO>, grid, kLongLanes, s, a);
    const int n = norm_lanes(a.F);
    return n > 512 ? launch_blk(norm_backward_kernel<IO, 1024>, grid, n, s, a)
                   : launch_blk(norm_backward_kernel<IO, 512>, grid, n, s, a);
}

snn_status norm_forward_entry(int io, const NormArgs& a, hipStream_t s) {
    return io == SNN_IO_F32 ? norm_forward_io<SNN_IO_F32>(a, s) : norm_forward_io<SNN_IO_BF16>(a, s);
}

snn_status norm_backward_entry(int io, const NormArgs& a, hipStream_t s) {
    const snn_status st = io == SNN_IO_F32 ? norm_backward_io<SNN_IO_F32>(a, s) : norm_backward_io<SNN_IO_BF16>(a, s);
    if (st != SNN_OK) return st;
    const ReduceOut out = {{a.gw_post, a.gscale, a.gw_pre}, {a.F, a.F, a.F}};
    return reduce_entry(a.part, a.groups, 3 * a.F, out, s);
}

}  // namespace snnlif
