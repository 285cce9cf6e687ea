// A block's gate, norm and scaled residual with the next block's norm, forward and backward,
// and the sums of partial results over workgroups.
//
// Rows of up to 8192 features are read once: a lane holds 8 of a row's features (16 bytes of
// bf16, two pieces of 16 bytes of fp32) and their parameters, a workgroup's lanes one row, and
// the workgroup walks rows with the next one's loads in flight.  A row costs two sums over the
// workgroup per direction, and more than one workgroup per CU hides them.  Longer rows go
// through the plain kernels, which read the row again for each sum.  Bound by memory.
#include "seq_device.h"

namespace snnlif {
namespace {

// -- Long rows ---------------------------------------------------------------------------

// Sum over the workgroup, in every lane.
__device__ __forceinline__ float block_sum(float v, float* lds) {
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0) lds[threadIdx.x / kWave] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kBlock / kWave; ++w) s += lds[w];
    return s;
}

template <int IO>
struct NormRow {
    const NormArgs& a;
    int64_t t, b;
    __device__ float gated(int64_t f) const {
        const float y = load1<IO>(at<IO>(a.y, t, b, f));
        if (a.z.p == nullptr) return y;
        const float z = load1<IO>(at<IO>(a.z, t, b, f));
        return y * (z * sigmoid(z));
    }
    __device__ float residual(int64_t f, float g, float k1) const {
        const float n = a.w_post != nullptr ? g * k1 * a.w_post[f] : g;
        const float r = a.r.p != nullptr ? load1<IO>(at<IO>(a.r, t, b, f)) : 0.0f;
        return a.scale != nullptr ? fmaf(a.scale[f], n, r) : r + n;
    }
};

template <int IO>
__global__ __launch_bounds__(kBlock) void norm_long_forward_kernel(NormArgs a) {
    __shared__ float lds[kBlock / kWave];
    const int64_t i = blockIdx.x;
    const NormRow<IO> row = {a, i / a.B, i % a.B};
    const int64_t t = row.t, b = row.b;
    if (t >= steps_of(a.lengths, b, a.T)) {
        for (int64_t f = threadIdx.x; f < a.F; f += kBlock) {
            store1<IO>(at_out<IO>(a.r_new, t, b, f), 0.0f);
            if (a.w_pre != nullptr) store1<IO>(at_out<IO>(a.u, t, b, f), 0.0f);
        }
        return;
    }
    float k1 = 0.0f, k2 = 0.0f;
    if (a.w_post != nullptr) {
        float s = 0.0f;
        for (int64_t f = threadIdx.x; f < a.F; f += kBlock) {
            const float g = row.gated(f);
            s = fmaf(g, g, s);
        }
        k1 = 1.0f / sqrtf(block_sum(s, lds) / float(a.F) + a.eps);
    }
    float s = 0.0f;
    for (int64_t f = threadIdx.x; f < a.F; f += kBlock) {
        const float r = row.residual(f, row.gated(f), k1);
        s = fmaf(r, r, s);
    }
    if (a.w_pre != nullptr) k2 = 1.0f / sqrtf(block_sum(s, lds) / float(a.F) + a.eps);
    for (int64_t f = threadIdx.x; f < a.F; f += kBlock) {
        const float r = row.residual(f, row.gated(f), k1);
        store1<IO>(at_out<IO>(a.r_new, t, b, f), r);
        if (a.w_pre != nullptr) store1<IO>(at_out<IO>(a.u, t, b, f), r * k2 * a.w_pre[f]);
    }
    if (a.rstd != nullptr && threadIdx.x == 0) {
        a.rstd[i] = k1;
        a.rstd[a.T * a.B + i] = k2;
    }
}

// Per row: with rn = r' k2, t = dL/du w_pre:  dL/dr' = dL/dr_new + k2 (t - rn mean(t rn));
// with gn = g k1, t = dL/dr' scale w_post:    dL/dg = k1 (t - gn mean(t gn)).
template <int IO>
__global__ __launch_bounds__(kBlock) void norm_long_backward_kernel(NormArgs a) {
    __shared__ float lds[kBlock / kWave];
    float* part = a.part + int64_t(blockIdx.x) * 3 * a.F;      // w_post, scale, w_pre
    for (int64_t f = threadIdx.x; f < a.F; f += kBlock) part[f] = part[a.F + f] = part[2 * a.F + f] = 0.0f;
    for (int64_t i = blockIdx.x; i < a.T * a.B; i += a.groups) {
        const NormRow<IO> row = {a, i / a.B, i % a.B};
        const int64_t t = row.t, b = row.b;
        if (t >= steps_of(a.lengths, b, a.T)) {
            for (int64_t f = threadIdx.x; f < a.F; f += kBlock) {
                store1<IO>(at_out<IO>(a.gy, t, b, f), 0.0f);
                if (a.z.p != nullptr) store1<IO>(at_out<IO>(a.gz, t, b, f), 0.0f);
                if (a.r.p != nullptr) store1<IO>(at_out<IO>(a.gr, t, b, f), 0.0f);
            }
            continue;
        }
        const float k1 = a.w_post != nullptr ? a.rstd_in[i] : 0.0f;
        const float k2 = a.w_pre != nullptr ? a.rstd_in[a.T * a.B + i] : 0.0f;
        const bool pre = a.w_pre != nullptr && a.gu.p != nullptr;
        float m2 = 0.0f, m1 = 0.0f;
        if (pre) {
            float s = 0.0f;
            for (int64_t f = threadIdx.x; f < a.F; f += kBlock) {
                const float rn = row.residual(f, row.gated(f), k1) * k2;
                s = fmaf(load1<IO>(at<IO>(a.gu, t, b, f)) * a.w_pre[f], rn, s);
            }
            m2 = block_sum(s, lds) / float(a.F);
        }
        const auto grad_r = [&](int64_t f, float& gw_pre) {
            float gr = a.gr_new.p != nullptr ? load1<IO>(at<IO>(a.gr_new, t, b, f)) : 0.0f;
            gw_pre = 0.0f;
            if (pre) {
                const float rn = row.residual(f, row.gated(f), k1) * k2, gu = load1<IO>(at<IO>(a.gu, t, b, f));
                gr = fmaf(k2, gu * a.w_pre[f] - rn * m2, gr);
                gw_pre = gu * rn;
            }
            return gr;
        };
        if (a.w_post != nullptr) {
            float s = 0.0f, unused;
            for (int64_t f = threadIdx.x; f < a.F; f += kBlock) {
                const float w = a.w_post[f] * (a.scale != nullptr ? a.scale[f] : 1.0f);
                s = fmaf(grad_r(f, unused) * w, row.gated(f) * k1, s);
            }
            m1 = block_sum(s, lds) / float(a.F);
        }
        for (int64_t f = threadIdx.x; f < a.F; f += kBlock) {
            float gw_pre;
            const float gr = grad_r(f, gw_pre), g = row.gated(f), gn = g * k1;
            const float gs = a.scale != nullptr ? gr * a.scale[f] : gr;      // dL/dn
            const float gg = a.w_post != nullptr ? k1 * (gs * a.w_post[f] - gn * m1) : gs;
            const float n = a.w_post != nullptr ? gn * a.w_post[f] : g;
            part[f] = fmaf(gs, gn, part[f]);
            part[a.F + f] = fmaf(gr, n, part[a.F + f]);
            part[2 * a.F + f] += gw_pre;
            if (a.r.p != nullptr) store1<IO>(at_out<IO>(a.gr, t, b, f), gr);
            if (a.z.p == nullptr) {
                store1<IO>(at_out<IO>(a.gy, t, b, f), gg);
            } else {
                const float z = load1<IO>(at<IO>(a.z, t, b, f)), s = sigmoid(z);
                store1<IO>(at_out<IO>(a.gz, t, b, f), gg * load1<IO>(at<IO>(a.y, t, b, f)) * silu_slope(z, s));
                store1<IO>(at_out<IO>(a.gy, t, b, f), gg * (z * s));
            }
        }
    }
}

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
    __device__ explicit Lane8(int64_t F) {
#pragma unroll
        for (int c = 0; c < N; ++c) {
            f[c] = int(c * blockDim.x + threadIdx.x) * V;
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
#pragma unroll
    for (int j = 0; j < kNormLane; ++j) g_post[j] = g_scale[j] = g_pre[j] = 0.0f;
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
    // the next row's loads have no registers beside 16 waves of one workgroup
    constexpr bool kAhead = MAXT < 1024;
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
            for (int j = 0; j < kNormLane; ++j) {
                rn[j] = k2 * fmaf(scale[j], gn[j] * w_post[j], rn[j]);
                g_pre[j] = fmaf(gu[j], rn[j], g_pre[j]);
                gu[j] *= w_pre[j];
                s = fmaf(gu[j], rn[j], s);
            }
            const float m = sum(s) * mean;
#pragma unroll
            for (int j = 0; j < kNormLane; ++j) gr[j] = fmaf(k2, fmaf(-m, rn[j], gu[j]), gr[j]);
            s = 0.0f;
        }
        if (a.r.p != nullptr) lane.store(a.gr, t, b, gr);
#pragma unroll
        for (int j = 0; j < kNormLane; ++j) {
            g_scale[j] = fmaf(gr[j], gn[j] * w_post[j], g_scale[j]);
            gr[j] *= scale[j];                                     // dL/dn
            g_post[j] = fmaf(gr[j], gn[j], g_post[j]);
            gr[j] *= w_post[j];
        }
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
    lane.put(part, g_post);
    lane.put(part + a.F, g_scale);
    lane.put(part + 2 * a.F, g_pre);
}

// 64 values per workgroup, its waves over the partial results.
__global__ __launch_bounds__(1024) void reduce_kernel(const float* part, int64_t P, int64_t stride, ReduceOut out) {
    __shared__ float lds[16][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, waves = blockDim.x / kWave;
    int64_t i = int64_t(blockIdx.x) * kWave + lane;
    const bool in = i < out.n[0] + out.n[1] + out.n[2];
    float s = 0.0f;
    if (in) {
#pragma unroll 8
        for (int64_t p = wave; p < P; p += waves) s += part[p * stride + i];
    }
    lds[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || !in) return;
    for (int w = 1; w < waves; ++w) s += lds[w][lane];
    int k = 0;
    while (i >= out.n[k]) i -= out.n[k++];
    if (out.p[k] != nullptr) out.p[k][i] = s;
}

}  // namespace

snn_status reduce_entry(const float* part, int64_t P, int64_t stride, const ReduceOut& out, hipStream_t s) {
    const int64_t n = out.n[0] + out.n[1] + out.n[2];
    const int waves = P >= 16 ? 16 : P >= 4 ? 4 : 1;
    return launch_blk(reduce_kernel, grid_for(n, kWave), waves * kWave, s, part, P, stride, out);
}

template <int IO>
static snn_status norm_forward_io(const NormArgs& a, hipStream_t s) {
    if (a.F > kNormRegs) return launch(norm_long_forward_kernel<IO>, dim3(unsigned(a.T * a.B)), s, a);
    const dim3 grid{unsigned(a.groups)};
    const int n = norm_lanes(a.F);
    return n > 512 ? launch_blk(norm_forward_kernel<IO, 1024>, grid, n, s, a)
                   : launch_blk(norm_forward_kernel<IO, 512>, grid, n, s, a);
}

template <int IO>
static snn_status norm_backward_io(const NormArgs& a, hipStream_t s) {
    const dim3 grid{unsigned(a.groups)};
    if (a.F > kNormRegs) return launch(norm_long_backward_kernel<IO>, grid, s, a);
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
