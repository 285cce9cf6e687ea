// A block's gate, norm and scaled residual with the next block's norm, forward and backward,
// and the sums of partial results over workgroups.
//
// A workgroup takes a row; bound by memory.
#include "seq_device.h"

namespace snnlif {
namespace {

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
__global__ __launch_bounds__(kBlock) void norm_forward_kernel(NormArgs a) {
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
__global__ __launch_bounds__(kBlock) void norm_backward_kernel(NormArgs a) {
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

// 64 values per workgroup, its waves over the partial results.
__global__ __launch_bounds__(1024) void reduce_kernel(const float* part, int64_t P, int64_t stride, ReduceOut out) {
    __shared__ float lds[16][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, waves = blockDim.x / kWave;
    int64_t i = int64_t(blockIdx.x) * kWave + lane;
    const bool in = i < out.n[0] + out.n[1] + out.n[2];
    float s = 0.0f;
    if (in)
        for (int64_t p = wave; p < P; p += waves) s += part[p * stride + i];
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

snn_status norm_forward_entry(int io, const NormArgs& a, hipStream_t s) {
    const dim3 grid(unsigned(a.T * a.B));
    return io == SNN_IO_F32 ? launch(norm_forward_kernel<SNN_IO_F32>, grid, s, a)
                            : launch(norm_forward_kernel<SNN_IO_BF16>, grid, s, a);
}

snn_status norm_backward_entry(int io, const NormArgs& a, hipStream_t s) {
    const dim3 grid{unsigned(a.groups)};
    const snn_status st = io == SNN_IO_F32 ? launch(norm_backward_kernel<SNN_IO_F32>, grid, s, a)
                                           : launch(norm_backward_kernel<SNN_IO_BF16>, grid, s, a);
    if (st != SNN_OK) return st;
    const ReduceOut out = {{a.gw_post, a.gscale, a.gw_pre}, {a.F, a.F, a.F}};
    return reduce_entry(a.part, a.groups, 3 * a.F, out, s);
}

}  // namespace snnlif
