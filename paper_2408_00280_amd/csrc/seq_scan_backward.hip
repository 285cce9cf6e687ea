// Selective state space scan, backward.
//
// With e[t] = a[t+1] dL/dh[t+1] carried down from the step after,
//   dL/dh = C dL/dy + e,  dL/dC += dL/dy h,  dL/dB += dL/dh d x,
//   dL/d(d) = sum_n dL/dh (A a h[t-1] + B x),  dL/dA += dL/dh d a h[t-1],
//   dL/dx = sum_n dL/dh B d + D dL/dy,  dL/ddt = dL/d(d) sigmoid(dt + dt_bias).
// Blocks of K steps go in reverse: from the state that the forward kept at the block's start
// the decays a and the products a h[t-1] of its steps are formed again in registers, then the
// recurrence runs down.  Lanes, waves and scalars are as in the forward.  The sums of dL/dB
// and dL/dC over the 64 features of a wave halve the number of values at each of the first
// three steps (8 values and 64 lanes to 1 value in 8 groups of lanes): 17 instructions for 4
// states.  Sums over tiles, sequences and steps go through partial results that further
// kernels add up in a fixed order.  Bound by the vector ALU.
#include "seq_scan.h"

namespace snnlif {
namespace {

// Sums v[0..7] over the 64 lanes; lane l gets the sum of v[l / 8].
__device__ __forceinline__ float reduce8(const float (&v)[8], int lane) {
    float a[4], b[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[i]), __float_as_uint(v[i + 4]), false, false);
        a[i] = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(a[i]), __float_as_uint(a[i + 2]), false, false);
        b[i] = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    const float lo = b[0] + dpp<kDppRor8>(b[0]), hi = b[1] + dpp<kDppRor8>(b[1]);
    float r = (lane & 8) ? hi : lo;
    r += dpp<kDppHalfMirror>(r);
    r += dpp<kDppXor2>(r);
    r += dpp<kDppXor1>(r);
    return r;
}

template <int IO, int K>
__global__ __launch_bounds__(K == 16 ? 512 : 1024) void scan_backward_kernel(ScanArgs a) {
    extern __shared__ float lds[];
    const ScanPlace p = scan_place(a);
    const int waves = a.plan.waves, sp = a.plan.sp;
    f32x4_t* sd = reinterpret_cast<f32x4_t*>(lds);               // [K][64] (d, d x, dL/dy, x)
    float2* sg = reinterpret_cast<float2*>(lds + K * kWave * 4); // [waves][K][64] (sum dh B, sum dh a h A)
    float* sbc = lds + K * kWave * (4 + 2 * waves);              // [K][2][sp]
    float rate[kSL], e[kSL], gA[kSL], gD = 0.0f, gbias = 0.0f;
    load_rates(a, p, rate);
    load_state(a, p, a.gh_out, e);
#pragma unroll
    for (int i = 0; i < kSL; ++i) gA[i] = 0.0f;
    const float skip = a.D != nullptr ? a.D[p.f] : 0.0f, bias = a.dt_bias != nullptr ? a.dt_bias[p.f] : 0.0f;
    const int64_t len = steps_of(a.lengths, p.b, a.T);
    const int64_t row = int64_t(a.G) * 2 * sp;
    // partial sums of this tile: [tile][t][b][g][2][sp]
    float* part = a.part_bc + p.tile * a.T * a.B * row;

    for (int64_t c = a.plan.blocks - 1; c >= 0; --c) {
        const int64_t t0 = c * K;
        const int n = int(max(int64_t(0), min(int64_t(K), len - t0)));
        for (int k = p.wave; k < K; k += waves) {
            f32x4_t d = {0.0f, 0.0f, 0.0f, 0.0f};
            if (k < n) {
                const float v = load1<IO>(at<IO>(a.dt, t0 + k, p.b, p.f)) + bias;
                d[3] = load1<IO>(at<IO>(a.x, t0 + k, p.b, p.f));
                d[2] = p.active ? load1<IO>(at<IO>(a.gy, t0 + k, p.b, p.f)) : 0.0f;
                d[0] = a.softplus ? softplus(v) : v;
                d[1] = p.active ? d[0] * d[3] : 0.0f;            // lanes behind the group add nothing
            }
            sd[k * kWave + p.lane] = d;
        }
        __syncthreads();
        if (n > 0) {
            float dec[K][kSL], ah[K][kSL], h[kSL];
            const float* bc = a.packed + (t0 * a.B + p.b) * row + p.g * 2 * sp + p.wave * kSL;
            if (c > 0) {
#pragma unroll
                for (int i = 0; i < kSL; ++i) {
                    const int s = p.wave * kSL + i;
                    h[i] = s < a.S ? a.saved[kept_at(a, p, c, s)] : 0.0f;
                }
            } else {
                load_state(a, p, a.h_in, h);
            }
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (k < n) {
                    const f32x4_t d = sd[k * kWave + p.lane];
                    const f32x4_t bv = scalar_load4(bc + k * a.B * row);
#pragma unroll
                    for (int i = 0; i < kSL; ++i) {
                        dec[k][i] = __builtin_amdgcn_exp2f(d[0] * rate[i]);
                        ah[k][i] = dec[k][i] * h[i];
                        h[i] = fmaf(d[1], bv[i], ah[k][i]);
                    }
                }
            }
#pragma unroll
            for (int k = K - 1; k >= 0; --k) {
                if (k < n) {
                    const f32x4_t d = sd[k * kWave + p.lane];
                    const f32x4_t bv = scalar_load4(bc + k * a.B * row), cv = scalar_load4(bc + k * a.B * row + sp);
                    float v[8], gx = 0.0f, gd = 0.0f;
#pragma unroll
                    for (int i = 0; i < kSL; ++i) {
                        const float dh = fmaf(cv[i], d[2], e[i]);
                        v[i] = dh * d[1];
                        v[kSL + i] = d[2] * fmaf(d[1], bv[i], ah[k][i]);
                        gx = fmaf(dh, bv[i], gx);
                        const float q = dh * ah[k][i];
                        gd = fmaf(q, rate[i], gd);
                        gA[i] = fmaf(q, d[0], gA[i]);
                        e[i] = dec[k][i] * dh;
                    }
                    sg[(p.wave * K + k) * kWave + p.lane] = {gx, gd};
                    const float r = reduce8(v, p.lane);
                    const int j = p.lane >> 3;
                    if ((p.lane & 7) == 0) sbc[(k * 2 + (j >> 2)) * sp + p.wave * kSL + (j & 3)] = r;
                }
            }
        }
        __syncthreads();
        for (int k = p.wave; k < K && t0 + k < a.T; k += waves) {
            float gx = 0.0f, gdt = 0.0f;
            if (k < n) {
                const f32x4_t d = sd[k * kWave + p.lane];
                float db = 0.0f, da = 0.0f;
                for (int w = 0; w < waves; ++w) {
                    const float2 g = sg[(w * K + k) * kWave + p.lane];
                    db += g.x;
                    da += g.y;
                }
                gx = fmaf(d[0], db, skip * d[2]);
                gdt = fmaf(d[3], db, da * kLn2);                 // rate is A log2 e
                if (a.softplus) gdt *= sigmoid(load1<IO>(at<IO>(a.dt, t0 + k, p.b, p.f)) + bias);
                gD = fmaf(d[2], d[3], gD);
                gbias += gdt;
            }
            if (p.active) {
                store1<IO>(at_out<IO>(a.gx, t0 + k, p.b, p.f), gx);
                store1<IO>(at_out<IO>(a.gdt, t0 + k, p.b, p.f), gdt);
            }
        }
        for (int i = threadIdx.x; i < K * 2 * sp; i += waves * kWave) {
            const int k = i / (2 * sp), s = i - k * 2 * sp;
            if (t0 + k < a.T) part[((t0 + k) * a.B + p.b) * row + p.g * 2 * sp + s] = k < n ? sbc[i] : 0.0f;
        }
        __syncthreads();
    }
    if (a.gh_in != nullptr) store_state(a, p, a.gh_in, e);
    float* pf = a.part_f + p.b * (a.F * (a.S + 2));
    store_state(a, {p.lane, p.wave, p.g, p.tile, 0, p.f, p.active}, pf, gA);
    float* s2 = lds;                                             // [waves][2][64]
    s2[(p.wave * 2) * kWave + p.lane] = gD;
    s2[(p.wave * 2 + 1) * kWave + p.lane] = gbias;
    __syncthreads();
    if (p.wave == 0 && p.active) {
        float sum[2] = {0.0f, 0.0f};
        for (int w = 0; w < waves; ++w) {
            sum[0] += s2[(w * 2) * kWave + p.lane];
            sum[1] += s2[(w * 2 + 1) * kWave + p.lane];
        }
        pf[a.F * a.S + p.f] = sum[0];
        pf[a.F * (a.S + 1) + p.f] = sum[1];
    }
}

// dL/dB and dL/dC: the sums over a group's tiles.
template <int IO>
__global__ __launch_bounds__(kBlock) void scan_join_kernel(ScanArgs a, int64_t n) {
    const int64_t i = int64_t(blockIdx.x) * kBlock + threadIdx.x;
    if (i >= n) return;
    const int s = int(i % a.S);
    const int64_t q = i / a.S, which = q & 1, r = q >> 1;
    const int64_t g = r % a.G, tb = r / a.G, b = tb % a.B, t = tb / a.B;
    const int64_t stride = a.T * a.B * a.G * 2 * a.plan.sp;
    const float* part = a.part_bc + (r * 2 + which) * a.plan.sp + s;
    float sum = 0.0f;
    for (int64_t j = 0; j < a.plan.tiles; ++j) sum += part[j * stride];
    store1<IO>(at_out<IO>(which ? a.gC : a.gB, t, b, g * a.S + s), sum);
}

template <int IO, int K>
snn_status backward_launch(const ScanArgs& a, hipStream_t s) {
    const int lds = K * 4 * (kWave * (4 + 2 * a.plan.waves) + 2 * a.plan.sp);
    hipLaunchKernelGGL((scan_backward_kernel<IO, K>), dim3(unsigned(a.plan.tiles * a.G * a.B)), dim3(a.plan.waves * kWave),
                       lds, s, a);
    if (hipGetLastError() != hipSuccess) return SNN_E_LAUNCH;
    const int64_t n = a.T * a.B * a.G * 2 * a.S;
    snn_status st = launch(scan_join_kernel<IO>, grid_for(n), s, a, n);
    if (st != SNN_OK) return st;
    const ReduceOut out = {{a.gA, a.gD, a.gdt_bias}, {a.F * a.S, a.F, a.F}};
    return reduce_entry(a.part_f, a.B, scan_partial_values(a.F, a.S), out, s);
}

}  // namespace

snn_status scan_backward_entry(int io, const ScanArgs& a, hipStream_t s) {
    if (a.plan.k == 16)
        return io == SNN_IO_F32 ? backward_launch<SNN_IO_F32, 16>(a, s) : backward_launch<SNN_IO_BF16, 16>(a, s);
    return io == SNN_IO_F32 ? backward_launch<SNN_IO_F32, 8>(a, s) : backward_launch<SNN_IO_BF16, 8>(a, s);
}

}  // namespace snnlif
