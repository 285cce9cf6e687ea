// Selective state space scan, forward.
//
// Per step, feature and state: a = 2^(d A log2 e), h = a h + (d x) B, y += C h: five vector
// instructions, one of them an exponential.  With S = 16 states that is more work than the
// few bytes per feature and step need to move, so the kernel is bound by the vector ALU.
// A lane is a feature, each wave of a workgroup holds 4 of its states in registers, and B and
// C come through scalar registers.  What belongs to a step but not to a state (the softplus,
// the sum of y over the waves) is shared out over the waves, K steps at a time, through LDS.
#include "seq_scan.h"

namespace snnlif {
namespace {

template <int IO>
__global__ __launch_bounds__(kBlock) void scan_pack_kernel(ScanArgs a, int64_t n) {
    const int64_t i = int64_t(blockIdx.x) * kBlock + threadIdx.x;
    if (i >= n) return;
    const int sp = a.plan.sp;
    const int s = int(i % sp);
    const int64_t q = i / sp, which = q & 1, r = q >> 1;     // r = (t B + b) G + g
    const int64_t g = r % a.G, tb = r / a.G, b = tb % a.B, t = tb / a.B;
    a.packed[i] = s < a.S ? load1<IO>(at<IO>(which ? a.Cm : a.Bm, t, b, g * a.S + s)) : 0.0f;
}

template <int IO, int K>
__global__ __launch_bounds__(1024) void scan_forward_kernel(ScanArgs a) {
    extern __shared__ float lds[];
    const ScanPlace p = scan_place(a);
    const int waves = a.plan.waves;
    float2* sd = reinterpret_cast<float2*>(lds);                 // [K][64] (d, d x)
    float* sy = lds + K * kWave * 2;                             // [waves][K][64]
    float rate[kSL], h[kSL];
    load_rates(a, p, rate);
    load_state(a, p, a.h_in, h);
    const float skip = a.D != nullptr ? a.D[p.f] : 0.0f, bias = a.dt_bias != nullptr ? a.dt_bias[p.f] : 0.0f;
    const int64_t len = steps_of(a.lengths, p.b, a.T);
    const int64_t row = int64_t(a.G) * 2 * a.plan.sp;            // packed values per (t, b)

    for (int64_t c = 0; c < a.plan.blocks; ++c) {
        const int64_t t0 = c * K;
        if (c > 0 && a.saved != nullptr && t0 < len) {
#pragma unroll
            for (int i = 0; i < kSL; ++i)
                if (p.active && p.wave * kSL + i < a.S) a.saved[kept_at(a, p, c, p.wave * kSL + i)] = h[i];
        }
        for (int k = p.wave; k < K; k += waves) {
            float2 d = {0.0f, 0.0f};
            if (t0 + k < len) {
                const float v = load1<IO>(at<IO>(a.dt, t0 + k, p.b, p.f)) + bias;
                d.x = a.softplus ? softplus(v) : v;
                d.y = d.x * load1<IO>(at<IO>(a.x, t0 + k, p.b, p.f));
            }
            sd[k * kWave + p.lane] = d;
        }
        __syncthreads();
        const int64_t n = min(int64_t(K), len - t0);
        for (int k = 0; k < n; ++k) {
            const float2 d = sd[k * kWave + p.lane];
            const float* bc = a.packed + ((t0 + k) * a.B + p.b) * row + p.g * 2 * a.plan.sp + p.wave * kSL;
            const f32x4_t bv = scalar_load4(bc), cv = scalar_load4(bc + a.plan.sp);
            float y = 0.0f;
#pragma unroll
            for (int i = 0; i < kSL; ++i) {
                h[i] = fmaf(__builtin_amdgcn_exp2f(d.x * rate[i]), h[i], d.y * bv[i]);
                y = fmaf(cv[i], h[i], y);
            }
            sy[(p.wave * K + k) * kWave + p.lane] = y;
        }
        __syncthreads();
        for (int k = p.wave; k < K && t0 + k < a.T; k += waves) {
            float y = 0.0f;
            if (t0 + k < len) {
                y = skip * load1<IO>(at<IO>(a.x, t0 + k, p.b, p.f));
                for (int w = 0; w < waves; ++w) y += sy[(w * K + k) * kWave + p.lane];
            }
            if (p.active) store1<IO>(at_out<IO>(a.y, t0 + k, p.b, p.f), y);
        }
    }
    if (a.h_out != nullptr) store_state(a, p, a.h_out, h);
}

template <int IO, int K>
snn_status forward_launch(const ScanArgs& a, hipStream_t s) {
    const int lds = K * kWave * 4 * (2 + a.plan.waves);
    hipLaunchKernelGGL((scan_forward_kernel<IO, K>), dim3(unsigned(a.plan.tiles * a.G * a.B)), dim3(a.plan.waves * kWave),
                       lds, s, a);
    return hipGetLastError() == hipSuccess ? SNN_OK : SNN_E_LAUNCH;
}

}  // namespace

snn_status scan_pack_entry(int io, const ScanArgs& a, hipStream_t s) {
    const int64_t n = a.T * a.B * a.G * 2 * a.plan.sp;
    return io == SNN_IO_F32 ? launch(scan_pack_kernel<SNN_IO_F32>, grid_for(n), s, a, n)
                            : launch(scan_pack_kernel<SNN_IO_BF16>, grid_for(n), s, a, n);
}

snn_status scan_forward_entry(int io, const ScanArgs& a, hipStream_t s) {
    if (a.plan.k == 16)
        return io == SNN_IO_F32 ? forward_launch<SNN_IO_F32, 16>(a, s) : forward_launch<SNN_IO_BF16, 16>(a, s);
    return io == SNN_IO_F32 ? forward_launch<SNN_IO_F32, 8>(a, s) : forward_launch<SNN_IO_BF16, 8>(a, s);
}

}  // namespace snnlif
