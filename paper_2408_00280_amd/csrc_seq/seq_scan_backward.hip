// Selective state space scan, backward.
//
// With e[t] = a[t+1] dL/dh[t+1] carried down from the step after,
//   dL/dh = C dL/dy + e,  dL/dC += dL/dy h,  dL/dB += dL/dh d x,
//   dL/d(d) = sum_n dL/dh (A a h[t-1] + B x),  dL/dA += dL/dh d a h[t-1],
//   dL/dx = sum_n dL/dh B d + D dL/dy,  dL/ddt = dL/d(d) sigmoid(dt + dt_bias).
// Blocks of K steps go in reverse: from the state that the forward kept at the block's start
// the decays and states of its steps are formed again in registers, then the recurrence runs
// down, dL/dh a h[t-1] as e[t-1] h[t-1].  Lanes and waves are as in the forward, and as there
// the next block is loaded while a block runs.  The sums of dL/dB and dL/dC over the 64 features
// of a wave halve the number of values at each of the first three steps (8 values and 64 lanes
// to 1 value in 8 groups of lanes): 17 instructions for 4 states.  Sums over tiles, sequences and
// steps go through partial results that one further kernel adds up in a fixed order.  Bound by
// the vector ALU, 80% busy (x[1024][8][4096] bf16 of 16 states: 444 us).
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

struct __align__(16) Step {
    float d, dx, gy, x;    // d, d x, dL/dy, x
};

// Adds one block's part of dL/dA, the first of those that a workgroup goes through, up to the
// sequence's last step: from memory, each step's state from the block's start.  Hardly a call
// needs it, so that it takes the kernel's arguments anew (a ScanArgs is all of them) rather than
// hold registers until then.
template <int IO, int K>
__device__ void add_block_rates(int t0, float (&gA)[kSL]) {
    auto args = __builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(args));
    ScanArgs a;
    __builtin_memcpy(&a, (const void*)args, sizeof(a));
    const ScanPlace p = scan_place(a);
    const Columns<IO> cx(a.x, p), cdt(a.dt, p), cgy(a.gy, p);
    const float bias = a.dt_bias != nullptr ? a.dt_bias[p.f] : 0.0f;
    float rate[kSL], from[kSL], e[kSL];
    load_rates(a, p, rate);
    if (t0 == 0) load_state(a, p, a.h_in, from);
    else StateColumn(a, p, a.saved).load(t0 / K - 1, from);
    segment_state<true>(a, p, rate, e);
#pragma unroll 1
    for (int t = p.len - 1; t >= t0; --t) {
        float h[kSL];
#pragma unroll
        for (int s = 0; s < kSL; ++s) h[s] = from[s];
#pragma unroll 1
        for (int i = t0; i <= t; ++i) {
            const float v = IoVec<IO, 1>::get(cdt.load(i), 0) + bias, d = a.softplus ? softplus(v) : v;
            const float dx = d * IoVec<IO, 1>::get(cx.load(i), 0), gy = IoVec<IO, 1>::get(cgy.load(i), 0);
#pragma unroll
            for (int s = 0; s < kSL; ++s) {
                if (s >= p.states) continue;
                const int64_t n = p.g * a.S + p.first + s;
                const float dec = __builtin_amdgcn_exp2f(d * rate[s]);
                if (i < t) {
                    h[s] = fmaf(dec, h[s], dx * load1<IO>(at<IO>(a.Bm, i, p.b, n)));
                } else {
                    e[s] = dec * fmaf(load1<IO>(at<IO>(a.Cm, t, p.b, n)), gy, e[s]);
                    gA[s] = fmaf(e[s] * h[s], d, gA[s]);
                }
            }
        }
    }
}

template <int NS>
struct BackwardLds {
    static constexpr int K = scan_keep(NS);
    Step sd[2][K][kWave];        // this block's, and the next one's as it is staged
    float slope[2][K][kWave];    // of the softplus
    StagedBC<NS, K> sbc[3];      // the last one zeros, for lanes without a feature
    float2 sg[NS][K][kWave];     // (sum dh B, sum dh a h A log2 e)
    float sgbc[K][NS][2 * kSL];  // dL/dB and dL/dC
};

// Waves per SIMD: 16 waves fill a CU; two of them, with 8-step blocks, are held to the 168 registers
// of three per SIMD (x[333][5][777]: a pass 73 us, 78 with 169 registers).
constexpr int backward_waves(int waves) { return waves > 8 ? 4 : waves == 2 ? 3 : 2; }

template <int IO, int NS, bool FULL>
__global__ __launch_bounds__(NS * kWave, backward_waves(NS)) void scan_backward_kernel(ScanArgs a) {
    constexpr int K = scan_keep(NS), R = K > NS ? K / NS : 1;
    // 4 waves per SIMD need no step read ahead, and have no registers for it
    constexpr bool kAhead = NS <= 8;
    extern __shared__ __align__(16) char lds[];
    auto& m = *reinterpret_cast<BackwardLds<NS>*>(lds);
    if (!scan_has_block(a)) return;
    const ScanPlace p = scan_place(a);
    float rate[kSL], e[kSL], gA[kSL], gD = 0.0f, gbias = 0.0f;
    load_rates(a, p, rate);
    // Lanes behind the group's last feature have steps and states of 0 and add nothing.  Their B
    // and C are zeros as well: 0 times an infinite one would not be.
    const StateColumn kept(a, p, a.saved);
    const auto load = [&](int64_t c, bool first, float (&v)[kSL]) {
#pragma unroll
        for (int s = 0; s < kSL; ++s) v[s] = 0.0f;
        if (!p.active) return;
        if (first) load_state(a, p, a.h_in, v);
        else if (p.states > 0) kept.load(c, v);
    };
    segment_state<true>(a, p, rate, e);
#pragma unroll
    for (int i = 0; i < kSL; ++i) {
        gA[i] = 0.0f;
        if (!p.active) e[i] = 0.0f;
    }
    float skip = a.D != nullptr ? a.D[p.f] : 0.0f, bias = a.dt_bias != nullptr ? a.dt_bias[p.f] : 0.0f;
    const Columns<IO> cx(a.x, p), cdt(a.dt, p), cgy(a.gy, p), cgx(a.gx, p), cgdt(a.gdt, p);
    const bool busy = p.states > 0;
    const int used = (a.S + kSL - 1) / kSL;

    struct Raw {
        typename IoVec<IO, 1>::raw x, dt, gy;
    };
    Raw raw[R];                  // of the next block
    const auto fetch_rows = [&](int t0) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int k = p.wave + r * NS;
            if (k < K && t0 >= p.t0 && t0 + k < p.len) raw[r] = {cx.load(t0 + k), cdt.load(t0 + k), cgy.load(t0 + k)};
        }
    };
    const auto stage_rows = [&](int t0, int to) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int k = p.wave + r * NS;
            Step d = {0.0f, 0.0f, 0.0f, 0.0f};
            float slope = 1.0f;
            if (k < K && t0 >= p.t0 && t0 + k < p.len) {
                const float v = IoVec<IO, 1>::get(raw[r].dt, 0) + bias, x = IoVec<IO, 1>::get(raw[r].x, 0);
                const float step = a.softplus ? softplus(v, slope) : v;
                if (p.active) d = {step, step * x, IoVec<IO, 1>::get(raw[r].gy, 0), x};
            }
            if (k < K) {
                m.sd[to][k][p.lane] = d;
                m.slope[to][k][p.lane] = slope;
            }
        }
    };

    int t0 = p.t0 + (p.t1 - 1 - p.t0) / K * K;
    for (; t0 >= p.t0 && t0 >= p.len; t0 -= K) {     // blocks behind the sequence's end
        for (int k = p.wave; k < K && t0 + k < p.t1; k += NS) {
            if (p.active) {
                cgx.store(t0 + k, 0.0f);
                cgdt.store(t0 + k, 0.0f);
            }
        }
    }
    BCColumns<IO, NS, K> cbc(a, p, t0);
    const auto fetch = [&](int t0) {
        cbc.template fetch<-1>(t0, p.t0, p.len);
        fetch_rows(t0);
    };
    const auto stage = [&](int t0, int to) {
        if (t0 >= p.t0) cbc.stage(t0, p.len, m.sbc[to]);
        stage_rows(t0, to);
    };
    fetch(t0);
    for (int i = threadIdx.x; i < K * NS * 2 * kSL; i += NS * kWave) m.sbc[2].v[0][0][i] = 0.0f;
    stage(t0, 0);
    fetch(t0 - K);
    float h[kSL], h_next[kSL];
    struct Ahead {
        Step d;
        f32x4_t b, c;
    } step, ahead;
    const auto read = [&](int block, int k) {
        const f32x4_t* bc = reinterpret_cast<const f32x4_t*>(m.sbc[p.active ? block : 2].v[k][p.wave]);
        return Ahead{m.sd[block][k][p.lane], bc[0], bc[1]};
    };
    load(t0 / K - 1, t0 <= 0, h);
    settle(skip);
    settle(bias);
    settle(rate);
    settle(e);
    settle(h);
    lds_barrier();
    int buf = 0, again = -1;
    for (; t0 >= p.t0; t0 -= K) {
        const int below = max(t0 - K, p.t0);
        if (busy) {
            step = read(buf, 0);
            float dec[K][kSL], hs[K + 1][kSL];       // decays, and the states before each step
#pragma unroll
            for (int s = 0; s < kSL; ++s) hs[0][s] = h[s];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (kAhead && k + 1 < K) ahead = read(buf, k + 1);
                if (!kAhead) step = read(buf, k);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int s = 0; s < kSL; ++s) {
                    dec[k][s] = __builtin_amdgcn_exp2f(step.d.d * rate[s]);
                    hs[k + 1][s] = fmaf(dec[k][s], hs[k][s], step.d.dx * step.b[s]);
                }
                __builtin_amdgcn_sched_barrier(0);
                if (kAhead && k + 1 < K) step = ahead;
            }
            // the sums over the wave run a step behind, beside the next step's recurrence
            float v[2 * kSL];
            const auto sum_up = [&](int k) {
                m.sgbc[k][p.wave][p.lane >> 3] = reduce8(v, p.lane);   // the same from 8 lanes
            };
#pragma unroll
            for (int k = K - 1; k >= 0; --k) {
                if (kAhead && k > 0) ahead = read(buf, k - 1);
                if (!kAhead) step = read(buf, k);
                if (k == K / 2) {                // half of the block's registers are free by now
                    load(below / K - 1, below == 0, h_next);
                }
                __builtin_amdgcn_sched_barrier(0);
                if (k < K - 1) sum_up(k + 1);
                const Step d = step.d;
                float gx = 0.0f, gd = 0.0f;
#pragma unroll
                for (int s = 0; s < kSL; ++s) {
                    const float b = step.b[s], dh = fmaf(step.c[s], d.gy, e[s]);
                    v[s] = dh * d.dx;
                    v[kSL + s] = d.gy * hs[k + 1][s];
                    const bool in = FULL || s < p.states;
                    gx = in ? fmaf(dh, b, gx) : gx;
                    e[s] = dec[k][s] * dh;
                    const float q = e[s] * hs[k][s];
                    gd = in ? fmaf(q, rate[s], gd) : gd;
                    gA[s] = fmaf(q, d.d, gA[s]);
                }
                m.sg[p.wave][k][p.lane] = {gx, gd};
                __builtin_amdgcn_sched_barrier(0);
                if (kAhead) step = ahead;
            }
            sum_up(0);
            // The steps behind the end have d = 0, and an infinite state or gradient times that is
            // NaN.  They come first: the sum of their block is formed again at the end, without
            // them (a branch in each step costs all blocks 7% of their time).
            if (t0 + K > p.len) {
                bool nan = false;
#pragma unroll
                for (int s = 0; s < kSL; ++s) nan |= gA[s] != gA[s];
                if (__builtin_amdgcn_ballot_w64(nan) != 0) {
                    again = t0;
#pragma unroll
                    for (int s = 0; s < kSL; ++s) gA[s] = 0.0f;
                }
            }
            settle(h_next);      // half a block after their load, and not with the next block's loads
#pragma unroll
            for (int s = 0; s < kSL; ++s) h[s] = h_next[s];
        }
        stage(t0 - K, buf ^ 1);
        fetch(t0 - 2 * K);
        lds_barrier();
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int k = p.wave + r * NS;
            if (k < K && t0 + k < p.t1) {
                float gx = 0.0f, gdt = 0.0f;
                if (t0 + k < p.len) {
                    const Step s = m.sd[buf][k][p.lane];
                    float2 g[NS];
                    float db = 0.0f, da = 0.0f;
#pragma unroll
                    for (int w = 0; w < NS; ++w) g[w] = m.sg[w][k][p.lane];
#pragma unroll
                    for (int w = 0; w < NS; ++w) {
                        db += w < used ? g[w].x : 0.0f;
                        da += w < used ? g[w].y : 0.0f;
                    }
                    gx = fmaf(s.d, db, a.D != nullptr ? skip * s.gy : 0.0f);
                    gdt = fmaf(s.x, db, da * kLn2) * m.slope[buf][k][p.lane];   // rate is A log2 e
                    gD = fmaf(s.gy, s.x, gD);
                    gbias += gdt;
                }
                if (p.active) {
                    cgx.store(t0 + k, gx);
                    cgdt.store(t0 + k, gdt);
                }
            }
        }
        {
            const int64_t row = int64_t(a.B) * a.G * (NS * 2 * kSL);
            float* part = a.part_bc + p.tile * a.T * row + (p.b * a.G + p.g) * (NS * 2 * kSL);
            for (int i = threadIdx.x; i < K * NS * 2 * kSL; i += NS * kWave) {
                const int k = i / (NS * 2 * kSL), j = i % (NS * 2 * kSL);
                if (t0 + k < p.len) part[(t0 + k) * row + j] = m.sgbc[k][0][j];
            }
        }
        lds_barrier();
        buf ^= 1;
    }
    if (again >= 0) add_block_rates<IO, K>(again, gA);
    if (a.gh_in != nullptr && p.t0 == 0) store_state(a, p, a.gh_in, e);
    float* pf = a.part_f + (blockIdx.y * a.B + p.b) * scan_partial_values(a.F, a.S);
#pragma unroll
    for (int i = 0; i < kSL; ++i)
        if (p.active && i < p.states) pf[p.f * a.S + p.first + i] = gA[i];
    m.sg[p.wave][0][p.lane] = {gD, gbias};
    lds_barrier();
    if (p.wave == 0 && p.active) {
        float2 sum = {0.0f, 0.0f};
        for (int w = 0; w < NS; ++w) {
            sum.x += m.sg[w][0][p.lane].x;
            sum.y += m.sg[w][0][p.lane].y;
        }
        pf[a.F * a.S + p.f] = sum.x;
        pf[a.F * (a.S + 1) + p.f] = sum.y;
    }
}

// The sums of the partial results: those of dL/dA, dL/dD and dL/d(dt_bias) over segments and
// sequences in the first `reduce` workgroups, dL/dB and dL/dC over a group's tiles in the others.
constexpr int kJoin = 1024;

template <int IO>
__global__ __launch_bounds__(kJoin) void scan_join_kernel(ScanArgs a, ReduceOut out, int64_t reduce, int64_t n) {
    __shared__ float lds[kJoin];
    const int64_t block = int64_t(blockIdx.z) * a.layer + blockIdx.x;
    if (block < reduce)
        return reduce_partials(a.part_f, a.plan.segments * a.B, scan_partial_values(a.F, a.S), out, block, lds);
    const int64_t i = (block - reduce) * kJoin + threadIdx.x;
    if (i >= n) return;
    const int waves = a.plan.waves, s = int(i % a.S);
    const int64_t q = i / a.S, which = q & 1, r = q >> 1;
    const int64_t g = r % a.G, tb = r / a.G, b = tb % a.B, t = tb / a.B;
    float sum = 0.0f;
    if (t < steps_of(a.lengths, b, a.T)) {
        const int64_t stride = a.T * a.B * a.G * waves * 2 * kSL;
        const float* part = a.part_bc + (r * waves + s / kSL) * 2 * kSL + which * kSL + s % kSL;
        for (int64_t j = 0; j < a.plan.tiles; ++j) sum += part[j * stride];
    }
    store1<IO>(at_out<IO>(which ? a.gC : a.gB, t, b, g * a.S + s), sum);
}

template <int IO, int NS, bool FULL>
snn_status backward_launch(const ScanArgs& a, hipStream_t s) {
    ScanArgs arg = a;
    void* argv[] = {&arg};
    const dim3 grid = scan_grid(a.plan, a.B, a.G, a.plan.segments);
    const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(scan_backward_kernel<IO, NS, FULL>), grid,
                                         dim3(NS * kWave), argv, sizeof(BackwardLds<NS>), s);
    return e == hipSuccess ? SNN_OK : SNN_E_LAUNCH;
}

template <int IO, bool FULL>
snn_status backward_states(const ScanArgs& a, hipStream_t s) {
    switch (a.plan.waves) {
        case 1: return backward_launch<IO, 1, FULL>(a, s);
        case 2: return backward_launch<IO, 2, FULL>(a, s);
        case 4: return backward_launch<IO, 4, FULL>(a, s);
        case 8: return backward_launch<IO, 8, FULL>(a, s);
        default: return backward_launch<IO, 16, FULL>(a, s);
    }
}

template <int IO>
snn_status backward_io(const ScanArgs& a, hipStream_t s) {
    const snn_status st = a.S % kSL == 0 ? backward_states<IO, true>(a, s) : backward_states<IO, false>(a, s);
    if (st != SNN_OK) return st;
    const ReduceOut out = {{a.gA, a.gD, a.gdt_bias}, {a.F * a.S, a.F, a.F}};
    const int64_t reduce = ceil_div(scan_partial_values(a.F, a.S), kWave), n = a.T * a.B * a.G * 2 * a.S;
    const dim3 grid = layered_grid(reduce + ceil_div(n, kJoin), kJoin);
    ScanArgs join = a;
    join.layer = grid.x;
    return launch_blk(scan_join_kernel<IO>, grid, kJoin, s, join, out, reduce, n);
}

}  // namespace

snn_status scan_backward_entry(int io, const ScanArgs& a, hipStream_t s) {
    return io == SNN_IO_F32 ? backward_io<SNN_IO_F32>(a, s) : backward_io<SNN_IO_BF16>(a, s);
}

}  // namespace snnlif
