// Selective state space scan over segments of the time axis, for shapes whose features and
// sequences do not fill the chip.
//
// A segment turns the state h before it into (product of its decays) h + (its state from
// zero), and the product of decays is 2^(A log2 e sum of d): the local kernel forms the state
// from zero and the sum of d of every segment at once, and the scan then runs on all segments at
// once, each from its own state.  Where there are few segments and the state is not updated in
// place its workgroups walk those before their own themselves, else the carry kernel walks them
// all first.  The backward does the same from the end with e[t] = a[t+1] dL/dh[t+1].  The local
// pass costs four vector instructions per state and step (20 cycles to the forward's 24) on top of
// the scan's own.
#include "seq_scan.h"

namespace snnlif {
namespace {

// One segment from zero: up the time axis h = a h + d x B, or down it e = a (e + C dL/dy).
// The blocks are staged as in the scan.
template <int IO, int NS, bool DOWN>
__global__ __launch_bounds__(NS * kWave) void scan_local_kernel(ScanArgs a) {
    constexpr int K = kScanBlock, R = K > NS ? K / NS : 1, U = 2;
    __shared__ float2 sd[3][K][kWave];           // (d, d x), or (d, dL/dy)
    __shared__ __align__(16) StagedBC<NS, K> sbc[3];
    if (!scan_has_block(a)) return;
    // the first segment's state is not needed further down, nor the last one's further up
    const ScanPlace p = scan_place(a, DOWN ? 1 : 0);
    float bias = a.dt_bias != nullptr ? a.dt_bias[p.f] : 0.0f;
    const Columns<IO> cv(DOWN ? a.gy : a.x, p), cdt(a.dt, p);
    const StateColumn out(a, p, a.part_h);
    const bool busy = p.states > 0;
    const int blocks = (p.t1 - p.t0 + K - 1) / K;
    const auto start = [&](int c) { return p.t0 + (DOWN ? blocks - 1 - c : c) * K; };
    BCColumns<IO, NS, K> cbc(a, p, start(0));
    float rate[kSL], h[kSL], sum = 0.0f;
    load_rates(a, p, rate);
    settle(bias);
    settle(rate);
#pragma unroll
    for (int s = 0; s < kSL; ++s) h[s] = 0.0f;

    typename IoVec<IO, 1>::raw vr[R], dr[R];
    const auto fetch = [&](int c) {
        const int t0 = c < blocks ? start(c) : p.len;
        cbc.template fetch<DOWN ? -1 : 1>(t0, p.t0, p.len);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int k = p.wave + r * NS;
            if (k < K && t0 + k < p.len) {
                vr[r] = cv.load(t0 + k);
                dr[r] = cdt.load(t0 + k);
            }
        }
    };
    const auto stage = [&](int c, int to) {
        const int t0 = c < blocks ? start(c) : p.len;
        cbc.stage(t0, p.len, sbc[to]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int k = p.wave + r * NS;
            float2 d = {0.0f, 0.0f};
            if (k < K && t0 + k < p.len && t0 + k < p.t1) {
                const float v = IoVec<IO, 1>::get(dr[r], 0) + bias;
                d.x = a.softplus ? softplus(v) : v;
                d.y = IoVec<IO, 1>::get(vr[r], 0) * (DOWN ? 1.0f : d.x);
            }
            if (k < K) sd[to][k][p.lane] = d;
        }
    };
    struct Step {
        float2 d;
        f32x4_t v;
    } step[U], ahead[U];
    const auto read = [&](int block, int k) {
        const int j = DOWN ? K - 1 - k : k;
        const f32x4_t* bc = reinterpret_cast<const f32x4_t*>(sbc[block].v[j][p.wave]);
        return Step{sd[block][j][p.lane], bc[DOWN ? 1 : 0]};
    };
    fetch(0);
    stage(0, 0);
    fetch(1);
    stage(1, 1);
    fetch(2);
    lds_barrier();
#pragma unroll
    for (int i = 0; i < U; ++i) step[i] = read(0, i);
    int now = 0;
    for (int c = 0; c < blocks; ++c) {
        const int next = now == 2 ? 0 : now + 1, last = now == 0 ? 2 : now - 1;
        stage(c + 2, last);
        fetch(c + 3);
        if (busy) {
#pragma unroll
            for (int u = 0; u < K; u += U) {
#pragma unroll
                for (int i = 0; i < U; ++i) ahead[i] = u + U < K ? read(now, u + U + i) : read(next, u + U - K + i);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    sum += step[i].d.x;
#pragma unroll
                    for (int s = 0; s < kSL; ++s) {
                        const float dec = __builtin_amdgcn_exp2f(step[i].d.x * rate[s]);
                        h[s] = DOWN ? dec * fmaf(step[i].v[s], step[i].d.y, h[s])
                                    : fmaf(dec, h[s], step[i].d.y * step[i].v[s]);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < U; ++i) step[i] = ahead[i];
            }
        }
        lds_barrier();
        now = next;
    }
    if (busy && p.active) {
        const int64_t seg = p.t0 / a.plan.steps;
        out.store(seg, h);
        if (p.wave == 0) a.part_d[(seg * a.B + p.b) * a.F + p.f] = sum;
    }
}

// A lane per sequence, state and feature walks the segments.  On return part_h[c] is the state
// before segment c (or e behind it), and the last one goes to h_out (gh_in).
template <bool DOWN>
__global__ __launch_bounds__(kBlock) void scan_carry_kernel(ScanArgs a, int64_t n) {
    const int64_t i = int64_t(blockIdx.x) * kBlock + threadIdx.x;
    if (i >= n) return;
    const int64_t states = n / (a.B * a.F), f = i % a.F, q = i / a.F, s = q % states, b = q / states;
    const bool in = s < a.S;
    const float rate = in ? rate_of(a.A[f * a.S + s]) : 0.0f;
    const float* from = DOWN ? a.gh_out : a.h_in;
    float h = in && from != nullptr ? from[(b * a.F + f) * a.S + s] : 0.0f;
    constexpr int U = 16;     // in flight at once (256 segments: 27 us, 41 with 4)
    for (int64_t c0 = 0; c0 < a.plan.segments; c0 += U) {
        float local[U], d[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (c0 + u + 1 < a.plan.segments) {
                const int64_t c = DOWN ? a.plan.segments - 1 - c0 - u : c0 + u;
                local[u] = a.part_h[c * n + i];
                d[u] = a.part_d[(c * a.B + b) * a.F + f];
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (c0 + u < a.plan.segments) {
                a.part_h[(DOWN ? a.plan.segments - 1 - c0 - u : c0 + u) * n + i] = h;
                if (c0 + u + 1 < a.plan.segments) h = decayed(0.5f * d[u] * rate, h) + local[u];
            }
        }
    }
}

template <int IO, bool DOWN, int NS>
snn_status local(const ScanArgs& a, hipStream_t s) {
    const dim3 grid = scan_grid(a.plan, a.B, a.G, a.plan.segments - 1);
    return launch_blk(scan_local_kernel<IO, NS, DOWN>, grid, NS * kWave, s, a);
}

template <int IO, bool DOWN>
snn_status split(const ScanArgs& a, hipStream_t s) {
    snn_status st;
    switch (a.plan.waves) {
        case 1: st = local<IO, DOWN, 1>(a, s); break;
        case 2: st = local<IO, DOWN, 2>(a, s); break;
        case 4: st = local<IO, DOWN, 4>(a, s); break;
        case 8: st = local<IO, DOWN, 8>(a, s); break;
        default: st = local<IO, DOWN, 16>(a, s); break;
    }
    if (st != SNN_OK || a.walk) return st;
    const int64_t n = a.B * scan_held_states(a.S) * a.F;
    return launch(scan_carry_kernel<DOWN>, grid_for(n), s, a, n);
}

}  // namespace

snn_status scan_split_entry(int io, bool down, const ScanArgs& a, hipStream_t s) {
    if (down) return io == SNN_IO_F32 ? split<SNN_IO_F32, true>(a, s) : split<SNN_IO_BF16, true>(a, s);
    return io == SNN_IO_F32 ? split<SNN_IO_F32, false>(a, s) : split<SNN_IO_BF16, false>(a, s);
}

}  // namespace snnlif
