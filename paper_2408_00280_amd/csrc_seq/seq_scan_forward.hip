// Selective state space scan, forward.
//
// Per step, feature and state: a = 2^(d A log2 e), h = a h + (d x) B, y += C h: five vector
// instructions, one of them an exponential at half rate.  With S = 16 states that is more
// work than the few bytes per feature and step need to move, so the kernel is bound by the
// vector ALU.  A lane is a feature and each wave of a workgroup holds 4 of its states in
// registers.  What belongs to a step but not to a state (the softplus, B and C, the sum of y
// over the waves) is shared out over the waves, K steps at a time, through LDS: while a
// block's steps run, the one after the next is loaded, and staged before the barrier that
// parts two blocks.  The vector ALU is 70 to 85% busy (x[1024][8][4096] bf16: 190 us).
#include "seq_scan.h"

namespace snnlif {
namespace {

template <int IO, int NS, int K, bool FULL>
__global__ __launch_bounds__(NS * kWave) void scan_forward_kernel(ScanArgs a) {
    constexpr int R = K > NS ? K / NS : 1, U = 2;   // U: steps read from LDS ahead
    __shared__ float2 sd[3][K][kWave];           // (d, d x): of this block, the next and the one being staged
    __shared__ float sy[2][NS][K][kWave];
    __shared__ __align__(16) StagedBC<NS, K> sbc[3];
    if (!scan_has_block(a)) return;
    const ScanPlace p = scan_place(a);
    float rate[kSL], h[kSL];
    load_rates(a, p, rate);
    segment_state<false>(a, p, rate, h);
    float skip = a.D != nullptr ? a.D[p.f] : 0.0f, bias = a.dt_bias != nullptr ? a.dt_bias[p.f] : 0.0f;
    settle(skip);
    settle(bias);
    settle(rate);
    settle(h);
    const Columns<IO> cx(a.x, p), cdt(a.dt, p), cy(a.y, p);
    BCColumns<IO, NS, K> cbc(a, p, p.t0);
    const StateColumn kept(a, p, a.saved);
    const bool busy = p.states > 0;              // waves behind the last state only share the rest
    const int used = (a.S + kSL - 1) / kSL;

    typename IoVec<IO, 1>::raw xr[R], dr[R];
    float xs[3][R];                              // D x of this wave's steps
    const auto fetch = [&](int t0) {
        cbc.template fetch<1>(t0, p.t0, p.len);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int k = p.wave + r * NS;
            if (k < K && t0 + k < p.len) {
                xr[r] = cx.load(t0 + k);
                dr[r] = cdt.load(t0 + k);
            }
        }
    };
    const auto stage = [&](int t0, int to, float (&skipped)[R]) {
        cbc.stage(t0, p.len, sbc[to]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int k = p.wave + r * NS;
            float2 d = {0.0f, 0.0f};             // behind the end: the state stays
            skipped[r] = 0.0f;
            if (k < K && t0 + k < p.len) {
                const float v = IoVec<IO, 1>::get(dr[r], 0) + bias, x = IoVec<IO, 1>::get(xr[r], 0);
                d.x = a.softplus ? softplus(v) : v;
                d.y = d.x * x;
                skipped[r] = a.D != nullptr ? skip * x : 0.0f;
            }
            if (k < K) sd[to][k][p.lane] = d;
        }
    };

    fetch(p.t0);
    stage(p.t0, 0, xs[0]);
    fetch(p.t0 + K);
    stage(p.t0 + K, 1, xs[1]);
    struct Step {
        float2 d;
        f32x4_t b, c;
    } step[U], ahead[U];
    const auto read = [&](int block, int k) {
        const f32x4_t* bc = reinterpret_cast<const f32x4_t*>(sbc[block].v[k][p.wave]);
        return Step{sd[block][k][p.lane], bc[0], bc[1]};
    };
    lds_barrier();
#pragma unroll
    for (int i = 0; i < U; ++i) step[i] = read(0, i);
    int now = 0, buf = 0;                        // block c: c % 3 and c % 2
    for (int t0 = p.t0; t0 < p.t1; t0 += K) {
        const int next = now == 2 ? 0 : now + 1, last = now == 0 ? 2 : now - 1;
        if (t0 < p.len) {
            if (a.saved != nullptr && t0 > 0 && (t0 & (a.plan.keep - 1)) == 0)
                if (busy && p.active) kept.store(t0 / a.plan.keep - 1, h);
            fetch(t0 + 2 * K);
            if (busy) {
#pragma unroll
                for (int u = 0; u < K; u += U) {
#pragma unroll
                    for (int i = 0; i < U; ++i)
                        ahead[i] = u + U < K ? read(now, u + U + i) : read(next, u + U - K + i);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int i = 0; i < U; ++i) {
                        float y = 0.0f;
#pragma unroll
                        for (int s = 0; s < kSL; ++s) {
                            h[s] = fmaf(__builtin_amdgcn_exp2f(step[i].d.x * rate[s]), h[s], step[i].d.y * step[i].b[s]);
                            y = FULL || s < p.states ? fmaf(step[i].c[s], h[s], y) : y;
                        }
                        sy[buf][p.wave][u + i][p.lane] = y;
                    }
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int i = 0; i < U; ++i) step[i] = ahead[i];
                }
            }
            // here, a block's steps after the last stores and the loads, neither is waited for long
            stage(t0 + 2 * K, last, xs[2]);
        }
        lds_barrier();
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int k = p.wave + r * NS;
            if (k < K && t0 + k < p.t1) {
                float y = 0.0f;
                if (t0 + k < p.len) {
                    float part[NS];
#pragma unroll
                    for (int w = 0; w < NS; ++w) part[w] = sy[buf][w][k][p.lane];
                    y = xs[0][r];
#pragma unroll
                    for (int w = 0; w < NS; ++w) y += w < used ? part[w] : 0.0f;
                }
                if (p.active) cy.store(t0 + k, y);
            }
            xs[0][r] = xs[1][r];
            xs[1][r] = xs[2][r];
        }
        now = next;
        buf ^= 1;
    }
    if (a.h_out != nullptr && p.t1 == a.T) store_state(a, p, a.h_out, h);
}

// Up to 4 states: one wave holds them all, so that steps and sums need no LDS and only B and C
// go through it; without the LDS of the shared form four times as many waves fit a CU.
template <int IO, bool FULL>
__global__ __launch_bounds__(kWave) void scan_forward_one_kernel(ScanArgs a) {
    constexpr int K = 8;
    __shared__ __align__(16) StagedBC<1, K> sbc[2];
    if (!scan_has_block(a)) return;
    const ScanPlace p = scan_place(a);
    float rate[kSL], h[kSL];
    load_rates(a, p, rate);
    segment_state<false>(a, p, rate, h);
    float skip = a.D != nullptr ? a.D[p.f] : 0.0f, bias = a.dt_bias != nullptr ? a.dt_bias[p.f] : 0.0f;
    settle(skip);
    settle(bias);
    settle(rate);
    settle(h);
    const Columns<IO> cx(a.x, p), cdt(a.dt, p), cy(a.y, p);
    const StateColumn kept(a, p, a.saved);
    BCColumns<IO, 1, K> cbc(a, p, p.t0);
    typename IoVec<IO, 1>::raw xr[K], dr[K];
    const auto fetch = [&](int t0) {
        cbc.template fetch<1>(t0, p.t0, p.len);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (t0 + k < p.len) {
                xr[k] = cx.load(t0 + k);
                dr[k] = cdt.load(t0 + k);
            }
        }
    };
    fetch(p.t0);
    int buf = 0;
    float ys[K];     // of the block before: stored once this block's loads have come, not waited for with them
    const auto put = [&](int t0) {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (t0 + k < p.len && p.active) cy.store(t0 + k, ys[k]);
    };
    for (int t0 = p.t0; t0 < p.t1; t0 += K, buf ^= 1) {
        const int n = min(K, p.len - t0);                        // steps inside the sequence
        if (n > 0) {
            if (a.saved != nullptr && t0 > 0 && (t0 & (a.plan.keep - 1)) == 0 && p.active)
                kept.store(t0 / a.plan.keep - 1, h);
            float x[K], d[K];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                x[k] = d[k] = 0.0f;                              // behind the end: the state stays
                if (k < n) {
                    const float v = IoVec<IO, 1>::get(dr[k], 0) + bias;
                    x[k] = IoVec<IO, 1>::get(xr[k], 0);
                    d[k] = a.softplus ? softplus(v) : v;
                }
            }
            cbc.stage(t0, p.len, sbc[buf]);
            if (t0 > p.t0) put(t0 - K);
            fetch(t0 + K);
            lds_barrier();
            const f32x4_t* bc = reinterpret_cast<const f32x4_t*>(sbc[buf].v[0][0]);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const f32x4_t b = bc[2 * k], c = bc[2 * k + 1];
                float y = a.D != nullptr ? skip * x[k] : 0.0f;
#pragma unroll
                for (int s = 0; s < kSL; ++s) {
                    h[s] = fmaf(__builtin_amdgcn_exp2f(d[k] * rate[s]), h[s], (d[k] * x[k]) * b[s]);
                    y = FULL || s < p.states ? fmaf(c[s], h[s], y) : y;
                }
                ys[k] = y;
            }
            if (t0 + K >= min(p.t1, p.len)) put(t0);             // the last block
        }
        for (int k = max(n, 0); k < K && t0 + k < p.t1; ++k)
            if (p.active) cy.store(t0 + k, 0.0f);
    }
    if (a.h_out != nullptr && p.t1 == a.T) store_state(a, p, a.h_out, h);
}

// One step: a feature's states lie over Q neighbouring lanes, 4 each, so that the state is read
// and written once, 16 bytes per lane and contiguously; y is their sum over the Q lanes.  A
// lane takes the same states of N sequences, whose loads are all in flight at once.  Bound by
// memory: the states are all but a few percent of what moves.
template <int IO, int Q, int N>
__global__ __launch_bounds__(kBlock) void scan_token_kernel(ScanArgs a) {
    const int64_t i = (int64_t(blockIdx.z) * a.layer + blockIdx.x) * kBlock + threadIdx.x;
    const unsigned F = unsigned(a.F), B = unsigned(a.B), n = (B + N - 1) / N * F, bf = min(unsigned(i / Q), n - 1);
    const bool active = i / Q < n;               // lanes behind the last feature compute it again
    const unsigned b0 = bf / F * N, f = bf % F, g = f / (F / unsigned(a.G));
    const int q = int(i) & (Q - 1), s0 = q * kSL, states = max(0, min(kSL, a.S - s0));
    const auto load4 = [&](const float* p, float (&v)[kSL]) {
        if (states == kSL) {
            const f32x4_t r = ld_nt<f32x4_t>(p);
#pragma unroll
            for (int j = 0; j < kSL; ++j) v[j] = r[j];
        } else {
#pragma unroll
            for (int j = 0; j < kSL; ++j) v[j] = j < states ? p[j] : 0.0f;
        }
    };
    const auto load_io = [&](const Rows& r, unsigned b, float (&v)[kSL]) {
        if (states == kSL) {
            load_vec<IO, kSL>(at<IO>(r, 0, b, int64_t(g) * a.S + s0), v);
        } else {
#pragma unroll
            for (int j = 0; j < kSL; ++j)
                v[j] = j < states ? load1<IO>(at<IO>(r, 0, b, int64_t(g) * a.S + s0 + j)) : 0.0f;
        }
    };
    float h[N][kSL], bv[N][kSL], cv[N][kSL], x[N], v[N], rate[kSL];
    bool on[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const unsigned b = b0 + k;
        on[k] = b < B && steps_of(a.lengths, b, a.T) > 0;
        if (b < B && a.h_in != nullptr) {
            load4(a.h_in + (int64_t(b) * F + f) * a.S + s0, h[k]);
        } else {
#pragma unroll
            for (int j = 0; j < kSL; ++j) h[k][j] = 0.0f;
        }
        if (on[k]) {
            load_io(a.Bm, b, bv[k]);
            load_io(a.Cm, b, cv[k]);
            x[k] = load1<IO>(at<IO>(a.x, 0, b, f));
            v[k] = load1<IO>(at<IO>(a.dt, 0, b, f));
        }
    }
    load4(a.A + int64_t(f) * a.S + s0, rate);
    const float bias = a.dt_bias != nullptr ? a.dt_bias[f] : 0.0f, skip = a.D != nullptr ? a.D[f] : 0.0f;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const unsigned b = b0 + k;
        float y = 0.0f;
        if (on[k]) {
            const float w = v[k] + bias, d = a.softplus ? softplus(w) : w;
#pragma unroll
            for (int j = 0; j < kSL; ++j) {
                h[k][j] = fmaf(__builtin_amdgcn_exp2f(d * rate_of(rate[j])), h[k][j], (d * x[k]) * bv[k][j]);
                y = j < states ? fmaf(cv[k][j], h[k][j], y) : y;
            }
            y = q == 0 && a.D != nullptr ? fmaf(skip, x[k], y) : y;
        }
        if (Q > 1) y += dpp<kDppXor1>(y);
        if (Q > 2) y += dpp<kDppXor2>(y);
        if (Q > 4) y += dpp<kDppHalfMirror>(y);
        if (Q > 8) y += dpp<kDppRor8>(y);
        if (!active || b >= B) continue;
        if (q == 0) store1<IO>(at_out<IO>(a.y, 0, b, f), y);
        if (a.h_out != nullptr) {
            float* to = a.h_out + (int64_t(b) * F + f) * a.S + s0;
            if (states == kSL) {
                const f32x4_t r = {h[k][0], h[k][1], h[k][2], h[k][3]};
                st_nt(to, r);
            } else {
#pragma unroll
                for (int j = 0; j < kSL - 1; ++j)
                    if (j < states) to[j] = h[k][j];
            }
        }
    }
}

template <int IO, int Q, int N>
snn_status token_sequences(ScanArgs a, hipStream_t s) {
    const dim3 grid = layered_grid(ceil_div(ceil_div(a.B, N) * a.F * Q, kBlock), kBlock);
    a.layer = grid.x;
    return launch(scan_token_kernel<IO, Q, N>, grid, s, a);
}

template <int IO, int Q>
snn_status token_lanes(const ScanArgs& a, hipStream_t s) {
    // several sequences per lane where that leaves 16 waves per CU
    if (a.B * a.F * Q >= int64_t(4) * 256 * 16 * kWave) return token_sequences<IO, Q, 4>(a, s);
    return token_sequences<IO, Q, 1>(a, s);
}

template <int IO>
snn_status token_states(const ScanArgs& a, hipStream_t s) {
    switch (a.plan.waves) {                      // the lanes per feature
        case 1: return token_lanes<IO, 1>(a, s);
        case 2: return token_lanes<IO, 2>(a, s);
        case 4: return token_lanes<IO, 4>(a, s);
        case 8: return token_lanes<IO, 8>(a, s);
        default: return token_lanes<IO, 16>(a, s);
    }
}

template <int IO, int NS, bool FULL>
snn_status forward_waves(const ScanArgs& a, hipStream_t s) {
    const dim3 grid = scan_grid(a.plan, a.B, a.G, a.plan.segments);
    if constexpr (NS == 1) return launch_blk(scan_forward_one_kernel<IO, FULL>, grid, kWave, s, a);
    // Up to two workgroups of four waves per CU have the LDS for blocks of 16 steps, whose
    // barriers are half as many (x[1024][8][4096]: 208 us to 219 with blocks of 8); more of
    // them hide the barriers themselves and need blocks of 8 to fit (x[4096][1][4096] in 16
    // segments: 89 us to 108 with blocks of 16).
    if constexpr (NS == 4) {
        if (int64_t(grid.x) * grid.y * grid.z <= 2 * 256)
            return launch_blk(scan_forward_kernel<IO, NS, 16, FULL>, grid, NS * kWave, s, a);
    }
    if constexpr (NS > 1) return launch_blk(scan_forward_kernel<IO, NS, 8, FULL>, grid, NS * kWave, s, a);
}

template <int IO, bool FULL>
snn_status forward_states(const ScanArgs& a, hipStream_t s) {
    switch (a.plan.waves) {
        case 1: return forward_waves<IO, 1, FULL>(a, s);
        case 2: return forward_waves<IO, 2, FULL>(a, s);
        case 4: return forward_waves<IO, 4, FULL>(a, s);
        case 8: return forward_waves<IO, 8, FULL>(a, s);
        default: return forward_waves<IO, 16, FULL>(a, s);
    }
}

template <int IO>
snn_status forward_io(const ScanArgs& a, hipStream_t s) {
    if (a.T == 1) return token_states<IO>(a, s);
    return a.S % kSL == 0 ? forward_states<IO, true>(a, s) : forward_states<IO, false>(a, s);
}

}  // namespace

snn_status scan_forward_entry(int io, const ScanArgs& a, hipStream_t s) {
    return io == SNN_IO_F32 ? forward_io<SNN_IO_F32>(a, s) : forward_io<SNN_IO_BF16>(a, s);
}

}  // namespace snnlif
