// Host side of the sequence operators (include/snn_seq.h): argument checks, the plans that
// size launches and workspaces, and the entries of the kernel translation units.  Plans
// depend only on the configuration and the shape, so that a forward, its backward and the
// size queries agree.
#pragma once
#include "lif_host.h"
#include "snn_seq.h"

#include <algorithm>

namespace snnlif {

constexpr int64_t kMaxSeqT = int64_t(1) << 30, kMaxSeqB = int64_t(1) << 24, kMaxSeqF = int64_t(1) << 24;
constexpr int64_t kMaxRows = int64_t(1) << 30, kMaxSpan = int64_t(1) << 44;
constexpr int kMaxTaps = 8, kMaxStates = 64;

inline snn_status check_io(int io) { return io == SNN_IO_F32 || io == SNN_IO_BF16 ? SNN_OK : SNN_E_PARAM; }
inline int64_t elem_bytes(int io) { return io == SNN_IO_F32 ? 4 : 2; }

inline snn_status check_seq_shape(int64_t T, int64_t B, int64_t F) {
    if (T < 0 || B < 0 || F < 0 || T > kMaxSeqT || B > kMaxSeqB || F > kMaxSeqF) return SNN_E_SHAPE;
    if (B > 0 && T > kMaxRows / B) return SNN_E_SHAPE;
    if (T > 0 && B > 0 && F > kMaxSpan / (T * B)) return SNN_E_SHAPE;
    return SNN_OK;
}

// Elements that a [T][B][X] tensor spans with its steps; -1 when a step is negative or the
// span is too long.  The step of an axis of length 1 is not used.
inline int64_t seq_span(const snn_seq* s, int64_t T, int64_t B, int64_t X) {
    int64_t span = X;
    for (const auto& [n, step] : {std::pair<int64_t, int64_t>{T, s->t}, {B, s->b}}) {
        if (n <= 1) continue;
        if (step < 0 || step > kMaxSpan / (n - 1)) return -1;
        span += (n - 1) * step;
        if (span > kMaxSpan) return -1;
    }
    return span;
}

inline snn_status check_in(const snn_seq* s, int64_t T, int64_t B, int64_t X, int io) {
    if (s == nullptr || s->data == nullptr) return SNN_E_NULL;
    if (seq_span(s, T, B, X) < 0) return SNN_E_SHAPE;
    return aligned_to(s->data, uintptr_t(elem_bytes(io))) ? SNN_OK : SNN_E_ALIGN;
}

// An output's rows must not overlap: one axis steps over rows, the other over whole runs of
// the first.
inline snn_status check_out(const snn_seq* s, int64_t T, int64_t B, int64_t X, int io) {
    const snn_status st = check_in(s, T, B, X, io);
    if (st != SNN_OK) return st;
    const auto nested = [X](int64_t n_in, int64_t in, int64_t n_out, int64_t out) {
        return (n_in <= 1 || in >= X) && (n_out <= 1 || out >= (n_in <= 1 ? X : (n_in - 1) * in + X));
    };
    return nested(B, s->b, T, s->t) || nested(T, s->t, B, s->b) ? SNN_OK : SNN_E_SHAPE;
}

inline snn_status first_error(std::initializer_list<snn_status> all) {
    for (snn_status s : all)
        if (s == SNN_E_NULL) return s;      // as everywhere: NULL before the rest
    for (snn_status s : all)
        if (s != SNN_OK) return s;
    return SNN_OK;
}

inline snn_status need(const void* p, uintptr_t align = 4) {
    return p == nullptr ? SNN_E_NULL : aligned_to(p, align) ? SNN_OK : SNN_E_ALIGN;
}
inline snn_status optional(const void* p, uintptr_t align = 4) { return p == nullptr ? SNN_OK : need(p, align); }

// A [T][B][X] tensor as the kernels take it.
struct Rows {
    const void* p;
    int64_t t, b;
};
inline Rows rows(const snn_seq* s) { return s == nullptr ? Rows{nullptr, 0, 0} : Rows{s->data, s->t, s->b}; }

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr int64_t kMaxBlocks = INT32_MAX;

// A launch has fewer than 2^32 threads along x.
constexpr int64_t kMaxThreads = (int64_t(1) << 32) - 1;

// Workgroups in layers along z, where there are too many for one; those behind the last have
// nothing to do.  Kernels take blockIdx.z * layer + blockIdx.x, layer being the grid's x.
inline dim3 layered_grid(int64_t blocks, int threads, int64_t y = 1) {
    const int64_t layers = ceil_div(blocks, (int64_t(1) << 31) / threads);
    return dim3(unsigned(ceil_div(blocks, layers)), unsigned(y), unsigned(layers));
}

// Bytes of a piece of a workspace: pieces start on 256-byte boundaries.
inline int64_t piece(int64_t bytes) { return (bytes + 255) / 256 * 256; }

// Sums of P partial results of n values each, in a fixed order: out[i] = sum_p part[p*stride + i].
// The n values go to up to three arrays one after the other (an array may be NULL).
struct ReduceOut {
    float* p[3];
    int64_t n[3];
};
snn_status reduce_entry(const float* part, int64_t P, int64_t stride, const ReduceOut& out, hipStream_t s);

// -- convolution -------------------------------------------------------------------------
inline snn_status check_conv_cfg(const snn_conv_cfg* c) {
    if (c == nullptr) return SNN_E_NULL;
    if (check_io(c->io) != SNN_OK || c->width < 1 || c->width > kMaxTaps) return SNN_E_PARAM;
    return c->act == SNN_ACT_NONE || c->act == SNN_ACT_SILU ? SNN_OK : SNN_E_PARAM;
}

// Lanes own V neighbouring features (the few left over one each) and walk `steps` steps of one
// sequence, U rows at a time; there are `chunks` such pieces of the time axis.  2^18 lanes in
// the forward and 2^17 in the backward, which holds more of a chunk and leaves a partial sum
// for each, did best of 2^16 to 2^19 (x[2048][8][4096] bf16: 62.5 of 62-74 us, 97 of 97-122 us).
// A chunk has U steps at least, as W-1 of them are read twice.
struct ConvPlan {
    int64_t lanes;   // per sequence and chunk
    int64_t steps, chunks;
};

constexpr int conv_vec(int io, bool backward) { return io == SNN_IO_F32 || backward ? 4 : 8; }
constexpr int conv_rows(bool backward) { return backward ? 4 : 8; }

inline ConvPlan conv_plan(const snn_conv_cfg* c, int64_t T, int64_t B, int64_t F, bool backward) {
    const int v = conv_vec(c->io, backward);
    ConvPlan p;
    p.lanes = F / v + F % v;
    const int64_t want = ceil_div(int64_t(1) << (backward ? 17 : 18), p.lanes * B);
    p.steps = std::max<int64_t>(8, ceil_div(T, want));
    p.chunks = ceil_div(T, p.steps);
    return p;
}

inline int64_t conv_partial(const snn_conv_cfg* c, int64_t F) { return F * (c->width + 1); }

inline int64_t conv_workspace(const snn_conv_cfg* c, int64_t T, int64_t B, int64_t F) {
    return piece(conv_plan(c, T, B, F, true).chunks * B * conv_partial(c, F) * 4);
}

struct ConvArgs {
    int64_t T, B, F;
    Rows x, y, gy, gx;      // y: forward; gy, gx: backward
    const float* weight;
    const float* bias;
    const void* state_in;
    const int32_t* lengths;
    void* state_out;        // forward
    const void* gstate_out; // backward
    void* gstate_in;
    float* part;
    ConvPlan plan;
};
snn_status conv_forward_entry(const snn_conv_cfg* c, const ConvArgs& a, hipStream_t s);
snn_status conv_backward_entry(const snn_conv_cfg* c, const ConvArgs& a, hipStream_t s);

// -- scan --------------------------------------------------------------------------------
inline snn_status check_scan_cfg(const snn_scan_cfg* c) {
    if (c == nullptr) return SNN_E_NULL;
    if (check_io(c->io) != SNN_OK || c->states < 1 || c->states > kMaxStates || c->groups < 1) return SNN_E_PARAM;
    return c->softplus == 0 || c->softplus == 1 ? SNN_OK : SNN_E_PARAM;
}

constexpr int kScanStates = 4;   // states per lane
constexpr int kScanBlock = 8;    // steps that the waves of the local pass share out at a time
constexpr int64_t kSplitWaves = 1024, kSplitGroups = 128, kSplitSteps = 128, kMaxSegments = 1024;
// Up to so many segments a workgroup of the scan walks those before its own itself (not on a state
// updated in place: scan_walks); a kernel that walks them all first costs a launch more and pays
// behind that (x[4096][1][1024], 64 segments: 60 us to 60 and the launch; x[1000][8][128], 32: 70
// to 77; x[4096][1][512], 128: 55 to 48).
constexpr int64_t kWalkSegments = 64;

// A workgroup owns 64 features of one group and one sequence, a feature per lane; each of its
// `waves` (a power of two) waves holds 4 of their states.  The forward keeps the state every
// `keep` steps for the backward, which holds that many steps' decays in registers: 16, but 8
// where 16 waves leave a wave half the registers, and where 1 or 2 waves stage a block's steps.
struct ScanPlan {
    int waves;
    int keep;
    int64_t tiles;      // workgroups per group
    int64_t steps;      // per segment of the time axis
    int64_t segments;
};

constexpr int scan_keep(int waves) { return waves == 4 || waves == 8 ? 16 : 8; }

// States as they are kept: whole lanes.
constexpr int64_t scan_held_states(int S) { return int64_t(S + kScanStates - 1) / kScanStates * kScanStates; }

// The time axis is cut into segments where the waves of one segment leave SIMDs (1024 of them)
// without two waves, or its workgroups half the CUs without one: the local pass then costs less
// than they do idle (x[4096][1][4096] runs in 154 us instead of 624; x[1024][8][4096], which has
// two waves per SIMD, gains nothing).  Four waves per SIMD are aimed for, with segments of 16
// steps or more (forward and backward of x[333][1][777], 7 states: 49 us, 58 with 32 or more),
// once the steps outweigh another launch.  Walking the segments takes a time per segment and the
// kernels one per step of them: their sum is least with about sqrt(2 T) segments (forward of
// x[4096][1][128]: 33 us with 86, 36 with 64 and 44 with 256; x[131072][1][64]: 147 us with 512,
// 165 with 362 and 164 with 724).
inline ScanPlan scan_plan(const snn_scan_cfg* c, int64_t T, int64_t B, int64_t F) {
    ScanPlan p;
    p.waves = 1;
    while (p.waves * kScanStates < c->states) p.waves *= 2;
    p.keep = scan_keep(p.waves);
    p.tiles = ceil_div(F / c->groups, kWave);
    p.steps = std::max<int64_t>(T, 1);
    p.segments = 1;
    const int64_t groups = p.tiles * c->groups * B, waves = groups * (scan_held_states(c->states) / kScanStates);
    const int64_t most = std::min({ceil_div(T, 16), int64_t(std::sqrt(2.0 * double(T))), kMaxSegments});
    const int64_t want = std::min(std::max<int64_t>(4096 / waves, 2), most);
    if ((waves <= kSplitWaves || groups <= kSplitGroups) && T >= kSplitSteps && want > 1) {
        p.steps = ceil_div(ceil_div(T, want), 16) * 16;      // whole blocks, in either direction
        if (p.waves == 16) {
            // One such workgroup fills a CU: the fewest rounds of the 256, weighed with their length
            // and 16 steps for a segment's start (x[442][2][2928] of 47 states, forward and backward:
            // 370 us with 5 segments, two rounds, 428 with 3, which are two as well).  8 waves
            // share a CU in the forward and lose there what the backward gains.
            const auto cost = [&](int64_t steps) { return ceil_div(groups * ceil_div(T, steps), 256) * (steps + 16); };
            // Half to twice the length; of as many segments the shortest are the cheapest.
            const auto blocks = [](int64_t steps) { return ceil_div(steps, 16) * 16; };
            const int64_t last = std::min(2 * p.steps, T - 1);
            int64_t steps = std::max({p.steps / 32 * 16, blocks(ceil_div(T, most)), int64_t(16)}), least = cost(p.steps);
            while (steps <= last) {
                if (const int64_t now = cost(steps); now < least) {
                    least = now;
                    p.steps = steps;
                }
                const int64_t n = ceil_div(T, steps);       // 2 at least, as steps < T
                steps = std::max(steps + 16, blocks(ceil_div(T, n - 1)));
            }
        }
        p.segments = ceil_div(T, p.steps);
    }
    return p;
}

inline int64_t scan_saved(const snn_scan_cfg* c, const ScanPlan& p, int64_t T, int64_t B, int64_t F) {
    return (ceil_div(T, p.keep) - 1) * B * F * scan_held_states(c->states) * 4;
}
inline int64_t scan_saved(const snn_scan_cfg* c, int64_t T, int64_t B, int64_t F) {
    return scan_saved(c, scan_plan(c, T, B, F), T, B, F);
}
// The segments' states and their sums of d.
inline int64_t scan_part_h(const snn_scan_cfg* c, const ScanPlan& p, int64_t B, int64_t F) {
    return p.segments > 1 ? p.segments * B * F * scan_held_states(c->states) * 4 : 0;
}
inline int64_t scan_part_d(const ScanPlan& p, int64_t B, int64_t F) { return p.segments > 1 ? p.segments * B * F * 4 : 0; }
inline int64_t scan_forward_workspace(const snn_scan_cfg* c, const ScanPlan& p, int64_t B, int64_t F) {
    return piece(scan_part_h(c, p, B, F)) + piece(scan_part_d(p, B, F));
}
inline int64_t scan_forward_workspace(const snn_scan_cfg* c, int64_t T, int64_t B, int64_t F) {
    return scan_forward_workspace(c, scan_plan(c, T, B, F), B, F);
}
constexpr int64_t scan_partial_values(int64_t F, int S) { return F * (S + 2); }
// dL/dB and dL/dC of every tile, as the waves hold them.
inline int64_t scan_partial_bc(const snn_scan_cfg* c, const ScanPlan& p, int64_t T, int64_t B) {
    return p.tiles * T * B * c->groups * p.waves * 2 * kScanStates * 4;
}
inline int64_t scan_backward_workspace(const snn_scan_cfg* c, const ScanPlan& p, int64_t T, int64_t B, int64_t F) {
    return piece(scan_part_h(c, p, B, F)) + piece(scan_part_d(p, B, F)) + piece(scan_partial_bc(c, p, T, B)) +
           piece(p.segments * B * scan_partial_values(F, c->states) * 4);
}
inline int64_t scan_backward_workspace(const snn_scan_cfg* c, int64_t T, int64_t B, int64_t F) {
    return scan_backward_workspace(c, scan_plan(c, T, B, F), T, B, F);
}

// Whether the scan's workgroups walk the segments before their own themselves, from the state at
// `from`.  In place the last segment's workgroup writes the state that the others start from, and
// nothing orders it behind them: then the carry kernel walks them, which has read the state
// before the scan starts.  One segment has no others, and its workgroups alone touch their state.
inline bool scan_walks(const ScanPlan& p, const void* from, const void* to) {
    return p.segments == 1 || (p.segments <= kWalkSegments && (to == nullptr || to != from));
}

struct ScanArgs {
    int64_t T, B, F;
    int S, G, softplus;
    bool walk;       // several segments: the workgroups walk them themselves
    Rows x, dt, Bm, Cm, y, gy, gx, gdt, gB, gC;
    const float *A, *D, *dt_bias, *h_in;
    const int32_t* lengths;
    float* h_out;
    float* saved;
    const float* gh_out;
    float *gA, *gD, *gdt_bias, *gh_in;
    float* part_bc;  // backward: [tiles][T][B][G][waves][B, C][4]
    float* part_f;   // backward: [segments][B] x (A [F][S], D [F], dt_bias [F])
    float* part_h;   // several segments: [segments][B][states][F] and [segments][B][F]
    float* part_d;
    ScanPlan plan;
    unsigned layer;  // workgroups of a layer of the grid
};
// Of the kernels whose workgroups own 64 features each.
inline dim3 scan_grid(const ScanPlan& p, int64_t B, int64_t G, int64_t segments) {
    return layered_grid(p.tiles * G * B, p.waves * kWave, segments);
}
snn_status scan_split_entry(int io, bool down, const ScanArgs& a, hipStream_t s);
snn_status scan_forward_entry(int io, const ScanArgs& a, hipStream_t s);
snn_status scan_backward_entry(int io, const ScanArgs& a, hipStream_t s);

// -- norm --------------------------------------------------------------------------------
inline snn_status check_norm_cfg(const snn_norm_cfg* c) {
    if (c == nullptr) return SNN_E_NULL;
    return check_io(c->io) == SNN_OK && c->eps > 0.0f && std::isfinite(c->eps) ? SNN_OK : SNN_E_PARAM;
}

// Rows of up to 8192 features stay in registers, 8 features per lane; longer ones are walked in
// pieces of that.
constexpr int kNormLane = 8, kNormRegs = 1024 * kNormLane;

inline int norm_lanes(int64_t F) {
    return int(ceil_div(std::min<int64_t>(F, kNormRegs), kNormLane * kWave) * kWave);
}

// Workgroups walk rows g, g + groups, ..., so that parameters are read once.  The backward's
// hold one partial sum of their gradients each, which 3 rows are to share at least (1250 rows of
// 1537 fp32 features: 28 us with the sums joined, to 37 with 1 or 2, and 30 with 4).  Up to 32
// waves per CU in the forward and 16 in the backward: whole rounds of the rows count for more.
inline int64_t norm_groups(int64_t T, int64_t B, int64_t F, bool backward) {
    const int64_t most = ceil_div(256 * (backward ? 16 : 32), norm_lanes(F) / kWave);
    return std::min<int64_t>(backward ? ceil_div(T * B, 3) : T * B, most);
}
inline int64_t norm_workspace(int64_t T, int64_t B, int64_t F) { return piece(norm_groups(T, B, F, true) * 3 * F * 4); }

struct NormArgs {
    int64_t T, B, F;
    float eps;
    Rows y, z, r, r_new, u, gr_new, gu, gy, gz, gr;
    const float *w_post, *scale, *w_pre;
    const int32_t* lengths;
    const float* rstd_in;
    float* rstd;
    float *gw_post, *gscale, *gw_pre;
    float* part;
    int64_t groups;
};
snn_status norm_forward_entry(int io, const NormArgs& a, hipStream_t s);
snn_status norm_backward_entry(int io, const NormArgs& a, hipStream_t s);

}  // namespace snnlif
