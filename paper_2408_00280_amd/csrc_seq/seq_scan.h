// What the scan's kernels share.
#pragma once
#include "seq_device.h"

namespace snnlif {

constexpr int kSL = kScanStates;   // states per lane

// The workgroup's place: 64 features of a group, one sequence, one segment of its steps.
struct ScanPlace {
    int lane, wave;
    int64_t g, tile, b;
    int64_t f;        // this lane's feature (the group's last for lanes behind it)
    bool active;
    int first, states;   // this wave's states
    int t0, t1, len;     // the segment, and the steps of the sequence
};

// The workgroup's number, and whether it has work: a grid of several layers ends with some that have none.
__device__ __forceinline__ unsigned scan_block(const ScanArgs& a) { return blockIdx.z * a.layer + blockIdx.x; }
__device__ __forceinline__ bool scan_has_block(const ScanArgs& a) {
    return scan_block(a) < unsigned(a.plan.tiles) * unsigned(a.G) * unsigned(a.B);
}

__device__ __forceinline__ ScanPlace scan_place(const ScanArgs& a, int first_segment = 0) {
    ScanPlace p;
    p.lane = threadIdx.x & (kWave - 1);
    p.wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const unsigned i = scan_block(a), tiles = unsigned(a.plan.tiles), per = unsigned(a.F / a.G);
    const unsigned q = i / tiles;
    p.tile = i % tiles;
    p.g = q % unsigned(a.G);
    p.b = q / unsigned(a.G);
    const unsigned j = unsigned(p.tile) * kWave + p.lane;
    p.active = j < per;
    p.f = p.g * per + (p.active ? j : per - 1);
    p.first = p.wave * kSL;
    p.states = min(kSL, a.S - p.first);
    p.t0 = int((blockIdx.y + first_segment) * a.plan.steps);
    p.t1 = int(min(a.T, p.t0 + a.plan.steps));
    p.len = __builtin_amdgcn_readfirstlane(steps_of(a.lengths, p.b, a.T));
    return p;
}

// Where S is not whole lanes (FULL = false in the kernels), the last wave leaves its states
// behind the last one out of its sums: B = C = 0 there, which gives 0 with finite values only.

// A log2(e), kept finite: steps behind a sequence's end have d = 0 and are to leave the state as
// it is, which 2^(0 A) does not where A is infinite or becomes so with the factor.
__device__ __forceinline__ float rate_of(float A) {
    const float r = A * kLog2e;
    return fabsf(r) == __builtin_inff() ? copysignf(__FLT_MAX__, r) : r;
}

// The rates of the lane's states, 0 behind the last.
__device__ __forceinline__ void load_rates(const ScanArgs& a, const ScanPlace& p, float (&r)[kSL]) {
#pragma unroll
    for (int i = 0; i < kSL; ++i) r[i] = i < p.states ? rate_of(a.A[p.f * a.S + p.first + i]) : 0.0f;
}

__device__ __forceinline__ void load_state(const ScanArgs& a, const ScanPlace& p, const float* from, float (&h)[kSL]) {
#pragma unroll
    for (int i = 0; i < kSL; ++i)
        h[i] = from != nullptr && i < p.states ? from[(p.b * a.F + p.f) * a.S + p.first + i] : 0.0f;
}

__device__ __forceinline__ void store_state(const ScanArgs& a, const ScanPlace& p, float* to, const float (&h)[kSL]) {
#pragma unroll
    for (int i = 0; i < kSL; ++i)
        if (p.active && i < p.states) to[(p.b * a.F + p.f) * a.S + p.first + i] = h[i];
}

// States by piece c of the time axis, features next to each other and whole waves' states:
// [c][b][wave][4][f].
struct StateColumn {
    float* p;
    int64_t piece, F;
    __device__ StateColumn(const ScanArgs& a, const ScanPlace& s, float* base) : F(a.F) {
        const int64_t waves = scan_held_states(a.S) / kSL;
        p = base + (s.b * waves + s.wave) * kSL * F + s.f;
        piece = a.B * waves * kSL * F;
    }
    __device__ void load(int64_t c, float (&h)[kSL]) const {
#pragma unroll
        for (int i = 0; i < kSL; ++i) h[i] = p[c * piece + i * F];
    }
    __device__ void store(int64_t c, const float (&h)[kSL]) const {
#pragma unroll
        for (int i = 0; i < kSL; ++i) p[c * piece + i * F] = h[i];
    }
};

// 2^x h over a segment, of half x, the sum of its steps times the rate.  The decays of a whole
// segment may multiply to 0 or to infinity in 32 bits where no step's does.  As the root twice, kept
// finite and above 0, they leave a state that is 0 or not finite as it is, as step by step, and
// take any other out of the type only where their product does.
__device__ __forceinline__ float decayed(float half, float h) {
    const float root = __builtin_amdgcn_fmed3f(__builtin_amdgcn_exp2f(half), __FLT_MIN__, __FLT_MAX__);
    return h * root * root;
}

// The state before this segment, or e behind it (DOWN): the workgroup walks the others' states and
// sums of d itself, or the carry kernel has walked them.
template <bool DOWN>
__device__ __forceinline__ void segment_state(const ScanArgs& a, const ScanPlace& p, const float (&rate)[kSL],
                                              float (&h)[kSL]) {
    StateColumn states(a, p, a.part_h);
    if (!a.walk) {
        if (p.states > 0) states.load(blockIdx.y, h);
        return;
    }
    load_state(a, p, DOWN ? a.gh_out : a.h_in, h);
    if (p.states <= 0) return;
    const int last = int(a.plan.segments) - 1, n = DOWN ? last - int(blockIdx.y) : int(blockIdx.y);
    const float* sums = a.part_d + ((DOWN ? last * a.B : 0) + p.b) * a.F + p.f;
    if (DOWN) states.p += last * states.piece;
    constexpr int U = 4, DIR = DOWN ? -1 : 1;
    for (int c0 = 0; c0 < n; c0 += U) {
        float l[U][kSL], d[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (c0 + u < n) {
                states.load(0, l[u]);
                d[u] = *sums;
                states.p += DIR * states.piece;
                sums += DIR * a.B * a.F;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (c0 + u < n) {
#pragma unroll
                for (int s = 0; s < kSL; ++s) h[s] = decayed(0.5f * d[u] * rate[s], h[s]) + l[u][s];
            }
        }
    }
}

// The lanes' columns of a [T][B][F] tensor: a row's address is the same for the whole wave and
// stays in scalar registers, a lane adds the offset of its feature.
template <int IO>
struct Columns {
    static constexpr int kBytes = IO == SNN_IO_F32 ? 4 : 2;
    const char* base;
    int64_t step;    // bytes
    unsigned lane;   // bytes
    __device__ Columns(const Rows& r, const ScanPlace& s)
        : base(static_cast<const char*>(r.p) + s.b * r.b * kBytes), step(r.t * kBytes), lane(unsigned(s.f) * kBytes) {}
    __device__ const char* row(int t) const {
        int64_t at = t * step;
        asm("" : "+s"(at));      // or the product moves to the vector ALU, as one with the lane's offset
        return base + at;
    }
    __device__ auto load(int t) const { return IoVec<IO, 1>::load(row(t) + lane, 0); }
    __device__ void store(int t, float v) const { store1<IO>(const_cast<char*>(row(t) + lane), v); }
};

// B and C of one step and group are the same for every lane of a wave.  Each block of steps is
// staged in LDS as float32, 4 of B and 4 of C per wave (zeros behind the last state and behind
// the sequence's end), one value per thread (two in 16-step blocks), and read back 16 bytes at a
// time with every lane at the same address.  Scalar loads, which would need no vector register,
// take too long to come to hide behind the few steps whose values fit the scalar registers.
template <int NS, int K>
struct StagedBC {
    static constexpr int N = K * 2 * kSL / kWave;    // values per thread
    float v[K][NS][2 * kSL];
};

template <int IO, int NS, int K>
struct BCColumns {
    static constexpr int N = StagedBC<NS, K>::N, kApart = kWave / (2 * kSL);   // steps between a thread's values
    const char* p;       // of the next block to fetch
    int64_t step;
    int k;
    bool in;
    typename IoVec<IO, 1>::raw raw[N];
    __device__ BCColumns(const ScanArgs& a, const ScanPlace& s, int t0) {
        const int j = threadIdx.x % (NS * 2 * kSL), n = j / (2 * kSL) * kSL + j % kSL;
        const Rows& r = (j & kSL) ? a.Cm : a.Bm;
        k = threadIdx.x / (NS * 2 * kSL);
        in = n < a.S;
        step = r.t * (IO == SNN_IO_F32 ? 4 : 2);
        p = static_cast<const char*>(at<IO>(r, t0 + k, s.b, s.g * a.S + (in ? n : 0)));
    }
    // Blocks one after the other, up (DIR = 1) or down the time axis.
    template <int DIR>
    __device__ void fetch(int t0, int first, int len) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (in && t0 >= first && t0 + k + i * kApart < len) raw[i] = IoVec<IO, 1>::load(p + i * kApart * step, 0);
        p += DIR * K * step;
    }
    __device__ void stage(int t0, int len, StagedBC<NS, K>& to) const {
#pragma unroll
        for (int i = 0; i < N; ++i)
            to.v[i * kApart + k][0][threadIdx.x % (NS * 2 * kSL)] =
                in && t0 + k + i * kApart < len ? IoVec<IO, 1>::get(raw[i], 0) : 0.0f;
    }
};

// Values loaded before a loop have come when it starts.  Left pending they are waited for at
// their use inside, in every round, and with them the loads and stores that the loop itself
// has under way by then.
__device__ __forceinline__ void settle(float& v) { asm volatile("" : "+v"(v)); }
template <int N>
__device__ __forceinline__ void settle(float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) settle(v[i]);
}

}  // namespace snnlif
