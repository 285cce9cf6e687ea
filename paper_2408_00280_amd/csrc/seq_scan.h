// What the scan's kernels share.
#pragma once
#include "seq_device.h"

namespace snnlif {

constexpr int kSL = 4;   // states per lane

// B and C of one step and group are the same for every lane of a wave: they are packed
// beforehand as float32 (4 per wave, zeros behind the last state) and read through the scalar
// cache, so that they cost no vector register and no vector instruction.
typedef const __attribute__((address_space(4))) f32x4_t* scalar_f32x4;

__device__ __forceinline__ f32x4_t scalar_load4(const float* p) {
    return *(scalar_f32x4)(reinterpret_cast<uintptr_t>(p));
}

// The workgroup's place: 64 features of a group, one sequence.
struct ScanPlace {
    int lane, wave;
    int64_t g, tile, b;
    int64_t f;        // this lane's feature (the group's last for lanes behind it)
    bool active;
};

__device__ __forceinline__ ScanPlace scan_place(const ScanArgs& a) {
    ScanPlace p;
    p.lane = threadIdx.x & (kWave - 1);
    p.wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t i = blockIdx.x, per = a.F / a.G;
    p.tile = i % a.plan.tiles;
    p.g = i / a.plan.tiles % a.G;
    p.b = i / (a.plan.tiles * a.G);
    const int64_t j = p.tile * kWave + p.lane;
    p.active = j < per;
    p.f = p.g * per + (p.active ? j : per - 1);
    return p;
}

// A[f][n] log2(e) of the lane's states, 0 behind the last (whose state then stays 0).
__device__ __forceinline__ void load_rates(const ScanArgs& a, const ScanPlace& p, float (&r)[kSL]) {
#pragma unroll
    for (int i = 0; i < kSL; ++i) {
        const int n = p.wave * kSL + i;
        r[i] = n < a.S ? a.A[p.f * a.S + n] * kLog2e : 0.0f;
    }
}

__device__ __forceinline__ void load_state(const ScanArgs& a, const ScanPlace& p, const float* from, float (&h)[kSL]) {
#pragma unroll
    for (int i = 0; i < kSL; ++i) {
        const int n = p.wave * kSL + i;
        h[i] = from != nullptr && n < a.S ? from[(p.b * a.F + p.f) * a.S + n] : 0.0f;
    }
}

__device__ __forceinline__ void store_state(const ScanArgs& a, const ScanPlace& p, float* to, const float (&h)[kSL]) {
#pragma unroll
    for (int i = 0; i < kSL; ++i) {
        const int n = p.wave * kSL + i;
        if (p.active && n < a.S) to[(p.b * a.F + p.f) * a.S + n] = h[i];
    }
}

// The state kept at the start of block c >= 1: [c-1][b][n][f].
__device__ __forceinline__ int64_t kept_at(const ScanArgs& a, const ScanPlace& p, int64_t c, int n) {
    return (((c - 1) * a.B + p.b) * a.S + n) * a.F + p.f;
}

}  // namespace snnlif
