// Device helpers of the sequence operators' kernels.
#pragma once
#include "lif_kernels.h"
#include "seq_host.h"

namespace snnlif {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;

template <int IO>
__device__ __forceinline__ const void* at(const Rows& r, int64_t t, int64_t b, int64_t f) {
    return static_cast<const char*>(r.p) + (t * r.t + b * r.b + f) * (IO == SNN_IO_F32 ? 4 : 2);
}
template <int IO>
__device__ __forceinline__ void* at_out(const Rows& r, int64_t t, int64_t b, int64_t f) {
    return const_cast<void*>(at<IO>(r, t, b, f));
}

template <int IO, int V>
__device__ __forceinline__ void load_vec(const void* p, float (&v)[V]) {
    const auto raw = IoVec<IO, V>::load(p, 0);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = IoVec<IO, V>::get(raw, j);
}

template <int IO>
__device__ __forceinline__ float load1(const void* p) {
    return IoVec<IO, 1>::get(IoVec<IO, 1>::load(p, 0), 0);
}
template <int IO>
__device__ __forceinline__ void store1(void* p, float v) {
    const float a[1] = {v};
    IoVec<IO, 1>::store(p, 0, a);
}

// V consecutive parameters.
template <int V>
__device__ __forceinline__ void load_params(const float* p, float (&v)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = p[j];
}

__device__ __forceinline__ int steps_of(const int32_t* lengths, int64_t b, int64_t T) {
    if (lengths == nullptr) return int(T);
    const int n = lengths[b];
    return n < 0 ? 0 : n > int(T) ? int(T) : n;
}

__device__ __forceinline__ float sigmoid(float u) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * u));
}
// Derivative of u * sigmoid(u) from s = sigmoid(u).
__device__ __forceinline__ float silu_slope(float u, float s) { return s * fmaf(u, 1.0f - s, 1.0f); }

// ln(1 + e^v) = max(v, 0) + ln(1 + e), e = e^-|v| <= 1.  ln(1 + e) loses e's low bits in the
// sum w = 1 + e; ln(w) e / (w - 1) puts them back (Kahan), as w - 1 is exact.
__device__ __forceinline__ float softplus_of(float v, float e) {
    const float w = 1.0f + e, d = w - 1.0f;
    const float l = (kLn2 * __builtin_amdgcn_logf(w)) * (e * __builtin_amdgcn_rcpf(d));
    return fmaxf(v, 0.0f) + (d == 0.0f ? e : l);
}
__device__ __forceinline__ float softplus(float v) {
    return softplus_of(v, __builtin_amdgcn_exp2f(-kLog2e * fabsf(v)));
}
// With its slope, the sigmoid of v.
__device__ __forceinline__ float softplus(float v, float& slope) {
    const float e = __builtin_amdgcn_exp2f(-kLog2e * fabsf(v)), r = __builtin_amdgcn_rcpf(1.0f + e);
    slope = v < 0.0f ? e * r : r;
    return softplus_of(v, e);
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
constexpr int kDppRor8 = 0x128, kDppHalfMirror = 0x141, kDppXor2 = 0x4E, kDppXor1 = 0xB1;

// Sum over the 64 lanes, in every lane, in a fixed order.
__device__ __forceinline__ float wave_sum(float v) {
    v += dpp<kDppXor1>(v);
    v += dpp<kDppXor2>(v);
    v += dpp<kDppHalfMirror>(v);
    v += dpp<kDppRor8>(v);
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Sums of partial results: V values of a workgroup, its threads over V values and the partial
// results, in a fixed order.
template <int V = kWave>
__device__ __forceinline__ void reduce_partials(const float* part, int64_t P, int64_t stride, const ReduceOut& out,
                                                int64_t block, float* lds) {
    const int value = threadIdx.x % V, walker = threadIdx.x / V, walkers = blockDim.x / V;
    int64_t i = block * V + value;
    const bool in = i < out.n[0] + out.n[1] + out.n[2];
    float s = 0.0f;
    if (in) {
#pragma unroll 8
        for (int64_t p = walker; p < P; p += walkers) s += part[p * stride + i];
    }
    lds[threadIdx.x] = s;
    __syncthreads();
    if (walker != 0 || !in) return;
    for (int w = 1; w < walkers; ++w) s += lds[w * V + value];
    int k = 0;
    while (i >= out.n[k]) i -= out.n[k++];
    if (out.p[k] != nullptr) out.p[k][i] = s;
}

// A barrier that orders the LDS only: loads from memory stay in flight over it.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

}  // namespace snnlif
