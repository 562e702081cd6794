// Device helpers of the gated norms: the gate functions and 8-value pieces of either type.
#pragma once
#include "common.h"

namespace ssm {

// sigmoid(v) = 1 / (1 + e^-v): relative error of a few 2^-24 wherever it is not tiny
__device__ __forceinline__ float sigmoid_f(float v) { return fast_rcp(1.0f + fast_exp2(-v * kLog2e)); }
__device__ __forceinline__ float gate_f(float v, int fn) {
    switch (fn) {   // the same for a whole launch
        case SSM_GATE_SIGMOID: return sigmoid_f(v);
        case SSM_GATE_SILU: return silu_f(v);
        case SSM_GATE_TANH: return tanhf(v);
        default: return v;
    }
}

template <typename T> __device__ __forceinline__ void read8(const T* p, float (&v)[8]) {
    T x[8];
    load16(p, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = to_f32(x[e]);
}
template <typename T> __device__ __forceinline__ void write8(T* p, const float (&v)[8]) {
    T x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = from_f32<T>(v[e]);
    store16(p, x);
}
// the same past the caches
__device__ __forceinline__ void write8_past(float* p, const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) __builtin_nontemporal_store(f32x4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]}, (f32x4*)p + i);
}

}  // namespace ssm
