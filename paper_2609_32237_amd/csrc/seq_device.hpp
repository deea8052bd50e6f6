// seq_device.hpp -- what the sequence kernels share on the device: element
// types, loads and stores at element alignment, the sigmoid.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace mi355seq {

constexpr int kWave = 64;

// Element types.  to_f is exact; of_f is the one rounding of an activation
// (to nearest, ties to even), done where it is written.
struct F32 {
    using T = float;
    static __device__ __forceinline__ float to_f(T v) { return v; }
    static __device__ __forceinline__ T of_f(float v) { return v; }
};
struct F16 {
    using T = _Float16;
    static __device__ __forceinline__ float to_f(T v) { return (float)v; }
    static __device__ __forceinline__ T of_f(float v) { return (T)v; }
};
struct BF16 {
    using T = __bf16;
    static __device__ __forceinline__ float to_f(T v) { return (float)v; }
    static __device__ __forceinline__ T of_f(float v) { return (T)v; }
};

// 1 / (1 + e^-v) with the hardware's exp2 and reciprocal (each within 1 ulp):
// 0 at -inf, 1 at +inf, relative error about |v| 2^-24 + 3e-7.
__device__ __forceinline__ float sigmoid(float v) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896340736f * v));
}

}  // namespace mi355seq
