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

// V consecutive elements in one access of up to 16 bytes.  Accesses need no
// more than element alignment: the hardware takes them at any address.
template <int BYTES>
struct Raw;
template <>
struct Raw<2> { using U = uint16_t; };
template <>
struct Raw<4> { using U = uint32_t; };
template <>
struct Raw<8> { using U = uint32_t __attribute__((ext_vector_type(2))); };
template <>
struct Raw<16> { using U = uint32_t __attribute__((ext_vector_type(4))); };

template <typename E, int V>
struct Pack {
    using T = typename E::T;
    using U = typename Raw<V * sizeof(T)>::U;
    struct __attribute__((packed, aligned(sizeof(T)))) Unaligned {
        U u;
    };
    U u;

    __device__ __forceinline__ void load(const T *p) { u = ((const Unaligned *)p)->u; }
    __device__ __forceinline__ void store(T *p) const { ((Unaligned *)p)->u = u; }
    __device__ __forceinline__ float get(int j) const {
        T v[V];
        __builtin_memcpy(v, &u, sizeof(u));
        return E::to_f(v[j]);
    }
    __device__ __forceinline__ void set(const float (&f)[V]) {
        T v[V];
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = E::of_f(f[j]);
        __builtin_memcpy(&u, v, sizeof(u));
    }
};

}  // namespace mi355seq
