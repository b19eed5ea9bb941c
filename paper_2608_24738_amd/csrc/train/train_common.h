// train_common.h -- element types, argument blocks and small device helpers
// shared by the kernels of the training operators (include/tm_train.h).
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cfloat>

#include "../edt_common.h"

namespace tmtrain {

using tmedt::Div32;
using tmedt::kWave;

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// Storage types: 16-bit floats are handled as their bit patterns.
struct f16 { uint16_t u; };
struct bf16 { uint16_t u; };

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(bf16 x) { return __uint_as_float(uint32_t(x.u) << 16); }
__device__ __forceinline__ float widen(f16 x) { return float(__builtin_bit_cast(_Float16, x.u)); }

// Round to nearest even, once, at the store.
template <typename T>
__device__ __forceinline__ T narrow(float x);
template <>
__device__ __forceinline__ float narrow<float>(float x) { return x; }
template <>
__device__ __forceinline__ f16 narrow<f16>(float x) { return {__builtin_bit_cast(uint16_t, _Float16(x))}; }
template <>
__device__ __forceinline__ bf16 narrow<bf16>(float x) { return {__builtin_bit_cast(uint16_t, __bf16(x))}; }

// V consecutive elements, loaded and stored in one piece of up to 16 bytes per
// instruction; the address is aligned to one element.
template <typename T, int V>
struct Pack { T v[V]; };

template <int V, typename T>
__device__ __forceinline__ Pack<T, V> load_pack(const T *p) {
    Pack<T, V> r;
    __builtin_memcpy(&r, p, sizeof r);
    return r;
}
// The first n elements; the rest are `fill`.
template <int V, typename T>
__device__ __forceinline__ Pack<T, V> load_pack(const T *p, uint32_t n, T fill) {
    if (n >= V) return load_pack<V>(p);
    Pack<T, V> r;
#pragma unroll
    for (int j = 0; j < V; ++j) r.v[j] = uint32_t(j) < n ? p[j] : fill;
    return r;
}
template <int V, typename T>
__device__ __forceinline__ void store_pack(T *p, const Pack<T, V> &r) {
    __builtin_memcpy(p, &r, sizeof r);
}
template <int V, typename T>
__device__ __forceinline__ void store_pack(T *p, const Pack<T, V> &r, uint32_t n) {
    if (n >= V) return store_pack<V>(p, r);
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (uint32_t(j) < n) p[j] = r.v[j];
}

// 2^x by the hardware's v_exp_f32 (results below 2^-126 flush to 0).
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

}  // namespace tmtrain
