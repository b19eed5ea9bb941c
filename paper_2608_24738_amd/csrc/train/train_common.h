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

// 2^x by the hardware's v_exp_f32 (results below 2^-126 flush to 0).
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

}  // namespace tmtrain
