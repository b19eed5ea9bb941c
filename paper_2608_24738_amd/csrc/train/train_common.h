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

// V consecutive elements as the 32-bit words they are loaded and stored in, in
// pieces of up to 16 bytes; the address is aligned to one element.  (Kept as
// words, because loads of separate elements are not merged again.)
template <typename T, int V>
struct Pack {
    static constexpr int kWords = (V * int(sizeof(T)) + 3) / 4;
    uint32_t w[kWords];

    __device__ __forceinline__ T at(int j) const {
        if constexpr (sizeof(T) == 8)
            return __builtin_bit_cast(T, uint64_t(w[2 * j + 1]) << 32 | w[2 * j]);
        else if constexpr (sizeof(T) == 4)
            return __builtin_bit_cast(T, w[j]);
        else if constexpr (sizeof(T) == 2)
            return __builtin_bit_cast(T, uint16_t(w[j / 2] >> (16 * (j & 1))));
        else
            return __builtin_bit_cast(T, uint8_t(w[j / 4] >> (8 * (j & 3))));
    }
    __device__ __forceinline__ void put(int j, T v) {
        if constexpr (sizeof(T) == 4)
            w[j] = __builtin_bit_cast(uint32_t, v);
        else if constexpr (sizeof(T) == 2)
            w[j / 2] = j & 1 ? (w[j / 2] & 0xffffu) | uint32_t(__builtin_bit_cast(uint16_t, v)) << 16
                             : (w[j / 2] & 0xffff0000u) | __builtin_bit_cast(uint16_t, v);
        else if constexpr (sizeof(T) == 1)
            w[j / 4] = (w[j / 4] & ~(0xffu << (8 * (j & 3)))) | uint32_t(__builtin_bit_cast(uint8_t, v)) << (8 * (j & 3));
        else {
            w[2 * j] = uint32_t(__builtin_bit_cast(uint64_t, v));
            w[2 * j + 1] = uint32_t(__builtin_bit_cast(uint64_t, v) >> 32);
        }
    }
};

template <int N> struct Words;
template <> struct Words<1> { typedef uint32_t type; };
template <> struct Words<2> { typedef uint32_t type __attribute__((ext_vector_type(2))); };
template <> struct Words<4> { typedef uint32_t type __attribute__((ext_vector_type(4))); };

// N words at an address aligned to A bytes.
template <int N, int A>
struct Piece {
    typedef typename Words<N>::type type __attribute__((aligned(A)));
};

template <int V, typename T>
__device__ __forceinline__ Pack<T, V> load_pack(const T *p) {
    Pack<T, V> r{};
    if constexpr (V * sizeof(T) < 4) {
#pragma unroll
        for (int j = 0; j < V; ++j) r.put(j, p[j]);
    } else {
        constexpr int N = Pack<T, V>::kWords < 4 ? Pack<T, V>::kWords : 4;
        static_assert(V * sizeof(T) % (4 * N) == 0);
#pragma unroll
        for (int i = 0; i < Pack<T, V>::kWords; i += N) {
            const typename Words<N>::type v = *reinterpret_cast<const typename Piece<N, alignof(T)>::type *>(
                reinterpret_cast<const char *>(p) + 4 * i);
            if constexpr (N == 1) {
                r.w[i] = v;
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) r.w[i + j] = v[j];
            }
        }
    }
    return r;
}
// The first n elements; the rest are `fill`.
template <int V, typename T>
__device__ __forceinline__ Pack<T, V> load_pack(const T *p, uint32_t n, T fill) {
    if (V == 1 || n >= V) return load_pack<V>(p);
    Pack<T, V> r{};
#pragma unroll
    for (int j = 0; j < V; ++j) r.put(j, uint32_t(j) < n ? p[j] : fill);
    return r;
}
template <int V, typename T>
__device__ __forceinline__ void store_pack(T *p, const Pack<T, V> &r) {
    if constexpr (V * sizeof(T) < 4) {
#pragma unroll
        for (int j = 0; j < V; ++j) p[j] = r.at(j);
    } else {
        constexpr int N = Pack<T, V>::kWords < 4 ? Pack<T, V>::kWords : 4;
#pragma unroll
        for (int i = 0; i < Pack<T, V>::kWords; i += N) {
            typename Words<N>::type v;
            if constexpr (N == 1) {
                v = r.w[i];
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) v[j] = r.w[i + j];
            }
            *reinterpret_cast<typename Piece<N, alignof(T)>::type *>(reinterpret_cast<char *>(p) + 4 * i) = v;
        }
    }
}
template <int V, typename T>
__device__ __forceinline__ void store_pack(T *p, const Pack<T, V> &r, uint32_t n) {
    if (V == 1 || n >= V) return store_pack<V>(p, r);
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (uint32_t(j) < n) p[j] = r.at(j);
}
// All but the first `skip` elements.
template <int V, typename T>
__device__ __forceinline__ void store_own(T *p, const Pack<T, V> &r, uint32_t skip) {
    if (V == 1 || skip == 0) return store_pack<V>(p, r);
#pragma unroll
    for (int j = 1; j < V; ++j)
        if (uint32_t(j) >= skip) p[j] = r.at(j);
}

// Makes the compiler take the elements out of their words again from here on:
// kept widened from pass to pass they would need twice the registers.
template <typename T, int V>
__device__ __forceinline__ void forget_widened(Pack<T, V> &r) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < Pack<T, V>::kWords; ++i) asm volatile("" : "+v"(r.w[i]));
    }
}

// V floats rounded to T.
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> narrow_pack(const float (&v)[V]) {
    Pack<T, V> r{};
    if constexpr (sizeof(T) == 2 && V % 2 == 0) {
        typedef float f2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            const f2 x = {v[j], v[j + 1]};
            if constexpr (__is_same(T, bf16)) {
                typedef __bf16 b2 __attribute__((ext_vector_type(2)));
                r.w[j / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, b2));
            } else {
                typedef _Float16 h2 __attribute__((ext_vector_type(2)));
                r.w[j / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, h2));
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) r.put(j, narrow<T>(v[j]));
    }
    return r;
}

// The largest of three by one instruction; fmaxf makes each operand quiet by
// another first.  A signalling NaN comes out as NaN, quiet ones are passed over.
__device__ __forceinline__ float max_of(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// 2^x by the hardware's v_exp_f32 (results below 2^-126 flush to 0).
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// Orders a wave's LDS writes and reads around it.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Reductions over a wave by data-parallel primitives: rows of 16 lanes by
// shifts, then across rows by two broadcasts; lane 63 ends with the result,
// which becomes uniform.  The order of the additions is fixed.
template <int Ctrl, int Rows>
__device__ __forceinline__ uint32_t dpp(uint32_t old, uint32_t x) {
    return uint32_t(__builtin_amdgcn_update_dpp(int(old), int(x), Ctrl, Rows, 0xf, false));
}
template <typename F>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t x, uint32_t none, F op) {
    x = op(x, dpp<0x111, 0xf>(none, x));                   // row_shr 1, 2, 4, 8
    x = op(x, dpp<0x112, 0xf>(none, x));
    x = op(x, dpp<0x114, 0xf>(none, x));
    x = op(x, dpp<0x118, 0xf>(none, x));
    x = op(x, dpp<0x142, 0xa>(none, x));                   // row_bcast 15 into rows 1 and 3, 31 into 2 and 3
    x = op(x, dpp<0x143, 0xc>(none, x));
    return uint32_t(__builtin_amdgcn_readlane(int(x), 63));
}
// The same over each row of 16 lanes, by rotations: every lane ends with the
// result, made in one order.
template <typename F>
__device__ __forceinline__ uint32_t row_reduce(uint32_t x, F op) {
    x = op(x, dpp<0x128, 0xf>(x, x));                      // row_ror 8, 4, 2, 1
    x = op(x, dpp<0x124, 0xf>(x, x));
    x = op(x, dpp<0x122, 0xf>(x, x));
    return op(x, dpp<0x121, 0xf>(x, x));
}
__device__ __forceinline__ float row_max(float x) {        // not of NaN
    return __uint_as_float(row_reduce(__float_as_uint(x), [](uint32_t a, uint32_t b) {
        return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    }));
}
__device__ __forceinline__ float row_sum(float x) {
    return __uint_as_float(row_reduce(__float_as_uint(x), [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }));
}
__device__ __forceinline__ uint64_t row_max(uint64_t x) {
    const auto most = [](uint32_t a, uint32_t b) { return max(a, b); };
    const uint32_t hi = row_reduce(uint32_t(x >> 32), most);
    const uint32_t lo = row_reduce(uint32_t(x >> 32) == hi ? uint32_t(x) : 0u, most);
    return uint64_t(hi) << 32 | lo;
}
__device__ __forceinline__ float wave_max(float x) {       // not of NaN
    return __uint_as_float(wave_reduce(__float_as_uint(x), 0xff800000u, [](uint32_t a, uint32_t b) {
        return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    }));
}
__device__ __forceinline__ float wave_sum(float x) {
    return __uint_as_float(wave_reduce(__float_as_uint(x), 0u, [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
    return wave_reduce(x, 0u, [](uint32_t a, uint32_t b) { return max(a, b); });
}
// By halves: the largest upper word, then the largest lower word that has it.
__device__ __forceinline__ uint64_t wave_max(uint64_t x) {
    const uint32_t hi = wave_max(uint32_t(x >> 32));
    const uint32_t lo = wave_max(uint32_t(x >> 32) == hi ? uint32_t(x) : 0u);
    return uint64_t(hi) << 32 | lo;
}

}  // namespace tmtrain
