// host_common.h -- what the host code of the training operators shares:
// element types, overlap of buffers, launches (include/tm_train.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../../include/tm_train.h"
#include "train_common.h"

namespace tmtrain {

constexpr uint64_t kLimit = uint64_t(1) << 31;

inline bool float_type(int dtype) { return dtype == TM_DTYPE_F32 || dtype == TM_DTYPE_F16 || dtype == TM_DTYPE_BF16; }
inline uint64_t float_bytes(int dtype) { return dtype == TM_DTYPE_F32 ? 4 : 2; }

constexpr uint64_t kFill = 1024;            // workgroups that keep the chip busy

inline uint32_t pow2_from(uint32_t n) {
    uint32_t p = 1;
    while (p < n) p <<= 1;
    return p;
}
inline uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

struct Range {
    const void *at;
    uint64_t bytes;
};
inline bool meet(const Range &a, const Range &b) {
    if (!a.at || !b.at || !a.bytes || !b.bytes) return false;
    const uintptr_t x = uintptr_t(a.at), y = uintptr_t(b.at);
    return x < y + b.bytes && y < x + a.bytes;
}
// No output may overlap an input or another output.
template <int NI, int NO>
inline bool aliased(const Range (&in)[NI], const Range (&out)[NO]) {
    for (int o = 0; o < NO; ++o) {
        for (int i = 0; i < NI; ++i)
            if (meet(out[o], in[i])) return true;
        for (int p = 0; p < o; ++p)
            if (meet(out[o], out[p])) return true;
    }
    return false;
}

template <typename Args>
int launch(void (*kernel)(Args), dim3 grid, dim3 block, size_t lds, hipStream_t s, const Args &args) {
    hipLaunchKernelGGL(kernel, grid, block, lds, s, args);
    return hipGetLastError() == hipSuccess ? TM_OK : TM_ERR_HIP;
}

// fn(T{}) with T the storage type of dtype.
template <typename F>
int by_type(int dtype, F fn) {
    if (dtype == TM_DTYPE_F32) return fn(float{});
    if (dtype == TM_DTYPE_BF16) return fn(bf16{});
    return fn(f16{});
}

// At least `blocks` < 2^31 workgroups, of up to 1024 threads.
inline dim3 row_grid(uint32_t blocks) {
    const uint32_t x = blocks < (1u << 21) ? blocks : 1u << 21;
    return dim3(x, uint32_t(ceil_div(blocks, x)));
}

}  // namespace tmtrain
