// bias.h -- a learned bias by buckets of distance, from a distance field or
// from the positions of queries and keys on a grid, and the gradient of its
// table (include/tm_train.h).
#pragma once

#include "train_common.h"

namespace tmtrain {

constexpr int kBiasMaxDim = 8;
constexpr uint32_t kMaxBuckets = 256;

// Where distances come from.  kField: an array; the others: positions.
enum Source { kFieldF32, kFieldI32, kOffset, kEuclid, kTaxicab, kChess };

struct BiasSource {
    const void *field;
    const float *edges;
    int32_t source, ndim;
    uint32_t buckets;
    uint32_t positions;                    // of one sample
    Div32 div_key;                         // key positions
    Div32 div_q[kBiasMaxDim], div_k[kBiasMaxDim];
    int32_t offset[kBiasMaxDim];           // first query's coordinates
    float sampling[kBiasMaxDim];
};

struct BiasArgs {
    BiasSource src;
    const void *table;
    const void *add;
    void *out;
    uint32_t heads, batch, field_batch;    // field_batch: samples with buckets of their own
    int32_t table_type;                    // tm_dtype
};

struct BiasGradArgs {
    BiasSource src;
    const void *grad;
    void *out;
    float *partial;
    uint32_t heads, batch, field_batch;
    int32_t table_type;
};

// The float32 distance of position p of sample b.  Every operation rounds by
// itself: a contraction could move a distance over an edge.
__device__ __forceinline__ float distance_at(const BiasSource &s, uint32_t b, uint32_t p) {
#pragma clang fp contract(off)
    if (s.source == kFieldF32) return static_cast<const float *>(s.field)[uint64_t(b) * s.positions + p];
    if (s.source == kFieldI32) return float(static_cast<const int32_t *>(s.field)[uint64_t(b) * s.positions + p]);
    uint32_t q = s.div_key.div(p), k = p - q * s.div_key.d;
    if (s.source == kOffset) return float(int32_t(k) - (int32_t(q) + s.offset[0]));
    float term[kBiasMaxDim];
    for (int a = s.ndim - 1; a >= 0; --a) {
        const uint32_t q1 = s.div_q[a].div(q), k1 = s.div_k[a].div(k);
        const int32_t delta = int32_t(k - k1 * s.div_k[a].d) - (int32_t(q - q1 * s.div_q[a].d) + s.offset[a]);
        const float v = float(delta) * s.sampling[a];
        term[a] = s.source == kEuclid ? v * v : fabsf(v);
        q = q1;
        k = k1;
    }
    float sum = term[0];
    for (int a = 1; a < s.ndim; ++a) sum = s.source == kChess ? fmaxf(sum, term[a]) : sum + term[a];
    return s.source == kEuclid ? sqrtf(sum) : sum;
}

// Number of edges <= d: between 0 and buckets - 1 whatever the edges hold.
__device__ __forceinline__ uint32_t bucket_of(const float *edges, uint32_t buckets, float d) {
    uint32_t lo = 0, hi = buckets - 1;
    while (lo < hi) {
        const uint32_t mid = (lo + hi) >> 1;
        if (edges[mid] <= d) lo = mid + 1; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ float table_at(const void *table, int32_t type, uint64_t i) {
    if (type == 6) return static_cast<const float *>(table)[i];
    if (type == 5) return widen(static_cast<const bf16 *>(table)[i]);
    return widen(static_cast<const f16 *>(table)[i]);
}
__device__ __forceinline__ void table_put(void *table, int32_t type, uint64_t i, float v) {
    if (type == 6) static_cast<float *>(table)[i] = v;
    else if (type == 5) static_cast<bf16 *>(table)[i] = narrow<bf16>(v);
    else static_cast<f16 *>(table)[i] = narrow<f16>(v);
}

template <typename T>
__global__ void __launch_bounds__(256) k_bias(BiasArgs a) {
    const uint32_t p = blockIdx.x * 256 + threadIdx.x;
    if (p >= a.src.positions) return;
    for (uint32_t b = 0; b < a.batch; ++b) {
        const uint32_t k = bucket_of(a.src.edges, a.src.buckets, distance_at(a.src, b, p));
        for (uint32_t h = 0; h < a.heads; ++h) {
            const uint64_t at = (uint64_t(b) * a.heads + h) * a.src.positions + p;
            float v = table_at(a.table, a.table_type, uint64_t(k) * a.heads + h);
            if (a.add) v += widen(static_cast<const T *>(a.add)[at]);
            static_cast<T *>(a.out)[at] = narrow<T>(v);
        }
    }
}

// One workgroup per bucket and head sums over every position.
template <typename T>
__global__ void __launch_bounds__(256) k_bias_grad(BiasGradArgs a) {
    __shared__ float part[256];
    const uint32_t k = blockIdx.x / a.heads, h = blockIdx.x - k * a.heads;
    float sum = 0.0f;
    for (uint32_t b = 0; b < a.batch; ++b)
        for (uint32_t p = threadIdx.x; p < a.src.positions; p += 256)
            if (bucket_of(a.src.edges, a.src.buckets, distance_at(a.src, b, p)) == k)
                sum += widen(static_cast<const T *>(a.grad)[(uint64_t(b) * a.heads + h) * a.src.positions + p]);
    part[threadIdx.x] = sum;
    __syncthreads();
    for (uint32_t w = 128; w; w >>= 1) {
        if (threadIdx.x < w) part[threadIdx.x] += part[threadIdx.x + w];
        __syncthreads();
    }
    if (threadIdx.x == 0) table_put(a.out, a.table_type, blockIdx.x, part[0]);
}

}  // namespace tmtrain
