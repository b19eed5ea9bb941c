// norm.h -- kernels of layer norm and its gradients (tm_layer_norm in
// include/tm_train.h).
//
// With m = mean x, r = 1 / sqrt(mean (x - m)^2 + eps) and t = (x - m) r:
//     y = t w + b,
//     dx = r (g w - mean(g w) - t mean(g w t)),   dw = sum g t,   db = sum g.
// Bound by memory: x is read once and y written once, and backwards x and g are
// read once and dx written once.  The mean is taken first, then the mean and the
// mean square of what it leaves, from the registers that hold the row: the first
// mean is off by its sum's rounding, which is much of a row far from zero (rows of
// 1000.1 came out as up to 0.02 instead of 0), and the second is that error.  A
// thread keeps its columns from row to row: weight, bias and the sums for dw and
// db stay in registers.
#pragma once

#include "train_common.h"

namespace tmtrain {

struct NormArgs {
    const void *x, *weight, *bias;
    uint64_t stride;            // of the rows of x, elements
    uint32_t rows, width;
    int32_t param_type;         // of weight, bias and their gradients
    float eps, share;           // share = 1 / width
    void *y;
    float2 *stats;              // m and r of each row
    const void *up;
    void *dx, *dw, *db;
    float *part;                // [parts][2][part_stride]: sums of g t and of g
    uint32_t part_stride, parts;
    uint32_t share_rows;        // rows of a workgroup of k_norm_columns
};

template <int V>
__device__ __forceinline__ void load_params(const void *p, int type, uint32_t c, uint32_t n, float other, float (&out)[V]) {
    const auto get = [&](auto *q) {
        using T = std::remove_const_t<std::remove_pointer_t<decltype(q)>>;
        const Pack<T, V> v = load_pack<V>(q + c, n, T{});
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = widen(v.at(i));
    };
    if (!p) {
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = other;
    } else if (type == TM_DTYPE_F32) {
        get(static_cast<const float *>(p));
    } else if (type == TM_DTYPE_BF16) {
        get(static_cast<const bf16 *>(p));
    } else {
        get(static_cast<const f16 *>(p));
    }
}
__device__ __forceinline__ void store_param(void *p, int type, uint32_t c, float v) {
    if (type == TM_DTYPE_F32)
        static_cast<float *>(p)[c] = v;
    else if (type == TM_DTYPE_BF16)
        static_cast<bf16 *>(p)[c] = narrow<bf16>(v);
    else
        static_cast<f16 *>(p)[c] = narrow<f16>(v);
}

// Sums of N values over the L threads of a row (16 lanes, a wave, or a workgroup).
template <int L, int N>
__device__ __forceinline__ void row_sums(float (&x)[N], float (*lds)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = L == 16 ? row_sum(x[i]) : wave_sum(x[i]);
    if constexpr (L > 64) {
        __syncthreads();                        // what is there is read
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) lds[threadIdx.x >> 6][i] = x[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = 0.0f;
        for (int w = 0; w < L / 64; ++w)
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] += lds[w][i];
    }
}

// What is left of a row around its first mean: the mean d of it, and r of the row.  Squares about the first mean are
// d^2 more.
struct RowRest {
    float d, r;
};
__device__ __forceinline__ RowRest row_rest(const NormArgs &p, const float (&sum)[2]) {
    const float d = sum[0] * p.share, var = fmaf(sum[1], p.share, -d * d);
    return {d, 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + p.eps)};
}

// L threads to a row, each with P pieces of 16 bytes, L pieces apart.  16384 x
// 2048 bf16: 24 us, 5.6 TB/s (23 by one mean); 3088 x 10995 float16, rows at odd
// addresses: 50 us (46).
template <typename T, int L, int P>
__global__ __launch_bounds__(L > 256 ? L : 256) void k_norm(NormArgs p) {
    constexpr int V = 16 / sizeof(T), kRows = L > 256 ? 1 : 256 / L;
    __shared__ float lds[L > 64 ? L / 64 : 1][1], lds2[L > 64 ? L / 64 : 1][2];
    const uint32_t lane = threadIdx.x % L;
    uint32_t left[P];           // elements of a piece that the row has
    float w[P][V], b[P][V];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const uint32_t c = (i * L + lane) * V;
        left[i] = c < p.width ? min(p.width - c, uint32_t(V)) : 0;
        if (left[i]) {
            load_params<V>(p.weight, p.param_type, c, left[i], 1.0f, w[i]);
            load_params<V>(p.bias, p.param_type, c, left[i], 0.0f, b[i]);
        }
    }
    const uint32_t step = gridDim.x * kRows;
    for (uint32_t row = blockIdx.x * kRows + threadIdx.x / L; row < p.rows; row += step) {
        const T *x = static_cast<const T *>(p.x) + row * p.stride;
        float v[P][V], sum[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < P; ++i) {
            Pack<T, V> q{};
            if (left[i]) q = load_pack<V>(x + (i * L + lane) * V, left[i], T{});
#pragma unroll
            for (int k = 0; k < V; ++k) {
                v[i][k] = widen(q.at(k));
                sum[0] += v[i][k];
            }
        }
        row_sums<L>(sum, lds);
        const float mean = sum[0] * p.share;
        float rest[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                v[i][k] = uint32_t(k) < left[i] ? v[i][k] - mean : 0.0f;
                rest[0] += v[i][k];
                rest[1] = fmaf(v[i][k], v[i][k], rest[1]);
            }
        row_sums<L>(rest, lds2);
        const RowRest s = row_rest(p, rest);
        if (p.stats && lane == 0) p.stats[row] = float2{mean + s.d, s.r};
        T *y = static_cast<T *>(p.y) + uint64_t(row) * p.width;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (!left[i]) continue;
            float o[V];
#pragma unroll
            for (int k = 0; k < V; ++k) o[k] = fmaf((v[i][k] - s.d) * s.r, w[i][k], b[i][k]);
            store_pack<V>(y + (i * L + lane) * V, narrow_pack<T>(o), left[i]);
        }
    }
}

// dx, and the workgroup's sums for dw and db.  16384 x 2048 bf16 with float32
// parameters: 44 us, 4.9 TB/s of what it moves (768 workgroups' sums are 6 % of it).
template <typename T, int L, int P, bool Sums>
__global__ __launch_bounds__(L > 256 ? L : 256) void k_norm_grad(NormArgs p) {
    constexpr int V = 16 / sizeof(T), kThreads = L > 256 ? L : 256, kRows = kThreads / L;
    constexpr int kGroups = L > 64 ? 1 : kThreads / 64;         // waves with rows of their own
    __shared__ float lds[L > 64 ? L / 64 : 1][2];
    __shared__ float both[Sums && kGroups > 1 ? 2 : 1][Sums && kGroups > 1 ? L * P * V : 1];
    const uint32_t lane = threadIdx.x % L;
    uint32_t left[P];
    float w[P][V], dw[P][V], db[P][V];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const uint32_t c = (i * L + lane) * V;
        left[i] = c < p.width ? min(p.width - c, uint32_t(V)) : 0;
        if (left[i]) load_params<V>(p.weight, p.param_type, c, left[i], 1.0f, w[i]);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            if (uint32_t(k) >= left[i]) w[i][k] = 0.0f;
            dw[i][k] = db[i][k] = 0.0f;
        }
    }
    const uint32_t step = gridDim.x * kRows;
    for (uint32_t row = blockIdx.x * kRows + threadIdx.x / L; row < p.rows; row += step) {
        const T *x = static_cast<const T *>(p.x) + row * p.stride;
        const T *up = static_cast<const T *>(p.up) + uint64_t(row) * p.width;
        Pack<T, V> xs[P], gs[P];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            xs[i] = gs[i] = Pack<T, V>{};
            if (!left[i]) continue;
            xs[i] = load_pack<V>(x + (i * L + lane) * V, left[i], T{});
            gs[i] = load_pack<V>(up + (i * L + lane) * V, left[i], T{});
        }
        const float2 s = p.stats[row];
        float sum[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float t = (widen(xs[i].at(k)) - s.x) * s.y, g = widen(gs[i].at(k));
                if constexpr (Sums) {
                    dw[i][k] = fmaf(g, t, dw[i][k]);
                    db[i][k] += g;
                }
                const float gw = g * w[i][k];
                sum[0] += gw;
                sum[1] = fmaf(gw, t, sum[1]);
            }
        if (!p.dx) continue;
        row_sums<L>(sum, lds);
        const float a = sum[0] * p.share, b = sum[1] * p.share;
        T *dx = static_cast<T *>(p.dx) + uint64_t(row) * p.width;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (!left[i]) continue;
            forget_widened(xs[i]);
            forget_widened(gs[i]);
            float o[V];
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float t = (widen(xs[i].at(k)) - s.x) * s.y;
                o[k] = (fmaf(widen(gs[i].at(k)), w[i][k], -a) - t * b) * s.y;
            }
            store_pack<V>(dx + (i * L + lane) * V, narrow_pack<T>(o), left[i]);
        }
    }
    if constexpr (Sums) {
        if constexpr (L == 16) {
#pragma unroll
            for (int i = 0; i < P; ++i)
#pragma unroll
                for (int k = 0; k < V; ++k)
#pragma unroll
                    for (int d = 16; d < 64; d <<= 1) {
                        dw[i][k] += __shfl_xor(dw[i][k], d);
                        db[i][k] += __shfl_xor(db[i][k], d);
                    }
        }
        if constexpr (kGroups > 1) {
            // the waves' sums, one after the other
            const uint32_t wave = threadIdx.x >> 6;
            const bool mine = (threadIdx.x & 63) < L;
            for (uint32_t q = 0; q < uint32_t(kGroups); ++q) {
                if (wave == q && mine)
#pragma unroll
                    for (int i = 0; i < P; ++i)
#pragma unroll
                        for (int k = 0; k < V; ++k) {
                            const uint32_t c = (k * P + i) * L + lane;          // lanes side by side
                            if (q) {
                                dw[i][k] += both[0][c];
                                db[i][k] += both[1][c];
                            }
                            if (q + 1 < uint32_t(kGroups)) {
                                both[0][c] = dw[i][k];
                                both[1][c] = db[i][k];
                            }
                        }
                __syncthreads();
            }
            if (wave + 1 != uint32_t(kGroups) || !mine) return;
        }
        float *to = p.part + uint64_t(blockIdx.x) * 2 * p.part_stride;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (!left[i]) continue;
            Pack<float, V> a, b;
#pragma unroll
            for (int k = 0; k < V; ++k) {
                a.put(k, dw[i][k]);
                b.put(k, db[i][k]);
            }
            store_pack<V>(to + (i * L + lane) * V, a);
            store_pack<V>(to + p.part_stride + (i * L + lane) * V, b);
        }
    }
}

// Rows longer than the registers of a workgroup hold (32768 elements of 16 bits): a workgroup to a row, which reads it
// again for each step, from the caches, and goes on to others.
constexpr int kLongThreads = 1024;

template <typename T>
__global__ __launch_bounds__(kLongThreads) void k_norm_long(NormArgs p) {
    constexpr int V = 16 / sizeof(T);
    __shared__ float lds[kLongThreads / 64][1], lds2[kLongThreads / 64][2];
    for (uint32_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(p.x) + row * p.stride;
        const uint32_t c0 = threadIdx.x * V, step = kLongThreads * V;
        float sum[1] = {0.0f};
        for (uint32_t c = c0; c < p.width; c += step) {
            const Pack<T, V> q = load_pack<V>(x + c, p.width - c, T{});
#pragma unroll
            for (int k = 0; k < V; ++k) sum[0] += widen(q.at(k));
        }
        row_sums<kLongThreads>(sum, lds);
        const float mean = sum[0] * p.share;
        float rest[2] = {0.0f, 0.0f};
        for (uint32_t c = c0; c < p.width; c += step) {
            const Pack<T, V> q = load_pack<V>(x + c, p.width - c, T{});
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float v = c + k < p.width ? widen(q.at(k)) - mean : 0.0f;
                rest[0] += v;
                rest[1] = fmaf(v, v, rest[1]);
            }
        }
        row_sums<kLongThreads>(rest, lds2);
        const RowRest s = row_rest(p, rest);
        if (p.stats && threadIdx.x == 0) p.stats[row] = float2{mean + s.d, s.r};
        T *y = static_cast<T *>(p.y) + uint64_t(row) * p.width;
        for (uint32_t c = c0; c < p.width; c += step) {
            const uint32_t n = p.width - c;
            const Pack<T, V> q = load_pack<V>(x + c, n, T{});
            float w[V], b[V], o[V];
            load_params<V>(p.weight, p.param_type, c, n, 1.0f, w);
            load_params<V>(p.bias, p.param_type, c, n, 0.0f, b);
#pragma unroll
            for (int k = 0; k < V; ++k) o[k] = fmaf((widen(q.at(k)) - mean - s.d) * s.r, w[k], b[k]);
            store_pack<V>(y + c, narrow_pack<T>(o), n);
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kLongThreads) void k_norm_long_grad(NormArgs p) {
    constexpr int V = 16 / sizeof(T);
    __shared__ float lds[kLongThreads / 64][2];
    for (uint32_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(p.x) + row * p.stride;
        const T *up = static_cast<const T *>(p.up) + uint64_t(row) * p.width;
        const float2 s = p.stats[row];
        const uint32_t c0 = threadIdx.x * V, step = kLongThreads * V;
        float sum[2] = {0.0f, 0.0f};
        for (uint32_t c = c0; c < p.width; c += step) {
            const uint32_t n = p.width - c;
            const Pack<T, V> q = load_pack<V>(x + c, n, T{}), g = load_pack<V>(up + c, n, T{});
            float w[V];
            load_params<V>(p.weight, p.param_type, c, n, 1.0f, w);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float gw = uint32_t(k) < n ? widen(g.at(k)) * w[k] : 0.0f;
                sum[0] += gw;
                sum[1] = fmaf(gw, (widen(q.at(k)) - s.x) * s.y, sum[1]);
            }
        }
        row_sums<kLongThreads>(sum, lds);
        const float a = sum[0] * p.share, b = sum[1] * p.share;
        T *dx = static_cast<T *>(p.dx) + uint64_t(row) * p.width;
        for (uint32_t c = c0; c < p.width; c += step) {
            const uint32_t n = p.width - c;
            const Pack<T, V> q = load_pack<V>(x + c, n, T{}), g = load_pack<V>(up + c, n, T{});
            float w[V], o[V];
            load_params<V>(p.weight, p.param_type, c, n, 1.0f, w);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float t = (widen(q.at(k)) - s.x) * s.y;
                o[k] = (fmaf(widen(g.at(k)), w[k], -a) - t * b) * s.y;
            }
            store_pack<V>(dx + c, narrow_pack<T>(o), n);
        }
    }
}

// The sums for dw and db of such rows: a thread to V columns, a workgroup to share_rows rows.
template <typename T>
__global__ __launch_bounds__(256) void k_norm_columns(NormArgs p) {
    constexpr int V = 16 / sizeof(T);
    const uint32_t c = (blockIdx.x * 256 + threadIdx.x) * V;
    if (c >= p.width) return;
    const uint32_t n = p.width - c, last = min(p.rows, (blockIdx.y + 1) * p.share_rows);
    Pack<float, V> dw{}, db{};
    for (uint32_t row = blockIdx.y * p.share_rows; row < last; ++row) {
        const Pack<T, V> q = load_pack<V>(static_cast<const T *>(p.x) + row * p.stride + c, n, T{});
        const Pack<T, V> g = load_pack<V>(static_cast<const T *>(p.up) + uint64_t(row) * p.width + c, n, T{});
        const float2 s = p.stats[row];
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const float gk = widen(g.at(k));
            dw.put(k, fmaf(gk, (widen(q.at(k)) - s.x) * s.y, dw.at(k)));
            db.put(k, db.at(k) + gk);
        }
    }
    float *to = p.part + uint64_t(blockIdx.y) * 2 * p.part_stride + c;
    store_pack<V>(to, dw);
    store_pack<V>(to + p.part_stride, db);
}

// dw (blockIdx.y = 0) and db from the parts, 768 of 2 x 2048: 4.6 us.  64 columns to a workgroup, parts over its 16 waves.
__global__ __launch_bounds__(1024) void k_norm_join(NormArgs p) {
    __shared__ float lds[16][64];
    void *to = blockIdx.y ? p.db : p.dw;
    if (!to) return;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    float sum = 0.0f;
    if (c < p.width)
#pragma unroll 8
        for (uint32_t i = wave; i < p.parts; i += 16) sum += p.part[(uint64_t(i) * 2 + blockIdx.y) * p.part_stride + c];
    lds[wave][lane] = sum;
    __syncthreads();
    if (wave || c >= p.width) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) sum += lds[w][lane];
    store_param(to, p.param_type, c, sum);
}

}  // namespace tmtrain
