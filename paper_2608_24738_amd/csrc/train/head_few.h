// head_few.h -- the kernels of head.h for up to kFewRows rows, such as one new
// token: bound by one read of the weight, which goes from memory to registers.
// Groups of kFewRows rows take the same way to their logits where there is so
// little work that tiles would leave most CUs without one, and go through long
// rows one step after the other.
#pragma once

#include "head.h"

namespace tmtrain {

constexpr int kFewWaves = 4;
constexpr int kFewClasses = 16 * kFewWaves;     // of a workgroup
constexpr int kFewSums = 8;
constexpr uint32_t kFewAhead = 8;                   // pieces of a row on their way to a lane

// The wave's classes, 16 from v0 on: each of its own, or waves share their row's columns.
struct FewPlace {
    uint32_t v0, share;
};
__device__ __forceinline__ FewPlace few_place(const HeadArgs &p) {
    const uint32_t wave = blockIdx.x * kFewWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    return {(wave >> p.few_shift) * 16, wave & ((1u << p.few_shift) - 1)};
}

// A lane's pieces of a row, round by round, of which lane group g has the g-th.
// Odd: rows may begin between two words, where loads take 2.5 times as long (log
// sums of 9 x 54800 x 703 float16 56 us, like this 26).  Such a row is read one
// element further on, and the first element of a piece is then the last one that
// the group before has read, in the first piece of a round that of the last.
template <typename T, bool Odd>
struct FewRow {
    typedef uint32_t Words __attribute__((ext_vector_type(4), aligned(4)));
    const T *row;
    uint32_t lane, carry;
    bool odd;
    __device__ __forceinline__ FewRow(const T *row_, uint32_t lane_, uint32_t k, uint32_t width) : row(row_), lane(lane_) {
        if constexpr (Odd) {
            odd = uintptr_t(row) & 2;
            carry = *reinterpret_cast<const uint16_t *>(row + min(k, width - 1));
        }
    }
    __device__ __forceinline__ u32x4 load(uint32_t k) const {
        if constexpr (Odd) {
            const Words d = *reinterpret_cast<const Words *>(row + k + odd);
            return u32x4{d[0], d[1], d[2], d[3]};
        } else {
            const auto x = load_pack<16 / int(sizeof(T))>(row + k);
            return u32x4{x.w[0], x.w[1], x.w[2], x.w[3]};
        }
    }
    // What `load` gave, in rising order of rounds.
    __device__ __forceinline__ u32x4 piece(u32x4 d) {
        if constexpr (Odd) {
            const uint32_t t = uint32_t(__shfl(int(d[3]), int((lane + 48) & 63))) >> 16, e = lane < 16 ? carry : t;
            carry = t;
            if (odd) d = u32x4{e | d[0] << 16, d[0] >> 16 | d[1] << 16, d[1] >> 16 | d[2] << 16, d[2] >> 16 | d[3] << 16};
        }
        return d;
    }
};

// h w of 16 classes from v0 on and 16 rows, of which the lane's is `row`: it
// holds classes v0 + 4 g + q of it.  Every wave of a workgroup calls it.
template <typename T, bool Odd>
__device__ __forceinline__ f32x4 few_logits(const HeadArgs &p, uint32_t first, FewPlace at, uint32_t row) {
    constexpr uint32_t V = 16 / sizeof(T), kRound = 4 * V;
    __shared__ f32x4 lds[kFewWaves][64];
    const uint32_t v0 = first + at.v0;
    const uint32_t lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    // several sums, so that none grows to the whole logit step by step
    f32x4 acc[kFewSums];
#pragma unroll
    for (int i = 0; i < kFewSums; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const uint32_t length = ((p.width + kRound - 1) / kRound + (1u << p.few_shift) - 1 >> p.few_shift) * kRound;
    const uint32_t end = v0 < p.classes ? min(p.width, (at.share + 1) * length) : 0;
    uint32_t k = at.share * length + g * V;
    FewRow<T, Odd> w(static_cast<const T *>(p.weight) + uint64_t(min(v0 + r, p.classes - 1)) * p.weight_stride, lane, k, p.width);
    FewRow<T, Odd> h(static_cast<const T *>(p.hidden) + row * p.hidden_stride, lane, k, p.width);
    // an odd row's loads take one element more, which the row must have
    const uint32_t limit = Odd ? min(end, p.width - 1) : end;
    for (; k - g * V + kFewAhead * kRound <= limit; k += kFewAhead * kRound) {
        u32x4 a[kFewAhead], b[kFewAhead];
#pragma unroll
        for (uint32_t i = 0; i < kFewAhead; ++i) a[i] = w.load(k + i * kRound);
#pragma unroll
        for (uint32_t i = 0; i < kFewAhead; ++i) b[i] = h.load(k + i * kRound);
#pragma unroll
        for (uint32_t i = 0; i < kFewAhead; ++i) acc[i % kFewSums] = multiply<T>(w.piece(a[i]), h.piece(b[i]), acc[i % kFewSums]);
    }
    if (k - g * V < end) {                              // fewer rounds, of which the last may be part of one
        const uint32_t at = k - g * V, whole = at < limit ? (limit - at) / kRound : 0;
        u32x4 a[kFewAhead], b[kFewAhead];
        Pack<T, int(V)> last_a{}, last_b{};
#pragma unroll
        for (uint32_t i = 0; i < kFewAhead; ++i) {
            if (i < whole) {
                a[i] = w.load(k + i * kRound);
                b[i] = h.load(k + i * kRound);
            }
        }
        const uint32_t last = k + whole * kRound;
        if (at + whole * kRound < end && last < p.width) {
            last_a = load_pack<int(V)>(w.row + last, p.width - last, T{});
            last_b = load_pack<int(V)>(h.row + last, p.width - last, T{});
        }
        const auto words = [](const Pack<T, int(V)> &x) { return u32x4{x.w[0], x.w[1], x.w[2], x.w[3]}; };
#pragma unroll
        for (uint32_t i = 0; i < kFewAhead; ++i)
            if (i < whole) acc[i % kFewSums] = multiply<T>(w.piece(a[i]), h.piece(b[i]), acc[i % kFewSums]);
        acc[0] = multiply<T>(words(last_a), words(last_b), acc[0]);
    }
#pragma unroll
    for (int d = kFewSums / 2; d; d /= 2)
#pragma unroll
        for (int i = 0; i < d; ++i) acc[i] += acc[i + d];
    if (p.few_shift) {
        const uint32_t wave = threadIdx.x >> 6;
        lds[wave][lane] = acc[0];
        __syncthreads();
        acc[0] = lds[wave - at.share][lane];
        for (uint32_t w = 1; w < 1u << p.few_shift; ++w) acc[0] += lds[wave - at.share + w][lane];
    }
    return acc[0];
}

// Sums over a workgroup's classes of its 16 rows, and the labels' x.  Bound by
// the weight's bytes: 32768 x 1024 bf16 13.8 us for up to 4 rows (4.8 TB/s),
// 131072 x 2048 95 (5.6 TB/s).
template <typename T, bool Odd>
__global__ __launch_bounds__(64 * kFewWaves) void k_few_sums(HeadArgs p) {
    __shared__ HeadSum lds[kFewWaves][kFewRows];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = blockIdx.y * kFewRows + (lane & 15);
    const FewPlace at = few_place(p);
    const uint32_t v = at.v0 + (lane >> 4) * 4;
    HeadSum sum = {kLowest, 0.0f};
    f32x4 x = few_logits<T, Odd>(p, 0, at, min(n, p.n - 1));
    if (at.v0 < p.classes && at.share == 0) {
        const int32_t y = n < p.n && p.label ? load_label(p.label, p.label_bytes, n, p.classes) : -1;
        if (y >= 0 && uint32_t(y) - v < 4) {
            const uint32_t q = uint32_t(y) - v;
            p.found[n] = q == 0 ? x[0] : q == 1 ? x[1] : q == 2 ? x[2] : x[3];
        }
        float most = -INFINITY;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (v + q >= p.classes) x[q] = -INFINITY;
            most = fmaxf(most, x[q]);
        }
        most = fmaxf(most, __shfl_xor(most, 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        sum.m = fmaxf(most, kLowest);
#pragma unroll
        for (int q = 0; q < 4; ++q) sum.s += exp2_hw((x[q] - sum.m) * p.c);
        sum.s += __shfl_xor(sum.s, 16);
        sum.s += __shfl_xor(sum.s, 32);
    }
    if (lane < 16) lds[wave][lane] = sum;
    __syncthreads();
    if (threadIdx.x >= 16) return;
    sum = lds[0][lane];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) sum = join(sum, lds[w][lane], p.c);
    if (n < p.n) p.part[uint64_t(n) * p.parts + blockIdx.x] = sum;
}

// The sums of a row over all parts, a workgroup to a row.  512 parts: 3.9 us, mostly a launch.
__global__ __launch_bounds__(256) void k_few_rows(HeadArgs p) {
    __shared__ HeadSum lds[4];
    constexpr int kAhead = 4;
    const HeadSum *part = p.part + uint64_t(blockIdx.x) * p.parts;
    HeadSum sum = {kLowest, 0.0f};
    for (uint32_t i = threadIdx.x; i < p.parts; i += 256 * kAhead) {
        HeadSum got[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) got[k] = i + 256 * k < p.parts ? part[i + 256 * k] : HeadSum{kLowest, 0.0f};
#pragma unroll
        for (int k = 0; k < kAhead; ++k) sum = join(sum, got[k], p.c);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum = join(sum, HeadSum{__shfl_xor(sum.m, d), __shfl_xor(sum.s, d)}, p.c);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x) return;
#pragma unroll
    for (int w = 1; w < 4; ++w) sum = join(sum, lds[w], p.c);
    head_store(p, blockIdx.x, p.found + blockIdx.x, sum);
}

// g in float32, [classes][kFewRows]; 0 for rows that take no part.
template <typename T, bool Odd>
__global__ __launch_bounds__(64 * kFewWaves) void k_few_slopes(HeadArgs p) {
    const uint32_t lane = threadIdx.x & 63, n = lane & 15;
    const FewPlace at = few_place(p);
    const uint32_t v = at.v0 + (lane >> 4) * 4;
    const f32x4 x = few_logits<T, Odd>(p, 0, at, min(n, p.n - 1));
    if (at.v0 >= p.classes || at.share) return;
    int32_t y = -1;
    HeadUp u = {0.0f, 0.0f};
    HeadSum s = {0.0f, 1.0f};
    bool in = n < p.n;
    if (in) {
        y = p.label ? load_label(p.label, p.label_bytes, n, p.classes) : -1;
        in = y >= 0 || p.all;
        u = head_up(p, n, y);
        s = p.stats[n];
        in = in && s.s != 0.0f;
    }
    const float b = u.b / s.s;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (v + q >= p.classes) break;
        float g = -b * exp2_hw((x[q] - s.m) * p.c);
        if (int32_t(v + q) == y) g += u.a;
        static_cast<float *>(p.slope)[uint64_t(v + q) * kFewRows + n] = in ? g : 0.0f;
    }
}

// g of the packed rows as the tiles read it, in G planes of S, for a piece: what
// k_head_slopes gives.  Rows from the last one to its 128 get zeros, and classes
// from the last one to its 64, which waves without classes of their own write.
template <typename T, typename S, int G, bool Odd>
__global__ __launch_bounds__(64 * kFewWaves) void k_few_tiles(HeadArgs p) {
    const uint32_t lane = threadIdx.x & 63, n = blockIdx.y * kFewRows + (lane & 15), count = *p.count;
    const FewPlace at = few_place(p);
    const uint32_t v = at.v0 + at.share * (kFewClasses >> p.few_shift) + (lane >> 4) * 4;
    const uint32_t rows = min(p.piece, p.classes - p.first);
    if (blockIdx.y * kFewRows >= ((count + 127) & ~127u)) return;
    const bool real = n < count;
    HeadRow r = {0.0f, 0.0f, 0.0f, -1};
    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
    if (blockIdx.y * kFewRows < count) {
        if (real) r = p.row[n];
        x = few_logits<T, Odd>(p, p.first, at, p.list[min(n, count - 1)]);
    }
    if (at.share && (blockIdx.x + 1 < gridDim.x || v >= ((rows + 63) & ~63u))) return;
    float g[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        g[q] = -r.b * exp2_hw((x[q] - r.m) * p.c);
        if (int32_t(p.first + v + q) == r.y) g[q] += r.a;
        if (!real || v + q >= rows) g[q] = 0.0f;
    }
    float ratio = 1.0f;
    if constexpr (__is_same(T, f16)) ratio = real ? p.inverse[n] / p.inverse[p.n_pad] : 1.0f;
    if constexpr (sizeof(T) == 2 && G == 1) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (r.y >= 0 && p.first + v + q == uint32_t(r.y)) keep_rest<T>(p, n, g[q], ratio);
    }
    const uint64_t to = uint64_t(n) * p.piece + v, plane = uint64_t(p.n_pad) * p.piece;
    Pack<S, 4> out[G];
    if (!__is_same(T, f16) || p.slope) {
        split(g, out);
#pragma unroll
        for (int k = 0; k < G; ++k) store_pack<4>(static_cast<S *>(p.slope) + to + k * plane, out[k]);
    }
    if constexpr (__is_same(T, f16)) {
        if (!p.slope_common) return;
#pragma unroll
        for (int q = 0; q < 4; ++q) g[q] *= ratio;
        split(g, out);
#pragma unroll
        for (int k = 0; k < G; ++k) store_pack<4>(static_cast<S *>(p.slope_common) + to + k * plane, out[k]);
    }
}

// dw = g^T h and the workgroup's share of dh = g w: a thread has C columns, its
// workgroup p.steps classes, which the rows of threads take in turn, several on
// their way at once.  N rows of hidden states.  Two workgroups to a CU: backward
// passes over 131072 x 2048 bf16 take 324 us for 1 row (g, then the weight read
// and written at 5 TB/s) and 350 for 8; one to a CU without loads ahead 518 for
// 1 row, four to a CU 321.
template <typename T, int N, int C>
__global__ __launch_bounds__(256) void k_few_outer(HeadArgs p) {
    const uint32_t d = (blockIdx.y * blockDim.x + threadIdx.x) * C;
    if (d >= p.width) return;
    const uint32_t left = p.width - d;
    float h[N][C], sum[N][C];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        Pack<T, C> x{};
        // what a row that takes no part holds reaches no gradient
        const bool in = uint32_t(n) < p.n &&
                        (p.all || (p.label && load_label(p.label, p.label_bytes, n, p.classes) >= 0));
        if (in && p.grad_weight)
            x = load_pack<C>(static_cast<const T *>(p.hidden) + n * p.hidden_stride + d, left, T{});
#pragma unroll
        for (int i = 0; i < C; ++i) {
            h[n][i] = widen(x.at(i));
            sum[n][i] = 0.0f;
        }
    }
    const uint32_t end = min(p.classes, (blockIdx.x + 1) * p.steps);
    constexpr uint32_t kClasses = N > 8 ? 2 : 4;         // on their way at once
    for (uint32_t v0 = blockIdx.x * p.steps + threadIdx.y; v0 < end; v0 += kClasses * blockDim.y) {
        float gv[kClasses][N];
        Pack<T, C> w[kClasses];
#pragma unroll
        for (uint32_t u = 0; u < kClasses; ++u) {
            const uint32_t v = min(v0 + u * blockDim.y, end - 1);
            const float *g = static_cast<const float *>(p.slope) + uint64_t(v) * kFewRows;
#pragma unroll
            for (int n = 0; n < N; ++n) gv[u][n] = g[n];
            if (p.grad_hidden) w[u] = load_pack<C>(static_cast<const T *>(p.weight) + v * p.weight_stride + d, left, T{});
        }
#pragma unroll
        for (uint32_t u = 0; u < kClasses; ++u) {
            const uint32_t v = v0 + u * blockDim.y;
            if (v >= end) break;
            if (p.grad_hidden) {
#pragma unroll
                for (int n = 0; n < N; ++n)
#pragma unroll
                    for (int i = 0; i < C; ++i) sum[n][i] = fmaf(gv[u][n], widen(w[u].at(i)), sum[n][i]);
            }
            if (p.grad_weight) {
                float x[C] = {};
#pragma unroll
                for (int n = 0; n < N; ++n)
#pragma unroll
                    for (int i = 0; i < C; ++i) x[i] = fmaf(gv[u][n], h[n][i], x[i]);
                store_pack<C>(static_cast<T *>(p.grad_weight) + uint64_t(v) * p.width + d, narrow_pack<T>(x), left);
            }
        }
    }
    if (!p.grad_hidden) return;
    const uint32_t split = blockIdx.x * blockDim.y + threadIdx.y;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        Pack<float, C> x;
#pragma unroll
        for (int i = 0; i < C; ++i) x.put(i, sum[n][i]);
        if (uint32_t(n) < p.n) store_pack<C>(p.sum + (uint64_t(split) * p.n + n) * p.sum_stride + d, x);
    }
}

// dh from the splits: 64 columns of a row to a workgroup, splits over its 16 waves.
template <typename T>
__global__ __launch_bounds__(1024) void k_few_join(HeadArgs p) {
    __shared__ float lds[16][64];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, d = blockIdx.x * 64 + lane, n = blockIdx.y;
    float sum = 0.0f;
    if (d < p.width)
#pragma unroll 8
        for (uint32_t s = wave; s < p.splits; s += 16) sum += p.sum[(uint64_t(s) * p.n + n) * p.sum_stride + d];
    lds[wave][lane] = sum;
    __syncthreads();
    if (wave || d >= p.width) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) sum += lds[w][lane];
    // rows that take no part: 0 x w is not 0 for every w
    const bool in = p.all || (p.label && load_label(p.label, p.label_bytes, n, p.classes) >= 0);
    static_cast<T *>(p.grad_hidden)[uint64_t(n) * p.width + d] = narrow<T>(in ? sum : 0.0f);
}

}  // namespace tmtrain
