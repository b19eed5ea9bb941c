// label_rows.h -- label log-probabilities where the classes of a position are
// a contiguous row, as in (N, C) or channels last.
//
// W waves run through a row, 8 (or 4) classes to a lane and load, with a
// running maximum per lane; the lanes' sums are joined at the end.  A long row
// among few is cut into `groups` parts, which k_label_rows_join puts together.
// Bound by the bytes of the logits; a row is read once.
//
// The k likeliest classes need no second reading either: a lane notes its
// largest logit and the load it came with.  The wave's likeliest class then is
// that of the lane that leads; only that lane's own classes, a 64 W-th of the
// row, are looked through again for its next one, by the whole wave.  After k
// rounds the waves' lists are merged by counting, for every candidate, the
// larger ones.
#pragma once

#include "label.h"

namespace tmtrain {

constexpr int kRowLoads = 4;                               // loads in flight per lane

struct RowPart {                                           // of one part of a row, followed by its k keys
    Sums sums;
};

// The sums of a wave's lanes together, the same in every lane.
__device__ __forceinline__ Sums wave_join(Sums r) {
    lift(r, wave_max(r.m));
    return {r.m, wave_sum(r.s), wave_sum(r.t), wave_sum(r.f)};
}

// Results of row n (outer o, inner i) by one thread.
template <typename T>
__device__ __forceinline__ void put_row(const LabelArgs &a, uint32_t n, const T *x, const Found &q) {
    if (a.logp) {
        const int32_t y = load_label(a.label, a.label_bytes, n, a.classes);
        a.logp[n] = y < 0 ? 0.0f : log_prob(q, widen(x[y]));
    }
    if (a.entropy) a.entropy[n] = q.entropy;
    if (a.mean) a.mean[n] = q.mean;
    if (a.stats) {
        a.stats[2 * uint64_t(n)] = q.m;
        a.stats[2 * uint64_t(n) + 1] = stats_logs(q);
    }
}
__device__ __forceinline__ void put_row_top(const LabelArgs &a, uint32_t o, uint32_t i, uint32_t rank, uint64_t key,
                                            const Found &q) {
    const int64_t at = o * a.ts[0] + rank * a.ts[1] + i * a.ts[2];
    a.index[at] = int32_t(~uint32_t(key));
    a.top[at] = log_prob(q, unordered(uint32_t(key >> 32)));
}

// The likeliest class of a lane below `floor`, found by the whole wave: the
// lane's loads begin at `first`, `stride` classes apart.
template <typename T, int V>
__device__ __forceinline__ uint64_t next_of(const T *x, uint32_t first, uint32_t end, uint32_t stride, uint64_t floor) {
    const uint32_t lane = threadIdx.x & 63;
    uint64_t best = 0;
    for (uint64_t c = first + uint64_t(lane) * stride; c < end; c += uint64_t(64) * stride) {
        const uint32_t n = min(uint32_t(V), end - uint32_t(c));
        const Pack<T, V> r = load_pack<V>(x + c, n, T{});
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const uint64_t key = top_key(widen(r.at(j)), uint32_t(c) + j);
            if (uint32_t(j) < n && key < floor && key > best) best = key;
        }
    }
    return wave_max(best);
}

template <typename T, int W, bool F>
__global__ void __launch_bounds__(W == 1 ? 256 : 64 * W, F ? 4 : 8) k_label_rows(LabelArgs a) {
    constexpr int V = 16 / sizeof(T);
    constexpr uint32_t kStride = 64 * W * V;               // classes between two loads of a lane
    __shared__ Sums sums[W];
    __shared__ uint64_t keys[W][32];
    const uint32_t lane = threadIdx.x & 63, wave = W == 1 ? 0 : threadIdx.x >> 6;
    const uint32_t t = wave * 64 + lane;
    const uint32_t n = W == 1 ? blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)
                              : a.div_groups.div(blockIdx.x);
    if (W == 1 && n >= a.n) return;                        // whole waves; nothing is shared between them
    const uint32_t part = W == 1 ? 0 : blockIdx.x - n * a.groups;
    const uint32_t o = a.div_inner.div(n), i = n - o * a.inner;
    const T *x = static_cast<const T *>(a.x) + o * a.xs[0] + i * a.xs[2];
    const float *field = F ? a.field + o * a.fs[0] + i * a.fs[2] : nullptr;
    // parts of whole strides
    const uint32_t strides = (a.classes + kStride - 1) / kStride, each = (strides + a.groups - 1) / a.groups;
    const uint32_t c0 = min(a.classes, part * each * kStride), end = min(a.classes, c0 + each * kStride);
    const uint32_t first = c0 + t * V;                     // of this lane

    Sums r = kNothing;
    float best = -INFINITY;                                // the lane's largest logit, and the first class of its load
    uint32_t from = first;
    const T none = narrow<T>(-INFINITY);                   // past the end
    const auto run = [&](Pack<T, V> (&held)[kRowLoads], uint32_t c) __attribute__((always_inline)) {
        float m = r.m;
#pragma unroll
        for (int u = 0; u < kRowLoads; ++u) {
            float most = widen(held[u].at(0));
#pragma unroll
            for (int j = 1; j < V; ++j) most = fmaxf(most, widen(held[u].at(j)));
            const bool leads = most > best;
            best = leads ? most : best;
            from = leads ? c + u * kStride : from;
            m = fmaxf(m, most);
        }
        lift(r, m);
#pragma unroll
        for (int u = 0; u < kRowLoads; ++u) forget_widened(held[u]);
        by_kind<T, F>(fabsf(m), a.entropy, [&](auto kind) __attribute__((always_inline)) {
            const typename decltype(kind)::type ref(m);
            Sums some = kNothing;
#pragma unroll
            for (int u = 0; u < kRowLoads; ++u) {
                const uint32_t at = c + u * kStride;
                Pack<float, V> phi{};
                if (ref.kMean && at < end) phi = load_field<V>(field + at * a.fs[1], a.fs[1], end - at);
#pragma unroll
                for (int j = 0; j < V; ++j) ref.take(some, widen(held[u].at(j)), phi.at(j));
            }
            ref.close(r, some);
        });
    };
    // whole rounds of loads, then one that asks at every load whether it is there
    uint32_t c = first;
    uint32_t left = end - min(end, c0 + wave * 64 * V);    // from the wave's first class on
    constexpr uint32_t kRound = kRowLoads * kStride;
    for (; left >= kRound - kStride + 64 * V; left -= min(left, kRound), c += kRound) {
        Pack<T, V> held[kRowLoads];
#pragma unroll
        for (int u = 0; u < kRowLoads; ++u) held[u] = load_pack<V>(x + c + u * kStride);
        run(held, c);
    }
    if (c < end) {
        Pack<T, V> held[kRowLoads];
#pragma unroll
        for (int u = 0; u < kRowLoads; ++u) {
            const uint32_t at = c + u * kStride;
            if (at < end) {
                held[u] = load_pack<V>(x + at, end - at, none);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) held[u].put(j, none);
            }
        }
        run(held, c);
    }
    r = wave_join(r);

    // the wave's k likeliest classes; lane j of the wave keeps the j-th
    uint64_t mine = 0;
    if (a.k) {
        // the lane's likeliest class, exactly: within the load that it came with
        uint64_t key = 0;
        if (first < end) {
            const uint32_t count = min(uint32_t(V), end - from);
            const Pack<T, V> again = load_pack<V>(x + from, count, none);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const uint64_t one = top_key(widen(again.at(j)), from + j);
                if (uint32_t(j) < count && one > key) key = one;
            }
        }
        for (uint32_t rank = 0; rank < a.k; ++rank) {
            const uint64_t lead = wave_max(key);
            if (lead == 0) break;                          // no classes are left
            if (lane == rank) mine = lead;
            if (rank + 1 == a.k) break;
            const int owner = __ffsll(static_cast<long long>(__ballot(key == lead))) - 1;
            const uint64_t next = next_of<T, V>(x, c0 + (wave * 64 + owner) * V, end, kStride, lead);
            if (int(lane) == owner) key = next;
        }
    }
    if constexpr (W == 1) {
        const Found q = found(r);
        if (lane == 0) put_row(a, n, x, q);
        if (lane < a.k) put_row_top(a, o, i, lane, mine, q);
    } else {
        if (lane == 0) sums[wave] = r;
        if (lane < a.k) keys[wave][lane] = mine;
        __syncthreads();
        const Sums all = wave_join(lane < W ? sums[lane] : kNothing);
        const Found q = found(all);
        char *out = static_cast<char *>(a.partial) + uint64_t(blockIdx.x) * (sizeof(RowPart) + a.k * 8);
        if (t == 0) {
            if (a.groups == 1) put_row(a, n, x, q);
            else reinterpret_cast<RowPart *>(out)->sums = all;
        }
        // a candidate's place is the number of larger ones; empty places (0) come last, in any order
        for (uint32_t j = t; j < W * a.k; j += 64 * W) {
            const uint64_t key = keys[j / a.k][j % a.k];
            uint32_t rank = 0;
            for (uint32_t w = 0; w < W; ++w)
                for (uint32_t v = 0; v < a.k; ++v)
                    rank += keys[w][v] > key || (key == 0 && w * a.k + v < j && keys[w][v] == 0);
            if (rank < a.k) {
                if (a.groups == 1) put_row_top(a, o, i, rank, key, q);
                else reinterpret_cast<uint64_t *>(out + sizeof(RowPart))[rank] = key;
            }
        }
    }
}

// Puts the parts of a row together, in their order.
constexpr uint32_t kRowMostParts = 64;

template <typename T>
__global__ void __launch_bounds__(256) k_label_rows_join(LabelArgs a) {
    __shared__ uint64_t keys[kRowMostParts * 32];
    const uint32_t n = blockIdx.x;
    const uint32_t o = a.div_inner.div(n), i = n - o * a.inner;
    const T *x = static_cast<const T *>(a.x) + o * a.xs[0] + i * a.xs[2];
    const uint64_t size = sizeof(RowPart) + a.k * 8;
    const char *in = static_cast<const char *>(a.partial) + uint64_t(n) * a.groups * size;
    Sums r = kNothing;
    for (uint32_t p = threadIdx.x & 63; p < a.groups; p += 64)
        r = join(r, reinterpret_cast<const RowPart *>(in + p * size)->sums);
    const Found q = found(wave_join(r));
    if (threadIdx.x == 0) put_row(a, n, x, q);
    const uint32_t count = a.groups * a.k;
    for (uint32_t j = threadIdx.x; j < count; j += 256)
        keys[j] = reinterpret_cast<const uint64_t *>(in + j / a.k * size + sizeof(RowPart))[j % a.k];
    __syncthreads();
    for (uint32_t j = threadIdx.x; j < count; j += 256) {
        const uint64_t key = keys[j];
        if (key == 0) continue;
        uint32_t rank = 0;
        for (uint32_t v = 0; v < count; ++v) rank += keys[v] > key;
        if (rank < a.k) put_row_top(a, o, i, rank, key, q);
    }
}

// Gradient of rows, with the forward call's statistics: part blockIdx.x of the
// rows' classes, 256 threads.
template <typename T, bool F>
__global__ void __launch_bounds__(256) k_label_grad_rows(LabelGradArgs a) {
    constexpr int V = 16 / sizeof(T);
    const uint32_t n = a.div_groups.div(blockIdx.x), part = blockIdx.x - n * a.groups;
    const uint32_t o = a.div_inner.div(n), i = n - o * a.inner;
    const T *x = static_cast<const T *>(a.x) + o * a.xs[0] + i * a.xs[2];
    T *out = static_cast<T *>(a.grad) + o * a.gs[0] + i * a.gs[2];
    const float *field = F ? a.field + o * a.fs[0] + i * a.fs[2] : nullptr;
    const uint32_t c0 = part * a.share, end = min(a.classes, c0 + a.share);
    const int32_t y = a.up_logp ? load_label(a.label, a.label_bytes, n, a.classes) : -1;
    Slope g;
    g.m = a.stats[2 * uint64_t(n)];
    g.logs = a.stats[2 * uint64_t(n) + 1];
    g.entropy = a.up_entropy ? a.entropy[n] : 0.0f;
    g.mean = F ? a.mean[n] : 0.0f;
    g.a = y < 0 || g.logs == INFINITY ? 0.0f : a.up_logp[n];
    g.h = a.up_entropy ? a.up_entropy[n] : 0.0f;
    g.f = F ? a.up_mean[n] : 0.0f;
    for (uint64_t c = c0 + threadIdx.x * V; c < end; c += 256 * V * 2) {
        Pack<T, V> held[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint64_t at = c + u * 256 * V;
            if (at < end) held[u] = load_pack<V>(x + at, end - uint32_t(at), T{});
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint64_t at = c + u * 256 * V;
            if (at >= end) break;
            Pack<float, V> phi{};
            if constexpr (F) phi = load_field<V>(field + at * a.fs[1], a.fs[1], end - uint32_t(at));
            float v[V];
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = slope_of<T, F>(g, a.up_entropy, widen(held[u].at(j)), phi.at(j));
            if (uint32_t(y) - uint32_t(at) < V) {          // false for y < 0
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (uint32_t(y) == uint32_t(at) + j) v[j] += g.a;
            }
            store_pack<V>(out + at, narrow_pack<T, V>(v), end - uint32_t(at));
        }
    }
}

}  // namespace tmtrain
