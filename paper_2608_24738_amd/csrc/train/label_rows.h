// label_rows.h -- label log-probabilities where the classes of a position are
// a contiguous row, as in (N, C) or channels last.
//
// W waves run through a row, 8 (or 4) classes to a lane and load, with a
// running maximum per lane; the lanes' sums are joined at the end.  Short rows
// among many are held by 16 lanes each (65536 x 512: 67 MB in 14 us, 4.9 TB/s).
// A long row among few is cut into `groups` parts, which k_label_rows_join puts
// together.
// Bound by the bytes of the logits; a row is read once (bf16 4096 x 32768 with
// the entropy: 268 MB in 44 us, 6.1 TB/s, the gradient 537 MB in 81 us, 6.6 TB/s;
// 512 x 50021 with 5 alternatives: 51 MB in 18.5 us, of them 6 the alternatives';
// 1 x 131072 likewise 10.8 us, all of it latency).
//
// The k likeliest classes need no second reading either: a lane notes its
// largest logit and the load it came with.  The k-th largest of the lanes'
// bests bounds the k likeliest classes from below, so only the k lanes at or
// above it, each with a 64 W-th of the row, are looked through again; what
// they hold at or above the bound is ranked by counting.
#pragma once

#include "label.h"

namespace tmtrain {

constexpr uint32_t kRowFound = 256;                        // classes at or above the bound that a row has room for
constexpr int kRowLoads = 4;                               // loads in flight per lane

struct RowPart {                                           // of one part of a row, followed by its k keys
    Sums sums;
};

// The sums of a wave's lanes together, the same in every lane.
__device__ __forceinline__ Sums wave_join(Sums r) {
    lift(r, wave_max(r.m));
    return {r.m, wave_sum(r.s), wave_sum(r.t), wave_sum(r.f)};
}

// The workgroup's number in a grid of two dimensions: one of them holds fewer
// than 2^32 threads.
__device__ __forceinline__ uint32_t block_number() { return blockIdx.y * gridDim.x + blockIdx.x; }

// Results of row n by one thread.
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
    // a row with NaN may have fewer classes in order than were asked for
    a.index[at] = key ? int32_t(~uint32_t(key)) : 0;
    a.top[at] = log_prob(q, unordered(uint32_t(key >> 32)));
}

// The k largest of `count` <= 64 falling lists of k keys in LDS, by one wave:
// lane j gets the j-th.  0 where there are no more.
__device__ __forceinline__ uint64_t merge_lists(const uint64_t *lists, uint32_t count, uint32_t k) {
    const uint32_t lane = threadIdx.x & 63;
    uint32_t at = 0;
    uint64_t mine = 0, key = lane < count ? lists[lane * k] : 0;
    for (uint32_t rank = 0; rank < k; ++rank) {
        const uint64_t lead = wave_max(key);
        if (lead == 0) break;
        if (lane == rank) mine = lead;
        if (key == lead) key = ++at < k ? lists[lane * k + at] : 0;
    }
    return mine;
}

// E: with the entropy, F: with a field (and the entropy), K: with the likeliest classes.
template <typename T, int W, bool E, bool F, bool K>
__global__ void __launch_bounds__(W == 1 ? 256 : 64 * W, K && !F ? 7 : 4) k_label_rows(LabelArgs a) {
    constexpr int V = 16 / sizeof(T);
    constexpr uint32_t kStride = 64 * W * V;               // classes between two loads of a lane
    constexpr int R = W == 1 ? 4 : 1;                      // rows of a workgroup
    __shared__ Sums sums[W];
    __shared__ uint64_t bests_of[K ? R : 1][W * 64], leads_of[K ? R : 1][W * 32], found_of[K ? R : 1][kRowFound];
    __shared__ uint64_t top_of[K ? R : 1][32];
    __shared__ uint32_t count_of[R];
    const uint32_t lane = threadIdx.x & 63, wave = W == 1 ? 0 : threadIdx.x >> 6;
    const uint32_t t = wave * 64 + lane;
    const uint32_t block = block_number();
    const uint32_t n = W == 1 ? block * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : a.div_groups.div(block);
    if (n >= a.n) return;                                  // whole waves, which share nothing, or whole workgroups
    const uint32_t part = W == 1 ? 0 : block - n * a.groups;
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
    // 16-bit logits, none of the likeliest asked for: a round against the
    // reference so far, which is as good as the maximum until a sum outgrows it
    const auto stride_over = [&](const Pack<T, V> (&held)[kRowLoads], uint32_t c) __attribute__((always_inline)) {
        const Ref<true, E, F> ref(r.m);
        Sums some = kNothing;
#pragma unroll
        for (int u = 0; u < kRowLoads; ++u) {
            Pack<float, V> phi{};
            if constexpr (F) phi = load_field<V>(field + (c + u * kStride) * a.fs[1], a.fs[1], V);
#pragma unroll
            for (int j = 0; j < V; ++j) ref.take(some, widen(held[u].at(j)), phi.at(j));
            __builtin_amdgcn_sched_barrier(0);             // one load's terms at a time: registers
        }
        if (!__all(some.s < 1e4f)) return false;           // nor NaN
        ref.close(r, some);
        return true;
    };
    const auto run = [&](auto &held, uint32_t c) __attribute__((always_inline)) {
        constexpr int N = sizeof(held) / sizeof(held[0]);
        float m = r.m;
#pragma unroll
        for (int u = 0; u < N; ++u) {
            float most = widen(held[u].at(0));
#pragma unroll
            for (int j = 1; j < V; ++j) most = fmaxf(most, widen(held[u].at(j)));
            if constexpr (K) {
                const bool leads = most > best;
                best = leads ? most : best;
                from = leads ? c + u * kStride : from;
            }
            m = fmaxf(m, most);
        }
        lift(r, m);
#pragma unroll
        for (int u = 0; u < N; ++u) forget_widened(held[u]);
        by_near<T>(fabsf(m), [&](auto near) __attribute__((always_inline)) {
            const Ref<decltype(near)::value, E, F> ref(m);
            Sums some = kNothing;
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const uint32_t at = c + u * kStride;
                Pack<float, V> phi{};
                if constexpr (F) phi = load_field<V>(field + at * a.fs[1], a.fs[1], end - at);
#pragma unroll
                for (int j = 0; j < V; ++j) ref.take(some, widen(held[u].at(j)), phi.at(j));
                __builtin_amdgcn_sched_barrier(0);         // one load's terms at a time: registers
            }
            ref.close(r, some);
        });
    };
    // whole rounds of loads, then one load after the other
    uint32_t c = first;
    constexpr uint32_t kRound = kRowLoads * kStride;
    uint32_t rounds = 0;                                   // of the wave, all of its lanes' loads whole
    const uint32_t own = end - min(end, c0 + wave * 64 * V);
    if (own >= kRound - kStride + 64 * V) rounds = (own - (kRound - kStride + 64 * V)) / kRound + 1;
    if (sizeof(T) == 2 && !K && rounds > 1) {
        Pack<T, V> first_load[1] = {load_pack<V>(x + c)};
        run(first_load, c);
        c += kStride;
        for (--rounds; rounds && __all(fabsf(r.m) <= kNear); --rounds, c += kRound) {
            Pack<T, V> held[kRowLoads];
#pragma unroll
            for (int u = 0; u < kRowLoads; ++u) held[u] = load_pack<V>(x + c + u * kStride);
            if (!stride_over(held, c)) break;
        }
    }
    for (; rounds; --rounds, c += kRound) {
        Pack<T, V> held[kRowLoads];
#pragma unroll
        for (int u = 0; u < kRowLoads; ++u) held[u] = load_pack<V>(x + c + u * kStride);
        run(held, c);
    }
    for (; c < end; c += kStride) {
        Pack<T, V> held[1] = {load_pack<V>(x + c, end - c, none)};
        run(held, c);
    }
    r = wave_join(r);

    if constexpr (W > 1) {
        if (lane == 0) sums[wave] = r;
    }
    const auto sync = [] {
        if constexpr (W == 1) wave_sync();
        else __syncthreads();
    };
    uint64_t mine = 0;                                     // lane j of the row's first wave: the j-th likeliest class
    if constexpr (K) {
        const uint32_t row = W == 1 ? threadIdx.x >> 6 : 0;
        uint64_t *const bests = bests_of[row] + wave * 64, *const leads = leads_of[row];
        uint64_t *const among = found_of[row], *const top = top_of[row];
        uint32_t *const count = &count_of[row];
        // the lane's likeliest class, exactly: within the load that it came with
        uint64_t key = 0;
        if (first < end) {
            const uint32_t have = min(uint32_t(V), end - from);
            const Pack<T, V> again = load_pack<V>(x + from, have, none);
            uint32_t at = ~0u;
#pragma unroll
            for (int j = V - 1; j >= 0; --j)
                if (uint32_t(j) < have && widen(again.at(j)) == best) at = from + j;
            if (at != ~0u) key = top_key(best, at);
        }
        // the k best lanes of the wave, in order
        bests[lane] = key;
        if (lane < a.k) leads[wave * a.k + lane] = 0;
        if (t < a.k) top[t] = 0;
        if (t == 0) *count = 0;
        wave_sync();
        uint32_t above = 0;
        for (int v = 0; v < 64; ++v) above += bests[v] > key;
        if (above < a.k && key) leads[wave * a.k + above] = key;
        sync();
        // the k-th best lane of the row (0: there are fewer)
        uint64_t least = 0;
        if (W == 1) {
            least = leads[a.k - 1];
        } else if (W * a.k <= 64) {
            const uint64_t one = lane < W * a.k ? leads[lane] : 0;
            above = 0;
            for (uint32_t v = 0; v < W * a.k; ++v) above += leads[v] > one;
            const uint64_t kth = __ballot(one != 0 && above == a.k - 1);
            if (kth) least = leads[__ffsll(static_cast<long long>(kth)) - 1];
        } else {
            bests[lane] = merge_lists(leads, W, a.k);
            wave_sync();
            least = bests[a.k - 1];
        }
        // what the lanes at or above it hold at or above it
        const float bound = least ? unordered(uint32_t(least >> 32)) : -INFINITY;
        for (uint64_t lanes = __ballot(key != 0 && key >= least); lanes; lanes &= lanes - 1) {
            const uint32_t owner = __ffsll(static_cast<long long>(lanes)) - 1;
            for (uint64_t at = c0 + (wave * 64 + owner) * V + uint64_t(lane) * kStride; at < end; at += 64 * kStride) {
                const uint32_t have = min(uint32_t(V), end - uint32_t(at));
                const Pack<T, V> again = load_pack<V>(x + at, have, none);
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (uint32_t(j) < have && widen(again.at(j)) >= bound) {
                        const uint64_t one = top_key(widen(again.at(j)), uint32_t(at) + j);
                        if (one >= least) {
                            const uint32_t place = atomicAdd(count, 1u);   // any order: they are ranked next
                            if (place < kRowFound) among[place] = one;
                        }
                    }
            }
        }
        sync();
        const uint32_t n_found = *count;
        if (n_found <= kRowFound) {
            if (wave == 0)
                for (uint32_t v = lane; v < n_found; v += 64) {
                    const uint64_t one = among[v];
                    above = 0;
                    for (uint32_t u = 0; u < n_found; ++u) above += among[u] > one;
                    if (above < a.k) top[above] = one;
                }
        } else {
            // one lane's classes hold most of the largest logits: one pass over the row for each
            uint64_t last = ~uint64_t(0);
            for (uint32_t rank = 0; rank < a.k; ++rank) {
                uint64_t next = 0;
                for (uint64_t at = first; at < end; at += kStride) {
                    const uint32_t have = min(uint32_t(V), end - uint32_t(at));
                    const Pack<T, V> again = load_pack<V>(x + at, have, none);
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const uint64_t one = top_key(widen(again.at(j)), uint32_t(at) + j);
                        if (uint32_t(j) < have && one < last && one > next) next = one;
                    }
                }
                next = wave_max(next);
                if (lane == 0) leads[wave] = next;
                sync();
                last = leads[0];
                for (int w = 1; w < W; ++w) last = last > leads[w] ? last : leads[w];
                sync();
                if (t == 0) top[rank] = last;
            }
        }
        wave_sync();
        if (wave == 0 && lane < a.k) mine = top[lane];
    } else if constexpr (W > 1) {
        __syncthreads();
    }
    if (wave > 0) return;
    if constexpr (W > 1) r = wave_join(lane < W ? sums[lane] : kNothing);
    if (W == 1 || a.groups == 1) {
        const Found q = found(r);
        if (lane == 0) put_row(a, n, x, q);
        if (K && lane < a.k) put_row_top(a, o, i, lane, mine, q);
    } else {
        char *out = static_cast<char *>(a.partial) + uint64_t(block) * (sizeof(RowPart) + a.k * 8);
        if (lane == 0) reinterpret_cast<RowPart *>(out)->sums = r;
        if (K && lane < a.k) reinterpret_cast<uint64_t *>(out + sizeof(RowPart))[lane] = mine;
    }
}

// Short rows among many: 16 lanes hold a row, four rows to a wave, and reduce
// by rotations.  The likeliest classes take a selection each, over the classes
// held.
constexpr uint32_t kShortRows = 16;                        // of a workgroup

// L: loads of a lane.
template <typename T, int L, bool E, bool F, bool K>
__global__ void __launch_bounds__(16 * kShortRows) k_label_rows_short(LabelArgs a) {
    constexpr int V = 16 / sizeof(T);
    const uint32_t lane = threadIdx.x & 15;
    const uint32_t n = block_number() * kShortRows + (threadIdx.x >> 4);
    if (n >= a.n) return;                                  // all 16 lanes
    const uint32_t o = a.div_inner.div(n), i = n - o * a.inner;
    const T *x = static_cast<const T *>(a.x) + o * a.xs[0] + i * a.xs[2];
    const float *field = F ? a.field + o * a.fs[0] + i * a.fs[2] : nullptr;
    const T none = narrow<T>(-INFINITY);
    Pack<T, V> held[L];
    uint32_t from[L];                              // the last load begins further back, its doubles are -inf
#pragma unroll
    for (int u = 0; u < L; ++u) {
        from[u] = min((u * 16 + lane) * V, a.classes - V);
        held[u] = load_pack<V>(x + from[u]);
    }
    Sums r = kNothing;
#pragma unroll
    for (int u = 0; u < L; ++u) {
        const uint32_t doubles = (u * 16 + lane) * V - from[u];
        if (doubles) {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (uint32_t(j) < doubles) held[u].put(j, none);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) r.m = fmaxf(r.m, widen(held[u].at(j)));
    }
    r.m = row_max(r.m);
    by_near<T>(fabsf(r.m), [&](auto near) __attribute__((always_inline)) {
        const Ref<decltype(near)::value, E, F> ref(r.m);
        Sums some = kNothing;
#pragma unroll
        for (int u = 0; u < L; ++u) {
            Pack<float, V> phi{};
            if constexpr (F) phi = load_field<V>(field + from[u] * a.fs[1], a.fs[1], V);
#pragma unroll
            for (int j = 0; j < V; ++j) ref.take(some, widen(held[u].at(j)), phi.at(j));
        }
        ref.close(r, some);
    });
    r.s = row_sum(r.s);
    if constexpr (E) r.t = row_sum(r.t);
    if constexpr (F) r.f = row_sum(r.f);
    const Found q = found(r);
    if (lane == 0) put_row(a, n, x, q);
    if constexpr (K) {
        float lx = INFINITY;                               // the last class found
        uint32_t lc = ~0u;
        for (uint32_t rank = 0; rank < a.k; ++rank) {
            float best = -INFINITY;
            uint32_t at = ~0u;
#pragma unroll
            for (int u = 0; u < L; ++u) {
                const uint32_t doubles = (u * 16 + lane) * V - from[u];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float v = widen(held[u].at(j));
                    const uint32_t c = from[u] + j;
                    const bool open = uint32_t(j) >= doubles && (v < lx || (v == lx && c > lc) || lc == ~0u) && v == v;
                    if (open && (v > best || at == ~0u)) {
                        best = v;
                        at = c;
                    }
                }
            }
            const uint64_t lead = row_max(at == ~0u ? uint64_t(0) : top_key(best, at));
            lx = unordered(uint32_t(lead >> 32));
            lc = ~uint32_t(lead);
            if (lane == (rank & 15)) put_row_top(a, o, i, rank, lead, q);
            if (lead == 0) lx = -INFINITY;                 // a row with NaN: nothing is behind it
        }
    }
}

// Puts the parts of a row together: a lane for each.
constexpr uint32_t kRowMostParts = 64;

template <typename T>
__global__ void __launch_bounds__(64) k_label_rows_join(LabelArgs a) {
    __shared__ uint64_t keys[kRowMostParts * 32];
    const uint32_t n = blockIdx.x, lane = threadIdx.x;
    const uint32_t o = a.div_inner.div(n), i = n - o * a.inner;
    const T *x = static_cast<const T *>(a.x) + o * a.xs[0] + i * a.xs[2];
    const uint64_t size = sizeof(RowPart) + a.k * 8;
    const char *in = static_cast<const char *>(a.partial) + uint64_t(n) * a.groups * size + lane * size;
    Sums r = kNothing;
    if (lane < a.groups) {
        r = reinterpret_cast<const RowPart *>(in)->sums;
        for (uint32_t j = 0; j < a.k; ++j) keys[lane * a.k + j] = reinterpret_cast<const uint64_t *>(in + sizeof(RowPart))[j];
    }
    const Found q = found(wave_join(r));
    if (lane == 0) put_row(a, n, x, q);
    __syncthreads();
    const uint64_t mine = merge_lists(keys, a.groups, a.k);
    if (lane < a.k) put_row_top(a, o, i, lane, mine, q);
}

// Gradient of rows, with the forward call's statistics: a workgroup to a part
// of a row, or a wave or 16 lanes to a row.
template <typename T, bool E, bool F>
__global__ void __launch_bounds__(256) k_label_grad_rows(LabelGradArgs a) {
    constexpr int V = 16 / sizeof(T);
    const uint32_t lanes = a.lanes, t = threadIdx.x & (lanes - 1);
    const uint32_t block = block_number();
    uint32_t at_part = block;
    if (lanes == 16) at_part = block * 16 + (threadIdx.x >> 4);
    if (lanes == 64) at_part = block * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t n = a.div_groups.div(at_part), part = at_part - n * a.groups;
    if (n >= a.n) return;
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
    const Slope all[1] = {g};
    by_near<T>(farthest(all), [&](auto near) __attribute__((always_inline)) {
        const Grad<decltype(near)::value, E, F> grad(g);
        for (uint32_t c = c0 + t * V; c < end; c += lanes * V * 2) {
            Pack<T, V> held[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t at = c + u * lanes * V;
                if (at < end) held[u] = load_pack<V>(x + at, end - at, T{});
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t at = c + u * lanes * V;
                if (at >= end) break;
                Pack<float, V> phi{};
                if constexpr (F) phi = load_field<V>(field + at * a.fs[1], a.fs[1], end - at);
                float v[V];
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = grad.at(widen(held[u].at(j)), phi.at(j), 0.0f);
                if (uint32_t(y) - at < V) {                // false for y < 0
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        if (uint32_t(y) == at + j) v[j] += g.a;
                }
                store_pack<V>(out + at, narrow_pack<T, V>(v), end - at);
            }
        }
    });
}

}  // namespace tmtrain
