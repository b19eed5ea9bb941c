// label_maps.h -- label log-probabilities where the classes of a position lie
// apart and neighbouring positions side by side, as in (B, C, *spatial).
//
// A thread owns V neighbouring positions (16 or 8 bytes of logits of one
// class), so a wave reads whole lines of every class plane.  Up to 32 classes
// are held in registers between the passes for the maximum, the sums and the likeliest
// classes (k_label_held): every logit is read once.  More run through in
// blocks of 8 with a running maximum (k_label_run); where there are few
// positions, the waves of a workgroup share the classes and join their sums.
// Class axes of any stride take the same kernels with one position to a thread.
//
// Bound by the bytes of logits, labels and outputs with few classes (bf16
// 8 x 4 x 128^3 with entropy and the likeliest class: 419 MB in 86 us, 4.9 TB/s;
// float32 with a field, forward 688 MB in 138 us, 5.0 TB/s, gradient 955 MB in
// 188 us, 5.1 TB/s; a copy reaches 5.2), by arithmetic, some 13 instructions a
// logit, with more of them (bf16 16 x 21 x 375 x 500: forward 141 MB in 37 us,
// gradient 267 MB in 50 us; 8 x 150 x 128^2 with the entropy: 42 MB in 22 us and
// 81 MB in 29 us).
#pragma once

#include <utility>

#include "label.h"

namespace tmtrain {

// Positions to a thread: 16 bytes, or 8 where the classes held would take more
// than 32 registers or running ones with their sums more than 128.
template <typename T, int C>
constexpr int kHeldV = (C <= 8 ? 16 : 8) / int(sizeof(T));
constexpr int kRunV = 4;

template <int V, typename L>
__device__ __forceinline__ void load_labels_as(const L *p, uint32_t classes, int32_t (&y)[V]) {
    const Pack<L, V> r = load_pack<V>(p);
#pragma unroll
    for (int j = 0; j < V; ++j) y[j] = int64_t(r.at(j)) >= 0 && int64_t(r.at(j)) < int64_t(classes) ? int32_t(r.at(j)) : -1;
}
template <int V>
__device__ __forceinline__ void load_labels(const void *p, int32_t bytes, uint64_t i, uint32_t classes,
                                            int32_t (&y)[V]) {
    if (bytes == 1)
        load_labels_as<V>(static_cast<const uint8_t *>(p) + i, classes, y);
    else if (bytes == 4)
        load_labels_as<V>(static_cast<const int32_t *>(p) + i, classes, y);
    else
        load_labels_as<V>(static_cast<const int64_t *>(p) + i, classes, y);
}

// Where a thread's positions lie.
template <int V>
struct Place {
    uint32_t o, i;              // outer, first inner position
    uint32_t skip;              // positions in front that are another thread's
    uint64_t at;                // in [outer][inner]
};
template <int V, typename Args>
__device__ __forceinline__ Place<V> place(const Args &a, uint32_t thread) {
    Place<V> r;
    r.o = a.div_groups.div(thread);
    // the last thread of an outer position takes whole loads, further back, and
    // writes what is its own: loads behind a branch would be waited for
    const uint32_t own = (thread - r.o * a.groups) * V;
    r.i = min(own, a.inner - V);
    r.skip = own - r.i;
    r.at = uint64_t(r.o) * a.inner + r.i;
    return r;
}

// One step of a selection over the classes, in rising number: the largest one
// behind `last` in the order of the alternatives.  NaN is never picked.
struct Pick {
    float x;
    int32_t c;                  // -1: none yet
};
__device__ __forceinline__ void consider(Pick &best, const Pick &last, float x, int32_t c) {
    const bool open = x < last.x || (x == last.x && c > last.c);
    if (open && (best.c < 0 || x > best.x)) best = {x, c};
}

template <int V>
__device__ __forceinline__ void put_top(const LabelArgs &a, const Place<V> &w, uint32_t rank, const Pick (&best)[V],
                                        const Found (&q)[V]) {
    const int64_t at = w.o * a.ts[0] + rank * a.ts[1] + w.i * a.ts[2];
    Pack<float, V> top{};
    Pack<int32_t, V> index{};
#pragma unroll
    for (int j = 0; j < V; ++j) {
        top.put(j, log_prob(q[j], best[j].x));
        index.put(j, max(best[j].c, 0));                   // NaN everywhere: no class is larger
    }
    if (V == 1 || a.ts[2] == 1) {
        store_own<V>(a.top + at, top, w.skip);
        store_own<V>(a.index + at, index, w.skip);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (uint32_t(j) >= w.skip) {
                a.top[at + j * a.ts[2]] = top.at(j);
                a.index[at + j * a.ts[2]] = index.at(j);
            }
    }
}

// Log-probability (xl: the labels' logits), entropy, mean, statistics.
template <int V>
__device__ __forceinline__ void put_found(const LabelArgs &a, const Place<V> &w, const int32_t (&y)[V],
                                          const float (&xl)[V], const Found (&q)[V]) {
    Pack<float, V> r{};
    if (a.logp) {
#pragma unroll
        for (int j = 0; j < V; ++j) r.put(j, y[j] < 0 ? 0.0f : log_prob(q[j], xl[j]));
        store_own<V>(a.logp + w.at, r, w.skip);
    }
    if (a.entropy) {
#pragma unroll
        for (int j = 0; j < V; ++j) r.put(j, q[j].entropy);
        store_own<V>(a.entropy + w.at, r, w.skip);
    }
    if (a.mean) {
#pragma unroll
        for (int j = 0; j < V; ++j) r.put(j, q[j].mean);
        store_own<V>(a.mean + w.at, r, w.skip);
    }
    if (a.stats) {
        Pack<float, 2 * V> st{};
#pragma unroll
        for (int j = 0; j < V; ++j) {
            st.put(2 * j, q[j].m);
            st.put(2 * j + 1, stats_logs(q[j]));
        }
        store_own<2 * V>(a.stats + 2 * w.at, st, 2 * w.skip);
    }
}

// Up to 32 logits may as well stay widened.
template <typename T, int V, int C>
__device__ __forceinline__ void forget_held(Pack<T, V> (&held)[C]) {
    if constexpr (V * C > 32) {
#pragma unroll
        for (int c = 0; c < C; ++c) forget_widened(held[c]);
    }
}

// The maxima of held classes, two at a time.
template <typename T, int V, int C>
__device__ __forceinline__ void held_maxima(Sums (&r)[V], const Pack<T, V> (&held)[C], uint32_t classes) {
#pragma unroll
    for (int c = 0; c < C; c += 2) {
        if (c + 1 < C && uint32_t(c + 1) < classes) {
#pragma unroll
            for (int j = 0; j < V; ++j)
                r[j].m = max_of(r[j].m, widen(held[c].at(j)), widen(held[c + 1 < C ? c + 1 : c].at(j)));
        } else if (uint32_t(c) < classes) {
#pragma unroll
            for (int j = 0; j < V; ++j) r[j].m = max_of(r[j].m, r[j].m, widen(held[c].at(j)));
        }
    }
}

// Classes whose field is held too; others' is read again for the gradient.
template <int C, int V, bool F>
constexpr int kFieldHeld = F && C * V <= 32 ? C : 1;

// The sums of held classes; r holds the maxima.
// The field is left in `phi` as far as that has room.
template <typename T, int V, int C, bool E, bool F, int P>
__device__ __forceinline__ void held_sums(Sums (&r)[V], Pack<T, V> (&held)[C], uint32_t classes, const float *field,
                                          const int64_t (&fs)[3], Pack<float, V> (&phi)[P]) {
    if constexpr (F && P == C) {
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (uint32_t(c) < classes) phi[c] = load_field<V>(field + c * fs[1], fs[2], V);
    }
    float size = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j) size = fmaxf(size, fabsf(r[j].m));
    forget_held(held);
    by_near<T>(size, [&](auto near) __attribute__((always_inline)) {
        typedef Ref<decltype(near)::value, E, F> R;
        Sums some[V];
#pragma unroll
        for (int j = 0; j < V; ++j) some[j] = kNothing;
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (uint32_t(c) < classes) {
                if (F && P != C) phi[0] = load_field<V>(field + c * fs[1], fs[2], V);
#pragma unroll
                for (int j = 0; j < V; ++j) R(r[j].m).take(some[j], widen(held[c].at(j)), F ? phi[P == C ? c : 0].at(j) : 0.0f);
            }
#pragma unroll
        for (int j = 0; j < V; ++j) R(r[j].m).close(r[j], some[j]);
    });
    forget_held(held);
}

// At most C classes, held in registers.  E: with the entropy, F: with a field
// (and the entropy, which then costs nothing).
template <typename T, int V, int C, bool E, bool F>
__global__ void __launch_bounds__(256) k_label_held(LabelArgs a) {
    const uint32_t thread = blockIdx.x * 256 + threadIdx.x;
    if (thread >= a.outer * a.groups) return;
    const Place<V> w = place<V>(a, thread);
    const T *x = static_cast<const T *>(a.x) + w.o * a.xs[0] + w.i * a.xs[2];
    Pack<T, V> held[C];
#pragma unroll
    for (int c = 0; c < C; ++c)
        if (uint32_t(c) < a.classes) held[c] = load_pack<V>(x + c * a.xs[1]);
    int32_t y[V];
    if (a.logp) load_labels<V>(a.label, a.label_bytes, w.at, a.classes, y);
    Sums r[V];
    float xl[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        r[j] = kNothing;
        xl[j] = 0.0f;
    }
    held_maxima(r, held, a.classes);
    const float *const field = F ? a.field + w.o * a.fs[0] + w.i * a.fs[2] : nullptr;
    Pack<float, V> phi[kFieldHeld<C, V, F>] = {};
    held_sums<T, V, C, E, F>(r, held, a.classes, field, a.fs, phi);
    Found q[V];
#pragma unroll
    for (int j = 0; j < V; ++j) q[j] = found(r[j]);
    if (a.logp) {
        // few classes: a comparison for each; of more, the label's logit is read once more
        if constexpr (C <= 8) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (y[j] == c) xl[j] = widen(held[c].at(j));
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) xl[j] = widen(x[max(y[j], 0) * a.xs[1] + j * a.xs[2]]);
        }
    }
    put_found<V>(a, w, y, xl, q);
    if (!a.k) return;
    forget_held(held);
    // the likeliest class is the first whose logit is the maximum; each other one takes a pass
    Pick best[V], last[V];
#pragma unroll
    for (int j = 0; j < V; ++j) best[j] = {r[j].m, 0};
#pragma unroll
    for (int c = C - 1; c >= 0; --c)
        if (uint32_t(c) < a.classes) {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (widen(held[c].at(j)) == r[j].m) best[j].c = c;
        }
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (q[j].dead) best[j].x = -INFINITY;
    put_top<V>(a, w, 0, best, q);
    for (uint32_t rank = 1; rank < a.k; ++rank) {
        forget_held(held);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            last[j] = best[j];
            best[j] = {-INFINITY, -1};
        }
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (uint32_t(c) < a.classes) {
#pragma unroll
                for (int j = 0; j < V; ++j) consider(best[j], last[j], widen(held[c].at(j)), c);
            }
        put_top<V>(a, w, rank, best, q);
    }
}

// Any number of classes, shared by the waves of a workgroup.
constexpr int kRunBlock = 8;                               // classes loaded at once
constexpr int kRunWaves = 8;                               // at most

template <typename T, int V, bool E, bool F>
__global__ void __launch_bounds__(64 * kRunWaves) k_label_run(LabelArgs a) {
    extern __shared__ float shared[];                      // [waves][V][4][64] sums, or [waves][V][2][64] picks
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const uint32_t threads = a.outer * a.groups;
    const uint32_t thread = min(blockIdx.x * 64 + lane, threads - 1);
    const bool mine = blockIdx.x * 64 + lane < threads && wave == 0;   // writes the results
    const Place<V> w = place<V>(a, thread);
    const T *x = static_cast<const T *>(a.x) + w.o * a.xs[0] + w.i * a.xs[2];
    const float *field = F ? a.field + w.o * a.fs[0] + w.i * a.fs[2] : nullptr;
    const uint32_t share = (a.classes + waves - 1) / waves;
    const uint32_t c0 = min(a.classes, wave * share), c1 = min(a.classes, c0 + share);
    Sums r[V];
    Pick best[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        r[j] = kNothing;
        best[j] = {-INFINITY, c0 < c1 ? int32_t(c0) : -1};
    }
    for (uint32_t c = c0; c < c1; c += kRunBlock) {
        Pack<T, V> held[kRunBlock];
#pragma unroll
        for (int u = 0; u < kRunBlock; ++u)
            if (c + u < c1) held[u] = load_pack<V>(x + (c + u) * a.xs[1]);
        float size = 0.0f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float m = r[j].m;
#pragma unroll
            for (int u = 0; u < kRunBlock; ++u)
                if (c + u < c1) m = fmaxf(m, widen(held[u].at(j)));
            lift(r[j], m);
            size = fmaxf(size, fabsf(m));
        }
#pragma unroll
        for (int u = 0; u < kRunBlock; ++u) forget_widened(held[u]);
        by_near<T>(size, [&](auto near) __attribute__((always_inline)) {
            typedef Ref<decltype(near)::value, E, F> R;
            Sums some[V];
#pragma unroll
            for (int j = 0; j < V; ++j) some[j] = kNothing;
#pragma unroll
            for (int u = 0; u < kRunBlock; ++u)
                if (c + u < c1) {
                    Pack<float, V> phi{};
                    if (F) phi = load_field<V>(field + (c + u) * a.fs[1], a.fs[2], V);
#pragma unroll
                    for (int j = 0; j < V; ++j) R(r[j].m).take(some[j], widen(held[u].at(j)), phi.at(j));
                }
#pragma unroll
            for (int j = 0; j < V; ++j) R(r[j].m).close(r[j], some[j]);
        });
        if (a.k) {
#pragma unroll
            for (int u = 0; u < kRunBlock; ++u)
                if (c + u < c1) {
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        if (widen(held[u].at(j)) > best[j].x) best[j] = {widen(held[u].at(j)), int32_t(c + u)};
                }
        }
    }
    if (waves > 1) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float *p = shared + ((wave * V + j) * 4) * 64 + lane;
            p[0] = r[j].m;
            p[64] = r[j].s;
            p[128] = r[j].t;
            p[192] = r[j].f;
        }
        __syncthreads();
        // every wave joins them all, in the same order
#pragma unroll
        for (int j = 0; j < V; ++j) {
            Sums all = kNothing;
            for (uint32_t v = 0; v < waves; ++v) {
                const float *p = shared + ((v * V + j) * 4) * 64 + lane;
                all = join(all, Sums{p[0], p[64], p[128], p[192]});
            }
            r[j] = all;
        }
        __syncthreads();
    }
    Found q[V];
#pragma unroll
    for (int j = 0; j < V; ++j) q[j] = found(r[j]);
    if (mine) {
        int32_t y[V];
        float xl[V];
        if (a.logp) {
            load_labels<V>(a.label, a.label_bytes, w.at, a.classes, y);
#pragma unroll
            for (int j = 0; j < V; ++j)
                xl[j] = y[j] >= 0 ? widen(x[y[j] * a.xs[1] + j * a.xs[2]]) : 0.0f;
        }
        put_found<V>(a, w, y, xl, q);
    }
    Pick last[V];
    for (uint32_t rank = 0; rank < a.k; ++rank) {
        if (rank) {
            // the first was found on the way; each other one is a pass over the classes
#pragma unroll
            for (int j = 0; j < V; ++j) best[j] = {-INFINITY, -1};
            for (uint32_t c = c0; c < c1; ++c) {
                const Pack<T, V> one = load_pack<V>(x + c * a.xs[1]);
#pragma unroll
                for (int j = 0; j < V; ++j) consider(best[j], last[j], widen(one.at(j)), int32_t(c));
            }
        }
        if (waves > 1) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float *p = shared + ((wave * V + j) * 2) * 64 + lane;
                p[0] = best[j].x;
                p[64] = __int_as_float(best[j].c);
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < V; ++j) {
                best[j] = {-INFINITY, -1};
                // shares of classes in rising number: of equal ones the first stays
                for (uint32_t v = 0; v < waves; ++v) {
                    const float *p = shared + ((v * V + j) * 2) * 64 + lane;
                    const int32_t c = __float_as_int(p[64]);
                    if (c >= 0 && (best[j].c < 0 || p[0] > best[j].x)) best[j] = {p[0], c};
                }
            }
            __syncthreads();
        }
        if (mine) put_top<V>(a, w, rank, best, q);
#pragma unroll
        for (int j = 0; j < V; ++j) last[j] = best[j];
    }
}

// ---------------------------------------------------------------------------
// Gradient.
// ---------------------------------------------------------------------------
template <int V>
__device__ __forceinline__ void load_upstream(const LabelGradArgs &a, const Place<V> &w, int32_t (&y)[V],
                                              Slope (&g)[V]) {
    if (a.up_logp) load_labels<V>(a.label, a.label_bytes, w.at, a.classes, y);
    Pack<float, V> ua{}, uh{}, uf{};
    if (a.up_logp) ua = load_pack<V>(a.up_logp + w.at);
    if (a.up_entropy) uh = load_pack<V>(a.up_entropy + w.at);
    if (a.up_mean) uf = load_pack<V>(a.up_mean + w.at);
#pragma unroll
    for (int j = 0; j < V; ++j) {
        if (!a.up_logp) y[j] = -1;
        g[j].a = y[j] < 0 || g[j].logs == INFINITY ? 0.0f : ua.at(j);
        g[j].h = uh.at(j);
        g[j].f = uf.at(j);
    }
}

// Where a thread's gradients begin.
template <typename T, int V>
__device__ __forceinline__ T *slopes(const LabelGradArgs &a, const Place<V> &w) {
    return static_cast<T *>(a.grad) + w.o * a.gs[0] + w.i * a.gs[2];
}
// The positions' slopes, prepared before the classes: each of these is behind a
// branch on their number, where nothing is shared with the one before.
template <typename G, int V>
struct Grads {
    G at[V];
    template <size_t... J>
    __device__ __forceinline__ Grads(const Slope (&g)[V], std::index_sequence<J...>) : at{G(g[J])...} {}
    __device__ __forceinline__ explicit Grads(const Slope (&g)[V]) : Grads(g, std::make_index_sequence<V>()) {}
};

// One class of V positions.
template <typename G, typename T, int V>
__device__ __forceinline__ void put_slope(const LabelGradArgs &a, T *out, const Place<V> &w, uint32_t c,
                                          const Pack<T, V> &x, const Pack<float, V> &phi, const int32_t (&y)[V],
                                          const Slope (&g)[V], const Grads<G, V> &grads) {
    out += c * a.gs[1];
    float v[V];
#pragma unroll
    for (int j = 0; j < V; ++j)
        v[j] = grads.at[j].at(widen(x.at(j)), phi.at(j), y[j] == int32_t(c) ? g[j].a : 0.0f);
    const Pack<T, V> r = narrow_pack<T, V>(v);
    if (V == 1 || a.gs[2] == 1) {
        store_own<V>(out, r, w.skip);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (uint32_t(j) >= w.skip) out[j * a.gs[2]] = r.at(j);
    }
}

// At most C classes: the sums are made anew, which reads nothing but the
// logits that the gradient needs anyway.
template <typename T, int V, int C, bool E, bool F>
__global__ void __launch_bounds__(256) k_label_grad_held(LabelGradArgs a) {
    const uint32_t thread = blockIdx.x * 256 + threadIdx.x;
    if (thread >= a.outer * a.groups) return;
    const Place<V> w = place<V>(a, thread);
    const T *x = static_cast<const T *>(a.x) + w.o * a.xs[0] + w.i * a.xs[2];
    Pack<T, V> held[C];
    const float *const field = F ? a.field + w.o * a.fs[0] + w.i * a.fs[2] : nullptr;
#pragma unroll
    for (int c = 0; c < C; ++c)
        if (uint32_t(c) < a.classes) {
            held[c] = load_pack<V>(x + c * a.xs[1]);
        }
    Sums r[V];
    Slope g[V];
#pragma unroll
    for (int j = 0; j < V; ++j) r[j] = kNothing;
    held_maxima(r, held, a.classes);
    Pack<float, V> phi[kFieldHeld<C, V, F>] = {};
    held_sums<T, V, C, E, F>(r, held, a.classes, field, a.fs, phi);
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const Found q = found(r[j]);
        g[j].m = q.m;
        g[j].logs = stats_logs(q);
        g[j].entropy = q.entropy;
        g[j].mean = q.mean;
    }
    int32_t y[V];
    load_upstream<V>(a, w, y, g);
    T *const out = slopes<T>(a, w);
    by_near<T>(farthest(g), [&](auto near) __attribute__((always_inline)) {
        const Grads<Grad<decltype(near)::value, E, F>, V> grads(g);
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (uint32_t(c) < a.classes) {
                constexpr bool kept = kFieldHeld<C, V, F> == C;
                if constexpr (F && !kept) phi[0] = load_field<V>(field + c * a.fs[1], a.fs[2], V);
                put_slope(a, out, w, c, held[c], phi[F && kept ? c : 0], y, g, grads);
            }
    });
}

// Any number of classes, with the forward call's statistics; blockIdx.y takes
// a share of the classes.
template <typename T, int V, bool E, bool F>
__global__ void __launch_bounds__(256) k_label_grad_run(LabelGradArgs a) {
    const uint32_t thread = blockIdx.x * 256 + threadIdx.x;
    if (thread >= a.outer * a.groups) return;
    const Place<V> w = place<V>(a, thread);
    const T *x = static_cast<const T *>(a.x) + w.o * a.xs[0] + w.i * a.xs[2];
    const uint32_t c0 = blockIdx.y * a.share, c1 = min(a.classes, c0 + a.share);
    Slope g[V];
    const Pack<float, 2 * V> st = load_pack<2 * V>(a.stats + 2 * w.at);
    Pack<float, V> entropy{}, mean{};
    if (E && a.up_entropy) entropy = load_pack<V>(a.entropy + w.at);
    if constexpr (F) mean = load_pack<V>(a.mean + w.at);
#pragma unroll
    for (int j = 0; j < V; ++j) {
        g[j].m = st.at(2 * j);
        g[j].logs = st.at(2 * j + 1);
        g[j].entropy = entropy.at(j);
        g[j].mean = mean.at(j);
    }
    int32_t y[V];
    load_upstream<V>(a, w, y, g);
    T *const out = slopes<T>(a, w);
    by_near<T>(farthest(g), [&](auto near) __attribute__((always_inline)) {
        const Grads<Grad<decltype(near)::value, E, F>, V> grads(g);
        for (uint32_t c = c0; c < c1; c += 4) {
            Pack<T, V> held[4];
            Pack<float, V> phi[F ? 4 : 1] = {};
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (c + u < c1) {
                    held[u] = load_pack<V>(x + (c + u) * a.xs[1]);
                    if constexpr (F)
                        phi[u] = load_field<V>(a.field + w.o * a.fs[0] + (c + u) * a.fs[1] + w.i * a.fs[2], a.fs[2],
                                               V);
                }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (c + u < c1)
                    put_slope(a, out, w, c + u, held[u], phi[F ? u : 0], y, g, grads);
        }
    });
}

}  // namespace tmtrain
