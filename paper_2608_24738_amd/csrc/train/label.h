// label.h -- log-probabilities of given labels, with the entropy, the expected
// field and the likeliest classes, and their gradient (include/tm_train.h).
//
// With m the largest logit, d_c = x_c - m, e_c = exp d_c and s = sum e_c:
//     l_c = d_c - log s,   entropy = log s - (sum e_c d_c) / s,
//     mean = (sum e_c field_c) / s.
// d and log s are kept apart: their difference loses nothing of a large m.
// m starts at the lowest finite float instead of -inf, so that d is never
// inf - inf: classes at -inf get e = 0, and s = 0 marks a position with no
// class left.
#pragma once

#include "train_common.h"

namespace tmtrain {

struct LabelArgs {
    const void *x;              // logits
    const void *label;
    const float *field;
    float *logp, *entropy, *mean, *top, *stats;
    int32_t *index;
    int64_t xs[3], fs[3];       // strides of logits and field: outer, class, inner
    uint32_t outer, classes, inner, k;
    int32_t label_bytes;        // 1 (unsigned), 4 or 8
    uint32_t n;                 // outer * inner
    Div32 div_inner;
};

struct LabelGradArgs {
    const void *x;
    const void *label;
    const float *field;
    const float *stats, *entropy, *mean;
    const float *up_logp, *up_entropy, *up_mean;
    void *grad;
    int64_t xs[3], fs[3], gs[3];
    uint32_t outer, classes, inner;
    int32_t label_bytes;
    uint32_t n;
    Div32 div_inner;
};

// The label of position i, or -1 where it lies outside [0, classes).
__device__ __forceinline__ int32_t load_label(const void *p, int32_t bytes, uint64_t i, uint32_t classes) {
    int64_t y;
    if (bytes == 1)
        y = static_cast<const uint8_t *>(p)[i];
    else if (bytes == 4)
        y = static_cast<const int32_t *>(p)[i];
    else
        y = static_cast<const int64_t *>(p)[i];
    return y >= 0 && y < int64_t(classes) ? int32_t(y) : -1;
}

// Logits in an order that whole numbers have: larger logits larger, -0 = +0,
// NaN below -inf, never 0.
__device__ __forceinline__ uint32_t ordered(float x) {
    if (x != x) return 1;
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t o) {
    if (o == 1) return __uint_as_float(0x7fc00000u);
    return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
// Larger logits first, equal ones by rising class; 0 is below every class.
__device__ __forceinline__ uint64_t top_key(float x, uint32_t c) { return uint64_t(ordered(x)) << 32 | ~c; }

struct Sums {
    float m, s, t, f;           // maximum, sum e, sum e d, sum e field
};

template <typename T>
__device__ Sums position_sums(const T *x, int64_t xs, const float *field, int64_t fs, uint32_t classes) {
    Sums r{-FLT_MAX, 0.0f, 0.0f, 0.0f};
    for (uint32_t c = 0; c < classes; ++c) r.m = fmaxf(r.m, widen(x[c * xs]));
    // sums of 256 classes at a time: the error of one long chain would grow with
    // the number of classes
    for (uint32_t first = 0; first < classes; first += 256) {
        float s = 0.0f, t = 0.0f, f = 0.0f;
        for (uint32_t c = first; c < min(classes, first + 256); ++c) {
            const float d = widen(x[c * xs]) - r.m;
            const float e = exp2_hw(d * kLog2e);
            s += e;
            t += e == 0.0f ? 0.0f : e * d;
            if (field) f += e == 0.0f ? 0.0f : e * field[c * fs];
        }
        r.s += s;
        r.t += t;
        r.f += f;
    }
    return r;
}

template <typename T>
__global__ void __launch_bounds__(256) k_label_logp(LabelArgs a) {
    const uint32_t n = blockIdx.x * 256 + threadIdx.x;
    if (n >= a.n) return;
    const uint32_t o = a.div_inner.div(n), i = n - o * a.inner;
    const T *x = static_cast<const T *>(a.x) + o * a.xs[0] + i * a.xs[2];
    const float *field = a.field ? a.field + o * a.fs[0] + i * a.fs[2] : nullptr;
    const Sums r = position_sums(x, a.xs[1], field, a.fs[1], a.classes);
    const bool dead = r.s == 0.0f;
    const float logs = logf(r.s);
    if (a.logp) {
        const int32_t y = load_label(a.label, a.label_bytes, n, a.classes);
        a.logp[n] = y < 0 ? 0.0f : dead ? -INFINITY : widen(x[y * a.xs[1]]) - r.m - logs;
    }
    if (a.entropy) a.entropy[n] = dead ? 0.0f : logs - r.t / r.s;
    if (a.mean) a.mean[n] = dead ? 0.0f : r.f / r.s;
    if (a.stats) {
        a.stats[2 * uint64_t(n)] = r.m;
        a.stats[2 * uint64_t(n) + 1] = dead ? INFINITY : logs;
    }
    uint64_t floor = ~uint64_t(0);
    for (uint32_t j = 0; j < a.k; ++j) {
        uint64_t best = 0;
        for (uint32_t c = 0; c < a.classes; ++c) {
            const uint64_t key = top_key(widen(x[c * a.xs[1]]), c);
            if (key < floor && key > best) best = key;
        }
        const uint64_t at = (uint64_t(o) * a.k + j) * a.inner + i;
        a.index[at] = int32_t(~uint32_t(best));
        a.top[at] = dead ? -INFINITY : unordered(best >> 32) - r.m - logs;
        floor = best;
    }
}

template <typename T>
__global__ void __launch_bounds__(256) k_label_logp_grad(LabelGradArgs a) {
    const uint32_t n = blockIdx.x * 256 + threadIdx.x;
    if (n >= a.n) return;
    const uint32_t o = a.div_inner.div(n), i = n - o * a.inner;
    const T *x = static_cast<const T *>(a.x) + o * a.xs[0] + i * a.xs[2];
    const float *field = a.field ? a.field + o * a.fs[0] + i * a.fs[2] : nullptr;
    T *g = static_cast<T *>(a.grad) + o * a.gs[0] + i * a.gs[2];
    float m, logs, entropy, mean;
    if (a.stats) {
        m = a.stats[2 * uint64_t(n)];
        logs = a.stats[2 * uint64_t(n) + 1];
        entropy = a.up_entropy ? a.entropy[n] : 0.0f;
        mean = a.up_mean ? a.mean[n] : 0.0f;
    } else {
        const Sums r = position_sums(x, a.xs[1], field, a.fs[1], a.classes);
        m = r.m;
        logs = r.s == 0.0f ? INFINITY : logf(r.s);
        entropy = logs - r.t / r.s;
        mean = r.f / r.s;
    }
    const bool dead = logs == INFINITY;
    const int32_t y = a.up_logp ? load_label(a.label, a.label_bytes, n, a.classes) : -1;
    const float ua = y < 0 || dead ? 0.0f : a.up_logp[n];
    const float uh = a.up_entropy ? a.up_entropy[n] : 0.0f;
    const float uf = a.up_mean ? a.up_mean[n] : 0.0f;
    for (uint32_t c = 0; c < a.classes; ++c) {
        const float l = widen(x[c * a.xs[1]]) - m - logs;
        const float p = exp2_hw(l * kLog2e);
        float slope = -ua;
        if (a.up_entropy) slope -= uh * (l + entropy);
        if (a.up_mean) slope += uf * (field[c * a.fs[1]] - mean);
        float v = p == 0.0f ? 0.0f : p * slope;
        if (int32_t(c) == y) v += ua;
        g[c * a.gs[1]] = narrow<T>(v);
    }
}

}  // namespace tmtrain
