// label.h -- what the kernels of the label log-probabilities share: arguments,
// the arithmetic of a running softmax, keys of the likeliest classes
// (include/tm_train.h).  label_maps.h has the kernels of class axes that lie
// apart, label_rows.h those of contiguous rows.
//
// With m the largest logit, d_c = x_c - m, e_c = exp d_c and s = sum e_c:
//     l_c = d_c - log s,   entropy = log s - (sum e_c d_c) / s,
//     mean = (sum e_c field_c) / s.
// d and log s are kept apart: their difference loses nothing of a large m.
// m runs: where it grows, the sums so far shrink by exp(old - new).  It starts
// at the lowest finite float instead of -inf, so that d is never inf - inf:
// classes at -inf get e = 0, and s = 0 marks a position with no class left.
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
    int64_t ts[3];              // strides of top and index: outer, rank, inner
    uint32_t outer, classes, inner, k;
    int32_t label_bytes;        // 1 (unsigned), 4 or 8
    uint32_t n;                 // outer * inner
    uint32_t groups;            // maps: threads along the inner positions; rows: workgroups of a row
    Div32 div_groups;
    Div32 div_inner;
    void *partial;              // rows: what the workgroups of a row found
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
    uint32_t groups;
    uint32_t share;             // classes of a workgroup
    Div32 div_groups;
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

// V elements `stride` apart, the first n of them.
template <int V>
__device__ __forceinline__ Pack<float, V> load_field(const float *p, int64_t stride, uint32_t n) {
    if (V == 1 || stride == 1) return load_pack<V>(p, n, 0.0f);
    Pack<float, V> r{};
#pragma unroll
    for (int j = 0; j < V; ++j) r.put(j, uint32_t(j) < n ? p[j * stride] : 0.0f);
    return r;
}

struct Sums {
    float m, s, t, f;           // maximum, sum e, sum e d, sum e field
};
constexpr Sums kNothing = {-FLT_MAX, 0.0f, 0.0f, 0.0f};

// d = x - m, not below -200: exp -200 is 0 in float32, and the products with d
// stay finite.  A NaN stays one.
__device__ __forceinline__ float below(float x, float m) {
    const float d = x - m;
    return d < -200.0f ? -200.0f : d;
}

// exp d for the sums of type T.  The rounding of d log2(e) is an error of up to
// 2^-24 |d|; float32 logits take it back to first order, 16-bit ones are
// rounded to 2^-9 themselves.
template <typename T>
__device__ __forceinline__ float exp_of(float d) {
    const float z = d * kLog2e;
    const float e = exp2_hw(z);
    if constexpr (sizeof(T) == 4) return fmaf(e, fmaf(d, kLog2e, -z) * kLn2, e);
    return e;
}

// The sums seen from a larger maximum.
__device__ __forceinline__ void lift(Sums &r, float m) {
    const float d = below(r.m, m);
    const float e = exp_of<float>(d);
    r.t = e * fmaf(d, r.s, r.t);
    r.s *= e;
    r.f *= e;
    r.m = m;
}
__device__ __forceinline__ Sums join(Sums a, Sums b) {
    const float m = fmaxf(a.m, b.m);
    lift(a, m);
    lift(b, m);
    return {m, a.s + b.s, a.t + b.t, a.f + b.f};
}

// One class more; field is read only if it is there.
template <typename T>
__device__ __forceinline__ void take(Sums &r, float x, bool entropy) {
    const float d = below(x, r.m);
    const float e = exp_of<T>(d);
    r.s += e;
    if (entropy) r.t = fmaf(e, d, r.t);
}
template <typename T>
__device__ __forceinline__ void take(Sums &r, float x, bool entropy, float field) {
    const float d = below(x, r.m);
    const float e = exp_of<T>(d);
    r.s += e;
    if (entropy) r.t = fmaf(e, d, r.t);
    r.f = fmaf(e, e == 0.0f ? 0.0f : field, r.f);
}

// What a position's sums say.
struct Found {
    float m, logs, entropy, mean;
    bool dead;                  // every class at -inf
};
__device__ __forceinline__ Found found(const Sums &r) {
    Found q;
    q.dead = r.s == 0.0f;
    q.m = r.m;
    q.logs = logf(r.s);
    q.entropy = q.dead ? 0.0f : q.logs - r.t / r.s;
    q.mean = q.dead ? 0.0f : r.f / r.s;
    return q;
}
__device__ __forceinline__ float log_prob(const Found &q, float x) {
    return q.dead ? -INFINITY : (x - q.m) - q.logs;
}
// As tm_label_logp_grad reads it: probabilities of a dead position become 0.
__device__ __forceinline__ float stats_logs(const Found &q) { return q.dead ? INFINITY : q.logs; }

// The gradient of one class: p (f (field - mean) - a - h (l + entropy)) and a more for the label's.
struct Slope {
    float m, logs, a, h, f, entropy, mean;
};
template <typename T, bool F>
__device__ __forceinline__ float slope_of(const Slope &g, bool entropy, float x, float field) {
    // x - m - log s; a dead position has log s = inf and so p = 0
    const float l = below(x - g.m, g.logs);
    const float p = exp_of<T>(l);
    float v = -g.a;
    if (entropy) v -= g.h * (l + g.entropy);
    if constexpr (F) v += g.f * (field - g.mean);
    return p == 0.0f ? 0.0f : p * v;
}

}  // namespace tmtrain
