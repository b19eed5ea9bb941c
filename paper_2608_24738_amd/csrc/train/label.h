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
    uint32_t lanes;             // rows: 16, 64 or 256 threads to a part
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

// exp d.  The rounding of d log2(e), an error of up to 2^-24 |d|, is taken
// back to first order.
__device__ __forceinline__ float exp_of(float d) {
    const float z = d * kLog2e;
    const float e = exp2_hw(z);
    return fmaf(e, fmaf(d, kLog2e, -z) * kLn2, e);
}

// The sums seen from a larger maximum.
__device__ __forceinline__ void lift(Sums &r, float m) {
    const float d = below(r.m, m);
    const float e = exp_of(d);
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

// Classes against a reference m.
//
// Near (16-bit logits, |m| <= kNear): z = x log2(e) - m log2(e) is one fused
// operation, off by 2^-24 |z|, which the logits' own rounding of 2^-9 hides.
// The rounding of m log2(e) is a common factor of every e and is taken out
// again at the end.  Otherwise (float32 logits, or products in which that
// factor would not be small, masks of the type's lowest value among them): d = x - m,
// with the rounding of d log2(e) taken back to first order.
constexpr float kNear = 1000.0f;                           // factor - 1 < 6e-5, its square below a rounding

template <bool Near, bool Entropy, bool Mean>
struct Ref {
    float m, mz;

    __device__ __forceinline__ explicit Ref(float m) : m(m), mz(m * kLog2e) {}

    __device__ __forceinline__ void take(Sums &r, float x, float field) const {
        float e;
        if constexpr (Near) {
            const float z = fmaf(x, kLog2e, -mz);
            e = exp2_hw(z);
            if constexpr (Entropy) r.t = fmaf(e, fmaxf(z, -300.0f), r.t);    // 0 times a finite number; NaN comes from e
        } else {
            const float d = below(x, m);
            e = exp_of(d);
            if constexpr (Entropy) r.t = fmaf(e, d, r.t);
        }
        r.s += e;
        if constexpr (Mean) r.f = fmaf(e, e == 0.0f ? 0.0f : field, r.f);
    }
    // r += the sums of the classes taken into `some`
    __device__ __forceinline__ void close(Sums &r, const Sums &some) const {
        if constexpr (Near) {
            const float off = fmaf(m, kLog2e, -mz) * kLn2;
            const float scale = 1.0f - off;
            r.s = fmaf(some.s, scale, r.s);
            if constexpr (Entropy) r.t = fmaf(fmaf(some.t, kLn2, -off * some.s), scale, r.t);   // z to d
            if constexpr (Mean) r.f = fmaf(some.f, scale, r.f);
        } else {
            r.s += some.s;
            if constexpr (Entropy) r.t += some.t;
            if constexpr (Mean) r.f += some.f;
        }
    }
};

template <bool B>
struct Bool { static constexpr bool value = B; };
// f(Bool<near>): whether references up to `size` from 0 are near for logits of
// type T.  Told apart here and not class by class.
template <typename T, typename F>
__device__ __forceinline__ void by_near(float size, F f) {
    if constexpr (sizeof(T) == 2) {
        if (size <= kNear) f(Bool<true>{});
        else f(Bool<false>{});
    } else {
        f(Bool<false>{});
    }
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
    q.logs = __builtin_amdgcn_logf(r.s) * kLn2;            // s is 0 or between 1/2 and 2^45: no subnormals
    const float one = __builtin_amdgcn_rcpf(r.s);          // within 1 ulp
    q.entropy = q.dead ? 0.0f : fmaf(-r.t, one, q.logs);
    q.mean = q.dead ? 0.0f : r.f * one;
    return q;
}
__device__ __forceinline__ float log_prob(const Found &q, float x) {
    return q.dead ? -INFINITY : (x - q.m) - q.logs;
}
// As tm_label_logp_grad reads it: probabilities of a dead position become 0.
__device__ __forceinline__ float stats_logs(const Found &q) { return q.dead ? INFINITY : q.logs; }

// The gradient of one class: p (f (field - mean) - a - h (l + entropy)) and a
// more for the label's, a being 0 where there is no label.
struct Slope {
    float m, logs, a, h, f, entropy, mean;
};

// A position's slope, prepared: the factor of p is base + per l (+ f field).
// p is the square of q = 2^z with z = (x - m - log s) log2(e) / 2, and its
// factor stands between the two: v_exp_f32 gives 0 below 2^-126, which for q
// is p = 2^-252, so that gradients among float32's smallest numbers come out
// whether p or the upstream gradient is small.  (A z made larger by a constant
// instead would be rounded as coarsely as the constant is large.)  Near as in
// Ref: c = (m + log s) log2(e) / 2 is rounded twice, which is a factor common to
// every p and a term common to every l.  Where p is close to 1 or l to minus
// the entropy, the gradient is what is left of a difference and shows them, so
// both are taken out, once for all classes; what stays is of second order,
// below 4e-9.
constexpr float kHalfLog2e = 0.5f * kLog2e;
constexpr float kGone = 1.0f / 604462909807314587353088.0f;   // q of p = 2^-158: the field is not looked at

template <bool Near, bool Entropy, bool Mean>
struct Grad {
    float base, per, f;         // per: of l, or of z
    float m, logs, c;

    __device__ __forceinline__ explicit Grad(const Slope &g)
        : base(-g.a), per(-g.h), f(g.f), m(g.m), logs(g.logs), c((g.m + g.logs) * kHalfLog2e) {
        if constexpr (Entropy) base = fmaf(per, g.entropy, base);
        if constexpr (Mean) base = fmaf(-f, g.mean, base);
        if constexpr (Near) {
            // m + log s - sum, exactly, and (m + log s) log2(e) / 2 - c
            const float sum = m + logs, part = sum - m;
            const float rest = (m - (sum - part)) + (logs - part);
            const float off = fmaf(rest, kHalfLog2e, fmaf(sum, kHalfLog2e, -c));
            const float scale = 1.0f - 2.0f * kLn2 * off;
            per *= 2.0f * kLn2;
            if constexpr (Entropy) base = fmaf(per, -off, base);
            base *= scale;
            if constexpr (Entropy) per *= scale;
            if constexpr (Mean) f *= scale;
        }
    }
    // extra: a for the label's class, else 0
    __device__ __forceinline__ float at(float x, float field, float extra) const {
        float q, l;
        if constexpr (Near) {
            l = fmaf(x, kHalfLog2e, -c);                   // z
            q = exp2_hw(l);
            l = fmaxf(l, -150.0f);                         // 0 times a finite number; NaN comes from q
        } else {
            l = below(x - m, logs);                        // a dead position has log s = inf and so q = 0
            const float z = l * kHalfLog2e;
            q = exp2_hw(z);
            q = fmaf(q, fmaf(l, kHalfLog2e, -z) * kLn2, q);      // as exp_of
        }
        float v = base;
        if constexpr (Entropy) v = fmaf(per, l, v);
        if constexpr (Mean) v = fmaf(f, q < kGone ? 0.0f : field, v);
        return fmaf(q * v, q, extra);
    }
};

// The largest distance from 0 among the positions' references; a dead one is far.
template <int V>
__device__ __forceinline__ float farthest(const Slope (&g)[V]) {
    float size = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j) size = fmaxf(size, fmaxf(fabsf(g[j].m), fabsf(g[j].logs)));
    return size;
}

}  // namespace tmtrain
