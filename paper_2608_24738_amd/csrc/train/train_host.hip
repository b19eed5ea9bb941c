// train_host.hip -- C-ABI of the training operators: argument checks, choice
// of kernel and launches (declared in include/tm_train.h).

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../../include/tm_train.h"
#include "bias.h"
#include "label_maps.h"
#include "label_rows.h"

using namespace tmtrain;

namespace {

constexpr uint64_t kLimit = uint64_t(1) << 31;

bool float_type(int dtype) { return dtype == TM_DTYPE_F32 || dtype == TM_DTYPE_F16 || dtype == TM_DTYPE_BF16; }
uint64_t float_bytes(int dtype) { return dtype == TM_DTYPE_F32 ? 4 : 2; }

constexpr uint64_t kFill = 1024;            // workgroups that keep the chip busy

uint32_t pow2_from(uint32_t n) {
    uint32_t p = 1;
    while (p < n) p <<= 1;
    return p;
}
uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

struct Range {
    const void *at;
    uint64_t bytes;
};
bool meet(const Range &a, const Range &b) {
    if (!a.at || !b.at || !a.bytes || !b.bytes) return false;
    const uintptr_t x = uintptr_t(a.at), y = uintptr_t(b.at);
    return x < y + b.bytes && y < x + a.bytes;
}
// No output may overlap an input or another output.
template <int NI, int NO>
bool aliased(const Range (&in)[NI], const Range (&out)[NO]) {
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

// fn(entropy, field) of the parts asked for; a field brings the entropy along.
template <typename F>
int by_parts(const void *entropy, const void *field, F fn) {
    if (field) return fn(Bool<true>{}, Bool<true>{});
    if (entropy) return fn(Bool<true>{}, Bool<false>{});
    return fn(Bool<false>{}, Bool<false>{});
}
template <int N>
struct Int { static constexpr int value = N; };
template <typename F>
int by_waves(uint32_t waves, F fn) {
    if (waves == 1) return fn(Int<1>{});
    if (waves == 2) return fn(Int<2>{});
    if (waves == 4) return fn(Int<4>{});
    if (waves == 8) return fn(Int<8>{});
    return fn(Int<16>{});
}
template <typename F>
int by_held(int held, F fn) {
    if (held == 4) return fn(Int<4>{});
    if (held == 8) return fn(Int<8>{});
    if (held == 16) return fn(Int<16>{});
    if (held == 24) return fn(Int<24>{});
    return fn(Int<32>{});
}

// ---------------------------------------------------------------------------
// Labels.
// ---------------------------------------------------------------------------

// Elements from a view's first to the end of its last, or 0 if a stride is
// negative or the view is too long to address.
uint64_t view_span(const uint64_t (&n)[3], const int64_t *strides) {
    uint64_t span = 1;
    for (int a = 0; a < 3; ++a) {
        if (strides[a] < 0) return 0;
        if (n[a] > 1 && uint64_t(strides[a]) > (uint64_t(1) << 58) / n[a]) return 0;
        span += (n[a] - 1) * uint64_t(strides[a]);
    }
    return span;
}

// Whether two elements of a view share an address.
bool self_overlap(const uint64_t (&n)[3], const int64_t *strides) {
    int order[3] = {0, 1, 2};
    for (int a = 1; a < 3; ++a)
        for (int b = a; b > 0 && strides[order[b]] < strides[order[b - 1]]; --b) {
            const int t = order[b];
            order[b] = order[b - 1];
            order[b - 1] = t;
        }
    uint64_t reach = 0;         // from the first to the last element of the axes so far
    for (int a : order) {
        if (n[a] < 2) continue;
        if (uint64_t(strides[a]) <= reach) return true;
        reach += (n[a] - 1) * uint64_t(strides[a]);
    }
    return false;
}

struct LabelShape {
    uint64_t n[3];              // outer, classes, inner
    uint64_t positions;
    uint64_t x_bytes, field_bytes, label_bytes;
};

int check_labels(const void *logits, int dtype, int64_t outer, int64_t classes, int64_t inner, const int64_t *strides,
                 const void *labels, int label_dtype, const float *field, const int64_t *field_strides,
                 LabelShape &s) {
    if (outer < 0 || inner < 0 || classes < 1 || !strides || (field && !field_strides)) return TM_ERR_SHAPE;
    for (int a = 0; a < 3; ++a)
        if (strides[a] < 0 || (field && field_strides[a] < 0)) return TM_ERR_SHAPE;
    if (!float_type(dtype)) return TM_ERR_DTYPE;
    if (labels && label_dtype != TM_DTYPE_U8 && label_dtype != TM_DTYPE_I32 && label_dtype != TM_DTYPE_I64)
        return TM_ERR_DTYPE;
    if (uint64_t(classes) >= kLimit || uint64_t(outer) >= kLimit || uint64_t(inner) >= kLimit ||
        uint64_t(outer) * uint64_t(inner) >= kLimit)
        return TM_ERR_TOO_LARGE;
    s.n[0] = uint64_t(outer);
    s.n[1] = uint64_t(classes);
    s.n[2] = uint64_t(inner);
    s.positions = s.n[0] * s.n[2];
    if (s.positions == 0) return TM_OK;
    if (!logits) return TM_ERR_NULL;
    const uint64_t span = view_span(s.n, strides), fspan = field ? view_span(s.n, field_strides) : 1;
    if (!span || !fspan) return TM_ERR_TOO_LARGE;
    s.x_bytes = span * float_bytes(dtype);
    s.field_bytes = field ? fspan * 4 : 0;
    s.label_bytes = label_dtype == TM_DTYPE_U8 ? 1 : label_dtype == TM_DTYPE_I32 ? 4 : 8;
    return TM_OK;
}

constexpr uint64_t kBusyThreads = 65536;     // four waves to a CU
constexpr uint64_t kRowBusyWaves = 4096;     // four waves to a SIMD

// How a request runs: on contiguous rows or on maps, with how many classes
// held, positions to a thread and waves to a row or position.
struct LabelPlan {
    bool rows;
    bool swap;                  // maps: the outer positions lie side by side, not the inner ones
    int wide;                   // maps: positions to a thread
    int held;                   // maps: classes held in registers, 0: they run through
    uint32_t waves;             // of a row, or sharing the classes of a map's positions
    uint32_t parts;             // of a row
    bool brief;                 // 16 lanes to a row
};

// Times below are of bf16 forward calls with the entropy, in us.
LabelPlan label_plan(int dtype, uint64_t outer, uint64_t classes, uint64_t inner, const int64_t *strides) {
    LabelPlan p{};
    const uint64_t n = outer * inner, vec = 16 / float_bytes(dtype);
    p.parts = 1;
    // Contiguous classes: lanes to a row (65536 x 64: 6 by 16 lanes, 10 by
    // threads, gradients 8 and 26; x 33: 6 and 6, 8 and 14). Up to 32 classes a
    // thread holds the row, and its gradient needs no statistics.
    if (strides[1] == 1 && classes > TM_LABEL_MAX_RECOMPUTE) {
        p.rows = true;
        // As many waves as fill the chip, each lane with at least one round of
        // loads (512 x 50021 with 5 alternatives: 8 waves 21, 16 waves 22;
        // 1024 x 32768: 1 to 4 waves 14.6, twice as many 15.9).
        const uint64_t most = ceil_div(classes, 64 * vec * kRowLoads), want = ceil_div(kRowBusyWaves, n);
        const uint64_t waves = std::min(most, want);
        // Many short rows: 16 lanes to a row (65536 x 100: 6, a wave to a row 25; x 512: 14 and 27).
        p.brief = n >= 4096 && classes <= 16 * vec * kRowLoads;
        p.waves = waves <= 1 ? 1 : waves <= 2 ? 2 : waves <= 4 ? 4 : waves <= 8 ? 8 : 16;
        // Few long rows: parts of one load to a lane of four waves, for a
        // second launch (1 x 131072: 4.8, without parts 11; 1 x 20000: 4.9, 4.5).
        if (want > 16 && classes > 32768) {
            p.waves = 4;
            p.parts = uint32_t(std::min<uint64_t>({kRowMostParts, ceil_div(classes, 64 * 4 * vec), ceil_div(want, 4)}));
        }
        return p;
    }
    p.swap = inner == 1 && outer > 1 && strides[0] == 1;
    const uint64_t in = p.swap ? outer : inner, out = p.swap ? 1 : outer;
    const int64_t step = p.swap ? strides[0] : strides[2];
    // Registers for as many classes as there are, which is waves to a SIMD (16 x 21 x 375 x 500, 24 or 32: forward
    // 38.8 and 39.7, gradient with the entropy 59 and 61.5; x 24: 42.4 and 43.5, 67 and 71).
    p.held = classes <= 4 ? 4 : classes <= 8 ? 8 : classes <= 16 ? 16 : classes <= 24 ? 24 : classes <= 32 ? 32 : 0;
    // Several positions to a thread where enough threads are left (4 x 4 x 512^2:
    // 6.0, one to a thread 6.5; 4 x 4 x 256^2, which leaves 32768: 4.3, 3.5).
    p.wide = p.held == 0 ? kRunV : int((p.held <= 8 ? 16 : 8) / float_bytes(dtype));
    if (step != 1 || in < uint64_t(p.wide) || out * ceil_div(in, p.wide) < kBusyThreads / (p.held ? 1 : 2)) p.wide = 1;
    // Waves that share many classes (8 x 150 x 128^2: 1, 2, 4, 8 waves 32, 25,
    // 17, 20; 16 x 64 x 100^2: 16, 13, 12, 17; 150 x 32^2: 14, 9, 6, 5).
    const uint64_t threads = out * ceil_div(in, p.wide);
    p.waves = uint32_t(std::max<uint64_t>(1, std::min<uint64_t>({kRunWaves, 3 * kBusyThreads / threads, classes / 16})));
    return p;
}

// At least `blocks` < 2^31 workgroups, of up to 1024 threads.
dim3 row_grid(uint32_t blocks) {
    const uint32_t x = std::min<uint32_t>(blocks, 1u << 21);
    return dim3(x, uint32_t(ceil_div(blocks, x)));
}

template <typename Args>
void swap_positions(Args &a) {
    a.inner = a.outer;
    a.outer = 1;
    std::swap(a.xs[0], a.xs[2]);
    std::swap(a.fs[0], a.fs[2]);
}

}  // namespace

extern "C" size_t tm_label_logp_workspace_size(int dtype, int64_t outer, int64_t classes, int64_t inner,
                                               const int64_t *strides, int top_k) {
    LabelShape s{};
    const void *some = reinterpret_cast<const void *>(uintptr_t(4096));
    if (check_labels(some, dtype, outer, classes, inner, strides, nullptr, 0, nullptr, nullptr, s) != TM_OK) return 0;
    if (s.positions == 0 || top_k < 0 || top_k > TM_LABEL_MAX_TOP) return 0;
    const LabelPlan p = label_plan(dtype, s.n[0], s.n[1], s.n[2], strides);
    return p.parts > 1 ? s.positions * p.parts * (sizeof(RowPart) + 8 * size_t(top_k)) : 0;
}

extern "C" int tm_label_logp(const void *logits, int dtype, int64_t outer, int64_t classes, int64_t inner,
                             const int64_t *strides, const void *labels, int label_dtype, const float *field,
                             const int64_t *field_strides, int top_k, float *out_logp, float *out_entropy,
                             float *out_mean, float *out_top, int32_t *out_index, float *out_stats, void *workspace,
                             size_t workspace_bytes, hipStream_t stream) {
    LabelShape s{};
    const int rc = check_labels(logits, dtype, outer, classes, inner, strides, labels, label_dtype, field,
                                field_strides, s);
    if (rc != TM_OK) return rc;
    if (top_k < 0 || top_k > TM_LABEL_MAX_TOP || top_k > classes) return TM_ERR_UNSUPPORTED;
    if (s.positions == 0) return TM_OK;
    if ((out_logp && !labels) || (out_mean && !field)) return TM_ERR_NULL;
    if (!out_logp && !out_entropy && !out_mean && !out_stats && !top_k) return TM_ERR_NO_OUTPUT;
    if (top_k > 0 && (!out_top || !out_index)) return TM_ERR_NO_OUTPUT;
    const size_t need = tm_label_logp_workspace_size(dtype, outer, classes, inner, strides, top_k);
    if (need && (!workspace || workspace_bytes < need || uintptr_t(workspace) % 8)) return TM_ERR_WORKSPACE;
    const uint64_t n4 = s.positions * 4;
    const Range in[] = {{logits, s.x_bytes}, {labels, s.positions * s.label_bytes}, {field, s.field_bytes}};
    const Range out[] = {{out_logp, n4}, {out_entropy, n4}, {out_mean, n4}, {out_stats, 2 * n4},
                         {top_k ? out_top : nullptr, n4 * uint64_t(top_k)},
                         {top_k ? out_index : nullptr, n4 * uint64_t(top_k)}, {need ? workspace : nullptr, need}};
    if (aliased(in, out)) return TM_ERR_ALIAS;
    LabelArgs a{};
    a.x = logits;
    a.label = labels;
    a.field = out_mean ? field : nullptr;
    a.logp = out_logp;
    a.entropy = out_entropy;
    a.mean = out_mean;
    a.top = out_top;
    a.index = out_index;
    a.stats = out_stats;
    for (int i = 0; i < 3; ++i) {
        a.xs[i] = strides[i];
        a.fs[i] = a.field ? field_strides[i] : 0;
    }
    a.outer = uint32_t(outer);
    a.classes = uint32_t(classes);
    a.inner = uint32_t(inner);
    a.k = uint32_t(top_k);
    a.label_bytes = int32_t(s.label_bytes);
    a.n = uint32_t(s.positions);
    LabelPlan p = label_plan(dtype, s.n[0], s.n[1], s.n[2], strides);
    // Many alternatives of rows of two loads a lane and more: a wave to a row, whose lanes' bests cost less than a pass
    // each (65536 x 500, 8 and 32 of them: 104 and 272 us, by 16 lanes 149 and 676; 5, about where the two meet: 86 and
    // 92; x 100 with 5, 8, 32: 81, 103, 265 and 30, 48, 197).
    if (top_k >= 8 && s.n[1] >= 32 * (16 / float_bytes(dtype))) p.brief = false;
    a.ts[0] = top_k * inner;
    a.ts[1] = inner;
    a.ts[2] = 1;
    if (p.swap) {
        swap_positions(a);
        std::swap(a.ts[0], a.ts[2]);
    }
    a.div_inner = Div32::make(a.inner);
    a.partial = workspace;
    return by_type(dtype, [&](auto t) {
        using T = decltype(t);
        if (p.rows) {
            a.groups = p.parts;
            a.div_groups = Div32::make(p.parts);
            if (s.positions * p.parts >= kLimit) return int(TM_ERR_TOO_LARGE);
            if (p.brief) {
                return by_parts(a.entropy, a.field, [&](auto e, auto f) {
                    constexpr bool E = decltype(e)::value, F = decltype(f)::value;
                    constexpr uint32_t load = 16 * 16 / sizeof(T);
                    return launch(a.classes <= load ? a.k ? k_label_rows_short<T, 1, E, F, true>
                                                          : k_label_rows_short<T, 1, E, F, false>
                                                    : a.k ? k_label_rows_short<T, kRowLoads, E, F, true>
                                                          : k_label_rows_short<T, kRowLoads, E, F, false>,
                                  row_grid(uint32_t(ceil_div(a.n, kShortRows))), dim3(16 * kShortRows), 0, stream, a);
                });
            }
            const int rc = by_waves(p.waves, [&](auto waves) {
                return by_parts(a.entropy, a.field, [&](auto e, auto f) {
                    constexpr int W = decltype(waves)::value;
                    constexpr bool E = decltype(e)::value, F = decltype(f)::value;
                    return launch(a.k ? k_label_rows<T, W, E, F, true> : k_label_rows<T, W, E, F, false>,
                                  row_grid(W == 1 ? (a.n + 3) / 4 : a.n * p.parts), dim3(W == 1 ? 256 : 64 * W), 0,
                                  stream, a);
                });
            });
            if (rc != TM_OK || p.parts == 1) return rc;
            return launch(k_label_rows_join<T>, dim3(a.n), dim3(64), 0, stream, a);
        }
        a.groups = uint32_t(ceil_div(a.inner, p.wide));
        a.div_groups = Div32::make(a.groups);
        const uint32_t threads = a.outer * a.groups;
        if (p.held) {
            return by_held(p.held, [&](auto held) {
                return by_parts(a.entropy, a.field, [&](auto e, auto f) {
                    constexpr int C = decltype(held)::value;
                    constexpr bool E = decltype(e)::value, F = decltype(f)::value;
                    return launch(p.wide > 1 ? k_label_held<T, kHeldV<T, C>, C, E, F> : k_label_held<T, 1, C, E, F>,
                                  dim3((threads + 255) / 256), dim3(256), 0, stream, a);
                });
            });
        }
        const size_t lds = p.waves > 1 ? size_t(p.waves) * p.wide * 1024 : 0;
        return by_parts(a.entropy, a.field, [&](auto e, auto f) {
            constexpr bool E = decltype(e)::value, F = decltype(f)::value;
            return launch(p.wide > 1 ? k_label_run<T, kRunV, E, F> : k_label_run<T, 1, E, F>, dim3((threads + 63) / 64),
                          dim3(64 * p.waves), lds, stream, a);
        });
    });
}

extern "C" int tm_label_logp_grad(const void *logits, int dtype, int64_t outer, int64_t classes, int64_t inner,
                                  const int64_t *strides, const void *labels, int label_dtype, const float *field,
                                  const int64_t *field_strides, const float *stats, const float *entropy,
                                  const float *mean, const float *up_logp, const float *up_entropy,
                                  const float *up_mean, void *out_grad, const int64_t *grad_strides,
                                  hipStream_t stream) {
    LabelShape s{};
    const int rc = check_labels(logits, dtype, outer, classes, inner, strides, labels, label_dtype, field,
                                field_strides, s);
    if (rc != TM_OK) return rc;
    if (!grad_strides) return TM_ERR_SHAPE;
    for (int a = 0; a < 3; ++a)
        if (grad_strides[a] < 0) return TM_ERR_SHAPE;
    if (s.positions == 0) return TM_OK;
    if (!up_logp && !up_entropy && !up_mean) return TM_ERR_NULL;
    if ((up_logp && !labels) || (up_mean && !field)) return TM_ERR_NULL;
    if (!stats && classes > TM_LABEL_MAX_RECOMPUTE) return TM_ERR_NULL;
    if (stats && ((up_entropy && !entropy) || (up_mean && !mean))) return TM_ERR_NULL;
    if (!out_grad) return TM_ERR_NO_OUTPUT;
    const uint64_t span = view_span(s.n, grad_strides);
    if (!span) return TM_ERR_TOO_LARGE;
    if (self_overlap(s.n, grad_strides)) return TM_ERR_ALIAS;
    const uint64_t n4 = s.positions * 4;
    const Range in[] = {{logits, s.x_bytes}, {labels, s.positions * s.label_bytes}, {field, s.field_bytes},
                        {stats, 2 * n4}, {entropy, n4}, {mean, n4}, {up_logp, n4}, {up_entropy, n4}, {up_mean, n4}};
    const Range out[] = {{out_grad, span * float_bytes(dtype)}};
    if (aliased(in, out)) return TM_ERR_ALIAS;
    LabelGradArgs a{};
    a.x = logits;
    a.label = labels;
    a.field = up_mean ? field : nullptr;
    a.stats = stats;
    a.entropy = entropy;
    a.mean = mean;
    a.up_logp = up_logp;
    a.up_entropy = up_entropy;
    a.up_mean = up_mean;
    a.grad = out_grad;
    for (int i = 0; i < 3; ++i) {
        a.xs[i] = strides[i];
        a.fs[i] = a.field ? field_strides[i] : 0;
        a.gs[i] = grad_strides[i];
    }
    a.outer = uint32_t(outer);
    a.classes = uint32_t(classes);
    a.inner = uint32_t(inner);
    a.label_bytes = int32_t(s.label_bytes);
    a.n = uint32_t(s.positions);
    LabelPlan p = label_plan(dtype, s.n[0], s.n[1], s.n[2], strides);
    // rows and 16-byte stores need the gradient to lie as the logits do
    if (p.rows && grad_strides[1] != 1) {
        p.rows = p.swap = false;
        p.wide = 1;
        p.held = 0;
    }
    if (grad_strides[p.swap ? 0 : 2] != 1) p.wide = 1;
    if (p.swap) {
        swap_positions(a);
        std::swap(a.gs[0], a.gs[2]);
    }
    a.div_inner = Div32::make(a.inner);
    return by_type(dtype, [&](auto t) {
        using T = decltype(t);
        if (p.rows) {
            // 16 lanes (65536 x 100: 10, a wave 25) or a wave to a row of up to
            // eight loads a lane; else a workgroup to eight loads a thread, or
            // to one where that leaves CUs idle.
            const uint64_t load = 16 / sizeof(T);
            if (s.n[1] <= 64 * 8 * load) {
                a.lanes = p.brief ? 16 : 64;
                a.share = uint32_t(s.n[1]);
            } else {
                a.lanes = 256;
                a.share = uint32_t(256 * load * (s.positions * ceil_div(s.n[1], 8 * 256 * load) < kFill ? 1 : 8));
            }
            a.groups = uint32_t(ceil_div(s.n[1], a.share));
            a.div_groups = Div32::make(a.groups);
            if (s.positions * a.groups >= kLimit) return int(TM_ERR_TOO_LARGE);
            const uint32_t blocks = a.lanes == 256 ? a.n * a.groups : uint32_t(ceil_div(a.n, 256 / a.lanes));
            return by_parts(a.up_entropy, a.field, [&](auto e, auto f) {
                constexpr bool E = decltype(e)::value, F = decltype(f)::value;
                return launch(k_label_grad_rows<T, E, F>, row_grid(blocks), dim3(256), 0, stream, a);
            });
        }
        a.groups = uint32_t(ceil_div(a.inner, p.wide));
        a.div_groups = Div32::make(a.groups);
        const uint32_t threads = a.outer * a.groups;
        const dim3 grid((threads + 255) / 256);
        if (p.held) {
            return by_held(p.held, [&](auto held) {
                return by_parts(a.up_entropy, a.field, [&](auto e, auto f) {
                    constexpr int C = decltype(held)::value;
                    constexpr bool E = decltype(e)::value, F = decltype(f)::value;
                    return launch(p.wide > 1 ? k_label_grad_held<T, kHeldV<T, C>, C, E, F>
                                             : k_label_grad_held<T, 1, C, E, F>, grid, dim3(256), 0, stream, a);
                });
            });
        }
        const uint64_t shares = std::min<uint64_t>({ceil_div(kBusyThreads, threads), ceil_div(s.n[1], 8), 65535});
        a.share = uint32_t(ceil_div(s.n[1], shares));
        return by_parts(a.up_entropy, a.field, [&](auto e, auto f) {
            constexpr bool E = decltype(e)::value, F = decltype(f)::value;
            return launch(p.wide > 1 ? k_label_grad_run<T, kRunV, E, F> : k_label_grad_run<T, 1, E, F>,
                          dim3(grid.x, uint32_t(ceil_div(s.n[1], a.share))), dim3(256), 0, stream, a);
        });
    });
}

// ---------------------------------------------------------------------------
// Biases.
// ---------------------------------------------------------------------------
namespace {

constexpr int64_t kMaxHeads = 1 << 16;
struct BiasShape {
    BiasSource src;
    uint64_t batch, field_batch;
    uint64_t field_bytes;       // of the distances
    uint64_t elements;          // batch * heads * positions
};

int check_field(const void *distances, int distance_dtype, int64_t batch, int64_t positions, BiasShape &s) {
    if (batch < 0 || positions < 0) return TM_ERR_SHAPE;
    if (distance_dtype != TM_DTYPE_F32 && distance_dtype != TM_DTYPE_I32) return TM_ERR_DTYPE;
    if (uint64_t(batch) >= kLimit || uint64_t(positions) >= kLimit) return TM_ERR_TOO_LARGE;
    s.src.source = distance_dtype == TM_DTYPE_F32 ? kFieldF32 : kFieldI32;
    s.src.field = distances;
    s.src.positions = uint32_t(positions);
    s.batch = s.field_batch = uint64_t(batch);
    s.field_bytes = s.batch * uint64_t(positions) * 4;
    if (!distances && s.field_bytes) return TM_ERR_NULL;
    return TM_OK;
}

int check_grid(int ndim, const int64_t *query_shape, const int64_t *key_shape, const int64_t *query_offset, int metric,
               const double *sampling, int64_t batch, BiasShape &s) {
    if (ndim < 1 || ndim > kBiasMaxDim) return TM_ERR_NDIM;
    if (!query_shape || !key_shape || batch < 0) return TM_ERR_SHAPE;
    if (metric < TM_METRIC_EUCLIDEAN || metric > TM_METRIC_OFFSET || (metric == TM_METRIC_OFFSET && ndim != 1))
        return TM_ERR_METRIC;
    uint64_t nq = 1, nk = 1;
    for (int a = 0; a < ndim; ++a) {
        if (query_shape[a] < 0 || key_shape[a] < 0) return TM_ERR_SHAPE;
        const int64_t off = query_offset ? query_offset[a] : 0, lim = int64_t(1) << 30;
        if (query_shape[a] > lim || key_shape[a] > lim || off > lim || off < -lim) return TM_ERR_TOO_LARGE;
        const double sp = sampling ? sampling[a] : 1.0;
        if (!std::isfinite(sp) || !(sp > 0.0) || !std::isfinite(float(sp)) || !(float(sp) > 0.0f))
            return TM_ERR_SAMPLING;
        s.src.offset[a] = int32_t(off);
        s.src.sampling[a] = float(sp);
        nq *= uint64_t(query_shape[a]);
        nk *= uint64_t(key_shape[a]);
        if (nq >= kLimit || nk >= kLimit) return TM_ERR_TOO_LARGE;
    }
    if (nq * nk >= kLimit || uint64_t(batch) >= kLimit) return TM_ERR_TOO_LARGE;
    uint64_t behind_q = 1, behind_k = 1;
    for (int a = ndim - 1; a >= 0 && nq * nk; --a) {
        s.src.div_q[a] = Div32::make(uint32_t(behind_q));
        s.src.div_k[a] = Div32::make(uint32_t(behind_k));
        behind_q *= uint64_t(query_shape[a]);
        behind_k *= uint64_t(key_shape[a]);
    }
    if (metric == TM_METRIC_OFFSET && s.src.sampling[0] != 1.0f) return TM_ERR_SAMPLING;
    s.src.source = metric == TM_METRIC_OFFSET ? kOffset : metric == TM_METRIC_EUCLIDEAN ? kEuclid
                   : metric == TM_METRIC_TAXICAB ? kTaxicab : kChess;
    s.src.ndim = ndim;
    s.src.positions = uint32_t(nq * nk);
    s.src.div_key = Div32::make(uint32_t(nk ? nk : 1));
    s.batch = uint64_t(batch);
    s.field_batch = 1;
    return TM_OK;
}

int check_table(int buckets, int64_t heads, const float *edges, int table_dtype, int value_dtype, BiasShape &s) {
    if (buckets < 1 || buckets > int(kMaxBuckets) || heads < 1) return TM_ERR_SHAPE;
    if (!float_type(table_dtype) || !float_type(value_dtype)) return TM_ERR_DTYPE;
    if (heads > kMaxHeads) return TM_ERR_TOO_LARGE;
    if (!edges && buckets > 1) return TM_ERR_NULL;
    const uint64_t lim = uint64_t(1) << 58;
    const uint64_t bh = s.batch * uint64_t(heads);          // below 2^54
    if (s.src.positions && bh > lim / s.src.positions) return TM_ERR_TOO_LARGE;
    s.src.edges = edges;
    s.src.buckets = uint32_t(buckets);
    s.src.span = pow2_from(s.src.buckets);
    s.elements = bh * s.src.positions;
    return TM_OK;
}

int run_bias(const BiasShape &s, const void *table, int table_dtype, int64_t heads, const void *add, void *out,
             int out_dtype, hipStream_t stream) {
    if (s.elements == 0) return TM_OK;
    if (!table) return TM_ERR_NULL;
    if (!out) return TM_ERR_NO_OUTPUT;
    const uint64_t bytes = s.elements * float_bytes(out_dtype);
    const Range in[] = {{s.src.field, s.field_bytes}, {table, s.src.buckets * uint64_t(heads) * float_bytes(table_dtype)},
                        {s.src.edges, 4 * uint64_t(s.src.buckets - 1)}, {add, bytes}};
    const Range outs[] = {{out, bytes}};
    if (aliased(in, outs)) return TM_ERR_ALIAS;
    BiasArgs a{};
    a.src = s.src;
    a.table = table;
    a.table_type = table_dtype;
    a.add = add;
    a.out = out;
    a.heads = uint32_t(heads);
    a.batch = uint32_t(s.batch);
    a.field_batch = uint32_t(s.field_batch);
    // Shares: all heads to a workgroup where the positions alone fill the chip,
    // else four heads at a time and then parts of the batch (one query and 4096
    // keys, 16 heads: 6.0 us, unshared 8.9; 512 x 512, 8 samples: 25, 38); a
    // share's table takes at most 36 KB of LDS.
    uint64_t vec = 16 / float_bytes(out_dtype);
    if (s.src.positions < vec) vec = 1;
    const uint64_t tiles = ceil_div(s.src.positions, kBiasThreads * vec);
    const uint64_t blocks = tiles * s.field_batch;
    const uint64_t quads = ceil_div(uint64_t(heads), 4);
    const uint64_t most = std::max<uint64_t>(1, 2048 / s.src.buckets);
    const uint64_t want = ceil_div(kFill, blocks);
    const uint64_t share = std::min(most, ceil_div(quads, std::min(quads, want)));
    const uint64_t shares = ceil_div(quads, share);
    uint64_t bshares = 1;
    if (s.field_batch == 1)
        bshares = std::min(std::min(s.batch, 65535 / shares), ceil_div(kFill, blocks * shares));
    const uint64_t bshare = s.field_batch == 1 ? ceil_div(s.batch, bshares) : 1;
    if (s.field_batch == 1) bshares = ceil_div(s.batch, bshare);
    if (blocks >= kLimit) return TM_ERR_TOO_LARGE;
    a.head_share = uint32_t(4 * share);
    a.row = uint32_t(4 * (share | 1));
    a.batch_share = uint32_t(bshare);
    a.batch_shares = uint32_t(bshares);
    a.tiles = uint32_t(blocks);
    a.div_tiles = Div32::make(uint32_t(tiles));
    // workgroups that go on, 16 to a CU (2 x 155 x 240 x 237, 3 heads: 62 us; 8 or 4 to a CU 70 and 67, one to
    // every tile 64)
    const uint64_t grid = std::min(blocks, std::max<uint64_t>(1, 4 * kFill / (shares * bshares)));
    const size_t lds = (size_t(s.src.buckets) * a.row + s.src.span) * 4;
    return by_type(out_dtype, [&](auto t) {
        using T = decltype(t);
        return launch(vec > 1 ? k_bias<T, 16 / sizeof(T)> : k_bias<T, 1>, dim3(uint32_t(grid), uint32_t(shares * bshares)), dim3(kBiasThreads), lds,
                      stream, a);
    });
}

template <typename F>
int by_blocks(int blocks, F fn) {
    if (blocks == 1) return fn(Int<1>{});
    if (blocks == 2) return fn(Int<2>{});
    return fn(Int<4>{});
}

uint64_t grad_splits_most(uint64_t head_groups) { return std::max<uint64_t>(64, 512 / head_groups); }
uint64_t grad_tile_rows(uint32_t buckets) { return std::max<uint64_t>(16, pow2_from(buckets)); }

int run_bias_grad(const BiasShape &s, const void *grad, int grad_dtype, int64_t heads, void *out, int table_dtype,
                  void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!out) return TM_ERR_NO_OUTPUT;
    if (!grad && s.elements) return TM_ERR_NULL;
    const size_t need = tm_bias_grad_workspace_size(int(s.src.buckets), heads);
    if (need && (!workspace || workspace_bytes < need || uintptr_t(workspace) % 16)) return TM_ERR_WORKSPACE;
    const Range in[] = {{s.src.field, s.field_bytes}, {s.src.edges, 4 * uint64_t(s.src.buckets - 1)},
                        {grad, s.elements * float_bytes(grad_dtype)}};
    const Range outs[] = {{out, s.src.buckets * uint64_t(heads) * float_bytes(table_dtype)},
                          {need ? workspace : nullptr, need}};
    if (aliased(in, outs)) return TM_ERR_ALIAS;
    BiasGradArgs a{};
    a.src = s.src;
    a.grad = grad;
    a.out = out;
    a.partial = static_cast<float *>(workspace);
    a.heads = uint32_t(heads);
    a.batch = uint32_t(s.batch);
    a.field_batch = uint32_t(s.field_batch);
    a.table_type = table_dtype;
    // Units of one step of positions and, where samples share the buckets, as many of
    // them as leave enough units; two workgroups of eight waves to a CU.
    const uint64_t groups = ceil_div(uint64_t(heads), 16);
    // Samples smaller than a load share steps, as many whole ones as fit.
    const bool few = s.src.positions && s.src.positions < 16 / float_bytes(grad_dtype);
    // Blocks of four heads to a load: up to 4 heads 16 us, two blocks for up to
    // 8 heads 19 us (8 x 512^2 bf16, 24 buckets); with four blocks 18 and 19.5.
    const int blocks = few ? 4 : heads <= 4 ? 1 : heads <= 8 ? 2 : 4;
    const uint64_t step = 256 / float_bytes(grad_dtype) * (4 / blocks);
    const uint64_t steps = ceil_div(s.src.positions, step);
    uint64_t shares = s.batch;
    a.batch_share = 1;
    if (s.field_batch == 1 && s.batch) {
        a.batch_share = uint32_t(std::min(s.batch, std::max<uint64_t>(1, s.batch * steps / 4096)));
        shares = ceil_div(s.batch, a.batch_share);
    }
    if (few) {
        a.batch_share = uint32_t(step / s.src.positions);
        shares = ceil_div(s.batch, a.batch_share);
    }
    const uint64_t units = steps * shares;                  // few: one step to a group
    if (units >= kLimit) return TM_ERR_TOO_LARGE;
    a.units = uint32_t(units);
    a.div_steps = Div32::make(few ? s.src.positions : uint32_t(std::max<uint64_t>(1, steps)));
    a.splits = uint32_t(std::max<uint64_t>(1, std::min(ceil_div(units, kGradWaves), grad_splits_most(groups))));
    a.tile_rows = uint32_t(grad_tile_rows(s.src.buckets));
    const int rc = by_type(grad_dtype, [&](auto t) {
        using T = decltype(t);
        const auto run = [&](auto n, auto f) {
            constexpr int B = decltype(n)::value;
            constexpr bool Few = decltype(f)::value;
            void (*const kernels[])(BiasGradArgs) = {k_bias_grad<T, 1, B, Few>, k_bias_grad<T, 2, B, Few>,
                                                     k_bias_grad<T, 4, B, Few>, k_bias_grad<T, 8, B, Few>,
                                                     k_bias_grad<T, 16, B, Few>};
            int tiles = 0;
            while ((16u << tiles) < a.tile_rows) ++tiles;
            return launch(kernels[tiles], dim3(a.splits, uint32_t(groups)), dim3(kGradThreads), 0, stream, a);
        };
        if (few) return run(Int<4>{}, Bool<true>{});
        return by_blocks(blocks, [&](auto n) { return run(n, Bool<false>{}); });
    });
    if (rc != TM_OK) return rc;
    return launch(k_bias_join, dim3(s.src.buckets, uint32_t(groups)), dim3(256), 0, stream, a);
}

}  // namespace

extern "C" int tm_distance_bias(const void *distances, int distance_dtype, int64_t batch, int64_t positions,
                                const void *table, int table_dtype, int buckets, int64_t heads, const float *edges,
                                const void *add, void *out, int out_dtype, hipStream_t stream) {
    BiasShape s{};
    int rc = check_field(distances, distance_dtype, batch, positions, s);
    if (rc == TM_OK) rc = check_table(buckets, heads, edges, table_dtype, out_dtype, s);
    return rc == TM_OK ? run_bias(s, table, table_dtype, heads, add, out, out_dtype, stream) : rc;
}

extern "C" int tm_relative_bias(int ndim, const int64_t *query_shape, const int64_t *key_shape,
                                const int64_t *query_offset, int metric, const double *sampling, int64_t batch,
                                const void *table, int table_dtype, int buckets, int64_t heads, const float *edges,
                                const void *add, void *out, int out_dtype, hipStream_t stream) {
    BiasShape s{};
    int rc = check_grid(ndim, query_shape, key_shape, query_offset, metric, sampling, batch, s);
    if (rc == TM_OK && !add && batch > 1) rc = TM_ERR_SHAPE;
    if (rc == TM_OK) rc = check_table(buckets, heads, edges, table_dtype, out_dtype, s);
    return rc == TM_OK ? run_bias(s, table, table_dtype, heads, add, out, out_dtype, stream) : rc;
}

extern "C" size_t tm_bias_grad_workspace_size(int buckets, int64_t heads) {
    if (buckets < 1 || buckets > int(kMaxBuckets) || heads < 1 || heads > kMaxHeads) return 0;
    const uint64_t groups = ceil_div(uint64_t(heads), 16);
    return grad_splits_most(groups) * groups * grad_tile_rows(uint32_t(buckets)) * 64;
}

extern "C" int tm_distance_bias_grad(const void *distances, int distance_dtype, int64_t batch, int64_t positions,
                                     const void *grad, int grad_dtype, int buckets, int64_t heads, const float *edges,
                                     void *out_grad, int table_dtype, void *workspace, size_t workspace_bytes,
                                     hipStream_t stream) {
    BiasShape s{};
    int rc = check_field(distances, distance_dtype, batch, positions, s);
    if (rc == TM_OK) rc = check_table(buckets, heads, edges, table_dtype, grad_dtype, s);
    return rc == TM_OK ? run_bias_grad(s, grad, grad_dtype, heads, out_grad, table_dtype, workspace, workspace_bytes,
                                       stream) : rc;
}

extern "C" int tm_relative_bias_grad(int ndim, const int64_t *query_shape, const int64_t *key_shape,
                                     const int64_t *query_offset, int metric, const double *sampling, int64_t batch,
                                     const void *grad, int grad_dtype, int buckets, int64_t heads, const float *edges,
                                     void *out_grad, int table_dtype, void *workspace, size_t workspace_bytes,
                                     hipStream_t stream) {
    BiasShape s{};
    int rc = check_grid(ndim, query_shape, key_shape, query_offset, metric, sampling, batch, s);
    if (rc == TM_OK) rc = check_table(buckets, heads, edges, table_dtype, grad_dtype, s);
    return rc == TM_OK ? run_bias_grad(s, grad, grad_dtype, heads, out_grad, table_dtype, workspace, workspace_bytes,
                                       stream) : rc;
}
