// head.h -- kernels of the log-probabilities from hidden states and a
// vocabulary's weight (tm_head_logp in include/tm_train.h).
//
// With x = h w^T, c = scale log2(e) and M the largest x of a row:
//     s = sum_v 2^(c (x_v - M)),   log sum exp (scale x) = scale M + ln 2 log2 s,
//     log p_y = ln 2 (c (x_y - M) - log2 s),   p_v = 2^(c (x_v - M)) / s.
// M is taken off first, which is exact for logits near it: the largest has the
// power 1, and what is left out of a sum next to 1 is no more than its rounding.
// M starts at -FLT_MAX instead of -inf, so that no difference is inf - inf:
// logits at -inf get 0, and s = 0 marks a row with no class left.
//
// The logits are never stored: a tile's pass over k ends in sums of its rows.
// The gradient computes them anew, a piece of the vocabulary at a time, as
//     g_nv = alpha_n 1[v = y_n] - beta_n p_nv,   alpha = scale up_logp,
//     beta = scale (up_logp - up_log_sum),
// and leaves g in the operands' type for the two products
//     dh = g w,   dw = g^T h.
// Its rounding to 16 bits is off by as much as that of the results, and most of
// that is the label's own term, the one number of a row that is not small.  What
// rounding takes from it is kept in float32, `rest`, and added to both products:
// of 4096 x 32768 x 1024 bf16 the gradients were 0.0024 off and are 0.0017, as
// float32's rounded once, for 955 us instead of 935.  With up to kFineRows rows
// or kFineClasses classes, of which few make up most of a result, g has two
// planes, 16 bits or more.  Beyond, they take longer: gradients of 300 x 131072 x
// 2048 bf16 1149 us instead of 827, of 512 rows 1545 and 1036, of 300 x 512 x 1000
// 43 and 38, of 300 x 256 x 1000 41 and 36; of 1000 x 128 x 1000 44 and 58, of 4000
// rows 61 and 66, of 300 rows 37 and 36, since a tile has most rows' labels there.
// Rows without a label take part only where the log sums are asked for: the
// rows that do are packed first, and the products run over those alone.
#pragma once

#include "label.h"
#include "product.h"

namespace tmtrain {

constexpr uint32_t kFewRows = 16;               // rows of hidden states that one matrix instruction holds
constexpr uint32_t kFineRows = 256;             // rows up to which g of 16-bit operands has two planes
constexpr uint32_t kFineClasses = 128;          // and classes
constexpr uint32_t kListChunk = 1024;           // rows that a workgroup counts

struct HeadSum {
    float m, s;                 // M, sum of 2^(c (h w - M))
};
constexpr float kLowest = -FLT_MAX;

// 2^(c (a - b)) for a <= b; 0 where a is kLowest and b is not.
__device__ __forceinline__ float shrink(float a, float b, float c) {
    return a == b ? 1.0f : exp2_hw(fmaxf((a - b) * c, -200.0f));
}

// inf - inf of the references of rows with +inf stays NaN in s.
__device__ __forceinline__ HeadSum join(HeadSum a, HeadSum b, float c) {
    const float m = fmaxf(a.m, b.m);
    return {m, a.s * shrink(a.m, m, c) + b.s * shrink(b.m, m, c)};
}

// A packed row, for the gradient.
struct HeadRow {
    float m;
    float a, b;                 // alpha, beta / s, for float16 times a power of two
    int32_t y;
};

struct HeadArgs {
    const void *hidden, *weight;
    uint64_t hidden_stride, weight_stride;      // elements
    const void *label;
    int32_t label_bytes;
    uint32_t n, classes, width;
    bool all;                   // rows without a label take part
    float scale, c;             // c = scale log2(e)
    float *logp, *log_sum;
    HeadSum *stats;             // of the rows in the caller's order
    const float *up_logp, *up_log_sum;
    void *grad_hidden, *grad_weight;
    // in the workspace
    uint32_t *count;            // packed rows
    uint32_t *chunk_count;      // of each chunk, then their exponents
    uint32_t pack_rows;         // of a workgroup, up to kPackRows
    uint32_t chunks;            // 0: few rows, which are counted where they are needed
    Div32 div_pieces;           // pieces of a packed row
    uint32_t *list;             // the packed rows' numbers
    int32_t *place;             // and where each row went, or -1
    HeadRow *row;
    float *inverse;             // float16: what takes a packed row's power of two back; then the common one's
    void *packed;               // packed hidden states [n_pad][width_pad]
    HeadSum *part;              // [parts][n_pad]
    float *found;               // h w of the packed rows' labels
    void *slope, *slope_common; // g [n_pad][piece]; float16: times its row's power of two, and the common one
    float *rest, *rest_common;  // g of 16 bits: what its rounding takes from the labels', for dh and float16's dw
    void *weight_laid;          // a piece's weights in whole steps, where they do not lie so
    float *sum;                 // dh by splits: [splits][rows of tiles][sum_stride]; few rows: [splits][n][sum_stride]
    uint32_t n_pad, width_pad, sum_stride;
    uint32_t parts;
    uint32_t first, piece;      // classes of the piece at hand, and its width
    uint32_t few_shift;         // few rows: 1 << few_shift waves share a row's columns
    uint32_t splits, steps;     // few rows: shares of the classes, and classes of one
    uint32_t blocks, most;      // of the product for dh: workgroups, splits that its k allows
    uint32_t tiles_m, tile_n;   // its tiles across the width, and the rows of one
    uint32_t weight_splits;     // of the product for dw, where the classes' tiles are few
    float *weight_sum;          // dw by splits: [splits][classes][sum_stride]
    bool add;                   // to the sums so far
};

// ---------------------------------------------------------------------------
// The packed rows.
// ---------------------------------------------------------------------------

// For float16, g is held times a power of two that brings |alpha| + |beta| to
// [2^14, 2^15): p is then exact to 11 bits down to 2^-29 of it, where as it
// stands everything below 2^-14 would lose bits.
constexpr int kSlopeExponent = 15;
__device__ __forceinline__ int exponent_of(float x) {       // 2^e > x, 0 for zeros and what is not finite
    if (!(x > 0.0f) || !(x <= FLT_MAX)) return 0;
    return max(-100, int(__builtin_amdgcn_frexp_expf(x)));
}
__device__ __forceinline__ float power(int e) { return __builtin_amdgcn_ldexpf(1.0f, e); }

struct HeadUp {
    float a, b;
};
__device__ __forceinline__ HeadUp head_up(const HeadArgs &p, uint32_t n, int32_t y) {
    const float a = y >= 0 && p.up_logp ? p.up_logp[n] : 0.0f;
    return {p.scale * a, p.scale * (a - (p.up_log_sum ? p.up_log_sum[n] : 0.0f))};
}

// The label of row n, and whether the row takes part.
__device__ __forceinline__ bool takes_part(const HeadArgs &p, uint32_t n, int32_t &y) {
    y = p.label ? load_label(p.label, p.label_bytes, n, p.classes) : -1;
    return y >= 0 || p.all;
}
// Of N rows, `step` apart, at once: what of them is before `end`.  Loads come first, none waits for another.
template <int N, typename F>
__device__ __forceinline__ void each_part(const HeadArgs &p, uint32_t n0, uint32_t step, uint32_t end, bool ups, F fn) {
    int32_t y[N];
    uint32_t n[N];
    float a[N] = {}, z[N] = {};
#pragma unroll
    for (int k = 0; k < N; ++k) n[k] = min(n0 + k * step, end - 1);
    const auto labels = [&](const auto *label) {
#pragma unroll
        for (int k = 0; k < N; ++k) y[k] = label[n[k]] < p.classes ? int32_t(label[n[k]]) : -1;
    };
    if (!p.label) {
#pragma unroll
        for (int k = 0; k < N; ++k) y[k] = -1;
    } else if (p.label_bytes == 1) {
        labels(static_cast<const uint8_t *>(p.label));
    } else if (p.label_bytes == 4) {
        labels(static_cast<const uint32_t *>(p.label));
    } else {
        labels(static_cast<const uint64_t *>(p.label));
    }
    if (ups && p.up_logp) {
#pragma unroll
        for (int k = 0; k < N; ++k) a[k] = p.up_logp[n[k]];
    }
    if (ups && p.up_log_sum) {
#pragma unroll
        for (int k = 0; k < N; ++k) z[k] = p.up_log_sum[n[k]];
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        if (n0 + k * step >= end || (y[k] < 0 && !p.all)) continue;
        const float up = y[k] >= 0 ? a[k] : 0.0f;
        fn(n[k], y[k], HeadUp{p.scale * up, p.scale * (up - z[k])});
    }
}
// Exponent of a row's slopes, kNoExponent for zeros.
constexpr int kNoExponent = -1000;
__device__ __forceinline__ int slope_exponent(HeadUp u) {
    const float size = fabsf(u.a) + fabsf(u.b);
    return size > 0.0f ? exponent_of(size) : kNoExponent;
}

// Adds up a workgroup's counts and takes the largest of its exponents: whole numbers, whose order does not matter.
__device__ __forceinline__ void tally(uint32_t mine, int most, uint32_t *found, int *top) {
    const uint32_t all = wave_reduce(mine, 0u, [](uint32_t a, uint32_t b) { return a + b; });
    const int best = int(wave_max(uint32_t(most - kNoExponent))) + kNoExponent;
    if ((threadIdx.x & 63) == 0) {
        atomicAdd(found, all);
        atomicMax(top, best);
    }
}

// Rows of each chunk that take part (and their largest exponent), where there are many chunks.
__global__ __launch_bounds__(256) void k_head_count(HeadArgs p) {
    __shared__ uint32_t found;
    __shared__ int top;
    if (threadIdx.x == 0) {
        found = 0;
        top = kNoExponent;
    }
    __syncthreads();
    const uint32_t last = min(p.n, (blockIdx.x + 1) * kListChunk);
    uint32_t mine = 0;
    int most = kNoExponent;
    each_part<kListChunk / 256>(p, blockIdx.x * kListChunk + threadIdx.x, 256, last, p.inverse, [&](uint32_t, int32_t, HeadUp u) {
        ++mine;
        if (p.inverse) most = max(most, slope_exponent(u));
    });
    tally(mine, most, &found, &top);
    __syncthreads();
    if (threadIdx.x == 0) {
        p.chunk_count[blockIdx.x] = found;
        p.chunk_count[gridDim.x + blockIdx.x] = uint32_t(top);
    }
}

template <typename T>
constexpr float kLargest = __is_same(T, bf16) ? 0x1.fep127f : __is_same(T, f16) ? 65504.0f : FLT_MAX;
// x in planes, each of what the ones before it leave: nothing of an infinity.  A number that the first plane would round
// to one is cut to the largest there, and the next plane has the rest.
template <typename T, int V, int P>
__device__ __forceinline__ void split(const float (&x)[V], Pack<T, V> (&out)[P]) {
    float rest[V];
#pragma unroll
    for (int j = 0; j < V; ++j) rest[j] = x[j];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        if (p == 0 && P > 1) {
            float head[V];
#pragma unroll
            for (int j = 0; j < V; ++j)
                head[j] = fabsf(x[j]) <= FLT_MAX ? fminf(fmaxf(x[j], -kLargest<T>), kLargest<T>) : x[j];
            out[0] = narrow_pack<T>(head);
#pragma unroll
            for (int j = 0; j < V; ++j) rest[j] = fabsf(x[j]) == INFINITY ? 0.0f : x[j] - widen(out[0].at(j));
            continue;
        }
        out[p] = narrow_pack<T>(rest);
#pragma unroll
        for (int j = 0; j < V; ++j) rest[j] -= widen(out[p].at(j));
    }
}

// What rounding to T takes from a label's g, for packed row n; 0 where that is no number.  For float16, `ratio` takes g to
// the common power of two.
template <typename T>
__device__ __forceinline__ void keep_rest(const HeadArgs &p, uint32_t n, float g, float ratio) {
    const auto lost = [](float x) {
        const float rest = x - widen(narrow<T>(x));
        return fabsf(rest) <= FLT_MAX ? rest : 0.0f;
    };
    if (p.rest) p.rest[n] = lost(g);
    if (__is_same(T, f16) && p.rest_common) p.rest_common[n] = lost(g * ratio);
}

// V elements as they are laid out: in P planes of S, `plane` elements apart.
template <typename T, typename S, int P, int V>
__device__ __forceinline__ void lay(const T *from, uint32_t n, S *to, uint64_t plane) {
    Pack<T, V> q{};
    if (n) q = load_pack<V>(from, n, T{});
    if constexpr (P == 1) {
        store_pack<V>(to, q);
    } else {
        float x[V];
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = widen(q.at(j));
        Pack<S, V> planes[P];
        split(x, planes);
#pragma unroll
        for (int k = 0; k < P; ++k) store_pack<V>(to + k * plane, planes[k]);
    }
}

// Packs the hidden states of kPackRows rows, in whole steps with zeros behind
// them, and writes where they went and what the gradient needs of them.  Every
// workgroup counts the rows before its own and all of them: one by one, or by the
// chunks' counts.  Behind the last one, workgroups leave zeros up to a multiple
// of 64.
// 4096 rows of 1024 bf16: 9.8 us (9 and 5 for chunks' counts); 509 rows 5.6.
constexpr uint32_t kPackRows = 8;
template <typename T, typename S, int P>
__global__ __launch_bounds__(256) void k_head_pack(HeadArgs p) {
    constexpr uint32_t V = 16 / sizeof(S);
    __shared__ uint32_t before, own, total;
    __shared__ int top;
    __shared__ uint32_t from[kPackRows];
    if (threadIdx.x == 0) {
        before = total = 0;
        top = kNoExponent;
    }
    __syncthreads();
    const uint32_t r0 = blockIdx.x * p.pack_rows, chunk = r0 / kListChunk;
    const bool exponents = p.inverse != nullptr;
    // the workgroup's own rows, a lane of the first wave to each
    const uint32_t own_row = r0 + threadIdx.x;
    const bool real_row = threadIdx.x < p.pack_rows && own_row < p.n;
    int32_t y = -1;
    const bool in = real_row && takes_part(p, own_row, y);
    uint32_t mine = 0, all = 0;
    int most = kNoExponent;
    const uint32_t last = p.chunks ? r0 : p.n;
    constexpr int kAhead = 8;
    for (uint32_t n0 = (p.chunks ? chunk * kListChunk : 0) + threadIdx.x; n0 < last; n0 += 256 * kAhead)
        each_part<kAhead>(p, n0, 256, last, exponents && !p.chunks, [&](uint32_t n, int32_t, HeadUp u) {
            mine += n < r0;
            all += !p.chunks;
            if (exponents && !p.chunks) most = max(most, slope_exponent(u));
        });
    for (uint32_t i = threadIdx.x; i < p.chunks; i += 256) {
        const uint32_t found = p.chunk_count[i];
        mine += i < chunk ? found : 0;
        all += found;
        if (exponents) most = max(most, int(p.chunk_count[p.chunks + i]));
    }
    tally(mine, most, &before, &top);
    tally(all, most, &total, &top);
    __syncthreads();
    if (threadIdx.x < 64) {
        const uint32_t n = own_row;
        const uint64_t set = __ballot(in);
        const uint32_t rank = __popcll(set & ((uint64_t(1) << threadIdx.x) - 1)), at = before + rank;
        if (threadIdx.x == 0) own = __popcll(set);
        const int common = top == kNoExponent ? 0 : top;
        if (threadIdx.x == 0 && blockIdx.x == 0 && exponents) p.inverse[p.n_pad] = power(common - kSlopeExponent);
        if (real_row && p.place) p.place[n] = in ? int32_t(at) : -1;
        if (real_row && !in && !p.row) {
            if (p.logp) p.logp[n] = 0.0f;
            if (p.stats) p.stats[n] = {0.0f, 1.0f};
        }
        if (in) {
            from[rank] = n;
            p.list[at] = n;
            if (p.row) {
                HeadUp u = head_up(p, n, y);
                const HeadSum s = p.stats[n];
                if (s.s == 0.0f) u = {0.0f, 0.0f};          // no class left
                HeadRow r = {s.m, u.a, s.s == 0.0f ? 0.0f : u.b / s.s, y};
                if (exponents) {
                    int e = slope_exponent(u);
                    if (e == kNoExponent) e = common;
                    r.a = __builtin_amdgcn_ldexpf(r.a, kSlopeExponent - e);
                    r.b = __builtin_amdgcn_ldexpf(r.b, kSlopeExponent - e);
                    p.inverse[at] = power(e - kSlopeExponent);
                }
                p.row[at] = r;
            }
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && blockIdx.x == 0) *p.count = total;
    const uint32_t pieces = p.width_pad / V;
    const uint64_t plane = uint64_t(p.n_pad) * p.width_pad;
    S *packed = static_cast<S *>(p.packed);
#pragma unroll 4
    for (uint32_t i = threadIdx.x; i < own * pieces; i += 256) {
        const uint32_t r = p.div_pieces.div(i), c = (i - r * pieces) * V;
        const bool real = c < p.width;
        lay<T, S, P, V>(static_cast<const T *>(p.hidden) + (real ? from[r] * p.hidden_stride + c : 0),
                        real ? p.width - c : 0, packed + uint64_t(before + r) * p.width_pad + c, plane);
    }
    for (uint32_t r = total + blockIdx.x; r < ((total + 63) & ~63u); r += gridDim.x)
        for (uint32_t i = threadIdx.x; i < pieces; i += 256)
            lay<T, S, P, V>(static_cast<const T *>(p.hidden), 0, packed + uint64_t(r) * p.width_pad + i * V, plane);
}

// The weights of the piece at hand, laid out likewise.
template <typename T, typename S, int P>
__global__ __launch_bounds__(256) void k_head_lay(HeadArgs p) {
    constexpr uint32_t V = 16 / sizeof(S);
    const uint32_t rows = min(p.piece, p.classes - p.first), pieces = p.width_pad / V;
    for (uint32_t r = blockIdx.x * blockDim.y + threadIdx.y; r < rows; r += gridDim.x * blockDim.y)
        for (uint32_t i = threadIdx.x; i < pieces; i += blockDim.x) {
            const uint32_t c = i * V;
            lay<T, S, P, V>(static_cast<const T *>(p.weight) + (p.first + r) * p.weight_stride + c,
                            c < p.width ? p.width - c : 0, static_cast<S *>(p.weight_laid) + uint64_t(r) * p.width_pad + c,
                            uint64_t(p.piece) * p.width_pad);
        }
}

// ---------------------------------------------------------------------------
// Products over tiles.
// ---------------------------------------------------------------------------

// The weights of the piece at hand, packed hidden states and g; S is the type they are held in, P the planes.
template <typename S, int P>
__device__ __forceinline__ Operand weight_rows(const HeadArgs &p) {
    const uint32_t rows = min(p.piece, p.classes - p.first);
    if (P > 1 || p.weight_laid)
        return {static_cast<const char *>(p.weight_laid), uint64_t(p.width_pad) * sizeof(S),
                uint64_t(p.piece) * p.width_pad * sizeof(S), rows, uint32_t(p.width_pad * sizeof(S) / 16)};
    return {static_cast<const char *>(p.weight) + uint64_t(p.first) * p.weight_stride * sizeof(S),
            p.weight_stride * sizeof(S), 0, rows, uint32_t(p.width * sizeof(S) / 16)};
}
template <typename S>
__device__ __forceinline__ Operand hidden_rows(const HeadArgs &p, uint32_t rows) {
    return {static_cast<const char *>(p.packed), uint64_t(p.width_pad) * sizeof(S),
            uint64_t(p.n_pad) * p.width_pad * sizeof(S), rows, uint32_t(p.width_pad * sizeof(S) / 16)};
}
template <typename S>
__device__ __forceinline__ Operand slope_rows(const HeadArgs &p, const void *at, uint32_t rows) {
    return {static_cast<const char *>(at), uint64_t(p.piece) * sizeof(S), uint64_t(p.n_pad) * p.piece * sizeof(S), rows,
            uint32_t(p.piece * sizeof(S) / 16)};
}
// The type that T is held in for a tile.
template <typename T, typename Tile>
using Held = std::conditional_t<Tile::kPlanes == 3, bf16, T>;

// Goes through the tiles of logits of `rows` classes and the packed rows, a
// workgroup taking several: the next tile's first step is on its way while
// before(place) has brought what finish(tile, place) needs, and finish runs.
template <typename T, typename Tile, typename Before, typename Finish>
__device__ __forceinline__ void each_tile(const HeadArgs &p, uint32_t rows, uint32_t count,
                                          typename Tile::Buffer &even, typename Tile::Buffer &odd, Before before,
                                          Finish finish) {
    typedef Held<T, Tile> S;
    const uint32_t tiles_n = (count + Tile::BN - 1) / Tile::BN;
    const uint32_t tiles_m = (rows + Tile::BM - 1) / Tile::BM;
    const uint32_t total = tiles_m * tiles_n, steps = p.width_pad / Tile::kStep;
    if (blockIdx.x >= total) return;
    Tile tile;
    const auto begin = [&](TilePlace at) {
        return tile.template begin<false, false>(weight_rows<S, Tile::kPlanes>(p), at.m * Tile::BM,
                                                 hidden_rows<S>(p, p.n_pad), at.n * Tile::BN, 0, even);
    };
    TilePlace at = tile_place(blockIdx.x, tiles_m, tiles_n);
    auto from = begin(at);
    for (uint32_t block = blockIdx.x;;) {
        tile.run(from, 0, steps, even, odd);
        const TilePlace now = at;
        before(tile, now);
        block += gridDim.x;
        const bool more = block < total;
        if (more) {
            at = tile_place(block, tiles_m, tiles_n);
            from = begin(at);
        }
        finish(tile, now);
        if (!more) return;
    }
}

// Sums of the packed rows over a tile's classes, one for each wave's classes,
// and the labels' x.  Bound by the matrix cores and what feeds them, at small
// widths also by the exponentials at a tile's end: 3891 rows of 4096 x 32768 x 1024
// bf16 232 to 243 us by machine (1080 to 1120 TFLOP/s), half of 8192 x 131072 x
// 2048 1610 to 1700 (1290 to 1370).
template <typename T, typename Tile>
__global__ __launch_bounds__(Tile::kThreads, Tile::kWaves / 4) void k_head_sums(HeadArgs p) {
    __shared__ __attribute__((aligned(1024))) typename Tile::Buffer even, odd;
    const uint32_t count = *p.count, rows = min(p.piece, p.classes - p.first);
    uint32_t wants[Tile::TN];                       // the labels' rows among the wave's
    each_tile<T, Tile>(p, rows, count, even, odd, [&](const Tile &tile, TilePlace at) {
#pragma unroll
        for (int j = 0; j < Tile::TN; ++j) {
            const uint32_t n = at.n * Tile::BN + tile.column(j);
            const int32_t y = n < count && p.label ? load_label(p.label, p.label_bytes, p.list[n], p.classes) : -1;
            wants[j] = y < 0 ? ~0u : uint32_t(y) - p.first - at.m * Tile::BM - tile.first_row();
        }
    }, [&](Tile &tile, TilePlace at) {
        const uint32_t part = (p.first / Tile::BM + at.m) * Tile::WM + tile.wave / Tile::WN;
        if ((at.m + 1) * Tile::BM > rows) {         // classes beyond the last
#pragma unroll
            for (int i = 0; i < Tile::TM; ++i)
#pragma unroll
                for (int j = 0; j < Tile::TN; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (at.m * Tile::BM + tile.row(i) + q >= rows) tile.acc[i][j][q] = -INFINITY;
        }
#pragma unroll
        for (int j = 0; j < Tile::TN; ++j) {
            const uint32_t n = at.n * Tile::BN + tile.column(j);
            const bool mine = wants[j] < 16u * Tile::TM && (wants[j] >> 3 & 3) == uint32_t(tile.lane >> 4);
            if (__any(mine)) {                      // few tiles hold a column's label
                float label = 0.0f;
#pragma unroll
                for (int i = 0; i < Tile::TM; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if ((wants[j] & ~24u) == Tile::pair_row(i) + q) label = tile.acc[i][j][q];
                if (mine) p.found[n] = label;
            }
            float most = -INFINITY;
#pragma unroll
            for (int i = 0; i < Tile::TM; ++i) {
                most = max_of(most, tile.acc[i][j][0], tile.acc[i][j][1]);
                most = max_of(most, tile.acc[i][j][2], tile.acc[i][j][3]);
            }
            most = fmaxf(most, __shfl_xor(most, 16));
            most = fmaxf(most, __shfl_xor(most, 32));
            const float m = fmaxf(most, kLowest);
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < Tile::TM; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) s += exp2_hw((tile.acc[i][j][q] - m) * p.c);
            s += __shfl_xor(s, 16);
            s += __shfl_xor(s, 32);
            if (n < count && tile.lane < 16) p.part[uint64_t(part) * p.n_pad + n] = {m, s};
        }
    });
}

// A row's results.
__device__ __forceinline__ void head_store(const HeadArgs &p, uint32_t n, const float *found, HeadSum sum) {
    const int32_t y = p.label ? load_label(p.label, p.label_bytes, n, p.classes) : -1;
    const float log_s = log2f(sum.s);
    if (p.logp) {
        float l = 0.0f;
        if (y >= 0) {
            l = fmaf(*found - sum.m, p.c, -log_s) * kLn2;
            if (sum.s == 0.0f) l = -INFINITY;
        }
        p.logp[n] = l;
    }
    if (p.log_sum) p.log_sum[n] = sum.s == 0.0f ? -INFINITY : fmaf(sum.m, p.scale, log_s * kLn2);
    if (p.stats) p.stats[n] = sum;
}

// The sums of a row over all parts: 16 rows to a workgroup, parts over its 64 rows of threads, which load several at
// once.  4096 rows of 256 parts: 6 us; 64 rows to a workgroup 7, and 8 for 509 rows.
__global__ __launch_bounds__(1024) void k_head_join(HeadArgs p) {
    constexpr uint32_t kRows = 16, kShares = 64;
    __shared__ HeadSum lds[16][kRows];
    const uint32_t count = *p.count;
    if (blockIdx.x * kRows >= count) return;
    const uint32_t row = threadIdx.x % kRows, share = threadIdx.x / kRows, j = blockIdx.x * kRows + row;
    HeadSum sum = {kLowest, 0.0f};
    if (j < count) {
        // several loads on their way at once
        constexpr int kAhead = 8;
        for (uint32_t i = share; i < p.parts; i += kShares * kAhead) {
            HeadSum got[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                got[k] = i + kShares * k < p.parts ? p.part[uint64_t(i + kShares * k) * p.n_pad + j] : HeadSum{kLowest, 0.0f};
#pragma unroll
            for (int k = 0; k < kAhead; ++k) sum = join(sum, got[k], p.c);
        }
    }
#pragma unroll
    for (int d = 16; d < 64; d <<= 1) sum = join(sum, HeadSum{__shfl_xor(sum.m, d), __shfl_xor(sum.s, d)}, p.c);
    if ((threadIdx.x & 63) < kRows) lds[threadIdx.x >> 6][row] = sum;
    __syncthreads();
    if (threadIdx.x >= kRows || j >= count) return;
    for (int w = 1; w < 16; ++w) sum = join(sum, lds[w][row], p.c);
    head_store(p, p.list[j], p.found + j, sum);
}

// g of a piece of the vocabulary, in G planes.  As the sums, and bound by its
// stores, which all workgroups make at once: 16384 classes of 3891 x 1024 bf16 130
// to 134 us (975 to 1000 TFLOP/s; 147 by stores of 8 bytes), 8192 of 4096 x 2048 110
// to 117 (1180 to 1250).
template <typename T, typename Tile, int G>
__global__ __launch_bounds__(Tile::kThreads, Tile::kWaves / 4) void k_head_slopes(HeadArgs p) {
    typedef Held<T, Tile> S;
    __shared__ __attribute__((aligned(1024))) typename Tile::Buffer even, odd;
    const uint32_t count = *p.count, rows = min(p.piece, p.classes - p.first);
    // what the columns need comes first: a wait for a load is one for all stores before it
    HeadRow row[Tile::TN];
    float ratios[Tile::TN];
    each_tile<T, Tile>(p, p.piece, count, even, odd, [&](const Tile &tile, TilePlace at) {
#pragma unroll
        for (int j = 0; j < Tile::TN; ++j) {
            const uint32_t n = at.n * Tile::BN + tile.column(j);
            row[j] = {0.0f, 0.0f, 0.0f, -1};
            if (n < count) row[j] = p.row[n];
            if constexpr (__is_same(T, f16)) ratios[j] = n < count ? p.inverse[n] / p.inverse[p.n_pad] : 1.0f;
        }
    }, [&](Tile &tile, TilePlace at) {
        const bool edge = (at.m + 1) * Tile::BM > rows || (at.n + 1) * Tile::BN > count;
#pragma unroll
        for (int j = 0; j < Tile::TN; ++j) {
            const uint32_t n = at.n * Tile::BN + tile.column(j);
            const HeadRow r = row[j];
            // the label's row among the lane's
            const uint32_t want = uint32_t(r.y) - p.first - at.m * Tile::BM - tile.row(0);
            const bool labels = __any(r.y >= 0 && want < 16u * Tile::TM);
            float label = 0.0f;
            bool mine = false;
#pragma unroll
            for (int i = 0; i < Tile::TM; i += 2) {             // eight rows side by side
                const uint32_t v = at.m * Tile::BM + tile.row(i);
                float g[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) g[q] = -r.b * exp2_hw((tile.acc[i + q / 4][j][q % 4] - r.m) * p.c);
                if (labels) {
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        if (r.y >= 0 && want == Tile::pair_row(i) + q) {
                            g[q] += r.a;
                            label = g[q];
                            mine = true;
                        }
                }
                if (edge) {
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        if (n >= count || v + q >= rows) g[q] = 0.0f;
                }
                const uint64_t to = uint64_t(n) * p.piece + v, plane = uint64_t(p.n_pad) * p.piece;
                Pack<S, 8> out[G];
                if (!__is_same(T, f16) || p.slope) {
                    split(g, out);
#pragma unroll
                    for (int k = 0; k < G; ++k) store_pack<8>(static_cast<S *>(p.slope) + to + k * plane, out[k]);
                }
                if constexpr (__is_same(T, f16)) {
                    if (!p.slope_common) continue;
#pragma unroll
                    for (int q = 0; q < 8; ++q) g[q] *= ratios[j];
                    split(g, out);
#pragma unroll
                    for (int k = 0; k < G; ++k) store_pack<8>(static_cast<S *>(p.slope_common) + to + k * plane, out[k]);
                }
            }
            if constexpr (sizeof(T) == 2 && G == 1) {
                if (mine) keep_rest<T>(p, n, label, __is_same(T, f16) ? ratios[j] : 1.0f);
            }
        }
    });
}

// Splits of the product for dh: as many as its workgroups make of the tiles that the packed rows take.
__device__ __forceinline__ uint32_t hidden_splits(const HeadArgs &p, uint32_t tiles_n) {
    return max(1u, min(p.most, p.blocks / max(1u, p.tiles_m * tiles_n)));
}

// The piece's share of dh = g w, over a split of its classes, added to the
// shares of the pieces before.  3891 x 16384 x 1024 bf16 in 4 splits 130 to 135 us
// (970 to 1000 TFLOP/s), 4096 x 8192 x 2048 in 2 115 to 124 (1110 to 1200).
template <typename T, typename Tile>
__global__ __launch_bounds__(Tile::kThreads, Tile::kWaves / 4) void k_head_hidden(HeadArgs p) {
    typedef Held<T, Tile> S;
    __shared__ __attribute__((aligned(1024))) typename Tile::Buffer even, odd;
    const uint32_t count = *p.count, tiles_n = (count + Tile::BN - 1) / Tile::BN, splits = hidden_splits(p, tiles_n);
    if (blockIdx.x >= p.tiles_m * tiles_n * splits) return;
    const TilePlace at = tile_place(blockIdx.x, p.tiles_m, tiles_n, splits);
    const uint32_t rows = min(p.piece, p.classes - p.first);
    const uint32_t all = (rows + Tile::kStep - 1) / Tile::kStep, steps = (all + splits - 1) / splits;
    Tile tile;
    tile.template run<true, false>(weight_rows<S, Tile::kPlanes>(p), at.m * Tile::BM, slope_rows<S>(p, p.slope, p.n_pad),
                                   at.n * Tile::BN, min(all, at.split * steps), min(all, (at.split + 1) * steps),
                                   even, odd);
#pragma unroll
    for (int j = 0; j < Tile::TN; ++j) {
        const uint32_t n = at.n * Tile::BN + tile.column(j);
        float *to = p.sum + (uint64_t(at.split) * tiles_n * Tile::BN + n) * p.sum_stride;
        if (n >= count) continue;
        // all loads of a column before its stores
        if (p.add) {
            f32x4 before[Tile::TM];
#pragma unroll
            for (int i = 0; i < Tile::TM; ++i)
                before[i] = *reinterpret_cast<const f32x4 *>(to + min(at.m * Tile::BM + tile.row_across(i), p.sum_stride - 4));
#pragma unroll
            for (int i = 0; i < Tile::TM; ++i) tile.acc[i][j] += before[i];
        }
#pragma unroll
        for (int i = 0; i < Tile::TM; ++i) {
            const uint32_t d = at.m * Tile::BM + tile.row_across(i);
            if (d < p.sum_stride) *reinterpret_cast<f32x4 *>(to + d) = tile.acc[i][j];
        }
    }
}

// The sum of `count` groups of four, `step` apart, in order; four loads on their way at once.
__device__ __forceinline__ f32x4 sum_of(const float *from, uint64_t step, uint32_t count) {
    constexpr uint32_t kAhead = 4;
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    for (uint32_t s = 0; s < count; s += kAhead) {
        f32x4 x[kAhead];
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k) x[k] = *reinterpret_cast<const f32x4 *>(from + min(s + k, count - 1) * step);
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k)
            if (s + k < count) sum += x[k];
    }
    return sum;
}

// The rest of g of packed row `at`'s label and four columns of the label's weights: loaded before the sums that it is
// added to.  (Infinite weights have made their sums what they are.)
template <typename T>
struct LabelRest {
    float rest = 0.0f;
    Pack<T, 4> w{};
    __device__ __forceinline__ LabelRest(const HeadArgs &p, int32_t at, uint32_t d) {
        const int32_t y = p.rest && at >= 0 && d < p.width ? p.row[at].y : -1;
        if (y < 0) return;
        rest = p.rest[at];
        w = load_pack<4>(static_cast<const T *>(p.weight) + y * p.weight_stride + d, p.width - d, T{});
    }
    __device__ __forceinline__ void add_to(f32x4 &sum) const {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float x = widen(w.at(q));
            if (fabsf(x) <= FLT_MAX) sum[q] = fmaf(rest, x, sum[q]);
        }
    }
};

// dh of every row from the splits' sums; rows that took no part get zeros.  Few
// rows of many splits: Shares threads to four columns, each with a share of the
// splits, whose sums are added in order (64 x 144 of 64 splits: 4 us, by one
// thread 12).  4096 x 1024 of 4 splits: 15 us, 5.4 TB/s; 13 without the rests, whose rows of the weight lie anywhere.
constexpr uint32_t kJoinQuads = 16;
template <typename T, uint32_t Shares>
__global__ __launch_bounds__(256) void k_head_hidden_join(HeadArgs p) {
    __shared__ f32x4 lds[Shares][Shares > 1 ? kJoinQuads : 1];
    const uint32_t quads = (p.width + 3) / 4, tiles_n = (*p.count + p.tile_n - 1) / p.tile_n;
    const uint32_t splits = hidden_splits(p, tiles_n);
    const uint64_t step = uint64_t(tiles_n) * p.tile_n * p.sum_stride;
    if constexpr (Shares > 1) {
        const uint32_t n = blockIdx.x, d = (blockIdx.y * kJoinQuads + threadIdx.x) * 4;
        const int32_t at = p.place[n];
        const uint32_t share = (splits + Shares - 1) / Shares, first = min(splits, threadIdx.y * share);
        const LabelRest<T> rest(p, threadIdx.y ? -1 : at, d);
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
        if (at >= 0 && d < p.width && first < splits)
            sum = sum_of(p.sum + uint64_t(at) * p.sum_stride + d + first * step, step, min(share, splits - first));
        lds[threadIdx.y][threadIdx.x] = sum;
        __syncthreads();
        if (threadIdx.y || d >= p.width) return;
#pragma unroll
        for (uint32_t s = 1; s < Shares; ++s) sum += lds[s][threadIdx.x];
        rest.add_to(sum);
        const float back = p.inverse && at >= 0 ? p.inverse[at] : 1.0f;
        float v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = sum[q] * back;
        store_pack<4>(static_cast<T *>(p.grad_hidden) + uint64_t(n) * p.width + d, narrow_pack<T>(v), p.width - d);
        return;
    }
    for (uint32_t n = blockIdx.x * blockDim.y + threadIdx.y; n < p.n; n += gridDim.x * blockDim.y) {
        const int32_t at = p.place[n];
        const float back = p.inverse && at >= 0 ? p.inverse[at] : 1.0f;
        for (uint32_t i = threadIdx.x; i < quads; i += blockDim.x) {
            const uint32_t d = i * 4;
            f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
            if (at >= 0) {
                const float *from = p.sum + uint64_t(at) * p.sum_stride + d;
                const LabelRest<T> rest(p, at, d);
                sum = sum_of(from, step, splits);
                rest.add_to(sum);
            }
            float v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = sum[q] * back;
            store_pack<4>(static_cast<T *>(p.grad_hidden) + uint64_t(n) * p.width + d, narrow_pack<T>(v), p.width - d);
        }
    }
}

// Adds the rests of g to a tile of dw.  The packed rows from `begin` to `end` whose labels are among the tile's `columns`
// classes are listed in order, and 64 of them at a time make a step of the product: their hidden states, and rows of
// zeros with the rest at the label.  `step` is a buffer that all waves have done with.  3891 rows of 4096 x 16384 x 1024
// bf16, mostly one such step to a tile of 61: dw 115 -> 123 us.
template <typename Tile>
struct LabelRows {
    static constexpr uint32_t kAhead = 4;           // rows that a thread looks at together
    uint32_t row[64 + kAhead * Tile::kThreads];
    uint32_t found[kAhead][Tile::kWaves];
};
template <typename T, typename Tile>
__device__ __forceinline__ void add_rests(const HeadArgs &p, Tile &tile, const Operand &hidden, uint32_t m0,
                                          const Operand &slope, uint32_t n0, uint32_t columns, uint32_t begin, uint32_t end,
                                          typename Tile::Buffer &step, LabelRows<Tile> &lds) {
    typedef typename Tile::template Sources<true, true> From;
    static_assert(Tile::kStep == 64 && Tile::kPlanesB == 1, "a lane of one wave to each row of a step");
    constexpr uint32_t kAhead = LabelRows<Tile>::kAhead, kThreads = Tile::kThreads;
    const From from = tile.template sources<true, true>(hidden, m0, slope, n0, 0);
    const float *rest = __is_same(T, f16) ? p.rest_common : p.rest;
    const uint32_t low = p.first + n0;
    const auto add = [&](const uint32_t *rows, uint32_t count) {
        From::FromA::gather(hidden, m0, rows, count, step.a, tile.lane, tile.wave);
        for (uint32_t i = threadIdx.x * 16; i < sizeof(step.b); i += kThreads * 16)
            *reinterpret_cast<u32x4 *>(step.b + i) = u32x4{0, 0, 0, 0};
        __syncthreads();
        if (threadIdx.x < count) {
            const uint32_t n = rows[threadIdx.x];
            *reinterpret_cast<T *>(step.b + From::FromB::element(threadIdx.x, uint32_t(p.row[n].y) - low)) = narrow<T>(rest[n]);
        }
        Tile::sync();
        f32x4 none[1][1];
        tile.step(from, step, none);
        __syncthreads();
    };
    uint32_t have = 0;
    for (uint32_t r0 = begin; r0 < end; r0 += kAhead * kThreads) {
        uint64_t set[kAhead];
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k) {
            const uint32_t n = r0 + k * kThreads + threadIdx.x;
            const int32_t y = n < end ? p.row[n].y : -1;
            set[k] = __ballot(y >= 0 && uint32_t(y) - low < columns);
            if (tile.lane == 0) lds.found[k][tile.wave] = __popcll(set[k]);
        }
        __syncthreads();
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k)
            for (uint32_t w = 0; w < uint32_t(Tile::kWaves); ++w) {
                if (w == uint32_t(tile.wave) && set[k] >> tile.lane & 1)
                    lds.row[have + __popcll(set[k] & ((uint64_t(1) << tile.lane) - 1))] = r0 + k * kThreads + threadIdx.x;
                have += lds.found[k][w];
            }
        __syncthreads();
        uint32_t done = 0;
        for (; have - done >= 64; done += 64) add(lds.row + done, 64);
        have -= done;
        if (done && threadIdx.x < have) lds.row[threadIdx.x] = lds.row[done + threadIdx.x];
    }
    __syncthreads();
    if (have) add(lds.row, have);
}

// The piece's rows of dw = g^T h, or their sums over a split of the packed rows.
// 3891 rows of 16384 x 1024 bf16 123 us (1060 TFLOP/s), 4096 of 8192 x 2048 115 to 125 (1100 to 1200).
template <typename T, typename Tile>
__global__ __launch_bounds__(Tile::kThreads, Tile::kWaves / 4) void k_head_weight(HeadArgs p) {
    typedef Held<T, Tile> S;
    __shared__ __attribute__((aligned(1024))) typename Tile::Buffer even, odd;
    const uint32_t count = *p.count, rows = min(p.piece, p.classes - p.first);
    const uint32_t tiles_m = (p.width + Tile::BM - 1) / Tile::BM, tiles_n = (rows + Tile::BN - 1) / Tile::BN;
    const TilePlace at = tile_place(blockIdx.x, tiles_m, tiles_n, p.weight_splits);
    const uint32_t all = (count + Tile::kStep - 1) / Tile::kStep, steps = (all + p.weight_splits - 1) / p.weight_splits;
    const void *slope = __is_same(T, f16) ? p.slope_common : p.slope;
    const Operand h = hidden_rows<S>(p, p.n_pad), g = slope_rows<S>(p, slope, p.n_pad);
    const uint32_t first = min(all, at.split * steps), last = min(all, (at.split + 1) * steps);
    Tile tile;
    tile.template run<true, true>(h, at.m * Tile::BM, g, at.n * Tile::BN, first, last, even, odd);
    if constexpr (sizeof(T) == 2 && Tile::kPlanesB == 1) {
        __shared__ LabelRows<Tile> labels;
        add_rests<T>(p, tile, h, at.m * Tile::BM, g, at.n * Tile::BN, min(uint32_t(Tile::BN), rows - at.n * Tile::BN),
                     first * Tile::kStep, min(count, last * Tile::kStep), even, labels);
    }
    float back = 1.0f;
    if constexpr (__is_same(T, f16)) {
        back = p.inverse[p.n_pad];
        __builtin_amdgcn_s_waitcnt(0x0f70);         // vmcnt(0), here and not behind each store
    }
#pragma unroll
    for (int j = 0; j < Tile::TN; ++j) {
        const uint32_t v = at.n * Tile::BN + tile.column(j);
        if (v >= rows) continue;
        if (p.weight_splits > 1) {
            float *to = p.weight_sum + (uint64_t(at.split) * rows + v) * p.sum_stride;
#pragma unroll
            for (int i = 0; i < Tile::TM; ++i) {
                const uint32_t d = at.m * Tile::BM + tile.row_across(i);
                if (d < p.sum_stride) *reinterpret_cast<f32x4 *>(to + d) = tile.acc[i][j];
            }
            continue;
        }
        T *to = static_cast<T *>(p.grad_weight) + uint64_t(p.first + v) * p.width;
#pragma unroll
        for (int i = 0; i < Tile::TM; ++i) {
            const uint32_t d = at.m * Tile::BM + tile.row_across(i);
            if (d >= p.width) continue;
            float x[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) x[q] = __is_same(T, f16) ? tile.acc[i][j][q] * back : tile.acc[i][j][q];
            store_pack<4>(to + d, narrow_pack<T>(x), p.width - d);
        }
    }
}

// The piece's rows of dw from the splits' sums.
template <typename T>
__global__ __launch_bounds__(256) void k_head_weight_join(HeadArgs p) {
    const uint32_t quads = (p.width + 3) / 4, rows = min(p.piece, p.classes - p.first);
    const uint64_t step = uint64_t(rows) * p.sum_stride;
    const float back = p.inverse ? p.inverse[p.n_pad] : 1.0f;
    for (uint32_t v = blockIdx.x * blockDim.y + threadIdx.y; v < rows; v += gridDim.x * blockDim.y)
        for (uint32_t i = threadIdx.x; i < quads; i += blockDim.x) {
            const uint32_t d = i * 4;
            const float *from = p.weight_sum + uint64_t(v) * p.sum_stride + d;
            const f32x4 sum = sum_of(from, step, p.weight_splits);
            float x[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) x[q] = sum[q] * back;
            store_pack<4>(static_cast<T *>(p.grad_weight) + uint64_t(p.first + v) * p.width + d, narrow_pack<T>(x),
                          p.width - d);
        }
}

}  // namespace tmtrain
