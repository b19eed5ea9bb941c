// bias.h -- a learned bias by buckets of distance, from a distance field or
// from the positions of queries and keys on a grid, and the gradient of its
// table (include/tm_train.h).
#pragma once

#include "train_common.h"

namespace tmtrain {

constexpr int kBiasMaxDim = 8;
constexpr uint32_t kMaxBuckets = 256;

// Where distances come from.  kField: an array; the others: positions.
enum Source { kFieldF32, kFieldI32, kOffset, kEuclid, kTaxicab, kChess };

struct BiasSource {
    const void *field;
    const float *edges;
    int32_t source, ndim;
    uint32_t buckets, span;                // span: buckets rounded up to a power of two
    uint32_t positions;                    // of one sample
    Div32 div_key;                         // key positions
    Div32 div_q[kBiasMaxDim], div_k[kBiasMaxDim];   // positions of the axes behind each axis
    int32_t offset[kBiasMaxDim];           // first query's coordinates
    float sampling[kBiasMaxDim];
};

struct BiasArgs {
    BiasSource src;
    const void *table;
    const void *add;
    void *out;
    uint32_t heads, batch, field_batch;    // field_batch: samples with buckets of their own
    int32_t table_type;                    // tm_dtype
    uint32_t head_share, row;              // heads of a workgroup, and their floats per bucket in LDS
    uint32_t batch_share, batch_shares;    // samples of a workgroup (relative)
    uint32_t tiles;                        // of 256 threads' positions, over all samples with buckets of their own
    Div32 div_tiles;                       // those of one sample
};

struct BiasGradArgs {
    BiasSource src;
    const void *grad;
    void *out;
    float *partial;                        // [splits][heads / 16][tile_rows][16]
    uint32_t heads, batch, field_batch;
    int32_t table_type;
    uint32_t splits, tile_rows;
    uint32_t units;                        // shares of the batch x steps of positions, or groups of samples
    uint32_t batch_share;                  // samples of a share: those of a unit have the same buckets; or of a group
    Div32 div_steps;                       // steps of a sample; or positions of one
};

// The float32 distance of position p of sample b.  Every operation rounds by
// itself: a contraction could move a distance over an edge.
__device__ __forceinline__ float distance_at(const BiasSource &s, uint32_t b, uint32_t p) {
#pragma clang fp contract(off)
    if (s.source == kFieldF32) return static_cast<const float *>(s.field)[uint64_t(b) * s.positions + p];
    if (s.source == kFieldI32) return float(static_cast<const int32_t *>(s.field)[uint64_t(b) * s.positions + p]);
    uint32_t q = s.div_key.div(p), k = p - q * s.div_key.d;
    if (s.source == kOffset) return float(int32_t(k) - (int32_t(q) + s.offset[0]));
    float sum = 0.0f;
    for (int a = 0; a < s.ndim; ++a) {
        const uint32_t qa = s.div_q[a].div(q), ka = s.div_k[a].div(k);
        q -= qa * s.div_q[a].d;
        k -= ka * s.div_k[a].d;
        const float v = float(int32_t(ka) - (int32_t(qa) + s.offset[a])) * s.sampling[a];
        // the first term is added to 0, which changes nothing
        if (s.source == kEuclid)
            sum = sum + v * v;
        else if (s.source == kTaxicab)
            sum = sum + fabsf(v);
        else
            sum = fmaxf(sum, fabsf(v));
    }
    return s.source == kEuclid ? sqrtf(sum) : sum;
}

// Edges in LDS, padded with NaN to one less than a power of two: no distance
// is at or past a NaN, so the count never leaves 0 .. buckets - 1, whatever the
// edges hold.
__device__ __forceinline__ void stage_edges(float *lds, const BiasSource &s, uint32_t threads) {
    for (uint32_t i = threadIdx.x; i + 1 < s.span; i += threads)
        lds[i] = i + 1 < s.buckets ? s.edges[i] : __uint_as_float(0x7fc00000u);
}
// Number of edges <= d, one bit of it a step.
__device__ __forceinline__ uint32_t bucket_of(const float *lds, uint32_t span, float d) {
    uint32_t k = 0;
    for (uint32_t step = span >> 1; step; step >>= 1)
        if (lds[k + step - 1] <= d) k += step;
    return k;
}

__device__ __forceinline__ float table_at(const void *table, int32_t type, uint64_t i) {
    if (type == 6) return static_cast<const float *>(table)[i];
    if (type == 5) return widen(static_cast<const bf16 *>(table)[i]);
    return widen(static_cast<const f16 *>(table)[i]);
}
__device__ __forceinline__ void table_put(void *table, int32_t type, uint64_t i, float v) {
    if (type == 6) static_cast<float *>(table)[i] = v;
    else if (type == 5) static_cast<bf16 *>(table)[i] = narrow<bf16>(v);
    else static_cast<f16 *>(table)[i] = narrow<f16>(v);
}

// ---------------------------------------------------------------------------
// Forward.  One thread owns V consecutive positions: it finds their buckets
// once and writes every head and sample of its workgroup's share with them,
// 16 bytes a store.  Workgroups go on to further positions rather than lay out
// the table again.  It lies in LDS by bucket, four heads to a 16-byte
// read, so a position's address serves all heads.  Bound by the bytes of add
// and out (bf16 scores of 2 x 16 x 2048 x 2048: 537 MB in 101 us, 5.3 TB/s; a
// field of 32 x 512^2 for 4 heads 168 MB in 33 us, 5.1 TB/s; float32 2 x 155 x
// 240 x 237, 3 heads, 282 MB in 56 us, 5.0 TB/s).
// ---------------------------------------------------------------------------
constexpr int kBiasThreads = 256;

template <typename T, int V>
__global__ void __launch_bounds__(kBiasThreads) k_bias(BiasArgs a) {
    extern __shared__ float lds[];
    float *const table = lds;                              // [buckets][row], row = heads of the share, padded
    float *const edges = lds + a.src.buckets * a.row;
    const uint32_t share = blockIdx.y / a.batch_shares, bshare = blockIdx.y - share * a.batch_shares;
    const uint32_t h0 = share * a.head_share, hn = min(a.head_share, a.heads - h0);
    stage_edges(edges, a.src, kBiasThreads);
    for (uint32_t i = threadIdx.x; i < a.src.buckets * a.row; i += kBiasThreads) {
        const uint32_t k = i / a.row, h = i - k * a.row;
        table[i] = h < hn ? table_at(a.table, a.table_type, uint64_t(k) * a.heads + h0 + h) : 0.0f;
    }
    __syncthreads();
    for (uint32_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        // field: samples are tiles' own; relative: this share of the batch, all with the same buckets
        const uint32_t fb = a.field_batch > 1 ? a.div_tiles.div(tile) : 0;
        const uint32_t own = ((tile - fb * a.div_tiles.d) * kBiasThreads + threadIdx.x) * V;
        if (own >= a.src.positions) continue;
        // the last thread reads whole loads, further back, and writes what is its own
        const uint32_t p0 = min(own, a.src.positions - V), skip = own - p0;
        float d[V];
        if (a.src.source == kFieldF32 || a.src.source == kFieldI32) {
            const Pack<int32_t, V> raw = load_pack<V>(static_cast<const int32_t *>(a.src.field) + uint64_t(fb) * a.src.positions + p0);
#pragma unroll
            for (int j = 0; j < V; ++j)
                d[j] = a.src.source == kFieldF32 ? __int_as_float(raw.at(j)) : float(raw.at(j));
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) d[j] = distance_at(a.src, fb, p0 + j);
        }
        uint32_t at[V];
#pragma unroll
        for (int j = 0; j < V; ++j) at[j] = bucket_of(edges, a.src.span, d[j]) * a.row;
        const uint32_t b0 = fb + bshare * a.batch_share;
        const uint32_t b1 = a.field_batch > 1 ? fb + 1 : min(a.batch, b0 + a.batch_share);
        for (uint32_t h = 0; h < hn; h += 4) {
            float4 v[V];
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = *reinterpret_cast<const float4 *>(table + at[j] + h);
            for (uint32_t b = b0; b < b1; ++b) {
                const uint64_t row = (uint64_t(b) * a.heads + h0 + h) * a.src.positions + p0;
                Pack<T, V> extra[4];
                if (a.add) {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (h + r < hn) extra[r] = load_pack<V>(static_cast<const T *>(a.add) + row + uint64_t(r) * a.src.positions);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if (h + r >= hn) break;
                    float out[V];
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float x = r == 0 ? v[j].x : r == 1 ? v[j].y : r == 2 ? v[j].z : v[j].w;
                        out[j] = a.add ? x + widen(extra[r].at(j)) : x;
                    }
                    store_own<V>(static_cast<T *>(a.out) + row + uint64_t(r) * a.src.positions, narrow_pack<T, V>(out), skip);
                }
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Gradient of the table: out[k][h] = sum over positions of [bucket = k] g[h],
// a matrix product with a matrix of ones and zeros.  A wave takes 16 heads and
// a step of positions: its lanes find the buckets and leave them in LDS; the
// ones and zeros are made in registers as the first operand of 16x16x32
// products (16 buckets x 32 positions; a "one" is 2.0, a single bit of either
// 16-bit format, and the sum is halved at the end) and the gradients are the
// second.  They are loaded 256 bytes of a head to 16 lanes, the next step's
// while one is added up, and change hands through LDS, since the operand wants
// 8 positions of one head in a lane.  (Loaded as the operand lies, with
// neighbouring lanes in different heads, every lane is an access of its own:
// 86 us instead of 81 for 2 x 16 x 2048 x 2048, 53 instead of 40 for 32 x 4 x
// 512^2.)  Fewer than 9 heads leave loads over for more positions.  Sums are
// float32 in the accumulators, in an order fixed by the sizes.  float32
// gradients are cut into three bf16 pieces of 8 bits, which lose nothing.  The
// first pieces have sums of their own: those of gradients of about one size are
// exact for 2^16 of them, and the others' are so much smaller that their
// roundings do not add up (32 x 2^20 positions of 0.1: off by 5 of 2^-24, in one
// sum by 166).
//
// With 16 heads bound by the gradients' bytes (bf16 2 x 16 x 2048 x 2048: 268 MB
// in 83 us, 3.2 TB/s right after the forward pass has written as much; without
// the loads 30 us), with few heads by the search of the buckets and the making
// of ones and zeros, 1.3 instructions a position and lane (bf16 32 x 4 x 512^2:
// 101 MB in 40 us; float32 4 x 3 x 990 x 990: 47 MB in 26 us).
//
// Each workgroup leaves its sums in the workspace; k_bias_join adds them up.
// Columns of heads that are not there hold anything and are not used.
//
// Zero times an infinity or NaN spreads it over the buckets of its tile.  A
// workgroup that finds a sum which is not finite goes over its positions once
// more (`clean`): what is not finite is noted by bucket and head and counts as
// zero.  bf16 and float32 gradients are taken a quarter as large, so that twice
// the largest one is in range.  Sums that were finite stay as they were.  (The
// first case with an infinity in each head: 122 us.)
//
// Samples of fewer positions than a load holds (Few) go into a step one behind
// the other, as many as fit, and are loaded element by element (131072 samples
// of one position, 16 heads, bf16: 4.7 MB in 13 us, bound by latency).
// ---------------------------------------------------------------------------
constexpr int kGradThreads = 512;
constexpr int kGradWaves = kGradThreads / kWave;
// Bytes of a head in LDS, a 16-bit value a position or three pieces; rows begin in different banks.
template <typename T>
constexpr int kGradRow = (sizeof(T) == 4 ? 3 * 128 : 256) + 16;

// Positions of a load of 256 bytes, and of a step with `Blocks` blocks of four heads.
template <typename T>
constexpr uint32_t kGradLoad = 256 / sizeof(T);
template <typename T, int Blocks>
constexpr uint32_t kGradStep = kGradLoad<T> * (4 / Blocks);

// A gradient of the second pass: 0 where it is not finite, with what it is left in `what`.
enum { kPlusInf = 1, kMinusInf = 2, kNaN = 4 };
template <typename T>
__device__ __forceinline__ T cleaned(T g, uint32_t &what) {
    const float x = widen(g);
    what = x != x ? kNaN : x == INFINITY ? kPlusInf : x == -INFINITY ? kMinusInf : 0;
    if (what) return T{};
    if constexpr (__is_same(T, f16)) return g;
    else return narrow<T>(0.25f * x);
}
__device__ __forceinline__ float noted(uint32_t what, float sum) {
    if (what & kNaN || (what & (kPlusInf | kMinusInf)) == (kPlusInf | kMinusInf)) return __uint_as_float(0x7fc00000u);
    return what == kPlusInf ? INFINITY : what == kMinusInf ? -INFINITY : sum;
}

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <bool B, typename X, typename Y>
struct Select { typedef X type; };
template <typename X, typename Y>
struct Select<false, X, Y> { typedef Y type; };

// Two ones (0x4000) or zeros: is either half of w the bucket?
__device__ __forceinline__ uint32_t match2(uint32_t w, uint32_t bucket2) {
    const u16x2 x = __builtin_bit_cast(u16x2, w ^ bucket2);
    const u16x2 one = {1, 1};
    const u16x2 hit = __builtin_elementwise_sub_sat(one, x);
    return __builtin_bit_cast(uint32_t, u16x2(hit << u16x2{14, 14}));
}

__device__ __forceinline__ f32x4 product(bf16, u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
}
__device__ __forceinline__ f32x4 product(f16, u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0,
                                                  0);
}

// One step of positions, for the samples of one share of the batch; Few: a
// group of samples from b0 on, as one.
struct Unit {
    uint32_t field, first;                 // sample of the distances, first position
    uint32_t b0, b1;
};
template <bool Few>
__device__ __forceinline__ Unit unit_at(const BiasGradArgs &a, uint32_t unit, uint32_t step) {
    if constexpr (Few) return {0, 0, unit * a.batch_share, unit * a.batch_share + 1};
    Unit u;
    const uint32_t share = a.div_steps.div(unit);
    u.field = a.field_batch > 1 ? share : 0;
    u.first = (unit - share * a.div_steps.d) * step;
    u.b0 = share * a.batch_share;
    u.b1 = min(a.batch, u.b0 + a.batch_share);
    return u;
}

// Tiles: buckets / 16, rounded up to a power of two.  Blocks of four heads: 1, 2 or 4 (Few: 4).
// Two workgroups to a CU, four waves to a SIMD, as far as the sums leave registers for it.
template <typename T, int Tiles, int Blocks, bool Few>
__global__ void __launch_bounds__(kGradThreads,
                                  !Few && (Tiles <= 4 || (Tiles == 8 && Blocks == 2 && sizeof(T) == 2)) ? 4 : 1)
    k_bias_grad(BiasGradArgs a) {
    constexpr uint32_t L = kGradLoad<T>, Step = kGradStep<T, Blocks>;
    constexpr int V = 16 / sizeof(T);
    __shared__ float edges[kMaxBuckets];
    __shared__ __align__(16) uint16_t ids[kGradWaves][Step];
    constexpr int Row = kGradRow<T>, Rows = 4 * Blocks * Row;
    // the rows of every wave, and after them the sums
    __shared__ __align__(16) char shared[kGradWaves * Rows > Tiles * 1024 ? kGradWaves * Rows : Tiles * 1024];
    __shared__ uint32_t odd[Tiles * 64];                   // [bucket][head], a byte each: what is not finite
    __shared__ uint32_t finite[kGradWaves];                // are a wave's sums?
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t col = lane & 15, group = lane >> 4;     // operand: row or column, block of 8 positions
    const uint32_t h0 = blockIdx.y * 16;
    stage_edges(edges, a.src, kGradThreads);
    __syncthreads();
    const uint32_t splat = col * 0x10001u;
    char *const mine = shared + wave * Rows;
    // Load i: head 4 (i % Blocks) + group, 16 bytes at piece col of 256-byte run
    // i / Blocks.  No load is behind a branch, where it would be waited for:
    // heads that are not there read the last one, and pieces past the end the
    // last V positions, whose doubles no bucket takes.
    const uint32_t last = a.src.positions - V;
    const auto fetch = [&](Pack<T, V> (&x)[4], const Unit &u, uint32_t b) __attribute__((always_inline)) {
        if constexpr (Few) {
            static_assert(Blocks == 4);
            // below 2^26 elements from the group's first
            const uint32_t b0 = __builtin_amdgcn_readfirstlane(u.b0), have = min(a.batch_share, a.batch - b0);
            const T *const g = static_cast<const T *>(a.grad) + uint64_t(b0) * a.heads * a.src.positions;
            uint32_t at_j[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const uint32_t s = a.div_steps.div(col * V + j), p = col * V + j - s * a.src.positions;
                at_j[j] = min(s, have - 1) * a.heads * a.src.positions + p;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t at_i = min(h0 + 4 * i + group, a.heads - 1) * a.src.positions;
                Pack<T, V> r{};
#pragma unroll
                for (int j = 0; j < V; ++j) r.put(j, g[at_j[j] + at_i]);
                x[i] = r;
            }
            return;
        }
        const T *g = static_cast<const T *>(a.grad) + uint64_t(b) * a.heads * a.src.positions;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t head = min(h0 + 4 * (i % Blocks) + group, a.heads - 1);
            x[i] = load_pack<V>(g + uint64_t(head) * a.src.positions + min(u.first + (i / Blocks) * L + col * V, last));
        }
    };
    constexpr int Lows = sizeof(T) == 4 ? Tiles : 1;
    f32x4 acc[Tiles] = {}, low[Lows] = {};                 // of the first pieces, of the others
    uint32_t present[Step / 64];                           // tiles with a bucket of 64 positions, a bit each
    const auto find = [&](const Unit &u) __attribute__((always_inline)) {
#pragma unroll
        for (uint32_t s = 0; s < Step / 64; ++s) {
            const uint32_t i = s * 64 + lane;
            uint32_t k;
            if constexpr (Few) {
                const uint32_t sample = a.div_steps.div(i), b = min(u.b0 + sample, a.batch - 1);
                k = bucket_of(edges, a.src.span,
                              distance_at(a.src, a.field_batch > 1 ? b : 0, i - sample * a.src.positions));
                if (sample >= a.batch_share || u.b0 + sample >= a.batch) k = 0xffffu;
            } else {
                const uint32_t piece = u.first + i / V * V, p = min(piece, last) + i % V;
                k = bucket_of(edges, a.src.span, distance_at(a.src, u.field, p));
                if (p < piece) k = 0xffffu;
            }
            ids[wave][i] = uint16_t(k);
            present[s] = 0;
#pragma unroll
            for (int t = 0; t < Tiles; ++t) present[s] |= uint32_t(__any(k >> 4 == uint32_t(t))) << t;
        }
    };
    const auto hand_over = [&](const Pack<T, V> &y, uint32_t row) __attribute__((always_inline)) {
        char *const to = mine + row * Row;
        if constexpr (sizeof(T) == 4) {
            uint32_t cut[4][3];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float g = __uint_as_float(y.w[e]);
                cut[e][0] = y.w[e] & 0xffff0000u;
                const float rest = g - __uint_as_float(cut[e][0]);
                cut[e][1] = __float_as_uint(rest) & 0xffff0000u;
                cut[e][2] = __float_as_uint(rest - __uint_as_float(cut[e][1]));
            }
#pragma unroll
            for (int c = 0; c < 3; ++c)
                *reinterpret_cast<u32x2 *>(to + c * 128 + col * 8) =
                    u32x2{__builtin_amdgcn_perm(cut[1][c], cut[0][c], 0x07060302u),
                          __builtin_amdgcn_perm(cut[3][c], cut[2][c], 0x07060302u)};
        } else {
            *reinterpret_cast<u32x4 *>(to + col * 16) = u32x4{y.w[0], y.w[1], y.w[2], y.w[3]};
        }
    };
    const auto add_up = [&](int run) __attribute__((always_inline)) {
        const char *const operand = mine + (col & (4 * Blocks - 1)) * Row + group * 16;
#pragma unroll
        for (uint32_t q = 0; q < L / 32; ++q) {
            u32x4 w = *reinterpret_cast<const u32x4 *>(&ids[wave][run * L + q * 32 + group * 8]);
            w ^= splat;
            constexpr int Parts = sizeof(T) == 4 ? 3 : 1;
            u32x4 part[Parts];
#pragma unroll
            for (int c = 0; c < Parts; ++c) part[c] = *reinterpret_cast<const u32x4 *>(operand + c * 128 + q * 64);
#pragma unroll
            for (int t = 0; t < Tiles; ++t) {
                if (Tiles > 1 && !(present[(run * L + q * 32) / 64] >> t & 1)) continue;
                u32x4 one;
#pragma unroll
                for (int j = 0; j < 4; ++j) one[j] = match2(w[j], t * 0x00100010u);
                typedef typename Select<sizeof(T) == 4, bf16, T>::type P;
#pragma unroll
                for (int c = 0; c < Parts; ++c) {
                    f32x4 &sum = c ? low[t % Lows] : acc[t];
                    sum = product(P{}, one, part[c], sum);
                }
            }
        }
    };
    // lane holds rows group * 4 .. + 3 of column col of each tile; waves add in turn
    float(*const sums)[16] = reinterpret_cast<float(*)[16]>(shared);
    const auto join_waves = [&]() __attribute__((always_inline)) {
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < Tiles * 256; i += kGradThreads) sums[i >> 4][i & 15] = 0.0f;
        __syncthreads();
        for (uint32_t w = 0; w < kGradWaves; ++w) {
            if (w == wave) {
#pragma unroll
                for (int t = 0; t < Tiles; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sums[t * 16 + group * 4 + r][col] += 0.5f * acc[t][r];
            }
            __syncthreads();
        }
    };
    uint32_t at = blockIdx.x * kGradWaves + wave;          // below 2^31 + 4096
    Unit u{};
    Pack<T, V> x[4];
    if (at < a.units) {
        u = unit_at<Few>(a, at, Step);
        fetch(x, u, u.b0);
    }
    while (at < a.units) {
        find(u);
        at += gridDim.x * kGradWaves;
        const Unit v = at < a.units ? unit_at<Few>(a, at, Step) : Unit{};
        for (uint32_t b = u.b0; b < u.b1; ++b) {
            // runs of 256 bytes change hands one after the other
#pragma unroll
            for (int run = 0; run < 4 / Blocks; ++run) {
                wave_sync();
#pragma unroll
                for (int i = 0; i < Blocks; ++i) hand_over(x[run * Blocks + i], 4 * i + group);
                wave_sync();
                if (run == 4 / Blocks - 1) {
                    // the gradients of the step after this one are on their way meanwhile
                    if (b + 1 < u.b1) fetch(x, u, b + 1);
                    else if (at < a.units) fetch(x, v, v.b0);
                }
                add_up(run);
            }
        }
        wave_sync();
        u = v;
    }
    const auto add_low = [&]() __attribute__((always_inline)) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int t = 0; t < Tiles; ++t) {
                acc[t] += low[t];
                low[t] = f32x4{};
            }
        }
    };
    add_low();
    bool whole = true;
#pragma unroll
    for (int t = 0; t < Tiles; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) whole &= __builtin_isfinite(acc[t][r]);
    whole = __all(whole);
    if (lane == 0) finite[wave] = whole;
    join_waves();
    float *const out = a.partial + (uint64_t(blockIdx.x) * gridDim.y + blockIdx.y) * (Tiles * 256);
    for (uint32_t i = threadIdx.x; i < Tiles * 256; i += kGradThreads) out[i] = sums[i >> 4][i & 15];
    uint32_t all = 1;
#pragma unroll
    for (int w = 0; w < kGradWaves; ++w) all &= finite[w];
    if (all) return;

    // once more, without what is not finite
    for (uint32_t i = threadIdx.x; i < Tiles * 64; i += kGradThreads) odd[i] = 0;
#pragma unroll
    for (int t = 0; t < Tiles; ++t) acc[t] = f32x4{};
    __syncthreads();
    for (at = blockIdx.x * kGradWaves + wave; at < a.units; at += gridDim.x * kGradWaves) {
        u = unit_at<Few>(a, at, Step);
        find(u);
        for (uint32_t b = u.b0; b < u.b1; ++b) {
            fetch(x, u, b);
#pragma unroll
            for (int run = 0; run < 4 / Blocks; ++run) {
                wave_sync();
#pragma unroll
                for (int i = 0; i < Blocks; ++i) {
                    Pack<T, V> y = x[run * Blocks + i];
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const uint32_t k = ids[wave][run * L + col * V + j], row = 4 * i + group;
                        uint32_t what;
                        y.put(j, cleaned(y.at(j), what));
                        if (what && k != 0xffffu) atomicOr(&odd[k * 4 + row / 4], what << (8 * (row & 3)));
                    }
                    hand_over(y, 4 * i + group);
                }
                wave_sync();
                add_up(run);
            }
        }
        wave_sync();
    }
    add_low();
    join_waves();
    for (uint32_t i = threadIdx.x; i < Tiles * 256; i += kGradThreads) {
        const float sum = sums[i >> 4][i & 15];
        const uint32_t row = i & (4 * Blocks - 1);
        if (!__builtin_isfinite(out[i]))
            out[i] = noted(odd[(i >> 4) * 4 + row / 4] >> (8 * (row & 3)) & 0xffu, __is_same(T, f16) ? sum : 4.0f * sum);
    }
}

// One workgroup per bucket and 16 heads: thread (slice, head) adds every 16th
// workgroup's sum, then the slices are added.
__global__ void __launch_bounds__(256) k_bias_join(BiasGradArgs a) {
    __shared__ float part[256];
    const uint32_t col = threadIdx.x & 15, slice = threadIdx.x >> 4;
    const uint32_t k = blockIdx.x, h0 = blockIdx.y * 16;
    const float *p = a.partial + (uint64_t(blockIdx.y) * a.tile_rows + k) * 16 + col;
    float sum = 0.0f;
    const uint64_t step = uint64_t(gridDim.y) * a.tile_rows * 16;
    for (uint32_t w = slice; w < a.splits; w += 16 * 8) {  // eight loads in flight
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = w + 16 * u < a.splits ? p[(w + 16 * u) * step] : 0.0f;
#pragma unroll
        for (int u = 0; u < 8; ++u) sum += v[u];
    }
    part[threadIdx.x] = sum;
    __syncthreads();
    for (uint32_t w = 8; w; w >>= 1) {
        if (slice < w) part[threadIdx.x] += part[threadIdx.x + 16 * w];
        __syncthreads();
    }
    sum = part[col];
    if (slice == 0 && h0 + col < a.heads) table_put(a.out, a.table_type, uint64_t(k) * a.heads + h0 + col, sum);
}

}  // namespace tmtrain
