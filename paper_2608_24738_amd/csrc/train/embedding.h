// embedding.h -- kernels of the lookup of a table's rows by given tokens, and
// of the table's gradient (tm_embedding in include/tm_train.h):
//     y_n = scale T[k_n],   dT[v] = scale sum over n with k_n = v of g_n.
//
// Both are bound by memory: y is written and its rows read once; g is read and
// dT written once.  For the gradient the numbers n are sorted by token, equal
// tokens by rising n, so that every row's sum has one order.  The sorted
// numbers are cut into chunks of one length: a row whose tokens lie within a
// chunk is summed and stored there, one that runs on over several leaves a sum
// in each, which are added in order; so the tokens' frequencies do not matter.
// Rows without a token are found by search among the sorted ones.
#pragma once

#include "label.h"

namespace tmtrain {

constexpr uint32_t kSortTile = 1024;            // tokens that a workgroup sorts at once
constexpr uint32_t kSortMost = 512;             // values of a digit
constexpr uint32_t kRangeTokens = 32768;        // that a workgroup lists at most
constexpr uint32_t kSortFew = 64;               // tiles whose counts each workgroup adds up by itself
constexpr uint32_t kClearRows = 64;             // rows of the table that a workgroup looks for

struct EmbeddingArgs {
    const void *table, *token;
    uint64_t stride;            // of the table's rows, elements
    int32_t token_bytes;
    uint32_t count, rows, width;
    float scale;
    void *y;
    uint32_t share;             // rows of a workgroup
    Div32 div_pieces;           // 16-byte pieces of a row
    // gradient
    const void *up;
    void *grad;
    uint32_t *key[2], *number[2];   // tokens (`rows` for one outside the table) and their numbers, two of each
    uint32_t *digits;           // [tile][values]: how often a tile has each value of the digit
    uint32_t *total;            // [values]: how often all have, where there are many tiles
    uint32_t tiles, values;
    uint32_t shift;             // of the digit at hand
    int32_t from;               // which of the two is read; -1: the tokens themselves
    const uint32_t *sorted_key, *sorted_number;
    float *part;                // [chunks][2][part_stride]
    uint32_t part_stride, chunk, chunks, sum_blocks;
};

// A workgroup copies p.share rows, its threads side by side over all their
// pieces.  16384 x 1024 bf16: 10.4 us, 5.2 TB/s; 60001 x 257 float32, no row of
// which is aligned: 14.3 us, 4.3 TB/s (threads along one row: 21).
template <typename T>
__global__ __launch_bounds__(256) void k_embedding(EmbeddingArgs p) {
    constexpr int V = 16 / sizeof(T);
    const uint32_t pieces = p.div_pieces.d;
    const uint64_t step = uint64_t(gridDim.x) * p.share;
    for (uint64_t n0 = uint64_t(blockIdx.x) * p.share; n0 < p.count; n0 += step) {
        const uint32_t total = uint32_t(min(uint64_t(p.share), p.count - n0)) * pieces;
        for (uint32_t i = blockIdx.y * 256 + threadIdx.x; i < total; i += gridDim.y * 256) {
            const uint32_t r = p.div_pieces.div(i), c = (i - r * pieces) * V;
            const uint64_t n = n0 + r;
            const int32_t k = load_label(p.token, p.token_bytes, n, p.rows);
            float v[V] = {};
            if (k >= 0) {
                const Pack<T, V> x = load_pack<V>(static_cast<const T *>(p.table) + k * p.stride + c, p.width - c, T{});
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = widen(x.at(j)) * p.scale;
            }
            store_pack<V>(static_cast<T *>(p.y) + n * p.width + c, narrow_pack<T>(v), p.width - c);
        }
    }
}

// ---------------------------------------------------------------------------
// Sorting: many tokens a digit at a time from the lowest, few in one launch.
// ---------------------------------------------------------------------------

__device__ __forceinline__ uint32_t sort_key(const EmbeddingArgs &p, uint32_t i) {
    if (p.from >= 0) return p.key[p.from][i];
    const int32_t k = load_label(p.token, p.token_bytes, i, p.rows);
    return k < 0 ? p.rows : uint32_t(k);
}

// How often each value of the digit occurs in a tile.
__global__ __launch_bounds__(256) void k_sort_count(EmbeddingArgs p) {
    __shared__ uint32_t found[kSortMost];
    for (uint32_t i = threadIdx.x; i < p.values; i += 256) found[i] = 0;
    __syncthreads();
    const uint32_t first = blockIdx.x * kSortTile, last = min(p.count, first + kSortTile);
    for (uint32_t i = first + threadIdx.x; i < last; i += 256)
        atomicAdd(&found[sort_key(p, i) >> p.shift & (p.values - 1)], 1u);
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < p.values; i += 256) p.digits[uint64_t(blockIdx.x) * p.values + i] = found[i];
}

// Many tiles: a wave to a value turns the tiles' counts into sums over the tiles before, and their total.
__global__ __launch_bounds__(256) void k_sort_tiles(EmbeddingArgs p) {
    const uint32_t lane = threadIdx.x & 63, value = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (value >= p.values) return;
    uint32_t before = 0;
    for (uint32_t t0 = 0; t0 < p.tiles; t0 += 64) {
        const uint32_t t = t0 + lane;
        const uint32_t x = t < p.tiles ? p.digits[uint64_t(t) * p.values + value] : 0;
        uint32_t up = x;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t o = __shfl_up(up, d);
            if (lane >= uint32_t(d)) up += o;
        }
        if (t < p.tiles) p.digits[uint64_t(t) * p.values + value] = before + up - x;
        before += __shfl(up, 63);
    }
    if (lane == 0) p.total[value] = before;
}

// Moves a tile's tokens to their places: first those with lower values, then
// those of earlier tiles, then of earlier waves, then of earlier rounds and lower
// lanes.  16 tiles 7.8 us, 59 tiles of two more bits 13: loads, counts and ranks
// wait for one another.
__global__ __launch_bounds__(256) void k_sort_move(EmbeddingArgs p) {
    constexpr uint32_t kWaves = 4, kRounds = kSortTile / 256;
    __shared__ uint32_t place[kSortMost];               // where a value's tokens of this tile begin
    __shared__ uint16_t wave_has[kWaves][kSortMost];    // how many a wave has, then how many before it
    __shared__ uint32_t scan[kWaves];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // a wave has a stretch of the tile and takes 64 of it a round
    const uint32_t first = blockIdx.x * kSortTile + wave * (kSortTile / kWaves);
    uint32_t key[kRounds], rank[kRounds];
#pragma unroll
    for (uint32_t r = 0; r < kRounds; ++r) {
        const uint32_t i = first + r * 64 + lane;
        key[r] = i < p.count ? sort_key(p, i) : 0;
    }
    for (uint32_t i = threadIdx.x; i < kWaves * kSortMost; i += 256) (&wave_has[0][0])[i] = 0;
    // sums over the lower values: two values to a thread, side by side
    uint32_t total[2] = {0, 0}, before[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint32_t v = threadIdx.x * 2 + j;
        if (v >= p.values) continue;
        if (p.tiles > kSortFew) {
            total[j] = p.total[v];
            before[j] = p.digits[uint64_t(blockIdx.x) * p.values + v];
        } else {
#pragma unroll 8
            for (uint32_t t = 0; t < p.tiles; ++t) {
                const uint32_t x = p.digits[t * p.values + v];
                total[j] += x;
                before[j] += t < blockIdx.x ? x : 0;
            }
        }
    }
    uint32_t up = total[0] + total[1];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = __shfl_up(up, d);
        if (lane >= uint32_t(d)) up += o;
    }
    if (lane == 63) scan[wave] = up;
    __syncthreads();
    up -= total[0] + total[1];
    for (uint32_t w = 0; w < wave; ++w) up += scan[w];
    place[threadIdx.x * 2] = up + before[0];
    place[threadIdx.x * 2 + 1] = up + total[0] + before[1];
#pragma unroll
    for (uint32_t r = 0; r < kRounds; ++r) {
        const uint32_t i = first + r * 64 + lane;
        const bool real = i < p.count;
        const uint32_t digit = key[r] >> p.shift & (p.values - 1);
        uint64_t same = __ballot(real);                 // lanes with this lane's digit
        for (uint32_t bit = 1; bit < p.values; bit <<= 1) {
            const uint64_t set = __ballot(digit & bit);
            same &= digit & bit ? set : ~set;
        }
        const uint64_t below = same & ((uint64_t(1) << lane) - 1);
        rank[r] = 0;
        if (real) rank[r] = wave_has[wave][digit] + __popcll(below);
        wave_sync();                                    // every lane has read before the first of each digit writes
        if (real && below == 0) wave_has[wave][digit] = uint16_t(rank[r] + __popcll(same));
        wave_sync();
    }
    __syncthreads();
    for (uint32_t v = threadIdx.x; v < p.values; v += 256) {
        uint32_t sum = 0;
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) {
            const uint32_t x = wave_has[w][v];
            wave_has[w][v] = uint16_t(sum);
            sum += x;
        }
    }
    __syncthreads();
    const int to = p.from == 0 ? 1 : 0;
#pragma unroll
    for (uint32_t r = 0; r < kRounds; ++r) {
        const uint32_t i = first + r * 64 + lane;
        if (i >= p.count) continue;
        const uint32_t digit = key[r] >> p.shift & (p.values - 1);
        const uint32_t at = place[digit] + wave_has[wave][digit] + rank[r];
        p.key[to][at] = key[r];
        p.number[to][at] = p.from < 0 ? i : p.number[p.from][i];
    }
}

// Few tokens: a workgroup to p.values of the table's rows, which reads all tokens,
// counts those of lower rows, lists its own and moves them to their places, first
// by row, then by wave, whose stretches follow one another, then in order.  Bound
// by the instructions of the first pass, some 25 for 64 tokens.  Sums and all of
// 50021 x 8: 64 tokens 13 us, 8192 22, 16384 24, 32768 29 (by tiles and digits 16384
// 38, 32768 43); 16384 times the same token 29.  K: tokens as unsigned numbers,
// of which negative ones are the largest.
template <typename K>
__global__ __launch_bounds__(1024) void k_sort_range(EmbeddingArgs p) {
    constexpr uint32_t kWaves = 16, kAhead = 8;
    static_assert(kRangeTokens * kSortMost <= uint64_t(1) << 32, "a number and a digit in 32 bits");
    extern __shared__ uint32_t list[];                  // numbers and digits, each wave's from its stretch on
    __shared__ uint16_t wave_has[kWaves][kSortMost];    // how many a wave has of a row, then where the next one goes
    __shared__ uint32_t scan[kWaves], lower[kWaves];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, low = blockIdx.x * p.values;
    const uint32_t stretch = (p.count + 1023) / 1024 * 64, first = wave * stretch, last = min(p.count, first + stretch);
    for (uint32_t i = threadIdx.x; i < kWaves * kSortMost; i += 1024) (&wave_has[0][0])[i] = 0;
    uint32_t less = 0, listed = first;
    for (uint32_t i0 = first; i0 < last; i0 += 64 * kAhead) {
        K token[kAhead];
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k)
            token[k] = static_cast<const K *>(p.token)[min(i0 + k * 64 + lane, p.count - 1)];
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k) {
            const uint32_t i = i0 + k * 64 + lane, digit = (token[k] < p.rows ? uint32_t(token[k]) : p.rows) - low;
            if (i < last && int32_t(digit) < 0) ++less;
            const uint64_t set = __ballot(i < last && digit < p.values);
            if (!set) continue;
            if (set >> lane & 1) list[listed + __popcll(set & ((uint64_t(1) << lane) - 1))] = i * kSortMost + digit;
            listed += __popcll(set);
        }
    }
    __syncthreads();
    // fn(number, digit, rank) of what the wave listed; counts it
    const auto each = [&](auto fn) {
        for (uint32_t j = first; j < listed; j += 64) {
            const bool real = j + lane < listed;
            const uint32_t x = list[min(j + lane, listed - 1)], digit = x % kSortMost;
            uint64_t same = __ballot(real);             // lanes with this lane's digit
            if (__any(digit != uint32_t(__builtin_amdgcn_readfirstlane(digit))))
                for (uint32_t bit = 1; bit < p.values; bit <<= 1) {
                    const uint64_t set = __ballot(digit & bit);
                    same &= digit & bit ? set : ~set;
                }
            const uint64_t below = same & ((uint64_t(1) << lane) - 1);
            uint32_t at = 0;
            if (real) at = wave_has[wave][digit] + __popcll(below);
            wave_sync();                                // every lane has read before the first of each digit writes
            if (real && below == 0) wave_has[wave][digit] = uint16_t(at + __popcll(same));
            wave_sync();
            if (real) fn(x / kSortMost, digit, at);
        }
    };
    each([](uint32_t, uint32_t, uint32_t) {});
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) less += __shfl_xor(less, d);
    if (lane == 0) lower[wave] = less;
    __syncthreads();
    uint32_t sum = 0;
    if (threadIdx.x < p.values)
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) sum += wave_has[w][threadIdx.x];
    uint32_t up = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = __shfl_up(up, d);
        if (lane >= uint32_t(d)) up += o;
    }
    if (lane == 63) scan[wave] = up;
    __syncthreads();
    if (threadIdx.x < p.values) {
        up -= sum;
        for (uint32_t w = 0; w < wave; ++w) up += scan[w];
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) {
            const uint32_t x = wave_has[w][threadIdx.x];
            wave_has[w][threadIdx.x] = uint16_t(up);
            up += x;
        }
    }
    __syncthreads();
    uint32_t before = 0;
#pragma unroll
    for (uint32_t w = 0; w < kWaves; ++w) before += lower[w];
    each([&](uint32_t i, uint32_t digit, uint32_t at) {
        p.key[0][before + at] = low + digit;
        p.number[0][before + at] = i;
    });
}

// ---------------------------------------------------------------------------
// Sums.
// ---------------------------------------------------------------------------

// First of n ascending keys that is >= k.
__device__ __forceinline__ uint32_t lower_bound(const uint32_t *key, uint32_t n, uint32_t k) {
    uint32_t lo = 0, hi = n;
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2;
        if (key[mid] < k)
            lo = mid + 1;
        else
            hi = mid;
    }
    return lo;
}

// The chunks' sums, and zeros in the rows without a token.  16384 tokens of 50021
// x 1024 bf16: 22.7 us, 6.1 TB/s; eight rows on their way to a thread.
template <typename T>
__global__ __launch_bounds__(256) void k_embedding_sums(EmbeddingArgs p) {
    constexpr int V = 16 / sizeof(T), kAhead = 8;
    __shared__ uint32_t absent[kClearRows];
    if (blockIdx.x >= p.sum_blocks) {
        const uint32_t v0 = (blockIdx.x - p.sum_blocks) * kClearRows, thread = threadIdx.y * blockDim.x + threadIdx.x;
        const uint32_t rows = min(kClearRows, p.rows - v0);
        if (thread < rows) {
            const uint32_t at = lower_bound(p.sorted_key, p.count, v0 + thread);
            absent[thread] = at == p.count || p.sorted_key[at] != v0 + thread;
        }
        __syncthreads();
        for (uint32_t r = threadIdx.y; r < rows; r += blockDim.y) {
            if (!absent[r]) continue;
            T *to = static_cast<T *>(p.grad) + uint64_t(v0 + r) * p.width;
            for (uint32_t c = (blockIdx.y * blockDim.x + threadIdx.x) * V; c < p.width; c += gridDim.y * blockDim.x * V)
                store_pack<V>(to + c, Pack<T, V>{}, p.width - c);
        }
        return;
    }
    const uint32_t c = (blockIdx.y * blockDim.x + threadIdx.x) * V, chunk = blockIdx.x * blockDim.y + threadIdx.y;
    if (c >= p.width || chunk >= p.chunks) return;
    const uint32_t n = p.width - c;
    const uint32_t first = chunk * p.chunk, last = min(p.count, first + p.chunk);
    const bool begun = first > 0 && p.sorted_key[first - 1] == p.sorted_key[first];
    const bool goes_on = last < p.count && p.sorted_key[last] == p.sorted_key[last - 1];
    float sum[V] = {};
    uint32_t run = first, now = p.sorted_key[first];
    const auto finish = [&](uint32_t end) {
        if (now >= p.rows) return;                      // tokens outside the table
        const bool head = run == first && begun, tail = end == last && goes_on;
        if (head || tail) {
            Pack<float, V> x;
#pragma unroll
            for (int j = 0; j < V; ++j) x.put(j, sum[j]);
            store_pack<V>(p.part + (uint64_t(chunk) * 2 + (head ? 0 : 1)) * p.part_stride + c, x);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) sum[j] *= p.scale;
            store_pack<V>(static_cast<T *>(p.grad) + uint64_t(now) * p.width + c, narrow_pack<T>(sum), n);
        }
    };
    for (uint32_t i0 = first; i0 < last; i0 += kAhead) {
        Pack<T, V> x[kAhead];
        uint32_t key[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const uint32_t i = min(i0 + k, last - 1);
            key[k] = p.sorted_key[i];
            x[k] = load_pack<V>(static_cast<const T *>(p.up) + uint64_t(p.sorted_number[i]) * p.width + c, n, T{});
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (i0 + k >= last) break;
            if (key[k] != now) {
                finish(i0 + k);
                run = i0 + k;
                now = key[k];
#pragma unroll
                for (int j = 0; j < V; ++j) sum[j] = 0.0f;
            }
#pragma unroll
            for (int j = 0; j < V; ++j) sum[j] += widen(x[k].at(j));
        }
    }
    finish(last);
}

// Rows whose tokens run over several chunks (5.4 us for 1024 chunks of 16 numbers): their sums, in the workgroup of
// the first such chunk, added by the rows of threads in shares and then in order.
template <typename T>
__global__ __launch_bounds__(256) void k_embedding_join(EmbeddingArgs p) {
    constexpr int V = 16 / sizeof(T);
    extern __shared__ float lds[];                      // [blockDim.y][blockDim.x][V]
    const uint32_t chunk = blockIdx.x, first = chunk * p.chunk, last = first + p.chunk;
    if (last >= p.count) return;
    const uint32_t k = p.sorted_key[last - 1], next = p.sorted_key[last], before = p.sorted_key[first > 0 ? first - 1 : 0];
    if (k >= p.rows || next != k) return;                                                // nothing runs on
    if (first > 0 && before == k) return;                                                // an earlier chunk's
    // the chunks that begin with the row, a thread to each
    const uint32_t threads = blockDim.x * blockDim.y, thread = threadIdx.y * blockDim.x + threadIdx.x;
    uint32_t chunks = 1;
    for (uint32_t found = threads; found == threads; chunks += found) {
        const uint64_t at = uint64_t(chunk + chunks + thread) * p.chunk;
        found = uint32_t(__syncthreads_count(at < p.count && p.sorted_key[at] == k));
    }
    const uint32_t share = (chunks + blockDim.y - 1) / blockDim.y;
    const uint32_t c = (blockIdx.y * blockDim.x + threadIdx.x) * V;
    float sum[V] = {};
    if (c < p.width) {
        const uint32_t stop = min(chunks, (threadIdx.y + 1) * share);
#pragma unroll 4
        for (uint32_t i = threadIdx.y * share; i < stop; ++i) {
            const Pack<float, V> x = load_pack<V>(p.part + (uint64_t(chunk + i) * 2 + (i == 0 ? 1 : 0)) * p.part_stride + c);
#pragma unroll
            for (int j = 0; j < V; ++j) sum[j] += x.at(j);
        }
    }
    float *mine = lds + (threadIdx.y * blockDim.x + threadIdx.x) * V;
#pragma unroll
    for (int j = 0; j < V; ++j) mine[j] = sum[j];
    __syncthreads();
    if (threadIdx.y || c >= p.width) return;
    for (uint32_t y = 1; y < blockDim.y; ++y)
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += lds[(y * blockDim.x + threadIdx.x) * V + j];
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] *= p.scale;
    store_pack<V>(static_cast<T *>(p.grad) + uint64_t(k) * p.width + c, narrow_pack<T>(sum), p.width - c);
}

}  // namespace tmtrain
