// rows_host.hip -- C-ABI of layer norm and of the lookup of a table's rows:
// argument checks, choice of kernel and launches (declared in
// include/tm_train.h).

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "host_common.h"

#include "embedding.h"
#include "norm.h"

using namespace tmtrain;

namespace {

template <int L_, int P_>
struct Held { static constexpr int L = L_, P = P_; };

// fn(threads to a row, pieces of 16 bytes of each): as few threads as hold a
// row in up to four pieces.  Returns UNSUPPORTED, without a call, for rows that
// no workgroup holds.
template <typename F>
int by_held_row(uint64_t pieces, F fn) {
    if (pieces <= 16) return fn(Held<16, 1>{});
    if (pieces <= 32) return fn(Held<16, 2>{});
    if (pieces <= 64) return fn(Held<64, 1>{});
    if (pieces <= 128) return fn(Held<64, 2>{});
    if (pieces <= 256) return fn(Held<64, 4>{});
    if (pieces <= 512) return fn(Held<256, 2>{});
    if (pieces <= 1024) return fn(Held<256, 4>{});
    if (pieces <= 2048) return fn(Held<1024, 2>{});
    if (pieces <= 4096) return fn(Held<1024, 4>{});
    return TM_ERR_UNSUPPORTED;
}

struct NormShape {
    uint64_t rows, width, size, pieces, x_bytes;
};

int check_norm(const void *x, int dtype, int64_t rows, int64_t width, int64_t stride, const void *params, int param_dtype,
               NormShape &s) {
    if (rows < 0 || width < 1 || stride < 0) return TM_ERR_SHAPE;
    if (!float_type(dtype) || (params && !float_type(param_dtype))) return TM_ERR_DTYPE;
    if (uint64_t(rows) >= kLimit || uint64_t(width) > (uint64_t(1) << 24)) return TM_ERR_TOO_LARGE;
    if (rows > 1 && uint64_t(stride) > (uint64_t(1) << 56) / uint64_t(rows)) return TM_ERR_TOO_LARGE;
    s.rows = uint64_t(rows);
    s.width = uint64_t(width);
    s.size = float_bytes(dtype);
    s.pieces = ceil_div(s.width * s.size, 16);
    s.x_bytes = rows ? ((s.rows - 1) * uint64_t(stride) + s.width) * s.size : 0;
    return rows && !x ? TM_ERR_NULL : TM_OK;
}

void norm_args(const NormShape &s, const void *x, int64_t stride, const void *weight, int param_dtype, NormArgs &a) {
    a.x = x;
    a.stride = uint64_t(stride);
    a.rows = uint32_t(s.rows);
    a.width = uint32_t(s.width);
    a.weight = weight;
    a.param_type = param_dtype;
    a.share = float(1.0 / double(s.width));
}

// Workgroups for rows that none holds: enough for the chip, since a grid has less than 2^32 threads.
dim3 long_grid(const NormShape &s) { return dim3(uint32_t(std::min<uint64_t>(s.rows, 2 * kFill))); }

// Workgroups whose sums for dw and db are added afterwards.
uint64_t norm_parts(const NormShape &s) {
    uint64_t parts = 0;
    const int rc = by_held_row(s.pieces, [&](auto held) {
        constexpr int L = decltype(held)::L;
        parts = std::min<uint64_t>(ceil_div(s.rows, L > 256 ? 1 : 256 / L), L > 256 ? 256 : 768);
        return int(TM_OK);
    });
    if (rc != TM_OK) parts = std::min<uint64_t>(s.rows, ceil_div(kFill, ceil_div(s.pieces, 256)));
    return parts;
}

}  // namespace

extern "C" int tm_layer_norm(const void *x, int dtype, int64_t rows, int64_t width, int64_t stride, const void *weight,
                             const void *bias, int param_dtype, double eps, void *out, float *out_stats,
                             hipStream_t stream) {
    NormShape s{};
    const int rc = check_norm(x, dtype, rows, width, stride, weight ? weight : bias, param_dtype, s);
    if (rc != TM_OK) return rc;
    if (!std::isfinite(eps) || !std::isfinite(float(eps)) || !(float(eps) > 0.0f)) return TM_ERR_SAMPLING;
    if (s.rows == 0) return TM_OK;
    if (!out) return TM_ERR_NO_OUTPUT;
    const uint64_t params = s.width * float_bytes(param_dtype);
    const Range in[] = {{x, s.x_bytes}, {weight, params}, {bias, params}};
    const Range outs[] = {{out, s.rows * s.width * s.size}, {out_stats, s.rows * 8}};
    if (aliased(in, outs)) return TM_ERR_ALIAS;
    NormArgs a{};
    norm_args(s, x, stride, weight, param_dtype, a);
    a.bias = bias;
    a.eps = float(eps);
    a.y = out;
    a.stats = reinterpret_cast<float2 *>(out_stats);
    return by_type(dtype, [&](auto t) {
        using T = decltype(t);
        const int rc = by_held_row(s.pieces, [&](auto held) {
            constexpr int L = decltype(held)::L, P = decltype(held)::P;
            const uint64_t blocks = ceil_div(s.rows, L > 256 ? 1 : 256 / L);
            return launch(k_norm<T, L, P>, dim3(uint32_t(std::min<uint64_t>(blocks, 2 * kFill))), dim3(L > 256 ? L : 256),
                          0, stream, a);
        });
        if (rc != TM_ERR_UNSUPPORTED) return rc;
        return launch(k_norm_long<T>, long_grid(s), dim3(kLongThreads), 0, stream, a);
    });
}

extern "C" size_t tm_layer_norm_grad_workspace_size(int dtype, int64_t rows, int64_t width) {
    NormShape s{};
    const void *some = reinterpret_cast<const void *>(uintptr_t(4096));
    if (check_norm(some, dtype, rows, width, 0, nullptr, 0, s) != TM_OK || s.rows == 0) return 0;
    return norm_parts(s) * 2 * ceil_div(s.width, 8) * 8 * 4;
}

extern "C" int tm_layer_norm_grad(const void *x, int dtype, int64_t rows, int64_t width, int64_t stride,
                                  const void *weight, int param_dtype, const float *stats, const void *up, void *out_x,
                                  void *out_weight, void *out_bias, void *workspace, size_t workspace_bytes,
                                  hipStream_t stream) {
    NormShape s{};
    const bool sums = out_weight || out_bias;
    const int rc = check_norm(x, dtype, rows, width, stride, sums || weight ? x : nullptr, param_dtype, s);
    if (rc != TM_OK) return rc;
    if (!out_x && !sums) return TM_ERR_NO_OUTPUT;
    if (s.rows && (!stats || !up)) return TM_ERR_NULL;
    const size_t need = sums ? tm_layer_norm_grad_workspace_size(dtype, rows, width) : 0;
    if (need && (!workspace || workspace_bytes < need || uintptr_t(workspace) % 16)) return TM_ERR_WORKSPACE;
    const uint64_t params = s.width * float_bytes(param_dtype), all = s.rows * s.width * s.size;
    const Range in[] = {{x, s.x_bytes}, {weight, params}, {stats, s.rows * 8}, {up, all}};
    const Range outs[] = {{out_x, all}, {out_weight, params}, {out_bias, params}, {need ? workspace : nullptr, need}};
    if (aliased(in, outs)) return TM_ERR_ALIAS;
    if (s.rows == 0 && !sums) return TM_OK;
    NormArgs a{};
    norm_args(s, x, stride, weight, param_dtype, a);
    a.stats = reinterpret_cast<float2 *>(const_cast<float *>(stats));
    a.up = up;
    a.dx = out_x;
    a.dw = out_weight;
    a.db = out_bias;
    a.part = static_cast<float *>(workspace);
    a.part_stride = uint32_t(ceil_div(s.width, 8) * 8);
    a.parts = s.rows ? uint32_t(norm_parts(s)) : 0;
    if (s.rows) {
        const int rc = by_type(dtype, [&](auto t) {
            using T = decltype(t);
            const int rc = by_held_row(s.pieces, [&](auto held) {
                constexpr int L = decltype(held)::L, P = decltype(held)::P;
                const uint64_t blocks = sums ? a.parts : std::min<uint64_t>(ceil_div(s.rows, L > 256 ? 1 : 256 / L), 2 * kFill);
                return launch(sums ? k_norm_grad<T, L, P, true> : k_norm_grad<T, L, P, false>, dim3(uint32_t(blocks)),
                              dim3(L > 256 ? L : 256), 0, stream, a);
            });
            if (rc != TM_ERR_UNSUPPORTED) return rc;
            if (out_x) {
                const int rc = launch(k_norm_long_grad<T>, long_grid(s), dim3(kLongThreads), 0, stream, a);
                if (rc != TM_OK) return rc;
            }
            if (!sums) return int(TM_OK);
            a.share_rows = uint32_t(ceil_div(s.rows, a.parts));
            a.parts = uint32_t(ceil_div(s.rows, a.share_rows));
            return launch(k_norm_columns<T>, dim3(uint32_t(ceil_div(s.pieces, 256)), a.parts), dim3(256), 0, stream, a);
        });
        if (rc != TM_OK) return rc;
    }
    if (!sums) return TM_OK;
    return launch(k_norm_join, dim3(uint32_t(ceil_div(s.width, 64)), 2), dim3(1024), 0, stream, a);
}

// ---------------------------------------------------------------------------
// Rows of a table.
// ---------------------------------------------------------------------------
namespace {

struct EmbeddingShape {
    uint64_t rows, width, count, size, token_bytes, pieces;
};

int check_embedding(int dtype, int64_t rows, int64_t width, const void *tokens, int token_dtype, int64_t count,
                    double scale, EmbeddingShape &s) {
    if (rows < 1 || width < 1 || count < 0) return TM_ERR_SHAPE;
    if (!float_type(dtype)) return TM_ERR_DTYPE;
    if (token_dtype != TM_DTYPE_U8 && token_dtype != TM_DTYPE_I32 && token_dtype != TM_DTYPE_I64) return TM_ERR_DTYPE;
    if (!std::isfinite(scale) || !std::isfinite(float(scale))) return TM_ERR_SAMPLING;
    if (uint64_t(rows) >= kLimit - 1 || uint64_t(count) >= kLimit || uint64_t(width) > (uint64_t(1) << 24))
        return TM_ERR_TOO_LARGE;
    if (count && !tokens) return TM_ERR_NULL;
    s.rows = uint64_t(rows);
    s.width = uint64_t(width);
    s.count = uint64_t(count);
    s.size = float_bytes(dtype);
    s.token_bytes = token_dtype == TM_DTYPE_U8 ? 1 : token_dtype == TM_DTYPE_I32 ? 4 : 8;
    s.pieces = ceil_div(s.width * s.size, 16);
    return TM_OK;
}

// Rows up to which a workgroup to a range of them sorts faster than tiles and digits: the whole gradient of 16384 tokens
// of 262144 x 8 takes 35 us and by digits 48, of 1000003 rows 85 and 71.
constexpr uint64_t kRangeRows = uint64_t(1) << 19;

// A workgroup's threads along a row, the rest for other rows.
dim3 row_block(uint64_t pieces) {
    const uint32_t x = uint32_t(std::min<uint64_t>(256, std::max<uint64_t>(8, pieces)));
    return dim3(x, 256 / x);
}

void embedding_args(const EmbeddingShape &s, const void *tokens, double scale, EmbeddingArgs &a) {
    a.token = tokens;
    a.token_bytes = int32_t(s.token_bytes);
    a.count = uint32_t(s.count);
    a.rows = uint32_t(s.rows);
    a.width = uint32_t(s.width);
    a.scale = float(scale);
}

// Layout of the gradient's workspace; returns its size.
uint64_t embedding_room(const EmbeddingShape &s, void *at, EmbeddingArgs &a, uint32_t &digits) {
    uint32_t bits = 1;
    while (s.rows >> bits) ++bits;                      // of the token that stands for none, `rows`
    digits = (bits + 8) / 9;
    const uint32_t each = (bits + digits - 1) / digits;
    a.values = 1u << each;
    a.tiles = uint32_t(ceil_div(s.count, kSortTile));
    // some 2048 chunks of 16 numbers at least
    a.chunk = 16;
    while (uint64_t(a.chunk) * 2048 < s.count) a.chunk *= 2;
    a.chunks = uint32_t(ceil_div(s.count, a.chunk));
    a.part_stride = uint32_t(ceil_div(s.width, 8) * 8);
    uint64_t used = 0;
    const auto take = [&](uint64_t words) {
        void *p = at ? static_cast<char *>(at) + used : nullptr;
        used += ceil_div(words * 4, 256) * 256;
        return p;
    };
    for (int i = 0; i < 2; ++i) {
        a.key[i] = static_cast<uint32_t *>(take(s.count));
        a.number[i] = static_cast<uint32_t *>(take(s.count));
    }
    a.digits = static_cast<uint32_t *>(take(uint64_t(a.tiles) * a.values));
    a.total = static_cast<uint32_t *>(take(a.values));
    a.part = static_cast<float *>(take(uint64_t(a.chunks) * 2 * a.part_stride));
    return used;
}

}  // namespace

extern "C" int tm_embedding(const void *table, int dtype, int64_t rows, int64_t width, int64_t stride,
                            const void *tokens, int token_dtype, int64_t count, double scale, void *out,
                            hipStream_t stream) {
    EmbeddingShape s{};
    const int rc = check_embedding(dtype, rows, width, tokens, token_dtype, count, scale, s);
    if (rc != TM_OK) return rc;
    if (stride < 0) return TM_ERR_SHAPE;
    if (rows > 1 && uint64_t(stride) > (uint64_t(1) << 56) / uint64_t(rows)) return TM_ERR_TOO_LARGE;
    if (s.count == 0) return TM_OK;
    if (!table) return TM_ERR_NULL;
    if (!out) return TM_ERR_NO_OUTPUT;
    const Range in[] = {{table, ((s.rows - 1) * uint64_t(stride) + s.width) * s.size}, {tokens, s.count * s.token_bytes}};
    const Range outs[] = {{out, s.count * s.width * s.size}};
    if (aliased(in, outs)) return TM_ERR_ALIAS;
    EmbeddingArgs a{};
    embedding_args(s, tokens, scale, a);
    a.table = table;
    a.stride = uint64_t(stride);
    a.y = out;
    // four pieces to a thread, unless that leaves CUs idle
    const uint64_t total = s.count * s.pieces;
    a.share = uint32_t(std::max<uint64_t>(1, (total >= 4 * 256 * kFill ? 1024 : 256) / s.pieces));
    a.div_pieces = Div32::make(uint32_t(s.pieces));
    const dim3 grid(uint32_t(std::min<uint64_t>(ceil_div(s.count, a.share), 1 << 20)), uint32_t(ceil_div(s.pieces, 4096)));
    return by_type(dtype, [&](auto t) { return launch(k_embedding<decltype(t)>, grid, dim3(256), 0, stream, a); });
}

extern "C" size_t tm_embedding_grad_workspace_size(int64_t rows, int64_t width, int64_t count) {
    EmbeddingShape s{};
    EmbeddingArgs a{};
    uint32_t digits;
    const void *some = reinterpret_cast<const void *>(uintptr_t(4096));
    if (check_embedding(TM_DTYPE_F32, rows, width, some, TM_DTYPE_I32, count, 1.0, s) != TM_OK || s.count == 0) return 0;
    return embedding_room(s, nullptr, a, digits);
}

extern "C" int tm_embedding_grad(const void *tokens, int token_dtype, int64_t count, const void *up, int dtype,
                                 int64_t rows, int64_t width, double scale, void *out_grad, void *workspace,
                                 size_t workspace_bytes, hipStream_t stream) {
    EmbeddingShape s{};
    const int rc = check_embedding(dtype, rows, width, tokens, token_dtype, count, scale, s);
    if (rc != TM_OK) return rc;
    if (!out_grad) return TM_ERR_NO_OUTPUT;
    if (s.count && !up) return TM_ERR_NULL;
    const size_t need = tm_embedding_grad_workspace_size(rows, width, count);
    if (need && (!workspace || workspace_bytes < need || uintptr_t(workspace) % 16)) return TM_ERR_WORKSPACE;
    const uint64_t bytes = s.rows * s.width * s.size;
    const Range in[] = {{tokens, s.count * s.token_bytes}, {up, s.count * s.width * s.size}};
    const Range outs[] = {{out_grad, bytes}, {need ? workspace : nullptr, need}};
    if (aliased(in, outs)) return TM_ERR_ALIAS;
    if (s.count == 0) {
        const FillArgs f{out_grad, bytes};
        return launch(k_fill_zeros<256>, dim3(uint32_t(std::min<uint64_t>(4 * kFill, ceil_div(bytes, 4096)))), dim3(256), 0,
                      stream, f);
    }
    EmbeddingArgs a{};
    uint32_t digits;
    embedding_args(s, tokens, scale, a);
    embedding_room(s, workspace, a, digits);
    a.up = up;
    a.grad = out_grad;
    a.from = -1;
    const uint32_t each = uint32_t(__builtin_ctz(a.values));
    if (s.count <= kRangeTokens && s.rows < kRangeRows) {
        // a workgroup to every CU, until each has kSortMost rows
        a.values = 1;
        while (a.values < kSortMost && a.values * 256 <= s.rows) a.values *= 2;
        const int rc = launch(s.token_bytes == 1   ? k_sort_range<uint8_t>
                              : s.token_bytes == 4 ? k_sort_range<uint32_t>
                                                   : k_sort_range<uint64_t>,
                              dim3(uint32_t(s.rows / a.values + 1)), dim3(1024), ceil_div(s.count, 1024) * 4096, stream, a);
        if (rc != TM_OK) return rc;
        a.from = 0;
    } else {
        for (uint32_t d = 0; d < digits; ++d, a.shift += each) {
            int rc = launch(k_sort_count, dim3(a.tiles), dim3(256), 0, stream, a);
            if (rc == TM_OK && a.tiles > kSortFew)
                rc = launch(k_sort_tiles, dim3(uint32_t(ceil_div(a.values, 4))), dim3(256), 0, stream, a);
            if (rc == TM_OK) rc = launch(k_sort_move, dim3(a.tiles), dim3(256), 0, stream, a);
            if (rc != TM_OK) return rc;
            a.from = a.from == 0 ? 1 : 0;
        }
    }
    a.sorted_key = a.key[a.from];
    a.sorted_number = a.number[a.from];
    const dim3 block = row_block(s.pieces);
    const uint32_t across = uint32_t(ceil_div(s.pieces, block.x));
    a.sum_blocks = uint32_t(ceil_div(a.chunks, block.y));
    const uint32_t clear = uint32_t(ceil_div(s.rows, kClearRows));
    return by_type(dtype, [&](auto t) {
        using T = decltype(t);
        const int rc = launch(k_embedding_sums<T>, dim3(a.sum_blocks + clear, across), block, 0, stream, a);
        if (rc != TM_OK || a.chunks == 1) return rc;
        return launch(k_embedding_join<T>, dim3(a.chunks, across), block, 256 * 16 / sizeof(T) * 4, stream, a);
    });
}
