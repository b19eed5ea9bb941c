// head_host.hip -- C-ABI of the log-probabilities from hidden states: argument
// checks, layout of the workspace, choice of kernel and launches (declared in
// include/tm_train.h).

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "head_few.h"
#include "host_common.h"

using namespace tmtrain;

namespace {

constexpr uint64_t kMaxWidth = uint64_t(1) << 20;      // 256 rows fit an offset of 32 bits
constexpr uint64_t kMostRows = uint64_t(1) << 26;       // a grid has 2^32 threads at most: 64 of k_head_join to a row,
constexpr uint64_t kMostClasses = uint64_t(1) << 30;    // 4 of k_few_sums to a class
constexpr uint64_t kPieceBytes = uint64_t(1) << 27;     // of g
constexpr uint64_t kLaidBytes = uint64_t(1) << 30;      // of weights laid out in whole steps
constexpr uint64_t kCus = 256;
constexpr uint64_t kJoinFew = 1 << 16;                  // groups of four columns of dh
constexpr uint64_t kMostSplits = 64;                    // of the product for dh
constexpr uint64_t kPlaneRows = 128;
constexpr uint64_t kNarrowRows = 64;
constexpr uint64_t kSmallRows = uint64_t(1) << 19;       // in groups of 16 to a grid's second dimension
constexpr double kSmallWork = 1 << 28;                  // rows x classes x width

struct HeadShape {
    uint64_t n, classes, width, size;
    uint64_t hidden_bytes, weight_bytes, label_bytes;
};

// Bytes from a matrix's first to the end of its last element, or 0 if it is too long to address.
uint64_t matrix_bytes(uint64_t rows, uint64_t width, uint64_t stride, uint64_t size) {
    if (rows > 1 && stride > (uint64_t(1) << 56) / rows) return 0;
    return ((rows - 1) * stride + width) * size;
}

int check_head(const void *hidden, int dtype, int64_t rows, int64_t classes, int64_t width, int64_t hidden_stride,
               const void *weight, int64_t weight_stride, int label_dtype, const void *labels, double scale,
               HeadShape &s) {
    if (rows < 0 || classes < 1 || width < 1 || hidden_stride < 0 || weight_stride < 0) return TM_ERR_SHAPE;
    if (!float_type(dtype)) return TM_ERR_DTYPE;
    if (labels && label_dtype != TM_DTYPE_U8 && label_dtype != TM_DTYPE_I32 && label_dtype != TM_DTYPE_I64)
        return TM_ERR_DTYPE;
    if (!std::isfinite(scale) || !std::isfinite(float(scale) * kLog2e) || !(float(scale) > FLT_MIN))
        return TM_ERR_SAMPLING;
    if (uint64_t(rows) >= kMostRows || uint64_t(classes) >= kMostClasses || uint64_t(width) > kMaxWidth)
        return TM_ERR_TOO_LARGE;
    s.n = uint64_t(rows);
    s.classes = uint64_t(classes);
    s.width = uint64_t(width);
    s.size = float_bytes(dtype);
    // workgroups of the smallest tiles
    if (ceil_div(s.n, 128) * ceil_div(s.classes, 128) >= kLimit ||
        ceil_div(std::max(s.n, s.classes), 64) * ceil_div(s.width, 128) >= kLimit)
        return TM_ERR_TOO_LARGE;
    s.label_bytes = label_dtype == TM_DTYPE_U8 ? 1 : label_dtype == TM_DTYPE_I32 ? 4 : 8;
    if (s.n == 0) return TM_OK;
    if (!hidden || !weight) return TM_ERR_NULL;
    s.hidden_bytes = matrix_bytes(s.n, s.width, uint64_t(hidden_stride), s.size);
    s.weight_bytes = matrix_bytes(s.classes, s.width, uint64_t(weight_stride), s.size);
    return s.hidden_bytes && s.weight_bytes ? TM_OK : TM_ERR_TOO_LARGE;
}

// A workspace, handed out front to back.
struct Room {
    char *at;
    uint64_t used;
    template <typename T>
    T *take(uint64_t count) {
        T *p = at ? reinterpret_cast<T *>(at + used) : nullptr;
        used += ceil_div(count * sizeof(T), 256) * 256;
        return p;
    }
};

uint64_t whole_tiles(uint64_t n) { return ceil_div(n, kTilePad) * kTilePad; }

// Whether single waves compute the logits sooner than tiles do, by microseconds: theirs go with the work in groups of
// rows, those of tiles, while CUs are without one, with the steps of k, and rows of no whole 128 bytes are laid out first.
// Forward passes: of 512 x 1024 x 512, 2^28, bf16 13 us and by tiles 18, float32 23 and 35; of 120 x 2504 x 3920 bf16 44
// and 61; of 64 x 1500 x 4000 float32 36 and 143; of 24 x 50021 x 777 bf16 36 and 54; of 1024 x 1024 x 512 bf16 20 and 17.
double small_work(const HeadShape &s) {
    return double(ceil_div(s.n, kFewRows) * kFewRows) * double(s.classes) * double(s.width) / kSmallWork;
}
double tile_rounds(const HeadShape &s) {
    return double(ceil_div(s.width, 64)) *
           std::max<uint64_t>(1, ceil_div(s.n, 128) * ceil_div(s.classes, 128) / (2 * kCus));
}
double laying_time(const HeadShape &s) { return 3 + double(s.classes * s.width * s.size) * 0.4e-6; }
bool small(const HeadShape &s) {
    const bool wide = s.size == 4;
    const double work = small_work(s), steps = tile_rounds(s) * (wide ? 2.2 : 0.65);
    const double laying = s.width * s.size % 128 ? laying_time(s) : 0;
    return s.n <= kSmallRows && (work <= 1 || 3 + work * (wide ? 17 : 10) <= 12 + steps + laying);
}
bool few(const HeadShape &s) { return s.n <= kFewRows || small(s); }
// The gradient of 16-bit operands reads and writes them at the tiles' pace from nine rows on (32768 x 1024 bf16: 8 rows
// 52 us and by tiles 70, 9 rows 71 and 67; float32 keeps to the kernels for few up to 16).
bool few_grad(const HeadShape &s) { return s.n <= (s.size == 4 ? kFewRows : 8); }

// Which 1 << shift waves share a row's columns in the kernels for few: as many as a workgroup has, unless the chip is
// full without (forward pass of 2514 x 14 x 3200 bf16 9 us, by single waves 13; 85 x 80 x 1926 float32 10 and 29).
uint32_t few_shift(const HeadShape &s) {
    const uint64_t waves = ceil_div(s.classes, 16) * ceil_div(s.n, kFewRows);
    uint32_t shift = 0;
    while (1 << shift < kFewWaves && waves << shift < 4 * kCus) ++shift;
    return shift;
}

// The same for g of the gradient, where either way packs the rows; weights that single waves would save from being laid
// out are those of a gradient without dh, which reads them so.  Whole gradients: of 300 x 513 x 512 bf16 37 us and by tiles
// 40, of 300 x 1024 x 1024 47 and 44, of 64 x 1500 x 4000 52 and 82, of 24 x 50021 x 777 135 and 119; float32, whose
// larger tiles of up to kPlaneRows rows take twice as long, of 100 x 5000 x 2047 175 and 233, of 300 x 1024 x 1024 77 and
// 80, of 17 x 131072 x 2047 1724 and 1422.
bool small_grad(const HeadShape &s, bool laid) {
    const bool wide = s.size == 4;
    const double steps = tile_rounds(s) * (!wide ? 0.65 : s.n > kNarrowRows && s.n <= kPlaneRows ? 4.3 : 2.2);
    return s.n <= kSmallRows && small_work(s) * (wide ? 17 : 10) <= 1 + steps + (laid ? laying_time(s) : 0);
}

// Floats go to the matrix cores as three 16-bit planes, unless the rows are few.  Forward and backward passes over 32768 x
// 1024: of 100 rows 89 and 244 us, in planes 134 and 235; of 128 rows 88 and 246, 132 and 238; of 129 rows 158 and 392,
// 147 and 303; of 256 rows 161 and 438, 146 and 336.  Over 131072 x 2048: of 100 rows 574 and 1729, 993 and 1927; of 200
// rows 1310 and 3333, 1134 and 2680.  (Where rows are laid out in either form, 100 x 20000 x 1000 takes 108 and 235, 85 and
// 171.)
bool planes(const HeadShape &s) { return s.size == 4 && s.n > kPlaneRows; }

// Workgroups that the chip holds at once.
template <typename Tile>
constexpr uint64_t kSlots = (2 * sizeof(typename Tile::Buffer) <= 80 * 1024 ? 2 : 1) * kCus;

// 16-bit operands whose g has two planes.
bool fine(const HeadShape &s) { return s.size == 2 && (s.n <= kFineRows || s.classes <= kFineClasses); }

// fn(tile): the larger of two, unless it leaves CUs without one or more than
// half of itself empty; `most` is how often k can be split, of which eight count:
// more cost what they write and read again (dh of 1024 x 8192 x 1024 bf16 by 16
// splits of the larger 69 us, by 8 of the smaller 63).
template <typename T, bool Across, typename F>
auto by_tile(const HeadShape &s, uint64_t m, uint64_t n, uint64_t most, F fn) {
    const bool large = ceil_div(m, 256) * ceil_div(n, planes(s) ? 128 : 256) * std::min<uint64_t>(most, 8) >= kCus && n > 128 && m > 128;
    if constexpr (std::is_same<T, float>::value) {
        if (planes(s)) return large ? fn(static_cast<LargeSplit *>(nullptr)) : fn(static_cast<SmallSplit *>(nullptr));
        if (n <= kNarrowRows) return fn(static_cast<NarrowTile *>(nullptr));
    }
    if constexpr (Across && sizeof(T) == 2) {
        if (fine(s)) return fn(static_cast<FineTile<T> *>(nullptr));
    }
    return large ? fn(static_cast<LargeTile<T, Across> *>(nullptr)) : fn(static_cast<SmallTile<T> *>(nullptr));
}
// The same where no kernel is meant.
template <bool Across, typename F>
auto by_tile_size(const HeadShape &s, uint64_t m, uint64_t n, uint64_t most, F fn) {
    return s.size == 4 ? by_tile<float, Across>(s, m, n, most, fn) : by_tile<bf16, Across>(s, m, n, most, fn);
}

// Tiles read whole steps of the weight's rows, 16 bytes at a time and with offsets of 32 bits: whether it is to be laid
// out for them.
bool to_lay(const void *p, uint64_t stride, const HeadShape &s) {
    return planes(s) || uintptr_t(p) % 16 || stride * s.size % 16 || s.width * s.size % 128 ||
           stride * s.size > kMostStride;
}

// Classes of a piece, in whole tiles, so that `bytes` hold a row of `each` for every class.
uint64_t piece_of(uint64_t classes, uint64_t each, uint64_t bytes) {
    const uint64_t most = std::max<uint64_t>(kTilePad, bytes / each / kTilePad * kTilePad);
    return whole_tiles(ceil_div(classes, ceil_div(classes, most)));
}

void head_sizes(const HeadShape &s, bool few, HeadArgs &a) {
    a.few_shift = few_shift(s);
    a.n = uint32_t(s.n);
    a.classes = uint32_t(s.classes);
    a.width = uint32_t(s.width);
    const uint64_t step = s.size == 4 ? 32 : 64;
    a.width_pad = uint32_t(ceil_div(s.width, step) * step);
    a.n_pad = uint32_t(few ? kFewRows : whole_tiles(s.n));
}

// Bytes of a laid out element, and of one of g.
uint64_t held(const HeadShape &s) { return planes(s) ? 6 : s.size; }
uint64_t slope_held(const HeadShape &s) { return fine(s) ? 4 : held(s); }

// Layout of the forward call's workspace; returns its size.
uint64_t head_room(const HeadShape &s, bool laid, void *at, HeadArgs &a) {
    Room room{static_cast<char *>(at), 0};
    head_sizes(s, few(s), a);
    a.found = room.take<float>(whole_tiles(s.n));
    if (few(s)) {
        a.parts = uint32_t(ceil_div(s.classes, kFewClasses >> a.few_shift));
        a.part = room.take<HeadSum>(uint64_t(a.parts) * a.n);
        return room.used;
    }
    a.parts = by_tile_size<false>(s, s.classes, s.n, 1, [&](auto *t) {
        using Tile = std::remove_pointer_t<decltype(t)>;
        return uint32_t(ceil_div(s.classes, Tile::BM) * Tile::WM);
    });
    a.piece = uint32_t(laid ? piece_of(s.classes, a.width_pad * held(s), kLaidBytes) : whole_tiles(s.classes));
    a.count = room.take<uint32_t>(1);
    a.chunk_count = room.take<uint32_t>(2 * ceil_div(s.n, kListChunk));
    a.list = room.take<uint32_t>(a.n_pad);
    a.packed = room.take<char>(uint64_t(a.n_pad) * a.width_pad * held(s));
    a.part = room.take<HeadSum>(uint64_t(a.parts) * a.n_pad);
    if (laid) a.weight_laid = room.take<char>(uint64_t(a.piece) * a.width_pad * held(s));
    return room.used;
}

// Classes of a workgroup of k_few_outer.
uint64_t few_share(const HeadShape &s) { return std::max<uint64_t>(16, ceil_div(s.classes, 2 * kCus)); }
// Columns of a thread of k_few_outer: what its registers hold of n rows, twice in float32.
uint32_t few_columns(const HeadShape &s) { return s.size == 4 ? 4 : 8; }
// and its block: as many threads as a row needs, up to 256, the rest for other classes.
dim3 few_block(const HeadShape &s) {
    const uint32_t x = std::min<uint32_t>(256, std::max<uint32_t>(16, pow2_from(uint32_t(ceil_div(s.width, few_columns(s))))));
    return dim3(x, 256 / x);
}

// Whether the gradient lays its weights out: for dh, and for g by tiles.
bool lays_grad(const HeadShape &s, const void *weight, uint64_t stride, bool hidden) {
    return !few_grad(s) && to_lay(weight, stride, s) && (hidden || !small_grad(s, true));
}

// Layout of the gradient's workspace.
uint64_t head_grad_room(const HeadShape &s, int dtype, bool laid, bool hidden, bool weight, void *at, HeadArgs &a) {
    Room room{static_cast<char *>(at), 0};
    head_sizes(s, few_grad(s), a);
    if (few_grad(s)) {
        a.sum_stride = uint32_t(ceil_div(s.width, 8) * 8);
        a.steps = uint32_t(few_share(s));
        a.splits = uint32_t(ceil_div(s.classes, a.steps) * few_block(s).y);
        a.slope = room.take<float>(s.classes * kFewRows);
        if (hidden) a.sum = room.take<float>(uint64_t(a.splits) * s.n * a.sum_stride);
        return room.used;
    }
    a.piece = uint32_t(piece_of(s.classes, a.n_pad * slope_held(s), kPieceBytes));
    a.sum_stride = uint32_t(ceil_div(s.width, 4) * 4);
    // dh: a workgroup to every CU (two of the small tiles, where LDS has room), which the kernel spreads over the tiles
    // that the packed rows take and splits of k, each of 4 steps at least
    const uint64_t steps = a.piece / (s.size == 4 ? 32 : 64);
    a.most = uint32_t(std::max<uint64_t>(1, std::min<uint64_t>(steps / 4, kMostSplits)));
    by_tile_size<true>(s, s.width, s.n, a.most, [&](auto *t) {
        using Tile = std::remove_pointer_t<decltype(t)>;
        a.tiles_m = uint32_t(ceil_div(s.width, Tile::BM));
        a.tile_n = Tile::BN;
        a.blocks = uint32_t(std::max(kSlots<Tile>, a.tiles_m * ceil_div(s.n, Tile::BN)));
        return 0;
    });
    // dw: likewise, for the tiles of the first piece (the last may be shorter)
    const uint64_t rows = std::min<uint64_t>(a.piece, s.classes);
    a.weight_splits = by_tile_size<true>(s, s.width, rows, 1, [&](auto *t) {
        using Tile = std::remove_pointer_t<decltype(t)>;
        const uint64_t tiles = ceil_div(s.width, Tile::BM) * ceil_div(rows, Tile::BN);
        return uint32_t(std::max<uint64_t>(1, std::min<uint64_t>({kSlots<Tile> / tiles, s.n / (8 * Tile::kStep), 32})));
    });
    a.count = room.take<uint32_t>(1);
    a.chunk_count = room.take<uint32_t>(2 * ceil_div(s.n, kListChunk));
    a.list = room.take<uint32_t>(a.n_pad);
    a.place = room.take<int32_t>(a.n_pad);
    a.row = room.take<HeadRow>(a.n_pad);
    if (dtype == TM_DTYPE_F16) a.inverse = room.take<float>(a.n_pad + 1);
    a.packed = room.take<char>(uint64_t(a.n_pad) * a.width_pad * held(s));
    const uint64_t slopes = uint64_t(a.n_pad) * a.piece * slope_held(s);
    if (hidden || dtype != TM_DTYPE_F16) a.slope = room.take<char>(slopes);
    if (weight && dtype == TM_DTYPE_F16) a.slope_common = room.take<char>(slopes);
    if (s.size == 2 && !fine(s)) {
        if (hidden || dtype != TM_DTYPE_F16) a.rest = room.take<float>(a.n_pad);
        if (weight && dtype == TM_DTYPE_F16) a.rest_common = room.take<float>(a.n_pad);
    }
    if (hidden) {
        const uint64_t rows = std::min<uint64_t>(uint64_t(a.most) * a.n_pad, uint64_t(a.blocks / a.tiles_m) * a.tile_n);
        a.sum = room.take<float>(rows * a.sum_stride);
    }
    if (weight && a.weight_splits > 1) a.weight_sum = room.take<float>(a.weight_splits * rows * a.sum_stride);
    if (laid) a.weight_laid = room.take<char>(uint64_t(a.piece) * a.width_pad * held(s));
    return room.used;
}

template <typename Tile>
dim3 tile_grid(uint64_t m, uint64_t n) {
    return dim3(uint32_t(ceil_div(m, Tile::BM) * ceil_div(n, Tile::BN)));
}
template <typename Tile>
dim3 lasting_grid(uint64_t m, uint64_t n) {
    return dim3(uint32_t(std::min<uint64_t>(tile_grid<Tile>(m, n).x, kSlots<Tile>)));
}

// The packed rows.
template <typename T>
int pack_rows(const HeadShape &s, HeadArgs &a, hipStream_t stream) {
    a.chunks = a.n <= 4 * kListChunk ? 0 : uint32_t(ceil_div(a.n, kListChunk));
    a.pack_rows = 1;
    while (a.pack_rows < kPackRows && a.n > 2 * kCus * a.pack_rows) a.pack_rows *= 2;
    if (a.chunks) {
        const int rc = launch(k_head_count, dim3(a.chunks), dim3(256), 0, stream, a);
        if (rc != TM_OK) return rc;
    }
    const bool split = std::is_same<T, float>::value && planes(s);
    a.div_pieces = Div32::make(uint32_t(a.width_pad * (split ? 2 : sizeof(T)) / 16));
    const dim3 grid(uint32_t(ceil_div(a.n, a.pack_rows)));
    if constexpr (std::is_same<T, float>::value) {
        if (split) return launch(k_head_pack<float, bf16, 3>, grid, dim3(256), 0, stream, a);
    }
    return launch(k_head_pack<T, T, 1>, grid, dim3(256), 0, stream, a);
}

// The weights of the piece at hand.
template <typename T>
int lay_piece(const HeadShape &s, const HeadArgs &a, hipStream_t stream) {
    const bool split = std::is_same<T, float>::value && planes(s);
    const uint64_t pieces = a.width_pad * (split ? 2 : sizeof(T)) / 16;
    const uint32_t x = uint32_t(std::min<uint64_t>(256, pow2_from(uint32_t(pieces))));
    const uint64_t rows = std::min(a.piece, a.classes - a.first);
    const dim3 block(x, 256 / x), grid(uint32_t(std::min<uint64_t>(ceil_div(rows, block.y), 4096)));
    if constexpr (std::is_same<T, float>::value) {
        if (split) return launch(k_head_lay<float, bf16, 3>, grid, block, 0, stream, a);
    }
    return launch(k_head_lay<T, T, 1>, grid, block, 0, stream, a);
}

// The joins' threads: along a row, four columns to each, the rest for other rows.
dim3 join_block(const HeadShape &s) {
    const uint32_t x = uint32_t(std::min<uint64_t>(256, pow2_from(uint32_t(ceil_div(s.width, 4)))));
    return dim3(x, 256 / x);
}
dim3 join_grid(uint64_t rows, const HeadShape &s) {
    return dim3(uint32_t(std::min<uint64_t>(ceil_div(rows, join_block(s).y), 4096)));
}

// Whether rows of 16-bit elements may begin between two words.
template <typename T>
bool odd_rows(const HeadArgs &a) {
    return sizeof(T) == 2 && ((uintptr_t(a.hidden) | uintptr_t(a.weight)) & 2 || (a.hidden_stride | a.weight_stride) & 1);
}

template <typename T>
int run_head(HeadArgs a, const HeadShape &s, hipStream_t stream) {
    if (few(s)) {
        const dim3 grid(a.parts, uint32_t(ceil_div(s.n, kFewRows)));
        const int rc = launch(odd_rows<T>(a) ? k_few_sums<T, sizeof(T) == 2> : k_few_sums<T, false>, grid,
                              dim3(64 * kFewWaves), 0, stream, a);
        return rc == TM_OK ? launch(k_few_rows, dim3(a.n), dim3(256), 0, stream, a) : rc;
    }
    int rc = pack_rows<T>(s, a, stream);
    for (uint64_t first = 0; rc == TM_OK && first < s.classes; first += a.piece) {
        a.first = uint32_t(first);
        if (a.weight_laid) rc = lay_piece<T>(s, a, stream);
        if (rc != TM_OK) break;
        // the tile is that of all classes: it says how many parts there are
        rc = by_tile<T, false>(s, s.classes, s.n, 1, [&](auto *t) {
            using Tile = std::remove_pointer_t<decltype(t)>;
            return launch(k_head_sums<T, Tile>, lasting_grid<Tile>(std::min<uint64_t>(a.piece, s.classes - first), s.n),
                          dim3(Tile::kThreads), 0, stream, a);
        });
    }
    return rc == TM_OK ? launch(k_head_join, dim3(uint32_t(ceil_div(s.n, 16))), dim3(1024), 0, stream, a) : rc;
}

template <typename T>
int run_few_grad(const HeadArgs &a, const HeadShape &s, hipStream_t stream) {
    int rc = launch(odd_rows<T>(a) ? k_few_slopes<T, sizeof(T) == 2> : k_few_slopes<T, false>,
                    dim3(uint32_t(ceil_div(s.classes, kFewClasses >> a.few_shift))), dim3(64 * kFewWaves), 0, stream, a);
    if (rc != TM_OK) return rc;
    const dim3 block = few_block(s);
    const dim3 grid(uint32_t(ceil_div(s.classes, a.steps)), uint32_t(ceil_div(s.width, block.x * few_columns(s))));
    constexpr int C = sizeof(T) == 4 ? 4 : 8;
    auto kernel = s.n == 1 ? k_few_outer<T, 1, C> : s.n <= 4 ? k_few_outer<T, 4, C> : k_few_outer<T, 8, C>;
    if constexpr (sizeof(T) == 4) {
        if (s.n > 8) kernel = k_few_outer<T, 16, 4>;
    }
    rc = launch(kernel, grid, block, 0, stream, a);
    if (rc != TM_OK || !a.grad_hidden) return rc;
    return launch(k_few_join<T>, dim3(uint32_t(ceil_div(s.width, 64)), a.n), dim3(1024), 0, stream, a);
}

template <typename T>
int run_head_grad(HeadArgs a, const HeadShape &s, hipStream_t stream) {
    if (few_grad(s)) return run_few_grad<T>(a, s, stream);
    const bool waves = small_grad(s, !a.grad_hidden && to_lay(a.weight, a.weight_stride, s));
    int rc = pack_rows<T>(s, a, stream);
    for (uint64_t first = 0; rc == TM_OK && first < s.classes; first += a.piece) {
        a.first = uint32_t(first);
        a.add = first > 0;
        if (a.weight_laid) rc = lay_piece<T>(s, a, stream);
        if (rc != TM_OK) break;
        if (waves) {
            const uint64_t rows = std::min<uint64_t>(a.piece, s.classes - first);
            const dim3 grid(uint32_t(ceil_div(rows, kFewClasses >> a.few_shift)), a.n_pad / kFewRows);
            auto kernel = k_few_tiles<T, T, 1, false>;
            if constexpr (sizeof(T) == 4) {
                if (planes(s)) kernel = k_few_tiles<T, bf16, 3, false>;
            } else if (odd_rows<T>(a)) {
                kernel = fine(s) ? k_few_tiles<T, T, 2, true> : k_few_tiles<T, T, 1, true>;
            } else if (fine(s)) {
                kernel = k_few_tiles<T, T, 2, false>;
            }
            rc = launch(kernel, grid, dim3(64 * kFewWaves), 0, stream, a);
        } else {
            rc = by_tile<T, false>(s, a.piece, s.n, 1, [&](auto *t) {
                using Tile = std::remove_pointer_t<decltype(t)>;
                constexpr int G = Tile::kPlanes;
                auto kernel = k_head_slopes<T, Tile, G>;
                if constexpr (sizeof(T) == 2) {
                    if (fine(s)) kernel = k_head_slopes<T, Tile, 2>;
                }
                return launch(kernel, lasting_grid<Tile>(a.piece, s.n), dim3(Tile::kThreads), 0, stream, a);
            });
        }
        if (rc == TM_OK && a.grad_hidden) {
            rc = by_tile<T, true>(s, s.width, s.n, a.most, [&](auto *t) {
                using Tile = std::remove_pointer_t<decltype(t)>;
                return launch(k_head_hidden<T, Tile>, dim3(a.blocks), dim3(Tile::kThreads), 0, stream, a);
            });
        }
        if (rc == TM_OK && a.grad_weight) {
            const uint64_t rows = std::min<uint64_t>(a.piece, s.classes - first);
            // the tile is that of the first piece, whose splits these are
            rc = by_tile<T, true>(s, s.width, std::min<uint64_t>(a.piece, s.classes), 1, [&](auto *t) {
                using Tile = std::remove_pointer_t<decltype(t)>;
                return launch(k_head_weight<T, Tile>, dim3(tile_grid<Tile>(s.width, rows).x * a.weight_splits),
                              dim3(Tile::kThreads), 0, stream, a);
            });
            if (rc == TM_OK && a.weight_splits > 1) {
                rc = launch(k_head_weight_join<T>, join_grid(rows, s), join_block(s), 0, stream, a);
            }
        }
    }
    if (rc != TM_OK || !a.grad_hidden) return rc;
    // few rows, which may have many splits
    const uint64_t quads = ceil_div(s.width, 4);
    if (s.n * quads <= kJoinFew)
        return launch(k_head_hidden_join<T, 16>, dim3(a.n, uint32_t(ceil_div(quads, kJoinQuads))), dim3(kJoinQuads, 16), 0,
                      stream, a);
    return launch(k_head_hidden_join<T, 1>, join_grid(s.n, s), join_block(s), 0, stream, a);
}

void head_args(const HeadShape &s, const void *hidden, int64_t hidden_stride, const void *weight, int64_t weight_stride,
               const void *labels, double scale, HeadArgs &a) {
    a.hidden = hidden;
    a.hidden_stride = uint64_t(hidden_stride);
    a.weight = weight;
    a.weight_stride = uint64_t(weight_stride);
    a.label = labels;
    a.label_bytes = int32_t(s.label_bytes);
    a.scale = float(scale);
    a.c = float(double(float(scale)) * 1.4426950408889634);
}

}  // namespace

extern "C" size_t tm_head_logp_workspace_size(int dtype, int64_t rows, int64_t classes, int64_t width,
                                              const void *weight, int64_t weight_stride) {
    HeadShape s{};
    HeadArgs a{};
    const void *some = reinterpret_cast<const void *>(uintptr_t(4096));
    if (check_head(some, dtype, rows, classes, width, 0, some, weight_stride, 0, nullptr, 1.0, s) != TM_OK || s.n == 0)
        return 0;
    return head_room(s, !few(s) && to_lay(weight, uint64_t(weight_stride), s), nullptr, a);
}

extern "C" int tm_head_logp(const void *hidden, int dtype, int64_t rows, int64_t classes, int64_t width,
                            int64_t hidden_stride, const void *weight, int64_t weight_stride, const void *labels,
                            int label_dtype, double scale, float *out_logp, float *out_log_sum, float *out_stats,
                            void *workspace, size_t workspace_bytes, hipStream_t stream) {
    HeadShape s{};
    const int rc = check_head(hidden, dtype, rows, classes, width, hidden_stride, weight, weight_stride, label_dtype,
                              labels, scale, s);
    if (rc != TM_OK) return rc;
    if (s.n == 0) return TM_OK;
    if (!labels && (out_logp || !out_log_sum)) return TM_ERR_NULL;
    if (!out_logp && !out_log_sum) return TM_ERR_NO_OUTPUT;
    const size_t need = tm_head_logp_workspace_size(dtype, rows, classes, width, weight, weight_stride);
    if (!workspace || workspace_bytes < need || uintptr_t(workspace) % 16) return TM_ERR_WORKSPACE;
    const Range in[] = {{hidden, s.hidden_bytes}, {weight, s.weight_bytes}, {labels, s.n * s.label_bytes}};
    const Range out[] = {{out_logp, s.n * 4}, {out_log_sum, s.n * 4}, {out_stats, s.n * 8}, {workspace, need}};
    if (aliased(in, out)) return TM_ERR_ALIAS;
    HeadArgs a{};
    head_args(s, hidden, hidden_stride, weight, weight_stride, labels, scale, a);
    head_room(s, !few(s) && to_lay(weight, a.weight_stride, s), workspace, a);
    a.all = out_log_sum != nullptr;
    a.logp = out_logp;
    a.log_sum = out_log_sum;
    a.stats = reinterpret_cast<HeadSum *>(out_stats);
    return by_type(dtype, [&](auto t) { return run_head<decltype(t)>(a, s, stream); });
}

extern "C" size_t tm_head_logp_grad_workspace_size(int dtype, int64_t rows, int64_t classes, int64_t width,
                                                   const void *weight, int64_t weight_stride, int for_hidden,
                                                   int for_weight) {
    HeadShape s{};
    HeadArgs a{};
    const void *some = reinterpret_cast<const void *>(uintptr_t(4096));
    if (check_head(some, dtype, rows, classes, width, 0, some, weight_stride, 0, nullptr, 1.0, s) != TM_OK || s.n == 0)
        return 0;
    return head_grad_room(s, dtype, lays_grad(s, weight, uint64_t(weight_stride), for_hidden != 0), for_hidden != 0,
                          for_weight != 0, nullptr, a);
}

extern "C" int tm_head_logp_grad(const void *hidden, int dtype, int64_t rows, int64_t classes, int64_t width,
                                 int64_t hidden_stride, const void *weight, int64_t weight_stride, const void *labels,
                                 int label_dtype, double scale, const float *stats, const float *up_logp,
                                 const float *up_log_sum, void *out_hidden, void *out_weight, void *workspace,
                                 size_t workspace_bytes, hipStream_t stream) {
    HeadShape s{};
    const int rc = check_head(hidden, dtype, rows, classes, width, hidden_stride, weight, weight_stride, label_dtype,
                              labels, scale, s);
    if (rc != TM_OK) return rc;
    if (s.n == 0 && !out_weight) return TM_OK;
    if (!out_hidden && !out_weight) return TM_ERR_NO_OUTPUT;
    if (s.n && ((!up_logp && !up_log_sum) || (up_logp && !labels) || !stats)) return TM_ERR_NULL;
    const uint64_t grad_bytes = s.classes * s.width * s.size;
    const size_t need = tm_head_logp_grad_workspace_size(dtype, rows, classes, width, weight, weight_stride,
                                                         out_hidden != nullptr, out_weight != nullptr);
    if (need && (!workspace || workspace_bytes < need || uintptr_t(workspace) % 16)) return TM_ERR_WORKSPACE;
    const Range in[] = {{hidden, s.hidden_bytes}, {weight, s.weight_bytes}, {labels, s.n * s.label_bytes},
                        {stats, s.n * 8}, {up_logp, s.n * 4}, {up_log_sum, s.n * 4}};
    const Range out[] = {{out_hidden, s.n * s.width * s.size}, {out_weight, grad_bytes}, {need ? workspace : nullptr, need}};
    if (aliased(in, out)) return TM_ERR_ALIAS;
    if (s.n == 0) {
        FillArgs f{out_weight, grad_bytes};
        return launch(k_fill_zeros<256>, dim3(uint32_t(std::min<uint64_t>(4 * kFill, ceil_div(grad_bytes, 4096)))), dim3(256), 0,
                      stream, f);
    }
    HeadArgs a{};
    head_args(s, hidden, hidden_stride, weight, weight_stride, labels, scale, a);
    head_grad_room(s, dtype, lays_grad(s, weight, a.weight_stride, out_hidden != nullptr), out_hidden != nullptr,
                   out_weight != nullptr, workspace, a);
    a.all = up_log_sum != nullptr;
    a.stats = reinterpret_cast<HeadSum *>(const_cast<float *>(stats));
    a.up_logp = up_logp;
    a.up_log_sum = up_log_sum;
    a.grad_hidden = out_hidden;
    a.grad_weight = out_weight;
    return by_type(dtype, [&](auto t) { return run_head_grad<decltype(t)>(a, s, stream); });
}
