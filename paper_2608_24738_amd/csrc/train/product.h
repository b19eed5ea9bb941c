// product.h -- tiles of a matrix product  C[m][n] = sum_k A[m][k] B[n][k]  on
// the matrix cores, for the kernels of head.h.  An operand lies along k (k side
// by side in a row, the rows are m or n) or across it (m or n side by side, the
// rows are k), so that none is ever turned in memory.
//
// A workgroup's tile goes through k in steps of 64 elements of 16 bits or 32
// floats.  A step of both operands is copied from memory straight to LDS, one
// step ahead of the one that is multiplied, into two buffers that are separate
// objects: the compiler then knows that a copy under way is not what is read,
// and waits for it at the barrier alone.
//
// A copy writes 64 pieces of 16 bytes side by side, one a lane, so the order of
// the pieces within a row of LDS is made by which piece a lane fetches.  Along
// k, the eight pieces of row r lie in the order piece ^ (r & 7); across it, the
// 32 bytes (floats: 64) that a read takes of a row lie in the order unit ^ u,
// with u another number for each of the rows that one instruction reads.  All
// reads then meet the banks alike.
//
// A lane of a matrix instruction holds 16 bytes of one m or n: 16-bit elements
// go in by one 16x16x32 instruction (k = 8 g + e for lane group g = lane / 16),
// floats by four 16x16x4 instructions, of which number e takes k = 4 g + e.
// Across k, 16-bit elements come from LDS by reads that turn blocks of 4 x 16,
// floats one by one.  Of the result, a lane holds rows m = 4 g .. 4 g + 3 in
// column n = lane % 16.  Rows of A along k come to LDS in another order, so that
// these are, of two blocks, eight rows of C side by side, 16 bytes of 16 bits.
#pragma once

#include <type_traits>
#include <utility>

#include "train_common.h"

namespace tmtrain {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kTilePad = 256;              // rows of laid out operands come in whole largest tiles

// acc += the products over one piece of k.
template <typename T>
__device__ __forceinline__ f32x4 multiply(u32x4 a, u32x4 b, f32x4 acc) {
    if constexpr (__is_same(T, bf16)) {
        typedef __bf16 b8 __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), acc, 0, 0, 0);
    } else if constexpr (__is_same(T, f16)) {
        typedef _Float16 h8 __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), acc, 0, 0, 0);
        return acc;
    }
}

// 16 bytes a lane from memory to LDS: lane l's go to `to` + 16 l.  One address
// for the wave and an offset of 32 bits a lane, which stays from step to step.
__device__ __forceinline__ void copy_to_lds(const char *from, uint32_t offset, char *to) {
    typedef const __attribute__((address_space(1))) uint32_t *Global;
    typedef __attribute__((address_space(3))) uint32_t *Local;
    __builtin_amdgcn_global_load_lds((Global)(from + offset), (Local)to, 16, 0, 0);
}

// Which tile of tiles_m x tiles_n a workgroup takes.  Workgroups go round robin
// over the eight XCDs: each gets one stretch of the tiles, so that its L2 holds
// what neighbouring tiles share, and a stretch goes down m over a few columns.
// Splits of k come one after the other: tiles that run together read the same k.
struct TilePlace {
    uint32_t m, n, split;
};
__device__ __forceinline__ TilePlace tile_place(uint32_t block, uint32_t tiles_m, uint32_t tiles_n, uint32_t splits = 1) {
    constexpr uint32_t kXcds = 8, kColumns = 4;
    const uint32_t total = tiles_m * tiles_n * splits;
    const uint32_t xcd = block % kXcds, share = total / kXcds, more = total % kXcds;
    uint32_t t = xcd * share + min(xcd, more) + block / kXcds;
    const uint32_t split = t / (tiles_m * tiles_n);
    t -= split * tiles_m * tiles_n;
    const uint32_t group = t / (kColumns * tiles_m), in = t - group * kColumns * tiles_m;
    const uint32_t columns = min(kColumns, tiles_n - group * kColumns);
    return {in / columns, group * kColumns + in % columns, split};
}

// One operand: rows `stride` <= kMostStride bytes apart, 16-byte aligned.  Along
// k, rows hold whole steps.
constexpr uint64_t kMostStride = uint64_t(1) << 23;     // 256 of them fit an offset of 32 bits
struct Operand {
    const char *at;
    uint64_t stride, plane;     // plane: bytes from one plane to the next
    uint32_t rows;              // rows beyond are read as the last one
    uint32_t pieces;            // of 16 bytes in a row; across k: those beyond are read as the last one
};

// Copies of an operand's steps to LDS, S elements of m or n by Waves waves, K
// elements of k a step (one or two instructions' worth).  Pairs: of 32 rows, row 4
// (2 g + b) + q goes to row 4 g + q of block b.
template <typename T, int S, int Waves, int K, bool Pairs>
struct Along {
    static constexpr uint32_t kRow = K * sizeof(T), kPieces = kRow / 16;    // 8 or 4 pieces in a row
    static constexpr uint32_t kAtOnce = 64 / kPieces;                       // rows of one copy
    static constexpr int kCopies = S / kAtOnce / Waves;
    const char *from;
    uint32_t offset[kCopies], place;

    static __device__ __forceinline__ uint32_t order(uint32_t r) { return kPieces == 8 ? r & 7 : r >> 1 & 3; }
    // The row that row r of LDS holds.
    static __device__ __forceinline__ uint32_t row_at(uint32_t r) {
        return Pairs ? (r & ~31u) | (r & 12) << 1 | (r & 16) >> 2 | (r & 3) : r;
    }
    __device__ __forceinline__ Along(const Operand &o, uint32_t m0, uint32_t first, int lane, int wave) {
        const uint32_t r = lane / kPieces, row = min(m0, o.rows - 1);       // tiles may lie behind the last row
        from = o.at + row * o.stride + uint64_t(first) * kRow;
#pragma unroll
        for (int i = 0; i < kCopies; ++i)
            offset[i] = min(row_at((i * Waves + wave) * kAtOnce + r), o.rows - 1 - row) * uint32_t(o.stride) +
                        (lane % kPieces ^ order(r)) * 16;
    }
    __device__ __forceinline__ void fetch(char *lds, uint32_t, int, int wave) {
#pragma unroll
        for (int i = 0; i < kCopies; ++i) copy_to_lds(from, offset[i], lds + (i * Waves + wave) * 1024);
        from += kRow;
    }
    // Where the lane's reads of block 0 begin, and the 16 bytes of block i in half of a step.
    __device__ __forceinline__ void reads(int lane, uint32_t block) {
        place = (block * 16 + (lane & 15)) * kRow + (((lane >> 4) ^ order(lane & 15)) * 16);
    }
    __device__ __forceinline__ u32x4 read(const char *lds, int i, int half) const {
        return *reinterpret_cast<const u32x4 *>(lds + (half ? place ^ 64 : place) + i * 16 * kRow);
    }
};

template <typename T, int S, int Waves, int K, int Blocks>
struct Across {
    static constexpr int kCopies = S * K * int(sizeof(T)) / 1024 / Waves;
    static constexpr uint32_t kRow = S * sizeof(T), kPieces = kRow / 16;    // of a row in LDS
    static constexpr uint32_t kUnits = S / 16;                              // of 16 elements
    const char *from;
    uint32_t stride, rows;
    uint32_t offset[kCopies];

    // Pieces of a unit, and the number that orders the units of row r.
    static constexpr uint32_t kUnitPieces = sizeof(T);
    static __device__ __forceinline__ uint32_t order(uint32_t r) {
        const uint32_t u = sizeof(T) == 4 ? r >> 2 & 3 : (r & 3) | (r >> 3 & 3) << 2;
        return u & (kUnits - 1);
    }
    static __device__ __forceinline__ uint32_t row_of(int i, int lane, int wave) {
        return (i * Waves + wave) * (64 / kPieces) + lane / kPieces;
    }
    __device__ __forceinline__ Across(const Operand &o, uint32_t m0, uint32_t first, int lane, int wave) {
        stride = uint32_t(o.stride);
        rows = o.rows;
        from = o.at + uint64_t(first) * K * stride;
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const uint32_t r = row_of(i, lane, wave);
            const uint32_t piece = m0 * sizeof(T) / 16 + (lane % kPieces ^ order(r) * kUnitPieces);
            offset[i] = r * stride + min(piece, o.pieces - 1) * 16;
        }
    }
    __device__ __forceinline__ void fetch(char *lds, uint32_t step, int lane, int wave) {
        if ((step + 1) * K > rows) {            // the last step
#pragma unroll
            for (int i = 0; i < kCopies; ++i) {
                const uint32_t r = row_of(i, lane, wave);
                offset[i] -= (r - min(r, rows - 1 - step * K)) * stride;
            }
        }
#pragma unroll
        for (int i = 0; i < kCopies; ++i) copy_to_lds(from, offset[i], lds + (i * Waves + wave) * 1024);
        from += uint64_t(K) * stride;
    }
    // A step of rows that a list of `count` >= 1 numbers gives; behind them the last one again.
    static __device__ __forceinline__ void gather(const Operand &o, uint32_t m0, const uint32_t *list, uint32_t count,
                                                  char *lds, int lane, int wave) {
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const uint32_t r = row_of(i, lane, wave), piece = m0 * sizeof(T) / 16 + (lane % kPieces ^ order(r) * kUnitPieces);
            copy_to_lds(o.at + list[min(r, count - 1)] * o.stride, min(piece, o.pieces - 1) * 16,
                        lds + (i * Waves + wave) * 1024);
        }
    }
    // Where element c of row r of a step lies.
    static __device__ __forceinline__ uint32_t element(uint32_t r, uint32_t c) {
        return r * kRow + (c / 16 ^ order(r)) * 16 * sizeof(T) + c % 16 * sizeof(T);
    }
    uint32_t place[Blocks];
    __device__ __forceinline__ void reads(int lane, uint32_t block) {
        const uint32_t c = lane & 15, g = lane >> 4;
#pragma unroll
        for (int i = 0; i < Blocks; ++i) {
            if constexpr (sizeof(T) == 4)
                place[i] = 4 * g * kRow + ((block + i) ^ order(4 * g)) * 64 + c * 4;
            else
                place[i] = (8 * g + (c >> 2)) * kRow + ((block + i) ^ order(8 * g + (c >> 2))) * 32 + (c & 3) * 8;
        }
    }
    __device__ __forceinline__ u32x4 read(const char *lds, int i, int half) const {
        u32x4 v;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = *reinterpret_cast<const uint32_t *>(lds + place[i] + (16 * half + e) * kRow);
        } else {
            typedef short s4 __attribute__((ext_vector_type(4)));
            typedef uint32_t u2 __attribute__((ext_vector_type(2)));
            typedef __attribute__((address_space(3))) s4 *Local;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const u2 q = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (Local)(lds + place[i] + (32 * half + 4 * e) * kRow)));
                v[2 * e] = q[0];
                v[2 * e + 1] = q[1];
            }
        }
        return v;
    }
};

// BM x BN elements by WM x WN waves.  An operand may lie in planes of T, whose
// sum it is.  Three of bf16 hold a float, x = h + m + l, exactly, since each
// takes eight more bits; a product of two is hh + hm + mh + mm + hl + lh, what is
// left out being below 2^-23 of it, and six instructions of 16 bits take less
// time than those of floats (2048 x 16384 x 1024: sums 300 us and 495).  All but
// hh have sums of their own: they are 2^-8 of the whole and add no rounding at
// its size.  An infinity has the planes inf, 0 and 0: hh then is what the product
// is, and hm and hl, inf times 0, are left out.  Two planes, of B alone, make 16
// or 22 bits of a number.
template <typename T, int BM_, int BN_, int WM_, int WN_, int PlanesA = 1, int PlanesB = PlanesA>
struct Tile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, kPlanes = PlanesA, kPlanesB = PlanesB;
    static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
    static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;              // 16 x 16 blocks of a wave
    static constexpr int kHalves = PlanesB == 1 ? 2 : 1;                    // instructions' worth of k in a step
    static constexpr int kStep = kHalves * 64 / int(sizeof(T));             // elements
    static constexpr int kPlaneA = BM * kHalves * 64, kPlaneB = BN * kHalves * 64;     // bytes of a plane's step

    struct Buffer {
        char a[PlanesA * kPlaneA], b[PlanesB * kPlaneB];
    };

    f32x4 acc[TM][TN];
    int lane, wave;

    __device__ __forceinline__ Tile() {
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    }
    // First row and column, in the tile, of what the lane holds of block i, j; rows for A along k, of which blocks 2 i
    // and 2 i + 1 have eight side by side, and across it.
    static_assert(TM % 2 == 0, "blocks in pairs");
    static constexpr __device__ __forceinline__ uint32_t pair_row(int i) { return i / 2 * 32 + i % 2 * 4; }
    __device__ __forceinline__ uint32_t first_row() const { return wave / WN * TM * 16; }
    __device__ __forceinline__ uint32_t row(int i) const { return first_row() + (lane >> 4) * 8 + pair_row(i); }
    __device__ __forceinline__ uint32_t row_across(int i) const { return first_row() + i * 16 + (lane >> 4) * 4; }
    __device__ __forceinline__ uint32_t column(int j) const { return ((wave % WN) * TN + j) * 16 + (lane & 15); }

    // Where a tile's operands come from, and the next step of both.
    template <bool AAcross, bool BAcross>
    struct Sources {
        typedef std::conditional_t<AAcross, Across<T, BM, kWaves, kStep, TM>, Along<T, BM, kWaves, kStep, true>> FromA;
        typedef std::conditional_t<BAcross, Across<T, BN, kWaves, kStep, TN>, Along<T, BN, kWaves, kStep, false>> FromB;
        // Waves with their operands at hand go first (4096 x 32768 x 1024: sums 246 -> 238 us); those that
        // read across k would hold up the others' reads (dw 121 -> 158), and planes leave time (sums of floats 309 -> 321).
        static constexpr bool kFirst = !AAcross && !BAcross && PlanesB == 1;
        FromA a[PlanesA];
        FromB b[PlanesB];

        template <size_t... I, size_t... J>
        __device__ __forceinline__ Sources(const Tile &t, const Operand &x, uint32_t m0, const Operand &y, uint32_t n0,
                                           uint32_t first, std::index_sequence<I...>, std::index_sequence<J...>)
            : a{FromA({x.at + I * x.plane, x.stride, 0, x.rows, x.pieces}, m0, first, t.lane, t.wave)...},
              b{FromB({y.at + J * y.plane, y.stride, 0, y.rows, y.pieces}, n0, first, t.lane, t.wave)...} {
            a[0].reads(t.lane, (t.wave / WN) * TM);
            b[0].reads(t.lane, (t.wave % WN) * TN);
        }
        __device__ __forceinline__ void fetch(const Tile &t, Buffer &s, uint32_t step) {
#pragma unroll
            for (int p = 0; p < PlanesA; ++p) a[p].fetch(s.a + p * kPlaneA, step, t.lane, t.wave);
#pragma unroll
            for (int p = 0; p < PlanesB; ++p) b[p].fetch(s.b + p * kPlaneB, step, t.lane, t.wave);
        }
    };

    // Sources for m0.. of A and n0.. of B from step `first` on.
    template <bool AAcross, bool BAcross>
    __device__ __forceinline__ Sources<AAcross, BAcross> sources(const Operand &a, uint32_t m0, const Operand &b,
                                                                 uint32_t n0, uint32_t first) const {
        return Sources<AAcross, BAcross>(*this, a, m0, b, n0, first, std::make_index_sequence<PlanesA>{},
                                         std::make_index_sequence<PlanesB>{});
    }
    // The same, with step `first` on its way.
    template <bool AAcross, bool BAcross>
    __device__ __forceinline__ Sources<AAcross, BAcross> begin(const Operand &a, uint32_t m0, const Operand &b, uint32_t n0,
                                                               uint32_t first, Buffer &even) const {
        auto from = sources<AAcross, BAcross>(a, m0, b, n0, first);
        from.fetch(*this, even, first);
        return from;
    }

    // A barrier behind which all waves' copies have arrived and all their reads are done.
    static __device__ __forceinline__ void sync() {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    }

    // acc += the products of the step in s; low: the small ones of three planes.
    template <typename From, typename Low>
    __device__ __forceinline__ void step(const From &from, const Buffer &s, Low &low) {
#pragma unroll
        for (int half = 0; half < kHalves; ++half) {
            u32x4 fa[PlanesA][TM], fb[PlanesB][TN];
#pragma unroll
            for (int p = 0; p < PlanesA; ++p)
#pragma unroll
                for (int i = 0; i < TM; ++i) fa[p][i] = from.a[0].read(s.a + p * kPlaneA, i, half);
#pragma unroll
            for (int p = 0; p < PlanesB; ++p)
#pragma unroll
                for (int j = 0; j < TN; ++j) fb[p][j] = from.b[0].read(s.b + p * kPlaneB, j, half);
            const auto add = [&](auto &to, int pa, int pb) {
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) to[i][j] = multiply<T>(fa[pa][i], fb[pb][j], to[i][j]);
            };
            if constexpr (From::kFirst) __builtin_amdgcn_s_setprio(1);
            add(acc, 0, 0);
            if constexpr (PlanesB == 2) add(acc, 0, 1);
            if constexpr (PlanesA == 3) {
                add(low, 0, 1);
                add(low, 1, 0);
                add(low, 1, 1);
                add(low, 0, 2);
                add(low, 2, 0);
            }
            if constexpr (From::kFirst) __builtin_amdgcn_s_setprio(0);
        }
    }

    // The products over steps [first, last), of which `even` has got the first.
    // Afterwards `even` can be filled again: all waves have done with it.
    template <typename From>
    __device__ __forceinline__ void run(From &from, uint32_t first, uint32_t last, Buffer &even, Buffer &odd) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        f32x4 low[PlanesA == 3 ? TM : 1][PlanesA == 3 ? TN : 1];
        if constexpr (PlanesA == 3) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) low[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        const auto work = [&](const Buffer &s) { step(from, s, low); };
        for (uint32_t k = first; k < last; k += 2) {
            sync();                             // even has arrived, odd is read
            if (k + 1 < last) from.fetch(*this, odd, k + 1);
            work(even);
            sync();
            if (k + 2 < last) from.fetch(*this, even, k + 2);
            if (k + 1 < last) work(odd);
        }
        if constexpr (PlanesA == 3) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        acc[i][j][q] += fabsf(acc[i][j][q]) == INFINITY ? 0.0f : low[i][j][q];
        }
    }
    template <bool AAcross, bool BAcross>
    __device__ __forceinline__ void run(const Operand &a, uint32_t m0, const Operand &b, uint32_t n0, uint32_t first,
                                        uint32_t last, Buffer &even, Buffer &odd) {
        if (first >= last) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            return;
        }
        auto from = begin<AAcross, BAcross>(a, m0, b, n0, first, even);
        run(from, first, last, even, odd);
    }
};

// Sixteen waves hide the reads' latency best (4096 x 32768 x 1024 bf16: sums 246 us, by eight 271); across k, of whose
// reads there are twice as many, eight waves of larger tiles (dh 137 and 135, dw 121 and 116).
template <typename T, bool Across> using LargeTile = std::conditional_t<Across, Tile<T, 256, 256, 2, 4>, Tile<T, 256, 256, 2, 8>>;
template <typename T> using SmallTile = Tile<T, 128, 128, 2, 4>;
// Few rows of floats, whose instructions would bound the larger tiles (17 x 131072 x 2048: 330 us, by 128 x 128 some 580).
typedef Tile<float, 128, 64, 4, 2> NarrowTile;
typedef Tile<bf16, 256, 128, 4, 2, 3> LargeSplit;
typedef Tile<bf16, 128, 128, 4, 2, 3> SmallSplit;
template <typename T> using FineTile = Tile<T, 256, 128, 4, 2, 1, 2>;

}  // namespace tmtrain
