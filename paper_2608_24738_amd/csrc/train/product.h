// product.h -- tiles of a matrix product  C[m][n] = sum_k A[m][k] B[n][k]  on
// the matrix cores, both operands with k side by side, for the kernels of
// head.h.
//
// A workgroup's tile goes through k in steps of 128 bytes a row (64 elements of
// 16 bits, 32 floats).  A step's rows of both operands are copied from memory
// straight to LDS, one step ahead of the one that is multiplied, into two
// buffers that are separate objects: the compiler then knows that a copy under
// way is not what is read, and waits for it at the barrier alone.
//
// In LDS the eight 16-byte pieces of row r lie in the order piece ^ (r & 7).
// A copy writes 64 pieces side by side, so the order is made by which piece a
// lane fetches; a read of one piece from each of 16 rows then meets all banks
// alike.
//
// A lane of a matrix instruction holds one piece of one row, whatever the type:
// 16-bit elements go in by one 16x16x32 instruction (k = 8 g + e for lane group
// g = lane / 16), floats by four 16x16x4 instructions, of which number e takes
// k = 4 g + e.  A and B agree on the order of k, which is all that matters.
// Of the result, a lane holds rows m = 4 g .. 4 g + 3 in column n = lane % 16.
#pragma once

#include "train_common.h"

namespace tmtrain {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kStepBytes = 128;            // of a row, in one step
constexpr uint32_t kTilePad = 256;              // rows of laid out operands come in whole largest tiles

template <typename T>
constexpr uint32_t kStep = kStepBytes / sizeof(T);

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

// 16 bytes a lane from memory to LDS: lane l's go to `to` + 16 l.
__device__ __forceinline__ void copy_to_lds(const char *from, char *to) {
    typedef const __attribute__((address_space(1))) uint32_t *Global;
    typedef __attribute__((address_space(3))) uint32_t *Local;
    __builtin_amdgcn_global_load_lds((Global)from, (Local)to, 16, 0, 0);
}

// What a row's pieces beyond its end are read from.
__device__ __attribute__((aligned(16))) const uint32_t kZeroPiece[4] = {0, 0, 0, 0};

// Which tile of tiles_m x tiles_n a workgroup takes.  Workgroups go round robin
// over the eight XCDs: each gets one stretch of the tiles, so that its L2 holds
// what neighbouring tiles share, and a stretch goes down m over a few columns.
struct TilePlace {
    uint32_t m, n;
};
__device__ __forceinline__ TilePlace tile_place(uint32_t block, uint32_t tiles_m, uint32_t tiles_n) {
    constexpr uint32_t kXcds = 8, kColumns = 4;
    const uint32_t total = tiles_m * tiles_n;
    const uint32_t xcd = block % kXcds, share = total / kXcds, more = total % kXcds;
    const uint32_t t = xcd * share + min(xcd, more) + block / kXcds;
    const uint32_t group = t / (kColumns * tiles_m), in = t - group * kColumns * tiles_m;
    const uint32_t columns = min(kColumns, tiles_n - group * kColumns);
    return {in / columns, group * kColumns + in % columns};
}

// One operand: rows of k, `stride` bytes apart, 16-byte aligned.
struct Operand {
    const char *at;
    uint64_t stride;
    uint32_t rows;              // rows beyond are read as the last one
    uint32_t pieces;            // whole pieces in a row, beyond them zeros; 0: rows hold whole steps
};

// BM x BN elements by WM x WN waves.
template <typename T, int BM_, int BN_, int WM_, int WN_>
struct Tile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
    static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
    static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;  // 16 x 16 blocks of a wave
    static constexpr int LM = BM / 8 / kWaves, LN = BN / 8 / kWaves;  // copies of a wave, eight rows each

    struct Buffer {
        char row[(BM + BN) * int(kStepBytes)];
    };

    f32x4 acc[TM][TN];
    int lane, wave;

    __device__ __forceinline__ Tile() {
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    // First row and column, in the tile, of what the lane holds of block i, j.
    __device__ __forceinline__ uint32_t row(int i) const { return ((wave / WN) * TM + i) * 16 + (lane >> 4) * 4; }
    __device__ __forceinline__ uint32_t column(int j) const { return ((wave % WN) * TN + j) * 16 + (lane & 15); }

    // Adds the products of rows m0.. of A and n0.. of B over steps [first, last).
    __device__ __forceinline__ void run(const Operand &a, uint32_t m0, const Operand &b, uint32_t n0, uint32_t first,
                                        uint32_t last, Buffer &even, Buffer &odd) {
        if (first >= last) return;
        const uint32_t r = lane >> 3, piece = (lane & 7) ^ r;
        const char *pa[LM], *pb[LN];
#pragma unroll
        for (int i = 0; i < LM; ++i)
            pa[i] = a.at + min(m0 + (i * kWaves + wave) * 8 + r, a.rows - 1) * a.stride + first * kStepBytes + piece * 16;
#pragma unroll
        for (int i = 0; i < LN; ++i)
            pb[i] = b.at + min(n0 + (i * kWaves + wave) * 8 + r, b.rows - 1) * b.stride + first * kStepBytes + piece * 16;
        const uint32_t ragged = a.pieces ? a.pieces / 8 : ~0u;        // the step that A's rows end in
        const auto fetch = [&](Buffer &s, uint32_t step) {
            if (step == ragged) {
                const bool out = step * 8 + piece >= a.pieces;
#pragma unroll
                for (int i = 0; i < LM; ++i)
                    pa[i] = out ? reinterpret_cast<const char *>(kZeroPiece) : pa[i];
            }
#pragma unroll
            for (int i = 0; i < LM; ++i) {
                copy_to_lds(pa[i], s.row + (i * kWaves + wave) * 1024);
                pa[i] += kStepBytes;
            }
#pragma unroll
            for (int i = 0; i < LN; ++i) {
                copy_to_lds(pb[i], s.row + BM * kStepBytes + (i * kWaves + wave) * 1024);
                pb[i] += kStepBytes;
            }
        };
        const uint32_t c = lane & 15, g = lane >> 4;
        const auto work = [&](const Buffer &s) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const char *at = s.row + c * kStepBytes + ((g + 4 * half) ^ (c & 7)) * 16;
                u32x4 fa[TM], fb[TN];
#pragma unroll
                for (int i = 0; i < TM; ++i)
                    fa[i] = *reinterpret_cast<const u32x4 *>(at + ((wave / WN) * TM + i) * 16 * kStepBytes);
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    fb[j] = *reinterpret_cast<const u32x4 *>(at + (BM + ((wave % WN) * TN + j) * 16) * kStepBytes);
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j] = multiply<T>(fa[i], fb[j], acc[i][j]);
            }
        };
        fetch(even, first);
        for (uint32_t k = first; k < last; k += 2) {
            __syncthreads();                    // even has arrived, odd is read
            if (k + 1 < last) fetch(odd, k + 1);
            work(even);
            __syncthreads();
            if (k + 2 < last) fetch(even, k + 2);
            if (k + 1 < last) work(odd);
        }
    }
};

template <typename T> using LargeTile = Tile<T, 256, 256, 2, 4>;
template <typename T> using SmallTile = Tile<T, 128, 128, 2, 2>;

}  // namespace tmtrain
