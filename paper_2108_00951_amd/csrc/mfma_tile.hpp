// A tile of C = A B^T on the matrix cores (gfx950): the product that the
// orthogonalised update (muon.hip) and the cross entropy (xent.hip) share.
//
// Both operands are stored along the summed axis: row r of A holds A[r, 0..K).
// A step of 128 bytes of a row holds
//   kBf16   64 bf16 values;
//   kHalf   64 fp16 values, scaled by a power of two;
//   kFp32   32 fp32 values as they are, for the fp32 matrix instructions
//           (32 x 32 x 2; 157 TFLOP/s): where a product waits for memory and a
//           pass that splits its operands would cost more than it saves;
//   kSplit  32 fp32 values as 32 fp16 high parts and then their 32 low parts:
//           v s = hi + lo with s a power of two, hi = fp16(v s),
//           lo = fp16(v s - hi).  The product is hi hi + hi lo + lo hi, three
//           fp16 products in fp32 accumulators: what is left out, lo lo and
//           the rounding of lo, is 2^-22 of a product at most, as much as an
//           fp32 product's own sums lose.  It runs at a third of the 16-bit
//           rate (2500 TFLOP/s), five times that of the fp32 matrix
//           instructions.  (The parts in planes of their own, 64 bytes of each
//           a step: 7 % slower.)
// A workgroup of WM x WN waves computes WM TM 32 rows by WN TN 32 columns, a
// wave TM x TN accumulators of the 32 x 32 x 16 instruction.  Steps go from
// memory straight to LDS (16 bytes a lane, no registers), into one of two
// buffers while the other one is multiplied (kStages buffers, where a tile is so
// narrow that one step in flight does not cover memory's latency).  In LDS a row's eight 16-byte
// units are permuted by the row's low bits, so that eight neighbouring rows
// lie in different banks; rows eight apart share theirs, and half of the cycles
// that LDS is busy count as conflicts.  A step's reads from LDS
// are spread between the products by scheduling groups.  Measured, 8192 x 8192
// x 4096, 256 x 256 tile: kSplit 441 TFLOP/s (1322 of fp16 products), kBf16
// 1124; without the groups 396 and 1056.  With 128 x 128 tiles 380 and 948,
// but 1024 x 4096 x 1024 runs at 286 and 532 against 131 and 288, since it has
// only 64 tiles of the larger kind for 256 compute units.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_common.hpp"
#include "launch.hpp"

#include <math.h>
#include <type_traits>

namespace efs {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

enum class Prec { kBf16, kHalf, kFp32, kSplit };

constexpr int kStepBytes = 128;   // of one row, a step of the summed axis
// values of a row in one step
template <Prec P>
constexpr int kStepValues = P == Prec::kSplit || P == Prec::kFp32 ? 32 : 64;

// Steps that `len` values take.
template <Prec P>
__host__ __device__ constexpr int64_t steps_of(int64_t len) {
    return (len + kStepValues<P> - 1) / kStepValues<P>;
}

// Bytes of a row of `len` values, padded with zeros to whole steps, and the
// values that it then holds.
template <Prec P>
__host__ __device__ constexpr int64_t row_bytes(int64_t len) {
    return steps_of<P>(len) * kStepBytes;
}
template <Prec P>
__host__ __device__ constexpr int32_t row_values(int64_t len) {
    return int32_t(steps_of<P>(len) * kStepValues<P>);
}

// `rows` >= 1 rows of `stride` bytes (a multiple of 16, as `base` is).  Rows
// past the last are read as the last: what they give is not used.
struct Operand {
    const char *base;
    int64_t stride;
    int32_t rows;
};

// The scaled value as its two halves.  An infinite or NaN value has no low
// part, so that it stays what it is.
__device__ __forceinline__ void split_value(float y, _Float16 &hi, _Float16 &lo) {
    hi = _Float16(y);
    const float h = float(hi);
    lo = fabsf(h) < INFINITY ? _Float16(__fsub_rn(y, h)) : _Float16(0.0f);
}

// Bytes from a split row's start to the high part of value c; its low part
// is 64 bytes further.
__device__ __forceinline__ int64_t split_offset(int32_t c) {
    return int64_t(c >> 5) * kStepBytes + (c & 31) * 2;
}

// Eight consecutive values of a split row, the first a multiple of eight.
__device__ __forceinline__ void store_split8(char *row, int32_t c, const float (&y)[8]) {
    f16x8 hi, lo;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        _Float16 h, l;
        split_value(y[k], h, l);
        hi[k] = h;
        lo[k] = l;
    }
    char *p = row + split_offset(c);
    *reinterpret_cast<f16x8 *>(p) = hi;
    *reinterpret_cast<f16x8 *>(p + 64) = lo;
}

typedef uint16_t u16x8_at2 __attribute__((ext_vector_type(8), aligned(2)));
typedef uint16_t u16x8_at4 __attribute__((ext_vector_type(8), aligned(4)));

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

template <Prec P, int WM, int WN, int TM, int TN, int kStages = 2>
struct MfmaTile {
    static constexpr int kRows = WM * TM * 32;
    static constexpr int kCols = WN * TN * 32;
    static constexpr int kThreads = WM * WN * kWave;
    static constexpr int kBufferBytes = (kRows + kCols) * kStepBytes;
    static constexpr int kLdsBytes = kStages * kBufferBytes;
    static constexpr int kLoadsA = kRows / 8 / (WM * WN);   // a wave's, 8 rows each
    static constexpr int kLoadsB = kCols / 8 / (WM * WN);
    static constexpr int kLoads = kLoadsA + kLoadsB;
    static constexpr int kTilesM = TM, kTilesN = TN;
    // Waiting for all loads but those of the kStages - 2 later steps: the
    // count's low four bits are bits 0..3 of the operand, its high two 14..15.
    static constexpr int kLater = (kStages - 2) * kLoads;
    static_assert(kStages >= 2 && kLater < 64, "six bits count the loads");
    static constexpr int kWaitLoads = 0x0f70 | (kLater & 15) | (kLater >> 4 << 14);
    // Loads between the products, where registers are left for it (64 x 64:
    // 21.5 -> 19.6 us for 256 x 256 x 2048, 128 x 128: 381 -> 391 TFLOP/s; the
    // largest kind loses 3 %).
    static constexpr bool kSpread = TM * TN <= 4;
    static constexpr int kWavesPerSimd = kThreads >= 256 ? 2 : 1;   // asked of the compiler

    f32x16 acc[TM][TN];

    // Row and column, within the workgroup's tile, of element e of acc[i][j]:
    // a lane holds one column and four consecutive rows in each eight.
    static __device__ __forceinline__ int row_of(int i, int e) {
        const int wave = threadIdx.x / kWave, half = (threadIdx.x & (kWave - 1)) >> 5;
        return (wave / WN * TM + i) * 32 + (e >> 2) * 8 + half * 4 + (e & 3);
    }
    static __device__ __forceinline__ int col_of(int j) {
        const int wave = threadIdx.x / kWave;
        return (wave % WN * TN + j) * 32 + (threadIdx.x & 31);
    }

    static __device__ __forceinline__ f32x16 mfma(f16x8 a, f16x8 b, f32x16 c) {
        if constexpr (P == Prec::kFp32) {
            // a lane's four values are four values of k, the same for a and b
            const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
            for (int k = 0; k < 4; ++k) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[k], y[k], c, 0, 0, 0);
            return c;
        } else if constexpr (P == Prec::kBf16)
            return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                           __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
        else
            return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }

    // acc = A[row0.., step0..step0+steps) B[col0.., ...)^T, in the operands'
    // scaled units.  `lds` has kLdsBytes, 16-byte aligned; it is free again
    // after a barrier.  Called by every thread of the workgroup.
    __device__ __forceinline__ void run(const Operand &a, const Operand &b, int32_t row0, int32_t col0,
                                        int32_t step0, int32_t steps, char *lds) {
        const int lane = threadIdx.x & (kWave - 1);
        const int wave = threadIdx.x / kWave;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

        // a load covers 8 rows of 128 bytes; lane l fills unit l % 8 of row
        // l / 8 in LDS, which holds unit (l % 8) ^ (row % 8) of memory
        const char *from[kLoads];
        const int unit = (lane & 7) ^ (lane >> 3);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const Operand &o = i < kLoadsA ? a : b;
            const int r = i < kLoadsA ? row0 + (wave * kLoadsA + i) * 8 + (lane >> 3)
                                      : col0 + (wave * kLoadsB + i - kLoadsA) * 8 + (lane >> 3);
            from[i] = o.base + int64_t(min(r, o.rows - 1)) * o.stride + unit * 16;
        }
        auto load = [&](int buffer, int32_t step) {
            char *to = lds + buffer * kBufferBytes;
            const int64_t off = int64_t(step) * kStepBytes;
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                __builtin_amdgcn_global_load_lds(
                    (global_void *)(from[i] + off),
                    (lds_void *)(to + (i < kLoadsA ? wave * kLoadsA + i : kRows / 8 + wave * kLoadsB + i - kLoadsA) * 1024),
                    16, 0, 0);
        };

        const int ra = wave / WN * TM * 32, rb = wave % WN * TN * 32;
        if (steps <= 0) return;
        // loads past the last step read the last again, into a buffer that
        // nothing reads: the loop has no branch, and counts its loads
        const int32_t last = step0 + steps - 1;
#pragma unroll
        for (int k = 0; k < kStages - 1; ++k) load(k, min(step0 + k, last));
        int buffer = 0;
        for (int32_t s = 0; s < steps; ++s) {
            // this step is in LDS once every wave's loads for it have come back
            // (those of later steps may be on their way), and every wave has
            // left the buffer that is loaded next
            __builtin_amdgcn_s_waitcnt(kWaitLoads);
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            const int next = buffer == 0 ? kStages - 1 : buffer - 1;
            const int32_t next_step = min(step0 + s + kStages - 1, last);
            if (!kSpread) load(next, next_step);

            const char *la = lds + buffer * kBufferBytes + ra * kStepBytes;
            const char *lb = lds + buffer * kBufferBytes + (kRows + rb) * kStepBytes;
            buffer = buffer + 1 == kStages ? 0 : buffer + 1;
            auto read = [&](const char *from, int tile, int q) {
                const int r = tile * 32 + (lane & 31);
                return *reinterpret_cast<const f16x8 *>(from + r * kStepBytes +
                                                        (((q * 2 + (lane >> 5)) ^ (r & 7)) * 16));
            };
            // the four quarters of a step, 16 values each; for kSplit the high
            // and low parts of the first 16 values, then of the second
            f16x8 fa[4][TM], fb[4][TN];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int at = P == Prec::kSplit ? (q >> 1) | ((q & 1) << 1) : q;
#pragma unroll
                for (int j = 0; j < TN; ++j) fb[q][j] = read(lb, j, at);
#pragma unroll
                for (int i = 0; i < TM; ++i) fa[q][i] = read(la, i, at);
            }
            if (kSpread) load(next, next_step);
            constexpr int kProducts = P == Prec::kSplit ? 6 : 4;
#pragma unroll
            for (int p = 0; p < kProducts; ++p) {
                const int qa = P == Prec::kSplit ? p / 3 * 2 + (p % 3 == 2) : p;
                const int qb = P == Prec::kSplit ? p / 3 * 2 + (p % 3 == 1) : p;
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j] = mfma(fa[qa][i], fb[qb][j], acc[i][j]);
            }
            // the first quarter's reads, then one read (and, spread, one load)
            // for every few products
            constexpr int kReads = 4 * (TM + TN), kFirst = TM + TN + 1;
            constexpr int kAll = kProducts * TM * TN * (P == Prec::kFp32 ? 4 : 1);
            constexpr int kSlots = kSpread && kLoads > kReads - kFirst ? kLoads : kReads - kFirst;
            constexpr int kEach = kAll * 3 / 4 / kSlots;
            __builtin_amdgcn_sched_group_barrier(0x100, kFirst, 0);
#pragma unroll
            for (int x = 0; x < kSlots; ++x) {
                __builtin_amdgcn_sched_group_barrier(0x8, kEach > 0 ? kEach : 1, 0);
                if (x < kReads - kFirst) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                if (kSpread && x < kLoads) __builtin_amdgcn_sched_group_barrier(0x20, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x8, kAll, 0);
        }
        __builtin_amdgcn_s_waitcnt(0x0f70);   // the loads that nothing reads
    }

    // The same of rows that are not laid out in steps: element (r, k) is
    // a[r * lda + k], k < len, at any alignment of the element type.  A lane
    // loads its own rows' values into registers, half of a step's 128 bytes of a
    // row, with zeros for values past len: the same values in the same order as
    // run's, and so the same sums.
    __device__ __forceinline__ void run_rows(const void *a, int64_t lda, int32_t rows_a, const void *b, int64_t ldb,
                                             int32_t rows_b, int32_t row0, int32_t col0, int32_t len) {
        static_assert(P == Prec::kBf16 || P == Prec::kFp32, "elements as they are stored");
        constexpr int kEach = P == Prec::kBf16 ? 8 : 4, kSize = 16 / kEach;   // elements of a load, bytes of one
        const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
        const char *from[TM + TN];
#pragma unroll
        for (int i = 0; i < TM + TN; ++i) {
            const int r = (lane & 31) + (i < TM ? row0 + (wave / WN * TM + i) * 32 : col0 + (wave % WN * TN + i - TM) * 32);
            from[i] = i < TM ? static_cast<const char *>(a) + min(r, rows_a - 1) * lda * kSize
                             : static_cast<const char *>(b) + min(r, rows_b - 1) * ldb * kSize;
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (i < TM)
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j][e] = 0.0f;
        }
        using u16x8u = std::conditional_t<P == Prec::kBf16, u16x8_at2, u16x8_at4>;
        f16x8 f[2][4][TM + TN];
        auto load = [&](f16x8 (&to)[4][TM + TN], int32_t k0) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int i = 0; i < TM + TN; ++i)
                    to[q][i] = __builtin_bit_cast(
                        f16x8, *reinterpret_cast<const u16x8u *>(from[i] + int64_t(k0 + (2 * q + (lane >> 5)) * kEach) * kSize));
        };
        auto load_last = [&](f16x8 (&to)[4][TM + TN], int32_t k0) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int32_t k = k0 + (2 * q + (lane >> 5)) * kEach;
#pragma unroll
                for (int i = 0; i < TM + TN; ++i) {
                    u16x8u v = {};
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (k + e * 2 / kSize < len)
                            v[e] = reinterpret_cast<const uint16_t *>(from[i] + int64_t(k) * kSize)[e];
                    to[q][i] = __builtin_bit_cast(f16x8, v);
                }
            }
        };
        auto multiply = [&](const f16x8 (&of)[4][TM + TN]) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j] = mfma(of[q][i], of[q][TM + j], acc[i][j]);
        };
        constexpr int kStep = 8 * kEach;
        const int32_t whole = len / kStep;
        if (whole > 0) load(f[0], 0);
        for (int32_t s = 0; s < whole; s += 2) {   // past the last, that one again
            load(f[1], min(s + 1, whole - 1) * kStep);
            multiply(f[0]);
            if (s + 1 == whole) break;
            load(f[0], min(s + 2, whole - 1) * kStep);
            multiply(f[1]);
        }
        if (whole * kStep < len) {
            load_last(f[0], whole * kStep);
            multiply(f[0]);
        }
    }
};

// A finished tile on its way out, a band of WM x 32 rows at a time through LDS,
// so that both a row's and a column's neighbours leave in 16-byte pieces.
// Straight from the accumulators (a lane holds one column) a row leaves two
// bytes a lane: 1024 x 4096 x 1024 then took 549 us for twelve matrices, with
// the product itself 240 of them; by bands 332.
template <class Tile>
struct Band {
    static constexpr int kRows = Tile::kRows / Tile::kTilesM;   // 32 of each row of waves
    static constexpr int kStride = Tile::kCols + 4;
    static constexpr int kGroups = Tile::kCols / 8;
    static constexpr int kUnits = kRows * kGroups / Tile::kThreads;   // of eight values, a thread's
    static constexpr int kBytes = kRows * kStride * 4;
    static_assert(kBytes <= Tile::kLdsBytes, "a band fits");
    static_assert(kUnits * Tile::kThreads == kRows * kGroups, "whole units");

    float *lds;

    // Row of the tile that row r of band i is.
    static __device__ __forceinline__ int tile_row(int i, int r) {
        return ((r >> 5) * Tile::kTilesM + i) * 32 + (r & 31);
    }
    // Unit k along the rows: eight columns from col() of row().
    static __device__ __forceinline__ int row(int k) { return (k * Tile::kThreads + int(threadIdx.x)) / kGroups; }
    static __device__ __forceinline__ int col(int k) { return (k * Tile::kThreads + int(threadIdx.x)) % kGroups * 8; }
    // Unit k along the columns: eight rows of the band from turned_row() of
    // column turned_col(); four neighbouring lanes have one column.
    static __device__ __forceinline__ int turned_row(int k) {
        const int u = k * Tile::kThreads + int(threadIdx.x);
        return u / (4 * Tile::kCols) * 32 + u % 4 * 8;
    }
    static __device__ __forceinline__ int turned_col(int k) {
        return (k * Tile::kThreads + int(threadIdx.x)) / 4 % Tile::kCols;
    }

    // acc[i][..] into LDS; a barrier on either side.
    template <int i>
    __device__ __forceinline__ void put(const Tile &tile) {
        __syncthreads();
        const int lane = threadIdx.x & (kWave - 1);
        const int first = (Tile::row_of(0, 0) / (Tile::kTilesM * 32)) * 32 + (lane >> 5) * 4;
#pragma unroll
        for (int j = 0; j < Tile::kTilesN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                lds[(first + (e >> 2) * 8 + (e & 3)) * kStride + Tile::col_of(j)] = tile.acc[i][j][e];
        __syncthreads();
    }
    __device__ __forceinline__ void get(int k, float (&v)[8]) const {
        const f32x4 *p = reinterpret_cast<const f32x4 *>(lds + row(k) * kStride + col(k));
        const f32x4 a = p[0], b = p[1];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            v[c] = a[c];
            v[4 + c] = b[c];
        }
    }
    __device__ __forceinline__ void set(int k, const float (&v)[8]) {
        f32x4 *p = reinterpret_cast<f32x4 *>(lds + row(k) * kStride + col(k));
        p[0] = f32x4{v[0], v[1], v[2], v[3]};
        p[1] = f32x4{v[4], v[5], v[6], v[7]};
    }
    __device__ __forceinline__ void get_turned(int k, float (&v)[8]) const {
        const float *p = lds + turned_row(k) * kStride + turned_col(k);
#pragma unroll
        for (int c = 0; c < 8; ++c) v[c] = p[c * kStride];
    }
};

// Calls f(integral constant i) for i = 0 .. N-1: the accumulators' first index
// has to be known to the compiler.
template <int N, int i = 0, class F>
__device__ __forceinline__ void each_band(F f) {
    if constexpr (i < N) {
        f(std::integral_constant<int, i>());
        each_band<N, i + 1>(f);
    }
}

// The shapes in use: 256 x 256 by eight waves (one workgroup a compute unit),
// 128 x 128 by four (two), 64 x 64 by four with two steps on their way (three).
template <Prec P>
using LargeTile = MfmaTile<P, 2, 4, 4, 2>;
template <Prec P>
using SmallTile = MfmaTile<P, 2, 2, 2, 2>;
template <Prec P>
using TinyTile = MfmaTile<P, 2, 2, 1, 1, 3>;

// For a few tokens against many rows: 64 x 32 TN by two waves, with two steps on
// their way in each of four workgroups a compute unit (TN = 1), or one in each
// of six where the fp32 instructions take longer than the loads.
template <Prec P, int TN>
using NarrowTile = MfmaTile<P, 2, 1, 1, TN, P == Prec::kFp32 ? 2 : 3>;

enum TileKind { kTiny, kSmall, kLarge };
constexpr int kTileKinds = 3;
constexpr int kTileSide[kTileKinds] = {64, 128, 256};

// What a product over tiles of one kind takes, in microseconds: `work` tiles
// times steps in all, `longest` steps of one tile.  Measured on kSplit steps:
// a tile's step takes 0.32, 0.63 and 1.7 us on its own, and 0.25, 0.76 and 2.4
// us of a compute unit where all are busy (270, 350 and 440 TFLOP/s), so that
// 256 x 1024 x 512 is fastest with the smallest kind (13.6 against 24.2 and 60
// us), 2048 x 4096 x 1024 with the middle one (63.6, 49.3, 64.8) and 4096 x
// 4096 x 4096 with the largest.
constexpr double kStepAlone[kTileKinds] = {0.32, 0.63, 1.7}, kStepBusy[kTileKinds] = {0.25, 0.76, 2.4};

inline double product_time(int kind, int64_t work, int64_t longest) {
    if (longest == 0) return 0.0;
    // rounds of the compute units, whole where few tiles share one
    double rounds = double(work) / double(longest) / device_cu_count();
    if (kind == kLarge && rounds > 1.0) rounds = ceil(rounds);
    if (kind == kSmall && rounds > 1.0) rounds = ceil(rounds * 2.0) / 2.0;
    return longest * fmax(rounds * kStepBusy[kind], kStepAlone[kind]);
}

inline TileKind best_tile(const int64_t (&work)[kTileKinds], int64_t longest) {
    TileKind best = kTiny;
    for (int k = kTiny + 1; k < kTileKinds; ++k)
        if (product_time(k, work[k], longest) < product_time(best, work[best], longest)) best = TileKind(k);
    return best;
}

// The workgroup's place in a grid whose consecutive places should share an
// XCD's cache: workgroups are dispatched to the eight XCDs in turn.
__device__ __forceinline__ uint32_t xcd_place(uint32_t id, uint32_t n) {
    const uint32_t x = id % kXcds, q = n / kXcds, r = n % kXcds;
    return x * q + min(x, r) + id / kXcds;
}

// Place t of a grid of rows x cols tiles, walked in bands of eight rows so
// that neighbours share the operands of eight tiles each way.
__device__ __forceinline__ void banded(uint32_t t, uint32_t rows, uint32_t cols, uint32_t &r, uint32_t &c) {
    constexpr uint32_t kBand = 8;
    const uint32_t band = t / (kBand * cols), in = t - band * kBand * cols;
    const uint32_t high = min(kBand, rows - band * kBand);
    r = band * kBand + in % high;
    c = in / high;
}

}  // namespace efs
