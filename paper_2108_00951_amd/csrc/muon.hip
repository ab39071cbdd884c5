// Orthogonalised update of weight matrices (the Muon form of the model update).
//
//   m <- beta m + avg ;  u = avg + beta m (Nesterov) or m        element by element
//   X0 = u / (||u||_F + eps), as an m x n matrix with m <= n (u^T where it is taller)
//   five times:  A = X X^T ;  B = b A + c A A ;  X <- a X + B X
//   x <- (1 - gamma decay) x - gamma sqrt(max(1, rows / cols)) X
//
// Every singular value of X0 goes through the odd polynomial
// a s + b s^3 + c s^5 of the step and tends to 1; the singular vectors stay.
//
// X and A are kept as split values (mfma_tile.hpp) scaled by 2^14, B by 2^12.
// No entry of a matrix is larger than its largest singular value, and with
// ||X0||_F <= 1 those of the iterates stay below 1.3, A's below 1.5 and B's
// (b s^2 + c s^4) below 3, so that the fp16 parts (65504 at most) do not
// overflow, and hold 22 bits of every entry above 2^-17 of that.  (At 2^10 the
// entries of a matrix whose norm eps outweighs lost some.)  Three fp16 products give the error of fp32 products
// (1.0-1.1 times at 256 x 256 to 256 x 1024, low-rank and ill-conditioned
// inputs among them); one product gives 1e-3, and iterating on the small Gram
// matrix alone, cheaper for wide matrices, 1e-4 to 1e-1.  a X is added in fp32
// to the product B X and not folded into B: twice the error otherwise where
// the singular values differ much.
//
// A call is a setup launch (the table of matrices), two passes over the
// elements (momentum and sums of squares; the split operands) and three
// products a step over all matrices together.  X X^T and A A are symmetric:
// tiles on and below the diagonal are computed and written to both places, so
// that a step is 3 m^2 n + m^3 operations instead of 4 m^2 n + 2 m^3.  X is
// kept along both axes, since X X^T sums over one and B X over the other (one
// copy, turned by LDS reads for B X, saves a third of what B X moves, but its
// loop runs 10 % slower: 2.75 against 3.05 ms for five matrices of 134 M, and
// no difference at 2600 x 650).
#include "mfma_tile.hpp"
#include "launch.hpp"

#include <math.h>

namespace efs {

namespace {

constexpr float kScale = 0x1p14f;          // of X and A in their split form
constexpr float kUnscale = 0x1p-14f;
constexpr float kScaleB = 0x1p12f;         // of B
constexpr float kUnscaleB = 0x1p-12f;
constexpr int kSumBlock = 256;
constexpr int kMaxChunks = 1024;           // partial sums of one matrix
constexpr int64_t kChunkMin = 4096;        // elements
constexpr int kPackTile = 64;
constexpr int kSetupBlock = 256;

enum Product { kGram, kPolynomial, kApply, kLast };

// Running counts over the matrices before one: where its tiles, sums and
// operands start.
struct Place {
    int64_t bytes;      // operands
    int32_t sym[kTileKinds];    // tiles on and below the diagonal of m x m
    int32_t full[kTileKinds];   // tiles of m x n
    int32_t chunks;     // partial sums
    int32_t packs;      // 64 x 64 tiles of the caller's matrix
    int32_t units;      // workgroups of a split X X^T
    int32_t parts;      // of which leave partial sums
};

struct Mat {
    int64_t src, dst;           // first element in the caller's arrays
    int32_t rows, cols;         // the caller's
    Place at;
};

struct Given {   // what the host passes of a matrix
    int64_t offset;
    int32_t rows, cols;
};
constexpr int kGivenPerLaunch = 192;
struct GivenArray {
    Given mat[kGivenPerLaunch];
};

__host__ __device__ inline int64_t low(const int32_t r, const int32_t c) { return r < c ? r : c; }
__host__ __device__ inline int64_t high(const int32_t r, const int32_t c) { return r < c ? c : r; }

__host__ __device__ inline int32_t chunks_of(int64_t size) {
    const int64_t c = (size + kChunkMin - 1) / kChunkMin;
    return int32_t(c < kMaxChunks ? c : kMaxChunks);
}

// Elements of one partial sum: whole pieces of eight.
__host__ __device__ inline int64_t chunk_of(int64_t size) {
    const int64_t c = chunks_of(size);
    return ((size + c - 1) / c + 7) / 8 * 8;
}

// Bytes of one X, X^T, A or B.
__host__ __device__ inline int64_t x_bytes(int64_t rows, int64_t len) { return rows * row_bytes<Prec::kSplit>(len); }

__host__ __device__ inline int64_t operand_bytes(int32_t rows, int32_t cols) {
    const int64_t m = low(rows, cols), n = high(rows, cols);
    return 2 * x_bytes(m, n) + 2 * x_bytes(n, m) + 2 * x_bytes(m, m);
}

// How many workgroups share a tile of X X^T, with about `most` steps each.
__host__ __device__ inline int32_t splits_of(int32_t rows, int32_t cols, int32_t most) {
    const int64_t steps = steps_of<Prec::kSplit>(high(rows, cols));
    const int64_t s = (steps + most / 2) / most;
    return int32_t(s < 1 ? 1 : s);
}

// Tiles along an axis (len + side can pass 32 bits).
__host__ __device__ inline int32_t tiles_along(int64_t len, int32_t side) { return int32_t((len + side - 1) / side); }

// `most`: steps of X X^T in one workgroup.
__host__ __device__ inline void advance(Place &p, int32_t rows, int32_t cols, int32_t most) {
    const int32_t m = int32_t(low(rows, cols)), n = int32_t(high(rows, cols));
    p.bytes += operand_bytes(rows, cols);
    for (int k = 0; k < kTileKinds; ++k) {
        const int32_t tm = tiles_along(m, kTileSide[k]), tn = tiles_along(n, kTileSide[k]);
        p.sym[k] += tm * (tm + 1) / 2;
        p.full[k] += tm * tn;
    }
    p.chunks += chunks_of(int64_t(rows) * cols);
    p.packs += tiles_along(rows, kPackTile) * tiles_along(cols, kPackTile);
    const int32_t tm = tiles_along(m, kTileSide[kTiny]), splits = splits_of(rows, cols, most);
    p.units += tm * (tm + 1) / 2 * splits;
    p.parts += splits > 1 ? tm * (tm + 1) / 2 * splits : 0;
}

__host__ __device__ inline void add(Place &p, const Place &q, int32_t times) {
    p.bytes += q.bytes * times;
    for (int k = 0; k < kTileKinds; ++k) {
        p.sym[k] += q.sym[k] * times;
        p.full[k] += q.full[k] * times;
    }
    p.chunks += q.chunks * times;
    p.packs += q.packs * times;
    p.units += q.units * times;
    p.parts += q.parts * times;
}

// Workspace: the table, the norms' partial sums, the operands, the partial
// sums of X X^T.
struct Layout {
    int64_t table, sums, operands, parts, total;
};

inline int64_t round256(int64_t v) { return (v + 255) / 256 * 256; }

inline Layout layout_of(int64_t nmat, const Place &end) {
    Layout l;
    l.table = 0;
    l.sums = round256((nmat + 1) * int64_t(sizeof(Mat)));
    l.operands = l.sums + round256(int64_t(end.chunks) * 8);
    l.parts = l.operands + round256(end.bytes);
    l.total = l.parts + int64_t(end.parts) * kTileSide[kTiny] * kTileSide[kTiny] * 4;
    return l;
}

// The caller's arrays, as both passes and the last product see them.
struct Io {
    const void *in;        // avg, or the matrices to orthogonalise
    float *m;              // momentum; null without
    void *out;             // x, or the orthogonalised matrices
    int64_t ld_in, ld_out; // elements between rows; 0: the matrix's own columns
    float beta, gamma, keep;   // keep = 1 - gamma decay
    float eps;
    int nesterov, bf16;
};

// A matrix's operands in the workspace: X twice, X^T twice, A, B.
struct Operands {
    char *base;
    int64_t m, n;
    int64_t x_row, t_row;   // bytes of a row of X (n values) and of X^T, A, B (m values)
    __device__ Operands(char *operands, const Mat &mat)
        : base(operands + mat.at.bytes), m(low(mat.rows, mat.cols)), n(high(mat.rows, mat.cols)),
          x_row(row_bytes<Prec::kSplit>(n)), t_row(row_bytes<Prec::kSplit>(m)) {}
    __device__ char *x(int k) const { return base + k * m * x_row; }
    __device__ char *xt(int k) const { return base + 2 * m * x_row + k * n * t_row; }
    __device__ char *a() const { return xt(2); }
    __device__ char *b() const { return a() + m * t_row; }
    __device__ Operand x_operand(int k) const { return Operand{x(k), x_row, int32_t(m)}; }
    __device__ Operand xt_operand(int k) const { return Operand{xt(k), t_row, int32_t(n)}; }
    __device__ Operand a_operand() const { return Operand{a(), t_row, int32_t(m)}; }
    __device__ Operand b_operand() const { return Operand{b(), t_row, int32_t(m)}; }
};

// The table.  Entry nmat holds the totals.  `first`: the matrices before
// `given`, already in the table.  With `given.mat` unused (batch), the matrices
// are alike and `stride` elements apart.
__global__ __launch_bounds__(kSetupBlock) void muon_setup_kernel(Mat *table, GivenArray given, int32_t first,
                                                                 int32_t count, int32_t batch, int32_t most,
                                                                 int64_t stride_in, int64_t stride_out) {
    if (batch) {   // alike: each place is a multiple
        for (int32_t i = blockIdx.x * kSetupBlock + threadIdx.x; i <= count; i += gridDim.x * kSetupBlock) {
            Place one = {};
            advance(one, given.mat[0].rows, given.mat[0].cols, most);
            Mat &t = table[i];
            t.src = i * stride_in;
            t.dst = i * stride_out;
            t.rows = given.mat[0].rows;
            t.cols = given.mat[0].cols;
            t.at = Place{};
            add(t.at, one, i);
        }
        return;
    }
    // at most kGivenPerLaunch: running sums by doubling distances
    __shared__ Place s_sum[kSetupBlock];
    const int32_t i = threadIdx.x;
    Place p = {};
    if (i == 0 && first > 0) p = table[first].at;
    if (i > 0 && i <= count) advance(p, given.mat[i - 1].rows, given.mat[i - 1].cols, most);
    for (int32_t d = 1; d <= count; d *= 2) {
        s_sum[i] = p;
        __syncthreads();
        if (i >= d) add(p, s_sum[i - d], 1);
        __syncthreads();
    }
    if (i > count) return;
    // entry first + count is the next launch's first, or the totals
    Mat &t = table[first + i];
    if (i < count) {
        t.src = given.mat[i].offset;
        t.dst = given.mat[i].offset;
        t.rows = given.mat[i].rows;
        t.cols = given.mat[i].cols;
    }
    if (i > 0 || first == 0) t.at = p;
}

// The last matrix whose count starts at or before `at`: none of them is
// empty, so the starts differ.  A wave looks at 64 of them at a time (every
// look is a way to memory and back before the kernel can start).
template <class F>
__device__ __forceinline__ int32_t matrix_of(const Mat *__restrict__ table, int32_t nmat, int32_t at, F start) {
    const int32_t lane = threadIdx.x & (kWave - 1);
    int32_t lo = 0, left = nmat;
    while (left > 1) {
        const int32_t step = (left + kWave - 1) / kWave, mine = lane * step;
        const bool before = mine < left && start(table[lo + mine].at) <= at;
        const int32_t passed = (__popcll(__ballot(before)) - 1) * step;
        lo += passed;
        left = min(step, left - passed);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

__device__ __forceinline__ float direction(const Io &io, float avg, float m) {
    return io.nesterov ? __fadd_rn(avg, __fmul_rn(io.beta, m)) : m;
}

__device__ __forceinline__ float read_in(const Io &io, int64_t i) {
    return io.bf16 ? float(static_cast<const __bf16 *>(io.in)[i]) : static_cast<const float *>(io.in)[i];
}

typedef __bf16 bf16x8u __attribute__((ext_vector_type(8), aligned(2)));

// Eight neighbours, at any alignment.
__device__ __forceinline__ void load8(const float *from, float (&v)[8]) {
    const f32x4u *p = reinterpret_cast<const f32x4u *>(from);
    const f32x4u a = p[0], b = p[1];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        v[k] = a[k];
        v[4 + k] = b[k];
    }
}

__device__ __forceinline__ void read_in8(const Io &io, int64_t i, float (&v)[8]) {
    if (io.bf16) {
        const bf16x8u a = *reinterpret_cast<const bf16x8u *>(static_cast<const __bf16 *>(io.in) + i);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = float(a[k]);
    } else {
        load8(static_cast<const float *>(io.in) + i, v);
    }
}

// What a matrix's values are divided by, from the sum of their squares.  Where 32
// bits do not reach to it (finite values near the largest), both are taken in
// units of 2^64.
struct Norm {
    float unit, norm;
    __device__ __forceinline__ float divide(float v) const { return __fdiv_rn(__fmul_rn(v, unit), norm); }
};

__device__ __forceinline__ Norm norm_of(double sum, float eps) {
    const float norm = __fadd_rn(float(sqrt(sum)), eps);
    if (norm == INFINITY && sum < INFINITY) return Norm{0x1p-64f, float((sqrt(sum) + double(eps)) * 0x1p-64)};
    return Norm{1.0f, norm};
}

// gamma sqrt(max(1, rows / cols))
__device__ __forceinline__ float step_scale(const Io &io, int32_t rows, int32_t cols) {
    return __fmul_rn(io.gamma, sqrtf(fmaxf(1.0f, __fdiv_rn(float(rows), float(cols)))));
}

// x after a step along o.
__device__ __forceinline__ float step_of(const Io &io, float x, float o, float scale) {
    return __fsub_rn(__fmul_rn(io.keep, x), __fmul_rn(scale, o));
}

// The orthogonalised value o of element `at`: into x, or out.
__device__ __forceinline__ void write_out(const Io &io, int64_t at, float o, float scale) {
    if (io.m != nullptr) {
        float *x = static_cast<float *>(io.out) + at;
        *x = step_of(io, *x, o, scale);
    } else if (io.bf16) {
        static_cast<__bf16 *>(io.out)[at] = __bf16(o);   // the one rounding to 8 bits
    } else {
        static_cast<float *>(io.out)[at] = o;
    }
}

// Eight of a row's values, scaled by 2^14, of which `left` are the matrix's.
__device__ __forceinline__ void write_out8(const Io &io, int64_t at, int32_t left, const float (&v)[8], float scale) {
    if (left < 8) {
        for (int e = 0; e < 8; ++e)
            if (e < left) write_out(io, at + e, __fmul_rn(v[e], kUnscale), scale);
        return;
    }
    if (io.bf16) {
        bf16x8u o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = __bf16(__fmul_rn(v[e], kUnscale));
        *reinterpret_cast<bf16x8u *>(static_cast<__bf16 *>(io.out) + at) = o;
        return;
    }
    f32x4u *p = reinterpret_cast<f32x4u *>(static_cast<float *>(io.out) + at);
    f32x4u o[2];
    if (io.m != nullptr) {
        o[0] = p[0];
        o[1] = p[1];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float u = __fmul_rn(v[e], kUnscale);
        o[e / 4][e % 4] = io.m != nullptr ? step_of(io, o[e / 4][e % 4], u, scale) : u;
    }
    p[0] = o[0];
    p[1] = o[1];
}

// First pass: the momentum in place, and each chunk's sum of u^2 in binary64
// (a fixed order: the same sum every time).  Bound by HBM: 300 us for 134 M
// elements (12 bytes each: 5.4 TB/s).
__global__ __launch_bounds__(kSumBlock) void muon_momentum_kernel(const Mat *__restrict__ table, int32_t nmat, Io io,
                                                                  double *sums) {
    __shared__ double s_f64[kWaves];
    const int32_t mi = matrix_of(table, nmat, blockIdx.x, [](const Place &p) { return p.chunks; });
    const Mat &mat = table[mi];
    const int64_t size = int64_t(mat.rows) * mat.cols;
    const int64_t chunk = chunk_of(size);
    const int64_t lo = chunk * (int64_t(blockIdx.x) - mat.at.chunks);
    const int64_t hi = min(size, lo + chunk);
    double sum = 0.0;
    if (io.m != nullptr) {
        const float *avg = static_cast<const float *>(io.in) + mat.src;
        float *m = io.m + mat.src;
        int64_t i = lo + int64_t(threadIdx.x) * 4;
        for (; i + 4 <= hi; i += kSumBlock * 4) {
            const f32x4u g = *reinterpret_cast<const f32x4u *>(avg + i);
            f32x4u v = *reinterpret_cast<const f32x4u *>(m + i);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                v[c] = __fadd_rn(__fmul_rn(io.beta, v[c]), g[c]);
                const double u = direction(io, g[c], v[c]);
                sum += u * u;
            }
            *reinterpret_cast<f32x4u *>(m + i) = v;
        }
        for (; i < hi; ++i) {   // the last matrix elements, fewer than four, of one thread
            const float g = avg[i];
            const float v = __fadd_rn(__fmul_rn(io.beta, m[i]), g);
            m[i] = v;
            const double u = direction(io, g, v);
            sum += u * u;
        }
    } else {
        const int64_t ld = io.ld_in ? io.ld_in : mat.cols;
#pragma unroll 2
        for (int64_t i = lo + int64_t(threadIdx.x) * 8; i < hi; i += kSumBlock * 8) {
            uint32_t r = uint32_t(i) / uint32_t(mat.cols), c = uint32_t(i) - r * uint32_t(mat.cols);
            float v[8] = {};
            if (c + 8 <= uint32_t(mat.cols)) {
                read_in8(io, mat.src + r * ld + c, v);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) {   // from one row into the next
                    if (i + k < hi) v[k] = read_in(io, mat.src + r * ld + c);
                    if (++c == uint32_t(mat.cols)) {
                        c = 0;
                        ++r;
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) sum += double(v[k]) * double(v[k]);
        }
    }
    sum = block_sum_f64(sum, s_f64);
    if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}

// Second pass: u / (||u|| + eps) as X and X^T, a 64 x 64 tile of the caller's
// matrix at a time (turned in LDS; its values are on their way while the norm's
// sums are added).  Bound by HBM: 441 us for 134 M elements
// (16 bytes each, with momentum: 4.9 TB/s).  Eight neighbouring lanes write two
// whole lines of a row, turned or not; with a row a lane the turned half took the
// whole to 563 us.
__global__ __launch_bounds__(kSumBlock) void muon_pack_kernel(const Mat *__restrict__ table, int32_t nmat, Io io,
                                                              const double *sums, char *operands) {
    __shared__ double s_f64[kWaves];
    __shared__ Norm s_norm;
    __shared__ float tile[kPackTile][kPackTile + 1];
    const int tid = threadIdx.x;
    const int32_t mi = matrix_of(table, nmat, blockIdx.x, [](const Place &p) { return p.packs; });
    const Mat &mat = table[mi];
    const int32_t across = tiles_along(mat.cols, kPackTile);
    const int32_t t = int32_t(blockIdx.x) - mat.at.packs;
    const int32_t r0 = t / across * kPackTile, c0 = t % across * kPackTile;
    const int64_t ld = io.ld_in ? io.ld_in : mat.cols;
    constexpr int kPieces = kPackTile * kPackTile / 8 / kSumBlock;   // of a thread, eight values each
    float in[kPieces][8], mom[kPieces][8];
#pragma unroll
    for (int q = 0; q < kPieces; ++q) {
        const int i = q * kSumBlock + tid;
        const int32_t r = r0 + i / 8, c = c0 + i % 8 * 8;
        const int64_t at = mat.src + r * ld + c;
#pragma unroll
        for (int k = 0; k < 8; ++k) in[q][k] = mom[q][k] = 0.0f;
        if (r >= mat.rows) continue;
        if (c + 8 <= mat.cols) {
            read_in8(io, at, in[q]);
            if (io.m != nullptr) load8(io.m + at, mom[q]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (c + k >= mat.cols) continue;
                in[q][k] = read_in(io, at + k);
                if (io.m != nullptr) mom[q][k] = io.m[at + k];
            }
        }
    }
    const int32_t nsums = chunks_of(int64_t(mat.rows) * mat.cols);
    double sum = 0.0;
    for (int32_t i = tid; i < nsums; i += kSumBlock) sum += sums[mat.at.chunks + i];
    sum = block_sum_f64(sum, s_f64);
    if (tid == 0) s_norm = norm_of(sum, io.eps);
    __syncthreads();
    const Norm norm = s_norm;
#pragma unroll
    for (int q = 0; q < kPieces; ++q) {
        const int i = q * kSumBlock + tid;
        const int32_t r = r0 + i / 8, c = c0 + i % 8 * 8;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float v = io.m != nullptr ? direction(io, in[q][k], mom[q][k]) : in[q][k];
            tile[i / 8][i % 8 * 8 + k] = r < mat.rows && c + k < mat.cols ? __fmul_rn(norm.divide(v), kScale) : 0.0f;
        }
    }
    __syncthreads();

    const Operands op(operands, mat);
    const bool wide = mat.rows <= mat.cols;
    // along the caller's rows, then along its columns; a thread writes eight
    // values of a row, both parts
#pragma unroll
    for (int turn = 0; turn < 2; ++turn) {
        const bool to_x = wide != bool(turn);
        char *base = to_x ? op.x(0) : op.xt(0);
        const int64_t stride = to_x ? op.x_row : op.t_row;
        const int32_t row_first = turn ? c0 : r0, col_first = turn ? r0 : c0;
        const int32_t row_end = turn ? mat.cols : mat.rows;
        const int32_t col_end = row_values<Prec::kSplit>(turn ? mat.rows : mat.cols);
        for (int i = tid; i < kPackTile * 8; i += kSumBlock) {
            const int r = i / 8, c = i % 8 * 8;
            if (row_first + r >= row_end || col_first + c >= col_end) continue;
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = turn ? tile[c + k][r] : tile[r][c + k];
            store_split8(base + (row_first + r) * stride, col_first + c, v);
        }
    }
}

// Where a tile's result goes, and what is added to it.
struct Target {
    int32_t row0, col0;
    bool diagonal;   // of a symmetric result: its other half is in the tile itself
    bool turned;     // rows of the result are X's columns
};

// Tile t on or below the diagonal.
template <class Tile>
__device__ __forceinline__ Target symmetric_tile(uint32_t t) {
    uint32_t r = uint32_t((sqrtf(8.0f * float(t) + 1.0f) - 1.0f) * 0.5f);
    while (r * (r + 1) / 2 > t) --r;
    while ((r + 1) * (r + 2) / 2 <= t) ++r;
    const uint32_t c = t - r * (r + 1) / 2;
    return Target{int32_t(r) * Tile::kRows, int32_t(c) * Tile::kCols, r == c, false};
}

// A product's tile on its way out.
template <int kProduct, class Tile>
__device__ __forceinline__ void finish(const Tile &tile, const Target &target, const Mat &mat, const Operands &op,
                                       int cur, float a, float b, float c, const Io &io, char *lds) {
    constexpr bool kSym = kProduct == kGram || kProduct == kPolynomial;
    const int32_t m = int32_t(op.m), n = int32_t(op.n);
    const bool turned = kProduct == kLast && target.turned;
    const int32_t row0 = target.row0, col0 = target.col0;
    const int32_t rows = turned ? n : m, cols = kSym ? m : turned ? m : n;
    const int32_t padded_cols = row_values<Prec::kSplit>(cols), padded_rows = row_values<Prec::kSplit>(rows);
    // what is added to the product: A, or X (turned: X^T)
    const char *add = kProduct == kPolynomial ? op.a() : turned ? op.xt(cur) : op.x(cur);
    const int64_t add_row = kProduct == kPolynomial || turned ? op.t_row : op.x_row;
    const float f_add = kProduct == kPolynomial ? b * (kScaleB * kUnscale) : a;
    const float f_acc = kProduct == kGram ? kUnscale : kProduct == kPolynomial ? c * (kScaleB * kUnscale * kUnscale) : kUnscaleB;
    // results: along the rows, and turned
    char *to = kProduct == kGram ? op.a() : kProduct == kPolynomial ? op.b() : op.x(cur ^ 1);
    char *to_t = kProduct == kGram ? op.a() : kProduct == kPolynomial ? op.b() : op.xt(cur ^ 1);
    const int64_t to_row = kSym ? op.t_row : op.x_row;
    const bool mirror = kProduct != kLast && !target.diagonal;
    const float scale = step_scale(io, mat.rows, mat.cols);
    const int64_t ld_out = io.ld_out ? io.ld_out : mat.cols;

    using Out = Band<Tile>;
    Out band{reinterpret_cast<float *>(lds)};
    each_band<Tile::kTilesM>([&](auto index) {
        constexpr int i = decltype(index)::value;
        f16x8 hi[Out::kUnits], lo[Out::kUnits];   // on their way while the band is put
        if (kProduct != kGram) {
#pragma unroll
            for (int k = 0; k < Out::kUnits; ++k) {
                const int32_t row = row0 + Out::tile_row(i, Out::row(k)), col = col0 + Out::col(k);
                if (row < rows && col < padded_cols) {
                    const char *p = add + row * add_row + split_offset(col);
                    hi[k] = *reinterpret_cast<const f16x8 *>(p);
                    lo[k] = *reinterpret_cast<const f16x8 *>(p + 64);
                }
            }
        }
        band.template put<i>(tile);
#pragma unroll
        for (int k = 0; k < Out::kUnits; ++k) {
            const int32_t row = row0 + Out::tile_row(i, Out::row(k)), col = col0 + Out::col(k);
            float v[8];
            band.get(k, v);
            const bool in = row < rows && col < padded_cols;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = __fmul_rn(v[e], f_acc);
                if (kProduct != kGram)
                    v[e] = __fadd_rn(__fmul_rn(f_add, __fadd_rn(float(hi[k][e]), float(lo[k][e]))), v[e]);
                if (!in || col + e >= cols) v[e] = 0.0f;   // the padding of both results
            }
            if (kProduct == kLast) {
                if (in) write_out8(io, mat.dst + row * ld_out + col, cols - col, v, scale);
            } else {
                if (mirror) band.set(k, v);
                if (in) store_split8(to + row * to_row, col, v);
            }
        }
        if (!mirror) return;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < Out::kUnits; ++k) {
            const int32_t row = row0 + Out::tile_row(i, Out::turned_row(k)), col = col0 + Out::turned_col(k);
            if (row >= padded_rows || col >= cols) continue;
            float v[8];
            band.get_turned(k, v);
            store_split8(to_t + col * op.t_row, row, v);
        }
    });
}

// One product of a step over all matrices, a tile a workgroup.
//   kGram        A = X X^T             tiles on and below the diagonal
//   kPolynomial  B = b A + c A A       the same
//   kApply       X' = a X + B X        into the other pair of buffers
//   kLast        the same, into the caller's x or out
// `cur`: which pair of buffers holds X.
// Large matrices are bound by the matrix cores: four of 4096 x 4096 and one of
// 4096 x 16384 take 1585 us for X X^T and 1022 for B on and below the diagonal
// (368 and 357 TFLOP/s of those tiles), and 2700 for a X + B X (407).  A matrix
// of few steps is bound by the stream of results instead: five gates of
// 2600 x 650 end B X in 12 bytes an element, 69 us in all.
template <int kProduct, class Tile>
__global__ __launch_bounds__(Tile::kThreads, Tile::kWavesPerSimd) void muon_product_kernel(
    const Mat *__restrict__ table, int32_t nmat, char *operands, int cur, float a, float b, float c, Io io) {
    __shared__ __align__(16) char lds[Tile::kLdsBytes];
    constexpr int kKind = Tile::kRows == kTileSide[kTiny] ? kTiny : Tile::kRows == kTileSide[kSmall] ? kSmall : kLarge;
    constexpr bool kSym = kProduct == kGram || kProduct == kPolynomial;
    static_assert(Tile::kRows == Tile::kCols, "tiles of the diagonal are square");
    const int32_t mi = matrix_of(table, nmat, blockIdx.x,
                                 [](const Place &p) { return kSym ? p.sym[kKind] : p.full[kKind]; });
    const Mat &mat = table[mi];
    const Operands op(operands, mat);
    const int32_t m = int32_t(op.m), n = int32_t(op.n);
    // a matrix's neighbouring tiles on one XCD; every XCD has a share of every matrix
    const Place &end = table[mi + 1].at;
    const int32_t begin = kSym ? mat.at.sym[kKind] : mat.at.full[kKind];
    const uint32_t t = xcd_place(blockIdx.x - begin, (kSym ? end.sym[kKind] : end.full[kKind]) - begin);
    Target target;
    if (kSym) {
        target = symmetric_tile<Tile>(t);
    } else {
        // the caller's orientation in the last product: its rows are X's
        // columns where the matrix is tall
        target.turned = kProduct == kLast && mat.rows > mat.cols;
        target.diagonal = false;
        const uint32_t tm = tiles_along(m, Tile::kRows), tn = tiles_along(n, Tile::kCols);
        uint32_t r, q;
        if (target.turned) banded(t, tn, tm, r, q);
        else banded(t, tm, tn, r, q);
        target.row0 = int32_t(r) * Tile::kRows;
        target.col0 = int32_t(q) * Tile::kCols;
    }

    Operand left, right;
    int64_t steps = steps_of<Prec::kSplit>(m);
    if (kProduct == kGram) {
        left = right = op.x_operand(cur);
        steps = steps_of<Prec::kSplit>(n);
    } else if (kProduct == kPolynomial) {
        left = right = op.a_operand();
    } else {
        left = target.turned ? op.xt_operand(cur) : op.b_operand();
        right = target.turned ? op.b_operand() : op.xt_operand(cur);
    }
    Tile tile;
    tile.run(left, right, target.row0, target.col0, 0, int32_t(steps), lds);
    finish<kProduct>(tile, target, mat, op, cur, a, b, c, io, lds);
}

// X X^T of few tiles: several workgroups share a long tile's steps and leave
// partial sums, as their registers hold them; the join adds them in order (five
// gates of 2600 x 650: 39 us and 7 for the join).
template <class Tile>
__global__ __launch_bounds__(Tile::kThreads, Tile::kWavesPerSimd) void muon_gram_kernel(const Mat *__restrict__ table, int32_t nmat,
                                                                                        char *operands, int cur,
                                                                                        int32_t most, f32x4 *parts,
                                                                                        Io io) {
    __shared__ __align__(16) char lds[Tile::kLdsBytes];
    static_assert(Tile::kRows == kTileSide[kTiny] && Tile::kTilesM == 1 && Tile::kTilesN == 1, "places count these");
    const int32_t mi = matrix_of(table, nmat, blockIdx.x, [](const Place &p) { return p.units; });
    const Mat &mat = table[mi];
    const Operands op(operands, mat);
    const uint32_t units = uint32_t(table[mi + 1].at.units - mat.at.units);
    const uint32_t splits = uint32_t(splits_of(mat.rows, mat.cols, most)), tiles = units / splits;
    const uint32_t u = xcd_place(blockIdx.x - mat.at.units, units);
    const uint32_t t = u % tiles, split = u / tiles;
    const Target target = symmetric_tile<Tile>(t);
    const int64_t steps = steps_of<Prec::kSplit>(op.n);
    const int32_t lo = int32_t(steps * split / splits), hi = int32_t(steps * (split + 1) / splits);
    const Operand x = op.x_operand(cur);
    Tile tile;
    tile.run(x, x, target.row0, target.col0, lo, hi - lo, lds);
    if (splits == 1) {
        finish<kGram>(tile, target, mat, op, cur, 0.0f, 0.0f, 0.0f, io, lds);
        return;
    }
    f32x4 *to = parts + (int64_t(mat.at.parts) + t * splits + split) * (4 * Tile::kThreads);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const f32x16 &v = tile.acc[0][0];
        to[q * Tile::kThreads + threadIdx.x] = f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
    }
}

template <class Tile>
__global__ __launch_bounds__(Tile::kThreads, Tile::kWavesPerSimd) void muon_gram_join_kernel(
    const Mat *__restrict__ table, int32_t nmat, char *operands, int cur, int32_t most, const f32x4 *parts, Io io) {
    __shared__ __align__(16) char lds[Band<Tile>::kBytes];
    const int32_t mi = matrix_of(table, nmat, blockIdx.x, [](const Place &p) { return p.sym[kTiny]; });
    const Mat &mat = table[mi];
    const int32_t splits = splits_of(mat.rows, mat.cols, most);
    if (splits == 1) return;
    const Operands op(operands, mat);
    const uint32_t t = blockIdx.x - mat.at.sym[kTiny];
    const f32x4 *from = parts + (int64_t(mat.at.parts) + int64_t(t) * splits) * (4 * Tile::kThreads) + threadIdx.x;
    Tile tile;
#pragma unroll
    for (int e = 0; e < 16; ++e) tile.acc[0][0][e] = 0.0f;
    for (int32_t s = 0; s < splits; ++s)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f32x4 v = from[(s * 4 + q) * Tile::kThreads];
#pragma unroll
            for (int e = 0; e < 4; ++e) tile.acc[0][0][4 * q + e] = __fadd_rn(tile.acc[0][0][4 * q + e], v[e]);
        }
    finish<kGram>(tile, symmetric_tile<Tile>(t), mat, op, cur, 0.0f, 0.0f, 0.0f, io, lds);
}

// ---- small matrices -------------------------------------------------------
// A matrix whose X fits in LDS as fp32 is one workgroup's from its gradient to
// its update: one launch, nothing in the workspace, the fp32 matrix
// instructions (16 x 16 x 4).  Rows are padded with zeros to 16 values and lie
// 4 values further apart, so that the 16 rows x 4 values that an instruction
// takes are in 64 different banks.  Bound by that one workgroup's instructions and
// round trips through LDS.  us, against tiles: 64 x 64 30 and 62, 256 of them 33 and
// 88; 2,048 of 32 x 32 68 and 201; 256 of 64 x 300 96 and 183; but one of 64 x 300 90
// and 80, of 64 x 450 129 and 86, of 16 x 2000 148 and 99.
constexpr int kLdsBlock = 512;
constexpr int kLdsWaves = kLdsBlock / kWave;
constexpr int kLdsMaxM = 64;
constexpr int kLdsFloats[2] = {8 << 10, 39 << 10};   // 32 KB: four a compute unit; 156 KB

// (past 32 bits for the longest axes, which no workgroup takes)
__host__ __device__ inline int64_t round16(int64_t v) { return (v + 15) / 16 * 16; }

// LDS of a matrix: X, A, B.
__host__ __device__ inline int64_t lds_floats(int32_t rows, int32_t cols) {
    const int64_t m = round16(low(rows, cols)), n = round16(high(rows, cols));
    return m * (n + 4) + 2 * m * (m + 4);
}

// 0, 1: the size of the workgroup that takes the matrix; -1: none does.
__host__ inline int lds_class(int32_t rows, int32_t cols) {
    if (low(rows, cols) > kLdsMaxM) return -1;
    const int64_t f = lds_floats(rows, cols);
    return f <= kLdsFloats[0] ? 0 : f <= kLdsFloats[1] ? 1 : -1;
}

// Two 16 x 16 tiles of one column of tiles: the sum over k < len (a multiple of
// 16) of left(i, row, k) right(k, col).  Lane l holds row l % 16 of the left,
// column l % 16 of the right, k = l / 16; of the result column l % 16, rows
// l / 16 * 4 + e.  The next 16 values of k are on their way from LDS while the
// present ones are multiplied.
template <class L, class R>
__device__ __forceinline__ void mfma_f32(int32_t len, f32x4 (&acc)[2], L left, R right) {
    const int row = threadIdx.x & 15, four = (threadIdx.x & (kWave - 1)) >> 4;
    float a[2][2][4], b[2][4];
    auto load = [&](int turn, int32_t k0) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int32_t k = k0 + 4 * q + four;
            b[turn][q] = right(k, row);
            a[turn][0][q] = left(0, row, k);
            a[turn][1][q] = left(1, row, k);
        }
    };
    auto multiply = [&](int turn) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                acc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[turn][i][q], b[turn][q], acc[i], 0, 0, 0);
    };
    acc[0] = acc[1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    load(0, 0);
    int32_t k = 16;
    for (; k + 16 < len; k += 32) {
        load(1, k);
        multiply(0);
        load(0, k + 16);
        multiply(1);
    }
    if (k < len) {
        load(1, k);
        multiply(0);
        multiply(1);
    } else {
        multiply(0);
    }
}

template <int kClass>
__global__ __launch_bounds__(kLdsBlock) void muon_lds_kernel(GivenArray given, bool batch, int64_t stride_in,
                                                             int64_t stride_out, Io io, int steps, float a, float b,
                                                             float c) {
    __shared__ float lds[kLdsFloats[kClass]];
    __shared__ double s_sum[kLdsWaves];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const Given mat = given.mat[batch ? 0 : blockIdx.x];
    const int64_t src = batch ? blockIdx.x * stride_in : mat.offset;
    const int64_t dst = batch ? blockIdx.x * stride_out : mat.offset;
    const int64_t ld_in = io.ld_in ? io.ld_in : mat.cols, ld_out = io.ld_out ? io.ld_out : mat.cols;
    const bool tall = mat.rows > mat.cols;
    const int32_t m = int32_t(round16(low(mat.rows, mat.cols))), n = int32_t(round16(high(mat.rows, mat.cols)));
    const int32_t lx = n + 4, la = m + 4;
    float *X = lds, *A = X + m * lx, *B = A + m * la;
    const int32_t size = mat.rows * mat.cols;
    // element i of the matrix: where it is in memory and in X
    auto place = [&](int32_t i, int64_t ld, int64_t &at, int32_t &to) {
        const int32_t r = int32_t(uint32_t(i) / uint32_t(mat.cols)), q = i - r * mat.cols;
        at = r * ld + q;
        to = tall ? q * lx + r : r * lx + q;
    };

    for (int32_t i = tid; i < m * lx; i += kLdsBlock) X[i] = 0.0f;
    __syncthreads();
    double sum = 0.0;
    constexpr int kAhead = 4;   // elements of a thread on their way together
    for (int32_t i0 = tid; i0 < size; i0 += kAhead * kLdsBlock) {
        float u[kAhead], v[kAhead];
        int64_t at[kAhead];
        int32_t to[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int32_t i = min(i0 + k * kLdsBlock, size - 1);
            place(i, ld_in, at[k], to[k]);
            u[k] = read_in(io, src + at[k]);
            v[k] = io.m != nullptr ? io.m[src + at[k]] : 0.0f;
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (i0 + k * kLdsBlock >= size) continue;
            if (io.m != nullptr) {
                v[k] = __fadd_rn(__fmul_rn(io.beta, v[k]), u[k]);
                io.m[src + at[k]] = v[k];
                u[k] = direction(io, u[k], v[k]);
            }
            X[to[k]] = u[k];
            sum += double(u[k]) * double(u[k]);
        }
    }
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
    if (lane == 0) s_sum[wave] = sum;
    __syncthreads();
    sum = 0.0;
    for (int w = 0; w < kLdsWaves; ++w) sum += s_sum[w];
    const Norm norm = norm_of(sum, io.eps);
    // the padding stays zero, also where the norm is zero, infinite or NaN
    for (int32_t i = tid; i < size; i += kLdsBlock) {
        int64_t at;
        int32_t to;
        place(i, 0, at, to);
        X[to] = norm.divide(X[to]);
    }
    __syncthreads();

    // A wave takes two tiles of a column: eight columns at a time, or four with
    // both halves of their rows where there are more than two rows of tiles.
    const int32_t tm = m / 16, tn = n / 16;
    const int halves = tm > 2 ? 2 : 1, columns = kLdsWaves / halves;
    const int first = wave % halves * 2, column = wave / halves;
    const int32_t last = (tm - 1) * 16;   // a second tile past the rows repeats the last
    const int32_t r0 = min(first * 16, last), r1 = min(first * 16 + 16, last);
    const int32_t row4 = (lane >> 4) * 4, col = lane & 15;
    for (int s = 0; s < steps; ++s) {
        f32x4 g[2];
        if (column < tm) {
            mfma_f32(n, g, [&](int i, int r, int k) { return X[((i ? r1 : r0) + r) * lx + k]; },
                     [&](int k, int q) { return X[(column * 16 + q) * lx + k]; });
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (first + i < tm)
#pragma unroll
                    for (int e = 0; e < 4; ++e) A[((i ? r1 : r0) + row4 + e) * la + column * 16 + col] = g[i][e];
        }
        __syncthreads();
        if (column < tm) {
            mfma_f32(m, g, [&](int i, int r, int k) { return A[((i ? r1 : r0) + r) * la + k]; },
                     [&](int k, int q) { return A[k * la + column * 16 + q]; });
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (first + i < tm)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int32_t at = ((i ? r1 : r0) + row4 + e) * la + column * 16 + col;
                        B[at] = __fadd_rn(__fmul_rn(b, A[at]), __fmul_rn(c, g[i][e]));
                    }
        }
        __syncthreads();
        for (int32_t t0 = 0; t0 < tn; t0 += columns) {
            const int32_t t = t0 + column;
            if (t < tn)
                mfma_f32(m, g, [&](int i, int r, int k) { return B[((i ? r1 : r0) + r) * la + k]; },
                         [&](int k, int q) { return X[k * lx + t * 16 + q]; });
            // a column is replaced where it is, once both halves have read it
            if (halves > 1) __syncthreads();
            if (t < tn) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (first + i < tm)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float *p = X + ((i ? r1 : r0) + row4 + e) * lx + t * 16 + col;
                            *p = __fadd_rn(__fmul_rn(a, *p), g[i][e]);
                        }
            }
        }
        __syncthreads();
    }
    const float scale = step_scale(io, mat.rows, mat.cols);
    for (int32_t i0 = tid; i0 < size; i0 += kAhead * kLdsBlock) {
        float v[kAhead];
        int64_t at[kAhead];
        int32_t from[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            place(min(i0 + k * kLdsBlock, size - 1), ld_out, at[k], from[k]);
            if (io.m != nullptr) v[k] = static_cast<const float *>(io.out)[dst + at[k]];
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (i0 + k * kLdsBlock >= size) continue;
            const float o = X[from[k]];
            if (io.m != nullptr)
                static_cast<float *>(io.out)[dst + at[k]] = step_of(io, v[k], o, scale);
            else
                write_out(io, dst + at[k], o, scale);
        }
    }
}

// What the products of all matrices come to: tiles times steps, and the most
// steps that one tile takes; X X^T, A A, B X.
struct Cost {
    int64_t work[3][kTileKinds], longest[3];
};

void add_cost(Cost &cost, int32_t rows, int32_t cols, int32_t times) {
    const int64_t steps_n = steps_of<Prec::kSplit>(high(rows, cols));
    const int64_t steps_m = steps_of<Prec::kSplit>(low(rows, cols));
    Place one = {};
    advance(one, rows, cols, INT32_MAX);
    for (int p = 0; p < 3; ++p) {
        const int64_t steps = p == 0 ? steps_n : steps_m;
        for (int k = 0; k < kTileKinds; ++k) cost.work[p][k] += steps * (p < 2 ? one.sym[k] : one.full[k]) * times;
        if (steps > cost.longest[p]) cost.longest[p] = steps;
    }
}

// The steps of X X^T that a workgroup takes where tiles are split, INT32_MAX
// where they are not: for three workgroups a compute unit, but 24 at least.
// Splitting costs a launch and the partial sums' way to memory and back, about
// 10 us (LSTM-sized gates, 330 tiles of 82 to 157 steps: 87 -> 59 us).
int32_t split_steps(const Cost &cost) {
    const double whole = product_time(best_tile(cost.work[0], cost.longest[0]),
                                      cost.work[0][best_tile(cost.work[0], cost.longest[0])], cost.longest[0]);
    const int64_t share = cost.work[0][kTiny] / (3 * device_cu_count());
    const int32_t most = int32_t(share < 24 ? 24 : share < (1 << 20) ? share : 1 << 20);
    const double split = fmax(most * kStepAlone[kTiny], cost.work[0][kTiny] * kStepBusy[kTiny] / device_cu_count()) + 10.0;
    return split < whole ? most : INT32_MAX;
}

// Everything that a call over these matrices is laid out by.
struct Job {
    Cost cost;
    Place end;
    int32_t nmat, most;
    uint32_t axes;   // bit k: a longer axis of 2^k to 2^(k+1) - 1
};

// Matrices that the workgroups of small ones do not take; `next` steps through
// rows and cols.  False where they need more workgroups than a grid has.
bool job_of(int32_t nmat, const int32_t *rows, const int32_t *cols, int32_t next, Job *job) {
    *job = {};
    auto each = [&](auto f) {
        for (int32_t i = 0; i < (next == 0 && nmat > 0 ? 1 : nmat); ++i) {
            const int32_t r = rows[i * next], c = cols[i * next];
            if (r != 0 && c != 0 && lds_class(r, c) < 0) f(r, c);
        }
    };
    const int32_t times = next == 0 ? nmat : 1;   // of each that is looked at
    int64_t count = 0;
    each([&](int32_t r, int32_t c) {
        Place one = {};
        advance(one, r, c, 8);   // no fewer workgroups than with any split
        count += (int64_t(one.packs) + one.full[kTiny] + one.chunks + one.units) * times;
        add_cost(job->cost, r, c, times);
        for (int bit = 0; bit < 31; ++bit) job->axes |= uint32_t((high(r, c) >> bit) == 1) << bit;
        job->nmat += times;
    });
    if (count > INT32_MAX) return false;
    job->most = split_steps(job->cost);
    each([&](int32_t r, int32_t c) {
        Place one = {};
        advance(one, r, c, job->most);
        add(job->end, one, times);
    });
    return true;
}

template <int kProduct>
void launch_product(const Job &job, const Mat *table, char *operands, f32x4 *parts, int cur, float a, float b,
                    float c, const Io &io, hipStream_t stream) {
    if (kProduct == kGram && job.most != INT32_MAX) {
        using Tile = TinyTile<Prec::kSplit>;
        muon_gram_kernel<Tile><<<job.end.units, Tile::kThreads, 0, stream>>>(table, job.nmat, operands, cur, job.most,
                                                                             parts, io);
        if (job.end.parts > 0)
            muon_gram_join_kernel<Tile><<<job.end.sym[kTiny], Tile::kThreads, 0, stream>>>(
                table, job.nmat, operands, cur, job.most, parts, io);
        return;
    }
    constexpr bool kSym = kProduct == kGram || kProduct == kPolynomial;
    constexpr int kCost = kProduct == kGram ? 0 : kProduct == kPolynomial ? 1 : 2;
    auto run = [&](auto tile, int kind) {
        using Tile = decltype(tile);
        muon_product_kernel<kProduct, Tile>
            <<<kSym ? job.end.sym[kind] : job.end.full[kind], Tile::kThreads, 0, stream>>>(table, job.nmat, operands,
                                                                                           cur, a, b, c, io);
    };
    switch (best_tile(job.cost.work[kCost], job.cost.longest[kCost])) {
        case kTiny: return run(TinyTile<Prec::kSplit>(), kTiny);
        case kSmall: return run(SmallTile<Prec::kSplit>(), kSmall);
        case kLarge: return run(LargeTile<Prec::kSplit>(), kLarge);
    }
}

void launch_lds(int kind, int32_t count, const GivenArray &given, bool batch, int64_t stride_in, int64_t stride_out,
                const Io &io, int steps, const float *coeffs, hipStream_t stream) {
    auto run = [&](auto kernel) {
        kernel<<<count, kLdsBlock, 0, stream>>>(given, batch, stride_in, stride_out, io, steps, coeffs[0], coeffs[1],
                                                coeffs[2]);
    };
    kind == 0 ? run(muon_lds_kernel<0>) : run(muon_lds_kernel<1>);
}

// The launches after the table.
hipError_t launch_steps(const Job &job, char *ws, const Io &io, int steps, const float *coeffs, hipStream_t stream) {
    const Layout l = layout_of(job.nmat, job.end);
    const Mat *table = reinterpret_cast<const Mat *>(ws + l.table);
    double *sums = reinterpret_cast<double *>(ws + l.sums);
    f32x4 *parts = reinterpret_cast<f32x4 *>(ws + l.parts);
    char *operands = ws + l.operands;
    muon_momentum_kernel<<<job.end.chunks, kSumBlock, 0, stream>>>(table, job.nmat, io, sums);
    muon_pack_kernel<<<job.end.packs, kSumBlock, 0, stream>>>(table, job.nmat, io, sums, operands);
    const float a = coeffs[0], b = coeffs[1], c = coeffs[2];
    int cur = 0;
    for (int s = 0; s < steps; ++s, cur ^= 1) {
        launch_product<kGram>(job, table, operands, parts, cur, a, b, c, io, stream);
        launch_product<kPolynomial>(job, table, operands, parts, cur, a, b, c, io, stream);
        if (s + 1 < steps) launch_product<kApply>(job, table, operands, parts, cur, a, b, c, io, stream);
        else launch_product<kLast>(job, table, operands, parts, cur, a, b, c, io, stream);
    }
    return hipGetLastError();
}

}  // namespace

bool muon_workspace_size(int32_t nmat, const int32_t *rows, const int32_t *cols, int32_t next, size_t *bytes) {
    Job job;
    if (!job_of(nmat, rows, cols, next, &job)) return false;
    *bytes = size_t(layout_of(job.nmat, job.end).total);
    return true;
}

hipError_t launch_muon_orthogonalize(const void *g, int64_t ld_g, int64_t stride_g, void *o, int64_t ld_o,
                                     int64_t stride_o, bool bf16, int32_t batch, int32_t rows, int32_t cols,
                                     int steps, const float *coeffs, float eps, void *workspace,
                                     hipStream_t stream) {
    Io io = {};
    io.in = g;
    io.out = o;
    io.ld_in = ld_g;
    io.ld_out = ld_o;
    io.eps = eps;
    io.bf16 = bf16;
    GivenArray given = {};
    given.mat[0] = Given{0, rows, cols};
    const int kind = lds_class(rows, cols);
    if (kind >= 0) {
        launch_lds(kind, batch, given, true, stride_g, stride_o, io, steps, coeffs, stream);
        return hipGetLastError();
    }
    Job job;
    job_of(batch, &rows, &cols, 0, &job);
    char *ws = static_cast<char *>(workspace);
    const int32_t blocks = (batch + kSetupBlock) / kSetupBlock;
    muon_setup_kernel<<<blocks < 64 ? blocks : 64, kSetupBlock, 0, stream>>>(
        reinterpret_cast<Mat *>(ws), given, 0, batch, 1, job.most, stride_g, stride_o);
    return launch_steps(job, ws, io, steps, coeffs, stream);
}

hipError_t launch_muon_apply(const float *avg, int32_t nmat, const int64_t *offsets, const int32_t *rows,
                             const int32_t *cols, float *x, float *m, float beta, float gamma, float decay,
                             bool nesterov, int steps, const float *coeffs, float eps, void *workspace,
                             hipStream_t stream) {
    Io io = {};
    io.in = avg;
    io.m = m;
    io.out = x;
    io.beta = beta;
    io.gamma = gamma;
    io.keep = float(1.0 - double(gamma) * double(decay));
    io.eps = eps;
    io.nesterov = nesterov;

    // the matrices of each kind, as many as a launch's arguments hold at a time
    char *ws = static_cast<char *>(workspace);
    Job job;
    job_of(nmat, rows, cols, 1, &job);
    for (int kind = -1; kind <= 1; ++kind) {
        GivenArray given;
        int32_t count = 0, before = 0;
        auto flush = [&]() {
            if (count == 0) return;
            if (kind >= 0)
                launch_lds(kind, count, given, false, 0, 0, io, steps, coeffs, stream);
            else
                muon_setup_kernel<<<1, kSetupBlock, 0, stream>>>(reinterpret_cast<Mat *>(ws), given, before, count, 0,
                                                                 job.most, 0, 0);
            before += count;
            count = 0;
        };
        // the tiles that take longest first (X X^T sums over the longer axis):
        // by the power of two of that axis
        for (int bit = kind < 0 ? 30 : 0; bit >= 0; --bit) {
            if (kind < 0 && (job.axes >> bit & 1) == 0) continue;
            for (int32_t i = 0; i < nmat; ++i) {
                if (rows[i] == 0 || cols[i] == 0 || (kind < 0 && (high(rows[i], cols[i]) >> bit) != 1)) continue;
                if (lds_class(rows[i], cols[i]) != kind) continue;
                if (count == kGivenPerLaunch) flush();
                given.mat[count++] = Given{offsets[i], rows[i], cols[i]};
            }
        }
        flush();
    }
    if (job.nmat == 0) return hipGetLastError();
    return launch_steps(job, ws, io, steps, coeffs, stream);
}

}  // namespace efs
