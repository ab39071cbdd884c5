// Softmax cross entropy of tokens against a vocabulary, and its gradients.
//
//   l = h w^T                                    T x V logits, never kept
//   lse_t = log sum_v exp l_tv ;  loss_t = lse_t - l_t,target
//   g = dloss_t (exp(l - lse_t) - [v = target_t])
//   dh = g w ;  dw = g^T h
//
// Forward: one product over tiles of vocabulary x tokens.  A tile ends as a
// maximum and a sum of exponentials for each of its tokens (8 bytes for 256
// logits); a second launch joins the tiles of a token.
// Backward: in pieces of the vocabulary.  A piece's logits are computed again
// and leave their tile as g, along both axes (the two products sum over one
// each); then g^T h gives the piece's rows of dw, and g w is added to dh's
// partial sums, in 32 bits.  The pieces' sums over v are split among several
// workgroups where dh has few tiles; each split has its own partial sums, so
// that the order of every addition is fixed.
//
// fp32 tensors are multiplied as split values (mfma_tile.hpp), scaled by a
// power of two that brings the tensor's largest finite magnitude to 2^14; g by
// 2^15 without dloss_t, which goes into h^T and into the last pass over dh.
// bf16 tensors are multiplied as they are; g is then rounded to bf16 (2^-9 of
// itself, as the results are when they are written).
//
// Tokens whose target is ignored count nowhere: what their rows of h hold is
// never used.
#include "mfma_tile.hpp"
#include "launch.hpp"

#include <algorithm>

namespace efs {

namespace {

constexpr int kPackBlock = 256;
constexpr int kPackTile = 64;
constexpr int kCheckBlock = 1024;
constexpr int kJoinTokens = kWave;
constexpr int kJoinSlices = 16;
constexpr int kGradShift = 15;          // g's scale in split form
constexpr int64_t kPieceBytes = int64_t(256) << 20;   // g along both axes, one piece

// What a call knows of its tensors.
struct Xent {
    const void *h, *w;
    int64_t ld_h, ld_w;
    const int64_t *target;
    int64_t ignore;
    int32_t tokens, vocab, hidden;
};

// Control words at the workspace's start.
struct Control {
    uint32_t status;
    uint32_t top[3];   // bits of the largest finite |h|, |w|, |dloss h|
};
enum { kTopH, kTopW, kTopWeighted };

// -1: the token does not count.
__device__ __forceinline__ int32_t target_of(const Xent &x, int32_t t) {
    const int64_t v = x.target[t];
    return v != x.ignore && v >= 0 && v < x.vocab ? int32_t(v) : -1;
}

// Exponent that brings a tensor's largest magnitude to [2^14, 2^15).
__device__ __forceinline__ int scale_exponent(uint32_t top) {
    return top == 0u ? 0 : 141 - max(int(top >> 23), 1);
}

__device__ __forceinline__ uint32_t finite_bits(float v) {
    const uint32_t b = magnitude_key(v);
    return b < 0x7f800000u ? b : 0u;
}

// One workgroup: the status word, and zeros for the magnitudes.
__global__ __launch_bounds__(kCheckBlock) void xent_check_kernel(Xent x, Control *control) {
    __shared__ uint32_t s_bad;
    if (threadIdx.x == 0) s_bad = 0u;
    __syncthreads();
    bool bad = false;
    for (int32_t t = threadIdx.x; t < x.tokens; t += kCheckBlock) {
        const int64_t v = x.target[t];
        bad |= v != x.ignore && (v < 0 || v >= x.vocab);
    }
    if (bad) s_bad = kXentBadTarget;
    __syncthreads();
    if (threadIdx.x == 0) control->status = s_bad;
    if (threadIdx.x < 3) control->top[threadIdx.x] = 0u;
}

// Largest finite magnitudes, fp32 tensors.  Workgroups [0, w_blocks) sweep w,
// the others h (rows that count) and, with dloss, dloss h.  A wave takes a row
// at a time.
__global__ __launch_bounds__(kPackBlock) void xent_top_kernel(Xent x, const float *dloss, uint32_t w_blocks,
                                                              Control *control) {
    __shared__ uint32_t s_wave[kWaves];
    const bool of_w = blockIdx.x < w_blocks;
    const uint32_t block = of_w ? blockIdx.x : blockIdx.x - w_blocks;
    const uint32_t blocks = of_w ? w_blocks : gridDim.x - w_blocks;
    const float *base = static_cast<const float *>(of_w ? x.w : x.h);
    const int64_t ld = of_w ? x.ld_w : x.ld_h;
    const int32_t rows = of_w ? x.vocab : x.tokens;
    const int lane = threadIdx.x & (kWave - 1);
    uint32_t top = 0u, weighted = 0u;
    for (int64_t r = int64_t(block) * kWaves + threadIdx.x / kWave; r < rows; r += int64_t(blocks) * kWaves) {
        if (!of_w && target_of(x, int32_t(r)) < 0) continue;
        const float *row = base + r * ld;
        const float f = !of_w && dloss != nullptr ? dloss[r] : 0.0f;
        int32_t c = lane * 4;
        for (; c + 4 <= x.hidden; c += kWave * 4) {
            const f32x4u v = *reinterpret_cast<const f32x4u *>(row + c);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                top = max(top, finite_bits(v[k]));
                weighted = max(weighted, finite_bits(__fmul_rn(f, v[k])));
            }
        }
        for (; c < x.hidden; ++c) {
            top = max(top, finite_bits(row[c]));
            weighted = max(weighted, finite_bits(__fmul_rn(f, row[c])));
        }
    }
    top = block_max(top, s_wave);
    __syncthreads();
    weighted = block_max(weighted, s_wave);
    if (threadIdx.x == 0) {
        atomicMax(&control->top[of_w ? kTopW : kTopH], top);
        if (!of_w) atomicMax(&control->top[kTopWeighted], weighted);
    }
}

// h or w as operands: `along` its rows, and `turned`, a row for each of its
// columns; either may be null.  Rows of h that do not count are zeros.  In
// split form the turned h holds dloss h.
template <Prec P>
__global__ __launch_bounds__(kPackBlock) void xent_pack_kernel(Xent x, bool of_w, const float *dloss, char *along,
                                                               char *turned, const Control *control) {
    __shared__ float tile[kPackTile][kPackTile + 1];
    __shared__ float s_weight[kPackTile];
    __shared__ bool s_counts[kPackTile];
    const int tid = threadIdx.x;
    const int32_t rows = of_w ? x.vocab : x.tokens, cols = x.hidden;
    const int64_t ld = of_w ? x.ld_w : x.ld_h;
    const int32_t across = (cols + kPackTile - 1) / kPackTile;
    const int32_t r0 = int32_t(blockIdx.x / across) * kPackTile, c0 = int32_t(blockIdx.x % across) * kPackTile;
    if (tid < kPackTile) {
        const int32_t r = r0 + tid;
        s_counts[tid] = r < rows && (of_w || target_of(x, r) >= 0);
        s_weight[tid] = P == Prec::kSplit && !of_w && dloss != nullptr && s_counts[tid] ? dloss[r] : 1.0f;
    }
    __syncthreads();
    for (int i = tid; i < kPackTile * kPackTile; i += kPackBlock) {
        const int r = i / kPackTile, c = i % kPackTile;
        float v = 0.0f;
        if (s_counts[r] && c0 + c < cols) {
            const int64_t at = int64_t(r0 + r) * ld + c0 + c;
            v = P == Prec::kBf16 ? float(static_cast<const __bf16 *>(of_w ? x.w : x.h)[at])
                                 : static_cast<const float *>(of_w ? x.w : x.h)[at];
        }
        tile[r][c] = v;
    }
    __syncthreads();
    const int e_along = P == Prec::kSplit ? scale_exponent(control->top[of_w ? kTopW : kTopH]) : 0;
    const int e_turned = P == Prec::kSplit ? scale_exponent(control->top[of_w ? kTopW : kTopWeighted]) : 0;
    constexpr int kPad = kStepValues<P>;
#pragma unroll
    for (int turn = 0; turn < 2; ++turn) {
        char *base = turn ? turned : along;
        if (base == nullptr) continue;
        const int64_t stride = row_bytes<P>(turn ? rows : cols);
        const int32_t row_first = turn ? c0 : r0, col_first = turn ? r0 : c0;
        const int32_t row_end = turn ? cols : rows;
        const int32_t col_end = ((turn ? rows : cols) + kPad - 1) / kPad * kPad;
        for (int i = tid; i < kPackTile * 8; i += kPackBlock) {
            const int r = turn ? i % kPackTile : i / 8, c = (turn ? i / kPackTile : i % 8) * 8;
            if (row_first + r >= row_end || col_first + c >= col_end) continue;
            char *row = base + int64_t(row_first + r) * stride;
            if constexpr (P == Prec::kBf16) {
                bf16x8 v;
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = __bf16(turn ? tile[c + k][r] : tile[r][c + k]);
                *reinterpret_cast<bf16x8 *>(row + int64_t(col_first + c) * 2) = v;
            } else {
                f16x8 hi, lo;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    float v = turn ? tile[c + k][r] : tile[r][c + k];
                    if (turn) v = __fmul_rn(s_weight[c + k], v);
                    _Float16 a, b;
                    split_value(ldexpf(v, turn ? e_turned : e_along), a, b);
                    hi[k] = a;
                    lo[k] = b;
                }
                char *p = row + split_offset(col_first + c);
                *reinterpret_cast<f16x8 *>(p) = hi;
                *reinterpret_cast<f16x8 *>(p + 64) = lo;
            }
        }
    }
}

// Maximum and sum of exponentials over some of a token's logits.
struct Part {
    float top, sum;
};

__device__ __forceinline__ Part join(Part a, Part b) {
    const float top = fmaxf(a.top, b.top);
    if (top == -INFINITY) return Part{top, a.sum + b.sum};   // nothing yet (or NaN, which stays in the sum)
    return Part{top, __fadd_rn(__fmul_rn(a.sum, expf(a.top - top)), __fmul_rn(b.sum, expf(b.top - top)))};
}

// The logits of a tile: rows are words, columns tokens.
template <Prec P>
__device__ __forceinline__ int logit_exponent(const Control *control) {
    return P == Prec::kSplit ? -(scale_exponent(control->top[kTopH]) + scale_exponent(control->top[kTopW])) : 0;
}

template <Prec P>
__device__ __forceinline__ float logit(float acc, int exponent) {
    return P == Prec::kSplit ? ldexpf(acc, exponent) : acc;
}

// Forward: parts[tile row][token], and the targets' logits.
template <Prec P, class Tile>
__global__ __launch_bounds__(Tile::kThreads, 2) void xent_forward_kernel(Xent x, Operand w, Operand h,
                                                                         const Control *control, Part *parts,
                                                                         float *target_logit) {
    __shared__ __align__(16) char lds[Tile::kLdsBytes];
    const uint32_t tv = (x.vocab + Tile::kRows - 1) / Tile::kRows, tt = (x.tokens + Tile::kCols - 1) / Tile::kCols;
    uint32_t r, c;
    banded(xcd_place(blockIdx.x, gridDim.x), tv, tt, r, c);
    const int32_t row0 = int32_t(r) * Tile::kRows, col0 = int32_t(c) * Tile::kCols;
    Tile tile;
    tile.run(w, h, row0, col0, 0, int32_t(row_bytes<P>(x.hidden) / kStepBytes), lds);
    const int exponent = logit_exponent<P>(control);
    Part *s_part = reinterpret_cast<Part *>(lds);   // [rows of waves][columns]
    constexpr int kHigh = Tile::kRows / (Tile::kTilesM * 32);
    const int wave_row = Tile::row_of(0, 0) / (Tile::kTilesM * 32);
    __syncthreads();   // every wave has read its last step
#pragma unroll
    for (int j = 0; j < Tile::kTilesN; ++j) {
        const int32_t t = col0 + Tile::col_of(j);
        const int32_t target = t < x.tokens ? target_of(x, t) : -1;
        Part p = {-INFINITY, 0.0f};
#pragma unroll
        for (int i = 0; i < Tile::kTilesM; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int32_t v = row0 + Tile::row_of(i, e);
                float l = logit<P>(tile.acc[i][j][e], exponent);
                if (v >= x.vocab) l = -INFINITY;
                if (v == target) target_logit[t] = l;
                tile.acc[i][j][e] = l;
                p.top = fmaxf(p.top, l);
            }
        const float shift = p.top == -INFINITY ? 0.0f : p.top;
#pragma unroll
        for (int i = 0; i < Tile::kTilesM; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) p.sum += expf(tile.acc[i][j][e] - shift);
        const Part q = {__shfl_xor(p.top, 32), __shfl_xor(p.sum, 32)};
        p = join(p, q);
        if ((threadIdx.x & 32) == 0) s_part[wave_row * Tile::kCols + Tile::col_of(j)] = p;
    }
    __syncthreads();
    for (int k = threadIdx.x; k < Tile::kCols; k += Tile::kThreads) {
        if (col0 + k >= x.tokens) continue;
        Part p = s_part[k];
#pragma unroll
        for (int i = 1; i < kHigh; ++i) p = join(p, s_part[i * Tile::kCols + k]);
        parts[int64_t(r) * x.tokens + col0 + k] = p;
    }
}

// A token's parts joined: lanes are tokens, waves take every 16th part.
__global__ __launch_bounds__(kJoinTokens *kJoinSlices) void xent_join_kernel(Xent x, const Part *parts, int32_t nparts,
                                                                             const float *target_logit, float *loss,
                                                                             float *lse) {
    __shared__ Part s_part[kJoinSlices][kJoinTokens];
    const int lane = threadIdx.x % kJoinTokens, slice = threadIdx.x / kJoinTokens;
    const int32_t t = int32_t(blockIdx.x) * kJoinTokens + lane;
    Part p = {-INFINITY, 0.0f};
    if (t < x.tokens)
        for (int32_t i = slice; i < nparts; i += kJoinSlices) p = join(p, parts[int64_t(i) * x.tokens + t]);
    s_part[slice][lane] = p;
    __syncthreads();
    if (slice != 0 || t >= x.tokens) return;
    for (int i = 1; i < kJoinSlices; ++i) p = join(p, s_part[i][lane]);
    const bool counts = target_of(x, t) >= 0;
    const float v = __fadd_rn(p.top, logf(p.sum));
    lse[t] = counts ? v : 0.0f;
    loss[t] = counts ? __fsub_rn(v, target_logit[t]) : 0.0f;
}

// Eight consecutive values of an operand's row, the first a multiple of eight.
template <Prec P>
__device__ __forceinline__ void store8(char *row, int32_t c, const float (&y)[8]) {
    if constexpr (P == Prec::kSplit) {
        store_split8(row, c, y);
    } else {
        bf16x8 v;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = __bf16(y[k]);
        *reinterpret_cast<bf16x8 *>(row + int64_t(c) * 2) = v;
    }
}

// Backward: g of words [v0, v0 + words), as g [token][word] and gt [word][token].
template <Prec P, class Tile>
__global__ __launch_bounds__(Tile::kThreads, 2) void xent_grad_kernel(Xent x, Operand w, Operand h, int32_t v0,
                                                                      int32_t words, const float *lse,
                                                                      const float *dloss, const Control *control,
                                                                      char *g, char *gt) {
    __shared__ __align__(16) char lds[Tile::kLdsBytes];
    const uint32_t tv = (words + Tile::kRows - 1) / Tile::kRows, tt = (x.tokens + Tile::kCols - 1) / Tile::kCols;
    uint32_t r, c;
    banded(xcd_place(blockIdx.x, gridDim.x), tv, tt, r, c);
    const int32_t row0 = int32_t(r) * Tile::kRows, col0 = int32_t(c) * Tile::kCols;
    Tile tile;
    tile.run(w, h, row0, col0, 0, int32_t(row_bytes<P>(x.hidden) / kStepBytes), lds);
    const int exponent = logit_exponent<P>(control);
    const int64_t g_row = row_bytes<P>(words), gt_row = row_bytes<P>(x.tokens);
    const int32_t words_end = int32_t(g_row / kStepBytes) * kStepValues<P>;
    const int32_t tokens_end = int32_t(gt_row / kStepBytes) * kStepValues<P>;
#pragma unroll
    for (int j = 0; j < Tile::kTilesN; ++j) {
        const int32_t t = col0 + Tile::col_of(j);
        const int32_t target = t < x.tokens ? target_of(x, t) : -1;
        const float shift = target >= 0 ? lse[t] : 0.0f;
        // bf16: dloss in g; split: in h^T and the last pass over dh
        const float weight = P == Prec::kSplit ? float(1 << kGradShift) : target >= 0 ? dloss[t] : 0.0f;
#pragma unroll
        for (int i = 0; i < Tile::kTilesM; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int32_t v = row0 + Tile::row_of(i, e);
                float p = 0.0f;   // tokens that do not count, and the padding
                if (target >= 0 && v < words) {
                    p = expf(logit<P>(tile.acc[i][j][e], exponent) - shift);
                    if (v0 + v == target) p = __fsub_rn(p, 1.0f);
                    p = __fmul_rn(p, weight);
                }
                tile.acc[i][j][e] = p;
            }
    }
    using Out = Band<Tile>;
    Out band{reinterpret_cast<float *>(lds)};
    each_band<Tile::kTilesM>([&](auto index) {
        constexpr int i = decltype(index)::value;
        band.template put<i>(tile);
#pragma unroll
        for (int k = 0; k < Out::kUnits; ++k) {
            float y[8];
            const int32_t v = row0 + Out::tile_row(i, Out::row(k)), t = col0 + Out::col(k);
            if (v < words && t < tokens_end) {
                band.get(k, y);
                store8<P>(gt + v * gt_row, t, y);
            }
        }
#pragma unroll
        for (int k = 0; k < Out::kUnits; ++k) {
            float y[8];
            const int32_t v = row0 + Out::tile_row(i, Out::turned_row(k)), t = col0 + Out::turned_col(k);
            if (t < x.tokens && v < words_end) {
                band.get_turned(k, y);
                store8<P>(g + t * g_row, v, y);
            }
        }
    });
}

// dw rows [v0, v0 + words) = g^T h.
template <Prec P, class Tile>
__global__ __launch_bounds__(Tile::kThreads, 2) void xent_dw_kernel(Xent x, Operand gt, Operand ht, int32_t v0,
                                                                    const Control *control, void *dw, int64_t ld) {
    __shared__ __align__(16) char lds[Tile::kLdsBytes];
    const uint32_t tv = (gt.rows + Tile::kRows - 1) / Tile::kRows, th = (x.hidden + Tile::kCols - 1) / Tile::kCols;
    uint32_t r, c;
    banded(xcd_place(blockIdx.x, gridDim.x), tv, th, r, c);
    const int32_t row0 = int32_t(r) * Tile::kRows, col0 = int32_t(c) * Tile::kCols;
    Tile tile;
    tile.run(gt, ht, row0, col0, 0, int32_t(row_bytes<P>(x.tokens) / kStepBytes), lds);
    const int exponent = P == Prec::kSplit ? -(kGradShift + scale_exponent(control->top[kTopWeighted])) : 0;
#pragma unroll
    for (int i = 0; i < Tile::kTilesM; ++i)
#pragma unroll
        for (int j = 0; j < Tile::kTilesN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int32_t v = row0 + Tile::row_of(i, e), k = col0 + Tile::col_of(j);
                if (v >= gt.rows || k >= x.hidden) continue;
                const int64_t at = (int64_t(v0) + v) * ld + k;
                if constexpr (P == Prec::kSplit) static_cast<float *>(dw)[at] = ldexpf(tile.acc[i][j][e], exponent);
                else static_cast<__bf16 *>(dw)[at] = __bf16(tile.acc[i][j][e]);
            }
}

// Partial sums of dh: split s adds its share of the piece's words to
// part[s][token][hidden] (or starts it, with the first piece).
template <Prec P, class Tile>
__global__ __launch_bounds__(Tile::kThreads, 2) void xent_dh_kernel(Xent x, Operand g, Operand wt, int32_t steps,
                                                                    int32_t splits, bool first, float *part) {
    __shared__ __align__(16) char lds[Tile::kLdsBytes];
    const uint32_t tt = (x.tokens + Tile::kRows - 1) / Tile::kRows, th = (x.hidden + Tile::kCols - 1) / Tile::kCols;
    const uint32_t place = xcd_place(blockIdx.x, gridDim.x);
    const uint32_t split = place / (tt * th);
    uint32_t r, c;
    banded(place % (tt * th), tt, th, r, c);
    const int32_t row0 = int32_t(r) * Tile::kRows, col0 = int32_t(c) * Tile::kCols;
    const int32_t lo = int32_t(int64_t(steps) * split / splits), hi = int32_t(int64_t(steps) * (split + 1) / splits);
    Tile tile;
    tile.run(g, wt, row0, col0, lo, hi - lo, lds);
    float *to = part + int64_t(split) * x.tokens * x.hidden;
#pragma unroll
    for (int i = 0; i < Tile::kTilesM; ++i)
#pragma unroll
        for (int j = 0; j < Tile::kTilesN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int32_t t = row0 + Tile::row_of(i, e), k = col0 + Tile::col_of(j);
                if (t >= x.tokens || k >= x.hidden) continue;
                float *p = to + int64_t(t) * x.hidden + k;
                *p = first ? tile.acc[i][j][e] : __fadd_rn(*p, tile.acc[i][j][e]);
            }
}

// dh from its partial sums.
template <Prec P>
__global__ __launch_bounds__(kPackBlock) void xent_dh_join_kernel(Xent x, const float *part, int32_t splits,
                                                                  const float *dloss, const Control *control,
                                                                  void *dh, int64_t ld) {
    const int exponent = P == Prec::kSplit ? -(kGradShift + scale_exponent(control->top[kTopW])) : 0;
    const int64_t size = int64_t(x.tokens) * x.hidden;
    for (int64_t i = int64_t(blockIdx.x) * kPackBlock + threadIdx.x; i < size; i += int64_t(gridDim.x) * kPackBlock) {
        const int32_t t = int32_t(i / x.hidden), k = int32_t(i - int64_t(t) * x.hidden);
        float v = 0.0f;
        if (target_of(x, t) >= 0) {
            for (int32_t s = 0; s < splits; ++s) v = __fadd_rn(v, part[s * size + i]);
            if (P == Prec::kSplit) v = __fmul_rn(ldexpf(v, exponent), dloss[t]);
        }
        const int64_t at = t * ld + k;
        if constexpr (P == Prec::kSplit) static_cast<float *>(dh)[at] = v;
        else static_cast<__bf16 *>(dh)[at] = __bf16(v);
    }
}

// dw of no tokens.
template <class T>
__global__ __launch_bounds__(kPackBlock) void xent_zero_kernel(T *dw, int64_t ld, int32_t rows, int32_t cols) {
    const int64_t size = int64_t(rows) * cols;
    for (int64_t i = int64_t(blockIdx.x) * kPackBlock + threadIdx.x; i < size; i += int64_t(gridDim.x) * kPackBlock)
        dw[i / cols * ld + i % cols] = T(0.0f);
}

int64_t round256(int64_t v) { return (v + 255) / 256 * 256; }
int64_t tiles(int64_t len, int tile) { return (len + tile - 1) / tile; }

// How a backward call is cut, and where everything is in the workspace.
struct Plan {
    int32_t piece;    // words
    int32_t splits;   // of a piece, for dh
    int64_t target_logit, parts, h_along, w_along, h_turned, w_turned, g, gt, dh, forward, total;
};

template <Prec P>
Plan plan_of(int32_t tokens, int32_t vocab, int32_t hidden) {
    constexpr int kTile = kTileSide[kLarge];
    Plan p;
    // whole large tiles of words, as many as the pieces' bytes allow
    if (tokens == 0) tokens = 1;   // (nothing is launched that reads them)
    const int64_t word = 2 * row_bytes<P>(tokens);
    int64_t piece = kPieceBytes / word / kTile * kTile;
    if (piece < 4 * kTile) piece = 4 * kTile;
    p.piece = int32_t(piece < vocab ? piece : vocab);
    // enough workgroups for the compute units, with eight steps each at least
    const int64_t dh_tiles = tiles(tokens, kTileSide[kSmall]) * tiles(hidden, kTileSide[kSmall]);
    const int64_t steps = row_bytes<P>(p.piece) / kStepBytes;
    int64_t splits = (512 + dh_tiles - 1) / dh_tiles;
    if (splits > steps / 8) splits = steps / 8;
    p.splits = int32_t(splits < 1 ? 1 : splits);

    int64_t at = 256;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += round256(bytes);
        return here;
    };
    p.target_logit = take(int64_t(tokens) * 4);
    p.parts = take(int64_t(tokens) * tiles(vocab, kTileSide[kTiny]) * 8);
    p.h_along = take(tokens * row_bytes<P>(hidden));
    p.w_along = take(vocab * row_bytes<P>(hidden));
    p.forward = at;
    p.h_turned = take(hidden * row_bytes<P>(tokens));
    p.w_turned = take(hidden * row_bytes<P>(vocab));
    p.g = take(tokens * row_bytes<P>(p.piece));
    p.gt = take(p.piece * row_bytes<P>(tokens));
    p.dh = take(int64_t(p.splits) * tokens * hidden * 4);
    p.total = at;
    return p;
}

// Calls run(tile, workgroups) with the kind of tile that rows x cols, `times`
// over with `steps` each, is fastest with.
template <Prec P, class F>
void with_tile(int64_t rows, int64_t cols, int64_t times, int64_t steps, F run) {
    int64_t n[kTileKinds], work[kTileKinds];
    for (int k = 0; k < kTileKinds; ++k) {
        n[k] = tiles(rows, kTileSide[k]) * tiles(cols, kTileSide[k]) * times;
        work[k] = n[k] * steps;
    }
    switch (best_tile(work, steps)) {
        case kTiny: return run(TinyTile<P>(), n[kTiny]);
        case kSmall: return run(SmallTile<P>(), n[kSmall]);
        case kLarge: return run(LargeTile<P>(), n[kLarge]);
    }
}

// Whether the tensor can be multiplied where it is: whole steps along its
// rows, 16-byte aligned.
template <Prec P>
bool direct(const void *p, int64_t ld, int32_t hidden) {
    return P == Prec::kBf16 && hidden % kStepValues<P> == 0 && ld % 8 == 0 &&
           reinterpret_cast<uintptr_t>(p) % 16 == 0;
}

// The operands of the logits, packed where they have to be.
template <Prec P>
void pack_operands(const Xent &x, const float *dloss, bool gradient, const Plan &plan, char *ws, Operand *h,
                   Operand *w, hipStream_t stream) {
    Control *control = reinterpret_cast<Control *>(ws);
    xent_check_kernel<<<1, kCheckBlock, 0, stream>>>(x, control);
    if (P == Prec::kSplit) {
        const uint32_t w_blocks = uint32_t(std::min<int64_t>(tiles(x.vocab, kWaves), device_cu_count() * 8));
        const uint32_t h_blocks = uint32_t(std::min<int64_t>(tiles(x.tokens, kWaves), device_cu_count() * 2));
        xent_top_kernel<<<w_blocks + h_blocks, kPackBlock, 0, stream>>>(x, dloss, w_blocks, control);
    }
    const bool direct_h = direct<P>(x.h, x.ld_h, x.hidden), direct_w = direct<P>(x.w, x.ld_w, x.hidden);
    auto pack = [&](bool of_w, bool in_place, int64_t along, int64_t turned) {
        if (in_place && !gradient) return;
        const int64_t blocks = tiles(of_w ? x.vocab : x.tokens, kPackTile) * tiles(x.hidden, kPackTile);
        xent_pack_kernel<P><<<uint32_t(blocks), kPackBlock, 0, stream>>>(
            x, of_w, dloss, in_place ? nullptr : ws + along, gradient ? ws + turned : nullptr, control);
    };
    pack(false, direct_h, plan.h_along, plan.h_turned);
    pack(true, direct_w, plan.w_along, plan.w_turned);
    const int64_t row = row_bytes<P>(x.hidden);
    *h = direct_h ? Operand{static_cast<const char *>(x.h), x.ld_h * 2, x.tokens}
                  : Operand{ws + plan.h_along, row, x.tokens};
    *w = direct_w ? Operand{static_cast<const char *>(x.w), x.ld_w * 2, x.vocab}
                  : Operand{ws + plan.w_along, row, x.vocab};
}

template <Prec P>
hipError_t forward(const Xent &x, float *loss, float *lse, char *ws, hipStream_t stream) {
    const Plan plan = plan_of<P>(x.tokens, x.vocab, x.hidden);
    const Control *control = reinterpret_cast<const Control *>(ws);
    Part *parts = reinterpret_cast<Part *>(ws + plan.parts);
    float *target_logit = reinterpret_cast<float *>(ws + plan.target_logit);
    Operand h, w;
    pack_operands<P>(x, nullptr, false, plan, ws, &h, &w, stream);
    int32_t nparts = 0;
    with_tile<P>(x.vocab, x.tokens, 1, row_bytes<P>(x.hidden) / kStepBytes, [&](auto tile, int64_t blocks) {
        using Tile = decltype(tile);
        nparts = int32_t(tiles(x.vocab, Tile::kRows));
        xent_forward_kernel<P, Tile><<<uint32_t(blocks), Tile::kThreads, 0, stream>>>(x, w, h, control, parts,
                                                                                      target_logit);
    });
    xent_join_kernel<<<uint32_t(tiles(x.tokens, kJoinTokens)), kJoinTokens * kJoinSlices, 0, stream>>>(
        x, parts, nparts, target_logit, loss, lse);
    return hipGetLastError();
}

template <Prec P>
hipError_t backward(const Xent &x, const float *lse, const float *dloss, void *dh, int64_t ld_dh, void *dw,
                    int64_t ld_dw, char *ws, hipStream_t stream) {
    const Plan plan = plan_of<P>(x.tokens, x.vocab, x.hidden);
    const Control *control = reinterpret_cast<const Control *>(ws);
    Operand h, w;
    pack_operands<P>(x, dloss, true, plan, ws, &h, &w, stream);
    const Operand ht{ws + plan.h_turned, row_bytes<P>(x.tokens), x.hidden};
    float *part = reinterpret_cast<float *>(ws + plan.dh);
    for (int64_t v0 = 0; v0 < x.vocab; v0 += plan.piece) {
        const int32_t words = int32_t(std::min<int64_t>(plan.piece, x.vocab - v0));
        const Operand w_piece{w.base + v0 * w.stride, w.stride, words};
        with_tile<P>(words, x.tokens, 1, row_bytes<P>(x.hidden) / kStepBytes, [&](auto tile, int64_t blocks) {
            using Tile = decltype(tile);
            xent_grad_kernel<P, Tile><<<uint32_t(blocks), Tile::kThreads, 0, stream>>>(
                x, w_piece, h, int32_t(v0), words, lse, dloss, control, ws + plan.g, ws + plan.gt);
        });
        const Operand gt{ws + plan.gt, row_bytes<P>(x.tokens), words};
        with_tile<P>(words, x.hidden, 1, row_bytes<P>(x.tokens) / kStepBytes, [&](auto tile, int64_t blocks) {
            using Tile = decltype(tile);
            xent_dw_kernel<P, Tile><<<uint32_t(blocks), Tile::kThreads, 0, stream>>>(x, gt, ht, int32_t(v0), control,
                                                                                     dw, ld_dw);
        });
        // a piece starts on a whole step of w^T: it is a multiple of 256 words
        const Operand g{ws + plan.g, row_bytes<P>(words), x.tokens};
        const Operand wt{ws + plan.w_turned + row_bytes<P>(v0), row_bytes<P>(x.vocab), x.hidden};
        const int32_t steps = int32_t(row_bytes<P>(words) / kStepBytes);
        with_tile<P>(x.tokens, x.hidden, plan.splits, steps / plan.splits, [&](auto tile, int64_t blocks) {
            using Tile = decltype(tile);
            xent_dh_kernel<P, Tile><<<uint32_t(blocks), Tile::kThreads, 0, stream>>>(x, g, wt, steps, plan.splits,
                                                                                     v0 == 0, part);
        });
    }
    const int64_t size = int64_t(x.tokens) * x.hidden;
    xent_dh_join_kernel<P><<<uint32_t(std::min<int64_t>(tiles(size, kPackBlock), device_cu_count() * 16)), kPackBlock,
                             0, stream>>>(x, part, plan.splits, dloss, control, dh, ld_dh);
    return hipGetLastError();
}

}  // namespace

size_t xent_workspace_size(int32_t tokens, int32_t vocab, int32_t hidden, bool bf16, bool gradient) {
    const Plan p = bf16 ? plan_of<Prec::kBf16>(tokens, vocab, hidden) : plan_of<Prec::kSplit>(tokens, vocab, hidden);
    return size_t(gradient ? p.total : p.forward);
}

hipError_t launch_xent_forward(const void *h, int64_t ld_h, const void *w, int64_t ld_w, const int64_t *target,
                               bool bf16, int32_t tokens, int32_t vocab, int32_t hidden, int64_t ignore, float *loss,
                               float *lse, void *workspace, hipStream_t stream) {
    const Xent x{h, w, ld_h, ld_w, target, ignore, tokens, vocab, hidden};
    char *ws = static_cast<char *>(workspace);
    return bf16 ? forward<Prec::kBf16>(x, loss, lse, ws, stream) : forward<Prec::kSplit>(x, loss, lse, ws, stream);
}

hipError_t launch_xent_backward(const void *h, int64_t ld_h, const void *w, int64_t ld_w, const int64_t *target,
                                bool bf16, int32_t tokens, int32_t vocab, int32_t hidden, int64_t ignore,
                                const float *lse, const float *dloss, void *dh, int64_t ld_dh, void *dw,
                                int64_t ld_dw, void *workspace, hipStream_t stream) {
    if (tokens == 0) {
        const uint32_t blocks =
            uint32_t(std::min<int64_t>(tiles(int64_t(vocab) * hidden, kPackBlock), device_cu_count() * 16));
        if (bf16) xent_zero_kernel<<<blocks, kPackBlock, 0, stream>>>(static_cast<__bf16 *>(dw), ld_dw, vocab, hidden);
        else xent_zero_kernel<<<blocks, kPackBlock, 0, stream>>>(static_cast<float *>(dw), ld_dw, vocab, hidden);
        return hipGetLastError();
    }
    const Xent x{h, w, ld_h, ld_w, target, ignore, tokens, vocab, hidden};
    char *ws = static_cast<char *>(workspace);
    return bf16 ? backward<Prec::kBf16>(x, lse, dloss, dh, ld_dh, dw, ld_dw, ws, stream)
                : backward<Prec::kSplit>(x, lse, dloss, dh, ld_dh, dw, ld_dw, ws, stream);
}

}  // namespace efs
