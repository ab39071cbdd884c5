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
// power of two that brings the tensor's largest finite magnitude to 2^14; g without
// dloss_t, which goes into h^T and into the last pass over dh.  Along the words, for
// dh, g is scaled by 2^15: what that loses is below p - 1's own rounding at the
// target.  Along the tokens, for dw, every word has a scale of its own, since a word
// that is no token's target has small p alone (xent_align_kernel).
// bf16 tensors are multiplied as they are for the logits.  For the gradients
// they are laid out as fp16, scaled in the same way (their 8 bits fit down to
// 2^-31 of the largest), so that g can be rounded to fp16's 11 bits.  In bf16 g
// would lose as much as the results do when they are written, and the same
// way for every token where dloss is one value (dh of 4096 tokens: 2.8e-3 off
// instead of 1.7e-3, the result's own rounding).
//
// Few tokens (64 at most; 128 forward, fp32): reading w is what counts.  Its
// rows are multiplied where they are, fp32 by the fp32 matrix instructions
// without the passes that split it (through LDS where they are whole steps,
// else straight into registers), and by the vector units for four tokens or
// fewer; a second launch joins the parts.  Backward,
// one launch leaves g in fp32, and one takes each block of w's rows to dh's
// partial sums and writes the same rows of dw; four tokens of fp32 or fewer take
// w's rows once for both.
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
constexpr int kJoinTokens = kWave;
constexpr int kJoinSlices = 16;
constexpr int kGradShift = 15;          // g's scale, and of a word's g beyond it:
constexpr int kWordShift = 8, kWordShiftMost = 136;   // a multiple, the largest
constexpr int64_t kPieceBytes = int64_t(256) << 20;   // g along both axes, one piece

// The form that the gradients' products take for tensors multiplied as P.
template <Prec P>
constexpr Prec kGradOf = P == Prec::kBf16 ? Prec::kHalf : P;

// A tensor's element as it is stored.
template <Prec P>
__device__ __forceinline__ float element(const void *p, int64_t i) {
    return P == Prec::kBf16 ? float(static_cast<const __bf16 *>(p)[i]) : static_cast<const float *>(p)[i];
}

// Eight consecutive elements, at any alignment.
template <Prec P>
__device__ __forceinline__ void load8(const void *p, int64_t i, float (&v)[8]) {
    if constexpr (P != Prec::kBf16) {
        const f32x4u *q = reinterpret_cast<const f32x4u *>(static_cast<const float *>(p) + i);
        const f32x4u a = q[0], b = q[1];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[k] = a[k];
            v[4 + k] = b[k];
        }
    } else {
        typedef __bf16 bf16x8u __attribute__((ext_vector_type(8), aligned(2)));
        const bf16x8u a = *reinterpret_cast<const bf16x8u *>(static_cast<const __bf16 *>(p) + i);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = float(a[k]);
    }
}

// Eight consecutive values of an operand's row, the first a multiple of eight.
template <Prec P>
__device__ __forceinline__ void store8(char *row, int32_t c, const float (&y)[8]) {
    if constexpr (P == Prec::kSplit) {
        store_split8(row, c, y);
    } else if constexpr (P == Prec::kHalf) {
        f16x8 v;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = _Float16(y[k]);
        *reinterpret_cast<f16x8 *>(row + int64_t(c) * 2) = v;
    } else {
        static_assert(P == Prec::kBf16, "fp32 operands are not laid out as they are");
        bf16x8 v;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = __bf16(y[k]);
        *reinterpret_cast<bf16x8 *>(row + int64_t(c) * 2) = v;
    }
}

// What a call knows of its tensors.
struct Xent {
    const void *h, *w;
    int64_t ld_h, ld_w;
    const int64_t *target;
    int64_t ignore;
    int32_t tokens, vocab, hidden;
};

// Control words at the workspace's start.
constexpr int kTopBlocksW = 768, kTopBlocksH = 128;   // workgroups that look for magnitudes, at most
struct Control {
    uint32_t status;
    // bits of the largest finite |w|, |h| and |dloss h| that each of those
    // found; a tensor's magnitude is the largest of them (atomics on one word
    // would take 13 ns each, one after the other)
    uint32_t w[kTopBlocksW], h[kTopBlocksH], weighted[kTopBlocksH];
    // and that (from the pass that lays the tensors out on)
    uint32_t top[3];
};
enum { kTopH, kTopW, kTopWeighted };
constexpr int kControlBytes = 8192;
static_assert(sizeof(Control) <= kControlBytes, "control words");

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

// The status word, by one workgroup.
__device__ __forceinline__ void write_status(const Xent &x, Control *control) {
    bool bad = false;
    for (int32_t t = threadIdx.x; t < x.tokens; t += blockDim.x) {
        const int64_t v = x.target[t];
        bad |= v != x.ignore && (v < 0 || v >= x.vocab);
    }
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) control->status = bad ? kXentBadTarget : 0u;
}

// Largest finite magnitudes.  Workgroups [0, w_blocks) sweep w, the others h
// (rows that count) and, with dloss, dloss h.  Eight elements a lane; rows with
// gaps, and those of h, are a wave's each.  Bound by HBM: 374 us for 131,072 x
// 4,096 words in fp32 (5.7 TB/s).
template <Prec P>
__global__ __launch_bounds__(kPackBlock) void xent_top_kernel(Xent x, const float *dloss, uint32_t w_blocks,
                                                              Control *control) {
    __shared__ uint32_t s_wave[kWaves];
    const bool of_w = blockIdx.x < w_blocks;
    const uint32_t block = of_w ? blockIdx.x : blockIdx.x - w_blocks;
    const uint32_t blocks = of_w ? w_blocks : gridDim.x - w_blocks;
    uint32_t top = 0u, weighted = 0u;
    if (of_w && x.ld_w == x.hidden) {   // without gaps: one vector
        constexpr int kAhead = 4;
        const int64_t size = int64_t(x.vocab) * x.hidden;
        const int64_t step = int64_t(blocks) * kPackBlock * 8;
        for (int64_t i = (int64_t(block) * kPackBlock + threadIdx.x) * 8; i < size; i += kAhead * step) {
            float v[kAhead][8] = {};
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                const int64_t at = i + q * step;
                if (at + 8 <= size) load8<P>(x.w, at, v[q]);
                else
                    for (int k = 0; k < 8; ++k)
                        if (at + k < size) v[q][k] = element<P>(x.w, at + k);
            }
#pragma unroll
            for (int q = 0; q < kAhead; ++q)
#pragma unroll
                for (int k = 0; k < 8; ++k) top = max(top, finite_bits(v[q][k]));
        }
    } else {
        const void *base = of_w ? x.w : x.h;
        const int64_t ld = of_w ? x.ld_w : x.ld_h;
        const int32_t rows = of_w ? x.vocab : x.tokens;
        const int lane = threadIdx.x & (kWave - 1);
        for (int64_t r = int64_t(block) * kWaves + threadIdx.x / kWave; r < rows; r += int64_t(blocks) * kWaves) {
            if (!of_w && target_of(x, int32_t(r)) < 0) continue;
            const float f = !of_w && dloss != nullptr ? dloss[r] : 0.0f;
            int32_t c = lane * 8;
            for (; c + 8 <= x.hidden; c += kWave * 8) {
                float v[8];
                load8<P>(base, r * ld + c, v);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    top = max(top, finite_bits(v[k]));
                    weighted = max(weighted, finite_bits(__fmul_rn(f, v[k])));
                }
            }
            for (; c < x.hidden; ++c) {   // the row's last elements, of one lane
                const float v = element<P>(base, r * ld + c);
                top = max(top, finite_bits(v));
                weighted = max(weighted, finite_bits(__fmul_rn(f, v)));
            }
        }
    }
    top = block_max(top, s_wave);
    __syncthreads();
    weighted = block_max(weighted, s_wave);
    if (threadIdx.x == 0) {
        (of_w ? control->w : control->h)[block] = top;
        if (!of_w) control->weighted[block] = weighted;
    }
}

// What that found, to every thread of a workgroup.
template <int kFrom>
__device__ __forceinline__ uint32_t largest_of(const uint32_t *words, int32_t n, uint32_t *s_wave) {
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < kFrom; i += kPackBlock)
        if (i + int(threadIdx.x) < n) top = max(top, words[i + threadIdx.x]);
    top = block_max(top, s_wave);
    __syncthreads();
    return top;
}

// h or w as operands: `along` its rows (for the logits), and `turned`, a row
// for each of its columns (for the gradients); either may be null.  Rows of h
// that do not count are zeros.  The turned h holds dloss h.  `found`: the
// magnitudes of this tensor that the control words hold.  Bound by HBM: w of
// 131,072 x 4,096 in fp32 takes 1244 us along both axes (12 bytes an element:
// 5.2 TB/s).
template <Prec P>
__global__ __launch_bounds__(kPackBlock) void xent_pack_kernel(Xent x, bool of_w, const float *dloss, char *along,
                                                               char *turned, int32_t found, Control *control) {
    constexpr Prec G = kGradOf<P>;
    __shared__ float tile[kPackTile][kPackTile + 1];
    __shared__ float s_weight[kPackTile];
    __shared__ bool s_counts[kPackTile];
    __shared__ uint32_t s_wave[kWaves];
    const int tid = threadIdx.x;
    const int32_t rows = of_w ? x.vocab : x.tokens, cols = x.hidden;
    const int64_t ld = of_w ? x.ld_w : x.ld_h;
    const int32_t across = (cols + kPackTile - 1) / kPackTile;
    const int32_t r0 = int32_t(blockIdx.x / across) * kPackTile, c0 = int32_t(blockIdx.x % across) * kPackTile;
    if (tid < kPackTile) {
        const int32_t r = r0 + tid;
        s_counts[tid] = r < rows && (of_w || target_of(x, r) >= 0);
        s_weight[tid] = !of_w && dloss != nullptr && s_counts[tid] ? dloss[r] : 1.0f;
    }
    __syncthreads();
    uint32_t top = 0u, weighted = 0u;
    if (found > 0) {
        top = of_w ? largest_of<kTopBlocksW>(control->w, found, s_wave) : largest_of<kTopBlocksH>(control->h, found, s_wave);
        weighted = of_w ? top : largest_of<kTopBlocksH>(control->weighted, found, s_wave);
        if (blockIdx.x == 0 && tid == 0) {   // for the products
            control->top[of_w ? kTopW : kTopH] = top;
            if (!of_w) control->top[kTopWeighted] = weighted;
        }
    }
    const void *base = of_w ? x.w : x.h;
    for (int i = tid; i < kPackTile * 8; i += kPackBlock) {
        const int r = i / 8, c = i % 8 * 8;
        float v[8] = {};
        if (s_counts[r]) {
            const int64_t at = int64_t(r0 + r) * ld + c0 + c;
            if (c0 + c + 8 <= cols) load8<P>(base, at, v);
            else
                for (int k = 0; k < 8; ++k)
                    if (c0 + c + k < cols) v[k] = element<P>(base, at + k);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) tile[r][c + k] = v[k];
    }
    __syncthreads();
    if (along != nullptr) {
        const int exponent = P == Prec::kSplit ? scale_exponent(top) : 0;
        const int64_t stride = row_bytes<P>(cols);
        const int32_t end = row_values<P>(cols);
        for (int i = tid; i < kPackTile * 8; i += kPackBlock) {
            const int r = i / 8, c = i % 8 * 8;
            if (r0 + r >= rows || c0 + c >= end) continue;
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = P == Prec::kSplit ? ldexpf(tile[r][c + k], exponent) : tile[r][c + k];
            store8<P>(along + int64_t(r0 + r) * stride, c0 + c, v);
        }
    }
    if (turned != nullptr) {
        const int exponent = scale_exponent(weighted);
        const int64_t stride = row_bytes<G>(rows);
        const int32_t end = row_values<G>(rows);
        for (int i = tid; i < kPackTile * 8; i += kPackBlock) {
            const int r = i / 8, c = i % 8 * 8;   // of the turned tile
            if (c0 + r >= cols || r0 + c >= end) continue;
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = ldexpf(__fmul_rn(s_weight[c + k], tile[c + k][r]), exponent);
            store8<G>(turned + int64_t(c0 + r) * stride, r0 + c, v);
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
__device__ __forceinline__ int logit_exponent(const Control *__restrict__ control) {
    return P == Prec::kSplit ? -(scale_exponent(control->top[kTopH]) + scale_exponent(control->top[kTopW])) : 0;
}

template <Prec P>
__device__ __forceinline__ float logit(float acc, int exponent) {
    return P == Prec::kSplit ? ldexpf(acc, exponent) : acc;
}

// Forward: parts[tile row][token], and the targets' logits.  kRows: from h and w
// as they are, whatever their alignment, and not from operands.
// Bound by the matrix cores for many tokens (2,048 x 131,072 x 4,096, bf16: 1.95
// ms, 1130 TFLOP/s; 4,096 x 131,072 x 4,096, fp32: 10.5 ms, 418), by reading w for
// few (a token x 33,278 x 1,024, bf16: 14.9 us, 4.6 TB/s).
template <Prec P, class Tile, bool kRows>
__global__ __launch_bounds__(Tile::kThreads, Tile::kWavesPerSimd) void xent_forward_kernel(Xent x, Operand w, Operand h,
                                                                         const Control *__restrict__ control, Part *parts,
                                                                         float *target_logit) {
    __shared__ __align__(16) char lds[kRows ? Tile::kRows / 32 * Tile::kCols * sizeof(Part) : Tile::kLdsBytes];
    const uint32_t tv = (x.vocab + Tile::kRows - 1) / Tile::kRows, tt = (x.tokens + Tile::kCols - 1) / Tile::kCols;
    uint32_t r, c;
    banded(xcd_place(blockIdx.x, gridDim.x), tv, tt, r, c);
    const int32_t row0 = int32_t(r) * Tile::kRows, col0 = int32_t(c) * Tile::kCols;
    Tile tile;
    if constexpr (kRows) tile.run_rows(x.w, x.ld_w, x.vocab, x.h, x.ld_h, x.tokens, row0, col0, x.hidden);
    else tile.run(w, h, row0, col0, 0, int32_t(steps_of<P>(x.hidden)), lds);
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

// A token's parts joined: lanes are tokens, waves take every 16th part (2,048
// tokens of 512 parts: 24 us).
__global__ __launch_bounds__(kJoinTokens *kJoinSlices) void xent_join_kernel(Xent x, const Part *parts, int32_t nparts,
                                                                             const float *target_logit, float *loss,
                                                                             float *lse, Control *control) {
    __shared__ Part s_part[kJoinSlices][kJoinTokens];
    if (blockIdx.x == 0) write_status(x, control);
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

// The same for few tokens: a workgroup each (5 us, a launch's own time).
__global__ __launch_bounds__(kPackBlock) void xent_join_few_kernel(Xent x, const Part *parts, int32_t nparts,
                                                                   const float *target_logit, float *loss,
                                                                   float *lse, Control *control) {
    __shared__ Part s_part[kWaves];
    const int32_t t = int32_t(blockIdx.x);
    if (t == 0) write_status(x, control);
    Part p = {-INFINITY, 0.0f};
    for (int32_t i = threadIdx.x; i < nparts; i += kPackBlock) p = join(p, parts[int64_t(i) * x.tokens + t]);
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) p = join(p, Part{__shfl_xor(p.top, off), __shfl_xor(p.sum, off)});
    if ((threadIdx.x & (kWave - 1)) == 0) s_part[threadIdx.x / kWave] = p;
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < kWaves; ++w) p = join(p, s_part[w]);
    const bool counts = target_of(x, t) >= 0;
    const float v = __fadd_rn(p.top, logf(p.sum));
    lse[t] = counts ? v : 0.0f;
    loss[t] = counts ? __fsub_rn(v, target_logit[t]) : 0.0f;
}

// A word's scale beyond 2^15 in one tile, from the largest |g| 2^15 of its tokens
// there: a multiple of kWordShift, so that most tiles of a word agree, which still
// leaves that value 2^7 or more.
__device__ __forceinline__ int word_shift(uint32_t top) {
    const int most = top == 0u ? kWordShiftMost : scale_exponent(top);   // -1 at |g| = 1
    return min(max(most, 0) / kWordShift * kWordShift, kWordShiftMost);
}

// Backward: g of words [v0, v0 + words), as g [token][word] and gt [word][token],
// and the words' shifts in this tile's tokens, shift [word][tile].
// Both are written from the tile, turned in LDS, so that no pass turns g; bound
// by the matrix cores (a piece of 8,192 words for 4,096 tokens of 4,096: 679 us in
// fp32, 405 TFLOP/s; of 16,384 in bf16 534 us, 1030).
template <Prec P, class Tile>
__global__ __launch_bounds__(Tile::kThreads, Tile::kWavesPerSimd) void xent_grad_kernel(Xent x, Operand w, Operand h, int32_t v0,
                                                                      int32_t words, const float *lse,
                                                                      const Control *__restrict__ control, char *g, char *gt,
                                                                      uint8_t *shifts) {
    __shared__ __align__(16) char lds[Tile::kLdsBytes];
    const uint32_t tv = (words + Tile::kRows - 1) / Tile::kRows, tt = (x.tokens + Tile::kCols - 1) / Tile::kCols;
    uint32_t r, c;
    banded(xcd_place(blockIdx.x, gridDim.x), tv, tt, r, c);
    const int32_t row0 = int32_t(r) * Tile::kRows, col0 = int32_t(c) * Tile::kCols;
    Tile tile;
    tile.run(w, h, row0, col0, 0, int32_t(steps_of<P>(x.hidden)), lds);
    const int exponent = logit_exponent<P>(control);
    constexpr Prec G = kGradOf<P>;
    const int64_t g_row = row_bytes<G>(words), gt_row = row_bytes<G>(x.tokens);
    const int32_t words_end = row_values<G>(words), tokens_end = row_values<G>(x.tokens);
#pragma unroll
    for (int j = 0; j < Tile::kTilesN; ++j) {
        const int32_t t = col0 + Tile::col_of(j);
        const int32_t target = t < x.tokens ? target_of(x, t) : -1;
        const float shift = target >= 0 ? lse[t] : 0.0f;
#pragma unroll
        for (int i = 0; i < Tile::kTilesM; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int32_t v = row0 + Tile::row_of(i, e);
                float p = 0.0f;   // tokens that do not count, and the padding
                if (target >= 0 && v < words) {
                    p = expf(logit<P>(tile.acc[i][j][e], exponent) - shift);
                    if (v0 + v == target) p = __fsub_rn(p, 1.0f);
                    p = __fmul_rn(p, float(1 << kGradShift));   // dloss: in h^T, and in the last pass over dh
                }
                tile.acc[i][j][e] = p;
            }
    }
    using Out = Band<Tile>;
    Out band{reinterpret_cast<float *>(lds)};
    each_band<Tile::kTilesM>([&](auto index) {
        constexpr int i = decltype(index)::value;
        band.template put<i>(tile);
        float top[Out::kUnits];
#pragma unroll
        for (int k = 0; k < Out::kUnits; ++k) {
            float y[8];
            band.get(k, y);
            top[k] = 0.0f;   // (NaN has no part in it)
#pragma unroll
            for (int e = 0; e < 8; ++e) top[k] = fmaxf(top[k], fabsf(y[e]));
        }
        // of the word: neighbouring lanes have its tokens
#pragma unroll
        for (int bit = 1; bit < Out::kGroups; bit *= 2)
#pragma unroll
            for (int k = 0; k < Out::kUnits; ++k) top[k] = fmaxf(top[k], __shfl_xor(top[k], bit));
#pragma unroll
        for (int k = 0; k < Out::kUnits; ++k) {
            float y[8];
            const int32_t v = row0 + Out::tile_row(i, Out::row(k)), t = col0 + Out::col(k);
            const int more = word_shift(__float_as_uint(top[k]));
            if (v < words && t < tokens_end) {
                band.get(k, y);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = ldexpf(y[e], more);
                store8<G>(gt + v * gt_row, t, y);
            }
            if (v < words && t == col0) shifts[int64_t(v) * tt + c] = uint8_t(more);
        }
#pragma unroll
        for (int k = 0; k < Out::kUnits; ++k) {
            float y[8];
            const int32_t v = row0 + Out::tile_row(i, Out::turned_row(k)), t = col0 + Out::turned_col(k);
            if (t < x.tokens && v < words_end) {
                band.get_turned(k, y);
                store8<G>(g + t * g_row, v, y);
            }
        }
    });
}

// Brings all tiles of a word in gt to the smallest of their shifts, row_shift [word].
// A wave takes a word; values whose tile has that shift already are not touched.
// Bound by the way to memory and back (11 and 16 us for those pieces, of which 2 to
// 4 MB are rewritten).
template <Prec G>
__global__ __launch_bounds__(kPackBlock) void xent_align_kernel(char *gt, int64_t gt_row, int32_t words,
                                                                int32_t tokens_end, int32_t width, int32_t tiles,
                                                                const uint8_t *__restrict__ shifts,
                                                                uint8_t *__restrict__ row_shift) {
    const int lane = threadIdx.x & (kWave - 1);
    const int32_t v = int32_t(blockIdx.x) * kWaves + threadIdx.x / kWave;
    if (v >= words) return;
    const uint8_t *mine = shifts + int64_t(v) * tiles;
    int least = kWordShiftMost;
    for (int32_t i = lane; i < tiles; i += kWave) least = min(least, int(mine[i]));
#pragma unroll
    for (int bit = 1; bit < kWave; bit *= 2) least = min(least, __shfl_xor(least, bit));
    if (lane == 0) row_shift[v] = uint8_t(least);
    char *row = gt + v * gt_row;
#pragma unroll 4
    for (int32_t t = lane * 8; t < tokens_end; t += kWave * 8) {
        const int down = least - int(mine[t / width]);
        if (down == 0) continue;
        float y[8];
        if constexpr (G == Prec::kSplit) {
            const char *p = row + split_offset(t);
            const f16x8 hi = *reinterpret_cast<const f16x8 *>(p), lo = *reinterpret_cast<const f16x8 *>(p + 64);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = ldexpf(__fadd_rn(float(hi[e]), float(lo[e])), down);
        } else {
            const f16x8 hi = *reinterpret_cast<const f16x8 *>(row + int64_t(t) * 2);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = ldexpf(float(hi[e]), down);
        }
        store8<G>(row, t, y);
    }
}

// dw rows [v0, v0 + words) = g^T h.  Bound by the matrix cores (the same pieces:
// 635 and 492 us, 433 and 1118 TFLOP/s).
template <Prec P, class Tile>
__global__ __launch_bounds__(Tile::kThreads, Tile::kWavesPerSimd) void xent_dw_kernel(Xent x, Operand gt, Operand ht, int32_t v0,
                                                                    const Control *__restrict__ control,
                                                                    const uint8_t *__restrict__ row_shift, void *dw,
                                                                    int64_t ld) {
    __shared__ __align__(16) char lds[Tile::kLdsBytes];
    const uint32_t tv = (gt.rows + Tile::kRows - 1) / Tile::kRows, th = (x.hidden + Tile::kCols - 1) / Tile::kCols;
    uint32_t r, c;
    banded(xcd_place(blockIdx.x, gridDim.x), tv, th, r, c);
    const int32_t row0 = int32_t(r) * Tile::kRows, col0 = int32_t(c) * Tile::kCols;
    uint32_t four[Tile::kTilesM][4];   // shifts of four neighbouring rows
#pragma unroll
    for (int i = 0; i < Tile::kTilesM; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            four[i][q] = reinterpret_cast<const uint32_t *>(row_shift)[min(row0 + Tile::row_of(i, 4 * q), gt.rows - 1) / 4];
    Tile tile;
    tile.run(gt, ht, row0, col0, 0, int32_t(steps_of<kGradOf<P>>(x.tokens)), lds);
    const int exponent = -(kGradShift + scale_exponent(control->top[kTopWeighted]));
#pragma unroll
    for (int i = 0; i < Tile::kTilesM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int32_t v = row0 + Tile::row_of(i, e);
            if (v >= gt.rows) continue;
            const int of_word = exponent - int(four[i][e >> 2] >> 8 * (e & 3) & 255u);
#pragma unroll
            for (int j = 0; j < Tile::kTilesN; ++j) {
                const int32_t k = col0 + Tile::col_of(j);
                if (k >= x.hidden) continue;
                const int64_t at = (int64_t(v0) + v) * ld + k;
                const float y = ldexpf(tile.acc[i][j][e], of_word);
                if constexpr (P == Prec::kSplit) static_cast<float *>(dw)[at] = y;
                else static_cast<__bf16 *>(dw)[at] = __bf16(y);
            }
        }
}

// Partial sums of dh: split s adds its share of the piece's words to
// part[s][token][hidden] (or starts it, with the first piece).  As dw (680 and 502
// us, 404 and 1095 TFLOP/s).
template <Prec P, class Tile>
__global__ __launch_bounds__(Tile::kThreads, Tile::kWavesPerSimd) void xent_dh_kernel(Xent x, Operand g, Operand wt, int32_t steps,
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

// dh from its partial sums: a stream (4,096 x 4,096: 40 us).
template <Prec P>
__global__ __launch_bounds__(kPackBlock) void xent_dh_join_kernel(Xent x, const float *part, int32_t splits,
                                                                  const float *dloss, Control *control, void *dh,
                                                                  int64_t ld) {
    if (blockIdx.x == 0) write_status(x, control);
    const int exponent = -(kGradShift + scale_exponent(control->top[kTopW]));
    const int64_t size = int64_t(x.tokens) * x.hidden;
    for (int64_t i = int64_t(blockIdx.x) * kPackBlock + threadIdx.x; i < size; i += int64_t(gridDim.x) * kPackBlock) {
        const int32_t t = int32_t(i / x.hidden), k = int32_t(i - int64_t(t) * x.hidden);
        float v = 0.0f;
        if (target_of(x, t) >= 0) {
            for (int32_t s = 0; s < splits; ++s) v = __fadd_rn(v, part[s * size + i]);
            v = __fmul_rn(ldexpf(v, exponent), dloss[t]);
        }
        const int64_t at = t * ld + k;
        if constexpr (P == Prec::kSplit) static_cast<float *>(dh)[at] = v;
        else static_cast<__bf16 *>(dh)[at] = __bf16(v);
    }
}

// One to four tokens: a wave takes rows of w, its lanes 16 bytes each along
// them, so that rows of any alignment come in whole lines, and multiplies on
// the vector units (kTok operations an element).  kGrad: g as
// xent_few_grad_kernel leaves it; else parts and target logits as
// xent_forward_kernel does.  A workgroup covers 64 words, a wave 16 of them, in
// one group or (more tokens: registers) two.  A call of 56,852 words x 2,758 (in
// brackets 2,752, whole steps), us, against the matrix cores: fp32, three tokens
// 126 and 268 (145, 155); eight, by a variant of this, 232 and 278 (240, 155); bf16,
// three tokens 76 and 110, eight 94 and 119.  bf16 rows in whole steps are as fast
// or faster through the matrix cores at any count (three tokens 61 either way, one
// token x 33,278 x 1,024 15 against 18).
constexpr int kDotTokens = 4, kDotWords = 64;
template <Prec P>
bool take_dot(int32_t tokens, bool in_steps) {
    return tokens <= kDotTokens && (P == Prec::kFp32 || !in_steps);
}

// Sums of N (a power of two) values over the wave's lanes; lane l gets that of
// value l / (64 / N).  A stage halves the values: each lane keeps one half and
// sends the other.
template <int N, int kBit = kWave / 2, int M>
__device__ __forceinline__ float sum_scattered(float (&v)[M]) {
    if constexpr (N > 1) {
        const bool upper = (threadIdx.x & kBit) != 0;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const float keep = upper ? v[i + N / 2] : v[i], send = upper ? v[i] : v[i + N / 2];
            v[i] = __fadd_rn(keep, __shfl_xor(send, kBit));
        }
        return sum_scattered<N / 2, kBit / 2>(v);
    } else if constexpr (kBit > 0) {
        v[0] = __fadd_rn(v[0], __shfl_xor(v[0], kBit));
        return sum_scattered<1, kBit / 2>(v);
    } else {
        return v[0];
    }
}

// 16 bytes of elements, at any alignment.
template <Prec P>
constexpr int kVec = P == Prec::kBf16 ? 8 : 4;
template <Prec P>
__device__ __forceinline__ void load_vec(const void *p, int64_t i, float (&v)[kVec<P>]) {
    if constexpr (P == Prec::kBf16) {
        load8<P>(p, i, v);
    } else {
        const f32x4u a = *reinterpret_cast<const f32x4u *>(static_cast<const float *>(p) + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = a[k];
    }
}

template <Prec P, int kTok, bool kGrad>
__global__ __launch_bounds__(kPackBlock) void xent_dot_kernel(Xent x, Part *__restrict__ parts,
                                                              float *__restrict__ target_logit,
                                                              const float *__restrict__ lse,
                                                              const float *__restrict__ dloss, float *__restrict__ g,
                                                              int64_t words_end) {
    constexpr int kRows = kTok <= 2 ? 16 : 8, kGroups = kDotWords / kWaves / kRows;
    constexpr int kSums = kRows * kTok, kSame = kWave / kSums;   // lanes that get one sum
    constexpr int kEach = kVec<P>;
    __shared__ Part s_part[kWaves][kTok];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int token = lane / kSame / kRows;   // of this lane's sum
    const bool there = token < x.tokens;
    const int32_t target = there ? target_of(x, token) : -1;
    const float shift = kGrad && target >= 0 ? lse[token] : 0.0f, weight = kGrad && target >= 0 ? dloss[token] : 0.0f;
    Part part = {-INFINITY, 0.0f};
    for (int group = 0; group < kGroups; ++group) {
        const int32_t v0 = int32_t(blockIdx.x) * kDotWords + (wave * kGroups + group) * kRows;
        float sum[kSums];   // [token][row]
#pragma unroll
        for (int i = 0; i < kSums; ++i) sum[i] = 0.0f;
        int32_t k = lane * kEach;
        for (; k + kEach <= x.hidden; k += kWave * kEach) {
            float w[kRows][kEach], h[kTok][kEach];
#pragma unroll
            for (int r = 0; r < kRows; ++r) load_vec<P>(x.w, min(v0 + r, x.vocab - 1) * x.ld_w + k, w[r]);
#pragma unroll
            for (int t = 0; t < kTok; ++t) load_vec<P>(x.h, min(t, x.tokens - 1) * x.ld_h + k, h[t]);
#pragma unroll
            for (int r = 0; r < kRows; ++r)
#pragma unroll
                for (int t = 0; t < kTok; ++t)
#pragma unroll
                    for (int e = 0; e < kEach; ++e) sum[t * kRows + r] = fmaf(w[r][e], h[t][e], sum[t * kRows + r]);
        }
        for (; k < x.hidden; ++k) {   // the rows' last values, of one lane
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const float w = element<P>(x.w, min(v0 + r, x.vocab - 1) * x.ld_w + k);
#pragma unroll
                for (int t = 0; t < kTok; ++t)
                    sum[t * kRows + r] = fmaf(w, element<P>(x.h, min(t, x.tokens - 1) * x.ld_h + k), sum[t * kRows + r]);
            }
        }
        float l = sum_scattered<kSums>(sum);
        const int32_t v = v0 + lane / kSame % kRows;
        if constexpr (kGrad) {
            if (there && lane % kSame == 0) {
                float p = 0.0f;
                if (target >= 0 && v < x.vocab) {
                    p = expf(l - shift);
                    if (v == target) p = __fsub_rn(p, 1.0f);
                    p = __fmul_rn(p, weight);
                }
                g[token * words_end + v] = p;
            }
        } else {
            if (v >= x.vocab) l = -INFINITY;
            if (v == target && lane % kSame == 0) target_logit[token] = l;
            // (a NaN has no maximum; it goes into the sum)
            part = join(part, l != l ? Part{-INFINITY, l} : Part{l, l == -INFINITY ? 0.0f : 1.0f});
        }
    }
    if constexpr (!kGrad) {
        // over the rows of a token, which are neighbouring lanes
#pragma unroll
        for (int bit = kSame; bit < kSame * kRows; bit *= 2)
            part = join(part, Part{__shfl_xor(part.top, bit), __shfl_xor(part.sum, bit)});
        if (lane % (kSame * kRows) == 0) s_part[wave][token] = part;
        __syncthreads();
        if (threadIdx.x < kTok && int(threadIdx.x) < x.tokens) {
            Part p = s_part[0][threadIdx.x];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) p = join(p, s_part[w][threadIdx.x]);
            parts[int64_t(blockIdx.x) * x.tokens + threadIdx.x] = p;
        }
    }
}

// One to four tokens, backward in one pass over w: a workgroup takes four words
// at a time with the whole hidden axis in its registers, 4 kSlots values a
// thread; the logits' sums meet in LDS, and the same registers serve
// dh += g w and dw = g h.  h and this workgroup's share of dh stay in registers
// throughout.  Bound by reading w and writing dw (three tokens x 56,852 x 2,758:
// 239 us, 5.2 TB/s; with the forward call 405).
constexpr int kOnceWords = 4;

template <int kTok, int kSlots>
__global__ __launch_bounds__(kPackBlock, 2) void xent_once_kernel(Xent x, const float *__restrict__ lse,
                                                                  const float *__restrict__ dloss,
                                                                  float *__restrict__ dw, int64_t ld_dw,
                                                                  float *__restrict__ part) {
    constexpr int kSums = kOnceWords * kTok, kSame = kWave / kSums;   // lanes that get one sum
    __shared__ float s_sum[2][kWaves][kSums], s_g[2][kSums];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    auto place = [&](int slot) { return (slot * kPackBlock + tid) * 4; };
    auto load = [&](const void *base, int64_t row, int slot, float (&v)[4]) {
        const int32_t k = place(slot);
        const float *p = static_cast<const float *>(base) + row + k;
        if (k + 4 <= x.hidden) {
            const f32x4u a = *reinterpret_cast<const f32x4u *>(p);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = a[e];
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = k + e < x.hidden ? p[e] : 0.0f;
        }
    };
    auto store = [&](float *row, int slot, const float (&v)[4]) {
        const int32_t k = place(slot);
        if (k + 4 <= x.hidden) {
            *reinterpret_cast<f32x4u *>(row + k) = f32x4u{v[0], v[1], v[2], v[3]};
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (k + e < x.hidden) row[k + e] = v[e];
        }
    };
    // h; zeros where a token does not count, whatever its row holds
    float h[kTok][kSlots][4], dh[kTok][kSlots][4];
#pragma unroll
    for (int t = 0; t < kTok; ++t) {
        const bool counts = t < x.tokens && target_of(x, t) >= 0;
#pragma unroll
        for (int q = 0; q < kSlots; ++q) {
#pragma unroll
            for (int e = 0; e < 4; ++e) h[t][q][e] = dh[t][q][e] = 0.0f;
            if (counts) load(x.h, t * x.ld_h, q, h[t][q]);
        }
    }
    // thread i < kSums: the sum of token i / 4 and word i % 4
    const int token = tid / kOnceWords;
    const int32_t target = tid < kSums && token < x.tokens ? target_of(x, token) : -1;
    const float shift = target >= 0 ? lse[token] : 0.0f, weight = target >= 0 ? dloss[token] : 0.0f;
    const int32_t groups = (x.vocab + kOnceWords - 1) / kOnceWords;
    int turn = 0;   // the other half of LDS may still be read
    for (int32_t group = blockIdx.x; group < groups; group += gridDim.x, turn ^= 1) {
        const int32_t v0 = group * kOnceWords;
        float w[kOnceWords][kSlots][4], sum[kSums];
#pragma unroll
        for (int r = 0; r < kOnceWords; ++r)
#pragma unroll
            for (int q = 0; q < kSlots; ++q) load(x.w, min(v0 + r, x.vocab - 1) * x.ld_w, q, w[r][q]);
#pragma unroll
        for (int t = 0; t < kTok; ++t)
#pragma unroll
            for (int r = 0; r < kOnceWords; ++r) {
                float l = 0.0f;
#pragma unroll
                for (int q = 0; q < kSlots; ++q)
#pragma unroll
                    for (int e = 0; e < 4; ++e) l = fmaf(w[r][q][e], h[t][q][e], l);
                sum[t * kOnceWords + r] = l;
            }
        const float mine = sum_scattered<kSums>(sum);
        if (lane % kSame == 0) s_sum[turn][wave][lane / kSame] = mine;
        __syncthreads();
        if (tid < kSums) {
            float l = s_sum[turn][0][tid], p = 0.0f;
#pragma unroll
            for (int k = 1; k < kWaves; ++k) l = __fadd_rn(l, s_sum[turn][k][tid]);
            const int32_t v = v0 + tid % kOnceWords;
            if (target >= 0 && v < x.vocab) {
                p = expf(l - shift);
                if (v == target) p = __fsub_rn(p, 1.0f);
                p = __fmul_rn(p, weight);
            }
            s_g[turn][tid] = p;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kOnceWords; ++r) {
            float g[kTok];
#pragma unroll
            for (int t = 0; t < kTok; ++t) g[t] = s_g[turn][t * kOnceWords + r];
#pragma unroll
            for (int q = 0; q < kSlots; ++q) {
                float y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    y[e] = 0.0f;
#pragma unroll
                    for (int t = 0; t < kTok; ++t) {
                        y[e] = fmaf(g[t], h[t][q][e], y[e]);
                        dh[t][q][e] = fmaf(g[t], w[r][q][e], dh[t][q][e]);
                    }
                }
                if (v0 + r < x.vocab) store(dw + (v0 + r) * ld_dw, q, y);
            }
        }
    }
    float *to = part + int64_t(blockIdx.x) * x.tokens * x.hidden;
#pragma unroll
    for (int t = 0; t < kTok; ++t)
        if (t < x.tokens)
#pragma unroll
            for (int q = 0; q < kSlots; ++q) store(to + int64_t(t) * x.hidden, q, dh[t][q]);
}

// Few tokens: g as fp32 [token][word], rows `words_end` long (a multiple of 64;
// zeros past the vocabulary and for tokens that do not count).  Bound by reading
// w: 16 tokens x 50,001 x 1,024, bf16: 20.7 us, 5.0 TB/s.
template <Prec P, class Tile, bool kRows>
__global__ __launch_bounds__(Tile::kThreads, Tile::kWavesPerSimd) void xent_few_grad_kernel(Xent x, Operand w, Operand h, const float *lse,
                                                                       const float *dloss, float *g,
                                                                       int64_t words_end) {
    __shared__ __align__(16) char lds[kRows ? 16 : Tile::kLdsBytes];
    const int32_t row0 = int32_t(blockIdx.x) * Tile::kRows;
    Tile tile;
    if constexpr (kRows) tile.run_rows(x.w, x.ld_w, x.vocab, x.h, x.ld_h, x.tokens, row0, 0, x.hidden);
    else tile.run(w, h, row0, 0, 0, int32_t(steps_of<P>(x.hidden)), lds);
#pragma unroll
    for (int j = 0; j < Tile::kTilesN; ++j) {
        const int32_t t = Tile::col_of(j);
        if (t >= x.tokens) continue;
        const int32_t target = target_of(x, t);
        const float shift = target >= 0 ? lse[t] : 0.0f, weight = target >= 0 ? dloss[t] : 0.0f;
#pragma unroll
        for (int i = 0; i < Tile::kTilesM; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int32_t v4 = row0 + Tile::row_of(i, 4 * q);
                f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
                if (target >= 0) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        float p = expf(tile.acc[i][j][4 * q + k] - shift);
                        if (v4 + k == target) p = __fsub_rn(p, 1.0f);
                        y[k] = v4 + k < x.vocab ? __fmul_rn(p, weight) : 0.0f;
                    }
                }
                *reinterpret_cast<f32x4 *>(g + t * words_end + v4) = y;
            }
    }
}

// Few tokens: dw, and dh's partial sums.  A workgroup takes 256 values of the
// hidden axis (a wave 64, a lane four neighbours: column c of product j is
// value 4 c + j) and every splits-th block of 32 words.
//   dw[word][value]  = sum over tokens  g[word][token] h[token][value]
//   dh[token][value] += sum over words  g[token][word] w[word][value]
// with dh and h in registers throughout, 16 kTok tokens at most.  w's rows serve
// as they come from memory: a lane loads four values of words four, four + 4,
// .., four + 28 of the block (four = lane / 16), and that is what an
// instruction takes of column 4 c + j, if the other operand's words are in the
// same order.
//   fp32: eight 16 x 16 x 4 instructions, a word of each lane each.
//   bf16: one 16 x 16 x 32 instruction for g's high part and one for its low
//   part (g = hi + lo in bf16, 16 bits of it); w and h are exact.  With the fp32
//   instructions a step of 16 tokens took 92 us here, the matrix cores 39 (w
//   read and dw written: 5.3 TB/s).
constexpr int kFewHidden = 256, kFewWords = 32;

__device__ __forceinline__ f32x4 mfma_16(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

template <Prec P, int kTok>
__global__ __launch_bounds__(kPackBlock) void xent_few_products_kernel(Xent x, const float *__restrict__ g,
                                                                       int64_t words_end, int32_t splits,
                                                                       void *__restrict__ dw, int64_t ld_dw,
                                                                       float *__restrict__ part) {
    constexpr bool kWide = P == Prec::kBf16;
    constexpr int kTokens = 16 * kTok, kStride = kFewWords + 1;
    // bf16: tokens in steps of the wide instruction's 32
    constexpr int kSteps = kWide ? (kTokens + 31) / 32 : 4 * kTok;
    __shared__ float s_g[2][kTokens * kStride];
    typedef __bf16 bf16x4u __attribute__((ext_vector_type(4), aligned(2)));
    using Vec = std::conditional_t<kWide, bf16x4u, f32x4>;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int col = lane & 15, four = lane >> 4;
    const int32_t split = int32_t(blockIdx.x) % splits;
    const int32_t k0 = int32_t(blockIdx.x) / splits * kFewHidden + wave * 64 + col * 4;   // this lane's values
    const int32_t left = min(4, x.hidden - k0);   // of which exist

    auto load4 = [&](const void *base, int64_t at, bool there) {
        Vec v = {};
        if (!there) return v;
        if constexpr (kWide) {
            const __bf16 *p = static_cast<const __bf16 *>(base) + at;
            if (left == 4) v = *reinterpret_cast<const bf16x4u *>(p);
            else
#pragma unroll
                for (int k = 0; k < 3; ++k)
                    if (k < left) v[k] = p[k];
        } else {
            const float *p = static_cast<const float *>(base) + at;
            if (left == 4) v = *reinterpret_cast<const f32x4u *>(p);
            else
#pragma unroll
                for (int k = 0; k < 3; ++k)
                    if (k < left) v[k] = p[k];
        }
        return v;
    };
    // g's block in LDS as [token][word]
    constexpr int kLoads = kTokens * kFewWords / kPackBlock;
    float next[kLoads];
    auto fetch = [&](int32_t block) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int t = (i * kPackBlock + tid) / kFewWords, v = (i * kPackBlock + tid) % kFewWords;
            next[i] = t < x.tokens ? g[t * words_end + int64_t(block) * kFewWords + v] : 0.0f;
        }
    };
    auto rows_of_w = [&](int32_t block, Vec (&w)[8]) {
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const int32_t v = block * kFewWords + 4 * s + four;
            w[s] = load4(x.w, v * x.ld_w + k0, v < x.vocab && left > 0);
        }
    };
    // column j of eight rows, as the wide instruction takes it
    auto column = [](const Vec (&v)[8], int j) {
        bf16x8 b;
#pragma unroll
        for (int s = 0; s < 8; ++s) b[s] = __bf16(v[s][j]);
        return b;
    };

    // h, once: token 4 s + four of each step, or 32 step + 4 i + four
    Vec h_narrow[kWide ? 1 : kSteps];
    bf16x8 h_wide[kWide ? kSteps : 1][4];
    f32x4 dh[kTok][4];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        auto row = [&](int32_t t) {
            return load4(x.h, t * x.ld_h + k0, t < x.tokens && left > 0 && target_of(x, t) >= 0);
        };
        if constexpr (kWide) {
            Vec v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = row(32 * s + 4 * i + four);
#pragma unroll
            for (int j = 0; j < 4; ++j) h_wide[s][j] = column(v, j);
        } else {
            h_narrow[s] = row(4 * s + four);
        }
    }
#pragma unroll
    for (int t = 0; t < kTok; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) dh[t][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const int32_t blocks = (x.vocab + kFewWords - 1) / kFewWords;
    int turn = 0;
    Vec w[8];
    if (split < blocks) {
        fetch(split);
        rows_of_w(split, w);
    }
    for (int32_t block = split; block < blocks; block += splits, turn ^= 1) {
        float *sg = s_g[turn];   // the other one may still be read
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int t = (i * kPackBlock + tid) / kFewWords, v = (i * kPackBlock + tid) % kFewWords;
            sg[t * kStride + v] = next[i];
        }
        const int32_t v0 = block * kFewWords;
        __syncthreads();
        // dh first: its rows of w make room for the next block's
        if constexpr (kWide) {
            bf16x8 b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = column(w, j);
            if (block + splits < blocks) {
                fetch(block + splits);
                rows_of_w(block + splits, w);
            }
#pragma unroll
            for (int t = 0; t < kTok; ++t) {
                bf16x8 hi, lo;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float v = sg[(t * 16 + col) * kStride + 4 * i + four];
                    hi[i] = __bf16(v);
                    lo[i] = __bf16(__fsub_rn(v, float(hi[i])));
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) dh[t][j] = mfma_16(lo, b[j], mfma_16(hi, b[j], dh[t][j]));
            }
        } else {
#pragma unroll
            for (int s = 0; s < 8; ++s)
#pragma unroll
                for (int t = 0; t < kTok; ++t) {
                    const float a = sg[(t * 16 + col) * kStride + 4 * s + four];
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        dh[t][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, w[s][j], dh[t][j], 0, 0, 0);
                }
            if (block + splits < blocks) {
                fetch(block + splits);
                rows_of_w(block + splits, w);
            }
        }
        // dw: two rows of 16 words, four columns of 16 values
#pragma unroll
        for (int r = 0; r < kFewWords / 16; ++r) {
            f32x4 acc[4] = {};
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                if constexpr (kWide) {
                    bf16x8 hi, lo;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int t = 32 * s + 4 * i + four;
                        const float v = t < kTokens ? sg[t * kStride + r * 16 + col] : 0.0f;
                        hi[i] = __bf16(v);
                        lo[i] = __bf16(__fsub_rn(v, float(hi[i])));
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[j] = mfma_16(lo, h_wide[s][j], mfma_16(hi, h_wide[s][j], acc[j]));
                } else {
                    const float a = sg[(4 * s + four) * kStride + r * 16 + col];
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, h_narrow[s][j], acc[j], 0, 0, 0);
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int32_t v = v0 + r * 16 + four * 4 + e;
                if (v >= x.vocab || left <= 0) continue;
                const int64_t at = v * ld_dw + k0;
                if constexpr (kWide) {
                    __bf16 *p = static_cast<__bf16 *>(dw) + at;
                    const bf16x4u y = {__bf16(acc[0][e]), __bf16(acc[1][e]), __bf16(acc[2][e]), __bf16(acc[3][e])};
                    if (left == 4) *reinterpret_cast<bf16x4u *>(p) = y;
                    else
#pragma unroll
                        for (int j = 0; j < 3; ++j)
                            if (j < left) p[j] = y[j];
                } else {
                    float *p = static_cast<float *>(dw) + at;
                    if (left == 4) *reinterpret_cast<f32x4u *>(p) = f32x4u{acc[0][e], acc[1][e], acc[2][e], acc[3][e]};
                    else
#pragma unroll
                        for (int j = 0; j < 3; ++j)
                            if (j < left) p[j] = acc[j][e];
                }
            }
        }
    }
    float *to = part + int64_t(split) * x.tokens * x.hidden;
#pragma unroll
    for (int t = 0; t < kTok; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int32_t token = t * 16 + four * 4 + e;
            if (token >= x.tokens) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j < left) to[int64_t(token) * x.hidden + k0 + j] = dh[t][j][e];
        }
}

// dh of few tokens from its partial sums.
template <Prec P>
__global__ __launch_bounds__(kPackBlock) void xent_few_join_kernel(Xent x, const float *__restrict__ part, int32_t splits, void *__restrict__ dh,
                                                                   int64_t ld, Control *control) {
    __shared__ float s_sum[kWaves][kWave];
    if (blockIdx.x == 0) write_status(x, control);
    // a wave takes every fourth split of 64 values
    const int64_t size = int64_t(x.tokens) * x.hidden;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t i = int64_t(blockIdx.x) * kWave + lane;
    float v = 0.0f;
    if (i < size)
#pragma unroll 8
        for (int32_t s = wave; s < splits; s += kWaves) v = __fadd_rn(v, part[s * size + i]);
    s_sum[wave][lane] = v;
    __syncthreads();
    if (wave != 0 || i >= size) return;
    for (int k = 1; k < kWaves; ++k) v = __fadd_rn(v, s_sum[k][lane]);
    const int32_t t = int32_t(i / x.hidden);
    const int64_t at = t * ld + (i - int64_t(t) * x.hidden);
    if (target_of(x, t) < 0) v = 0.0f;
    if constexpr (P == Prec::kBf16) static_cast<__bf16 *>(dh)[at] = __bf16(v);
    else static_cast<float *>(dh)[at] = v;
}

// The status word of a call without tokens.
__global__ void xent_clear_kernel(Control *control) { control->status = 0u; }

// dw of no tokens.
template <class T>
__global__ __launch_bounds__(kPackBlock) void xent_zero_kernel(T *dw, int64_t ld, int32_t rows, int32_t cols) {
    const int64_t size = int64_t(rows) * cols;
    for (int64_t i = int64_t(blockIdx.x) * kPackBlock + threadIdx.x; i < size; i += int64_t(gridDim.x) * kPackBlock)
        dw[i / cols * ld + i % cols] = T(0.0f);
}

int64_t round256(int64_t v) { return (v + 255) / 256 * 256; }
int64_t tiles(int64_t len, int tile) { return (len + tile - 1) / tile; }

// Few tokens: reading w takes longer than multiplying it.  65,536 words x 2,048, us,
// where they are against laid out first: a step of fp32 with 16 tokens 499 and 1283,
// with 64 864 and 1306; of bf16 225 and 526, 344 and 532.  (dh of more than 64 does
// not fit xent_few_products_kernel's registers.)  Forward of fp32 with 64: 221 and
// 449; with 65, 96 and 128 the two are near each other (491 and 453, 517 and 449, 489
// and 448), and a call of loss alone does without a copy of the head.  Forward of
// bf16 with 64: 53 and 77; with 65 and 128, 58 and 66, 64 and 69.
constexpr int32_t kFewTokens = 64;
template <Prec P>
constexpr int32_t kFewForward = P == Prec::kFp32 ? 128 : 64;

// Whether backward takes w in one pass, and by how many workgroups: fp32, and
// rows that fill a workgroup's registers (half of them, of the shortest) but no
// more.  A step of three tokens x 56,852 x 2,758: 403 us against 620 in two
// passes, of 1 x 1,000 x 512 31 against 41, of 4 x 100,000 x 512 135 against 162.
constexpr int32_t kOnceHidden = 4096, kOnceLeast = 512;
bool take_once(int32_t tokens, int32_t hidden, bool fp32) {
    return fp32 && tokens <= kDotTokens && hidden >= kOnceLeast && hidden <= kOnceHidden;
}
// Two to a compute unit, or four where rows are short and leave lanes idle (3 x
// 33,278 x 700: 85 -> 77 us; 2 x 50,001 x 1,024 would take 136 for 128); with eight
// groups of words each at least.
int32_t once_blocks(int32_t vocab, int32_t hidden) {
    return int32_t(std::min<int64_t>(tiles(vocab, kOnceWords * 8), hidden <= kPackBlock * 3 ? 1024 : 512));
}

// How a backward call is cut, and where everything is in the workspace.
struct Plan {
    int32_t piece;    // words
    int32_t splits;   // of a piece, for dh
    int32_t few_splits;
    int64_t target_logit, parts, h_along, w_along, forward;
    int64_t h_turned, w_turned, g, gt, shifts, row_shift, dh;   // or, of few tokens,
    int64_t few_g, few_dh;
    int64_t total;
};

// The kind of tile that rows x cols, `times` over with `steps` each, is fastest
// with, and how many there are of each.
TileKind tile_kind(int64_t rows, int64_t cols, int64_t times, int64_t steps, int64_t (&n)[kTileKinds]) {
    int64_t work[kTileKinds];
    for (int k = 0; k < kTileKinds; ++k) {
        n[k] = tiles(rows, kTileSide[k]) * tiles(cols, kTileSide[k]) * times;
        work[k] = n[k] * steps;
    }
    return best_tile(work, steps);
}

// Calls run(tile, workgroups) with it.
template <Prec P, class F>
void with_tile(int64_t rows, int64_t cols, int64_t times, int64_t steps, F run) {
    int64_t n[kTileKinds];
    switch (tile_kind(rows, cols, times, steps, n)) {
        case kTiny: return run(TinyTile<P>(), n[kTiny]);
        case kSmall: return run(SmallTile<P>(), n[kSmall]);
        case kLarge: return run(LargeTile<P>(), n[kLarge]);
    }
}

// The forward product's (few tokens: tiles of 64 words).
template <Prec P>
TileKind forward_tile(int32_t tokens, int32_t vocab, int32_t hidden) {
    int64_t n[kTileKinds];
    return tokens <= kFewForward<P == Prec::kSplit ? Prec::kFp32 : P> ? kTiny
                                                                     : tile_kind(vocab, tokens, 1, steps_of<P>(hidden), n);
}

template <Prec P>
Plan plan_of(int32_t tokens, int32_t vocab, int32_t hidden) {
    constexpr Prec G = kGradOf<P>;
    constexpr int kTile = kTileSide[kLarge];
    Plan p = {};
    // whole large tiles of words, as many as the pieces' bytes allow
    if (tokens == 0) tokens = 1;   // (nothing is launched that reads them)
    const int64_t word = 2 * row_bytes<G>(tokens);
    int64_t piece = kPieceBytes / word / kTile * kTile;
    if (piece < 4 * kTile) piece = 4 * kTile;
    p.piece = int32_t(piece < vocab ? piece : vocab);
    // as many as two workgroups a compute unit take in one round, with eight
    // steps each at least
    const int64_t dh_tiles = tiles(tokens, kTileSide[kSmall]) * tiles(hidden, kTileSide[kSmall]);
    const int64_t steps = steps_of<G>(p.piece);
    int64_t splits = 512 / dh_tiles;
    if (splits > steps / 8) splits = steps / 8;
    p.splits = int32_t(splits < 1 ? 1 : splits);

    int64_t at = kControlBytes;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += round256(bytes);
        return here;
    };
    p.target_logit = take(int64_t(tokens) * 4);
    p.parts = take(int64_t(tokens) * tiles(vocab, kTileSide[forward_tile<P>(tokens, vocab, hidden)]) * 8);
    // few tokens read h and w where they are
    const bool laid_out = tokens > kFewForward<P == Prec::kSplit ? Prec::kFp32 : P>;
    auto take_along = [&]() {
        p.h_along = take(tokens * row_bytes<P>(hidden));
        p.w_along = take(vocab * row_bytes<P>(hidden));
    };
    if (laid_out) take_along();
    p.forward = at;
    if (tokens <= kFewTokens) {
        // the workgroups that three to a compute unit make, with eight blocks of
        // words each at least
        int64_t n = tiles(768, int(tiles(hidden, kFewHidden)));
        n = std::min(n, tiles(vocab, kFewWords * 8));
        if (take_once(tokens, hidden, P == Prec::kSplit || P == Prec::kFp32)) n = once_blocks(vocab, hidden);
        p.few_splits = int32_t(n);
        p.few_g = take(tokens * tiles(vocab, 64) * 64 * 4);
        p.few_dh = take(n * tokens * hidden * 4);
        p.total = at;
        return p;
    }
    if (!laid_out) take_along();
    p.h_turned = take(hidden * row_bytes<G>(tokens));
    p.w_turned = take(hidden * row_bytes<G>(vocab));
    p.g = take(tokens * row_bytes<G>(p.piece));
    p.gt = take(p.piece * row_bytes<G>(tokens));
    p.shifts = take(p.piece * tiles(tokens, kTileSide[kTiny]));   // of the smallest tiles
    p.row_shift = take(p.piece);
    p.dh = take(int64_t(p.splits) * tokens * hidden * 4);
    p.total = at;
    return p;
}

// Whether the tensor can be multiplied where it is: whole steps along its
// rows, 16-byte aligned.
template <Prec P>
bool direct(const void *p, int64_t ld, int32_t hidden) {
    return P != Prec::kSplit && hidden % kStepValues<P> == 0 && ld % (P == Prec::kFp32 ? 4 : 8) == 0 &&
           reinterpret_cast<uintptr_t>(p) % 16 == 0;
}

// The operands of the logits, laid out where they have to be; with `gradient`
// those of the gradients' products too.
template <Prec P>
void pack_operands(const Xent &x, const float *dloss, bool gradient, const Plan &plan, char *ws, Operand *h,
                   Operand *w, hipStream_t stream) {
    Control *control = reinterpret_cast<Control *>(ws);
    constexpr int kSize = P == Prec::kBf16 ? 2 : 4;
    const int64_t row = row_bytes<P>(x.hidden);
    // the largest magnitudes, where a scale needs them
    uint32_t w_blocks = 0, h_blocks = 0;
    if (P == Prec::kSplit || gradient) {
        w_blocks = uint32_t(std::min<int64_t>(tiles(x.vocab, kWaves), kTopBlocksW));
        h_blocks = uint32_t(std::min<int64_t>(tiles(x.tokens, kWaves), kTopBlocksH));
        xent_top_kernel<P><<<w_blocks + h_blocks, kPackBlock, 0, stream>>>(x, dloss, w_blocks, control);
    }
    auto pack = [&](bool of_w, const void *p, int64_t ld, int32_t rows, int64_t along, int64_t turned) {
        const bool in_place = direct<P>(p, ld, x.hidden);
        if (!in_place || gradient) {
            const int64_t blocks = tiles(rows, kPackTile) * tiles(x.hidden, kPackTile);
            xent_pack_kernel<P><<<uint32_t(blocks), kPackBlock, 0, stream>>>(
                x, of_w, dloss, in_place ? nullptr : ws + along, gradient ? ws + turned : nullptr,
                int32_t(of_w ? w_blocks : h_blocks), control);
        }
        return in_place ? Operand{static_cast<const char *>(p), ld * kSize, rows} : Operand{ws + along, row, rows};
    };
    *h = pack(false, x.h, x.ld_h, x.tokens, plan.h_along, plan.h_turned);
    *w = pack(true, x.w, x.ld_w, x.vocab, plan.w_along, plan.w_turned);
}

// Calls run with the narrow tile of `tokens`, kMost at most.
template <Prec P, int32_t kMost, class F>
void with_narrow_tile(int32_t tokens, F run) {
    static_assert(kMost == 64 || kMost == 128, "whole tiles");
    if (tokens <= 32) run(NarrowTile<P, 1>());
    else if (kMost == 64 || tokens <= 64) run(NarrowTile<P, 2>());
    else if constexpr (kMost == 128) run(NarrowTile<P, 4>());
}

// Few tokens: the operands are the tensors themselves.
template <Prec P>
Operand operand_of(const void *p, int64_t ld, int32_t rows) {
    return Operand{static_cast<const char *>(p), ld * (P == Prec::kBf16 ? 2 : 4), rows};
}

template <Prec P>
hipError_t forward_few(const Xent &x, const Plan &plan, float *loss, float *lse, char *ws, hipStream_t stream) {
    Control *control = reinterpret_cast<Control *>(ws);
    Part *parts = reinterpret_cast<Part *>(ws + plan.parts);
    float *target_logit = reinterpret_cast<float *>(ws + plan.target_logit);
    const bool in_steps = direct<P>(x.w, x.ld_w, x.hidden) && direct<P>(x.h, x.ld_h, x.hidden);
    const Operand h = operand_of<P>(x.h, x.ld_h, x.tokens), w = operand_of<P>(x.w, x.ld_w, x.vocab);
    int32_t nparts = int32_t(tiles(x.vocab, kDotWords));
    auto dot = [&](auto kernel) {
        kernel<<<uint32_t(nparts), kPackBlock, 0, stream>>>(x, parts, target_logit, nullptr, nullptr, nullptr, 0);
    };
    if (take_dot<P>(x.tokens, in_steps))
        x.tokens == 1   ? dot(xent_dot_kernel<P, 1, false>)
        : x.tokens == 2 ? dot(xent_dot_kernel<P, 2, false>)
                        : dot(xent_dot_kernel<P, 4, false>);
    else with_narrow_tile<P, kFewForward<P>>(x.tokens, [&](auto tile) {
        using Tile = decltype(tile);
        static_assert(Tile::kRows == kDotWords, "parts of as many words");
        auto run = [&](auto kernel) {
            kernel<<<uint32_t(nparts), Tile::kThreads, 0, stream>>>(x, w, h, control, parts, target_logit);
        };
        in_steps ? run(xent_forward_kernel<P, Tile, false>) : run(xent_forward_kernel<P, Tile, true>);
    });
    xent_join_few_kernel<<<uint32_t(x.tokens), kPackBlock, 0, stream>>>(x, parts, nparts, target_logit, loss, lse,
                                                                        control);
    return hipGetLastError();
}

template <Prec P>
hipError_t backward_few(const Xent &x, const Plan &plan, const float *lse, const float *dloss, void *dh, int64_t ld_dh,
                        void *dw, int64_t ld_dw, char *ws, hipStream_t stream) {
    const bool in_steps = direct<P>(x.w, x.ld_w, x.hidden) && direct<P>(x.h, x.ld_h, x.hidden);
    const Operand h = operand_of<P>(x.h, x.ld_h, x.tokens), w = operand_of<P>(x.w, x.ld_w, x.vocab);
    float *g = reinterpret_cast<float *>(ws + plan.few_g), *part = reinterpret_cast<float *>(ws + plan.few_dh);
    auto finish = [&]() {
        xent_few_join_kernel<P><<<uint32_t(tiles(int64_t(x.tokens) * x.hidden, kWave)), kPackBlock, 0, stream>>>(
            x, part, plan.few_splits, dh, ld_dh, reinterpret_cast<Control *>(ws));
        return hipGetLastError();
    };
    if constexpr (P == Prec::kFp32)
        if (take_once(x.tokens, x.hidden, true)) {
            auto once = [&](auto kernel) {
                kernel<<<uint32_t(plan.few_splits), kPackBlock, 0, stream>>>(x, lse, dloss, static_cast<float *>(dw), ld_dw,
                                                                             part);
            };
            auto with_slots = [&](auto slots) {
                constexpr int n = decltype(slots)::value;
                x.tokens == 1   ? once(xent_once_kernel<1, n>)
                : x.tokens == 2 ? once(xent_once_kernel<2, n>)
                                : once(xent_once_kernel<4, n>);
            };
            switch (tiles(x.hidden, kPackBlock * 4)) {
                case 1: with_slots(std::integral_constant<int, 1>()); break;
                case 2: with_slots(std::integral_constant<int, 2>()); break;
                case 3: with_slots(std::integral_constant<int, 3>()); break;
                case 4: with_slots(std::integral_constant<int, 4>()); break;
            }
            return finish();
        }
    const int64_t words_end = tiles(x.vocab, kDotWords) * kDotWords;
    auto dot = [&](auto kernel) {
        kernel<<<uint32_t(words_end / kDotWords), kPackBlock, 0, stream>>>(x, nullptr, nullptr, lse, dloss, g, words_end);
    };
    if (take_dot<P>(x.tokens, in_steps))
        x.tokens == 1   ? dot(xent_dot_kernel<P, 1, true>)
        : x.tokens == 2 ? dot(xent_dot_kernel<P, 2, true>)
                        : dot(xent_dot_kernel<P, 4, true>);
    else with_narrow_tile<P, kFewTokens>(x.tokens, [&](auto tile) {
        using Tile = decltype(tile);
        static_assert(Tile::kRows == kDotWords, "g's rows end with the tiles");
        auto run = [&](auto kernel) {
            kernel<<<uint32_t(tiles(x.vocab, Tile::kRows)), Tile::kThreads, 0, stream>>>(x, w, h, lse, dloss, g,
                                                                                         words_end);
        };
        in_steps ? run(xent_few_grad_kernel<P, Tile, false>) : run(xent_few_grad_kernel<P, Tile, true>);
    });
    const uint32_t blocks = uint32_t(tiles(x.hidden, kFewHidden) * plan.few_splits);
    auto run = [&](auto kernel) {
        kernel<<<blocks, kPackBlock, 0, stream>>>(x, g, words_end, plan.few_splits, dw, ld_dw, part);
    };
    if (x.tokens <= 16) run(xent_few_products_kernel<P, 1>);
    else if (x.tokens <= 32) run(xent_few_products_kernel<P, 2>);
    else run(xent_few_products_kernel<P, 4>);
    return finish();
}

template <Prec P>
hipError_t forward(const Xent &x, float *loss, float *lse, char *ws, hipStream_t stream) {
    const Plan plan = plan_of<P>(x.tokens, x.vocab, x.hidden);
    Control *control = reinterpret_cast<Control *>(ws);
    Part *parts = reinterpret_cast<Part *>(ws + plan.parts);
    float *target_logit = reinterpret_cast<float *>(ws + plan.target_logit);
    constexpr Prec F = P == Prec::kSplit ? Prec::kFp32 : P;
    if (x.tokens <= kFewForward<F>) return forward_few<F>(x, plan, loss, lse, ws, stream);
    Operand h, w;
    pack_operands<P>(x, nullptr, false, plan, ws, &h, &w, stream);
    int32_t nparts = 0;
    with_tile<P>(x.vocab, x.tokens, 1, steps_of<P>(x.hidden), [&](auto tile, int64_t blocks) {
        using Tile = decltype(tile);
        nparts = int32_t(tiles(x.vocab, Tile::kRows));
        xent_forward_kernel<P, Tile, false><<<uint32_t(blocks), Tile::kThreads, 0, stream>>>(x, w, h, control, parts,
                                                                                             target_logit);
    });
    xent_join_kernel<<<uint32_t(tiles(x.tokens, kJoinTokens)), kJoinTokens * kJoinSlices, 0, stream>>>(
        x, parts, nparts, target_logit, loss, lse, control);
    return hipGetLastError();
}

template <Prec P>
hipError_t backward(const Xent &x, const float *lse, const float *dloss, void *dh, int64_t ld_dh, void *dw,
                    int64_t ld_dw, char *ws, hipStream_t stream) {
    constexpr Prec G = kGradOf<P>;
    const Plan plan = plan_of<P>(x.tokens, x.vocab, x.hidden);
    Control *control = reinterpret_cast<Control *>(ws);
    constexpr Prec F = P == Prec::kSplit ? Prec::kFp32 : P;
    if (x.tokens <= kFewTokens) return backward_few<F>(x, plan, lse, dloss, dh, ld_dh, dw, ld_dw, ws, stream);
    Operand h, w;
    pack_operands<P>(x, dloss, true, plan, ws, &h, &w, stream);
    const int64_t t_row = row_bytes<G>(x.tokens), v_row = row_bytes<G>(x.vocab);
    const Operand ht{ws + plan.h_turned, t_row, x.hidden};
    float *part = reinterpret_cast<float *>(ws + plan.dh);
    for (int64_t v0 = 0; v0 < x.vocab; v0 += plan.piece) {
        const int32_t words = int32_t(std::min<int64_t>(plan.piece, x.vocab - v0));
        const Operand w_piece{w.base + v0 * w.stride, w.stride, words};
        uint8_t *shifts = reinterpret_cast<uint8_t *>(ws + plan.shifts), *row_shift = shifts;
        with_tile<P>(words, x.tokens, 1, steps_of<P>(x.hidden), [&](auto tile, int64_t blocks) {
            using Tile = decltype(tile);
            xent_grad_kernel<P, Tile><<<uint32_t(blocks), Tile::kThreads, 0, stream>>>(
                x, w_piece, h, int32_t(v0), words, lse, control, ws + plan.g, ws + plan.gt, shifts);
            const int32_t across = int32_t(tiles(x.tokens, Tile::kCols));
            if (across == 1) return;   // a word's only shift
            row_shift = reinterpret_cast<uint8_t *>(ws + plan.row_shift);
            xent_align_kernel<G><<<uint32_t(tiles(words, kWaves)), kPackBlock, 0, stream>>>(
                ws + plan.gt, t_row, words, row_values<G>(x.tokens), Tile::kCols, across, shifts, row_shift);
        });
        const Operand gt{ws + plan.gt, t_row, words};
        with_tile<G>(words, x.hidden, 1, steps_of<G>(x.tokens), [&](auto tile, int64_t blocks) {
            using Tile = decltype(tile);
            xent_dw_kernel<P, Tile><<<uint32_t(blocks), Tile::kThreads, 0, stream>>>(x, gt, ht, int32_t(v0), control,
                                                                                     row_shift, dw, ld_dw);
        });
        // a piece starts on a whole step of w^T: it is a multiple of 256 words
        const int64_t g_row = row_bytes<G>(words);
        const Operand g{ws + plan.g, g_row, x.tokens};
        const Operand wt{ws + plan.w_turned + row_bytes<G>(v0), v_row, x.hidden};
        const int32_t steps = int32_t(steps_of<G>(words));
        with_tile<G>(x.tokens, x.hidden, plan.splits, steps / plan.splits, [&](auto tile, int64_t blocks) {
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

hipError_t launch_xent_clear(void *workspace, hipStream_t stream) {
    xent_clear_kernel<<<1, 1, 0, stream>>>(static_cast<Control *>(workspace));
    return hipGetLastError();
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
