// Layer norm and its gradients.
//
//   y  = (x - mean) rstd w + b                     rows of x; mean, rstd of a row
//   g  = dy w ;  h = (x - mean) rstd
//   dx = rstd (g - mean(g) - h mean(g h))
//   dw = sum over the rows of dy h ;  db = sum over the rows of dy
//
// Bytes bound it: x in and y out, x and dy in and dx out.  Measured on one MI355X, 16,384 x
// 4,096 bf16: forward 54 us (5.0 TB/s), backward 76 us (5.3 TB/s, and 25 MB of partial
// sums) and 5 for their join; 700 x 650 fp32: forward 4.9 us, backward 4.2 and 5.1 for
// the columns behind it (each by itself, under a profiler; 7.2 for both as nodes of a
// graph); one row of 1,024: 2.6 us, a launch and two sums over a wave.  A row is read
// once and stays in the registers of one wave, 256 or 1,024 threads, which are left with
// the same columns row after row, so that the weights are read once too and the
// sums of dw and db stay in registers until the workgroup ends.  These partial
// sums go to the workspace and a second launch adds them in order, or, of few rows, sums
// columns of all of them: no atomics, and the same bits each time.
//
// The mean is taken first and the squares of x - mean after it: a row whose mean
// is large against its spread loses nothing by them.  What the rounding of the
// mean itself leaves, the sum of x - mean, is taken off again (it is also what
// makes x - mean right in the backward pass, from the mean as it was stored).
#include "rows.hpp"
#include "launch.hpp"

#include <math.h>

namespace efs {

namespace {

struct Norm {
    const void *x, *weight, *bias, *dy;
    void *out;              // y or dx
    float *mean, *rstd;     // forward: may be NULL
    float *partial;         // backward: [groups][2][width], NULL: no partial sums of dw and db
    float *sums;            // backward of long rows: [rows][4]
    float *rest;            // backward of few rows: [rows], the mean of x - mean; NULL: not kept
    void *dweight, *dbias;  // backward of few rows: written by columns
    int32_t groups;         // backward: workgroups that take rows
    int64_t ld_x, ld_dy, ld_out;
    int32_t rows, width;
    float eps;
    bool past;              // y or dx goes past the caches
};

template <typename T>
constexpr int kRowPack = 16 / sizeof(T);

constexpr int kLong = 1024;   // threads of the longest rows

// The sums of M values over the kThreads threads that hold a row, in each of
// them.  One barrier: the next call takes another buffer, and the one after it
// comes behind that one's barrier.
template <int kThreads, int M>
__device__ __forceinline__ void row_sums(float (&v)[M], float (*buffer)[M]) {
#pragma unroll
    for (int m = 0; m < M; ++m) v[m] = wave_sum(v[m]);
    if (kThreads > kWave) {
        constexpr int kRowWaves = kThreads / kWave;
        const int wave = threadIdx.x / kWave, first = wave / kRowWaves * kRowWaves;
        if ((threadIdx.x & (kWave - 1)) == 0)
#pragma unroll
            for (int m = 0; m < M; ++m) buffer[wave][m] = v[m];
        __syncthreads();
#pragma unroll
        for (int m = 0; m < M; ++m) v[m] = 0.0f;
#pragma unroll
        for (int w = 0; w < kRowWaves; ++w)
#pragma unroll
            for (int m = 0; m < M; ++m) v[m] += buffer[first + w][m];
    }
}

// This thread's columns of a row of weights; `absent` where there are none.
template <typename F, int N, int kPacks, int kThreads>
__device__ __forceinline__ void load_columns(const void *row, int width, float absent, float (&v)[kPacks][N]) {
#pragma unroll
    for (int k = 0; k < kPacks; ++k) {
        const int at = (k * kThreads + threadIdx.x % kThreads) * N;
#pragma unroll
        for (int i = 0; i < N; ++i) v[k][i] = absent;
        if (row != nullptr && at < width) load_pack<N>(static_cast<const F *>(row) + at, width - at, v[k]);
    }
}

// This thread's packs of a row of `width` elements (0: none there).
template <int N, int kPacks, int kThreads, typename T>
__device__ __forceinline__ void load_row(const T *row, int lane, int width, Pack<T, N> (&v)[kPacks]) {
#pragma unroll
    for (int k = 0; k < kPacks; ++k) {
        const int at = (k * kThreads + lane) * N;
#pragma unroll
        for (int i = 0; i < N; ++i) v[k][i] = T(0.0f);
        if (at < width) v[k] = load_raw<N>(row + at, width - at);
    }
}

struct Moments {
    float mean, rstd, rest;   // rest: mean of x - (the mean that was subtracted)
};

// From the sums of x - m and of its squares.
__device__ __forceinline__ Moments moments(float m, float sum, float squares, int width, float eps) {
    const float n = float(width), rest = sum / n;
    const float var = (squares - sum * rest) / n;
    // a constant row's sums can leave less than 0; NaN stays.  Where the spread is
    // larger than the mean, the differences are rounded more coarsely than the sum was
    return Moments{m * m > var ? m + rest : m, 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + eps), rest};
}

template <typename T, typename F, int kThreads, int kPacks>
__global__ __launch_bounds__(kThreads < kBlock ? kBlock : kThreads) void norm_forward_kernel(const Norm a) {
    constexpr int N = kRowPack<T>, kSize = kThreads < kBlock ? kBlock : kThreads, kGroups = kSize / kThreads;
    __shared__ float s_sum[kSize / kWave][1], s_squares[kSize / kWave][2];
    const int lane = threadIdx.x % kThreads, group = threadIdx.x / kThreads;
    float w[kPacks][N], b[kPacks][N];
    load_columns<F, N, kPacks, kThreads>(a.weight, a.width, 1.0f, w);
    load_columns<F, N, kPacks, kThreads>(a.bias, a.width, 0.0f, b);
    const int64_t step = int64_t(gridDim.x) * kGroups;
    const T *const rows = static_cast<const T *>(a.x);
    int64_t row = int64_t(blockIdx.x) * kGroups + group;
    Pack<T, N> next[kPacks];   // a row on its way while the one before it is worked on
    load_row<N, kPacks, kThreads>(rows + row * a.ld_x, lane, row < a.rows ? a.width : 0, next);
    // (a wave's own rows end where it likes; groups of waves are one to a workgroup)
    for (; row < a.rows; row += step) {
        float x[kPacks][N];
        float sum[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < kPacks; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                x[k][i] = float(next[k][i]);
                sum[0] += x[k][i];
            }
        load_row<N, kPacks, kThreads>(rows + (row + step) * a.ld_x, lane, row + step < a.rows ? a.width : 0, next);
        row_sums<kThreads>(sum, s_sum);
        const float m = sum[0] / float(a.width);
        float rest[2] = {0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < kPacks; ++k) {
            const int at = (k * kThreads + lane) * N;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                x[k][i] = at + i < a.width ? x[k][i] - m : 0.0f;
                rest[0] += x[k][i];
                rest[1] = fmaf(x[k][i], x[k][i], rest[1]);
            }
        }
        row_sums<kThreads>(rest, s_squares);
        const Moments s = moments(m, rest[0], rest[1], a.width, a.eps);
        if (lane == 0 && a.mean != nullptr) a.mean[row] = s.mean;
        if (lane == 0 && a.rstd != nullptr) a.rstd[row] = s.rstd;
        T *to = static_cast<T *>(a.out) + row * a.ld_out;
#pragma unroll
        for (int k = 0; k < kPacks; ++k) {
            const int at = (k * kThreads + lane) * N;
            if (at >= a.width) break;
#pragma unroll
            for (int i = 0; i < N; ++i) x[k][i] = fmaf((x[k][i] - s.rest) * s.rstd, w[k][i], b[k][i]);
            store_pack<N>(to + at, a.width - at, x[k], a.past);
        }
    }
}

// Rows too long for registers, one workgroup each, read three times.

template <typename T, typename F>
__global__ __launch_bounds__(kLong) void norm_forward_long_kernel(const Norm a) {
    constexpr int N = kRowPack<T>;
    __shared__ float s_sum[kLong / kWave][1], s_squares[kLong / kWave][2];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *from = static_cast<const T *>(a.x) + row * a.ld_x;
        float sum[1] = {0.0f}, rest[2] = {0.0f, 0.0f};
        for (int at = threadIdx.x * N; at < a.width; at += kLong * N) {
            float x[N];
            load_pack<N>(from + at, a.width - at, x);
#pragma unroll
            for (int i = 0; i < N; ++i) sum[0] += x[i];
        }
        row_sums<kLong>(sum, s_sum);
        const float m = sum[0] / float(a.width);
        for (int at = threadIdx.x * N; at < a.width; at += kLong * N) {
            float x[N];
            load_pack<N>(from + at, a.width - at, x);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float c = at + i < a.width ? x[i] - m : 0.0f;
                rest[0] += c;
                rest[1] = fmaf(c, c, rest[1]);
            }
        }
        row_sums<kLong>(rest, s_squares);
        const Moments s = moments(m, rest[0], rest[1], a.width, a.eps);
        if (threadIdx.x == 0 && a.mean != nullptr) a.mean[row] = s.mean;
        if (threadIdx.x == 0 && a.rstd != nullptr) a.rstd[row] = s.rstd;
        T *to = static_cast<T *>(a.out) + row * a.ld_out;
        for (int at = threadIdx.x * N; at < a.width; at += kLong * N) {
            float x[N], w[N], b[N];
            load_pack<N>(from + at, a.width - at, x);
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = 1.0f, b[i] = 0.0f;
            if (a.weight != nullptr) load_pack<N>(static_cast<const F *>(a.weight) + at, a.width - at, w);
            if (a.bias != nullptr) load_pack<N>(static_cast<const F *>(a.bias) + at, a.width - at, b);
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = fmaf((x[i] - m - s.rest) * s.rstd, w[i], b[i]);
            store_pack<N>(to + at, a.width - at, x, a.past);
        }
    }
}

// What a row's gradient needs of its sums: dx = rstd g - even - slope (x - mean - rest).
struct Slopes {
    float rest, even, slope;
};

// From the sums of x - mean, of g and of g (x - mean).
__device__ __forceinline__ Slopes slopes(const float (&s)[3], float rstd, int width) {
    const float n = float(width), rest = s[0] / n, along = (s[2] - rest * s[1]) * rstd;
    return Slopes{rest, rstd * (s[1] / n), rstd * rstd * (along / n)};
}

template <typename T, typename F, int kThreads, int kPacks, int kSize>
__global__ __launch_bounds__(kSize) void norm_backward_kernel(const Norm a) {
    constexpr int N = kRowPack<T>, kGroups = kSize / kThreads;
    __shared__ float s_sums[2][kSize / kWave][3];
    __shared__ float s_join[kGroups > 1 ? (kGroups - 1) * kThreads * N : 1];
    const int lane = threadIdx.x % kThreads, group = threadIdx.x / kThreads;
    float w[kPacks][N], dw[kPacks][N], db[kPacks][N];
    load_columns<F, N, kPacks, kThreads>(a.weight, a.width, 1.0f, w);
#pragma unroll
    for (int k = 0; k < kPacks; ++k)
#pragma unroll
        for (int i = 0; i < N; ++i) dw[k][i] = db[k][i] = 0.0f;
    int turn = 0;
    const int64_t step = int64_t(a.groups) * kGroups;
    const T *const xs = static_cast<const T *>(a.x), *const dys = static_cast<const T *>(a.dy);
    Pack<T, N> next_x[kPacks], next_dy[kPacks];   // a row on its way while the one before it is worked on
    float next_mean = 0.0f, next_rstd = 0.0f;
    const auto fetch = [&](int64_t row) {
        const bool there = row < a.rows;
        load_row<N, kPacks, kThreads>(xs + row * a.ld_x, lane, there ? a.width : 0, next_x);
        load_row<N, kPacks, kThreads>(dys + row * a.ld_dy, lane, there ? a.width : 0, next_dy);
        next_mean = there ? a.mean[row] : 0.0f, next_rstd = there ? a.rstd[row] : 0.0f;
    };
    // (16 waves' registers do not hold two rows)
    constexpr bool kFetchAhead = kThreads < kLong;
    if (kFetchAhead) fetch(int64_t(blockIdx.x) * kGroups + group);
    for (int64_t first = int64_t(blockIdx.x) * kGroups; first < a.rows; first += step) {
        const int64_t row = first + group;
        const bool there = row < a.rows;   // (all groups meet at the barrier)
        if (!kFetchAhead) fetch(row);
        const float mean = next_mean, rstd = next_rstd;
        float x[kPacks][N], dy[kPacks][N];
#pragma unroll
        for (int k = 0; k < kPacks; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) x[k][i] = float(next_x[k][i]), dy[k][i] = float(next_dy[k][i]);
        if (kFetchAhead) fetch(row + step);
        float s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < kPacks; ++k) {
            const int at = (k * kThreads + lane) * N;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                x[k][i] = at + i < a.width ? x[k][i] - mean : 0.0f;
                db[k][i] += dy[k][i];
                const float g = dy[k][i] * w[k][i];
                s[0] += x[k][i];
                s[1] += g;
                s[2] = fmaf(g, x[k][i], s[2]);
            }
        }
        row_sums<kThreads>(s, s_sums[turn]);
        turn ^= 1;
        const Slopes p = slopes(s, rstd, a.width);
        if (a.rest != nullptr && there && lane == 0) a.rest[row] = p.rest;
        T *to = static_cast<T *>(a.out) + row * a.ld_out;
#pragma unroll
        for (int k = 0; k < kPacks; ++k) {
            const int at = (k * kThreads + lane) * N;
            float dx[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float c = x[k][i] - p.rest;
                dw[k][i] = fmaf(dy[k][i], c * rstd, dw[k][i]);
                dx[i] = fmaf(rstd, dy[k][i] * w[k][i], -p.even) - p.slope * c;
            }
            if (there && at < a.width) store_pack<N>(to + at, a.width - at, dx, a.past);
        }
    }
    if (a.partial == nullptr) return;
    // the groups' sums in order, then this workgroup's to the workspace
    float *to = a.partial + int64_t(blockIdx.x) * 2 * a.width;
#pragma unroll
    for (int k = 0; k < kPacks; ++k) {
        const int at = (k * kThreads + lane) * N;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            float v[N];
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = which == 0 ? dw[k][i] : db[k][i];
            if (kGroups > 1) {
                __syncthreads();
                if (group > 0)
#pragma unroll
                    for (int i = 0; i < N; ++i) s_join[((group - 1) * N + i) * kThreads + lane] = v[i];
                __syncthreads();
                if (group == 0)
                    for (int o = 0; o < kGroups - 1; ++o)
#pragma unroll
                        for (int i = 0; i < N; ++i) v[i] += s_join[(o * N + i) * kThreads + lane];
            }
            if (group == 0 && at < a.width) store_pack<N>(to + which * int64_t(a.width) + at, a.width - at, v);
        }
    }
}

// Long rows: their sums first, a workgroup a row ...
template <typename T, typename F>
__global__ __launch_bounds__(kLong) void norm_sums_kernel(const Norm a) {
    constexpr int N = kRowPack<T>;
    __shared__ float s_sums[2][kLong / kWave][3];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float mean = a.mean[row];
        float s[3] = {0.0f, 0.0f, 0.0f};
        for (int at = threadIdx.x * N; at < a.width; at += kLong * N) {
            float x[N], dy[N], w[N];
            load_pack<N>(static_cast<const T *>(a.x) + row * a.ld_x + at, a.width - at, x);
            load_pack<N>(static_cast<const T *>(a.dy) + row * a.ld_dy + at, a.width - at, dy);
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = 1.0f;
            if (a.weight != nullptr) load_pack<N>(static_cast<const F *>(a.weight) + at, a.width - at, w);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float c = at + i < a.width ? x[i] - mean : 0.0f, g = dy[i] * w[i];
                s[0] += c;
                s[1] += g;
                s[2] = fmaf(g, c, s[2]);
            }
        }
        row_sums<kLong>(s, s_sums[turn]);
        turn ^= 1;
        if (threadIdx.x < 3) a.sums[row * 4 + threadIdx.x] = s[threadIdx.x];
    }
}

// ... then columns of some rows, each thread the same ones.
template <typename T, typename F>
__global__ __launch_bounds__(kBlock) void norm_backward_long_kernel(const Norm a, int32_t rows_each) {
    constexpr int N = kRowPack<T>;
    const int at = (blockIdx.x * kBlock + threadIdx.x) * N;
    if (at >= a.width) return;
    float w[N], dw[N], db[N];
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = 1.0f, dw[i] = db[i] = 0.0f;
    if (a.weight != nullptr) load_pack<N>(static_cast<const F *>(a.weight) + at, a.width - at, w);
    const int64_t lo = int64_t(blockIdx.y) * rows_each, hi = min(lo + rows_each, int64_t(a.rows));
    for (int64_t row = lo; row < hi; ++row) {
        const float mean = a.mean[row], rstd = a.rstd[row];
        const float s[3] = {a.sums[row * 4], a.sums[row * 4 + 1], a.sums[row * 4 + 2]};
        const Slopes p = slopes(s, rstd, a.width);
        float x[N], dy[N], dx[N];
        load_pack<N>(static_cast<const T *>(a.x) + row * a.ld_x + at, a.width - at, x);
        load_pack<N>(static_cast<const T *>(a.dy) + row * a.ld_dy + at, a.width - at, dy);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float c = x[i] - mean - p.rest;
            db[i] += dy[i];
            dw[i] = fmaf(dy[i], c * rstd, dw[i]);
            dx[i] = fmaf(rstd, dy[i] * w[i], -p.even) - p.slope * c;
        }
        store_pack<N>(static_cast<T *>(a.out) + row * a.ld_out + at, a.width - at, dx, a.past);
    }
    if (a.partial == nullptr) return;
    float *to = a.partial + int64_t(blockIdx.y) * 2 * a.width + at;
    store_pack<N>(to, a.width - at, dw);
    store_pack<N>(to + a.width, a.width - at, db);
}

// dw and db: the workgroups' sums in order, each wave a run of them.
constexpr int kJoin = 1024, kJoinWaves = kJoin / kWave;

template <typename F>
__global__ __launch_bounds__(kJoin) void norm_join_kernel(const float *__restrict__ partial, int32_t parts, int32_t width,
                                                          F *dweight, F *dbias) {
    __shared__ float s_sum[kJoinWaves][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t column = int64_t(blockIdx.x) * kWave + lane, columns = 2 * int64_t(width);
    const int each = (parts + kJoinWaves - 1) / kJoinWaves, lo = min(wave * each, parts), hi = min(lo + each, parts);
    float sum = 0.0f;
    if (column < columns) {
#pragma unroll 8
        for (int p = lo; p < hi; ++p) sum += partial[p * columns + column];
    }
    s_sum[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && column < columns) {
#pragma unroll
        for (int w = 1; w < kJoinWaves; ++w) sum += s_sum[w][lane];
        if (column < width) {
            if (dweight != nullptr) dweight[column] = F(sum);
        } else if (dbias != nullptr) {
            dbias[column - width] = F(sum);
        }
    }
}

// Few rows: dw and db of kColumns columns from all rows, which stay in L2, in a launch
// behind that of the rows, which leaves what the rounding of each row's mean left.
// (Columns beside the rows in one launch, 4.2 us of 700 x 650 fp32 where these two take
// 7.2, do not have that: with a mean of 1,000 spreads dw was off by 1.7e-5 of it.  Rows
// beyond 8 spreads summed once more for it, by every workgroup, took 174.)
constexpr int kColumnsBlock = 1024, kRowsAhead = 8;

template <typename T, typename F, int kColumns>
__global__ __launch_bounds__(kColumnsBlock) void norm_columns_kernel(const Norm a) {
    __shared__ float s_part[kColumnsBlock / kWave][2][kColumns];
    constexpr int kSlots = kColumnsBlock / kColumns;   // a thread's rows: its slot's, every kSlots
    const int64_t column = int64_t(blockIdx.x) * kColumns + threadIdx.x % kColumns;
    const int slot = threadIdx.x / kColumns;
    const T *x = static_cast<const T *>(a.x) + column, *dy = static_cast<const T *>(a.dy) + column;
    float dw = 0.0f, db = 0.0f;
    if (column < a.width) {
        for (int first = slot; first < a.rows; first += kSlots * kRowsAhead) {
            float v[kRowsAhead], c[kRowsAhead], mean[kRowsAhead], rest[kRowsAhead], rstd[kRowsAhead];
#pragma unroll
            for (int j = 0; j < kRowsAhead; ++j) {   // on their way at once; behind the last row: the last again
                const int row = min(first + j * kSlots, a.rows - 1);
                v[j] = float(dy[row * a.ld_dy]), c[j] = float(x[row * a.ld_x]);
                mean[j] = a.mean[row], rest[j] = a.rest[row], rstd[j] = a.rstd[row];
            }
#pragma unroll
            for (int j = 0; j < kRowsAhead; ++j) {
                if (first + j * kSlots >= a.rows) break;
                dw = fmaf(v[j], (c[j] - mean[j] - rest[j]) * rstd[j], dw);
                db += v[j];
            }
        }
    }
#pragma unroll
    for (int off = kColumns; off < kWave; off <<= 1) dw += __shfl_xor(dw, off), db += __shfl_xor(db, off);
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    if (lane < kColumns) s_part[wave][0][lane] = dw, s_part[wave][1][lane] = db;
    __syncthreads();
    if (threadIdx.x >= 2 * kColumns || column >= a.width) return;
    const int which = threadIdx.x / kColumns;
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kColumnsBlock / kWave; ++w) sum += s_part[w][which][threadIdx.x % kColumns];
    F *to = static_cast<F *>(which == 0 ? a.dweight : a.dbias);
    if (to != nullptr) to[column] = F(sum);
}

// How a row is held: threads and packs of each.
struct Hold {
    int threads, packs;   // 0: too long for registers
};

// Forward: up to four packs of 8 bf16 or 4 fp32 values a thread, 16,384 values.
Hold forward_hold(int32_t width, int pack) {
    const int packs = (width + pack - 1) / pack;
    if (width > kLong * 16) return Hold{0, 0};
    for (int threads = kWave; threads <= kLong; threads *= 4)
        for (int k = 1; k <= 4; k *= 2)
            if (packs <= threads * k) return Hold{threads, k};
    return Hold{0, 0};
}

// Backward: two packs, beside which a thread holds those of dy, the weights and both sums.
Hold backward_hold(int32_t width, int pack) {
    const int packs = (width + pack - 1) / pack;
    for (int threads = kWave; threads <= kLong; threads *= 4)
        for (int k = 1; k <= 2; k *= 2)
            if (packs <= threads * k) return Hold{threads, k};
    return Hold{0, 0};
}

// Whether dw and db are summed over columns of all rows, which are read a second
// time for that, from L2, instead of by rows with a join.  us of replays of a graph,
// against the join: 700 x 650 fp32 7.2 and 10.3, 1 x 1,024 bf16 5.2 and 6.6, 300 x 4,096
// 8.0 and 13.7, 768 x 2,000 fp32 11.8 and 13.6, 512 x 64 5.9 and 5.0; beyond: 1,024 x 64
// 7.1 and 5.4, 1,024 x 1,024 bf16 9.9 and 8.2, 512 x 4,096 fp32 13.6 and 12.2, 2,048 x
// 1,500 24.3 and 15.5.  kWide: 16 columns a workgroup, not 8 (300 x 4,096 bf16 8.0 and
// 13.2, 512 x 2,000 8.1 and 7.5, 700 x 650 fp32 8.8 and 7.2).
constexpr int kFewRows = 768, kWide = 2048;
constexpr int64_t kFewElements = 3 << 19;

bool few_rows(int32_t rows, int32_t width, Hold h) {
    return h.threads != 0 && rows <= kFewRows && int64_t(rows) * width <= kFewElements;
}

// Workgroups of the backward pass, whose partial sums the workspace holds: no more
// than run at once, three a compute unit (two: 143 us where three take 135 for 16,384 x
// 4,096 with the forward call, four 146: more partial sums, and a second round).
int backward_groups(int32_t rows, Hold h) {
    const int64_t each = h.threads == 0 ? 8 : h.threads < kBlock ? kBlock / h.threads : 1;
    const int64_t groups = (rows + each - 1) / each, most = h.threads == kLong ? 256 : 768;
    return int(groups < most ? groups : most);
}

template <typename T, typename F, int kThreads, int kPacks>
void forward(const Norm &a, hipStream_t stream) {
    constexpr int kSize = kThreads < kBlock ? kBlock : kThreads, kGroups = kSize / kThreads;
    const int64_t groups = (int64_t(a.rows) + kGroups - 1) / kGroups, most = int64_t(device_cu_count()) * (2048 / kSize);
    norm_forward_kernel<T, F, kThreads, kPacks><<<uint32_t(groups < most ? groups : most), kSize, 0, stream>>>(a);
}

template <typename T, typename F, int kThreads, int kPacks>
void backward(const Norm &a, hipStream_t stream) {
    constexpr int kSize = kThreads < kBlock ? kBlock : kThreads;
    norm_backward_kernel<T, F, kThreads, kPacks, kSize><<<uint32_t(a.groups), kSize, 0, stream>>>(a);
}

template <typename T, typename F, int kColumns>
void columns(const Norm &a, hipStream_t stream) {
    norm_columns_kernel<T, F, kColumns><<<uint32_t((a.width + kColumns - 1) / kColumns), kColumnsBlock, 0, stream>>>(a);
}

template <typename T, typename F>
hipError_t run_forward(const Norm &a, hipStream_t stream) {
    const Hold h = forward_hold(a.width, kRowPack<T>);
    switch (h.threads * 8 + h.packs) {
        case 64 * 8 + 1: forward<T, F, 64, 1>(a, stream); break;
        case 64 * 8 + 2: forward<T, F, 64, 2>(a, stream); break;
        case 64 * 8 + 4: forward<T, F, 64, 4>(a, stream); break;
        case 256 * 8 + 2: forward<T, F, 256, 2>(a, stream); break;
        case 256 * 8 + 4: forward<T, F, 256, 4>(a, stream); break;
        case 1024 * 8 + 2: forward<T, F, 1024, 2>(a, stream); break;
        case 1024 * 8 + 4:   // (16,384 bf16 values are two packs)
            if constexpr (sizeof(T) == 4) forward<T, F, 1024, 4>(a, stream);
            break;
        default: {
            const int64_t most = int64_t(device_cu_count()) * 2;
            norm_forward_long_kernel<T, F><<<uint32_t(a.rows < most ? a.rows : most), kLong, 0, stream>>>(a);
        }
    }
    return hipGetLastError();
}

template <typename T, typename F>
hipError_t run_backward(Norm a, void *workspace, hipStream_t stream) {
    const Hold h = backward_hold(a.width, kRowPack<T>);
    a.groups = backward_groups(a.rows, h);
    int parts = a.groups;
    const bool gradients = a.dweight != nullptr || a.dbias != nullptr;
    // (rows that are overwritten in place are not there for the columns)
    if (gradients && a.out != a.x && a.out != a.dy && few_rows(a.rows, a.width, h)) {
        a.rest = static_cast<float *>(workspace);
    } else if (gradients) {
        a.partial = static_cast<float *>(workspace) + (h.threads == 0 ? int64_t(a.rows) * 4 : 0);
    }
    a.sums = static_cast<float *>(workspace);
    if (a.rows > 0) switch (h.threads * 8 + h.packs) {
        case 64 * 8 + 1: backward<T, F, 64, 1>(a, stream); break;
        case 64 * 8 + 2: backward<T, F, 64, 2>(a, stream); break;
        case 256 * 8 + 1: backward<T, F, 256, 1>(a, stream); break;
        case 256 * 8 + 2: backward<T, F, 256, 2>(a, stream); break;
        case 1024 * 8 + 1: backward<T, F, 1024, 1>(a, stream); break;
        case 1024 * 8 + 2: backward<T, F, 1024, 2>(a, stream); break;
        default: {
            const int64_t most = int64_t(device_cu_count()) * 2;
            norm_sums_kernel<T, F><<<uint32_t(a.rows < most ? a.rows : most), kLong, 0, stream>>>(a);
            const int64_t each = (int64_t(a.rows) + a.groups - 1) / a.groups;
            parts = int((a.rows + each - 1) / each);
            const int across = (a.width + kBlock * kRowPack<T> - 1) / (kBlock * kRowPack<T>);
            norm_backward_long_kernel<T, F><<<dim3(across, parts), kBlock, 0, stream>>>(a, int32_t(each));
        }
    }
    if (a.rest != nullptr) {
        if (a.width >= kWide) columns<T, F, 16>(a, stream);
        else columns<T, F, 8>(a, stream);
    }
    if (a.partial != nullptr)
        norm_join_kernel<F><<<uint32_t((2 * int64_t(a.width) + kWave - 1) / kWave), kJoin, 0, stream>>>(
            a.partial, parts, a.width, static_cast<F *>(a.dweight), static_cast<F *>(a.dbias));
    return hipGetLastError();
}

}  // namespace

hipError_t launch_layernorm_forward(const void *x, int64_t ld_x, const void *weight, const void *bias, void *y,
                                    int64_t ld_y, bool bf16, bool weight_bf16, int32_t rows, int32_t width, float eps,
                                    float *mean, float *rstd, hipStream_t stream) {
    Norm a{};
    a.x = x, a.weight = weight, a.bias = bias, a.out = y, a.mean = mean, a.rstd = rstd;
    a.ld_x = ld_x, a.ld_out = ld_y, a.rows = rows, a.width = width, a.eps = eps;
    a.past = int64_t(rows) * width * (bf16 ? 2 : 4) >= kPastCaches;
    if (bf16 && weight_bf16) return run_forward<__bf16, __bf16>(a, stream);
    if (bf16) return run_forward<__bf16, float>(a, stream);
    if (weight_bf16) return run_forward<float, __bf16>(a, stream);
    return run_forward<float, float>(a, stream);
}

// [sums of long rows][partial sums of dw and db], as much as either type of x takes; or
// [rests of few rows]
size_t layernorm_workspace_size(int32_t rows, int32_t width) {
    size_t most = 0;
    for (int pack = kRowPack<float>; pack <= kRowPack<__bf16>; pack *= 2) {
        const Hold h = backward_hold(width, pack);
        const size_t bytes = size_t(backward_groups(rows, h)) * 2 * size_t(width) * sizeof(float) +
                             (h.threads == 0 ? size_t(rows) * 4 * sizeof(float) : 0);
        most = bytes > most ? bytes : most;
    }
    const size_t rests = rows <= kFewRows ? size_t(rows) * sizeof(float) : 0;
    return 16 + (most > rests ? most : rests);
}

hipError_t launch_layernorm_backward(const void *x, int64_t ld_x, const void *weight, const float *mean,
                                     const float *rstd, const void *dy, int64_t ld_dy, void *dx, int64_t ld_dx, bool bf16,
                                     bool weight_bf16, int32_t rows, int32_t width, void *dweight, void *dbias,
                                     void *workspace, hipStream_t stream) {
    Norm a{};
    a.x = x, a.weight = weight, a.dy = dy, a.out = dx;
    a.mean = const_cast<float *>(mean), a.rstd = const_cast<float *>(rstd);
    a.ld_x = ld_x, a.ld_dy = ld_dy, a.ld_out = ld_dx, a.rows = rows, a.width = width;
    a.past = int64_t(rows) * width * (bf16 ? 2 : 4) >= kPastCaches;
    a.dweight = dweight, a.dbias = dbias;
    if (bf16 && weight_bf16) return run_backward<__bf16, __bf16>(a, workspace, stream);
    if (bf16) return run_backward<__bf16, float>(a, workspace, stream);
    if (weight_bf16) return run_backward<float, __bf16>(a, workspace, stream);
    return run_backward<float, float>(a, workspace, stream);
}

}  // namespace efs
