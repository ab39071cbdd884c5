// Words' vectors looked up, and the gradient of their table.
//
//   out[t]    = scale * table[ids[t]]
//   dtable[v] = scale * sum over the tokens t with ids[t] = v, in their order, of dout[t]
//
// Nothing but bytes: the rows that are looked up in, out; dout in, the table's
// gradient out, whole, since words without a token get zeros.
//
// The gradient sorts the tokens by word without a pass that has to wait for
// another: a workgroup owns some consecutive words, looks through all ids twice
// (they stay in L2: 16,384 of them are 128 KiB) and so knows by itself how many
// tokens the words before its own have, and which tokens, in their order, each
// of its own has.  The same workgroup then writes its words' rows: zeros, or
// the sum of a word's few rows.  A word of kHot tokens or more is left to two
// more launches that cut the sorted tokens into pieces of kHot whatever their
// words, sum each piece, and join the pieces of a word in order: no word is
// summed by one wave, and nothing depends on which workgroup comes first.
#include "rows.hpp"
#include "launch.hpp"

#include <math.h>

namespace efs {

namespace {

constexpr int kGradBlock = 512;
constexpr int kGradWaves = kGradBlock / kWave;
constexpr int kMaxWords = 1024;        // of one workgroup
constexpr int kHot = 32;               // tokens; a lane of a half wave each
constexpr int kAhead = 8;              // loads of a lane on their way at once
constexpr int kJoinBlock = 512;
constexpr int kJoinWaves = kJoinBlock / kWave;

// Flags beside a sorted token.
constexpr uint32_t kIsHot = 1u << 31, kIsFirst = 1u << 30, kTokenMask = kIsFirst - 1;

struct Lookup {
    const void *table;
    void *out;
    const int64_t *ids;
    int64_t ld_table, ld_out, ignore;
    int32_t tokens, vocab, width, parts, lanes_log2;
    float scale;
    uint32_t *status;
};

// A row's packs are dealt to 1..64 lanes, kLookAhead to each; longer rows are
// several units.
constexpr int kLookAhead = 4;

template <typename T, typename F>
__global__ __launch_bounds__(kBlock) void embed_forward_kernel(const Lookup a) {
    constexpr int N = kPack<T, F>;
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
    const int64_t units = int64_t(a.tokens) * a.parts, step = (int64_t(gridDim.x) * kBlock) >> a.lanes_log2;
    for (int64_t unit = (int64_t(blockIdx.x) * kBlock + threadIdx.x) >> a.lanes_log2; unit < units; unit += step) {
        const int32_t token = int32_t(unit / a.parts), part = int32_t(unit % a.parts);
        const int64_t id = a.ids[token];
        const bool known = id >= 0 && id < a.vocab, counts = known && id != a.ignore;
        if (!known && id != a.ignore && lane == 0 && part == 0 && a.status != nullptr)
            atomicOr(a.status, kEmbedBadId);
        const F *from = static_cast<const F *>(a.table) + (counts ? id : 0) * a.ld_table;
        T *to = static_cast<T *>(a.out) + int64_t(token) * a.ld_out;
        const int first = (part * kLookAhead * lanes + lane) * N;
        float v[kLookAhead][N];
    #pragma unroll
        for (int k = 0; k < kLookAhead; ++k) {
            const int at = first + k * lanes * N;
    #pragma unroll
            for (int i = 0; i < N; ++i) v[k][i] = 0.0f;
            if (counts && at < a.width) load_pack<N>(from + at, a.width - at, v[k]);
        }
    #pragma unroll
        for (int k = 0; k < kLookAhead; ++k) {
            const int at = first + k * lanes * N;
            if (at >= a.width) break;
            if (counts) {   // (a row that does not count is +0 whatever the scale)
    #pragma unroll
                for (int i = 0; i < N; ++i) v[k][i] = __fmul_rn(v[k][i], a.scale);
            }
            store_pack<N>(to + at, a.width - at, v[k]);
        }
    }
}

struct Sorted {
    uint32_t token;   // with flags
    int32_t word;
};

struct Spread {
    const void *dout;
    void *dtable;
    const int64_t *ids;
    int64_t ld_dout, ld_dtable, ignore;
    int32_t tokens, vocab, width, words;   // words: of one workgroup
    float scale;
    int accumulate;
    uint32_t *status;
    int32_t *count;       // tokens that count, all words together
    Sorted *list;         // [tokens]
    int32_t *lengths;     // [pieces] tokens of the word that starts in a piece
    float *partial;       // [pieces][2][width]
};

// The row of a word from its sum: scaled, added to what is there or written.
template <typename F, int N>
__device__ __forceinline__ void put_row(const Spread &a, int64_t word, int at, float (&sum)[N]) {
    F *to = static_cast<F *>(a.dtable) + word * a.ld_dtable + at;
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = __fmul_rn(sum[i], a.scale);
    if (a.accumulate) {
        float old[N];
        load_pack<N>(to, a.width - at, old);
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] = __fadd_rn(old[i], sum[i]);
    }
    store_pack<N>(to, a.width - at, sum);
}

// Sum of the rows of dout whose numbers are token(0..n-1), at one lane's
// columns, in that order; kAhead loads on their way.
template <typename T, int N, typename Token>
__device__ __forceinline__ void sum_rows(const Spread &a, int at, int n, Token token, float (&sum)[N]) {
    const T *rows = static_cast<const T *>(a.dout) + at;
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = 0.0f;
    for (int j = 0; j < n; j += kAhead) {
        float v[kAhead][N];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (j + k < n) load_pack<N>(rows + int64_t(token(j + k)) * a.ld_dout, a.width - at, v[k]);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (j + k < n) {
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] = __fadd_rn(sum[i], v[k][i]);
            }
    }
}

template <typename T, typename F>
__global__ __launch_bounds__(kGradBlock) void embed_grad_kernel(const Spread a) {
    constexpr int N = kPack<T, F>;
    extern __shared__ uint32_t s_mem[];
    uint32_t *s_at = s_mem;                              // [kGradWaves][words]
    uint32_t *s_start = s_mem + kGradWaves * a.words;    // [words] in the sorted list
    uint32_t *s_total = s_start + a.words;               // [words]
    __shared__ uint32_t s_wave[kGradWaves];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t first = int64_t(blockIdx.x) * a.words;
    const int words = int(min(int64_t(a.words), a.vocab - first));
    for (int i = threadIdx.x; i < kGradWaves * a.words; i += kGradBlock) s_at[i] = 0u;
    __syncthreads();

    // each wave counts its share of the tokens, and all that come before this workgroup's words
    const int share = (a.tokens + kGradBlock - 1) / kGradBlock * kWave;   // whole rounds
    const int lo = min(wave * share, a.tokens), hi = min(lo + share, a.tokens);
    uint32_t before = 0;
    bool bad = false;
    uint32_t *mine = s_at + wave * a.words;
    for (int t = lo; t < hi; t += kAhead * kWave) {
        int64_t id[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) id[k] = t + k * kWave + lane < hi ? a.ids[t + k * kWave + lane] : a.ignore;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (id[k] == a.ignore) continue;
            if (id[k] < 0 || id[k] >= a.vocab) bad = true;
            else if (id[k] < first) ++before;
            else if (id[k] < first + words) atomicAdd(&mine[id[k] - first], 1u);
        }
    }
    if (bad && blockIdx.x == 0 && a.status != nullptr) atomicOr(a.status, kEmbedBadId);
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) before += __shfl_xor(before, off);
    if (lane == 0) s_wave[wave] = before;
    __syncthreads();
    uint32_t base = 0;
#pragma unroll
    for (int w = 0; w < kGradWaves; ++w) base += s_wave[w];

    // where each word's tokens start, and each wave's among them
    for (int r0 = 0; r0 < words; r0 += kGradBlock) {
        const int r = r0 + threadIdx.x;
        uint32_t total = 0;
        if (r < words)
            for (int w = 0; w < kGradWaves; ++w) total += s_at[w * a.words + r];
        uint32_t upto = total;   // inclusive, over the wave and then the workgroup
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const uint32_t left = __shfl_up(upto, off);
            if (lane >= off) upto += left;
        }
        __syncthreads();
        if (lane == kWave - 1) s_wave[wave] = upto;
        __syncthreads();
        uint32_t start = base + upto - total;
        for (int w = 0; w < kGradWaves; ++w) {
            if (w < wave) start += s_wave[w];
            base += s_wave[w];
        }
        if (r < words) {
            s_start[r] = start;
            s_total[r] = total;
            for (int w = 0; w < kGradWaves; ++w) {
                const uint32_t n = s_at[w * a.words + r];
                s_at[w * a.words + r] = start;
                start += n;
            }
        }
    }
    if (first + words >= a.vocab && threadIdx.x == 0) *a.count = int32_t(base);
    __syncthreads();

    // the tokens into their places, in order: a wave takes them as they come, and
    // lanes with the same word count those below them
    for (int t = lo; t < hi; t += kAhead * kWave) {
        int64_t id[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) id[k] = t + k * kWave + lane < hi ? a.ids[t + k * kWave + lane] : a.ignore;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const bool in = id[k] != a.ignore && id[k] >= first && id[k] < first + words;
            const int r = int(id[k] - first);
            uint64_t left = __ballot(in);
            while (left != 0) {
                const int leader = __ffsll((unsigned long long)left) - 1;
                const int word = __shfl(r, leader);
                const uint64_t same = __ballot(in && r == word);
                if (in && r == word) {
                    const uint32_t start = mine[word], at = start + lanes_below(same), n = s_total[word];
                    uint32_t token = uint32_t(t + k * kWave + lane);
                    if (n >= uint32_t(kHot)) {
                        token |= kIsHot;
                        if (at == s_start[word]) {
                            token |= kIsFirst;
                            a.lengths[at / kHot] = int32_t(n);
                        }
                    }
                    a.list[at] = Sorted{token, int32_t(first) + word};
                    if (lane == leader) mine[word] = start + uint32_t(__popcll(same));
                }
                left &= ~same;
            }
        }
    }
    __syncthreads();

    // the rows: a wave takes a word's 64 packs of columns
    const int parts = (a.width + kWave * N - 1) / (kWave * N);
    for (int u = wave; u < words * parts; u += kGradWaves) {
        const int r = u / parts, at = (u % parts * kWave + lane) * N;
        const int n = int(s_total[r]);
        if (n >= kHot || (n == 0 && a.accumulate)) continue;
        if (at >= a.width) continue;
        float sum[N];
        const Sorted *list = a.list + s_start[r];
        if (n == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] = 0.0f;
            store_pack<N>(static_cast<F *>(a.dtable) + (first + r) * a.ld_dtable + at, a.width - at, sum);
        } else {
            sum_rows<T, N>(a, at, n, [&](int j) { return list[j].token; }, sum);
            put_row<F, N>(a, first + r, at, sum);
        }
    }
}

// Sums of one piece of kHot sorted tokens, of those whose word has kHot tokens
// or more: at most two such words meet a piece, one that is there at its first
// token (slot 0) and one that starts behind it (slot 1).
template <typename T, typename F>
__global__ __launch_bounds__(kBlock) void embed_pieces_kernel(const Spread a) {
    constexpr int N = kPack<T, F>;
    const int lane = threadIdx.x & (kWave - 1);
    const int parts = (a.width + kWave * N - 1) / (kWave * N);
    const int64_t units = ((*a.count + int64_t(kHot) - 1) / kHot) * parts;
    for (int64_t unit = int64_t(blockIdx.x) * kWaves + threadIdx.x / kWave; unit < units;
         unit += int64_t(gridDim.x) * kWaves) {
        const int64_t piece = unit / parts, begin = piece * kHot;
        const int at = (int(unit % parts) * kWave + lane) * N;
        const int n = int(min(int64_t(kHot), *a.count - begin));
        Sorted s{0u, -1};
        if (lane < n) s = a.list[begin + lane];
        const uint64_t hot = __ballot((s.token & kIsHot) != 0u);
        if (hot == 0) continue;
        const uint32_t token = s.token & kTokenMask;
        const uint64_t head = hot & 1u ? __ballot(s.word == __shfl(s.word, 0) && lane < n) : 0;
    #pragma unroll
        for (int slot = 0; slot < 2; ++slot) {
            const uint64_t lanes = slot == 0 ? head : hot & ~head;
            if (lanes == 0) continue;
            const int from = __ffsll((unsigned long long)lanes) - 1, many = int(__popcll(lanes));
            float sum[N];
            sum_rows<T, N>(a, min(at, a.width - 1), many, [&](int j) { return __builtin_amdgcn_readlane(token, from + j); }, sum);
            if (at < a.width) {
                float *to = a.partial + (piece * 2 + slot) * int64_t(a.width) + at;
                store_pack<N>(to, a.width - at, sum);
            }
        }
    }
}

// The pieces of a word, in order, from the piece in which it starts: each wave
// sums a run of them, and the first joins the waves' sums.
template <typename T, typename F>
__global__ __launch_bounds__(kJoinBlock) void embed_join_kernel(const Spread a) {
    constexpr int N = kPack<T, F>;
    __shared__ float s_sum[kJoinWaves][kWave * N];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t piece = blockIdx.x, begin = piece * kHot;
    const int n = int(min(int64_t(kHot), *a.count - begin));
    if (n <= 0) return;
    Sorted s{0u, -1};
    if (lane < n) s = a.list[begin + lane];
    const uint64_t starts = __ballot((s.token & kIsFirst) != 0u);
    if (starts == 0) return;   // the same for every wave
    const int from = __ffsll((unsigned long long)starts) - 1;
    const int word = __shfl(s.word, from);
    const int64_t pieces = (begin + from + a.lengths[piece] - 1) / kHot - piece + 1;
    const int64_t each = (pieces + kJoinWaves - 1) / kJoinWaves;
    const int64_t lo = min(wave * each, pieces), hi = min(lo + each, pieces);
    const int parts = (a.width + kWave * N - 1) / (kWave * N);
    for (int part = blockIdx.y; part < parts; part += gridDim.y) {
        const int at = (part * kWave + lane) * N;
        float sum[N];
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] = 0.0f;
        if (at < a.width)
            for (int64_t j = lo; j < hi; j += kAhead) {
                float v[kAhead][N];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    const int64_t slot = (piece + j + k) * 2 + (j + k == 0 && from != 0);
                    if (j + k < hi) load_pack<N>(a.partial + slot * a.width + at, a.width - at, v[k]);
                }
#pragma unroll
                for (int k = 0; k < kAhead; ++k)
                    if (j + k < hi) {
#pragma unroll
                        for (int i = 0; i < N; ++i) sum[i] = __fadd_rn(sum[i], v[k][i]);
                    }
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) s_sum[wave][i * kWave + lane] = sum[i];
        __syncthreads();
        if (wave == 0 && at < a.width) {
            for (int w = 1; w < kJoinWaves; ++w)
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] = __fadd_rn(sum[i], s_sum[w][i * kWave + lane]);
            put_row<F, N>(a, word, at, sum);
        }
    }
}

int64_t pieces_of(int32_t tokens) { return tokens < kHot ? 0 : (int64_t(tokens) + kHot - 1) / kHot; }

// A grid's threads are counted in 32 bits; the kernels step on where it ends.
uint32_t grid_of(int64_t groups) { return uint32_t(groups < (1 << 20) ? groups : 1 << 20); }

size_t up16(size_t bytes) { return (bytes + 15) & ~size_t(15); }

// Words of one workgroup: enough of them that looking through the ids (16 bytes
// a token at the rate of L2) stays below a tenth of writing their rows, and few
// enough that there are some workgroups for every compute unit.
int words_per_workgroup(int32_t tokens, int32_t vocab, int64_t row_bytes) {
    const int64_t scan = 24 * int64_t(tokens) / row_bytes;
    int64_t words = vocab / (8 * int64_t(device_cu_count()));
    if (words < scan) words = scan;
    return int(words < 1 ? 1 : words > kMaxWords ? kMaxWords : words);
}

template <typename T, typename F>
hipError_t spread(Spread a, hipStream_t stream) {
    constexpr int N = kPack<T, F>;
    a.words = words_per_workgroup(a.tokens, a.vocab, int64_t(a.width) * int(sizeof(F)));
    const uint32_t groups = uint32_t((a.vocab + a.words - 1) / a.words);
    const size_t lds = size_t(a.words) * (kGradWaves + 2) * sizeof(uint32_t);
    embed_grad_kernel<T, F><<<groups, kGradBlock, lds, stream>>>(a);
    const int64_t pieces = pieces_of(a.tokens);
    if (pieces > 0) {
        const int64_t parts = (a.width + kWave * N - 1) / (kWave * N);
        embed_pieces_kernel<T, F><<<grid_of((pieces * parts + kWaves - 1) / kWaves), kBlock, 0, stream>>>(a);
        embed_join_kernel<T, F><<<dim3(uint32_t(pieces), uint32_t(parts < 64 ? parts : 64)), kJoinBlock, 0, stream>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embed_forward(const void *table, int64_t ld_table, bool table_bf16, const int64_t *ids, void *out,
                                int64_t ld_out, bool bf16, int32_t tokens, int32_t vocab, int32_t width, float scale,
                                int64_t ignore, uint32_t *status, hipStream_t stream) {
    Lookup a{table, out, ids, ld_table, ld_out, ignore, tokens, vocab, width, 0, 0, scale, status};
    const int pack = bf16 && table_bf16 ? 8 : 4, packs = (width + pack - 1) / pack;
    while ((1 << a.lanes_log2) < kWave && (1 << a.lanes_log2) < packs) ++a.lanes_log2;
    const int each = kLookAhead << a.lanes_log2;
    a.parts = (packs + each - 1) / each;
    const int64_t threads = (int64_t(tokens) * a.parts) << a.lanes_log2;
    const uint32_t groups = grid_of((threads + kBlock - 1) / kBlock);
    if (bf16 && table_bf16) embed_forward_kernel<__bf16, __bf16><<<groups, kBlock, 0, stream>>>(a);
    else if (bf16) embed_forward_kernel<__bf16, float><<<groups, kBlock, 0, stream>>>(a);
    else if (table_bf16) embed_forward_kernel<float, __bf16><<<groups, kBlock, 0, stream>>>(a);
    else embed_forward_kernel<float, float><<<groups, kBlock, 0, stream>>>(a);
    return hipGetLastError();
}

// [16 bytes: tokens that count][list][lengths][partial sums]
size_t embed_workspace_size(int32_t tokens, int32_t width) {
    const size_t pieces = size_t(pieces_of(tokens));
    return 16 + up16(size_t(tokens) * sizeof(Sorted)) + up16(pieces * sizeof(int32_t)) +
           up16(pieces * 2 * size_t(width) * sizeof(float));
}

hipError_t launch_embed_backward(const void *dout, int64_t ld_dout, bool bf16, const int64_t *ids, void *dtable,
                                 int64_t ld_dtable, bool table_bf16, int32_t tokens, int32_t vocab, int32_t width,
                                 float scale, int64_t ignore, bool accumulate, uint32_t *status, void *workspace,
                                 hipStream_t stream) {
    char *ws = static_cast<char *>(workspace);
    Spread a{};
    a.dout = dout, a.dtable = dtable, a.ids = ids;
    a.ld_dout = ld_dout, a.ld_dtable = ld_dtable, a.ignore = ignore;
    a.tokens = tokens, a.vocab = vocab, a.width = width;
    a.scale = scale, a.accumulate = accumulate, a.status = status;
    a.count = reinterpret_cast<int32_t *>(ws);
    ws += 16;
    a.list = reinterpret_cast<Sorted *>(ws);
    ws += up16(size_t(tokens) * sizeof(Sorted));
    a.lengths = reinterpret_cast<int32_t *>(ws);
    ws += up16(size_t(pieces_of(tokens)) * sizeof(int32_t));
    a.partial = reinterpret_cast<float *>(ws);
    if (bf16 && table_bf16) return spread<__bf16, __bf16>(a, stream);
    if (bf16) return spread<__bf16, float>(a, stream);
    if (table_bf16) return spread<float, __bf16>(a, stream);
    return spread<float, float>(a, stream);
}

}  // namespace efs
