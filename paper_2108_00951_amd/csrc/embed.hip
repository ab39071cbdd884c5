// Words' vectors looked up, and the gradient of their table.
//
//   out[t]    = scale * table[ids[t]]
//   dtable[v] = scale * sum over the tokens t with ids[t] = v, in their order, of dout[t]
//
// Bytes bound both: the rows that are looked up in and out; dout in, the table's
// gradient out, whole, since words without a token get zeros.  Measured on one MI355X
// (a copy reaches 6.0 to 6.3 TB/s, zeros alone 6.9):
//   32,768 rows of 4,096 bf16 looked up              77 us, 4.7 TB/s (5.6 with the rows
//                                                    that several XCDs fetch)
//   gradient, 131,072 x 2,048 fp32, 16,384 tokens    167 us, 6.8 TB/s
//   gradient, 33,278 x 650 fp32, 700 tokens          18 us, 4.9 TB/s
//   gradient, 64 tokens added to 33,278 x 1,024      4.2 us
//
// The gradient of few tokens is one launch: a workgroup for each token and 64 packs
// of columns looks through all ids, ends if an earlier token has the same, and else
// sums the rows of its word's tokens; others write the zeros of words without a
// token.  Up to 1,024 tokens, or 4,096 where the rows are short: 1,520 x 23,472 x 499
// takes 17 us so and 33 by the other way, 2,241 x 48,840 x 4,095 90 and 29.
//
// More tokens are sorted by word, without a pass that has to wait for another: a
// workgroup owns some consecutive words and looks through all ids (they stay in L2:
// 16,384 of them are 128 KiB), so that it knows by itself how many tokens the words
// before its own have, and which tokens, in their order, each of its own has (13 us
// for 16,384 tokens, 35 for 65,536, 117 for 262,144, which are 7, 13 and 20 % of the call
// at 131,072 x 2,048; the workgroup of the hottest words is the last: 57 us for 16,384
// tokens of which half are its own).  A second
// launch takes the sorted tokens in pieces of kHot, writes the rows of words with
// fewer than kHot tokens and sums those of other words piece by piece; a third joins
// the pieces of a word in order.  So no word is summed by one wave, and nothing depends
// on which workgroup comes first.
#include "rows.hpp"
#include "launch.hpp"

#include <type_traits>

namespace efs {

namespace {

constexpr int kFew = 4096;             // tokens that need no sorting, with short rows
constexpr int kFewAny = 1024;          // with rows of any length
constexpr int kFewRounds = kFew / kBlock;
constexpr int kFewAlone = 16;          // rows that one wave sums
constexpr int kSortBlock = 1024;
constexpr int kSortWaves = kSortBlock / kWave;
constexpr int kSortAhead = 16;         // rounds of ids that a wave keeps
constexpr int kMaxWords = 960;         // of one sorting workgroup: 60 KiB of LDS
constexpr int kHot = 32;               // tokens; a lane of a half wave each
constexpr int kAhead = 8;              // loads of a lane on their way at once
constexpr int kJoinBlock = 512;
constexpr int kJoinWaves = kJoinBlock / kWave;
constexpr int64_t kFewBytes = 32768;   // of the table's rows that a workgroup of few tokens writes
constexpr int kMaxRows = 1024;         // of one such workgroup
constexpr int64_t kTileBytes = kSortBlock * 16, kRowTile = kBlock * 16;   // cleared by one, 16 bytes a thread

struct Lookup {
    const void *table;
    void *out;
    const int64_t *ids;
    int64_t ld_table, ld_out, ignore;
    int32_t tokens, vocab, width, parts, lanes_log2;
    float scale;
    bool past;            // the results go past the caches
    uint32_t *status;
};

// A row's packs are dealt to 1..64 lanes, kLookAhead to each; longer rows are
// several units.  (1, 2, 4 and 8 of them: 84, 77, 80 and 98 us for 32,768 x 4,096 bf16.)
constexpr int kLookAhead = 2;

template <typename T, typename F>
__global__ __launch_bounds__(kBlock) void embed_forward_kernel(const Lookup a) {
    constexpr int N = kPack<T, F>;
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
    const uint32_t units = uint32_t(a.tokens) * uint32_t(a.parts), step = (gridDim.x * kBlock) >> a.lanes_log2;
    for (uint32_t unit = (blockIdx.x * kBlock + threadIdx.x) >> a.lanes_log2; unit < units; unit += step) {
        const int32_t token = int32_t(unit / uint32_t(a.parts)), part = int32_t(unit % uint32_t(a.parts));
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
            store_pack<N>(to + at, a.width - at, v[k], a.past);
        }
    }
}

struct Sorted {
    int32_t token, word;
};

struct Spread {
    const void *dout;
    void *dtable;
    const int64_t *ids;
    int64_t ld_dout, ld_dtable, ignore;
    int32_t tokens, vocab, width;
    int32_t words, rows;  // of one workgroup that sorts, that writes rows
    int32_t sums, clears;   // workgroups that sum rows, that clear rows
    int32_t sorts;        // workgroups that sort, before those that clear
    int64_t tiles;        // that these clear
    uint64_t share;       // of the workgroups that sum, times 2^32
    float scale;
    bool accumulate, past;
    uint32_t *status;
    int32_t *start;       // [vocab + 1] in the sorted list
    Sorted *list;         // [tokens]
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
    store_pack<N>(to, a.width - at, sum, a.past);
}

// Sum of the rows row(0..n-1) at one lane's columns (at < width), in that order.
template <int N, int kLoads, typename Row>
__device__ __forceinline__ void sum_rows(int left, int n, Row row, float (&sum)[N]) {
    typedef typename std::remove_cv<typename std::remove_pointer<decltype(row(0))>::type>::type T;
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = 0.0f;
    for (int j = 0; j < n; j += kLoads) {
        Pack<T, N> v[kLoads];
#pragma unroll
        for (int k = 0; k < kLoads; ++k)
            if (j + k < n) v[k] = load_raw<N>(row(j + k), left);
#pragma unroll
        for (int k = 0; k < kLoads; ++k)
            if (j + k < n) {
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] = __fadd_rn(sum[i], float(v[k][i]));
            }
    }
}

// Zeros into the rows of [first, first + rows) that empty(r) says.
template <typename F, typename Empty>
__device__ __forceinline__ void clear_rows(const Spread &a, int64_t first, int rows, Empty empty) {
    constexpr int N = 16 / sizeof(F);
    const uint32_t packs = uint32_t(a.width + N - 1) / N;
    const float zero[N] = {};
    for (uint32_t u = threadIdx.x; u < uint32_t(rows) * packs; u += blockDim.x) {
        const uint32_t r = u / packs;
        const int at = int(u - r * packs) * N;
        if (empty(int(r))) store_pack<N>(static_cast<F *>(a.dtable) + (first + r) * a.ld_dtable + at, a.width - at, zero, a.past);
    }
}

__device__ __forceinline__ bool counts(const Spread &a, int64_t id) { return id != a.ignore && id >= 0 && id < a.vocab; }

// The workgroups that sum (which >= 0: the how manieth) among those that clear
// (which < 0: -1 - the how manieth), evenly spread: the ones wait for what they
// read, the others fill the memory's time.
__device__ __forceinline__ int dealt(const Spread &a) {
    const uint64_t b = blockIdx.x;
    const int before = int((b * a.share) >> 32), upto = int(((b + 1) * a.share) >> 32);
    return upto > before ? before : -1 - (int(b) - before);
}

// Up to kFew tokens: a token's word, a workgroup for 64 packs of columns; or rows of
// words without a token.
template <typename T, typename F>
__global__ __launch_bounds__(kBlock) void embed_few_kernel(const Spread a) {
    constexpr int N = kPack<T, F>;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int group = dealt(a);
    if (group < 0) {
        __shared__ uint8_t s_there[kMaxRows];
        const int64_t first = int64_t(-1 - group) * a.rows;
        const int rows = int(min(int64_t(a.rows), a.vocab - first));
        for (int r = threadIdx.x; r < rows; r += kBlock) s_there[r] = 0;
        __syncthreads();
        for (int t = threadIdx.x; t < a.tokens; t += kBlock) {
            const int64_t id = a.ids[t];
            if (id != a.ignore && id >= first && id < first + rows) s_there[id - first] = 1;
        }
        __syncthreads();
        clear_rows<F>(a, first, rows, [&](int r) { return s_there[r] == 0; });
        return;
    }

    __shared__ int32_t s_count[kFewRounds * kWaves];
    __shared__ int32_t s_token[kFew];
    __shared__ float s_sum[kWaves][kWave * N];
    const int parts = (a.width + kWave * N - 1) / (kWave * N), token = group / parts, part = group % parts;
    const int64_t word = a.ids[token];
    if (!counts(a, word)) {
        if (word != a.ignore && part == 0 && threadIdx.x == 0 && a.status != nullptr) atomicOr(a.status, kEmbedBadId);
        return;
    }
    // the tokens of the same word, a bit each; an earlier one's workgroup sums them
    const int rounds = (a.tokens + kBlock - 1) / kBlock;
    uint64_t mine[kFewRounds];
    bool earlier = false;
#pragma unroll
    for (int k = 0; k < kFewRounds; ++k) {
        mine[k] = 0;
        if (k >= rounds) continue;
        const int t = k * kBlock + int(threadIdx.x);
        const bool same = t < a.tokens && a.ids[t] == word;
        earlier = earlier || (same && t < token);
        mine[k] = __ballot(same);
        if (lane == 0) s_count[k * kWaves + wave] = int(__popcll(mine[k]));
    }
    if (__syncthreads_or(earlier)) return;
    int n = 0;
    for (int k = 0; k < rounds; ++k)   // in the order of the tokens: round by round, wave by wave
#pragma unroll
        for (int w = 0; w < kWaves; ++w) n += s_count[k * kWaves + w];
    int before = 0, next = 0;
#pragma unroll
    for (int k = 0; k < kFewRounds; ++k) {
        if (k >= rounds) continue;
        before = next;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const int c = s_count[k * kWaves + w];
            before += w < wave ? c : 0;
            next += c;
        }
        if ((mine[k] >> lane) & 1u) s_token[before + int(lanes_below(mine[k]))] = k * kBlock + int(threadIdx.x);
    }
    __syncthreads();
    const T *dout = static_cast<const T *>(a.dout);
    if (n <= kFewAlone) {   // a wave's columns each, in one of four workgroups
        const int at = ((part + wave) * kWave + lane) * N;
        if (part % kWaves != 0 || at >= a.width) return;
        float sum[N];
        sum_rows<N, kAhead>(a.width - at, n, [&](int j) { return dout + int64_t(s_token[j]) * a.ld_dout + at; }, sum);
        put_row<F, N>(a, word, at, sum);
        return;
    }
    // a wave's tokens each
    const int each = (n + kWaves - 1) / kWaves, lo = min(wave * each, n), hi = min(lo + each, n);
    const int at = (part * kWave + lane) * N;
    float sum[N] = {};
    if (at < a.width)
        sum_rows<N, 2 * kAhead>(a.width - at, hi - lo,
                                [&](int j) { return dout + int64_t(s_token[lo + j]) * a.ld_dout + at; }, sum);
#pragma unroll
    for (int i = 0; i < N; ++i) s_sum[wave][i * kWave + lane] = sum[i];
    __syncthreads();
    if (wave == 0 && at < a.width) {
        for (int w = 1; w < kWaves; ++w)
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] = __fadd_rn(sum[i], s_sum[w][i * kWave + lane]);
        put_row<F, N>(a, word, at, sum);
    }
}

// Zeros into a tile of the table, words with tokens or not: the rows of those, no more
// than there are tokens, are written again.
template <typename F>
__device__ __forceinline__ void clear_table(const Spread &a, int64_t tile) {
    constexpr int N = 16 / sizeof(F);
    const float zero[N] = {};
    if (a.ld_dtable == a.width) {   // without gaps: whole lines, whatever the rows
        F *const table = static_cast<F *>(a.dtable);
        const int64_t ahead = int64_t(reinterpret_cast<uintptr_t>(table) % 128 / sizeof(F)), all = int64_t(a.vocab) * a.width;
        const int64_t e = (tile * kSortBlock + threadIdx.x) * N - ahead;
        if (e >= 0 && e + N <= all) return store_pack<N>(table + e, N, zero, a.past);
        for (int i = 0; i < N; ++i)
            if (e + i >= 0 && e + i < all) table[e + i] = F(0.0f);
        return;
    }
    const int64_t first = tile * a.rows;
    clear_rows<F>(a, first, int(min(int64_t(a.rows), a.vocab - first)), [](int) { return true; });
}

// The tokens by word: the list, and where each word's start in it.  Workgroups behind
// a.sorts clear the table meanwhile.
template <typename F>
__global__ __launch_bounds__(kSortBlock) void embed_sort_kernel(const Spread a) {
    if (int(blockIdx.x) >= a.sorts) {
        for (int64_t tile = int64_t(blockIdx.x) - a.sorts; tile < a.tiles; tile += a.clears) clear_table<F>(a, tile);
        return;
    }
    extern __shared__ uint32_t s_mem[];
    uint32_t *s_at = s_mem;                              // [kSortWaves][words]
    __shared__ uint32_t s_wave[kSortWaves];
    static_assert(kMaxWords <= kSortBlock, "a thread a word");
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t first = int64_t(blockIdx.x) * a.words;
    const int words = int(min(int64_t(a.words), a.vocab - first));
    for (int i = threadIdx.x; i < kSortWaves * a.words; i += kSortBlock) s_at[i] = 0u;
    __syncthreads();

    // each wave counts its share of the tokens, and all that come before this workgroup's words
    const int share = (a.tokens + kSortBlock - 1) / kSortBlock * kWave;   // whole rounds
    const int lo = min(wave * share, a.tokens), hi = min(lo + share, a.tokens);
    int32_t id[kSortAhead];      // -1: does not count
    uint64_t in[kSortAhead];     // the lanes whose token is one of this workgroup's words
    const uint32_t from = uint32_t(first), vocab = uint32_t(a.vocab);
    const auto fetch = [&](int t) {
        int64_t wide[kSortAhead];
#pragma unroll
        for (int k = 0; k < kSortAhead; ++k)
            wide[k] = t + k * kWave + lane < hi ? a.ids[t + k * kWave + lane] : a.ignore;
#pragma unroll
        for (int k = 0; k < kSortAhead; ++k) {
            const bool word = uint32_t(wide[k] >> 32) == 0u && uint32_t(wide[k]) < vocab;
            id[k] = word && wide[k] != a.ignore ? int32_t(wide[k]) : -1;
            in[k] = __ballot(uint32_t(id[k]) - from < uint32_t(words));
            if (blockIdx.x == 0 && !word && wide[k] != a.ignore && a.status != nullptr) atomicOr(a.status, kEmbedBadId);
        }
    };
    uint32_t before = 0;   // of the wave
    uint32_t *mine = s_at + wave * a.words;
    for (int t = lo; t < hi; t += kSortAhead * kWave) {
        fetch(t);
#pragma unroll
        for (int k = 0; k < kSortAhead; ++k) {
            before += uint32_t(__popcll(__ballot(uint32_t(id[k]) < from)));
            if (in[k] != 0 && uint32_t(id[k]) - from < uint32_t(words)) atomicAdd(&mine[uint32_t(id[k]) - from], 1u);
        }
    }
    if (lane == 0) s_wave[wave] = before;
    __syncthreads();
    uint32_t base = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) base += s_wave[w];

    // where each word's tokens start, and each wave's among them (a thread a word)
    const int r = threadIdx.x;
    uint32_t total = 0;
    if (r < words)
        for (int w = 0; w < kSortWaves; ++w) total += s_at[w * a.words + r];
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
    for (int w = 0; w < wave; ++w) start += s_wave[w];
    if (r < words) {
        a.start[first + r] = int32_t(start);
        if (first + r == a.vocab - 1) a.start[a.vocab] = int32_t(start + total);
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t n = s_at[w * a.words + r];
            s_at[w * a.words + r] = start;
            start += n;
        }
    }
    __syncthreads();

    // the tokens into their places, in order: a wave takes them as they come, and
    // lanes with the same word count those below them
    for (int t = lo; t < hi; t += kSortAhead * kWave) {
        if (hi - lo > kSortAhead * kWave) fetch(t);   // (else they are there)
#pragma unroll
        for (int k = 0; k < kSortAhead; ++k) {
            const int own = id[k] - int(first);
            uint64_t left = in[k], same = 0;
            if (left == 0) continue;
            while (left != 0) {   // a word at a time: the lanes that have it
                const int word = __builtin_amdgcn_readlane(own, __ffsll((unsigned long long)left) - 1);
                const uint64_t its = __ballot(own == word);
                same = own == word ? its : same;
                left &= ~its;
            }
            // the lanes of a word read its place before one of them moves it on
            const bool its = (in[k] >> lane) & 1u;
            const uint32_t at = its ? mine[own] : 0u, below = lanes_below(same);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (its) {
                a.list[at + below] = Sorted{t + k * kWave + lane, int32_t(first) + own};
                if (below == 0u) mine[own] = at + uint32_t(__popcll(same));
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }
}

// How many tokens a word has.
__device__ __forceinline__ int tokens_of(const Spread &a, int word) { return a.start[word + 1] - a.start[word]; }

// One piece of kHot sorted tokens at a lane's columns.  share < kShares: words with
// fewer than kHot that start in that share of the piece are summed, all of their
// tokens, and their rows written (a whole piece for a wave, its loads waited for the
// rows that it had stored: 229 us where this takes 167).  kShares: of words with
// more, the sums of those tokens that lie in the piece; at most two such words meet
// it, one that is there at its first token (slot 0) and one that starts behind it
// (slot 1).
constexpr int kShares = 4;

template <typename T, typename F>
__device__ __forceinline__ void sum_piece(const Spread &a, int32_t piece, int share, int at) {
    constexpr int N = kPack<T, F>;
    static_assert(2 * kHot == kWave, "a piece, and what words that start in it have in the next");
    const int lane = threadIdx.x & (kWave - 1);
    const int64_t place = int64_t(piece) * kHot + lane;
    const bool there = place < a.start[a.vocab];
    Sorted s{0, -1};
    int from = -1, n = 0;   // of the word: its first place, its tokens
    if (there) {
        s = a.list[place];
        from = a.start[s.word];
        n = a.start[s.word + 1] - from;
    }
    const uint64_t in_piece = (uint64_t(1) << kHot) - 1;
    const uint64_t hot = __ballot(n >= kHot) & in_piece;
    const uint64_t firsts = __ballot(there && from == place && n < kHot) & in_piece;
    const uint64_t lasts = __ballot(there && from + n - 1 == place);
    // tokens of words that start in the share and are not hot
    const int64_t lo = place - lane + share * (kHot / kShares), hi = lo + kHot / kShares;
    uint64_t todo = share < kShares ? __ballot(there && n < kHot && from >= lo && from < hi) : 0;
    const T *rows = static_cast<const T *>(a.dout) + min(at, a.width - 1);
    const int left = max(a.width - at, 1);
    const auto row = [&](int j) { return rows + int64_t(__builtin_amdgcn_readlane(s.token, j)) * a.ld_dout; };
    float sum[N] = {};
    while (todo != 0) {
        constexpr int kLoads = 2 * kAhead;
        Pack<T, N> v[kLoads];
        uint64_t now = todo;
#pragma unroll
        for (int k = 0; k < kLoads; ++k)
            if (todo != 0) {
                v[k] = load_raw<N>(row(__ffsll((unsigned long long)todo) - 1), left);
                todo &= todo - 1;
            }
#pragma unroll
        for (int k = 0; k < kLoads; ++k)
            if (now != 0) {
                const int j = __ffsll((unsigned long long)now) - 1;
                now &= now - 1;
                if ((firsts >> j) & 1u)
#pragma unroll
                    for (int i = 0; i < N; ++i) sum[i] = 0.0f;
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] = __fadd_rn(sum[i], float(v[k][i]));
                if ((lasts >> j) & 1u && at < a.width) put_row<F, N>(a, __builtin_amdgcn_readlane(s.word, j), at, sum);
            }
    }
    if (share < kShares || hot == 0) return;
    const uint64_t head = hot & 1u ? __ballot(s.word == __builtin_amdgcn_readlane(s.word, 0) && there) & in_piece : 0;
#pragma unroll
    for (int slot = 0; slot < 2; ++slot) {
        const uint64_t lanes = slot == 0 ? head : hot & ~head;
        if (lanes == 0) continue;
        const int first = __ffsll((unsigned long long)lanes) - 1;
        sum_rows<N, 2 * kAhead>(left, int(__popcll(lanes)), [&](int j) { return row(first + j); }, sum);
        if (at < a.width)
            store_pack<N>(a.partial + (int64_t(piece) * 2 + slot) * a.width + at, a.width - at, sum);
    }
}

// A piece's columns a wave.  kClear: and among these workgroups, those that clear rows
// without a token, whose bytes are whole tiles.
template <typename T, typename F, bool kClear>
__global__ __launch_bounds__(kBlock) void embed_rows_kernel(const Spread a) {
    constexpr int N = kPack<T, F>;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int parts = (a.width + kWave * N - 1) / (kWave * N);
    const int group = kClear ? dealt(a) : int(blockIdx.x);
    if (kClear && group < 0) {
        constexpr int kZeros = 16 / sizeof(F), kElements = kRowTile / sizeof(F);
        const uint32_t across = uint32_t(a.width) / kElements;
        const float zero[kZeros] = {};
        for (uint32_t tile = uint32_t(-1 - group); tile < uint32_t(a.tiles); tile += uint32_t(a.clears)) {
            const int32_t word = int32_t(tile / across);
            F *to = static_cast<F *>(a.dtable) + word * a.ld_dtable + int64_t(tile % across) * kElements;
            if (tokens_of(a, word) == 0) store_pack<kZeros>(to + threadIdx.x * kZeros, kZeros, zero, true);
        }
        return;
    }
    const uint32_t each = uint32_t(parts) * (kShares + 1), units = (uint32_t(a.start[a.vocab]) + kHot - 1) / kHot * each;
    for (uint32_t u = uint32_t(group * kWaves + wave); u < units; u += uint32_t(a.sums) * kWaves) {
        const uint32_t piece = u / each, rest = u - piece * each, share = rest / uint32_t(parts);
        sum_piece<T, F>(a, int32_t(piece), int(share), (int(rest - share * uint32_t(parts)) * kWave + lane) * N);
    }
}

// The pieces of a word, in order, from the piece in which it starts: each wave
// sums a run of them, and the first joins the waves' sums.  A workgroup looks for
// words in as many pieces as it has waves.
template <typename T, typename F>
__global__ __launch_bounds__(kJoinBlock) void embed_join_kernel(const Spread a) {
    constexpr int N = kPack<T, F>;
    __shared__ float s_sum[kJoinWaves][kWave * N];
    __shared__ int32_t s_word[kJoinWaves], s_from[kJoinWaves], s_length[kJoinWaves];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t piece0 = int64_t(blockIdx.x) * kJoinWaves;
    {
        const int64_t piece = piece0 + wave;
        const int64_t place = piece * kHot + lane;
        const bool there = lane < kHot && place < a.start[a.vocab];
        const int word = there ? a.list[place].word : 0;
        const int n = there ? tokens_of(a, word) : 0;
        // one lane at most; lane 0 alone writes what it found (two lanes' stores to one
        // word are in no order that the compiler has to keep)
        const uint64_t starts = __ballot(n >= kHot && a.start[word] == place);
        const int from = starts != 0 ? __ffsll((unsigned long long)starts) - 1 : 0;
        const int its_word = __builtin_amdgcn_readlane(word, from), length = __builtin_amdgcn_readlane(n, from);
        if (lane == 0) {
            s_word[wave] = starts != 0 ? its_word : -1;
            s_from[wave] = from;
            s_length[wave] = length;
        }
    }
    __syncthreads();
    const int parts = (a.width + kWave * N - 1) / (kWave * N);
    for (int i = 0; i < kJoinWaves; ++i) {
        const int word = s_word[i], from = s_from[i];
        if (word < 0) continue;   // the same for every wave
        const int64_t piece = piece0 + i, pieces = (int64_t(from) + s_length[i] - 1) / kHot + 1;
        const int64_t each = (pieces + kJoinWaves - 1) / kJoinWaves;
        const int64_t lo = min(wave * each, pieces), hi = min(lo + each, pieces);
        for (int part = blockIdx.y; part < parts; part += gridDim.y) {
            const int at = (part * kWave + lane) * N;
            float sum[N] = {};
            if (at < a.width)
                sum_rows<N, kAhead>(a.width - at, int(hi - lo), [&](int j) {
                    const int64_t slot = (piece + lo + j) * 2 + (lo + j == 0 && from != 0);
                    return static_cast<const float *>(a.partial) + slot * a.width + at;
                }, sum);
            __syncthreads();
#pragma unroll
            for (int k = 0; k < N; ++k) s_sum[wave][k * kWave + lane] = sum[k];
            __syncthreads();
            if (wave == 0 && at < a.width) {
                for (int w = 1; w < kJoinWaves; ++w)
#pragma unroll
                    for (int k = 0; k < N; ++k) sum[k] = __fadd_rn(sum[k], s_sum[w][k * kWave + lane]);
                put_row<F, N>(a, word, at, sum);
            }
        }
    }
}

int64_t pieces_of(int32_t tokens) { return (int64_t(tokens) + kHot - 1) / kHot; }

// A grid's threads are counted in 32 bits; the kernels step on where it ends.
uint32_t grid_of(int64_t groups) { return uint32_t(groups < (1 << 20) ? groups : 1 << 20); }

// Whether all ids are looked through for every token and 64 packs of its columns.
bool few(int32_t tokens, int64_t parts) { return tokens <= kFewAny || tokens * parts <= kFew; }

size_t up16(size_t bytes) { return (bytes + 15) & ~size_t(15); }

// The workgroups that sum among all (dealt()), rounded up: as many as there are come out.
uint64_t share_of(const Spread &a) {
    const uint64_t all = uint64_t(a.sums) + uint64_t(a.clears);
    return all == 0 ? 0 : ((uint64_t(a.sums) << 32) + all - 1) / all;
}

template <typename T, typename F>
hipError_t spread(Spread a, hipStream_t stream) {
    constexpr int N = kPack<T, F>;
    const int64_t parts = (a.width + kWave * N - 1) / (kWave * N);
    const int64_t row_bytes = int64_t(a.width) * int(sizeof(F));
    if (few(a.tokens, parts)) {
        const int64_t rows = kFewBytes / row_bytes;
        a.rows = int32_t(rows > kMaxRows ? kMaxRows : rows);
        if (a.rows <= a.vocab >> 22) a.rows = (a.vocab >> 22) + 1;   // (a grid's threads again)
        a.clears = a.accumulate ? 0 : (a.vocab + a.rows - 1) / a.rows;
        a.sums = int32_t(a.tokens * parts);
        a.share = share_of(a);
        embed_few_kernel<T, F><<<uint32_t(a.sums) + uint32_t(a.clears), kBlock, 0, stream>>>(a);
        return hipGetLastError();
    }
    // How rows without a token are cleared.  Large tables whose rows are whole tiles of 4
    // KiB: by the second launch, which knows those rows, and in the order of the table.
    // Others, all of the table while the tokens are sorted.  16,384 tokens x 131,072 x 2,048
    // fp32 took 183 us by the first and 212 by the second; where tiles meet several rows,
    // 131,072 x 1,056 fp32 130 and 116, 1,055 bf16 91 and 75, 1,000,000 x 64 96 and 76.
    const bool whole = !a.accumulate && a.past && row_bytes % kRowTile == 0 && a.ld_dtable * int(sizeof(F)) % 128 == 0 &&
                       reinterpret_cast<uintptr_t>(a.dtable) % 128 == 0;
    a.rows = int32_t(kTileBytes / row_bytes < 1 ? 1 : kTileBytes / row_bytes);
    a.tiles = a.accumulate || whole ? 0 : a.ld_dtable != a.width ? (a.vocab + a.rows - 1) / a.rows :
              (a.vocab * row_bytes + 127 + kTileBytes - 1) / kTileBytes;
    a.clears = int32_t(grid_of(a.tiles));
    const int each = (a.vocab + device_cu_count() - 1) / device_cu_count();
    a.words = each > kMaxWords ? kMaxWords : each;
    a.sorts = (a.vocab + a.words - 1) / a.words;
    const size_t lds = size_t(a.words) * kSortWaves * sizeof(uint32_t);
    embed_sort_kernel<F><<<uint32_t(a.sorts + a.clears), kSortBlock, lds, stream>>>(a);
    const int64_t pieces = pieces_of(a.tokens);
    a.sums = int32_t(grid_of((pieces * parts * (kShares + 1) + kWaves - 1) / kWaves));
    if (whole) {
        a.tiles = a.vocab * (row_bytes / kRowTile);
        a.clears = int32_t(a.tiles < 1 << 23 ? a.tiles : 1 << 23);
        a.share = share_of(a);
        embed_rows_kernel<T, F, true><<<uint32_t(a.sums) + uint32_t(a.clears), kBlock, 0, stream>>>(a);
    } else {
        embed_rows_kernel<T, F, false><<<uint32_t(a.sums), kBlock, 0, stream>>>(a);
    }
    embed_join_kernel<T, F><<<dim3(uint32_t((pieces + kJoinWaves - 1) / kJoinWaves), uint32_t(parts < 64 ? parts : 64)), kJoinBlock, 0,
                              stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embed_forward(const void *table, int64_t ld_table, bool table_bf16, const int64_t *ids, void *out,
                                int64_t ld_out, bool bf16, int32_t tokens, int32_t vocab, int32_t width, float scale,
                                int64_t ignore, uint32_t *status, hipStream_t stream) {
    Lookup a{table, out, ids, ld_table, ld_out, ignore, tokens, vocab, width, 0, 0, scale, false, status};
    a.past = int64_t(tokens) * width * (bf16 ? 2 : 4) >= kPastCaches;
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

// [list][where words start][partial sums]; few tokens need none.  (Types whose
// packs are longer are few no later.)
size_t embed_workspace_size(int32_t tokens, int32_t vocab, int32_t width) {
    if (few(tokens, (int64_t(width) + kWave * 4 - 1) / (kWave * 4))) return 16;
    return up16(size_t(tokens) * sizeof(Sorted)) + up16((size_t(vocab) + 1) * sizeof(int32_t)) +
           up16(size_t(pieces_of(tokens)) * 2 * size_t(width) * sizeof(float));
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
    a.past = !accumulate && int64_t(vocab) * width * (table_bf16 ? 2 : 4) >= kPastCaches;
    a.list = reinterpret_cast<Sorted *>(ws);
    ws += up16(size_t(tokens) * sizeof(Sorted));
    a.start = reinterpret_cast<int32_t *>(ws);
    ws += up16((size_t(vocab) + 1) * sizeof(int32_t));
    a.partial = reinterpret_cast<float *>(ws);
    if (bf16 && table_bf16) return spread<__bf16, __bf16>(a, stream);
    if (bf16) return spread<__bf16, float>(a, stream);
    if (table_bf16) return spread<float, __bf16>(a, stream);
    return spread<float, float>(a, stream);
}

}  // namespace efs
