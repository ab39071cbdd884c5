// C ABI of libefsparse.so: host-side argument validation, status codes and
// dispatch to the kernel launchers.  Nothing here touches the device until
// every argument has been checked; nothing here allocates or synchronises.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <cstdlib>

#include "../../include/efsparse.h"
#include "launch.hpp"
#include "device_common.hpp"

static_assert(efs::kMaxApplyWorkers == EFS_MAX_WORKERS, "worker limit differs from the header");
static_assert(efs::kSparseTruncated == EFS_SPARSE_TRUNCATED, "status bit differs from the header");
static_assert(efs::kSparseBadIndex == EFS_SPARSE_BAD_INDEX, "status bit differs from the header");
static_assert(efs::kMaxSegments == EFS_SEG_MAX, "segment limit differs from the header");
static_assert(efs::kStaticScratchBytes == EFS_STATIC_SCRATCH_BYTES, "scratch size differs from the header");
static_assert(efs::kMuonMaxMatrices == EFS_MUON_MAX_MATRICES, "matrix limit differs from the header");
static_assert(efs::kMuonMaxSteps == EFS_MUON_MAX_STEPS, "step limit differs from the header");
static_assert(efs::kXentMaxTokens == EFS_XENT_MAX_TOKENS, "token limit differs from the header");
static_assert(efs::kXentMaxVocab == EFS_XENT_MAX_VOCAB, "vocabulary limit differs from the header");
static_assert(efs::kXentMaxHidden == EFS_XENT_MAX_HIDDEN, "hidden limit differs from the header");
static_assert(efs::kXentBadTarget == EFS_XENT_BAD_TARGET, "status bit differs from the header");
static_assert(efs::kEmbedMaxTokens == EFS_EMBED_MAX_TOKENS, "token limit differs from the header");
static_assert(efs::kEmbedMaxVocab == EFS_EMBED_MAX_VOCAB, "vocabulary limit differs from the header");
static_assert(efs::kEmbedMaxWidth == EFS_EMBED_MAX_WIDTH, "width limit differs from the header");
static_assert(efs::kEmbedBadId == EFS_EMBED_BAD_ID, "status bit differs from the header");
static_assert(efs::kNormMaxWidth == EFS_NORM_MAX_WIDTH, "width limit differs from the header");
static_assert(efs::kAdamwMaxTensors == EFS_ADAMW_MAX_TENSORS, "tensor limit differs from the header");
static_assert(sizeof(efs::Telemetry) == EFS_TELEMETRY_BYTES, "telemetry layout differs from the header");

namespace {

thread_local char g_message[256] = "";
thread_local efs_status g_sticky = EFS_OK;  // last non-OK status on this thread

efs_status fail(efs_status s, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_message, sizeof g_message, fmt, ap);
    va_end(ap);
    g_sticky = s;
    return s;
}

efs_status check_launch(hipError_t err, const char *what) {
    if (err != hipSuccess)
        return fail(EFS_EHIP, "%s: kernel launch failed: %s", what, hipGetErrorString(err));
    return EFS_OK;
}

bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int64_t kMaxLen = INT32_MAX;

// Whether two vectors of d floats share any byte.
bool overlap(const float *a, const float *b, int64_t d) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + uintptr_t(d) * 4 && y < x + uintptr_t(d) * 4;
}

// Memory that a tensor takes, in bytes: rows of `width`, `ld` apart (0: not so
// regular), over `span` from the first's start to the last's end.
struct Rows {
    uintptr_t at;
    int64_t ld, width, span;
};

Rows rows_of(const void *p, int64_t rows, int64_t ld, int64_t cols, int64_t size) {
    return Rows{reinterpret_cast<uintptr_t>(p), ld * size, cols * size, ((rows - 1) * ld + cols) * size};
}

// A batch of matrices: their rows, where the matrices are whole rows apart; where
// their rows take turns, as wide as all of them.
Rows rows_of_batch(const void *p, int64_t batch, int64_t stride, int64_t rows, int64_t ld, int64_t cols, int64_t size) {
    if (rows == 1) ld = batch > 1 && stride >= cols ? stride : cols;   // a row each
    const int64_t wide = (batch - 1) * stride + cols;
    Rows r = rows_of(p, rows, ld, cols, size);
    r.span += (batch - 1) * stride * size;
    if (batch > 1 && stride % ld != 0) {
        r.width = wide * size;
        if (wide > ld) r.ld = 0;
    }
    return r;
}

// Whether two tensors can share a byte: their spans do, unless the rows of both
// are as far apart throughout and take different columns of that.
bool meet(const Rows &a, const Rows &b) {
    if (a.at >= b.at + uintptr_t(b.span) || b.at >= a.at + uintptr_t(a.span)) return false;
    // a single row fits the other's
    const int64_t ld = a.span == a.width ? b.ld : b.span == b.width || a.ld == b.ld ? a.ld : 0;
    if (ld == 0) return true;
    const uintptr_t row = uintptr_t(ld), apart = a.at < b.at ? (b.at - a.at) % row : (row - (a.at - b.at) % row) % row;
    return apart < uintptr_t(a.width) || apart + uintptr_t(b.width) > row;
}

// A tensor of a call, under its name; what is written meets no other one.
struct Given {
    const char *name;
    Rows rows;
    bool written;
};

Given flat(const char *name, const void *p, int64_t bytes, bool written) {
    return Given{name, Rows{bytes == 0 ? 0 : reinterpret_cast<uintptr_t>(p), bytes, bytes, bytes}, written};
}

template <int N>
efs_status check_apart(const char *name, const Given (&given)[N]) {
    for (int i = 0; i < N; ++i)
        for (int j = 0; j < i; ++j)
            if ((given[i].written || given[j].written) && meet(given[i].rows, given[j].rows))
                return fail(EFS_EINVAL, "%s: %s and %s must not overlap", name, given[j].name, given[i].name);
    return EFS_OK;
}

// Memory of a list of tensors, of which each is a run of bytes.
struct Span {
    uintptr_t at, end;
    const char *name;
    bool written;
};

// Sees spans in ascending order and says which two share a byte that one of them writes.
struct SpanSweep {
    Span last = {0, 0, "", false}, last_written = {0, 0, "", false};   // those that reach furthest

    const char *add(const Span &s) {
        const char *met = nullptr;
        if (s.at < last_written.end) met = last_written.name;
        else if (s.written && s.at < last.end) met = last.name;
        if (s.end > last.end) last = s;
        if (s.written && s.end > last_written.end) last_written = s;
        return met;
    }
};

// One array of a call's list of tensors: pointers, bytes of each element (of the
// states of 8 bits: 0).
struct Column {
    const char *name;
    const void *const *at;   // NULL: none; entries may be NULL
    int64_t size;
    bool written;
};

Span span_of(const Column &c, const int64_t *sizes, int32_t i) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(c.at[i]);
    const uintptr_t bytes = c.size == 0 ? uintptr_t(efs::adamw_state_size(sizes[i])) : uintptr_t(sizes[i] * c.size);
    return Span{at, at + bytes, c.name, c.written};
}

// Something that is read beside the lists (NULL: nothing).
Span span_at(const char *name, const void *p, uintptr_t bytes) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    return Span{at, p == nullptr ? at : at + bytes, name, false};
}

// Whether what is written meets anything else, over all tensors of all columns.
// Layers of flat vectors come in ascending order and are merged as they are;
// others are sorted.
template <int N>
efs_status check_lists(const char *name, const Column (&columns)[N], const int64_t *sizes, int32_t count) {
    const auto there = [&](int c, int32_t i) {
        return columns[c].at != nullptr && columns[c].at[i] != nullptr && sizes[i] > 0;
    };
    bool ascending = true;
    int64_t spans = 0;
    for (int c = 0; c < N && columns[c].at != nullptr; ++c) {
        uintptr_t before = 0;
        for (int32_t i = 0; i < count; ++i)
            if (there(c, i)) {
                const uintptr_t at = reinterpret_cast<uintptr_t>(columns[c].at[i]);
                ascending = ascending && at >= before;
                before = at;
                ++spans;
            }
    }
    SpanSweep sweep;
    if (ascending) {
        int32_t next[N] = {};
        for (;;) {
            int least = -1;
            for (int c = 0; c < N; ++c) {
                if (columns[c].at == nullptr) continue;
                while (next[c] < count && !there(c, next[c])) ++next[c];
                if (next[c] < count && (least < 0 || columns[c].at[next[c]] < columns[least].at[next[least]])) least = c;
            }
            if (least < 0) return EFS_OK;
            const Span s = span_of(columns[least], sizes, next[least]++);
            if (const char *met = sweep.add(s))
                return fail(EFS_EINVAL, "%s: tensors of %s and %s must not overlap", name, met, s.name);
        }
    }
    Span *all = static_cast<Span *>(std::malloc(size_t(spans) * sizeof(Span)));
    if (all == nullptr) return fail(EFS_ESPACE, "%s: no host memory to check %lld tensors", name, (long long)spans);
    int64_t n = 0;
    for (int c = 0; c < N; ++c)
        for (int32_t i = 0; i < count; ++i)
            if (there(c, i)) all[n++] = span_of(columns[c], sizes, i);
    std::sort(all, all + n, [](const Span &a, const Span &b) { return a.at < b.at; });
    efs_status s = EFS_OK;
    for (int64_t i = 0; i < n && s == EFS_OK; ++i)
        if (const char *met = sweep.add(all[i]))
            s = fail(EFS_EINVAL, "%s: tensors of %s and %s must not overlap", name, met, all[i].name);
    std::free(all);
    return s;
}

int g_cu_count[64];  // per device; 0 = not queried yet

}  // namespace

namespace efs {

int device_cu_count() {
    int dev = 0;
    int cus = 256;
    if (hipGetDevice(&dev) == hipSuccess && dev >= 0 && dev < 64) {
        if (g_cu_count[dev] == 0) {
            int v = 0;
            if (hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess &&
                v > 0)
                g_cu_count[dev] = v;
            else
                g_cu_count[dev] = 256;
        }
        cus = g_cu_count[dev];
    }
    return cus;
}

uint32_t balanced_grid(int64_t work_tiles, int workgroups_per_cu) {
    if (work_tiles < 1) work_tiles = 1;
    const int64_t resident = int64_t(device_cu_count()) * workgroups_per_cu;
    const int64_t per_wg = (work_tiles + resident - 1) / resident;
    return uint32_t((work_tiles + per_wg - 1) / per_wg);
}

}  // namespace efs

extern "C" {

const char *efs_status_string(efs_status s) {
    switch (s) {
        case EFS_OK: return "ok";
        case EFS_EINVAL: return "invalid argument";
        case EFS_ESPACE: return "workspace too small";
        case EFS_EHIP: return "HIP runtime error";
    }
    return "unknown status";
}

const char *efs_last_error_message(void) { return g_message; }

efs_status efs_last_error(void) {
    if (hipPeekAtLastError() != hipSuccess) return EFS_EHIP;
    const efs_status s = g_sticky;
    g_sticky = EFS_OK;
    return s;
}

static efs_status ht_common(const char *name, const float *g, float *e, int64_t d, float lr,
                            float lambda, int32_t *idx, float *val, int64_t cap, uint32_t *counter,
                            void *telemetry, void *stream) {
    if (d < 0 || d > kMaxLen) return fail(EFS_EINVAL, "%s: d=%lld outside [0, 2^31-1]", name, (long long)d);
    if (d > 0 && (g == nullptr || e == nullptr)) return fail(EFS_EINVAL, "%s: g or e is NULL", name);
    if (!aligned(g, 4) || !aligned(e, 4)) return fail(EFS_EINVAL, "%s: g and e must be 4-byte aligned", name);
    if (!std::isfinite(lr)) return fail(EFS_EINVAL, "%s: lr must be finite", name);
    if (std::isnan(lambda) || lambda < 0.0f) return fail(EFS_EINVAL, "%s: lambda must be >= 0 and not NaN", name);
    if (cap < 0 || cap > kMaxLen) return fail(EFS_EINVAL, "%s: cap=%lld outside [0, 2^31-1]", name, (long long)cap);
    if (cap > 0 && (idx == nullptr || val == nullptr)) return fail(EFS_EINVAL, "%s: idx or val is NULL", name);
    if (!aligned(idx, 4) || !aligned(val, 4)) return fail(EFS_EINVAL, "%s: idx and val must be 4-byte aligned", name);
    if (counter == nullptr || !aligned(counter, 8)) return fail(EFS_EINVAL, "%s: counter must be non-NULL and 8-byte aligned", name);
    return check_launch(efs::launch_ht(g, e, d, lr, lambda, idx, val, cap, counter, telemetry,
                                       static_cast<hipStream_t>(stream)),
                        name);
}

efs_status ht_compress(const float *g, float *e, int64_t d, float lr, float lambda,
                       int32_t *idx, float *val, int64_t cap, uint32_t *counter,
                       void *stream) {
    return ht_common("ht_compress", g, e, d, lr, lambda, idx, val, cap, counter, nullptr, stream);
}

efs_status ht_compress_telemetry(const float *g, float *e, int64_t d, float lr, float lambda,
                                 int32_t *idx, float *val, int64_t cap, uint32_t *counter,
                                 void *telemetry, void *stream) {
    if (telemetry == nullptr || !aligned(telemetry, 8))
        return fail(EFS_EINVAL, "ht_compress_telemetry: telemetry must be non-NULL and 8-byte aligned");
    return ht_common("ht_compress_telemetry", g, e, d, lr, lambda, idx, val, cap, counter,
                     telemetry, stream);
}

size_t topk_workspace_bytes(int64_t d, int64_t k) {
    if (d < 0 || d > kMaxLen || k < 0 || k > d) return 0;
    return efs::topk_workspace_size(d, k);
}

size_t topk_path_flag_offset(void) { return efs::topk_path_flag_offset(); }

efs_status topk_compress(const float *g, float *e, int64_t d, float lr, int64_t k,
                         int32_t *idx, float *val, void *workspace, size_t workspace_bytes,
                         void *stream) {
    if (d < 0 || d > kMaxLen) return fail(EFS_EINVAL, "topk_compress: d=%lld outside [0, 2^31-1]", (long long)d);
    if (k < 0 || k > d) return fail(EFS_EINVAL, "topk_compress: k=%lld outside [0, d]", (long long)k);
    if (d > 0 && (g == nullptr || e == nullptr)) return fail(EFS_EINVAL, "topk_compress: g or e is NULL");
    if (!aligned(g, 4) || !aligned(e, 4)) return fail(EFS_EINVAL, "topk_compress: g and e must be 4-byte aligned");
    if (!std::isfinite(lr)) return fail(EFS_EINVAL, "topk_compress: lr must be finite");
    if (k > 0 && (idx == nullptr || val == nullptr)) return fail(EFS_EINVAL, "topk_compress: idx or val is NULL");
    if (!aligned(idx, 4) || !aligned(val, 4)) return fail(EFS_EINVAL, "topk_compress: idx and val must be 4-byte aligned");
    if (d > 0 && (workspace == nullptr || !aligned(workspace, 16)))
        return fail(EFS_EINVAL, "topk_compress: workspace must be non-NULL and 16-byte aligned");
    if (d > 0 && workspace_bytes < efs::topk_workspace_size(d, k))
        return fail(EFS_ESPACE, "topk_compress: workspace has %zu bytes, needs %zu", workspace_bytes,
                    efs::topk_workspace_size(d, k));
    return check_launch(efs::launch_topk(g, e, d, lr, k, idx, val, workspace,
                                         static_cast<hipStream_t>(stream)),
                        "topk_compress");
}

size_t topk_segmented_workspace_bytes(int32_t nseg, int64_t k_total) {
    if (nseg < 1 || nseg > efs::kMaxSegments || k_total < 0 || k_total > kMaxLen) return 0;
    return efs::topk_segmented_workspace_size(nseg, k_total);
}

size_t topk_segmented_status_offset(void) { return efs::topk_segmented_status_offset(); }

size_t topk_segmented_bracket_offset(void) { return efs::topk_segmented_bracket_offset(); }

efs_status topk_segmented_compress(const float *g, float *e, int64_t d, float lr, int32_t nseg,
                                   const int64_t *offsets, const int64_t *k, int64_t k_total,
                                   int32_t *idx, float *val, void *workspace,
                                   size_t workspace_bytes, void *stream) {
    const char *name = "topk_segmented_compress";
    if (d < 0 || d > kMaxLen) return fail(EFS_EINVAL, "%s: d=%lld outside [0, 2^31-1]", name, (long long)d);
    if (nseg < 1 || nseg > efs::kMaxSegments)
        return fail(EFS_EINVAL, "%s: nseg=%d outside [1, %d]", name, nseg, efs::kMaxSegments);
    if (k_total < 0 || k_total > d) return fail(EFS_EINVAL, "%s: k_total=%lld outside [0, d]", name, (long long)k_total);
    if (d > 0 && (g == nullptr || e == nullptr)) return fail(EFS_EINVAL, "%s: g or e is NULL", name);
    if (!aligned(g, 4) || !aligned(e, 4)) return fail(EFS_EINVAL, "%s: g and e must be 4-byte aligned", name);
    if (!std::isfinite(lr)) return fail(EFS_EINVAL, "%s: lr must be finite", name);
    if (offsets == nullptr || k == nullptr || !aligned(offsets, 8) || !aligned(k, 8))
        return fail(EFS_EINVAL, "%s: offsets and k must be non-NULL and 8-byte aligned", name);
    if (k_total > 0 && (idx == nullptr || val == nullptr)) return fail(EFS_EINVAL, "%s: idx or val is NULL", name);
    if (!aligned(idx, 4) || !aligned(val, 4)) return fail(EFS_EINVAL, "%s: idx and val must be 4-byte aligned", name);
    if (d == 0) return EFS_OK;
    if (workspace == nullptr || !aligned(workspace, 16))
        return fail(EFS_EINVAL, "%s: workspace must be non-NULL and 16-byte aligned", name);
    const size_t need = efs::topk_segmented_workspace_size(nseg, k_total);
    if (workspace_bytes < need)
        return fail(EFS_ESPACE, "%s: workspace has %zu bytes, needs %zu", name, workspace_bytes, need);
    return check_launch(efs::launch_topk_segmented(g, e, d, lr, nseg, offsets, k, k_total, idx, val,
                                                   workspace, static_cast<hipStream_t>(stream)),
                        name);
}

size_t sparse_apply_workspace_bytes(int32_t n_workers, int64_t d, int64_t total_cap) {
    if (n_workers < 1 || n_workers > efs::kMaxApplyWorkers || d < 0 || d > kMaxLen ||
        total_cap < 0 || total_cap > int64_t(UINT32_MAX))
        return 0;
    return efs::apply_workspace_size(n_workers, d, total_cap);
}

size_t sparse_accumulate_workspace_bytes(int32_t n_workers, int64_t d, int64_t total_cap) {
    return sparse_apply_workspace_bytes(n_workers, d, total_cap);
}

size_t sparse_bucket_workspace_bytes(int32_t n_workers, int64_t d) {
    if (n_workers < 1 || n_workers > efs::kMaxApplyWorkers || d < 0 || d > kMaxLen) return 0;
    return efs::apply_bucket_workspace_size(n_workers, d);
}

size_t sparse_status_offset(void) { return efs::apply_status_offset(); }

// Checks shared by sparse_accumulate, sparse_accumulate_static and
// sparse_apply: the payload arrays and the output (x).  Returns EFS_OK when
// they are valid, with the sum of the capacities in *total.
static efs_status check_payload_args(const char *name, const int32_t *const *idx,
                                     const float *const *val, const uint32_t *const *counts,
                                     const int64_t *caps, int32_t n_workers, int64_t d,
                                     const float *x, int64_t *total_out) {
    if (n_workers < 1 || n_workers > efs::kMaxApplyWorkers)
        return fail(EFS_EINVAL, "%s: n_workers=%d outside [1, %d]", name, n_workers,
                    efs::kMaxApplyWorkers);
    if (d < 0 || d > kMaxLen) return fail(EFS_EINVAL, "%s: d=%lld outside [0, 2^31-1]", name, (long long)d);
    if (idx == nullptr || val == nullptr || caps == nullptr)
        return fail(EFS_EINVAL, "%s: idx, val and caps must be host arrays", name);
    if (d > 0 && (x == nullptr || !aligned(x, 16)))
        return fail(EFS_EINVAL, "%s: the output must be non-NULL and 16-byte aligned", name);
    int64_t total = 0;
    for (int32_t w = 0; w < n_workers; ++w) {
        if (caps[w] < 0 || caps[w] > kMaxLen)
            return fail(EFS_EINVAL, "%s: caps[%d]=%lld outside [0, 2^31-1]", name, w, (long long)caps[w]);
        if (caps[w] > 0 && (idx[w] == nullptr || val[w] == nullptr))
            return fail(EFS_EINVAL, "%s: payload %d has a NULL pointer", name, w);
        if (!aligned(idx[w], 4) || !aligned(val[w], 4))
            return fail(EFS_EINVAL, "%s: payload %d is not 4-byte aligned", name, w);
        if (counts != nullptr && counts[w] != nullptr && !aligned(counts[w], 4))
            return fail(EFS_EINVAL, "%s: count %d is not 4-byte aligned", name, w);
        total += caps[w];
    }
    if (total > int64_t(UINT32_MAX))
        return fail(EFS_EINVAL, "%s: total capacity %lld exceeds 2^32-1 pairs", name, (long long)total);
    *total_out = total;
    return EFS_OK;
}

// Bytes the call needs of a workspace of `have` bytes: 0 when it holds the
// bucketed layout or the packed one, else the packed layout's size.
static size_t workspace_shortfall(int32_t n_workers, int64_t d, int64_t total, size_t have) {
    if (have >= efs::apply_bucket_workspace_size(n_workers, d)) return 0;
    const size_t need = efs::apply_workspace_size(n_workers, d, total);
    return have >= need ? 0 : need;
}

// The payload checks plus the workspace (pointer, alignment, size).
static efs_status check_payloads(const char *name, const int32_t *const *idx,
                                 const float *const *val, const uint32_t *const *counts,
                                 const int64_t *caps, int32_t n_workers, int64_t d, const float *x,
                                 const void *workspace, size_t workspace_bytes) {
    int64_t total = 0;
    const efs_status s = check_payload_args(name, idx, val, counts, caps, n_workers, d, x, &total);
    if (s != EFS_OK || d == 0) return s;
    if (workspace == nullptr || !aligned(workspace, 16))
        return fail(EFS_EINVAL, "%s: workspace must be non-NULL and 16-byte aligned", name);
    // the bucketed layout whenever the workspace holds it, else the packed one
    const size_t need = workspace_shortfall(n_workers, d, total, workspace_bytes);
    if (need != 0)
        return fail(EFS_ESPACE, "%s: workspace has %zu bytes, needs %zu", name, workspace_bytes, need);
    return EFS_OK;
}

efs_status sparse_accumulate(const int32_t *const *idx, const float *const *val,
                             const uint32_t *const *counts, const int64_t *caps,
                             int32_t n_workers, int64_t d, float *out, void *workspace,
                             size_t workspace_bytes, void *stream) {
    const efs_status s = check_payloads("sparse_accumulate", idx, val, counts, caps, n_workers, d,
                                        out, workspace, workspace_bytes);
    if (s != EFS_OK || d == 0) return s;
    return check_launch(efs::launch_apply(idx, val, counts, caps, n_workers, d, EFS_APPLY_AVERAGE,
                                          out, nullptr, 0.0f, 0.0f, workspace, workspace_bytes,
                                          static_cast<hipStream_t>(stream)),
                        "sparse_accumulate");
}

efs_status sparse_accumulate_static(const int32_t *const *idx, const float *const *val,
                                    const uint32_t *const *counts, const int64_t *caps,
                                    int32_t n_workers, int64_t d, float *out, void *stream) {
    const char *name = "sparse_accumulate_static";
    int64_t total = 0;
    const efs_status s = check_payload_args(name, idx, val, counts, caps, n_workers, d, out, &total);
    if (s != EFS_OK || d == 0) return s;
    const size_t need = workspace_shortfall(n_workers, d, total, efs::kStaticScratchBytes);
    if (need != 0)
        return fail(EFS_ESPACE, "%s: the payloads need %zu bytes of scratch; the library holds %zu "
                    "per device (use sparse_accumulate with a workspace)", name, need,
                    efs::kStaticScratchBytes);
    void *scratch = nullptr;
    const hipError_t err = efs::static_scratch(&scratch);
    if (err != hipSuccess)
        return fail(EFS_EHIP, "%s: no scratch on the current device: %s", name, hipGetErrorString(err));
    return check_launch(efs::launch_apply(idx, val, counts, caps, n_workers, d, EFS_APPLY_AVERAGE,
                                          out, nullptr, 0.0f, 0.0f, scratch,
                                          efs::kStaticScratchBytes,
                                          static_cast<hipStream_t>(stream)),
                        name);
}

efs_status sparse_apply(const int32_t *const *idx, const float *const *val,
                        const uint32_t *const *counts, const int64_t *caps, int32_t n_workers,
                        int64_t d, int mode, float *x, float *m, float beta, float gamma,
                        void *workspace, size_t workspace_bytes, void *stream) {
    if (mode < EFS_APPLY_AVERAGE || mode > EFS_APPLY_MOMENTUM)
        return fail(EFS_EINVAL, "sparse_apply: mode %d is not one of EFS_APPLY_*", mode);
    if (mode == EFS_APPLY_MOMENTUM && d > 0) {
        if (m == nullptr || !aligned(m, 16))
            return fail(EFS_EINVAL, "sparse_apply: m must be non-NULL and 16-byte aligned");
        if (m == x) return fail(EFS_EINVAL, "sparse_apply: m and x must not alias");
    }
    if (mode == EFS_APPLY_MOMENTUM && (!std::isfinite(beta) || !std::isfinite(gamma)))
        return fail(EFS_EINVAL, "sparse_apply: beta and gamma must be finite");
    const efs_status s = check_payloads("sparse_apply", idx, val, counts, caps, n_workers, d, x,
                                        workspace, workspace_bytes);
    if (s != EFS_OK || d == 0) return s;
    return check_launch(efs::launch_apply(idx, val, counts, caps, n_workers, d, mode, x, m, beta,
                                          gamma, workspace, workspace_bytes,
                                          static_cast<hipStream_t>(stream)),
                        "sparse_apply");
}

// What the two orthogonalising calls check alike.  next: from one matrix's
// entry of rows and cols to the next's (0: all alike).
static efs_status check_muon(const char *name, int32_t nmat, const int32_t *rows, const int32_t *cols,
                             int32_t next, int32_t steps, float eps, const void *workspace, size_t workspace_bytes,
                             int64_t *used) {
    if (steps < 1 || steps > efs::kMuonMaxSteps)
        return fail(EFS_EINVAL, "%s: steps=%d outside [1, %d]", name, steps, efs::kMuonMaxSteps);
    if (!std::isfinite(eps) || eps < 0.0f) return fail(EFS_EINVAL, "%s: eps must be finite and >= 0", name);
    size_t need = 0;
    if (!efs::muon_workspace_size(nmat, rows, cols, next, &need))
        return fail(EFS_EINVAL, "%s: the matrices are too many for one call", name);
    if (workspace == nullptr || !aligned(workspace, 16))
        return fail(EFS_EINVAL, "%s: workspace must be non-NULL and 16-byte aligned", name);
    if (workspace_bytes < need)
        return fail(EFS_ESPACE, "%s: workspace has %zu bytes, needs %zu", name, workspace_bytes, need);
    *used = int64_t(need);
    return EFS_OK;
}

size_t muon_workspace_bytes(int32_t nmat, const int32_t *rows, const int32_t *cols) {
    if (nmat < 0 || nmat > efs::kMuonMaxMatrices || (nmat > 0 && (rows == nullptr || cols == nullptr))) return 0;
    for (int32_t i = 0; i < nmat; ++i)
        if (rows[i] < 0 || cols[i] < 0 || int64_t(rows[i]) * cols[i] > kMaxLen) return 0;
    size_t bytes = 0;
    return efs::muon_workspace_size(nmat, rows, cols, 1, &bytes) ? bytes : 0;
}

efs_status muon_orthogonalize(const void *g, int64_t ld_g, int64_t stride_g, void *out, int64_t ld_out,
                              int64_t stride_out, int dtype, int32_t batch, int32_t rows, int32_t cols,
                              int32_t steps, const float *coeffs, float eps, void *workspace,
                              size_t workspace_bytes, void *stream) {
    const char *name = "muon_orthogonalize";
    static const float kCoeffs[3] = {3.4445f, -4.7750f, 2.0315f};
    if (dtype != EFS_FP32 && dtype != EFS_BF16)
        return fail(EFS_EINVAL, "%s: dtype %d is neither EFS_FP32 nor EFS_BF16", name, dtype);
    if (batch < 0 || batch > efs::kMuonMaxMatrices)
        return fail(EFS_EINVAL, "%s: batch=%d outside [0, %d]", name, batch, efs::kMuonMaxMatrices);
    if (rows < 0 || cols < 0 || int64_t(rows) * cols > kMaxLen)
        return fail(EFS_EINVAL, "%s: %d x %d is negative or has more than 2^31-1 elements", name, rows, cols);
    if (coeffs == nullptr) coeffs = kCoeffs;
    for (int k = 0; k < 3; ++k)
        if (!std::isfinite(coeffs[k])) return fail(EFS_EINVAL, "%s: coeffs must be finite", name);
    if (batch == 0 || rows == 0 || cols == 0) return EFS_OK;
    const uintptr_t size = dtype == EFS_BF16 ? 2 : 4;
    if (g == nullptr || out == nullptr || !aligned(g, size) || !aligned(out, size))
        return fail(EFS_EINVAL, "%s: g and out must be non-NULL and aligned to their type", name);
    if (ld_g < cols || ld_out < cols || ld_g > kMaxLen || ld_out > kMaxLen)
        return fail(EFS_EINVAL, "%s: ld_g and ld_out must be in [cols, 2^31-1]", name);
    if (stride_g < 0 || stride_out < 0 || stride_g > INT64_MAX / 4 / (int64_t(batch) + 1) ||
        stride_out > INT64_MAX / 4 / (int64_t(batch) + 1))
        return fail(EFS_EINVAL, "%s: stride_g or stride_out is negative or too large", name);
    // one matrix after the other, or their rows in turn
    if (batch > 1 && stride_out < (int64_t(rows) - 1) * ld_out + cols &&
        (stride_out < cols || ld_out < (int64_t(batch) - 1) * stride_out + cols))
        return fail(EFS_EINVAL, "%s: the matrices of out overlap", name);
    // a matrix is written when it has been read, but others may not have been
    if (batch > 1 && (g != out || ld_g != ld_out || stride_g != stride_out) &&
        meet(rows_of_batch(g, batch, stride_g, rows, ld_g, cols, size),
             rows_of_batch(out, batch, stride_out, rows, ld_out, cols, size)))
        return fail(EFS_EINVAL, "%s: out overlaps g and is not g itself", name);
    int64_t used = 0;
    efs_status s = check_muon(name, batch, &rows, &cols, 0, steps, eps, workspace, workspace_bytes, &used);
    if (s != EFS_OK) return s;
    const Given given[3] = {{"g", rows_of_batch(g, batch, stride_g, rows, ld_g, cols, size), false},
                            {"out", rows_of_batch(out, batch, stride_out, rows, ld_out, cols, size), false},
                            flat("workspace", workspace, used, true)};   // (g and out: above)
    s = check_apart(name, given);
    if (s != EFS_OK) return s;
    return check_launch(efs::launch_muon_orthogonalize(g, ld_g, stride_g, out, ld_out, stride_out,
                                                       dtype == EFS_BF16, batch, rows, cols, steps, coeffs,
                                                       eps, workspace, static_cast<hipStream_t>(stream)),
                        name);
}

efs_status muon_apply(const float *avg, float *x, float *m, int64_t d, int32_t nmat, const int64_t *offsets,
                      const int32_t *rows, const int32_t *cols, float beta, float gamma, float decay,
                      int nesterov, int32_t steps, float eps, void *workspace, size_t workspace_bytes,
                      void *stream) {
    const char *name = "muon_apply";
    static const float kCoeffs[3] = {3.4445f, -4.7750f, 2.0315f};
    if (d < 0 || d > kMaxLen) return fail(EFS_EINVAL, "%s: d=%lld outside [0, 2^31-1]", name, (long long)d);
    if (nmat < 0 || nmat > efs::kMuonMaxMatrices)
        return fail(EFS_EINVAL, "%s: nmat=%d outside [0, %d]", name, nmat, efs::kMuonMaxMatrices);
    if (nmat > 0 && (offsets == nullptr || rows == nullptr || cols == nullptr))
        return fail(EFS_EINVAL, "%s: offsets, rows and cols must be host arrays", name);
    if (!std::isfinite(beta) || !std::isfinite(gamma) || !std::isfinite(decay))
        return fail(EFS_EINVAL, "%s: beta, gamma and decay must be finite", name);
    if (nesterov != 0 && nesterov != 1) return fail(EFS_EINVAL, "%s: nesterov must be 0 or 1", name);
    int64_t end = 0;
    bool any = false;
    for (int32_t i = 0; i < nmat; ++i) {
        if (rows[i] < 0 || cols[i] < 0 || int64_t(rows[i]) * cols[i] > kMaxLen)
            return fail(EFS_EINVAL, "%s: matrix %d of %d x %d is negative or has more than 2^31-1 elements", name,
                        i, rows[i], cols[i]);
        const int64_t size = int64_t(rows[i]) * cols[i];
        if (offsets[i] < end || offsets[i] > d - size)
            return fail(EFS_EINVAL, "%s: matrix %d starts before the one before it ends, or ends past d", name, i);
        end = offsets[i] + size;
        any = any || size > 0;
    }
    if (!any) return EFS_OK;
    if (avg == nullptr || x == nullptr || m == nullptr || !aligned(avg, 4) || !aligned(x, 4) || !aligned(m, 4))
        return fail(EFS_EINVAL, "%s: avg, x and m must be non-NULL and 4-byte aligned", name);
    if (overlap(avg, x, d) || overlap(avg, m, d) || overlap(x, m, d))
        return fail(EFS_EINVAL, "%s: avg, x and m must not overlap", name);
    int64_t used = 0;
    efs_status s = check_muon(name, nmat, rows, cols, 1, steps, eps, workspace, workspace_bytes, &used);
    if (s != EFS_OK) return s;
    const Given given[4] = {flat("avg", avg, d * 4, false), flat("x", x, d * 4, true), flat("m", m, d * 4, true),
                            flat("workspace", workspace, used, true)};
    s = check_apart(name, given);
    if (s != EFS_OK) return s;
    return check_launch(efs::launch_muon_apply(avg, nmat, offsets, rows, cols, x, m, beta, gamma, decay,
                                               nesterov != 0, steps, kCoeffs, eps, workspace,
                                               static_cast<hipStream_t>(stream)),
                        name);
}

static bool xent_sizes_ok(int32_t tokens, int32_t vocab, int32_t hidden, int dtype) {
    return tokens >= 0 && tokens <= efs::kXentMaxTokens && vocab >= 1 && vocab <= efs::kXentMaxVocab &&
           hidden >= 1 && hidden <= efs::kXentMaxHidden && int64_t(tokens) * vocab <= int64_t(1) << 38 &&
           (dtype == EFS_FP32 || dtype == EFS_BF16);
}

size_t xent_workspace_bytes(int32_t tokens, int32_t vocab, int32_t hidden, int dtype, int gradient) {
    if (!xent_sizes_ok(tokens, vocab, hidden, dtype) || gradient < 0 || gradient > 1) return 0;
    return efs::xent_workspace_size(tokens, vocab, hidden, dtype == EFS_BF16, gradient != 0);
}

size_t xent_status_offset(void) { return 0; }

// What both directions check alike.  Their rows: pointer, elements between them.
static efs_status check_xent(const char *name, const void *h, int64_t ld_h, const void *w, int64_t ld_w,
                             const int64_t *target, int dtype, int32_t tokens, int32_t vocab, int32_t hidden,
                             bool gradient, const void *workspace, size_t workspace_bytes, int64_t *used) {
    if (dtype != EFS_FP32 && dtype != EFS_BF16)
        return fail(EFS_EINVAL, "%s: dtype %d is neither EFS_FP32 nor EFS_BF16", name, dtype);
    if (!xent_sizes_ok(tokens, vocab, hidden, dtype))
        return fail(EFS_EINVAL, "%s: %d tokens, %d words or %d values a row are outside the limits", name, tokens,
                    vocab, hidden);
    if (tokens == 0) return EFS_OK;
    const uintptr_t size = dtype == EFS_BF16 ? 2 : 4;
    if (h == nullptr || w == nullptr || !aligned(h, size) || !aligned(w, size))
        return fail(EFS_EINVAL, "%s: h and w must be non-NULL and aligned to their type", name);
    if (ld_h < hidden || ld_w < hidden || ld_h > kMaxLen || ld_w > kMaxLen)
        return fail(EFS_EINVAL, "%s: ld_h and ld_w must be in [hidden, 2^31-1]", name);
    if (target == nullptr || !aligned(target, 8))
        return fail(EFS_EINVAL, "%s: target must be non-NULL and 8-byte aligned", name);
    if (workspace == nullptr || !aligned(workspace, 16))
        return fail(EFS_EINVAL, "%s: workspace must be non-NULL and 16-byte aligned", name);
    const size_t need = efs::xent_workspace_size(tokens, vocab, hidden, dtype == EFS_BF16, gradient);
    if (workspace_bytes < need)
        return fail(EFS_ESPACE, "%s: workspace has %zu bytes, needs %zu", name, workspace_bytes, need);
    *used = int64_t(need);
    return EFS_OK;
}

// A call without tokens: the status word is cleared where there is one.
static efs_status clear_xent_status(const char *name, void *workspace, size_t workspace_bytes, void *stream) {
    if (workspace == nullptr || workspace_bytes < sizeof(uint32_t) || !aligned(workspace, 4)) return EFS_OK;
    return check_launch(efs::launch_xent_clear(workspace, static_cast<hipStream_t>(stream)), name);
}

efs_status xent_forward(const void *h, int64_t ld_h, const void *w, int64_t ld_w, const int64_t *target,
                        int dtype, int32_t tokens, int32_t vocab, int32_t hidden, int64_t ignore_index,
                        float *loss, float *lse, void *workspace, size_t workspace_bytes, void *stream) {
    const char *name = "xent_forward";
    int64_t used = 0;
    efs_status s = check_xent(name, h, ld_h, w, ld_w, target, dtype, tokens, vocab, hidden, false, workspace,
                              workspace_bytes, &used);
    if (s != EFS_OK) return s;
    if (tokens == 0) return clear_xent_status(name, workspace, workspace_bytes, stream);
    if (loss == nullptr || lse == nullptr || !aligned(loss, 4) || !aligned(lse, 4))
        return fail(EFS_EINVAL, "%s: loss and lse must be non-NULL and 4-byte aligned", name);
    const int64_t size = dtype == EFS_BF16 ? 2 : 4, t = tokens;
    const Given given[6] = {{"h", rows_of(h, t, ld_h, hidden, size), false},
                            {"w", rows_of(w, vocab, ld_w, hidden, size), false},
                            flat("target", target, t * 8, false), flat("loss", loss, t * 4, true),
                            flat("lse", lse, t * 4, true), flat("workspace", workspace, used, true)};
    s = check_apart(name, given);
    if (s != EFS_OK) return s;
    return check_launch(efs::launch_xent_forward(h, ld_h, w, ld_w, target, dtype == EFS_BF16, tokens, vocab,
                                                 hidden, ignore_index, loss, lse, workspace,
                                                 static_cast<hipStream_t>(stream)),
                        name);
}

efs_status xent_backward(const void *h, int64_t ld_h, const void *w, int64_t ld_w, const int64_t *target,
                         int dtype, int32_t tokens, int32_t vocab, int32_t hidden, int64_t ignore_index,
                         const float *lse, const float *dloss, void *dh, int64_t ld_dh, void *dw, int64_t ld_dw,
                         void *workspace, size_t workspace_bytes, void *stream) {
    const char *name = "xent_backward";
    int64_t used = 0;
    efs_status s = check_xent(name, h, ld_h, w, ld_w, target, dtype, tokens, vocab, hidden, true, workspace,
                              workspace_bytes, &used);
    if (s != EFS_OK) return s;
    const uintptr_t size = dtype == EFS_BF16 ? 2 : 4;
    if (dw == nullptr || !aligned(dw, size) || ld_dw < hidden || ld_dw > kMaxLen)
        return fail(EFS_EINVAL, "%s: dw must be non-NULL and aligned to its type, ld_dw in [hidden, 2^31-1]", name);
    if (tokens == 0) {
        const efs_status cleared = clear_xent_status(name, workspace, workspace_bytes, stream);
        if (cleared != EFS_OK) return cleared;
    } else {
        if (dh == nullptr || !aligned(dh, size) || ld_dh < hidden || ld_dh > kMaxLen)
            return fail(EFS_EINVAL, "%s: dh must be non-NULL and aligned to its type, ld_dh in [hidden, 2^31-1]",
                        name);
        if (lse == nullptr || dloss == nullptr || !aligned(lse, 4) || !aligned(dloss, 4))
            return fail(EFS_EINVAL, "%s: lse and dloss must be non-NULL and 4-byte aligned", name);
        const int64_t t = tokens;
        const Given given[8] = {{"h", rows_of(h, t, ld_h, hidden, size), false},
                                {"w", rows_of(w, vocab, ld_w, hidden, size), false},
                                {"dh", rows_of(dh, t, ld_dh, hidden, size), true},
                                {"dw", rows_of(dw, vocab, ld_dw, hidden, size), true},
                                flat("target", target, t * 8, false), flat("lse", lse, t * 4, false),
                                flat("dloss", dloss, t * 4, false), flat("workspace", workspace, used, true)};
        s = check_apart(name, given);
        if (s != EFS_OK) return s;
    }
    return check_launch(efs::launch_xent_backward(h, ld_h, w, ld_w, target, dtype == EFS_BF16, tokens, vocab,
                                                  hidden, ignore_index, lse, dloss, dh, ld_dh, dw, ld_dw,
                                                  workspace, static_cast<hipStream_t>(stream)),
                        name);
}

static bool dtype_ok(int dtype) { return dtype == EFS_FP32 || dtype == EFS_BF16; }

static int64_t dtype_size(int dtype) { return dtype == EFS_BF16 ? 2 : 4; }

// A matrix of a call: non-NULL, aligned to its type, its rows no closer than they are long.
static efs_status check_rows(const char *name, const char *what, const void *p, int64_t ld, int32_t cols, int dtype) {
    if (p == nullptr || !aligned(p, uintptr_t(dtype_size(dtype))))
        return fail(EFS_EINVAL, "%s: %s must be non-NULL and aligned to its type", name, what);
    if (ld < cols || ld > kMaxLen) return fail(EFS_EINVAL, "%s: ld_%s must be in [%d, 2^31-1]", name, what, cols);
    return EFS_OK;
}

// What both directions of the lookup check alike.
static efs_status check_embed(const char *name, int table_dtype, const int64_t *ids, int dtype, int32_t tokens,
                              int32_t vocab, int32_t width, float scale, const uint32_t *status) {
    if (!dtype_ok(dtype) || !dtype_ok(table_dtype))
        return fail(EFS_EINVAL, "%s: a dtype is neither EFS_FP32 nor EFS_BF16", name);
    if (tokens < 0 || tokens > efs::kEmbedMaxTokens || vocab < 1 || vocab > efs::kEmbedMaxVocab || width < 1 ||
        width > efs::kEmbedMaxWidth)
        return fail(EFS_EINVAL, "%s: %d tokens, %d words or %d values a row are outside the limits", name, tokens,
                    vocab, width);
    if (!std::isfinite(scale)) return fail(EFS_EINVAL, "%s: scale must be finite", name);
    if (tokens > 0 && (ids == nullptr || !aligned(ids, 8)))
        return fail(EFS_EINVAL, "%s: ids must be non-NULL and 8-byte aligned", name);
    if (!aligned(status, 4)) return fail(EFS_EINVAL, "%s: status must be 4-byte aligned", name);
    return EFS_OK;
}

efs_status embed_forward(const void *table, int64_t ld_table, int table_dtype, const int64_t *ids, void *out,
                         int64_t ld_out, int dtype, int32_t tokens, int32_t vocab, int32_t width, float scale,
                         int64_t ignore_index, uint32_t *status, void *stream) {
    const char *name = "embed_forward";
    efs_status s = check_embed(name, table_dtype, ids, dtype, tokens, vocab, width, scale, status);
    if (s != EFS_OK || tokens == 0) return s;
    if ((s = check_rows(name, "table", table, ld_table, width, table_dtype)) != EFS_OK) return s;
    if ((s = check_rows(name, "out", out, ld_out, width, dtype)) != EFS_OK) return s;
    const Given given[4] = {{"table", rows_of(table, vocab, ld_table, width, dtype_size(table_dtype)), false},
                            {"out", rows_of(out, tokens, ld_out, width, dtype_size(dtype)), true},
                            flat("ids", ids, int64_t(tokens) * 8, false),
                            flat("status", status, status != nullptr ? 4 : 0, true)};
    if ((s = check_apart(name, given)) != EFS_OK) return s;
    return check_launch(efs::launch_embed_forward(table, ld_table, table_dtype == EFS_BF16, ids, out, ld_out,
                                                  dtype == EFS_BF16, tokens, vocab, width, scale, ignore_index, status,
                                                  static_cast<hipStream_t>(stream)),
                        name);
}

size_t embed_workspace_bytes(int32_t tokens, int32_t vocab, int32_t width) {
    if (tokens < 0 || tokens > efs::kEmbedMaxTokens || vocab < 1 || vocab > efs::kEmbedMaxVocab || width < 1 ||
        width > efs::kEmbedMaxWidth || int64_t(tokens) * vocab > int64_t(1) << 38)
        return 0;
    return efs::embed_workspace_size(tokens, vocab, width);
}

efs_status embed_backward(const void *dout, int64_t ld_dout, int dtype, const int64_t *ids, void *dtable,
                          int64_t ld_dtable, int table_dtype, int32_t tokens, int32_t vocab, int32_t width,
                          float scale, int64_t ignore_index, int accumulate, uint32_t *status, void *workspace,
                          size_t workspace_bytes, void *stream) {
    const char *name = "embed_backward";
    efs_status s = check_embed(name, table_dtype, ids, dtype, tokens, vocab, width, scale, status);
    if (s != EFS_OK) return s;
    const size_t need = embed_workspace_bytes(tokens, vocab, width);
    if (need == 0) return fail(EFS_EINVAL, "%s: %d tokens x %d words are more than 2^38", name, tokens, vocab);
    if (accumulate != 0 && accumulate != 1) return fail(EFS_EINVAL, "%s: accumulate must be 0 or 1", name);
    if ((s = check_rows(name, "dtable", dtable, ld_dtable, width, table_dtype)) != EFS_OK) return s;
    if (tokens > 0 && (s = check_rows(name, "dout", dout, ld_dout, width, dtype)) != EFS_OK) return s;
    if (workspace == nullptr || !aligned(workspace, 16))
        return fail(EFS_EINVAL, "%s: workspace must be non-NULL and 16-byte aligned", name);
    if (workspace_bytes < need)
        return fail(EFS_ESPACE, "%s: workspace has %zu bytes, needs %zu", name, workspace_bytes, need);
    const Given given[5] = {{"dtable", rows_of(dtable, vocab, ld_dtable, width, dtype_size(table_dtype)), true},
                            tokens > 0 ? Given{"dout", rows_of(dout, tokens, ld_dout, width, dtype_size(dtype)), false}
                                       : flat("dout", nullptr, 0, false),
                            flat("ids", ids, int64_t(tokens) * 8, false),
                            flat("status", status, status != nullptr ? 4 : 0, true),
                            flat("workspace", workspace, int64_t(need), true)};
    if ((s = check_apart(name, given)) != EFS_OK) return s;
    if (tokens == 0 && accumulate) return EFS_OK;
    return check_launch(efs::launch_embed_backward(dout, ld_dout, dtype == EFS_BF16, ids, dtable, ld_dtable,
                                                   table_dtype == EFS_BF16, tokens, vocab, width, scale, ignore_index,
                                                   accumulate != 0, status, workspace,
                                                   static_cast<hipStream_t>(stream)),
                        name);
}

// What both directions of the norm check alike.
static efs_status check_norm(const char *name, const void *x, int64_t ld_x, const void *weight, int dtype,
                             int weight_dtype, int32_t rows, int32_t width) {
    if (!dtype_ok(dtype) || !dtype_ok(weight_dtype))
        return fail(EFS_EINVAL, "%s: a dtype is neither EFS_FP32 nor EFS_BF16", name);
    if (rows < 0 || width < 1 || width > efs::kNormMaxWidth)
        return fail(EFS_EINVAL, "%s: %d rows of %d values are outside the limits", name, rows, width);
    if (!aligned(weight, uintptr_t(dtype_size(weight_dtype))))
        return fail(EFS_EINVAL, "%s: weight must be aligned to its type", name);
    return rows == 0 ? EFS_OK : check_rows(name, "x", x, ld_x, width, dtype);
}

// Rows that are written: they may be those of an input itself, and then meet nothing of it.
static Given given_rows(const char *name, const void *p, int64_t rows, int64_t ld, int64_t width, int dtype, bool written) {
    if (rows == 0) return flat(name, nullptr, 0, written);
    return Given{name, rows_of(p, rows, ld, width, dtype_size(dtype)), written};
}

efs_status layernorm_forward(const void *x, int64_t ld_x, const void *weight, const void *bias, void *y, int64_t ld_y,
                             int dtype, int weight_dtype, int32_t rows, int32_t width, float eps, float *mean,
                             float *rstd, void *stream) {
    const char *name = "layernorm_forward";
    efs_status s = check_norm(name, x, ld_x, weight, dtype, weight_dtype, rows, width);
    if (s != EFS_OK) return s;
    if (!aligned(bias, uintptr_t(dtype_size(weight_dtype))))
        return fail(EFS_EINVAL, "%s: bias must be aligned to its type", name);
    if (!std::isfinite(eps) || eps < 0.0f) return fail(EFS_EINVAL, "%s: eps must be finite and >= 0", name);
    if (!aligned(mean, 4) || !aligned(rstd, 4)) return fail(EFS_EINVAL, "%s: mean and rstd must be 4-byte aligned", name);
    if (rows == 0) return EFS_OK;
    if ((s = check_rows(name, "y", y, ld_y, width, dtype)) != EFS_OK) return s;
    const bool itself = y == x && (ld_y == ld_x || rows == 1);
    const int64_t row = int64_t(width) * dtype_size(weight_dtype);
    const Given given[6] = {given_rows("x", x, itself ? 0 : rows, ld_x, width, dtype, false),
                            given_rows("y", y, rows, ld_y, width, dtype, true),
                            flat("weight", weight, weight != nullptr ? row : 0, false),
                            flat("bias", bias, bias != nullptr ? row : 0, false),
                            flat("mean", mean, mean != nullptr ? int64_t(rows) * 4 : 0, true),
                            flat("rstd", rstd, rstd != nullptr ? int64_t(rows) * 4 : 0, true)};
    if ((s = check_apart(name, given)) != EFS_OK) return s;
    return check_launch(efs::launch_layernorm_forward(x, ld_x, weight, bias, y, ld_y, dtype == EFS_BF16,
                                                      weight_dtype == EFS_BF16, rows, width, eps, mean, rstd,
                                                      static_cast<hipStream_t>(stream)),
                        name);
}

size_t layernorm_workspace_bytes(int32_t rows, int32_t width) {
    if (rows < 0 || width < 1 || width > efs::kNormMaxWidth) return 0;
    return efs::layernorm_workspace_size(rows, width);
}

efs_status layernorm_backward(const void *x, int64_t ld_x, const void *weight, const float *mean, const float *rstd,
                              const void *dy, int64_t ld_dy, void *dx, int64_t ld_dx, int dtype, int weight_dtype,
                              int32_t rows, int32_t width, void *dweight, void *dbias, void *workspace,
                              size_t workspace_bytes, void *stream) {
    const char *name = "layernorm_backward";
    efs_status s = check_norm(name, x, ld_x, weight, dtype, weight_dtype, rows, width);
    if (s != EFS_OK) return s;
    const uintptr_t size = uintptr_t(dtype_size(weight_dtype));
    if (!aligned(dweight, size) || !aligned(dbias, size))
        return fail(EFS_EINVAL, "%s: dweight and dbias must be aligned to their type", name);
    if (rows > 0) {
        if ((s = check_rows(name, "dy", dy, ld_dy, width, dtype)) != EFS_OK) return s;
        if ((s = check_rows(name, "dx", dx, ld_dx, width, dtype)) != EFS_OK) return s;
        if (mean == nullptr || rstd == nullptr || !aligned(mean, 4) || !aligned(rstd, 4))
            return fail(EFS_EINVAL, "%s: mean and rstd must be non-NULL and 4-byte aligned", name);
    }
    if (workspace == nullptr || !aligned(workspace, 16))
        return fail(EFS_EINVAL, "%s: workspace must be non-NULL and 16-byte aligned", name);
    const size_t need = efs::layernorm_workspace_size(rows, width);
    if (workspace_bytes < need)
        return fail(EFS_ESPACE, "%s: workspace has %zu bytes, needs %zu", name, workspace_bytes, need);
    const bool is_x = dx == x && (ld_dx == ld_x || rows == 1), is_dy = dx == dy && (ld_dx == ld_dy || rows == 1);
    const int64_t row = int64_t(width) * int64_t(size), each = int64_t(rows) * 4;
    const Given given[9] = {given_rows("x", x, is_x ? 0 : rows, ld_x, width, dtype, false),
                            given_rows("dy", dy, is_dy ? 0 : rows, ld_dy, width, dtype, false),
                            given_rows("dx", dx, rows, ld_dx, width, dtype, true),
                            flat("weight", weight, weight != nullptr ? row : 0, false),
                            flat("mean", mean, each, false),
                            flat("rstd", rstd, each, false),
                            flat("dweight", dweight, dweight != nullptr ? row : 0, true),
                            flat("dbias", dbias, dbias != nullptr ? row : 0, true),
                            flat("workspace", workspace, int64_t(need), true)};
    if ((s = check_apart(name, given)) != EFS_OK) return s;
    if (rows == 0 && dweight == nullptr && dbias == nullptr) return EFS_OK;
    return check_launch(efs::launch_layernorm_backward(x, ld_x, weight, mean, rstd, dy, ld_dy, dx, ld_dx,
                                                       dtype == EFS_BF16, weight_dtype == EFS_BF16, rows, width,
                                                       dweight, dbias, workspace, static_cast<hipStream_t>(stream)),
                        name);
}

size_t adamw_state_bytes(int64_t size) {
    if (size < 0 || size > kMaxLen) return 0;
    return efs::adamw_state_size(size);
}

// One array of tensors: there, and every tensor that is not empty aligned.
static efs_status check_list(const char *name, const char *what, const void *const *list, const int64_t *sizes,
                             int32_t count, uintptr_t align, bool optional) {
    if (list == nullptr) return fail(EFS_EINVAL, "%s: %s must be a host array", name, what);
    for (int32_t i = 0; i < count; ++i)
        if (sizes[i] > 0 && ((list[i] == nullptr && !optional) || !aligned(list[i], align)))
            return fail(EFS_EINVAL, "%s: tensor %d of %s must be non-NULL and %d-byte aligned", name, i, what,
                        int(align));
    return EFS_OK;
}

static efs_status check_sizes(const char *name, const int64_t *sizes, int32_t count) {
    if (count < 0 || count > efs::kAdamwMaxTensors)
        return fail(EFS_EINVAL, "%s: count=%d outside [0, %d]", name, count, efs::kAdamwMaxTensors);
    if (count > 0 && sizes == nullptr) return fail(EFS_EINVAL, "%s: sizes must be a host array", name);
    for (int32_t i = 0; i < count; ++i)
        if (sizes[i] < 0 || sizes[i] > kMaxLen)
            return fail(EFS_EINVAL, "%s: tensor %d has %lld elements, not 0 to 2^31-1", name, i, (long long)sizes[i]);
    return EFS_OK;
}

static const void *const *as_list(const void *list) { return static_cast<const void *const *>(list); }

efs_status adamw_apply(const void *const *g, int grad_dtype, float *const *x, void *const *copies, void *const *m,
                       void *const *v, int state, const int64_t *sizes, const float *decays, int32_t count,
                       float gamma, float beta1, float beta2, float eps, int64_t step, const int64_t *step_device,
                       const float *factors, uint32_t seed, void *stream) {
    const char *name = "adamw_apply";
    if (!dtype_ok(grad_dtype)) return fail(EFS_EINVAL, "%s: grad_dtype is neither EFS_FP32 nor EFS_BF16", name);
    if (state != EFS_STATE_32 && state != EFS_STATE_8)
        return fail(EFS_EINVAL, "%s: state is neither EFS_STATE_32 nor EFS_STATE_8", name);
    efs_status s = check_sizes(name, sizes, count);
    if (s != EFS_OK) return s;
    if (!std::isfinite(gamma) || !std::isfinite(eps) || eps < 0.0f)
        return fail(EFS_EINVAL, "%s: gamma and eps must be finite, eps >= 0", name);
    if (!(beta1 >= 0.0f && beta1 < 1.0f && beta2 >= 0.0f && beta2 < 1.0f))
        return fail(EFS_EINVAL, "%s: beta1 and beta2 must be in [0, 1)", name);
    if (step_device == nullptr && step < 1) return fail(EFS_EINVAL, "%s: step must be >= 1", name);
    if (!aligned(step_device, 8) || !aligned(factors, 4))
        return fail(EFS_EINVAL, "%s: step_device must be 8-byte and factors 4-byte aligned", name);
    if (count == 0) return EFS_OK;
    const bool bytes = state == EFS_STATE_8;
    const uintptr_t held = bytes ? 16 : 4;
    if ((s = check_list(name, "g", g, sizes, count, uintptr_t(dtype_size(grad_dtype)), false)) != EFS_OK) return s;
    if ((s = check_list(name, "x", as_list(x), sizes, count, 4, false)) != EFS_OK) return s;
    if ((s = check_list(name, "m", as_list(m), sizes, count, held, false)) != EFS_OK) return s;
    if ((s = check_list(name, "v", as_list(v), sizes, count, held, false)) != EFS_OK) return s;
    if (copies != nullptr && (s = check_list(name, "copies", as_list(copies), sizes, count, 2, true)) != EFS_OK) return s;
    for (int32_t i = 0; decays != nullptr && i < count; ++i)
        if (!std::isfinite(decays[i])) return fail(EFS_EINVAL, "%s: decays must be finite", name);
    const Column columns[5] = {{"g", g, dtype_size(grad_dtype), false},
                               {"x", as_list(x), 4, true},
                               {"m", as_list(m), bytes ? 0 : 4, true},
                               {"v", as_list(v), bytes ? 0 : 4, true},
                               {"copies", as_list(copies), 2, true}};
    if ((s = check_lists(name, columns, sizes, count)) != EFS_OK) return s;
    const Span read[2] = {span_at("step_device", step_device, 8), span_at("factors", factors, 8)};
    for (const Column &c : columns)
        for (int32_t i = 0; c.written && c.at != nullptr && i < count; ++i)
            for (const Span &r : read) {
                if (c.at[i] == nullptr || sizes[i] == 0) continue;
                const Span t = span_of(c, sizes, i);
                if (t.at < r.end && r.at < t.end)
                    return fail(EFS_EINVAL, "%s: tensors of %s and %s must not overlap", name, c.name, r.name);
            }
    const efs::AdamwArgs args{g,    x,     m,     v,   copies, sizes,       decays,  count, grad_dtype == EFS_BF16, bytes,
                              gamma, beta1, beta2, eps, step,   step_device, factors, seed};
    return check_launch(efs::launch_adamw(args, static_cast<hipStream_t>(stream)), name);
}

static efs_status state_call(const char *name, bool write, float *const *m, float *const *v, void *const *m8,
                             void *const *v8, const int64_t *sizes, int32_t count, void *stream) {
    efs_status s = check_sizes(name, sizes, count);
    if (s != EFS_OK || count == 0) return s;
    if ((s = check_list(name, "m", as_list(m), sizes, count, 4, false)) != EFS_OK) return s;
    if ((s = check_list(name, "v", as_list(v), sizes, count, 4, false)) != EFS_OK) return s;
    if ((s = check_list(name, "m8", as_list(m8), sizes, count, 16, false)) != EFS_OK) return s;
    if ((s = check_list(name, "v8", as_list(v8), sizes, count, 16, false)) != EFS_OK) return s;
    const Column columns[4] = {{"m", as_list(m), 4, !write},
                               {"v", as_list(v), 4, !write},
                               {"m8", as_list(m8), 0, write},
                               {"v8", as_list(v8), 0, write}};
    if ((s = check_lists(name, columns, sizes, count)) != EFS_OK) return s;
    return check_launch(efs::launch_adamw_state(write, m, v, m8, v8, sizes, count, static_cast<hipStream_t>(stream)),
                        name);
}

efs_status adamw_read_state(void *const *m8, void *const *v8, float *const *m, float *const *v, const int64_t *sizes,
                            int32_t count, void *stream) {
    return state_call("adamw_read_state", false, m, v, m8, v8, sizes, count, stream);
}

efs_status adamw_write_state(float *const *m, float *const *v, void *const *m8, void *const *v8, const int64_t *sizes,
                             int32_t count, void *stream) {
    return state_call("adamw_write_state", true, m, v, m8, v8, sizes, count, stream);
}

// The probes address at most INT32_MAX tiles (one workgroup each in the
// one-tile-per-workgroup shape).
constexpr int64_t kProbeMaxElements = int64_t(INT32_MAX) * efs::kTile;

efs_status efs_copy_probe(const float *src, float *dst, int64_t n, void *stream) {
    if (n < 0 || n > kProbeMaxElements)
        return fail(EFS_EINVAL, "efs_copy_probe: n = %lld outside [0, %lld]", (long long)n,
                    (long long)kProbeMaxElements);
    if (n > 0 && (src == nullptr || dst == nullptr || !aligned(src, 16) || !aligned(dst, 16)))
        return fail(EFS_EINVAL, "efs_copy_probe: src and dst must be non-NULL and 16-byte aligned");
    return check_launch(efs::launch_copy(src, dst, n, false, static_cast<hipStream_t>(stream)),
                        "efs_copy_probe");
}

efs_status efs_stream_probe(const float *x, float *y, int64_t n, int mode, void *stream) {
    if (n < 0 || n > kProbeMaxElements)
        return fail(EFS_EINVAL, "efs_stream_probe: n = %lld outside [0, %lld]", (long long)n,
                    (long long)kProbeMaxElements);
    if (mode < 0 || mode > 7) return fail(EFS_EINVAL, "efs_stream_probe: mode %d outside 0..7", mode);
    const bool per_tile = (mode & 4) != 0;
    mode &= 3;
    if (n > 0 && (x == nullptr || y == nullptr || !aligned(x, 16) || !aligned(y, 16)))
        return fail(EFS_EINVAL, "efs_stream_probe: x and y must be non-NULL and 16-byte aligned");
    if (mode == 0)
        return check_launch(efs::launch_copy(x, y, n, per_tile, static_cast<hipStream_t>(stream)),
                            "efs_stream_probe");
    return check_launch(
        efs::launch_stream_probe(x, y, n, mode, per_tile, static_cast<hipStream_t>(stream)),
        "efs_stream_probe");
}

}  // extern "C"
