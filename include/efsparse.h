/*
 * efsparse — error-feedback gradient sparsification on MI355X (gfx950).
 *
 * C ABI of libefsparse.so.  Implements the per-worker compression step of
 * "Rethinking gradient sparsification as total error minimization"
 * (arXiv 2108.00951), Algorithm 1 (distributed EF SGD):
 *
 *     p      = e + lr * g                 EF accumulate
 *     Delta  = C(p)                       compress (hard threshold or Top-k)
 *     e'     = p - Delta                  error update
 *     avg    = (1/n) sum_i Delta_i        exchange and average
 *
 * Conventions shared by every entry point
 *   - Every array argument is a DEVICE pointer owned by the caller; the
 *     library never allocates, frees or synchronises.  Work is enqueued on
 *     `stream` (a hipStream_t; NULL means the legacy default stream) and is
 *     complete only when that stream is.
 *   - Arguments are validated on the host before anything is enqueued.  On a
 *     non-OK status nothing was enqueued, except EFS_EHIP, which reports a
 *     launch failure (kernels launched before it stay enqueued).
 *     efs_last_error_message() then describes the failure (per thread).
 *   - Arithmetic is IEEE binary32 with round to nearest even; the accumulate
 *     is a multiply followed by a separately rounded add (never fused);
 *     subnormals are kept.
 *   - Indices are 0-based int32; d must not exceed INT32_MAX.
 *   - Payload pair order is unspecified (consumers must not rely on it).
 *     Payload values are the kept entries of p, unscaled.
 */
#ifndef EFSPARSE_H
#define EFSPARSE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum efs_status {
    EFS_OK = 0,
    EFS_EINVAL = 1,   /* an argument failed validation; nothing enqueued      */
    EFS_ESPACE = 2,   /* workspace smaller than the query said; nothing enqueued */
    EFS_EHIP = 3      /* the HIP runtime rejected a launch                      */
} efs_status;

/* A counter object: EFS_COUNTER_WORDS uint32 words (16 bytes) of device
 * memory, 8-byte aligned, zero-filled once by the caller before first use.
 * Word 0 receives the payload count k_t of the last completed call; the
 * other words are the library's and are back at zero whenever no call that
 * uses the object is in flight.  One object must not be used by two calls
 * that may run concurrently. */
#define EFS_COUNTER_WORDS 4

/* Hard-threshold sparsifier with error feedback (Algorithm 1 with the
 * hard-threshold compressor C_lambda of section 4.2:
 * S_lambda(p) = { i : |p_i| >= lambda }).
 *
 *   g        [d] fp32, read only: the stochastic gradient g_t.
 *   e        [d] fp32, in place: e_t on entry, e_{t+1} on completion
 *            (+0.0f at kept coordinates, p_i elsewhere).  Must not overlap g
 *            or the payload.
 *   d        vector length, 0 <= d <= INT32_MAX.
 *   lr       step size gamma (finite).
 *   lambda   threshold in the units of p (lambda >= 0, not NaN; +inf keeps
 *            nothing).  Algorithm 1 writes the compressor as gamma*C(p/gamma);
 *            for the threshold of C in those units pass gamma*lambda here.
 *   idx,val  [cap] payload (int32 index, fp32 value p_i), unordered; only the
 *            first min(k_t, cap) slots are written.  May be NULL when cap == 0.
 *   cap      payload capacity, >= 0.
 *   counter  counter object (see above); word 0 receives k_t, the TRUE
 *            count even when it exceeds cap (then the payload is truncated
 *            and must be treated as invalid; e' is complete regardless).
 * Pointers g and e must be 4-byte aligned.  NaN entries of p are never kept. */
efs_status ht_compress(const float *g, float *e, int64_t d, float lr, float lambda,
                       int32_t *idx, float *val, int64_t cap, uint32_t *counter,
                       void *stream);

/* A telemetry object: EFS_TELEMETRY_BYTES of device memory, 8-byte aligned,
 * zero-filled by the caller before the first call; every call adds to it:
 *   double   err2_part[32] partial sums whose total is the sum over calls of
 *                          ||e_{t+1}||^2, the total error of Remark 4
 *                          (section 3) when the calls are the iterations
 *                          t = 0..T-1 (sum the 32 values to read it);
 *   double   sent_total    sum over calls of k_t (average density =
 *                          sent_total / (calls * d), the measure of data
 *                          volume used in section 6);
 *   uint32_t max_abs_bits  running max of |e_{t+1}| as the bit pattern of a
 *                          non-negative float (the hard threshold keeps it
 *                          below lambda: the absolute-compressor bound of
 *                          section 5);
 *   uint32_t calls         number of calls accumulated;
 *   16 bytes reserved.
 * The norm is summed in binary64, each workgroup adding its share into one
 * of the 32 parts with an atomic (one word for all of them serialises), so
 * its last bits can vary with the order of the additions. */
#define EFS_TELEMETRY_BYTES 288

/* ht_compress, and in the same pass the telemetry above added to
 * `telemetry` (device pointer, see EFS_TELEMETRY_BYTES). */
efs_status ht_compress_telemetry(const float *g, float *e, int64_t d, float lr, float lambda,
                                 int32_t *idx, float *val, int64_t cap, uint32_t *counter,
                                 void *telemetry, void *stream);

/* Bytes of device workspace topk_compress needs for (d, k). */
size_t topk_workspace_bytes(int64_t d, int64_t k);

/* Top-k sparsifier with error feedback (Algorithm 1 with Top-k, the
 * per-iteration optimum of Lemma 2): keeps the k coordinates of largest |p|.
 * Magnitudes are ranked by the bit pattern of |p| (so -0 and +0 tie, NaN
 * ranks above +inf); equal magnitudes go to the lower index.
 *
 *   g, e, d, lr   as for ht_compress.
 *   k             0 <= k <= d.
 *   idx, val      [k] payload of exactly k pairs (unordered).
 *   workspace     device memory of at least topk_workspace_bytes(d, k)
 *                 bytes, 16-byte aligned; contents need no initialisation.
 *                 The library keeps the last three thresholds in it and how
 *                 far its predictions were off: a following call on the same
 *                 workspace whose k-th magnitude lies near the predicted one
 *                 (the error-feedback case; within 6 to 12 % at most) selects
 *                 from a small candidate set instead of two more passes over p.
 *                 Results never depend on what the workspace held.  Not
 *                 shareable between concurrent calls.
 */
efs_status topk_compress(const float *g, float *e, int64_t d, float lr, int64_t k,
                         int32_t *idx, float *val, void *workspace,
                         size_t workspace_bytes, void *stream);

/* Byte offset, within a Top-k workspace, of a uint32 that is 1 after a call
 * that selected from the candidate set around the previous threshold and 0
 * after one that ran the full radix select (a diagnostic; read it after the
 * call has completed). */
size_t topk_path_flag_offset(void);

/* Layer-wise Top-k EF step (Appendix C.5: the sparsifier applied to each
 * layer's tensor on its own; Algorithm 1 for the error):
 *     p = e + lr*g ;  in every segment s = [offsets[s], offsets[s+1]) keep the
 *     min(k[s], size_s) entries of largest |p| (equal magnitudes: lower index
 *     first, as topk_compress ranks them) ;  e' = p with +0 at every kept entry.
 *
 *   g, e        as for topk_compress (e in/out, in place).
 *   nseg        number of segments, 1 <= nseg <= EFS_SEG_MAX.
 *   offsets     DEVICE int64[nseg + 1], 8-byte aligned: offsets[0] = 0,
 *               non-decreasing, offsets[nseg] = d (empty segments allowed).
 *   k           DEVICE int64[nseg], 8-byte aligned: k[s] >= 0; values above
 *               a segment's size keep the whole segment.
 *   k_total     capacity of idx/val; must be >= sum of min(k[s], size_s).
 *   idx, val    payload: segment s's pairs occupy
 *               [kout_s, kout_s + min(k[s], size_s)), kout the exclusive
 *               prefix of those counts; order within a segment unspecified.
 *   workspace   >= topk_segmented_workspace_bytes(nseg, k_total) bytes,
 *               16-byte aligned: per-segment tables and histograms (36 KiB per
 *               segment), a candidate region of 16*k_total + 4096*nseg
 *               (key, index) pairs, a work list of one 8-byte entry per
 *               512 of those pairs or payload slots, and 32 KiB of flags
 *               over groups of tiles.  Results never depend on its contents.
 *               Not shareable between concurrent calls.
 * Host-visible arguments are checked before anything is launched (EFS_EINVAL,
 * EFS_ESPACE).  offsets and k live on the device and are checked there: a
 * layout that breaks the rules above, or a k_total below the sum, makes the
 * call change nothing (no payload written, e untouched) and leaves the uint32
 * at topk_segmented_status_offset() in the workspace at 1 (0 after an
 * accepted call).  d == 0 is a no-op. */
#define EFS_SEG_MAX 65536
size_t topk_segmented_workspace_bytes(int32_t nseg, int64_t k_total);
size_t topk_segmented_status_offset(void);

/* Byte offset, within a layer-wise Top-k workspace, of a uint32 counting the
 * segments of the last completed call that selected among the keys in a
 * bracket around the threshold predicted from that segment's earlier calls
 * (instead of the full radix select; a diagnostic, read after the call has
 * completed). */
size_t topk_segmented_bracket_offset(void);
efs_status topk_segmented_compress(const float *g, float *e, int64_t d, float lr, int32_t nseg,
                                   const int64_t *offsets, const int64_t *k, int64_t k_total,
                                   int32_t *idx, float *val, void *workspace,
                                   size_t workspace_bytes, void *stream);

/* Exchange-and-average of n workers' payloads on one device (Algorithm 1:
 * the average (1/n) sum_i Delta_i of the compressed updates; App. C.6.2,
 * Algorithm 2: DECOMPRESS then AGGREGATE):
 *     out = (sum over w = 0..n-1, in that order, of decompress(payload_w)) / n
 * with fp32 adds in worker order and one IEEE division by (float)n at every
 * coordinate (untouched coordinates are +0).
 *
 *   idx, val   HOST arrays of n_workers device pointers; payload w has
 *              indices idx[w][0..c_w) (distinct within one payload) and
 *              values val[w][0..c_w).
 *   counts     HOST array of n_workers device pointers to the uint32 count of
 *              each payload (word 0 of ht_compress's counter object, which
 *              stays on the device), or NULL entries / a NULL array meaning
 *              c_w = caps[w].
 *   caps       HOST array of n_workers capacities; c_w = min(*counts[w],
 *              caps[w]).  A count above its capacity (a truncated
 *              hard-threshold payload) is averaged over its caps[w] pairs and
 *              reported in the status word (EFS_SPARSE_TRUNCATED).
 *   n_workers  1 <= n_workers <= EFS_MAX_WORKERS; sum of caps <= 2^32 - 1.
 *   d          length of out; d == 0 is a no-op.
 *   out        [d] fp32, 16-byte aligned, overwritten.
 *   workspace  device memory, 16-byte aligned, in one of two layouts chosen
 *              by workspace_bytes:
 *                bucketed, when workspace_bytes >=
 *                sparse_bucket_workspace_bytes(n_workers, d) (about 8 n d
 *                bytes): a 256-byte control block, an 8-byte counter per
 *                (range of 4096 coordinates, worker) and a bucket of 4096
 *                8-byte slots per counter.  Two launches.
 *                packed, otherwise; needs at least
 *                sparse_accumulate_workspace_bytes(n_workers, d, sum of caps)
 *                bytes: the control block, an 8-byte counter and a 4-byte
 *                segment start per (range, worker), and 8 bytes per payload
 *                slot for the pairs grouped by range.  Four launches.
 *              Both give the same bits.  (sparse_apply's EFS_APPLY_SGD with
 *              one payload uses neither: one launch, and words of the control
 *              block with an epoch of their own.)  Contents need no
 *              initialisation: each counter carries a 40-bit tag of the epoch
 *              of the call that wrote it (the control block's epoch, advanced by
 *              every call that uses the counters), so a counter of an earlier
 *              call reads as zero, also where a call of another layout or other
 *              sizes has overwritten half of it since, as does arbitrary content
 *              except when its tag bits equal the current tag (probability 2^-40
 *              per counter for random bytes).  Calls on one workspace must be
 *              ordered (one stream, or synchronised streams); concurrent
 *              calls on one workspace race.
 * Payload entries with an index outside [0, d) are skipped and reported in
 * the status word (EFS_SPARSE_BAD_INDEX).  The status word is the uint32 at
 * sparse_status_offset() in the workspace: the EFS_SPARSE_* bits of the last
 * completed call (0: every payload was whole and in range).  The counts are
 * read on the device, so these are reported there and not as an efs_status. */
#define EFS_MAX_WORKERS 64
#define EFS_SPARSE_TRUNCATED 1u
#define EFS_SPARSE_BAD_INDEX 2u
/* Bytes of the packed and of the bucketed workspace layout; 0 if the
 * arguments are out of range. */
size_t sparse_accumulate_workspace_bytes(int32_t n_workers, int64_t d, int64_t total_cap);
size_t sparse_bucket_workspace_bytes(int32_t n_workers, int64_t d);
size_t sparse_status_offset(void);
efs_status sparse_accumulate(const int32_t *const *idx, const float *const *val,
                             const uint32_t *const *counts, const int64_t *caps,
                             int32_t n_workers, int64_t d, float *out, void *workspace,
                             size_t workspace_bytes, void *stream);

/* sparse_accumulate for callers that cannot allocate device memory (code
 * under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc): the same operation with the same bits, the pairs grouped in a
 * scratch array of EFS_STATIC_SCRATCH_BYTES that the library holds on each
 * device it runs on (from the library's first use of that device until the
 * process ends) instead of in a caller's workspace.  The call allocates
 * nothing.
 *
 *   idx, val, counts, caps, n_workers, d, out, stream
 *              as for sparse_accumulate.
 * Returns EFS_ESPACE, with nothing launched, when the payloads need more
 * than EFS_STATIC_SCRATCH_BYTES: the bucketed layout is used when
 * sparse_bucket_workspace_bytes(n_workers, d) fits in the scratch, else the
 * packed one, which needs sparse_accumulate_workspace_bytes(n_workers, d,
 * sum of caps).  EFS_EINVAL on any other invalid argument, EFS_EHIP if the
 * scratch cannot be found on the current device.  Every call on one device
 * shares that device's scratch; nothing in it needs clearing between calls
 * (its counters carry epoch tags), but calls that overlap on one device
 * (from concurrent streams or host threads) race and must be ordered by the
 * caller.  The status word of these calls stays in the scratch and is not
 * reported. */
#define EFS_STATIC_SCRATCH_BYTES ((size_t)64 << 20)
efs_status sparse_accumulate_static(const int32_t *const *idx, const float *const *val,
                                    const uint32_t *const *counts, const int64_t *caps,
                                    int32_t n_workers, int64_t d, float *out, void *stream);

/* Exchange-and-average fused with the model update that follows it.
 *
 *   avg = (sum over w = 0..n-1, in that order, of decompress(payload_w)) / n
 * exactly as sparse_accumulate computes it (fp32 adds in worker order, one
 * IEEE division by (float)n), then, by mode:
 *   EFS_APPLY_AVERAGE   x = avg at every coordinate (x is the output; the
 *                       same call as sparse_accumulate).
 *   EFS_APPLY_SGD       x = x - avg (Algorithm 1, model update).  Only
 *                       coordinates that some payload touches are written;
 *                       the others keep x, which equals x - (+0) for every
 *                       value except a signalling NaN.
 *   EFS_APPLY_MOMENTUM  m = beta*m + avg, then x = x - gamma*(avg + m) with the
 *                       new m, at every coordinate (Appendix C.6.2,
 *                       Algorithm 2: EF SGD with momentum and gradient
 *                       compression; the paper writes the momentum factor
 *                       as lambda and the learning rate as gamma).
 * Every operation is one separately rounded fp32 operation, in the order
 * written (no fused multiply-add).
 *
 *   idx, val, counts, caps, n_workers, d, workspace, status word
 *              as for sparse_accumulate (the same workspace layouts, chosen
 *              the same way).
 *   x          [d] fp32, 16-byte aligned, read and written in place (mode
 *              EFS_APPLY_AVERAGE only writes it).  Must not overlap a payload.
 *   m          [d] fp32 momentum, 16-byte aligned, read and written in place;
 *              used by EFS_APPLY_MOMENTUM only (may be NULL otherwise).
 *   beta, gamma  momentum factor and learning rate (finite); used by
 *              EFS_APPLY_MOMENTUM only.
 * Returns EFS_ESPACE if the workspace is too small, EFS_EINVAL on any other
 * invalid argument; nothing is launched then.  d == 0 is a no-op. */
enum { EFS_APPLY_AVERAGE = 0, EFS_APPLY_SGD = 1, EFS_APPLY_MOMENTUM = 2 };

/* Workspace bytes of sparse_apply's packed layout (the same as
 * sparse_accumulate_workspace_bytes); 0 if the arguments are out of range. */
size_t sparse_apply_workspace_bytes(int32_t n_workers, int64_t d, int64_t total_cap);

efs_status sparse_apply(const int32_t *const *idx, const float *const *val,
                        const uint32_t *const *counts, const int64_t *caps, int32_t n_workers,
                        int64_t d, int mode, float *x, float *m, float beta, float gamma,
                        void *workspace, size_t workspace_bytes, void *stream);

/* Element types of the operators that take more than one. */
enum { EFS_FP32 = 0, EFS_BF16 = 1 };

/* Newton-Schulz orthogonalisation of a batch of matrices: with the singular
 * value decomposition G = U S V^T of one matrix, the result approximates
 * U V^T (the direction that the orthogonalised model update takes,
 * muon_apply).  With X = G / (||G||_F + eps), transposed where it has more
 * rows than columns, `steps` times
 *     A = X X^T ;  B = b A + c A A ;  X = a X + B X
 * and the last X, transposed back.  The norm is summed in binary64.  Whatever the
 * type, matrices of up to 64 rows or columns whose X fits one workgroup's LDS are
 * iterated in binary32.  Others keep 22 bits of every entry of X, A and B, of
 * small entries to 2^-39 (no singular value of X is above 1.99): where eps
 * outweighs the norm so far that the entries of G / (||G||_F + eps) are below
 * 2^-38 they vanish.
 *
 *   g          batch matrices of rows x cols; element (i, r, c) is
 *              g[i * stride_g + r * ld_g + c] (in elements; ld_g >= cols).  Read
 *              only; matrices may overlap (stride_g = 0 repeats one).
 *   out        the same with ld_out, stride_out; matrices must not overlap
 *              each other.  May be g itself (the same pointer, ld and stride):
 *              a matrix of g is not read any more when its result is written.
 *              A batch must not overlap g in any other way; other columns of
 *              the same rows are no overlap (of rows that take turns, past all of
 *              them).
 *   dtype      EFS_FP32 or EFS_BF16, of g and out.
 *   batch, rows, cols   >= 0; rows * cols <= INT32_MAX, batch <=
 *              EFS_MUON_MAX_MATRICES.  0 of any: a call that does nothing.
 *   steps      1..EFS_MUON_MAX_STEPS (5 is usual).
 *   coeffs     HOST float[3] a, b, c (finite), or NULL for 3.4445, -4.7750,
 *              2.0315.  Iterates are held in a form that reaches to singular
 *              values s of 1.99, with |b s^2 + c s^4| below 15, which
 *              coefficients that keep the singular values near 1 stay below;
 *              beyond it they become infinite.
 *   eps        added to the norm (finite, >= 0): a matrix of zeros gives zeros
 *              (with eps = 0 NaN, as 0 / 0).
 *   workspace  >= muon_workspace_bytes for these matrices (16 to 24 bytes an
 *              element, more where an axis is short, since both are padded to 32
 *              values: 1 x 100,000 takes 285), 16-byte aligned;
 *              contents need no initialisation and are not kept.  Must not
 *              overlap the matrices.  Not shareable between concurrent calls.
 * A matrix that holds NaN or infinities gives NaN; the others of the batch
 * are not affected. */
#define EFS_MUON_MAX_MATRICES 65536
#define EFS_MUON_MAX_STEPS 64
/* Bytes for nmat matrices of rows[i] x cols[i] (HOST arrays); 0 if the
 * arguments are out of range. */
size_t muon_workspace_bytes(int32_t nmat, const int32_t *rows, const int32_t *cols);
efs_status muon_orthogonalize(const void *g, int64_t ld_g, int64_t stride_g, void *out,
                              int64_t ld_out, int64_t stride_out, int dtype, int32_t batch,
                              int32_t rows, int32_t cols, int32_t steps, const float *coeffs,
                              float eps, void *workspace, size_t workspace_bytes, void *stream);

/* Model update of a flat vector's weight matrices from the averaged update,
 * orthogonalised matrix by matrix (the update of Algorithm 2, App. C.6.2, with
 * the direction orthogonalised; it takes what sparse_accumulate writes):
 *     m = beta * m + avg ;  u = avg + beta * m (nesterov) or m ;
 *     O = muon_orthogonalize(u) with the default coefficients ;
 *     x = (1 - gamma * decay) * x - gamma * sqrt(max(1, rows / cols)) * O
 * each a separately rounded fp32 operation in the order written.
 *
 *   avg        fp32 vector of d elements, read only.
 *   x, m       fp32 vectors of d elements, in place.  avg, x and m must not
 *              overlap.  Any 4-byte alignment.
 *   d          0..INT32_MAX.
 *   nmat, offsets, rows, cols
 *              HOST arrays: matrix i is the row-major rows[i] x cols[i] at
 *              offsets[i] of each vector.  In ascending order and not
 *              overlapping; nmat <= EFS_MUON_MAX_MATRICES; empty matrices are
 *              skipped.  Elements outside every matrix keep x and m.
 *   beta, gamma, decay   finite.
 *   nesterov   0 or 1.
 *   steps, eps, workspace   as for muon_orthogonalize (a matrix whose u is zero
 *              only decays). */
efs_status muon_apply(const float *avg, float *x, float *m, int64_t d, int32_t nmat,
                      const int64_t *offsets, const int32_t *rows, const int32_t *cols, float beta,
                      float gamma, float decay, int nesterov, int32_t steps, float eps,
                      void *workspace, size_t workspace_bytes, void *stream);

/* Softmax cross entropy of tokens against a vocabulary: the loss whose
 * gradient a language model's largest matrix sends through the compression.
 * The logits l = h w^T are never kept: tiles of them are formed, reduced and
 * dropped.
 *     lse[t]  = log(sum over v of exp(l[t, v]))
 *     loss[t] = lse[t] - l[t, target[t]]
 *
 *   h          tokens x hidden hidden states, row t at h + t * ld_h elements.
 *   w          vocab x hidden output head, row v at w + v * ld_w.
 *   target     DEVICE int64[tokens], 8-byte aligned.  A token whose target is
 *              ignore_index does not count: its loss and lse are 0, and its row
 *              of h may hold anything.  So does, with EFS_XENT_BAD_TARGET in the
 *              status word, one whose target is neither that nor in [0, vocab).
 *   dtype      EFS_FP32 or EFS_BF16, of h and w.  fp32: up to 64 tokens
 *              (xent_forward: 128) products of fp32.  With more, 22 bits of every
 *              element count, of those below 2^-17 of the tensor's largest finite
 *              magnitude to 2^-39 of that.  bf16: the logits are exact products;
 *              above 64 tokens the gradients take w and dloss h in 11 bits, of
 *              small elements to 2^-39 of the largest.  All sums are fp32.
 *   tokens     0..EFS_XENT_MAX_TOKENS (0: nothing to do but to clear the status
 *              word, where a workspace is given); vocab
 *              1..EFS_XENT_MAX_VOCAB; hidden 1..EFS_XENT_MAX_HIDDEN; tokens x
 *              vocab at most 2^38.
 *   loss, lse  fp32[tokens], overwritten.  They and the workspace must not
 *              overlap each other or an input.
 *   workspace  >= xent_workspace_bytes(tokens, vocab, hidden, dtype, 0) bytes,
 *              16-byte aligned; contents need no initialisation.  Up to 64
 *              tokens (xent_forward of fp32: 128) h and w are read where they
 *              are.  With more, the bytes hold a copy of both, which bf16 rows
 *              that are multiples of 64 long and 16-byte aligned do without.
 *              Not shareable between concurrent calls.
 * A row of h that holds NaN or infinities gives NaN or infinities for its token
 * alone (and NaN in all of dw); w has to be finite. */
#define EFS_XENT_MAX_TOKENS (1 << 22)
#define EFS_XENT_MAX_VOCAB (1 << 24)
#define EFS_XENT_MAX_HIDDEN (1 << 18)
#define EFS_XENT_BAD_TARGET 1u
/* Bytes for xent_forward (gradient = 0) or both calls (1); 0 if the arguments
 * are out of range. */
size_t xent_workspace_bytes(int32_t tokens, int32_t vocab, int32_t hidden, int dtype, int gradient);
/* Byte offset, in that workspace, of a uint32 with the EFS_XENT_* bits of the
 * last completed call (read it after the call has completed). */
size_t xent_status_offset(void);
efs_status xent_forward(const void *h, int64_t ld_h, const void *w, int64_t ld_w,
                        const int64_t *target, int dtype, int32_t tokens, int32_t vocab,
                        int32_t hidden, int64_t ignore_index, float *loss, float *lse,
                        void *workspace, size_t workspace_bytes, void *stream);

/* Gradients of the sum over t of dloss[t] * loss[t]:
 *     g[t, v] = dloss[t] * (exp(l[t, v] - lse[t]) - [v == target[t]])
 *     dh = g w ;  dw = g^T h
 * The logits are formed again, a piece of the vocabulary at a time.  Up to 64
 * tokens g is held in fp32 (bf16: in 16 bits).  Above, g / dloss is held in 22
 * bits (bf16: 11), of small elements to 2^-32 of the largest of the word for
 * dw, whatever its size, and to 2^-40 for dh, of which p - 1 at the target loses
 * more.
 *
 *   h .. ignore_index   as for xent_forward.
 *   lse        fp32[tokens] as xent_forward left it.
 *   dloss      fp32[tokens]: 1 / (tokens that count) for their mean.  Not used
 *              where the token does not count.
 *   dh, dw     tokens x hidden and vocab x hidden of dtype, rows ld_dh and
 *              ld_dw elements apart, overwritten (dh is 0 where a token does
 *              not count; dw is 0 with no tokens).  They and the workspace must
 *              not overlap each other or an input (other columns of the same rows
 *              are no overlap).  bf16: each result is rounded once more.
 *   workspace  >= xent_workspace_bytes(.., 1). */
efs_status xent_backward(const void *h, int64_t ld_h, const void *w, int64_t ld_w,
                         const int64_t *target, int dtype, int32_t tokens, int32_t vocab,
                         int32_t hidden, int64_t ignore_index, const float *lse,
                         const float *dloss, void *dh, int64_t ld_dh, void *dw, int64_t ld_dw,
                         void *workspace, size_t workspace_bytes, void *stream);

/* Words' vectors: out[t] = scale * table[ids[t]], the start of a language model.
 *
 *   table      vocab x width, row v at table + v * ld_table elements, read only.
 *   ids        DEVICE int64[tokens], 8-byte aligned.  A token whose id is
 *              ignore_index does not count: its row of out is 0.  So is, with
 *              EFS_EMBED_BAD_ID in the status word, that of an id which is
 *              neither ignore_index nor in [0, vocab).
 *   out        tokens x width, rows ld_out elements apart, overwritten; must not
 *              overlap table, ids or status.
 *   dtype, table_dtype   EFS_FP32 or EFS_BF16, of out and of table.
 *   tokens     0..EFS_EMBED_MAX_TOKENS; vocab 1..EFS_EMBED_MAX_VOCAB; width
 *              1..EFS_EMBED_MAX_WIDTH.
 *   scale      finite; the product is one fp32 operation, rounded once more for
 *              bf16.
 *   status     DEVICE uint32, 4-byte aligned, zero-filled by the caller before its
 *              first use, or NULL: calls that meet a bad id set bits in it, and
 *              no call clears it. */
#define EFS_EMBED_MAX_TOKENS (1 << 22)
#define EFS_EMBED_MAX_VOCAB (1 << 24)
#define EFS_EMBED_MAX_WIDTH (1 << 18)
#define EFS_EMBED_BAD_ID 1u
efs_status embed_forward(const void *table, int64_t ld_table, int table_dtype, const int64_t *ids, void *out,
                         int64_t ld_out, int dtype, int32_t tokens, int32_t vocab, int32_t width, float scale,
                         int64_t ignore_index, uint32_t *status, void *stream);

/* Gradient of the table:
 *     dtable[v] = scale * sum over the tokens t with ids[t] = v of dout[t]
 * and 0 for words without a token that counts.  The sums are fp32, always in
 * the same order: a call on the same inputs gives the same bits.
 *
 *   dout       tokens x width of dtype, rows ld_dout elements apart, read only.
 *              Rows of tokens that do not count are not read.
 *   dtable     vocab x width of table_dtype, rows ld_dtable elements apart: a
 *              layer of the flat gradient vector, say.
 *   accumulate 0: every row is overwritten.  1: the rows of words with a token
 *              have their sum added (one fp32 addition, rounded once more for
 *              bf16), others keep what they hold: an output head that shares its
 *              weights, after xent_backward.
 *   ids, status, scale, ignore_index, limits   as for embed_forward; tokens x
 *              vocab at most 2^38.
 *   workspace  >= embed_workspace_bytes(tokens, vocab, width) bytes, 16-byte
 *              aligned; contents need no initialisation and are not kept.  Not
 *              shareable between concurrent calls.
 * dtable, status and the workspace must not overlap each other or an input
 * (other columns of the same rows are no overlap). */
/* Bytes; 0 if the arguments are out of range. */
size_t embed_workspace_bytes(int32_t tokens, int32_t vocab, int32_t width);
efs_status embed_backward(const void *dout, int64_t ld_dout, int dtype, const int64_t *ids, void *dtable,
                          int64_t ld_dtable, int table_dtype, int32_t tokens, int32_t vocab, int32_t width,
                          float scale, int64_t ignore_index, int accumulate, uint32_t *status, void *workspace,
                          size_t workspace_bytes, void *stream);

/* Layer norm of every row of x:
 *     mean = sum(x) / width ;  rstd = 1 / sqrt(sum((x - mean)^2) / width + eps)
 *     y = (x - mean) * rstd * weight + bias
 * in fp32; bf16 results are rounded once.
 *
 *   x, y       rows x width of dtype, rows ld_x and ld_y elements apart.  y may be
 *              x itself (the same pointer and ld); it must not overlap x in any
 *              other way (other columns of the same rows are no overlap), nor
 *              anything else.
 *   weight, bias   [width] of weight_dtype, aligned to it; NULL: 1 and 0.
 *   dtype, weight_dtype   EFS_FP32 or EFS_BF16.
 *   rows       0..INT32_MAX; width 1..EFS_NORM_MAX_WIDTH.
 *   eps        finite, >= 0 (a constant row gives bias; with eps = 0 NaN).
 *   mean, rstd fp32[rows], overwritten, for the gradients; each may be NULL.
 * A row that holds NaN or infinities, or whose sum or sum of squares passes
 * fp32's range, gives NaN or zeros; the others are not affected (in the gradients:
 * dweight and dbias take it in). */
#define EFS_NORM_MAX_WIDTH (1 << 18)
efs_status layernorm_forward(const void *x, int64_t ld_x, const void *weight, const void *bias, void *y,
                             int64_t ld_y, int dtype, int weight_dtype, int32_t rows, int32_t width, float eps,
                             float *mean, float *rstd, void *stream);

/* Its gradients, with g = dy * weight and h = (x - mean) * rstd:
 *     dx = rstd * (g - sum(g) / width - h * sum(g * h) / width)     (of its row)
 *     dweight = sum over the rows of dy * h ;  dbias = sum over the rows of dy
 * Sums are fp32, always in the same order.
 *
 *   x, weight, dtype, weight_dtype, rows, width   as for layernorm_forward.
 *   mean, rstd fp32[rows] as layernorm_forward left them.
 *   dy         rows x width of dtype, rows ld_dy elements apart.
 *   dx         the same with ld_dx, overwritten.  May be dy or x itself (the
 *              same pointer and ld).
 *   dweight, dbias   [width] of weight_dtype, overwritten (0 with no rows); each may
 *              be NULL.
 *   workspace  >= layernorm_workspace_bytes(rows, width) bytes, 16-byte aligned;
 *              contents need no initialisation and are not kept.  Not shareable
 *              between concurrent calls.
 * What is written must not overlap anything else. */
/* Bytes; 0 if the arguments are out of range. */
size_t layernorm_workspace_bytes(int32_t rows, int32_t width);
efs_status layernorm_backward(const void *x, int64_t ld_x, const void *weight, const float *mean, const float *rstd,
                              const void *dy, int64_t ld_dy, void *dx, int64_t ld_dx, int dtype, int weight_dtype,
                              int32_t rows, int32_t width, void *dweight, void *dbias, void *workspace,
                              size_t workspace_bytes, void *stream);

/* AdamW over many tensors at once: the update of the parameters that muon_apply
 * leaves as they are (norms, biases, embeddings, output heads), from the averaged
 * gradient.  With t the number of the step, from 1 on,
 *     m = beta1 * m + (1 - beta1) * g
 *     v = beta2 * v + ((1 - beta2) * g) * g
 *     x = (1 - gamma * decay) * x - alpha * (m / (root * sqrt(v) + eps))
 *     alpha = gamma / (1 - beta1^t) ;  root = 1 / sqrt(1 - beta2^t)
 * each a separately rounded fp32 operation in the order written; 1 - beta1, 1 -
 * beta2, 1 - gamma * decay, alpha and root are computed in binary64 and rounded.
 *
 *   g, x, m, v, sizes   HOST arrays of `count` device pointers (and lengths, 0 to
 *              INT32_MAX elements): tensors of their own or layers of flat vectors.
 *              g: of grad_dtype, read only; x: fp32, in place; m, v: in place, of
 *              state.  Aligned to their type; states of 8 bits to 16 bytes.
 *   copies     HOST array of device pointers to bf16 that receive the new x
 *              rounded, or NULL (in which entries may be NULL).
 *   decays     HOST float[count] (finite), or NULL for 0.
 *   count      0..EFS_ADAMW_MAX_TENSORS, of which those of length 0 are skipped
 *              (their pointers are not looked at).
 *   state      EFS_STATE_32: m[i] and v[i] are fp32[sizes[i]], zero before the
 *              first step.  EFS_STATE_8: adamw_state_bytes(sizes[i]) bytes each,
 *              zero-filled before the first step; see below.
 *   gamma, beta1, beta2, eps   finite; 0 <= beta < 1, eps >= 0 (with eps = 0 an
 *              element that never had a gradient becomes NaN, as 0 / 0).
 *   step       t >= 1, where step_device is NULL.
 *   step_device   DEVICE int64, 8-byte aligned, with t in it (below 1: as 1), or
 *              NULL: for calls in a captured graph, which the caller advances
 *              between them.
 *   factors    DEVICE float[2], 4-byte aligned, or NULL for 1, 1: gamma is
 *              multiplied by the first (a schedule), every element of g by the
 *              second (one over a loss scale, a clipped norm's factor).
 *   seed       of the random rounding of states of 8 bits.
 * A tensor that is written, its states among them, must not overlap any other,
 * step_device or factors.
 * NaN or infinities in g spoil their own elements alone.
 *
 * States of 8 bits.  256 consecutive elements share a power of two s for m and one
 * for r = sqrt(v): the largest finite magnitude lies in [2^7, 2^8) * s (s is
 * 2^-102 where it is below 2^-95).  m is kept as a sign and a value of 3 bits
 * below its leading one, from 2^-6 s on (smaller: in steps of 2^-9 s); r as one
 * of 4 bits (steps of 2^-10 s), of which no r > 0 becomes 0.  A value between two
 * others is rounded up with the share of its distance from the lower one, by a
 * hash of (seed, the tensor's place in the list, t, element): the same call
 * gives the same bits.  A magnitude that is infinite or NaN is kept as NaN; one
 * that is finite stays so (rounded down where the next m or v is 2^128).  x is
 * computed from m and v before they are rounded.  The state of n elements is
 * ceil(n / 256) * 256 bytes (a byte an element, zeros behind the last), then a
 * float s for each 256. */
#define EFS_ADAMW_MAX_TENSORS 65536
enum { EFS_STATE_32 = 0, EFS_STATE_8 = 1 };
/* Bytes of m (or of v) of `size` elements in 8 bits; 0 if size is out of range. */
size_t adamw_state_bytes(int64_t size);
efs_status adamw_apply(const void *const *g, int grad_dtype, float *const *x, void *const *copies, void *const *m,
                       void *const *v, int state, const int64_t *sizes, const float *decays, int32_t count,
                       float gamma, float beta1, float beta2, float eps, int64_t step, const int64_t *step_device,
                       const float *factors, uint32_t seed, void *stream);

/* States of 8 bits as values and back, for checkpoints: adamw_read_state writes
 * the m and v that m8 and v8 stand for; adamw_write_state is its inverse, rounding
 * to nearest (ties up).  HOST arrays of device pointers as for adamw_apply; m and
 * v fp32.  What is written must not overlap anything else. */
efs_status adamw_read_state(void *const *m8, void *const *v8, float *const *m, float *const *v, const int64_t *sizes,
                            int32_t count, void *stream);
efs_status adamw_write_state(float *const *m, float *const *v, void *const *m8, void *const *v8, const int64_t *sizes,
                             int32_t count, void *stream);

/* Streaming copy dst[0..n) = src[0..n) with the same 16-byte access pattern
 * and grid as the hard-threshold kernel: the reference transfer for
 * measurements, not part of the method.  src and dst 16-byte aligned,
 * 0 <= n <= INT32_MAX * 4096. */
efs_status efs_copy_probe(const float *src, float *dst, int64_t n, void *stream);

/* Streaming bandwidth probes over n floats with the same tile shape as the
 * compression kernels (measurement aids, not part of the method):
 *   mode 0  copy       y = x                (4n bytes read, 4n written)
 *   mode 1  read       sum of x, discarded  (4n read; y[0..255] reserved)
 *   mode 2  write      y = constant         (4n written)
 *   mode 3  2R1W       y = y + 0.5 x        (8n read, 4n written; the
 *                                            access pattern of ht_compress)
 * plus 4: the same traffic with one workgroup per 4096-element tile instead
 * of the hard threshold's persistent grid.  Modes 1-3 (5-7) cover whole
 * 4096-element tiles only.  x and y 16-byte aligned, 0 <= n <=
 * INT32_MAX * 4096; for mode 1 (5), y must hold at least 256 floats.  Other
 * modes: EFS_EINVAL. */
efs_status efs_stream_probe(const float *x, float *y, int64_t n, int mode, void *stream);

/* Static text for a status code. */
const char *efs_status_string(efs_status status);

/* Detail of the last non-OK status returned on the calling thread. */
const char *efs_last_error_message(void);

/* Sticky status for callers that check once after a sequence of calls:
 * EFS_EHIP when the HIP runtime holds an error left by an earlier
 * asynchronous launch on this thread (hipPeekAtLastError, not cleared);
 * otherwise the last non-OK status any call returned on this thread since
 * the previous efs_last_error (which clears it), or EFS_OK.  Conditions
 * that only the device sees are reported on the device: a hard-threshold
 * count above the capacity in the counter object (compare it with cap), a
 * truncated payload or an index out of range in the average's status word. */
efs_status efs_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* EFSPARSE_H */
