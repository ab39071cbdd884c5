// Host-side launchers of the efsparse kernels.  Arguments arrive here
// already validated by the C ABI layer (abi.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace efs {

hipError_t launch_ht(const float *g, float *e, int64_t d, float lr, float lambda,
                     int32_t *idx, float *val, int64_t cap, uint32_t *counter,
                     void *telemetry, hipStream_t stream);

size_t topk_workspace_size(int64_t d, int64_t k);
size_t topk_path_flag_offset();
hipError_t launch_topk(const float *g, float *e, int64_t d, float lr, int64_t k,
                       int32_t *idx, float *val, void *workspace, hipStream_t stream);

// Layer-wise Top-k (topk_seg.hip).
constexpr int32_t kMaxSegments = 1 << 16;
size_t topk_segmented_workspace_size(int32_t nseg, int64_t k_total);
size_t topk_segmented_status_offset();
size_t topk_segmented_bracket_offset();
hipError_t launch_topk_segmented(const float *g, float *e, int64_t d, float lr, int32_t nseg,
                                 const int64_t *offsets, const int64_t *k, int64_t k_total,
                                 int32_t *idx, float *val, void *workspace, hipStream_t stream);

// Exchange-and-average, alone (mode 0) or fused with the model update
// (apply.hip).  Status bits of the last call, at apply_status_offset() in the
// workspace.
constexpr int kMaxApplyWorkers = 64;
constexpr uint32_t kSparseTruncated = 1u;   // a count exceeded its payload's capacity
constexpr uint32_t kSparseBadIndex = 2u;    // an index outside [0, d) was ignored
// Workspace of the packed layout (four launches) and of the bucketed one
// (two launches, taken whenever the workspace holds it).
size_t apply_workspace_size(int32_t n, int64_t d, int64_t total_cap);
size_t apply_bucket_workspace_size(int32_t n, int64_t d);
size_t apply_status_offset();
hipError_t launch_apply(const int32_t *const *idx, const float *const *val,
                        const uint32_t *const *counts, const int64_t *caps, int32_t n,
                        int64_t d, int mode, float *x, float *m, float beta, float gamma,
                        void *workspace, size_t workspace_bytes, hipStream_t stream);

// Scratch held by the library per device for sparse_accumulate_static
// (scratch.hip): its device address on the current device.
constexpr size_t kStaticScratchBytes = size_t(64) << 20;
hipError_t static_scratch(void **ptr);

// Orthogonalised update of weight matrices (muon.hip).  muon_workspace_size
// returns false where the matrices together need more workgroups than a grid
// has; `next` steps through rows and cols (0: all matrices alike).
constexpr int32_t kMuonMaxMatrices = 1 << 16;
constexpr int32_t kMuonMaxSteps = 64;
bool muon_workspace_size(int32_t nmat, const int32_t *rows, const int32_t *cols, int32_t next, size_t *bytes);
hipError_t launch_muon_orthogonalize(const void *g, int64_t ld_g, int64_t stride_g, void *o, int64_t ld_o,
                                     int64_t stride_o, bool bf16, int32_t batch, int32_t rows, int32_t cols,
                                     int steps, const float *coeffs, float eps, void *workspace,
                                     hipStream_t stream);
hipError_t launch_muon_apply(const float *avg, int32_t nmat, const int64_t *offsets, const int32_t *rows,
                             const int32_t *cols, float *x, float *m, float beta, float gamma, float decay,
                             bool nesterov, int steps, const float *coeffs, float eps, void *workspace,
                             hipStream_t stream);

// Softmax cross entropy over a vocabulary and its gradients (xent.hip).
constexpr uint32_t kXentBadTarget = 1u;   // a target neither ignored nor in the vocabulary
constexpr int32_t kXentMaxTokens = 1 << 22, kXentMaxVocab = 1 << 24, kXentMaxHidden = 1 << 18;
size_t xent_workspace_size(int32_t tokens, int32_t vocab, int32_t hidden, bool bf16, bool gradient);
hipError_t launch_xent_clear(void *workspace, hipStream_t stream);
hipError_t launch_xent_forward(const void *h, int64_t ld_h, const void *w, int64_t ld_w, const int64_t *target,
                               bool bf16, int32_t tokens, int32_t vocab, int32_t hidden, int64_t ignore, float *loss,
                               float *lse, void *workspace, hipStream_t stream);
hipError_t launch_xent_backward(const void *h, int64_t ld_h, const void *w, int64_t ld_w, const int64_t *target,
                                bool bf16, int32_t tokens, int32_t vocab, int32_t hidden, int64_t ignore,
                                const float *lse, const float *dloss, void *dh, int64_t ld_dh, void *dw,
                                int64_t ld_dw, void *workspace, hipStream_t stream);

// Words looked up and the gradient of their table (embed.hip).
constexpr uint32_t kEmbedBadId = 1u;   // an id neither ignored nor in the table
constexpr int32_t kEmbedMaxTokens = 1 << 22, kEmbedMaxVocab = 1 << 24, kEmbedMaxWidth = 1 << 18;
hipError_t launch_embed_forward(const void *table, int64_t ld_table, bool table_bf16, const int64_t *ids, void *out,
                                int64_t ld_out, bool bf16, int32_t tokens, int32_t vocab, int32_t width, float scale,
                                int64_t ignore, uint32_t *status, hipStream_t stream);
size_t embed_workspace_size(int32_t tokens, int32_t vocab, int32_t width);
hipError_t launch_embed_backward(const void *dout, int64_t ld_dout, bool bf16, const int64_t *ids, void *dtable,
                                 int64_t ld_dtable, bool table_bf16, int32_t tokens, int32_t vocab, int32_t width,
                                 float scale, int64_t ignore, bool accumulate, uint32_t *status, void *workspace,
                                 hipStream_t stream);

// Layer norm and its gradients (norm.hip).  weight, bias, dweight, dbias, mean
// and rstd of the forward call may be NULL.
constexpr int32_t kNormMaxWidth = 1 << 18;
hipError_t launch_layernorm_forward(const void *x, int64_t ld_x, const void *weight, const void *bias, void *y,
                                    int64_t ld_y, bool bf16, bool weight_bf16, int32_t rows, int32_t width, float eps,
                                    float *mean, float *rstd, hipStream_t stream);
size_t layernorm_workspace_size(int32_t rows, int32_t width);
hipError_t launch_layernorm_backward(const void *x, int64_t ld_x, const void *weight, const float *mean,
                                     const float *rstd, const void *dy, int64_t ld_dy, void *dx, int64_t ld_dx, bool bf16,
                                     bool weight_bf16, int32_t rows, int32_t width, void *dweight, void *dbias,
                                     void *workspace, hipStream_t stream);

// AdamW over a list of tensors (adamw.hip).  Arrays of `count` on the host.
constexpr int32_t kAdamwMaxTensors = 1 << 16;
constexpr int kAdamwBlock = 256;   // elements of an 8-bit state with one scale
struct AdamwArgs {
    const void *const *g;
    float *const *x;
    void *const *m, *const *v, *const *copy;   // copy: may be NULL
    const int64_t *size;
    const float *decay;                        // may be NULL
    int32_t count;
    bool bf16, bytes;                          // of g; states in 8 bits
    float gamma, beta1, beta2, eps;
    int64_t step;
    const int64_t *step_device;                // may be NULL
    const float *factors;                      // may be NULL
    uint32_t seed;
};
hipError_t launch_adamw(const AdamwArgs &args, hipStream_t stream);
size_t adamw_state_size(int64_t size);
// write: the states of 8 bits from m and v; else these from the states.
hipError_t launch_adamw_state(bool write, float *const *m, float *const *v, void *const *m8, void *const *v8,
                              const int64_t *size, int32_t count, hipStream_t stream);

hipError_t launch_copy(const float *src, float *dst, int64_t n, bool per_tile, hipStream_t stream);
hipError_t launch_stream_probe(const float *x, float *y, int64_t n, int mode, bool per_tile,
                               hipStream_t stream);

// Compute units of the current device (queried once per device).
int device_cu_count();

// Grid for a grid-stride pass in which every workgroup stays resident: the
// fewest tiles per workgroup that the resident workgroups allow, and just
// enough workgroups to cover the tiles at that count (so no workgroup does
// more than one tile beyond any other).
uint32_t balanced_grid(int64_t work_tiles, int workgroups_per_cu);

}  // namespace efs
