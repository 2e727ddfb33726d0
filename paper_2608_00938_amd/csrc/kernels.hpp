// Internal launchers of the gfx950 kernels; the C ABI in grace_api.hip calls
// them after validating every argument.  Each returns the launch's HIP status.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/grace.h"

namespace grace {

// launch(first, count) for workgroups first .. first + count - 1 until all are under
// way: one launch takes fewer than 2^32 threads, 2^22 of the largest workgroups.
template <class F>
hipError_t launch_in_parts(int64_t workgroups, F launch) {
  constexpr int64_t kMost = (int64_t)1 << 21;
  for (int64_t first = 0; first < workgroups; first += kMost) {
    launch((uint32_t)first, (uint32_t)(workgroups - first < kMost ? workgroups - first : kMost));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Cross-attention, beam-as-query: grid over (request, head, beam tile).
hipError_t launch_cross_attn(const void* q, const void* enc_k, const void* enc_v,
                             const int32_t* enc_off, void* out, int32_t B, int32_t M, int32_t H,
                             int32_t d, int32_t sum_L, float scale, bool bf16, hipStream_t stream);

// Paged rearrangement + append.  k_slab/v_slab point at slab `step` of the pools.
hipError_t launch_kv_append(void* k_slab, void* v_slab, const int32_t* table_prev,
                            int32_t* table_next, const int32_t* parents, const void* k_new,
                            const void* v_new, int32_t R, int32_t M, int32_t T_max, int32_t step,
                            int32_t row_bytes, bool copy_k, bool copy_v, int32_t* err_flag,
                            hipStream_t stream);

// Paged self-attention over step+1 tokens.
hipError_t launch_self_attn_step(const void* q, const void* k_pool, const void* v_pool,
                                 const int32_t* table, void* out, int32_t R, int32_t H, int32_t d,
                                 int32_t T_max, int32_t step, float scale, bool bf16,
                                 hipStream_t stream);

// Fused append + attend: table update, slab write (unless aliased) and
// self-attention over step+1 tokens in one pass.  R = B*M rows this step,
// parents index B*M_prev previous rows, pool slabs have row stride R_s.
hipError_t launch_self_attn_fused(const void* q, const void* k_new, const void* v_new,
                                  void* k_pool, void* v_pool, const int32_t* table_prev,
                                  int32_t* table_next, const int32_t* parents, void* out, int32_t R,
                                  int32_t M, int32_t M_prev, int32_t R_s, int32_t H, int32_t d,
                                  int32_t T_max, int32_t step, float scale, bool bf16, bool copy_k,
                                  bool copy_v, int32_t* err_flag, hipStream_t stream);

// Beam candidate scores: prev[r] + log_softmax(logits[r]), -inf where filtered.
hipError_t launch_beam_scores(const void* logits, const float* prev, const uint32_t* mask,
                              float* cand, float* row_max, int32_t R, int32_t V, bool bf16,
                              hipStream_t stream);

// Per-request top-k over M*V candidates; k <= beam_topk_max_k(); workspace of
// beam_topk_workspace_bytes(B, M, V) bytes, 8-byte aligned.
hipError_t launch_beam_topk(const float* cand, const float* row_max, int32_t B, int32_t M,
                            int32_t V, int32_t k, void* workspace, int32_t* parents,
                            int32_t* tokens, float* scores, hipStream_t stream);
size_t beam_topk_workspace_bytes(int32_t B, int32_t M, int32_t V);
int32_t beam_topk_max_k();

// Score update and top-k in one: the same outputs as launch_beam_scores then
// launch_beam_topk, with the candidates recomputed from the logits instead of
// written out; workspace of beam_step_workspace_bytes(B, M, V) bytes.
hipError_t launch_beam_step(const void* logits, const float* prev, const uint32_t* mask,
                            int32_t B, int32_t M, int32_t V, int32_t k, bool bf16, void* workspace,
                            int32_t* parents, int32_t* tokens, float* scores, hipStream_t stream);
size_t beam_step_workspace_bytes(int32_t B, int32_t M, int32_t V);

// CD + GTM filter words of every beam row; next trie node of every new beam.
hipError_t launch_gtm_mask(const grace_gtm_index& index, const grace_gtm_user& user,
                           const int32_t* node_ids, int32_t R, int32_t M, uint32_t* mask,
                           int32_t* err_flag, hipStream_t stream);
hipError_t launch_trie_advance(const grace_gtm_index& index, const int32_t* node_prev,
                               const int32_t* parents, const int32_t* tokens, int32_t B,
                               int32_t M_prev, int32_t k, int32_t* node_next, int32_t* err_flag,
                               hipStream_t stream);

// Norm of R rows of D elements (D <= rms_norm_max_d()): h = x + residual (residual
// may be null), sum = h if not null, out = h / rms(h) * weight in out_dtype, with
// a scale per row for GRACE_E4M3.
hipError_t launch_rms_norm(const void* x, const void* residual, const void* weight, int32_t R,
                           int32_t D, float eps, int32_t dtype, int32_t out_dtype, void* sum,
                           void* out, float* out_scale, hipStream_t stream);
int32_t rms_norm_max_d();

// out [R, N] = act(x_scale w_scale x w^T + bias) + residual, x [R, K] and w [N, K]
// in dtype, bias, residual and out in out_dtype; scales, bias and residual may be
// null; residual may be out itself.
hipError_t launch_linear(const void* x, const float* x_scale, const void* w, const float* w_scale,
                         const void* bias, const void* residual, int32_t R, int32_t N, int32_t K,
                         int32_t act, int32_t dtype, int32_t out_dtype, void* out,
                         hipStream_t stream);

// A token of every row by temperature, top-k, top-p and min-p (each per request, or
// null), and prev (or 0) + its log-probability.
hipError_t launch_sample(const void* logits, const float* uniform, const float* prev,
                         const uint32_t* mask, const float* temperature, const int32_t* top_k,
                         const float* top_p, const float* min_p, int32_t B, int32_t M, int32_t V,
                         bool bf16, int32_t* tokens, float* scores, hipStream_t stream);

// Debug builds: add the device-check counters of the attention kernels' source
// files to acc[0 .. 7] and clear them (synchronous); release builds return
// hipErrorNotSupported.
hipError_t debug_take_cross(uint32_t* acc);
hipError_t debug_take_self(uint32_t* acc);

}  // namespace grace
