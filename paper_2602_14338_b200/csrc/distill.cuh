// The calls of distill.cu with what another loss that is linear in the log-probs of one token per row needs besides: with K = 1, logits
// of zero and no teacher_lse, kl_t is -log p_t,y and dz_tv = grad_scale w_i (p_tv - 1[v = y_t]).
#pragma once

#include "common.cuh"

struct AeroListed {
  const float* z_gain = nullptr;        // bf16 rows: log-probs with lmhead::Params::z_gain [T]
  // K = 1, every row of the kept rollouts with a token in [0,V): its logit, an fp32 dot product [T], and the rows' weights [T] in place
  // of w; the passes that make these (and the outputs of rows that no kept rollout owns) are left out.
  const float* z = nullptr;
  const float* row_weights = nullptr;
  // bf16 rows: factors of the rows' gradients that are left out of dz [T], on top of the weights.  They go on the finished rows of dH and,
  // rounded once, on the rows of H that enter dW: with one listed token per row the largest entry of dz is close to its weight,
  // and one weight for all tokens of a rollout would be rounded with the same error in all of them.
  const float* row_factor = nullptr;
  // One-call step whose rows fit one chunk: called when the rows' log-probs are there and before the factors are used, to write
  // these on the context's stream.
  int (*between)(void* arg) = nullptr;
  void* arg = nullptr;
};

// (loss may be NULL: not wanted)
int aero_distill_fwd_listed(const AeroListed& ex, aero_ctx* ctx, const aero_cfg* cfg, int64_t T, int32_t d, int32_t V,
                            int32_t R, int32_t K, const void* H, const void* W, const int32_t* ids, const float* logits,
                            const float* teacher_lse, const int64_t* cs, const float* w, const uint8_t* keep, float* lse,
                            float* kl, float* loss, float* metrics, void* workspace, size_t workspace_bytes);
int aero_distill_bwd_listed(const AeroListed& ex, aero_ctx* ctx, const aero_cfg* cfg, int64_t T, int32_t d, int32_t V,
                            int32_t R, int32_t K, const void* H, const void* W, const int32_t* ids, const float* logits,
                            const float* teacher_lse, const int64_t* cs, const float* w, const uint8_t* keep,
                            const float* lse, float grad_scale, void* dH, void* dW, int32_t dw_dtype, int accumulate_dW,
                            void* workspace, size_t workspace_bytes);
int aero_distill_fwd_bwd_listed(const AeroListed& ex, aero_ctx* ctx, const aero_cfg* cfg, int64_t T, int32_t d, int32_t V,
                                int32_t R, int32_t K, const void* H, const void* W, const int32_t* ids, const float* logits,
                                const float* teacher_lse, const int64_t* cs, const float* w, const uint8_t* keep, float* lse,
                                float* kl, float* loss, float* metrics, float grad_scale, void* dH, void* dW,
                                int32_t dw_dtype, int accumulate_dW, void* workspace, size_t workspace_bytes);

// The calls' argument checks alone.
int aero_distill_check(aero_ctx* ctx, const aero_cfg* cfg, int64_t T, int32_t d, int32_t V, int32_t R, int32_t K, const void* H,
                       const void* W, const int32_t* ids, const float* logits, const int64_t* cs, const float* w, const uint8_t* keep,
                       const void* workspace);
int aero_distill_check_grads(const aero_cfg* cfg, int64_t T, const void* dH, const void* dW, int32_t dw_dtype, int accumulate_dW);

// Whether the backward can run in so much workspace.
bool aero_distill_bwd_fits(const aero_cfg* cfg, int64_t T, int32_t d, int32_t V, int32_t R, int32_t K, int32_t dw_dtype,
                           size_t workspace_bytes);

// Whether a one-call step with so much workspace takes all rows in one chunk.
bool aero_distill_one_chunk(const aero_ctx* ctx, int64_t T, int32_t d, int32_t V, int32_t R, int32_t K, int32_t dw_dtype,
                            size_t workspace_bytes);
