// The preference loss on pairs of rollouts through the lm_head.  With logp_t the log-prob of token t of rollout i,
//   r_i = sum_t (logp_t - ref_t), or its mean over the scored tokens;   m_p = beta (r_c - r_r) - margin
//   loss = sum_p u_p l(m_p),   coef_i = (sum_{p: c = i} - sum_{p: r = i}) u_p beta l'(m_p) [/ scored tokens of i]
//   dz_tv = grad_scale coef_i (1[v = y_t] - p_tv),   dH = dz W,   dW (+)= dz^T H
// Everything between H, W and the log-probs, and between coef and dH, dW, is distillation's with one listed token per row
// (distill.cuh); what is here are the sums over rollouts and pairs.  The gradient of a row needs all rows of all of its rollout's
// pairs, so the one-call step computes the log-probs of a chunk, then coef, then the chunk's gradients; rows that do not fit
// one chunk of the workspace take the separate passes, which compute the logits twice (8 d V FLOP per token instead of 6).
// The kernels here read 12 bytes per token and 8 bytes per pair and rollout: microseconds beside the products.  All sums are in
// 64 bits and have a fixed order.
#include "distill.cuh"
#include "entry.cuh"
#include "loss_common.cuh"

namespace {

constexpr int kPairBlocks = 148, kThreads = 128;

struct PrefArgs {
  long long T;
  int V, R, P;
  int kind, mean;
  double beta, margin, smoothing;
  const int32_t* y;
  const float* ref;               // NULL: no reference
  const int64_t* cs;
  const int32_t* pairs;           // [P][2]
  const float* weight;            // NULL: 1 / counted pairs
  uint8_t* keep;                  // rollouts in some counted pair
  int* counted;                   // pairs counted
  double* r;                      // [R] log ratios
  int* scored;                    // [R]
  double* slope;                  // [P] d loss / d r_chosen
  double* partials;               // [kPairBlocks][kPartialStride]
  float* logp;                    // in: minus the log-probs
  float* ratio;
  float* margins;
  float* coef;
  float* w;                       // [R] -coef
  float* wrow;                    // [T], or NULL
  uint32_t* status;
};

// A pair that counts: both rollouts exist.  (-1, -1) is an empty place.
__device__ __forceinline__ bool pair_of(const PrefArgs& a, int p, int* c, int* r) {
  *c = a.pairs[2 * (long long)p];
  *r = a.pairs[2 * (long long)p + 1];
  return *c >= 0 && *c < a.R && *r >= 0 && *r < a.R;
}

__global__ void __launch_bounds__(256) pref_mark_kernel(PrefArgs a) {
  int n = 0;
  bool bad = false;
  for (int p = blockIdx.x * 256 + threadIdx.x; p < a.P; p += gridDim.x * 256) {
    int c, r;
    if (pair_of(a, p, &c, &r)) {
      a.keep[c] = 1;
      a.keep[r] = 1;
      ++n;
    } else {
      bad |= c != -1 || r != -1;
    }
  }
  n = __reduce_add_sync(0xffffffffu, n);
  if ((threadIdx.x & 31) == 0 && n) atomicAdd(a.counted, n);
  if (bad) aero_raise(a.status, AERO_ST_BAD_PAIR);
}

// Sum over the block's threads; every thread gets it.
__device__ __forceinline__ double block_sum(double v, double* sh) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  v = sh[0];
  for (int w = 1; w < kThreads / 32; ++w) v += sh[w];
  return v;
}

// Rows a .. b of a rollout, none where its offsets leave [0, T].
__device__ __forceinline__ bool rows_of(const PrefArgs& a, int i, long long* t0, long long* t1) {
  *t0 = a.cs[i];
  *t1 = a.cs[i + 1];
  return *t0 >= 0 && *t1 >= *t0 && *t1 <= a.T;
}

// A block per rollout: its log ratio, and its tokens' log-probs (which arrive negated).
__global__ void __launch_bounds__(kThreads) pref_ratio_kernel(PrefArgs a) {
  __shared__ double sh[kThreads / 32];
  for (int i = blockIdx.x; i < a.R; i += gridDim.x) {
    long long t0, t1;
    double sum = 0.0;
    int n = 0;
    if (!rows_of(a, i, &t0, &t1)) {
      if (threadIdx.x == 0) aero_raise(a.status, AERO_ST_BAD_OFFSETS);
    } else if (a.keep[i]) {
      for (long long t = t0 + threadIdx.x; t < t1; t += kThreads) {
        const float lp = 0.f - a.logp[t];
        const int v = a.y[t];
        a.logp[t] = lp;
        if (v >= 0 && v < a.V) {
          sum += (double)lp - (a.ref ? (double)a.ref[t] : 0.0);
          ++n;
        }
      }
    }
    sum = block_sum(sum, sh);
    n = (int)block_sum((double)n, sh);
    if (threadIdx.x == 0) {
      if (a.mean && n > 0) sum /= n;
      a.r[i] = sum;
      a.scored[i] = n;
      a.ratio[i] = (float)sum;
    }
  }
}

__global__ void __launch_bounds__(kThreads) pref_pairs_kernel(PrefArgs a) {
  __shared__ double sh[kThreads / 32];
  double part[kPartialStride] = {0.0, 0.0, 0.0, 0.0, 0.0};
  const int n = *a.counted;
  for (int p = blockIdx.x * kThreads + threadIdx.x; p < a.P; p += gridDim.x * kThreads) {
    int c, r;
    double slope = 0.0, m = 0.0;
    if (pair_of(a, p, &c, &r)) {
      const double u = a.weight ? (double)a.weight[p] : 1.0 / n, rc = a.r[c], rr = a.r[r];
      m = a.beta * (rc - rr) - a.margin;
      double l;
      if (a.kind == AERO_PREF_LOGISTIC) {
        const double e = exp(-fabs(m)), s = log1p(e);                  // softplus(-|m|)
        const double down = m > 0.0 ? e / (1.0 + e) : 1.0 / (1.0 + e); // sigmoid(-m)
        l = (1.0 - a.smoothing) * (fmax(-m, 0.0) + s) + a.smoothing * (fmax(m, 0.0) + s);
        if (m != m) l = m;                                             // (fmax would drop it)
        slope = a.smoothing * (1.0 - down) - (1.0 - a.smoothing) * down;
      } else if (a.kind == AERO_PREF_SQUARE) {
        l = (m - 0.5) * (m - 0.5);
        slope = 2.0 * (m - 0.5);
      } else {
        l = m < 1.0 ? 1.0 - m : (m != m ? m : 0.0);
        slope = m < 1.0 ? -1.0 : (m != m ? m : 0.0);
      }
      slope *= u * a.beta;
      part[0] -= u * l;                                                // (the finalising kernel returns minus this sum)
      part[1] += rc > rr ? 1.0 : 0.0;
      part[2] += a.beta * rc;
      part[3] += a.beta * rr;
      part[4] += 1.0;
    }
    a.slope[p] = slope;
    a.margins[p] = (float)m;
  }
  for (int k = 0; k < kPartialStride; ++k) {
    const double s = block_sum(part[k], sh);
    if (threadIdx.x == 0) a.partials[(size_t)blockIdx.x * kPartialStride + k] = s;
  }
}

// A block per rollout walks all pairs in order for its own.  (A rollout is in few of them, but a list per rollout would take a sort
// to have a fixed order; 65536 pairs are 2 us of a block beside 1 to 2 us of the whole GPU for one token's products.)
__global__ void __launch_bounds__(kThreads) pref_coef_kernel(PrefArgs a) {
  __shared__ double sh[kThreads / 32];
  for (int i = blockIdx.x; i < a.R; i += gridDim.x) {
    double sum = 0.0;
    if (a.keep[i]) {
      const int2* pairs = reinterpret_cast<const int2*>(a.pairs);
#pragma unroll 4
      for (int p = threadIdx.x; p < a.P; p += kThreads) {
        const int2 q = pairs[p];
        if (q.x == i) sum += a.slope[p];
        if (q.y == i) sum -= a.slope[p];
      }
    }
    sum = block_sum(sum, sh);
    if (a.mean && a.scored[i] > 0) sum /= a.scored[i];
    const float coef = (float)sum;
    if (threadIdx.x == 0) {
      a.coef[i] = coef;
      a.w[i] = -coef;
    }
    long long t0, t1;
    if (a.wrow && a.keep[i] && rows_of(a, i, &t0, &t1))
      for (long long t = t0 + threadIdx.x; t < t1; t += kThreads) a.wrow[t] = -coef;
  }
}

// The backward alone: rollouts with a gradient, and their weights.
__global__ void __launch_bounds__(256) pref_weights_kernel(int R, const float* __restrict__ coef, uint8_t* __restrict__ keep,
                                                           float* __restrict__ w) {
  for (int i = blockIdx.x * 256 + threadIdx.x; i < R; i += gridDim.x * 256) {
    keep[i] = coef[i] != 0.f ? 1 : 0;
    w[i] = -coef[i];
  }
}

struct Ws {
  uint8_t* keep;                  // starts at zero, with counted
  int* counted;
  float* zeros;                   // [T]: the listed tokens' teacher logits
  float* w;                       // [R]
  double* r;
  int* scored;
  double* slope;
  double* partials;
  size_t zero_bytes;
  char* rest;
  size_t head_bytes;
};

Ws carve(void* base, int64_t T, int32_t R, int32_t P) {
  Ws s = {};
  char* p = static_cast<char*>(base);
  size_t off = 0;
  auto take = [&](size_t bytes) { char* q = p + off; off += aero_align_up(bytes, 256); return q; };
  s.counted = reinterpret_cast<int*>(take(4));
  s.keep = reinterpret_cast<uint8_t*>(take((size_t)R + 1));
  s.zeros = reinterpret_cast<float*>(take((size_t)(T + 1) * 4));
  s.w = reinterpret_cast<float*>(take((size_t)(R + 1) * 4));
  s.zero_bytes = off;
  s.r = reinterpret_cast<double*>(take((size_t)(R + 1) * 8));
  s.scored = reinterpret_cast<int*>(take((size_t)(R + 1) * 4));
  s.slope = reinterpret_cast<double*>(take((size_t)(P + 1) * 8));
  s.partials = reinterpret_cast<double*>(take((size_t)kPairBlocks * kPartialStride * 8));
  s.rest = p + off;
  s.head_bytes = off;
  return s;
}

int grid_for(long long n, int per, int most) {
  const long long blocks = (n + per - 1) / per;
  return (int)(blocks < 1 ? 1 : (blocks < most ? blocks : most));
}

int check_pref(const aero_pref_cfg* pc, int32_t P, const int32_t* pairs) {
  if (!pc || P < 0 || (P > 0 && !pairs)) return AERO_ERR_INVALID;
  if (pc->kind != AERO_PREF_LOGISTIC && pc->kind != AERO_PREF_SQUARE && pc->kind != AERO_PREF_HINGE) return AERO_ERR_UNSUPPORTED;
  if (!(fabsf(pc->beta) < INFINITY) || !(fabsf(pc->margin) < INFINITY) || !(pc->label_smoothing >= 0.f && pc->label_smoothing <= 1.f))
    return AERO_ERR_INVALID;
  if (reinterpret_cast<uintptr_t>(pairs) % 8) return AERO_ERR_INVALID;
  return AERO_OK;
}

int check_call(aero_ctx* ctx, const aero_cfg* cfg, const aero_pref_cfg* pc, int64_t T, int32_t d, int32_t V, int32_t R, int32_t P,
               const void* H, const void* W, const int32_t* y, const int64_t* cs, const int32_t* pairs, const float* logp,
               const float* lse, const float* ratio, const float* margin, const float* coef, const float* loss, const Ws& s,
               const void* workspace) {
  int rc = check_pref(pc, P, pairs);
  if (rc) return rc;
  if (!cfg || !workspace || !loss || (R > 0 && (!ratio || !coef)) || (P > 0 && !margin) || (T > 0 && (!logp || !lse)))
    return AERO_ERR_INVALID;
  return aero_distill_check(ctx, cfg, T, d, V, R, 1, H, W, y, s.zeros, cs, s.w, s.keep, workspace);
}

// What stands between the log-probs and the gradients.
struct Between {
  aero_ctx* ctx;
  PrefArgs a;
  float *loss, *metrics;

  int run(float* wrow) {
    a.wrow = wrow;
    const int rollouts = grid_for(a.R, 1, 65535);
    if (a.R > 0) pref_ratio_kernel<<<rollouts, kThreads, 0, ctx->stream>>>(a);
    const int blocks = grid_for(a.P, kThreads, kPairBlocks);
    pref_pairs_kernel<<<blocks, kThreads, 0, ctx->stream>>>(a);
    if (a.R > 0) pref_coef_kernel<<<rollouts, kThreads, 0, ctx->stream>>>(a);
    ctx->launches += a.R > 0 ? 3 : 1;
    AERO_CUDA_TRY(cudaGetLastError());
    return aero_loss_finalize(ctx, a.partials, blocks, kPartialStride, loss, metrics, 0);
  }
  static int call(void* self, float* wrow) { return static_cast<Between*>(self)->run(wrow); }
};

int begin(aero_ctx* ctx, const Ws& s, const PrefArgs& a) {
  AERO_CUDA_TRY(cudaMemsetAsync(s.counted, 0, s.zero_bytes, ctx->stream));
  if (a.P > 0) {
    pref_mark_kernel<<<grid_for(a.P, 256, 592), 256, 0, ctx->stream>>>(a);
    ctx->launches += 1;
  }
  AERO_CUDA_TRY(cudaGetLastError());
  return AERO_OK;
}

PrefArgs args_of(aero_ctx* ctx, const aero_pref_cfg* pc, int64_t T, int32_t V, int32_t R, int32_t P, const int32_t* y,
                 const float* ref, const int64_t* cs, const int32_t* pairs, const float* weight, const Ws& s, float* logp, float* ratio,
                 float* margin, float* coef) {
  return {T, V, R, P, pc->kind, pc->mean, pc->beta, pc->margin, pc->label_smoothing, y, ref, cs, pairs, weight, s.keep, s.counted,
          s.r, s.scored, s.slope, s.partials, logp, ratio, margin, coef, s.w, nullptr, ctx->d_status};
}

}  // namespace

extern "C" {

void aero_pref_cfg_default(aero_pref_cfg* pc) {
  if (!pc) return;
  pc->kind = AERO_PREF_LOGISTIC; pc->mean = 0; pc->beta = 0.1f; pc->margin = 0.f; pc->label_smoothing = 0.f;
}

size_t aero_pref_fwd_workspace_bytes(int64_t T, int32_t d, int32_t V, int32_t R, int32_t P) {
  const size_t inner = aero_distill_fwd_workspace_bytes(T, d, V, R, 1);
  return inner == 0 || P < 0 ? 0 : carve(nullptr, T, R, P).head_bytes + inner;
}

size_t aero_pref_bwd_workspace_bytes(int64_t T, int32_t d, int32_t V, int32_t R, int64_t chunk_tokens, int32_t dw_dtype) {
  const size_t inner = aero_distill_bwd_workspace_bytes(T, d, V, R, 1, chunk_tokens, dw_dtype);
  return inner == 0 ? 0 : carve(nullptr, T, R, 0).head_bytes + inner;
}

size_t aero_pref_fwd_bwd_workspace_bytes(int64_t T, int32_t d, int32_t V, int32_t R, int32_t P, int64_t chunk_tokens, int32_t dw_dtype) {
  size_t inner = aero_distill_fwd_bwd_workspace_bytes(T, d, V, R, 1, chunk_tokens, dw_dtype);
  if (inner == 0 || P < 0) return 0;
  for (const size_t other : {aero_distill_fwd_workspace_bytes(T, d, V, R, 1),
                             aero_distill_bwd_workspace_bytes(T, d, V, R, 1, chunk_tokens, dw_dtype)})
    if (other > inner) inner = other;
  return carve(nullptr, T, R, P).head_bytes + inner;
}

int aero_pref_fwd(aero_ctx* ctx, const aero_cfg* cfg, const aero_pref_cfg* pc, int64_t T, int32_t d, int32_t V, int32_t R, int32_t P,
                  const void* H, const void* W, const int32_t* y, const float* ref_logp, const int64_t* cs, const int32_t* pairs,
                  const float* pair_weight, float* logp, float* lse, float* ratio, float* margin, float* coef, float* loss,
                  float* metrics, void* workspace, size_t workspace_bytes) {
  AeroRange nv("aero_pref_fwd");
  const Ws s = carve(workspace, T > 0 ? T : 0, R > 0 ? R : 0, P > 0 ? P : 0);
  int rc = check_call(ctx, cfg, pc, T, d, V, R, P, H, W, y, cs, pairs, logp, lse, ratio, margin, coef, loss, s, workspace);
  if (rc) return rc;
  if (workspace_bytes < aero_pref_fwd_workspace_bytes(T, d, V, R, P)) return AERO_ERR_WORKSPACE;
  if ((rc = aero_check_ctx(ctx))) return rc;
  Between b = {ctx, args_of(ctx, pc, T, V, R, P, y, ref_logp, cs, pairs, pair_weight, s, logp, ratio, margin, coef), loss, metrics};
  AeroListed ex;
  ex.gain = true;
  if ((rc = begin(ctx, s, b.a))) return rc;
  if ((rc = aero_distill_fwd_listed(ex, ctx, cfg, T, d, V, R, 1, H, W, y, s.zeros, nullptr, cs, s.w, s.keep, lse, logp, nullptr,
                                    nullptr, s.rest, workspace_bytes - s.head_bytes)))
    return rc;
  return b.run(nullptr);
}

int aero_pref_bwd(aero_ctx* ctx, const aero_cfg* cfg, int64_t T, int32_t d, int32_t V, int32_t R, const void* H, const void* W,
                  const int32_t* y, const int64_t* cs, const float* coef, const float* lse, float grad_scale, void* dH, void* dW,
                  int32_t dw_dtype, int accumulate_dW, void* workspace, size_t workspace_bytes) {
  AeroRange nv("aero_pref_bwd");
  const Ws s = carve(workspace, T > 0 ? T : 0, R > 0 ? R : 0, 0);
  if (!cfg || !workspace || (R > 0 && !coef) || (T > 0 && !lse)) return AERO_ERR_INVALID;
  int rc = aero_distill_check(ctx, cfg, T, d, V, R, 1, H, W, y, s.zeros, cs, s.w, s.keep, workspace);
  if (rc || (rc = aero_distill_check_grads(cfg, T, dH, dW, dw_dtype, accumulate_dW))) return rc;
  if (workspace_bytes < s.head_bytes || !aero_distill_bwd_fits(cfg, T, d, V, R, 1, dw_dtype, workspace_bytes - s.head_bytes))
    return AERO_ERR_WORKSPACE;
  if ((rc = aero_check_ctx(ctx))) return rc;
  AERO_CUDA_TRY(cudaMemsetAsync(s.zeros, 0, (size_t)T * 4, ctx->stream));
  if (R > 0) {
    pref_weights_kernel<<<grid_for(R, 256, 592), 256, 0, ctx->stream>>>(R, coef, s.keep, s.w);
    ctx->launches += 1;
    AERO_CUDA_TRY(cudaGetLastError());
  }
  return aero_distill_bwd_listed({}, ctx, cfg, T, d, V, R, 1, H, W, y, s.zeros, nullptr, cs, s.w, s.keep, lse, grad_scale, dH, dW,
                                 dw_dtype, accumulate_dW, s.rest, workspace_bytes - s.head_bytes);
}

int aero_pref_fwd_bwd(aero_ctx* ctx, const aero_cfg* cfg, const aero_pref_cfg* pc, int64_t T, int32_t d, int32_t V, int32_t R,
                      int32_t P, const void* H, const void* W, const int32_t* y, const float* ref_logp, const int64_t* cs,
                      const int32_t* pairs, const float* pair_weight, float* logp, float* lse, float* ratio, float* margin,
                      float* coef, float* loss, float* metrics, float grad_scale, void* dH, void* dW, int32_t dw_dtype,
                      int accumulate_dW, void* workspace, size_t workspace_bytes) {
  AeroRange nv("aero_pref_fwd_bwd");
  const Ws s = carve(workspace, T > 0 ? T : 0, R > 0 ? R : 0, P > 0 ? P : 0);
  int rc = check_call(ctx, cfg, pc, T, d, V, R, P, H, W, y, cs, pairs, logp, lse, ratio, margin, coef, loss, s, workspace);
  if (rc || (rc = aero_distill_check_grads(cfg, T, dH, dW, dw_dtype, accumulate_dW))) return rc;
  if (workspace_bytes < s.head_bytes) return AERO_ERR_WORKSPACE;
  const size_t room = workspace_bytes - s.head_bytes;
  const bool one_chunk = cfg->dtype == AERO_BF16 && T > 0 && R > 0 && aero_distill_one_chunk(ctx, T, d, V, R, 1, dw_dtype, room);
  if (!one_chunk && (room < aero_distill_fwd_workspace_bytes(T, d, V, R, 1) || !aero_distill_bwd_fits(cfg, T, d, V, R, 1, dw_dtype, room)))
    return AERO_ERR_WORKSPACE;
  if ((rc = aero_check_ctx(ctx))) return rc;
  Between b = {ctx, args_of(ctx, pc, T, V, R, P, y, ref_logp, cs, pairs, pair_weight, s, logp, ratio, margin, coef), loss, metrics};
  AeroListed ex;
  ex.gain = true;
  if ((rc = begin(ctx, s, b.a))) return rc;
  if (one_chunk) {
    ex.between = Between::call;
    ex.arg = &b;
    return aero_distill_fwd_bwd_listed(ex, ctx, cfg, T, d, V, R, 1, H, W, y, s.zeros, nullptr, cs, s.w, s.keep, lse, logp, nullptr,
                                       nullptr, grad_scale, dH, dW, dw_dtype, accumulate_dW, s.rest, room);
  }
  if ((rc = aero_distill_fwd_listed(ex, ctx, cfg, T, d, V, R, 1, H, W, y, s.zeros, nullptr, cs, s.w, s.keep, lse, logp, nullptr,
                                    nullptr, s.rest, room)))
    return rc;
  if ((rc = b.run(nullptr))) return rc;
  return aero_distill_bwd_listed({}, ctx, cfg, T, d, V, R, 1, H, W, y, s.zeros, nullptr, cs, s.w, s.keep, lse, grad_scale, dH, dW,
                                 dw_dtype, accumulate_dW, s.rest, room);
}

}  // extern "C"
