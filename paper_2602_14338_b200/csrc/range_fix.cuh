// Rows in which bf16 could not hold exp(z - c_t) (a logit more than ~87 above the shift; MODE_FWD_P lists
// them): their dz rows recomputed from H and W.
#pragma once

#include "loss_common.cuh"

constexpr int kRangeCap = 1024;      // rows per chunk the step can redo after a saturated exp(z - c_t)

struct RangeArgs {
  const int* rows;          // chunk-local rows (tile in chunk * 128 + row in tile) listed by the forward
  const int* count;
  int cap;
  __nv_bfloat16* dz;        // tiled as above
  int nblk;
  const int32_t* tile_row;
  int tile_begin;
  long long T;
  int d, V;
  const int32_t* y;
  const float* lse;
  const float* g;
  const float* logp;        // log-prob of y, or NULL (taken from the recomputed logit)
  float grad_scale;
  const __nv_bfloat16* H;   // [T, d]
  const __nv_bfloat16* W;   // [V, d]
  __nv_bfloat16* Hs;        // row-factor form: the row's copy of H (unscaled here); NULL otherwise
  float* row_scale;         // row-factor form: set to 1 for a redone row
  const float* ent;         // entropy term: H_t and ent_coef * w_i per row; both NULL without the term
  const float* row_et;
};

// The forward could not hold exp(z - c_t) of these rows in bf16: write their dz rows from the
// definition, one warp per (row, vocabulary column), logits as fp32 dot products of the bf16
// operands.  Rare by construction (a logit ~87 above the row's first ones), so speed is no concern;
// without listed rows the kernel reads one word and returns.
static __global__ void __launch_bounds__(256) range_fix_kernel(RangeArgs a) {
  const int n = min(*a.count, a.cap);
  if (n == 0) return;
  const int lane = threadIdx.x & 31;
  const long long warp0 = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const long long nwarps = (long long)gridDim.x * 8;
  const long long ldz = (long long)a.nblk * 64;
  for (long long u = warp0; u < (long long)n * ldz; u += nwarps) {
    const int e = (int)(u / ldz), v = (int)(u % ldz);
    const int local = a.rows[e], lt = local / 128, r = local % 128;
    const long long row = (long long)a.tile_row[a.tile_begin + lt] + r;
    if (row >= a.T) continue;
    const float coef = a.g[row] * a.grad_scale;
    const float et = a.row_et != nullptr ? a.row_et[row] * a.grad_scale : 0.f;
    float val = 0.f;
    if (v < a.V && (coef != 0.f || et != 0.f)) {
      const uint4* h = reinterpret_cast<const uint4*>(a.H + row * a.d);
      const uint4* w = reinterpret_cast<const uint4*>(a.W + (long long)v * a.d);
      float acc = 0.f;
      for (int k = lane; k < a.d / 8; k += 32) {
        const uint4 hv = h[k], wv = w[k];
        const __nv_bfloat162* hp = reinterpret_cast<const __nv_bfloat162*>(&hv);
        const __nv_bfloat162* wp = reinterpret_cast<const __nv_bfloat162*>(&wv);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float2 x = __bfloat1622float2(hp[q]), yv = __bfloat1622float2(wp[q]);
          acc = fmaf(x.x, yv.x, acc);
          acc = fmaf(x.y, yv.y, acc);
        }
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
      const float lpv = v == a.y[row] && a.logp != nullptr ? a.logp[row] : acc - a.lse[row];
      val = v == a.y[row] ? -coef * expm1f(lpv) : -coef * __expf(lpv);
      if (et != 0.f) val = fmaf(et * __expf(lpv), lpv + a.ent[row], val);
    }
    if (lane == 0) a.dz[(((size_t)lt * a.nblk + v / 64) * 128 + r) * 64 + v % 64] = __float2bfloat16_rn(val);
    if (a.Hs != nullptr && v == 0) {
      // the row's factor is already in its dz entries: unit factor, plain copy of the H row
      if (lane == 0) a.row_scale[row] = 1.f;
      const uint4* src = reinterpret_cast<const uint4*>(a.H + row * a.d);
      uint4* dst = reinterpret_cast<uint4*>(a.Hs + ((size_t)lt * 128 + r) * a.d);
      for (int k = lane; k < a.d / 8; k += 32) dst[k] = src[k];
    }
  }
}
