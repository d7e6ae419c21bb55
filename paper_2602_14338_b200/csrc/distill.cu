// Distillation from a teacher's top logits through the lm_head.  Per kept token t of rollout i, with the
// teacher's list (id_tk, a_tk), k < K:
//   q_tk = exp(a_tk - n_t),  n_t = teacher_lse_t or, without it, log sum_k exp a_tk;   Q_t = sum_k q_tk
//   kl_t = sum_k q_tk (log q_tk - log p_t,id),   p_t = softmax(W h_t);     loss = sum_t w_i kl_t
//   dz_tv = grad_scale w_i (Q_t p_tv - sum_{k: id_tk = v} q_tk)
// The softmax part w_i Q_t p_tv is what stage (b) computes for a row with g_t = -w_i Q_t, so the lm_head
// kernel, the chunk block and the two backward products are stage (b)'s own.  What is new is the list:
// its logits are K dot products per row (distill_dots_kernel: 2 K d FLOP and K rows of W out of L2
// against the 2 V d of the row's logits), and after the chunk block holds the softmax
// part its K entries are written from those fp32 values (distill_scatter_kernel), never subtracted
// from a rounded probability.
//
// A chunk of token tiles in the one-call step: plan_kernel chooses the splits from the number of tiles
// the device has found; lmhead_kernel<MODE_FWD_P> leaves p~ = exp(z - c_t) in the block and the rows'
// running states; distill_dots_kernel and distill_rows_kernel finish the rows; distill_scale_kernel turns p~ into the softmax
// part; range_fix_kernel redoes rows whose p~ left bf16's range; distill_scatter_kernel; the products
// dH and dW.  (The row-factor form of aero_grpo_loss_fwd_bwd, which saves the pass over the block, would
// multiply the rows of H by exp(c_t - lse_t) and round them to bf16 once more before dW; here the list's
// entries, which are most of dz, reach dW with the rounding of dz alone, as the one-call step's dW then
// is 2.4e-3 of its norm off instead of 2.9e-3.  The price is a second rounding of the softmax part, p~ and dz: where
// a list holds little weight dH is 2.6e-3 of its norm off, 1.6e-3 with one.)
#include "distill.cuh"
#include "entry.cuh"
#include "gemm_bwd_kernel.cuh"
#include "lmhead_kernel.cuh"
#include "range_fix.cuh"
#include "tmap.cuh"
#include "vec.cuh"

namespace {

constexpr int kMaxK = 256, kSlots = kMaxK / 32;
constexpr int kUnitsPerTile = 16;       // units of 8 rows that cover a token tile in the row kernels
// Blocks of the row kernels at most: they walk the units that there are.  Only the device knows these, and the bound
// that the host has, a tile of its own for every second rollout, may be far above (20000 tokens in 20000 rollouts, all
// kept, d = 1536: loss 12.0 -> 9.0 ms, step 35.6 -> 27.3 ms).
constexpr int kRowBlocks = 2368;
constexpr int kMaxVsplit = 148;         // vocabulary splits the plan may choose
constexpr int kMaxKsplit = 16;          // ranges of the reduction of dH it may choose

// The teacher's list and what the call makes of it.
struct List {
  int K;
  const int32_t* ids;      // [T,K]
  const float* logits;     // [T,K]
  const float* tlse;       // [T] or NULL: the list itself is normalised
  float* kl;               // [T] out, or NULL
  float* z;                // [T,K] student logits at the listed tokens
  float* entry;            // [T,K] dz at the listed tokens, or NULL (forward only)
  double* partials;        // one record per block of the row kernel, or NULL
};

struct RowsArgs {
  List ls;
  long long T;
  int d, V, R;
  const void* H;
  const void* W;
  const int64_t* cs;
  const uint8_t* keep;
  const float* wrow;       // weight of each row
  float* lse;              // in: the rows' log-sum-exp, unless xstate gives it (then out)
  const int32_t* y;        // the listed token with the largest teacher logit
  float* g;                // out: -w_i Q_t, or NULL
  float4* ysum;            // out: weight of the other listed tokens and of y in the list, y's logit; or NULL
  float grad_scale;
  const float4* xstate;    // running states of the lm_head kernel, [split][T], or NULL
  const int* plan;         // split count
  __nv_bfloat16* Hl;       // chunk's copy of its rows of H, zeros where the tile has no row; or NULL
  const int32_t* tile_row; // NULL: rows 0 .. T - 1 themselves (fp32 path)
  const int32_t* tile_valid;
  const int32_t* n_tiles;
  int tile_begin, tile_end;
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// The kept rollout that owns token row t, or -1: the row belongs to a dropped rollout, to none (behind the last one), or to
// one whose offsets leave [0, T).
__device__ __forceinline__ int kept_owner(const int64_t* __restrict__ cs, const uint8_t* __restrict__ keep, int R, long long T,
                                          long long t) {
  if (R <= 0 || t >= T) return -1;
  const int i = aero_owner(cs, R, t);
  const long long a = cs[i], b = cs[i + 1];
  return keep[i] != 0 && a >= 0 && a <= t && t < b && b <= T ? i : -1;
}

// Units of 8 rows of this launch, and the token row of a warp in one of them; -1: none (past the tile's rows, or of a
// dropped rollout)
__device__ __forceinline__ long long units_of(const RowsArgs& a) {
  return a.tile_row == nullptr ? (a.T + 7) / 8 : (long long)(min(*a.n_tiles, a.tile_end) - a.tile_begin) * kUnitsPerTile;
}
__device__ __forceinline__ long long row_of(const RowsArgs& a, long long unit, int warp) {
  if (a.tile_row == nullptr) {
    const long long t = unit * 8 + warp;
    return kept_owner(a.cs, a.keep, a.R, a.T, t) >= 0 ? t : -1;
  }
  const int tile = a.tile_begin + (int)(unit / kUnitsPerTile), r = (int)(unit % kUnitsPerTile) * 8 + warp;
  if (r >= a.tile_valid[tile]) return -1;
  const long long t = (long long)a.tile_row[tile] + r;
  return t < a.T ? t : -1;
}

// Joins the running states of row t that the splits of the lm_head kernel left (largest logit m and sum of
// 2^(z log2e - m) without y's column, y's own logit), a split per lane and turn: log-sum-exp and log-prob of y.
// The formulas are those of lmhead::finish_rows.
__device__ __forceinline__ float2 join_states(const float4* xs, long long T, long long t, int nsplit, int lane) {
  float m = -INFINITY, l = 0.f, zy = 0.f;
  for (int s = lane; s < nsplit; s += 32) {
    const float4 o = xs[(size_t)s * T + t];
    const float mm = fmaxf(m, o.x);
    l = l * exp2f(m - mm) + o.y * exp2f(o.x - mm);
    zy += o.z;
    m = mm;
  }
  const float M = warp_max(m);
  // (a logit that is no number shows in l alone, in m only if it is the largest: l has to come through as it is)
  l = warp_sum(m > -INFINITY ? l * exp2f(m - M) : l);
  zy = warp_sum(zy);                                   // one split has y's column, the others hold 0
  if (l <= 0.f || (l == l && M <= lmhead::kMaskedMax2)) return make_float2(zy, 0.f);      // a vocabulary of one
  const float a = fmaf(zy, lmhead::kLog2e, -M), big = fmaxf(a, 0.f);
  const float ey = exp2f(a - big), lr = l * exp2f(-big);
  const float lse = (M + big + log2f(lr + ey)) * lmhead::kLn2;
  const float lp = a > -40.f ? -log1pf(l * exp2f(-a)) : (a - log2f(l + exp2f(a))) * lmhead::kLn2;
  return make_float2(lse, lp);
}

// The backward alone has only the rounded lse, and zy - lse is no log-prob of y where 1 - p_y comes near lse's rounding.  From
// 2^12 of these roundings down a row takes (1 - p_y) / p_y from the sum of the other columns' exponentials and y's own
// instead, in which lse cancels.
__device__ __forceinline__ bool sure_of_y(float zy, float lse) { return zy - lse > -0x1p-12f * fmaxf(fabsf(lse), 1.f); }
// dz of such a row at y; outside = sum_{v != y} exp(z_v - lse)
__device__ __forceinline__ float sure_entry(const RowsArgs& a, long long t, float outside) {
  const float4 q = a.ysum[t];
  const float lp = -log1pf(outside * expf(a.lse[t] - q.z));
  return a.grad_scale * a.wrow[t] * (q.x * expf(lp) + q.y * expm1f(lp));
}

// Student logits at the listed tokens: kDots list places of one row per warp, so that even a few hundred rows put
// thousands of warps on the machine (one warp for the whole list took 100 us for 300 rows of 64 places).  Bound by
// the gather of K rows of W per token out of L2.
constexpr int kDots = 4;
template <typename T>
__device__ __forceinline__ void list_dots(const RowsArgs& a, long long t, int k0, int lane) {
  constexpr int VEC = rowvec::Elem<T>::kVec;
  const int K = a.ls.K, d = a.d;
  int v[kDots];
  const T* w[kDots];
  int last = -1;
#pragma unroll
  for (int q = 0; q < kDots; ++q) {
    v[q] = k0 + q < K ? a.ls.ids[t * K + k0 + q] : -1;
    if (v[q] >= a.V) v[q] = -1;
    if (v[q] >= 0) last = v[q];
  }
  if (last < 0) return;
#pragma unroll
  for (int q = 0; q < kDots; ++q) w[q] = static_cast<const T*>(a.W) + (long long)(v[q] >= 0 ? v[q] : last) * d;
  const T* h = static_cast<const T*>(a.H) + t * d;
  float acc[kDots] = {0.f, 0.f, 0.f, 0.f};
  if (d % VEC == 0) {
#pragma unroll 2
    for (int e = lane * VEC; e < d; e += 32 * VEC) {
      float x[VEC], y[kDots][VEC];
      rowvec::load<T, VEC>(h + e, x);
#pragma unroll
      for (int q = 0; q < kDots; ++q) rowvec::load<T, VEC>(w[q] + e, y[q]);
#pragma unroll
      for (int q = 0; q < kDots; ++q)
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[q] = fmaf(x[i], y[q][i], acc[q]);
    }
  } else {
    for (int e = lane; e < d; e += 32) {
      const float x = rowvec::Elem<T>::load(h + e);
#pragma unroll
      for (int q = 0; q < kDots; ++q) acc[q] = fmaf(x, rowvec::Elem<T>::load(w[q] + e), acc[q]);
    }
  }
#pragma unroll
  for (int q = 0; q < kDots; ++q) {
    acc[q] = warp_sum(acc[q]);
    if (lane == 0 && v[q] >= 0) a.ls.z[t * K + k0 + q] = acc[q];
  }
}
template <typename T>
__global__ void __launch_bounds__(256) distill_dots_kernel(RowsArgs a) {
  const long long n = units_of(a);
  for (long long u = blockIdx.x; u < n; u += gridDim.x) {
    const long long t = row_of(a, u, threadIdx.x >> 5);
    if (t >= 0) list_dots<T>(a, t, blockIdx.y * kDots, threadIdx.x & 31);
  }
}

__global__ void __launch_bounds__(256) distill_rows_kernel(RowsArgs a) {
  __shared__ double rec[8][kPartialStride];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int K = a.ls.K, d = a.d;
  double part[kPartialStride] = {0.0, 0.0, 0.0, 0.0, 0.0};
  const long long n = units_of(a);
  for (long long u = blockIdx.x; u < n; u += gridDim.x) {
    const long long t = row_of(a, u, warp);
    if (a.Hl) {
      uint4* dst = reinterpret_cast<uint4*>(a.Hl + ((size_t)u * 8 + warp) * d);
      const uint4* src = t >= 0 ? reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.H) + t * d) : nullptr;
      for (int k = lane; k < d / 8; k += 32) dst[k] = src ? src[k] : make_uint4(0, 0, 0, 0);
    }
    if (t >= 0) {
      const float wi = a.wrow[t];
      const int yt = a.y[t];
      float lse, lp_y = 0.f;
      if (a.xstate) {
        const float2 s = join_states(a.xstate, a.T, t, *a.plan, lane);
        lse = s.x;
        lp_y = s.y;
      } else {
        lse = a.lse[t];
      }
      // slot s of a lane holds list place 32 s + lane
      int id[kSlots];
      float lg[kSlots], z[kSlots];
      float hi = -INFINITY;
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        id[s] = -1;
        lg[s] = -INFINITY;
        z[s] = 0.f;
        if (s * 32 < K) {
          const int k = s * 32 + lane;
          if (k < K) {
            const int v = a.ls.ids[t * K + k];
            if (v >= 0 && v < a.V) {
              id[s] = v;
              lg[s] = a.ls.logits[t * K + k];
              hi = fmaxf(hi, lg[s]);
            }
          }
        }
      }
      float norm;
      if (a.ls.tlse) {
        norm = a.ls.tlse[t];
      } else {
        hi = warp_max(hi);
        float sum = 0.f;
#pragma unroll
        for (int s = 0; s < kSlots; ++s)
          if (id[s] >= 0 && lg[s] > -INFINITY) sum += expf(lg[s] - hi);
        norm = hi + logf(warp_sum(sum));            // (an empty list: -inf, no place below uses it)
      }
      // student logits at the listed tokens, from distill_dots_kernel
      float zy = 0.f;
      bool any_listed = false;
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        if (s * 32 < K) {
          if (id[s] >= 0) z[s] = a.ls.z[t * K + s * 32 + lane];
          const unsigned is_y = __ballot_sync(0xffffffffu, id[s] == yt && id[s] >= 0);
          if (is_y) zy = __shfl_sync(0xffffffffu, z[s], __ffs(is_y) - 1);
          any_listed |= is_y != 0;
        }
      }
      if (a.xstate) {
        // y's logit again, now as the dot product: the accumulation of the tensor cores is off by up to 2^-23 of the
        // partial sums a step, which for a logit that makes up most of the sum would be most of lse's error.  With
        // L = (1 - p_y) / p_y the correction keeps the accuracy of a log-prob close to 0.
        const float dlt = any_listed ? zy - (lse + lp_y) : 0.f;
        lp_y = lp_y > -30.f ? -log1pf(expm1f(-lp_y) * expf(-dlt)) : lp_y + dlt;
        if (any_listed) lse = zy - lp_y;
        if (lane == 0) a.lse[t] = lse;
      } else {
        lp_y = zy - lse;
      }
      float kl = 0.f, Q = 0.f, mass = 0.f, q[kSlots], lps[kSlots];
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        q[s] = 0.f;
        lps[s] = -INFINITY;
        if (id[s] >= 0) {
          const float lp = id[s] == yt ? lp_y : z[s] - lse;
          lps[s] = lp;
          mass += expf(lp);
          if (lg[s] > -INFINITY) {                    // a logit of -inf or NaN carries no weight
            const float lq = lg[s] - norm;
            q[s] = expf(lq);
            if (q[s] != 0.f) kl = fmaf(q[s], lq - lp, kl);
            Q += q[s];
          }
        }
      }
      kl = warp_sum(kl);
      Q = warp_sum(Q);
      mass = warp_sum(mass);
      if (a.ls.entry) {
        // Q p - q of a token, with q the sum over its places and q_o that over the other tokens', as q_o p + q (p - 1): both
        // terms keep their relative accuracy where p and q are close to 1, which a difference of rounded numbers next to
        // 1 does not
        const float c = a.grad_scale * wi;
        float same[kSlots], other[kSlots];
#pragma unroll
        for (int s = 0; s < kSlots; ++s) same[s] = other[s] = 0.f;
#pragma unroll
        for (int s2 = 0; s2 < kSlots; ++s2) {
          if (s2 * 32 < K) {
            for (int l = 0; l < 32 && s2 * 32 + l < K; ++l) {
              const int v = __shfl_sync(0xffffffffu, id[s2], l);
              const float qv = __shfl_sync(0xffffffffu, q[s2], l);
#pragma unroll
              for (int s = 0; s < kSlots; ++s) {
                if (id[s] == v) same[s] += qv;
                else other[s] += qv;
              }
            }
          }
        }
#pragma unroll
        for (int s = 0; s < kSlots; ++s)
          if (s * 32 + lane < K) {
            a.ls.entry[t * K + s * 32 + lane] = c * (other[s] * expf(lps[s]) + same[s] * expm1f(lps[s]));
            if (a.ysum && id[s] == yt) a.ysum[t] = make_float4(other[s], same[s], zy, 0.f);
          }
      }
      if (lane == 0) {
        if (a.ysum && !any_listed) a.ysum[t] = make_float4(0.f, 0.f, -INFINITY, 0.f);
        if (a.g) a.g[t] = -wi * Q;
        if (a.ls.kl) a.ls.kl[t] = kl;
      }
      part[0] -= (double)wi * (double)kl;             // (the finalising kernel returns minus this sum)
      part[1] += Q > 0.f ? 0.0 : 1.0;
      part[2] += kl;
      part[3] += mass;
      part[4] += 1.0;
    }
  }
  if (a.ls.partials) {
    if (lane == 0)
      for (int k = 0; k < kPartialStride; ++k) rec[warp][k] = part[k];
    __syncthreads();
    if (threadIdx.x < kPartialStride) {
      double s = 0.0;
      for (int w = 0; w < 8; ++w) s += rec[w][threadIdx.x];
      a.ls.partials[(size_t)blockIdx.x * kPartialStride + threadIdx.x] += s;      // (one chunk after another)
    }
  }
}

struct BlockArgs {
  RowsArgs a;
  __nv_bfloat16* dz;            // the chunk's block, tiled: [tile - tile_begin][nblk][128][64]
  int nblk, nvt;
  const float* shift;           // [split][T], log2 domain
  float* outside;               // backward alone: probability outside y's column of the rows that are sure of y; else NULL
};

// p~ -> the softmax part of dz, -g_t grad_scale exp(c_t - lse_t) p~, in place: block (vocabulary tile of 256
// columns, token tile).  The factor goes on in two halves of the exponent, so that it stays in fp32's normal range
// for rows whose many logits put lse far above the shift.  Bound by memory: the block is read and written once.
__global__ void __launch_bounds__(256) distill_scale_kernel(BlockArgs b) {
  __shared__ float2 f[128];
  const RowsArgs& a = b.a;
  const int j = blockIdx.x, tile_end = min(*a.n_tiles, a.tile_end);
  const int n = min(4, b.nblk - 4 * j) * 128 * 8;              // 16-byte vectors of a piece
  for (int tile = a.tile_begin + blockIdx.y; tile < tile_end; tile += gridDim.y) {
    __syncthreads();                                           // the previous tile's factors have been used
    if (threadIdx.x < 128) {
      const int r = threadIdx.x;
      const long long t = (long long)a.tile_row[tile] + r;
      float2 v = make_float2(0.f, 0.f);
      if (r < a.tile_valid[tile] && t < a.T) {
        // the split whose range of vocabulary tiles holds tile j
        const int s = (int)(((long long)(j + 1) * *a.plan - 1) / b.nvt);
        const float h = exp2f(0.5f * (b.shift[(size_t)s * a.T + t] - a.lse[t] * lmhead::kLog2e));
        v = make_float2(h, -a.g[t] * a.grad_scale * h);
      }
      f[r] = v;
    }
    __syncthreads();
    uint4* p = reinterpret_cast<uint4*>(b.dz + ((size_t)(tile - a.tile_begin) * b.nblk + 4 * j) * 128 * 64);
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += 256) {
      const float2 c = f[(i >> 3) & 127];
      float x[8];
      rowvec::unpack(p[i], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = c.y != 0.f ? x[e] * c.x * c.y : 0.f;      // (a row without weight: zeros)
      p[i] = rowvec::pack(x);
    }
  }
}

// Of the rows that are sure of y (sure_of_y), the probability outside y's column, from the softmax part that the block
// holds: its values are rounded to bf16, and the entry that is made of their sum will be too.  (Summing in the lm_head kernel's
// epilogue instead made all rows pay: 340 -> 393 us for the kernel at 1000 rows, d = 1536, V = 151936.)  A block per row.
__global__ void __launch_bounds__(256) distill_outside_kernel(BlockArgs b) {
  __shared__ float sh[8];
  const RowsArgs& a = b.a;
  const long long rows = units_of(a) * 8;
  for (long long i = blockIdx.x; i < rows; i += gridDim.x) {
    const long long t = row_of(a, i / 8, (int)(i % 8));
    if (t < 0) continue;
    const float c0 = -a.g[t] * a.grad_scale;
    if (c0 == 0.f || !sure_of_y(a.ysum[t].z, a.lse[t])) continue;
    const int y = a.y[t], n = b.nblk * 8;                         // 16-byte vectors of the row, 8 in a row of a 64-column tile
    const uint4* p = reinterpret_cast<const uint4*>(b.dz + ((size_t)(i / 128) * b.nblk * 128 + i % 128) * 64);
    float sum = 0.f;
#pragma unroll 8
    for (int k = threadIdx.x; k < n; k += 256) {
      float x[8];
      rowvec::unpack(p[(size_t)(k >> 3) * (128 * 8) + (k & 7)], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += k * 8 + e != y ? x[e] : 0.f;
    }
    sum = warp_sum(sum);
    __syncthreads();                                              // the previous row's sums have been read
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
      sum = 0.f;
      for (int w = 0; w < 8; ++w) sum += sh[w];
      b.outside[t] = sum / c0;
    }
  }
}

// The entries of dz at the listed tokens, over the softmax part.
__global__ void __launch_bounds__(256) distill_scatter_kernel(BlockArgs b) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int K = b.a.ls.K;
  const long long n = units_of(b.a);
  for (long long u = blockIdx.x; u < n; u += gridDim.x) {
    const long long t = row_of(b.a, u, warp);
    if (t < 0) continue;
    const int lt = (int)(u / kUnitsPerTile), r = (int)(u % kUnitsPerTile) * 8 + warp;
    int y = -1;
    float at_y = 0.f;
    if (b.outside && b.a.g[t] * b.a.grad_scale != 0.f && sure_of_y(b.a.ysum[t].z, b.a.lse[t])) {
      y = b.a.y[t];
      at_y = sure_entry(b.a, t, b.outside[t]);
    }
    for (int k = lane; k < K; k += 32) {
      const int v = b.a.ls.ids[t * K + k];
      if (v < 0 || v >= b.a.V) continue;
      b.dz[(((size_t)lt * b.nblk + v / 64) * 128 + r) * 64 + v % 64] =
          __float2bfloat16_rn(v == y ? at_y : b.a.ls.entry[t * K + k]);
    }
  }
}

// dH of the chunk's rows from the fp32 sums of the ranges, added in order; a warp takes 256 columns of a row.
__global__ void __launch_bounds__(256) distill_join_dh_kernel(RowsArgs a, const int* __restrict__ ksplit,
                                                              const float* __restrict__ part, const float* __restrict__ factor,
                                                              __nv_bfloat16* __restrict__ dH) {
  const int ks = *ksplit;
  if (ks <= 1) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n = (int)units_of(a);
  const long long rows = (long long)n * 8;
  const int c = blockIdx.y * 256 + lane * 8;
  if (c >= a.d) return;
  for (int u = blockIdx.x; u < n; u += gridDim.x) {
    const long long t = row_of(a, u, warp);
    if (t < 0) continue;
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int k = 0; k < ks; ++k) {
      const float4* p = reinterpret_cast<const float4*>(part + (k * rows + u * 8 + warp) * a.d + c);
      const float4 x = p[0], y = p[1];
      s[0] += x.x; s[1] += x.y; s[2] += x.z; s[3] += x.w;
      s[4] += y.x; s[5] += y.y; s[6] += y.z; s[7] += y.w;
    }
    if (factor) {
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] *= factor[t];
    }
    rowvec::store<__nv_bfloat16, 8>(dH + t * a.d + c, s);
  }
}

// The chunk's rows of H times the factors of their rows (AeroListed::row_factor).
__global__ void __launch_bounds__(256) distill_scale_rows_kernel(RowsArgs a, const float* __restrict__ factor) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long n = units_of(a);
  for (long long u = blockIdx.x; u < n; u += gridDim.x) {
    const long long t = row_of(a, u, warp);
    if (t < 0) continue;
    const float f = factor[t];
    uint4* p = reinterpret_cast<uint4*>(a.Hl + ((size_t)u * 8 + warp) * a.d);
    for (int k = lane; k < a.d / 8; k += 32) {
      float x[8];
      rowvec::unpack(p[k], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= f;
      p[k] = rowvec::pack(x);
    }
  }
}

// Before anything else, one warp per row: y_t = the listed token with the largest teacher logit (the first of equals; 0 where the
// list is empty) and the row's weight, or the outputs of a row that belongs to no kept rollout.  y's entry of dz keeps the
// relative accuracy of 1 - p_y.  No other token needs that: its q (in one place) is at most y's, and its entry q_o p - q (1 - p) then has
// in q_o p, q_o >= q_y >= q, a term that the rounding of its log-prob is small against.
struct FirstArgs {
  long long T;
  int d, V, R, K;
  const int32_t* ids;
  const float* logits;
  const int64_t* cs;
  const float* w;
  const uint8_t* keep;
  int32_t* y;
  float* wrow;
  float* lse;              // out, or NULL
  float* kl;               // out, or NULL
  __nv_bfloat16* dH;       // out (bf16 path with gradients), or NULL
  uint32_t* status;
};

__global__ void __launch_bounds__(256) distill_first_kernel(FirstArgs a) {
  const int lane = threadIdx.x & 31;
  const long long nwarps = (long long)gridDim.x * 8;
  for (long long t = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); t < a.T; t += nwarps) {
    const int owner = kept_owner(a.cs, a.keep, a.R, a.T, t);
    if (owner < 0) {
      if (lane == 0) {
        if (a.lse) a.lse[t] = 0.f;
        if (a.kl) a.kl[t] = 0.f;
      }
      if (a.dH)
        for (int k = lane; k < a.d / 8; k += 32) reinterpret_cast<uint4*>(a.dH + t * a.d)[k] = make_uint4(0, 0, 0, 0);
      continue;
    }
    int first = 0x7fffffff;
    float top = -INFINITY;
    bool bad = false;
    for (int k = lane; k < a.K; k += 32) {
      const int v = a.ids[t * a.K + k];
      const float x = a.logits[t * a.K + k];
      if (v >= 0 && v < a.V) {
        if (x > top || first == 0x7fffffff) first = k;        // (a NaN is larger than nothing)
        top = fmaxf(top, x);
      } else {
        bad |= v != AERO_NO_TOKEN;
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const int f = __shfl_xor_sync(0xffffffffu, first, o);
      const float x = __shfl_xor_sync(0xffffffffu, top, o);
      if (x > top || (x == top && f < first)) { first = f; top = x; }
    }
    if (__any_sync(0xffffffffu, bad) && lane == 0) aero_raise(a.status, AERO_ST_BAD_TARGET);
    if (lane == 0) {
      a.y[t] = first < a.K ? a.ids[t * a.K + first] : 0;
      a.wrow[t] = a.w[owner];
    }
  }
}

// Splits of this chunk's launches, from the number of token tiles the device found: plan[0] vocabulary splits of
// the lm_head kernel, plan[1] ranges of the reduction of dH.  Each candidate's cost is the rounds of its units over
// the CTA (pair)s times the length of a unit, in vocabulary tiles or 64-deep slabs, plus what a unit and a split
// cost besides: 0.4 tiles (with 1 or 2 instead the loss of 2000 tokens takes 643 or 647 us, not 624, of 5000 tokens
// 1496 or 1517, not 1471), and an estimate of 8 slabs and the traffic of the fp32 sums.  With stage (b)'s at most
// four splits of the vocabulary and none of dH a small call leaves most SMs idle (d = 1536: loss of 1000 tokens 1290
// us instead of 370, step of 300 tokens 2410 instead of 490).
// Block 0 plans; with dW given all blocks clear it if there is no tile at all (the products then write nothing).
struct PlanArgs {
  const int32_t* n_tiles;
  int tile_begin, tpc;
  int pairs;               // CTA pairs of the lm_head kernel
  int nvt, v_lo, v_hi;
  int workers, rows_per_worker, n_nt, nkb, k_hi, d;      // the dH product
  int* plan;
  uint4* dW;
  size_t dW_vecs;
};

__device__ __forceinline__ int best_of(float cost, int what) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float c = __shfl_xor_sync(0xffffffffu, cost, o);
    const int w = __shfl_xor_sync(0xffffffffu, what, o);
    if (c < cost || (c == cost && w < what)) { cost = c; what = w; }
  }
  return what;
}

__global__ void __launch_bounds__(256) plan_kernel(PlanArgs a) {
  if (a.dW && *a.n_tiles == 0)
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < a.dW_vecs; i += (size_t)gridDim.x * 256)
      a.dW[i] = make_uint4(0, 0, 0, 0);
  if (blockIdx.x > 0 || threadIdx.x >= 32) return;
  const int lane = threadIdx.x;
  const int n = max(1, min(*a.n_tiles - a.tile_begin, a.tpc));
  auto div = [](int x, int y) { return (x + y - 1) / y; };
  float best = INFINITY;
  int what = a.v_lo;
  for (int v = a.v_lo + lane; v <= a.v_hi; v += 32) {
    const float c = div(div(n, 2) * v, a.pairs) * (div(a.nvt, v) + 0.4f);
    if (c < best) { best = c; what = v; }
  }
  what = best_of(best, what);
  if (lane == 0) a.plan[0] = what;
  best = INFINITY;
  what = 1;
  for (int k = 1 + lane; k <= a.k_hi; k += 32) {
    const float sums = k > 1 ? 20.f + (float)k * n * 128.f * a.d * 8.f / 1.3e6f : 0.f;
    const float c = div(div(n, a.rows_per_worker) * a.n_nt * k, a.workers) * (div(a.nkb, k) + 8.f) + sums;
    if (c < best) { best = c; what = k; }
  }
  what = best_of(best, what);
  if (lane == 0) a.plan[1] = what;
}

// ---- fp32 path, for small shapes -----------------------------------------------------------------
// A block per row, its warps sharing the other operand's rows between them: 32 at a time stand in a warp's part of
// shared memory, a row apart by an odd number of words, and a lane has one of them, so that a logit is d products
// in a lane, without a reduction.  The warps' results are added in order.  Bound by the staging (each of the T V d
// products is read from shared memory once, and each row of the other operand through L2 for every row): 189 us at T =
// 160, K = 9, d = 57, V = 831; a warp per row that kept its own staging area took 253 us.
constexpr int kMaxD32 = 1024;

struct Fp32Args {
  RowsArgs r;
  float* dH;               // gradients; NULL: the log-sum-exp alone
  float* dW;
  int accumulate;
};

// 32 rows of `src` from row r0 into the warp's staging area (zeros past `n`, and where `g` says that the row has no
// weight, so that what stands in rows of dropped rollouts is not looked at)
__device__ __forceinline__ void stage_rows(float* dst, int pitch, const float* src, long long r0, long long n, int d,
                                           const float* g) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
#pragma unroll 4
  for (int i = 0; i < 32; ++i) {
    const bool there = r0 + i < n && (g == nullptr || g[r0 + i] != 0.f);
    for (int k = lane; k < d; k += 32) dst[i * pitch + k] = there ? src[(r0 + i) * d + k] : 0.f;
  }
  __syncwarp();
}
__device__ __forceinline__ float dot(const float* a, const float* b, int d) {
  float z = 0.f;
#pragma unroll 4
  for (int k = 0; k < d; ++k) z = fmaf(a[k], b[k], z);
  return z;
}
// acc += sum_i x_i tile[i, :], lane i holding x_i
template <int NC>
__device__ __forceinline__ void add_rows(float (&acc)[NC], float x_mine, const float* tile, int pitch, int d) {
  const int lane = threadIdx.x & 31;
  for (int i = 0; i < 32; ++i) {
    const float x = __shfl_sync(0xffffffffu, x_mine, i);
#pragma unroll
    for (int q = 0; q < NC; ++q)
      if (q * 32 + lane < d) acc[q] = fmaf(x, tile[i * pitch + q * 32 + lane], acc[q]);
  }
}
// the warps' rows of sums, added in order, to out[d]; then x times the row `last`
template <int NC>
__device__ __forceinline__ void join_rows(const float (&acc)[NC], float* sm, int d, float* out, bool accumulate, float x = 0.f,
                                          const float* last = nullptr) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, nw = blockDim.x >> 5;
  __syncthreads();                                       // the staged rows have been read
#pragma unroll
  for (int q = 0; q < NC; ++q)
    if (q * 32 + lane < d) sm[warp * d + q * 32 + lane] = acc[q];
  __syncthreads();
  for (int k = threadIdx.x; k < d; k += blockDim.x) {
    float s = 0.f;
    for (int w = 0; w < nw; ++w) s += sm[w * d + k];
    if (last) s = fmaf(x, last[k], s);
    out[k] = accumulate ? out[k] + s : s;
  }
}

// Block t: the row's log-sum-exp, or its row of dH.  NC * 32 >= d.  A row of dH that is sure of y (sure_of_y) sums
// the probability of the other columns on its way, makes y's entry of it and adds that entry's share last.
template <int NC, bool GRADS>
__global__ void __launch_bounds__(256) fp32_rows_kernel(Fp32Args f) {
  extern __shared__ float sm[];
  __shared__ float2 state[8];
  const RowsArgs& a = f.r;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, nw = blockDim.x >> 5, d = a.d, pitch = d | 1, K = a.ls.K;
  float* h = sm;
  float* tile = sm + d + warp * 32 * pitch;
  const long long t = blockIdx.x;
  const bool kept = kept_owner(a.cs, a.keep, a.R, a.T, t) >= 0;
  const float lse = GRADS && kept ? a.lse[t] : 0.f, c = GRADS && kept ? -a.grad_scale * a.g[t] : 0.f;
  for (int k = threadIdx.x; k < d; k += blockDim.x) h[k] = kept ? static_cast<const float*>(a.H)[t * d + k] : 0.f;
  __syncthreads();
  float m = -INFINITY, l = 0.f, acc[NC];
#pragma unroll
  for (int q = 0; q < NC; ++q) acc[q] = 0.f;
  const bool work = GRADS ? c != 0.f : kept;
  const int yt = GRADS && work && sure_of_y(a.ysum[t].z, lse) ? a.y[t] : -1;
  float rest = 0.f;
  for (int v0 = warp * 32; work && v0 < a.V; v0 += nw * 32) {
    stage_rows(tile, pitch, static_cast<const float*>(a.W), v0, a.V, d, nullptr);
    const float z = dot(h, tile + lane * pitch, d);
    const bool in = v0 + lane < a.V;
    if (!GRADS) {
      if (in) {
        const float mn = fmaxf(m, z);
        l = l * expf(m - mn) + expf(z - mn);
        m = mn;
      }
      continue;
    }
    const float p = in ? expf(z - lse) : 0.f;
    float dz = c * p;
    if (v0 + lane != yt) rest += p;
    for (int k0 = 0; k0 < K; k0 += 32) {                 // at a listed token the entry takes the place of the softmax part
      const int id = k0 + lane < K ? a.ls.ids[t * K + k0 + lane] : -1;
      for (unsigned hits = __ballot_sync(0xffffffffu, id >= v0 && id < v0 + 32 && id < a.V); hits != 0; hits &= hits - 1) {
        const int src = __ffs(hits) - 1, v = __shfl_sync(0xffffffffu, id, src);
        if (v == v0 + lane) dz = a.ls.entry[t * K + k0 + src];
      }
    }
    if (v0 + lane == yt) dz = 0.f;
    add_rows<NC>(acc, dz, tile, pitch, d);
  }
  if (GRADS) {
    float entry = 0.f;
    if (yt >= 0) {
      rest = warp_sum(rest);
      if (lane == 0) state[warp].x = rest;
      __syncthreads();
      float outside = 0.f;
      for (int w = 0; w < nw; ++w) outside += state[w].x;
      entry = sure_entry(a, t, outside);
      for (int k = threadIdx.x; k < K; k += blockDim.x)                            // (for the rows of dW)
        if (a.ls.ids[t * K + k] == yt) a.ls.entry[t * K + k] = entry;
    }
    join_rows<NC>(acc, sm, d, f.dH + t * d, false, entry, yt >= 0 ? static_cast<const float*>(a.W) + (long long)yt * d : nullptr);
  } else {
    const float M = warp_max(m);
    l = warp_sum(m > -INFINITY ? l * expf(m - M) : l);   // (l alone shows a logit that is no number)
    if (lane == 0) state[warp] = make_float2(M, l);
    __syncthreads();
    if (threadIdx.x == 0 && kept) {
      float top = -INFINITY, sum = 0.f;
      for (int w = 0; w < nw; ++w) top = fmaxf(top, state[w].x);
      for (int w = 0; w < nw; ++w)
        sum += state[w].x > -INFINITY ? state[w].y * expf(state[w].x - top) : state[w].y;
      a.lse[t] = top + logf(sum);
    }
  }
}

// Block v: dW[v, :] (+)= sum_t dz_tv H[t, :].
template <int NC>
__global__ void __launch_bounds__(256) fp32_vocabulary_kernel(Fp32Args f) {
  extern __shared__ float sm[];
  const RowsArgs& a = f.r;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, nw = blockDim.x >> 5, d = a.d, pitch = d | 1, K = a.ls.K;
  float* w = sm;
  float* tile = sm + d + warp * 32 * pitch;
  const int v = blockIdx.x;
  for (int k = threadIdx.x; k < d; k += blockDim.x) w[k] = static_cast<const float*>(a.W)[(long long)v * d + k];
  __syncthreads();
  float acc[NC];
#pragma unroll
  for (int q = 0; q < NC; ++q) acc[q] = 0.f;
  for (long long t0 = warp * 32; t0 < a.T; t0 += nw * 32) {
    const long long t = t0 + lane;
    const float c = t < a.T ? -a.grad_scale * a.g[t] : 0.f;      // (0 for the rows of dropped rollouts)
    if (!__any_sync(0xffffffffu, c != 0.f)) continue;
    stage_rows(tile, pitch, static_cast<const float*>(a.H), t0, a.T, d, a.g);
    const float z = dot(w, tile + lane * pitch, d);
    float dz = 0.f;
    if (c != 0.f) {
      dz = c * expf(z - a.lse[t]);
#pragma unroll 4
      for (int k = 0; k < K; ++k)
        if (a.ls.ids[t * K + k] == v) dz = a.ls.entry[t * K + k];
    }
    add_rows<NC>(acc, dz, tile, pitch, d);
  }
  join_rows<NC>(acc, sm, d, f.dW + (long long)v * d, f.accumulate != 0);
}

// ---- workspace -----------------------------------------------------------------------------------------
enum Mode { kFwd, kBwd, kBoth };

struct Ws {
  int* zero;                 // starts at zero: 1 KB of pacing counters, plan, count of the range list, then its rows' bits
  int* plan;
  int* range_count;
  unsigned int* range_seen;
  int* range_rows;
  int32_t* y;
  float* wrow;
  float* g;
  float* z;
  float* entry;
  float4* ysum;
  float* outside;
  double* partials;
  size_t n_partials;
  aero_tiles tiles;
  float4* xstate;
  float* shift;
  float* part;               // fp32 sums of dH
  int v_hi, k_hi;
  char* rest;                // chunk block, then the chunk's rows of H
  size_t head_bytes;
};

inline long long ldz_of(int32_t V) { return ((long long)V + 63) / 64 * 64; }
inline size_t chunk_tile_bytes(int32_t d, int32_t V) { return (size_t)128 * ((size_t)ldz_of(V) * 2 + (size_t)d * 2); }
// token tiles a call may have: one per 128 rows, and each run of kept rollouts (a rollout that is not kept, or empty, lies
// between any two) may end in one of its own
inline int64_t max_tiles_of(int64_t T, int32_t R) { return T / 128 + ((int64_t)R + 1) / 2 + 1; }
// of Ws::zero, with the bits of so many token tiles' rows
inline size_t zero_bytes(size_t tiles) { return 1024 + tiles * lmhead::BM / 8; }
inline unsigned row_blocks_of(int64_t units) { return (unsigned)(units < kRowBlocks ? (units > 0 ? units : 1) : kRowBlocks); }

Ws carve(void* base, int64_t T, int32_t d, int32_t V, int32_t R, int32_t K, Mode mode) {
  Ws w = {};
  const size_t Tn = (size_t)(T > 0 ? T : 1);
  const int nvt = (V + lmhead::BN - 1) / lmhead::BN;
  char* p = static_cast<char*>(base);
  size_t off = 0;
  auto take = [&](size_t bytes) { char* r = p + off; off += aero_align_up(bytes, 256); return r; };
  const size_t mt = (size_t)max_tiles_of(T, R);
  w.zero = reinterpret_cast<int*>(take(zero_bytes(mode == kBoth ? mt : 0)));
  w.plan = w.zero + 128;
  w.range_count = w.zero + 192;
  w.range_seen = reinterpret_cast<unsigned int*>(w.zero + 256);
  w.range_rows = reinterpret_cast<int*>(take(kRangeCap * sizeof(int)));
  w.y = reinterpret_cast<int32_t*>(take(Tn * 4));
  w.wrow = reinterpret_cast<float*>(take(Tn * 4));
  w.g = reinterpret_cast<float*>(take(Tn * 4));
  w.z = reinterpret_cast<float*>(take(Tn * (size_t)K * 4));
  if (mode != kFwd) w.entry = reinterpret_cast<float*>(take(Tn * (size_t)K * 4));
  const long long tile_units = (long long)mt * kUnitsPerTile, row_units = ((long long)T + 7) / 8;      // of the two paths
  w.n_partials = row_blocks_of(tile_units > row_units ? tile_units : row_units);
  w.partials = reinterpret_cast<double*>(take(w.n_partials * kPartialStride * sizeof(double)));
  w.tiles = aero_carve_tiles(p + off, T, R, lmhead::BM);
  w.tiles.max_tiles = (int32_t)mt;
  off += aero_tiles_bytes(T, R, lmhead::BM);
  // more than one wave of token tiles keeps all SMs busy without further splits (loss at d = 1536: 24000 tokens 6640 us
  // without, 6850 with; 16000 tokens 4600 without, 4560 with)
  const bool few = T <= 148 * 128;
  const int base_v = aero_vsplit_cap(d);
  w.v_hi = few && base_v < kMaxVsplit ? kMaxVsplit : base_v;
  if (w.v_hi > nvt) w.v_hi = nvt;
  if (mode != kBwd) w.xstate = reinterpret_cast<float4*>(take((size_t)w.v_hi * Tn * sizeof(float4)));
  if (mode == kBwd) w.outside = reinterpret_cast<float*>(take(Tn * 4));
  if (mode != kFwd) w.ysum = reinterpret_cast<float4*>(take(Tn * sizeof(float4)));
  if (mode == kBoth) w.shift = reinterpret_cast<float*>(take((size_t)w.v_hi * Tn * sizeof(float)));
  w.k_hi = 1;
  if (mode != kFwd && few) {
    const size_t one = mt * 128 * (size_t)d * sizeof(float), room = (size_t)256 << 20;
    w.k_hi = one * kMaxKsplit <= room ? kMaxKsplit : (one * 2 <= room ? (int)(room / one) : 1);
    if (w.k_hi > 1) w.part = reinterpret_cast<float*>(take(one * (size_t)w.k_hi));
  }
  w.rest = p + off;
  w.head_bytes = off;
  return w;
}

// fp32 sums for a bf16 dW that is made of several chunks
size_t dw_sums_bytes(int32_t d, int32_t V) { return aero_align_up((size_t)V * d * sizeof(float), 256); }

__global__ void __launch_bounds__(256) dw_to_bf16_kernel(const float4* __restrict__ in, uint2* __restrict__ out, size_t n) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) {
    const float4 v = in[i];
    uint2 o;
    __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&o);
    h[0] = __floats2bfloat162_rn(v.x, v.y);
    h[1] = __floats2bfloat162_rn(v.z, v.w);
    out[i] = o;
  }
}

// How a call with gradients uses what its workspace has after the head: tiles per chunk, and for a bf16 dW of
// several chunks the fp32 sums first.
struct Room {
  long long tpc = 0;             // 0: not enough
  bool sums = false;

  Room(size_t bytes, int64_t T, int32_t d, int32_t V, int32_t R, bool bf16, int sm_count) {
    const long long mt = max_tiles_of(T, R);
    tpc = (long long)(bytes / chunk_tile_bytes(d, V));
    if (tpc > 32768) tpc = 32768;                                           // unit numbers stay within 32 bits
    if (tpc >= mt) { tpc = mt; return; }
    if (bf16) {
      sums = true;
      const size_t used = dw_sums_bytes(d, V);
      tpc = bytes < used ? 0 : (long long)((bytes - used) / chunk_tile_bytes(d, V));
      if (tpc > 32768) tpc = 32768;
    }
    if (sm_count > 0 && tpc > sm_count) tpc = tpc / sm_count * sm_count;                    // whole waves of token tiles
  }
};

size_t grads_workspace(int64_t T, int32_t d, int32_t V, int32_t R, int32_t K, int64_t chunk_tokens, int32_t dw_dtype, Mode mode) {
  if (T < 0 || d <= 0 || V <= 0 || R < 0 || K <= 0) return 0;
  if (chunk_tokens < 128) chunk_tokens = 128;
  int64_t tiles = (chunk_tokens + 127) / 128;
  const int64_t mt = max_tiles_of(T, R);
  if (tiles > mt) tiles = mt;
  return carve(nullptr, T, d, V, R, K, mode).head_bytes + (size_t)tiles * chunk_tile_bytes(d, V) +
         (dw_dtype == AERO_BF16 && tiles < mt ? dw_sums_bytes(d, V) : 0);
}

struct Call {
  aero_ctx* ctx;
  int64_t T;
  int32_t d, V, R, K;
  const void *H, *W;
  const int32_t* ids;
  const float* logits;
  const float* tlse;
  const int64_t* cs;
  const float* w;
  const uint8_t* keep;
  AeroListed ex;
};

// What the caller has already takes the workspace's place.
Ws with_given(Ws s, const Call& c) {
  if (c.ex.z) {
    s.y = const_cast<int32_t*>(c.ids);
    s.wrow = const_cast<float*>(c.ex.row_weights);
    s.z = const_cast<float*>(c.ex.z);
  }
  return s;
}

int check_call(const aero_cfg* cfg, const Call& c, const void* ws) {
  if (!c.ctx || !cfg || c.T < 0 || c.T >= (int64_t)1 << 31 || c.d <= 0 || c.V <= 0 || c.R < 0 || c.K <= 0) return AERO_ERR_INVALID;
  if (!c.W || !c.cs || !ws || !aero_aligned256(ws)) return AERO_ERR_INVALID;
  if (c.T > 0 && (!c.H || !c.ids || !c.logits)) return AERO_ERR_INVALID;
  if (c.R > 0 && (!c.w || !c.keep)) return AERO_ERR_INVALID;
  if (cfg->dtype != AERO_BF16 && cfg->dtype != AERO_FP32) return AERO_ERR_UNSUPPORTED;
  if (c.K > kMaxK) return AERO_ERR_UNSUPPORTED;
  if (cfg->dtype == AERO_BF16 ? c.d % 64 != 0 : c.d > kMaxD32) return AERO_ERR_UNSUPPORTED;
  if (!aero_aligned16(c.H) || !aero_aligned16(c.W)) return AERO_ERR_INVALID;
  return AERO_OK;
}

// dW of type dw_dtype: fp32 (added to or overwritten) or, for bf16 rows, bf16 (overwritten)
int check_dw(const aero_cfg* cfg, const void* dH, const void* dW, int32_t dw_dtype, int accumulate_dW) {
  if (!aero_aligned16(dH) || !aero_aligned16(dW)) return AERO_ERR_INVALID;
  if (dw_dtype != AERO_FP32 && dw_dtype != AERO_BF16) return AERO_ERR_UNSUPPORTED;
  if (dw_dtype == AERO_BF16 && cfg->dtype != AERO_BF16) return AERO_ERR_UNSUPPORTED;
  if (dw_dtype == AERO_BF16 && accumulate_dW) return AERO_ERR_INVALID;
  return AERO_OK;
}

unsigned row_grid(int64_t T) {
  const long long blocks = (T + 7) / 8;
  return (unsigned)(blocks < 65535 ? blocks : 65535);
}

RowsArgs rows_of(const Call& c, const Ws& s, float* lse, float* kl, bool partials, float grad_scale) {
  RowsArgs a = {};
  a.ls = {c.K, c.ids, c.logits, c.tlse, kl, s.z, s.entry, partials ? s.partials : nullptr};
  a.T = c.T; a.d = c.d; a.V = c.V; a.R = c.R; a.H = c.H; a.W = c.W; a.cs = c.cs; a.keep = c.keep; a.wrow = s.wrow;
  a.lse = lse; a.y = s.y; a.g = s.g; a.grad_scale = grad_scale; a.plan = s.plan;
  return a;
}

int start(const Call& c, const Ws& s, float* lse, float* kl, void* dH16, bool partials, long long chunk_tiles = 0) {
  aero_ctx* ctx = c.ctx;
  AERO_CUDA_TRY(cudaMemsetAsync(s.zero, 0, zero_bytes((size_t)chunk_tiles), ctx->stream));
  if (partials) AERO_CUDA_TRY(cudaMemsetAsync(s.partials, 0, s.n_partials * kPartialStride * sizeof(double), ctx->stream));
  if (c.T == 0 || c.ex.z) return AERO_OK;
  const FirstArgs f = {c.T, c.d, c.V, c.R, c.K, c.ids, c.logits, c.cs, c.w, c.keep, s.y, s.wrow, lse, kl, static_cast<__nv_bfloat16*>(dH16),
                       ctx->d_status};
  distill_first_kernel<<<row_grid(c.T), 256, 0, ctx->stream>>>(f);
  ctx->launches += 1;
  AERO_CUDA_TRY(cudaGetLastError());
  return AERO_OK;
}

// ---- fp32 path -------------------------------------------------------------------------------------------
// list logits and rows: all T at once, 8 per block
int rows_fp32(const RowsArgs& a, aero_ctx* ctx, bool given) {
  const unsigned blocks = row_blocks_of((a.T + 7) / 8);
  if (!given) distill_dots_kernel<float><<<dim3(blocks, (unsigned)((a.ls.K + kDots - 1) / kDots)), 256, 0, ctx->stream>>>(a);
  distill_rows_kernel<<<blocks, 256, 0, ctx->stream>>>(a);
  ctx->launches += given ? 1 : 2;
  AERO_CUDA_TRY(cudaGetLastError());
  return AERO_OK;
}

// a block per row of `rows`, of as many warps (up to eight) as have work and room for their staged rows
template <typename K>
int launch_fp32(aero_ctx* ctx, K kernel, const Fp32Args& f, long long rows, long long others) {
  const int d = f.r.d;
  const size_t per_warp = (size_t)32 * (d | 1) * sizeof(float);
  int warps = (int)((200 * 1024) / per_warp);
  if (warps > 8) warps = 8;
  if (warps > (others + 31) / 32) warps = (int)((others + 31) / 32);
  const size_t smem = d * sizeof(float) + warps * per_warp;
  AERO_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  kernel<<<(unsigned)rows, warps * 32, smem, ctx->stream>>>(f);
  ctx->launches += 1;
  AERO_CUDA_TRY(cudaGetLastError());
  return AERO_OK;
}

int fwd_fp32(const Call& c, const Ws& s, float* lse, float* kl, float* loss, float* metrics) {
  aero_ctx* ctx = c.ctx;
  int rc = start(c, s, lse, kl, nullptr, loss != nullptr);
  if (rc) return rc;
  if (c.T > 0 && c.R > 0) {
    RowsArgs a = rows_of(c, s, lse, kl, loss != nullptr, 1.f);
    a.ls.entry = nullptr;
    if ((rc = launch_fp32(ctx, fp32_rows_kernel<1, false>, {a, nullptr, nullptr, 0}, c.T, c.V))) return rc;
    if ((rc = rows_fp32(a, ctx, c.ex.z != nullptr))) return rc;
  }
  if (!loss) return AERO_OK;
  return aero_loss_finalize(ctx, s.partials, (int)s.n_partials, kPartialStride, loss, metrics, 0);
}

int bwd_fp32(const Call& c, const Ws& s, const float* lse, float grad_scale, float* dH, float* dW, int accumulate) {
  aero_ctx* ctx = c.ctx;
  int rc = start(c, s, nullptr, nullptr, nullptr, false);
  if (rc) return rc;
  if (c.T == 0 || c.R == 0) {
    if (!accumulate) AERO_CUDA_TRY(cudaMemsetAsync(dW, 0, (size_t)c.V * c.d * sizeof(float), ctx->stream));
    if (c.T > 0) AERO_CUDA_TRY(cudaMemsetAsync(dH, 0, (size_t)c.T * c.d * sizeof(float), ctx->stream));
    return AERO_OK;
  }
  AERO_CUDA_TRY(cudaMemsetAsync(s.g, 0, (size_t)c.T * sizeof(float), ctx->stream));      // rows of dropped rollouts
  Fp32Args f = {rows_of(c, s, const_cast<float*>(lse), nullptr, false, grad_scale), dH, dW, accumulate};
  f.r.ysum = s.ysum;
  if ((rc = rows_fp32(f.r, ctx, c.ex.z != nullptr))) return rc;
  // sums of a row: 4 or 32 registers a lane (T = 160, d = 57, V = 831, forward and gradients: 189 or 267 us)
  const bool narrow = c.d <= 128;
  rc = launch_fp32(ctx, narrow ? fp32_rows_kernel<4, true> : fp32_rows_kernel<kMaxD32 / 32, true>, f, c.T, c.V);
  if (rc) return rc;
  return launch_fp32(ctx, narrow ? fp32_vocabulary_kernel<4> : fp32_vocabulary_kernel<kMaxD32 / 32>, f, c.V, c.T);
}

// ---- bf16 path on the tensor cores -------------------------------------------------------------------------
struct Grads {
  float grad_scale;
  __nv_bfloat16* dH;
  float* dW;                 // fp32 dW, or the sums of a bf16 one
  __nv_bfloat16* dW16;       // bf16 dW that the products write themselves, or NULL
  int accumulate;
  long long tpc;
  __nv_bfloat16* block;      // [tpc][ldz / 64][128][64]
};

int lmhead_launch(const Call& c, const Ws& s, lmhead::Params p, const CUtensorMap& tmH, const CUtensorMap& tmW,
                  const CUtensorMap& tmDZ, Mode mode) {
  aero_ctx* ctx = c.ctx;
  p.T = c.T; p.d = c.d; p.V = c.V; p.R = c.R;
  p.tile_row = s.tiles.tile_row; p.tile_valid = s.tiles.tile_valid; p.n_tiles = s.tiles.n_tiles;
  p.y = s.y; p.status = ctx->d_status; p.plan = s.plan;
  p.sync_ctr = reinterpret_cast<unsigned int*>(s.zero);
  // the meetings pay over launches of many units per pair; a few milliseconds do not drift apart (without / with them:
  // loss of 1000 tokens 371 / 379 us, step of 300 tokens 492 / 513, of 4096 tokens at d = 3584 8090 / 8150)
  p.nsync = c.T > (int64_t)ctx->sm_count * lmhead::BM ? aero_nsync(ctx) : 0;
  p.w_hint = aero_w_hint(ctx, mode != kFwd); p.k_zigzag = aero_k_zigzag(ctx);
  auto kern = mode == kFwd ? lmhead::lmhead_kernel<lmhead::MODE_FWD>
                           : (mode == kBoth ? lmhead::lmhead_kernel<lmhead::MODE_FWD_P> : lmhead::lmhead_kernel<lmhead::MODE_DZ>);
  if (c.ex.z_gain && mode != kBwd) {
    kern = mode == kFwd ? lmhead::lmhead_kernel<lmhead::MODE_FWD_GAIN> : lmhead::lmhead_kernel<lmhead::MODE_FWD_P_GAIN>;
    p.z_gain = c.ex.z_gain;
  }
  AERO_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)lmhead::SMEM_BYTES));
  const int pairs = ctx->sm_count / 2 > 0 ? ctx->sm_count / 2 : 1;
  kern<<<2 * pairs, lmhead::THREADS, lmhead::SMEM_BYTES, ctx->stream>>>(tmH, tmW, tmDZ, p);
  ctx->launches += 1;
  AERO_CUDA_TRY(cudaGetLastError());
  return AERO_OK;
}

int plan_launch(const Call& c, const Ws& s, long long begin, long long tpc, bool pairs, void* clear, size_t clear_bytes) {
  aero_ctx* ctx = c.ctx;
  PlanArgs a = {};
  a.n_tiles = s.tiles.n_tiles; a.tile_begin = (int)begin; a.tpc = (int)tpc;
  a.pairs = ctx->sm_count / 2 > 0 ? ctx->sm_count / 2 : 1;
  a.nvt = (c.V + lmhead::BN - 1) / lmhead::BN;
  a.v_lo = aero_vsplit(ctx, c.d, c.V);
  a.v_hi = ctx->tune_vsplit > 0 || s.v_hi < a.v_lo ? a.v_lo : s.v_hi;
  a.workers = pairs ? a.pairs : ctx->sm_count;
  a.rows_per_worker = pairs ? 2 : 1;
  a.n_nt = (c.d + gemmbwd::BN - 1) / gemmbwd::BN;
  a.nkb = (int)(ldz_of(c.V) / gemmbwd::BK);
  a.k_hi = s.k_hi < a.nkb ? s.k_hi : a.nkb;
  a.d = c.d;
  a.plan = s.plan;
  a.dW = static_cast<uint4*>(clear);
  a.dW_vecs = clear_bytes / 16;
  plan_kernel<<<clear ? 4 * ctx->sm_count : 1, 256, 0, ctx->stream>>>(a);
  ctx->launches += 1;
  AERO_CUDA_TRY(cudaGetLastError());
  return AERO_OK;
}

int fwd_tc(const Call& c, const Ws& s, float* lse, float* kl, float* loss, float* metrics) {
  aero_ctx* ctx = c.ctx;
  int rc = start(c, s, lse, kl, nullptr, loss != nullptr);
  if (rc) return rc;
  if (c.T > 0 && c.R > 0) {
    if ((rc = aero_build_tiles(ctx, c.T, c.R, c.cs, c.keep, lmhead::BM, s.tiles))) return rc;
    if ((rc = plan_launch(c, s, 0, s.tiles.max_tiles, false, nullptr, 0))) return rc;
    const CUtensorMapDataType BF = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    CUtensorMap tmH, tmW;
    if ((rc = aero_make_tmap_2d(ctx, &tmH, BF, 2, c.H, c.T, c.d, c.d, lmhead::BM, lmhead::BK))) return rc;
    if ((rc = aero_make_tmap_2d(ctx, &tmW, BF, 2, c.W, c.V, c.d, c.d, lmhead::BNH, lmhead::BK))) return rc;
    lmhead::Params p = {};
    p.tile_begin = 0; p.tile_end = s.tiles.max_tiles;
    p.xstate = s.xstate;
    if ((rc = lmhead_launch(c, s, p, tmH, tmW, tmH, kFwd))) return rc;
    RowsArgs a = rows_of(c, s, lse, kl, loss != nullptr, 1.f);
    a.xstate = s.xstate;
    a.tile_row = s.tiles.tile_row; a.tile_valid = s.tiles.tile_valid; a.n_tiles = s.tiles.n_tiles;
    a.tile_begin = 0; a.tile_end = s.tiles.max_tiles;
    const unsigned blocks = row_blocks_of((int64_t)s.tiles.max_tiles * kUnitsPerTile);
    if (!c.ex.z) distill_dots_kernel<__nv_bfloat16><<<dim3(blocks, (unsigned)((c.K + kDots - 1) / kDots)), 256, 0, ctx->stream>>>(a);
    distill_rows_kernel<<<blocks, 256, 0, ctx->stream>>>(a);
    ctx->launches += c.ex.z ? 1 : 2;
    AERO_CUDA_TRY(cudaGetLastError());
  }
  if (!loss) return AERO_OK;
  return aero_loss_finalize(ctx, s.partials, (int)s.n_partials, kPartialStride, loss, metrics, 0);
}

// Gradients, with (kBoth) or without (kBwd: lse is given) the forward.
int grads_tc(const Call& c, const Ws& s, Mode mode, float* lse, float* kl, const Grads& gr) {
  aero_ctx* ctx = c.ctx;
  const int d = c.d, V = c.V;
  const long long tpc = gr.tpc, listed_tiles = mode == kBoth ? tpc : 0;
  const bool sums = mode == kBoth && !c.ex.between;      // (the loss of another caller is its own)
  int rc = start(c, s, mode == kBoth ? lse : nullptr, kl, gr.dH, sums, listed_tiles);
  if (rc) return rc;
  if (c.T == 0 || c.R == 0) {
    if (gr.dW16) AERO_CUDA_TRY(cudaMemsetAsync(gr.dW16, 0, (size_t)V * d * 2, ctx->stream));
    else if (!gr.accumulate) AERO_CUDA_TRY(cudaMemsetAsync(gr.dW, 0, (size_t)V * d * sizeof(float), ctx->stream));
    return AERO_OK;
  }
  if ((rc = aero_build_tiles(ctx, c.T, c.R, c.cs, c.keep, lmhead::BM, s.tiles))) return rc;
  const long long ldz = ldz_of(V);
  const uint64_t nblk = (uint64_t)(ldz / 64);
  __nv_bfloat16* Hl = gr.block + (size_t)tpc * lmhead::BM * (size_t)ldz;
  const bool pairs = aero_gemm_pairs(ctx, d);
  const CUtensorMapDataType BF = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  CUtensorMap tmH, tmW, tmDZ_st, tmDZ_k, tmDZ_mn, tmW_mn, tmH_mn;
  const uint32_t bn = (uint32_t)((pairs ? gemmbwd::PBNH : gemmbwd::BN) / 64);   // CTA pairs: each stages half of the B slab
  if ((rc = aero_make_tmap_2d(ctx, &tmH, BF, 2, c.H, c.T, d, d, lmhead::BM, 64))) return rc;
  if ((rc = aero_make_tmap_2d(ctx, &tmW, BF, 2, c.W, V, d, d, lmhead::BNH, 64))) return rc;
  if ((rc = aero_make_tmap_dz(ctx, &tmDZ_st, gr.block, (uint64_t)tpc, nblk, 32, 1))) return rc;
  if ((rc = aero_make_tmap_dz(ctx, &tmDZ_k, gr.block, (uint64_t)tpc, nblk, gemmbwd::BM, 1))) return rc;
  if ((rc = aero_make_tmap_dz(ctx, &tmDZ_mn, gr.block, (uint64_t)tpc, nblk, 64, gemmbwd::BM / 64))) return rc;
  if ((rc = aero_make_tmap_blocked(ctx, &tmW_mn, c.W, V, d, d, 64, bn))) return rc;
  if ((rc = aero_make_tmap_blocked(ctx, &tmH_mn, Hl, tpc * lmhead::BM, d, d, 64, bn))) return rc;
  auto k_dh = pairs ? gemmbwd::gemm_pair_kernel<gemmbwd::KIND_DH> : gemmbwd::gemm_kernel<gemmbwd::KIND_DH>;
  auto k_dw = pairs ? gemmbwd::gemm_pair_kernel<gemmbwd::KIND_DW> : gemmbwd::gemm_kernel<gemmbwd::KIND_DW>;
  const int dh_smem = (int)(pairs ? gemmbwd::PSMEM_BYTES : gemmbwd::SMEM_BYTES), dw_smem = dh_smem + (int)gemmbwd::OUT_EXTRA;
  AERO_CUDA_TRY(cudaFuncSetAttribute(k_dh, cudaFuncAttributeMaxDynamicSharedMemorySize, dh_smem));
  AERO_CUDA_TRY(cudaFuncSetAttribute(k_dw, cudaFuncAttributeMaxDynamicSharedMemorySize, dw_smem));
  CUtensorMap tmO = tmDZ_k;
  if (gr.dW16) rc = aero_make_tmap_2d(ctx, &tmO, BF, 2, gr.dW16, V, d, d, 32, 64);
  else if (!gr.accumulate) rc = aero_make_tmap_2d(ctx, &tmO, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, gr.dW, V, d, d, 32, 32);
  if (rc) return rc;
  const int gemm_grid = pairs ? 2 * (ctx->sm_count / 2 > 0 ? ctx->sm_count / 2 : 1) : ctx->sm_count;
  const bool many = c.T > (int64_t)ctx->sm_count * lmhead::BM;

  for (long long begin = 0; begin < s.tiles.max_tiles; begin += tpc) {
    const long long end = begin + tpc < s.tiles.max_tiles ? begin + tpc : s.tiles.max_tiles;
    const unsigned row_blocks = row_blocks_of((end - begin) * kUnitsPerTile);
    void* clear = begin > 0 || gr.accumulate ? nullptr : (gr.dW16 ? static_cast<void*>(gr.dW16) : static_cast<void*>(gr.dW));
    if (begin > 0) AERO_CUDA_TRY(cudaMemsetAsync(s.zero, 0, zero_bytes((size_t)listed_tiles), ctx->stream));
    if ((rc = plan_launch(c, s, begin, tpc, pairs, clear, (size_t)V * d * (gr.dW16 ? 2 : 4)))) return rc;
    RowsArgs a = rows_of(c, s, lse, kl, sums, gr.grad_scale);
    a.tile_row = s.tiles.tile_row; a.tile_valid = s.tiles.tile_valid; a.n_tiles = s.tiles.n_tiles;
    a.tile_begin = (int)begin; a.tile_end = (int)end; a.Hl = Hl;
    lmhead::Params p = {};
    p.tile_begin = (int)begin; p.tile_end = (int)end;
    p.dz = gr.block; p.ldz = ldz;
    if (!c.ex.z) {
      distill_dots_kernel<__nv_bfloat16><<<dim3(row_blocks, (unsigned)((c.K + kDots - 1) / kDots)), 256, 0, ctx->stream>>>(a);
      ctx->launches += 1;
    }
    BlockArgs b = {a, gr.block, (int)nblk, (V + lmhead::BN - 1) / lmhead::BN, s.shift, s.outside};
    if (mode == kBoth) {
      p.xstate = s.xstate; p.shift_out = s.shift;
      p.range_rows = s.range_rows; p.range_count = s.range_count; p.range_seen = s.range_seen; p.range_cap = kRangeCap;
      if ((rc = lmhead_launch(c, s, p, tmH, tmW, tmDZ_st, kBoth))) return rc;
      a.xstate = s.xstate;
      distill_rows_kernel<<<row_blocks, 256, 0, ctx->stream>>>(a);
      distill_scale_kernel<<<dim3((unsigned)b.nvt, (unsigned)(end - begin < 64 ? end - begin : 64)), 256, 0, ctx->stream>>>(b);
      RangeArgs f = {};
      f.rows = s.range_rows; f.count = s.range_count; f.cap = kRangeCap; f.dz = gr.block; f.nblk = (int)nblk;
      f.tile_row = s.tiles.tile_row; f.tile_begin = (int)begin; f.T = c.T; f.d = d; f.V = V; f.y = s.y;
      f.lse = lse; f.g = s.g; f.grad_scale = gr.grad_scale;
      f.H = static_cast<const __nv_bfloat16*>(c.H); f.W = static_cast<const __nv_bfloat16*>(c.W);
      range_fix_kernel<<<2 * ctx->sm_count, 256, 0, ctx->stream>>>(f);
      ctx->launches += 3;
    } else {
      a.ysum = s.ysum;
      b.a.ysum = s.ysum;
      distill_rows_kernel<<<row_blocks, 256, 0, ctx->stream>>>(a);
      ctx->launches += 1;
      p.lse_in = lse; p.g_in = s.g; p.grad_scale = gr.grad_scale;
      if ((rc = lmhead_launch(c, s, p, tmH, tmW, tmDZ_st, kBwd))) return rc;
      distill_outside_kernel<<<row_blocks_of((end - begin) * lmhead::BM), 256, 0, ctx->stream>>>(b);
      ctx->launches += 1;
    }
    distill_scatter_kernel<<<row_blocks, 256, 0, ctx->stream>>>(b);
    if (c.ex.between && (rc = c.ex.between(c.ex.arg))) return rc;
    if (c.ex.row_factor) {
      distill_scale_rows_kernel<<<row_blocks, 256, 0, ctx->stream>>>(a, c.ex.row_factor);
      ctx->launches += 1;
    }
    gemmbwd::Params gp = {};
    gp.T = c.T; gp.d = d; gp.V = V; gp.ldz = ldz;
    gp.tile_row = s.tiles.tile_row; gp.tile_valid = s.tiles.tile_valid; gp.n_tiles = s.tiles.n_tiles;
    gp.tile_begin = (int)begin; gp.tpc = (int)tpc;
    gp.dH = gr.dH; gp.dW = gr.dW; gp.status = ctx->d_status;
    gp.out = gr.dW16 ? gemmbwd::kOutBf16 : (begin == 0 && !gr.accumulate ? gemmbwd::kOutFp32 : 0);
    gp.h_local = 1;
    gp.row_scale = c.ex.row_factor;
    gp.ksplit = s.k_hi > 1 ? s.plan + 1 : nullptr; gp.part = s.part;
    gp.nsync = many ? aero_gemm_sync(ctx) : 0;
    gp.sync_ctr = reinterpret_cast<unsigned int*>(s.zero) + 4;
    k_dh<<<gemm_grid, gemmbwd::THREADS, dh_smem, ctx->stream>>>(tmDZ_k, tmW_mn, tmDZ_k, gp);
    if (s.k_hi > 1) {
      distill_join_dh_kernel<<<dim3(row_blocks, (unsigned)((d + 255) / 256)), 256, 0, ctx->stream>>>(a, s.plan + 1, s.part, c.ex.row_factor, gr.dH);
      ctx->launches += 1;
    }
    gp.sync_ctr = reinterpret_cast<unsigned int*>(s.zero) + 8;
    k_dw<<<gemm_grid, gemmbwd::THREADS, dw_smem, ctx->stream>>>(tmDZ_mn, tmH_mn, tmO, gp);
    ctx->launches += 3;
    AERO_CUDA_TRY(cudaGetLastError());
  }
  return AERO_OK;
}

// Shared by the two calls with gradients: where dW goes, the chunks, the rounding of its sums at the end.
int grads_call(const Call& c, const Ws& s, Mode mode, const Room& room, float* lse, float* kl, float grad_scale, void* dH,
               void* dW, int32_t dw_dtype, int accumulate_dW) {
  Grads gr = {};
  gr.grad_scale = grad_scale;
  gr.dH = static_cast<__nv_bfloat16*>(dH);
  gr.accumulate = accumulate_dW;
  gr.tpc = room.tpc;
  const size_t sums = room.sums ? dw_sums_bytes(c.d, c.V) : 0;
  gr.block = reinterpret_cast<__nv_bfloat16*>(s.rest + sums);
  if (room.sums) gr.dW = reinterpret_cast<float*>(s.rest);
  else if (dw_dtype == AERO_BF16) gr.dW16 = static_cast<__nv_bfloat16*>(dW);
  else gr.dW = static_cast<float*>(dW);
  const int rc = grads_tc(c, s, mode, lse, kl, gr);
  if (rc || !room.sums) return rc;
  dw_to_bf16_kernel<<<8 * c.ctx->sm_count, 256, 0, c.ctx->stream>>>(reinterpret_cast<const float4*>(gr.dW),
                                                                    static_cast<uint2*>(dW), (size_t)c.V * c.d / 4);
  c.ctx->launches += 1;
  AERO_CUDA_TRY(cudaGetLastError());
  return AERO_OK;
}

}  // namespace

int aero_distill_fwd_listed(const AeroListed& ex, aero_ctx* ctx, const aero_cfg* cfg, int64_t T, int32_t d, int32_t V,
                            int32_t R, int32_t K, const void* H, const void* W, const int32_t* ids, const float* logits,
                            const float* teacher_lse, const int64_t* cs, const float* w, const uint8_t* keep, float* lse,
                            float* kl, float* loss, float* metrics, void* workspace, size_t workspace_bytes) {
  const Call c = {ctx, T, d, V, R, K, H, W, ids, logits, teacher_lse, cs, w, keep, ex};
  int rc = check_call(cfg, c, workspace);
  if (rc) return rc;
  if (T > 0 && (!lse || !kl)) return AERO_ERR_INVALID;
  if (workspace_bytes < aero_distill_fwd_workspace_bytes(T, d, V, R, K)) return AERO_ERR_WORKSPACE;
  if ((rc = aero_check_ctx(ctx))) return rc;
  const Ws s = with_given(carve(workspace, T, d, V, R, K, kFwd), c);
  return cfg->dtype == AERO_FP32 ? fwd_fp32(c, s, lse, kl, loss, metrics) : fwd_tc(c, s, lse, kl, loss, metrics);
}

int aero_distill_bwd_listed(const AeroListed& ex, aero_ctx* ctx, const aero_cfg* cfg, int64_t T, int32_t d, int32_t V,
                            int32_t R, int32_t K, const void* H, const void* W, const int32_t* ids, const float* logits,
                            const float* teacher_lse, const int64_t* cs, const float* w, const uint8_t* keep,
                            const float* lse, float grad_scale, void* dH, void* dW, int32_t dw_dtype, int accumulate_dW,
                            void* workspace, size_t workspace_bytes) {
  const Call c = {ctx, T, d, V, R, K, H, W, ids, logits, teacher_lse, cs, w, keep, ex};
  int rc = check_call(cfg, c, workspace);
  if (rc) return rc;
  if (!dW || (T > 0 && (!lse || !dH))) return AERO_ERR_INVALID;
  if ((rc = check_dw(cfg, dH, dW, dw_dtype, accumulate_dW))) return rc;
  const Ws s = with_given(carve(workspace, T, d, V, R, K, kBwd), c);
  if (workspace_bytes < s.head_bytes) return AERO_ERR_WORKSPACE;
  const Room room(workspace_bytes - s.head_bytes, T, d, V, R, dw_dtype == AERO_BF16, ctx->sm_count);
  if (cfg->dtype == AERO_BF16 && room.tpc < 1) return AERO_ERR_WORKSPACE;
  if ((rc = aero_check_ctx(ctx))) return rc;
  if (cfg->dtype == AERO_FP32)
    return bwd_fp32(c, s, lse, grad_scale, static_cast<float*>(dH), static_cast<float*>(dW), accumulate_dW);
  return grads_call(c, s, kBwd, room, const_cast<float*>(lse), nullptr, grad_scale, dH, dW, dw_dtype, accumulate_dW);
}

int aero_distill_fwd_bwd_listed(const AeroListed& ex, aero_ctx* ctx, const aero_cfg* cfg, int64_t T, int32_t d, int32_t V,
                                int32_t R, int32_t K, const void* H, const void* W, const int32_t* ids, const float* logits,
                                const float* teacher_lse, const int64_t* cs, const float* w, const uint8_t* keep, float* lse,
                                float* kl, float* loss, float* metrics, float grad_scale, void* dH, void* dW,
                                int32_t dw_dtype, int accumulate_dW, void* workspace, size_t workspace_bytes) {
  const Call c = {ctx, T, d, V, R, K, H, W, ids, logits, teacher_lse, cs, w, keep, ex};
  int rc = check_call(cfg, c, workspace);
  if (rc) return rc;
  if (!dW || (T > 0 && (!lse || !kl || !dH))) return AERO_ERR_INVALID;
  if ((rc = check_dw(cfg, dH, dW, dw_dtype, accumulate_dW))) return rc;
  const Ws s = with_given(carve(workspace, T, d, V, R, K, kBoth), c);
  if (workspace_bytes < s.head_bytes) return AERO_ERR_WORKSPACE;
  const Room room(workspace_bytes - s.head_bytes, T, d, V, R, dw_dtype == AERO_BF16, ctx->sm_count);
  if (cfg->dtype == AERO_BF16 && room.tpc < 1) return AERO_ERR_WORKSPACE;
  if ((rc = aero_check_ctx(ctx))) return rc;
  if (cfg->dtype == AERO_FP32) {
    if ((rc = fwd_fp32(c, s, lse, kl, loss, metrics))) return rc;
    return bwd_fp32(c, s, lse, grad_scale, static_cast<float*>(dH), static_cast<float*>(dW), accumulate_dW);
  }
  if ((rc = grads_call(c, s, kBoth, room, lse, kl, grad_scale, dH, dW, dw_dtype, accumulate_dW)) || !loss) return rc;
  return aero_loss_finalize(ctx, s.partials, (int)s.n_partials, kPartialStride, loss, metrics, 0);
}

int aero_distill_check(aero_ctx* ctx, const aero_cfg* cfg, int64_t T, int32_t d, int32_t V, int32_t R, int32_t K, const void* H,
                       const void* W, const int32_t* ids, const float* logits, const int64_t* cs, const float* w, const uint8_t* keep,
                       const void* workspace) {
  return check_call(cfg, {ctx, T, d, V, R, K, H, W, ids, logits, nullptr, cs, w, keep, {}}, workspace);
}

int aero_distill_check_grads(const aero_cfg* cfg, int64_t T, const void* dH, const void* dW, int32_t dw_dtype, int accumulate_dW) {
  if (!dW || (T > 0 && !dH)) return AERO_ERR_INVALID;
  return check_dw(cfg, dH, dW, dw_dtype, accumulate_dW);
}

bool aero_distill_bwd_fits(const aero_cfg* cfg, int64_t T, int32_t d, int32_t V, int32_t R, int32_t K, int32_t dw_dtype,
                           size_t workspace_bytes) {
  const size_t head = carve(nullptr, T, d, V, R, K, kBwd).head_bytes;
  return workspace_bytes >= head &&
         (cfg->dtype == AERO_FP32 || Room(workspace_bytes - head, T, d, V, R, dw_dtype == AERO_BF16, 0).tpc >= 1);
}

bool aero_distill_one_chunk(const aero_ctx* ctx, int64_t T, int32_t d, int32_t V, int32_t R, int32_t K, int32_t dw_dtype,
                            size_t workspace_bytes) {
  const size_t head = carve(nullptr, T, d, V, R, K, kBoth).head_bytes;
  return workspace_bytes >= head &&
         Room(workspace_bytes - head, T, d, V, R, dw_dtype == AERO_BF16, ctx->sm_count).tpc >= max_tiles_of(T, R);
}

extern "C" {

size_t aero_distill_fwd_workspace_bytes(int64_t T, int32_t d, int32_t V, int32_t R, int32_t K) {
  if (T < 0 || d <= 0 || V <= 0 || R < 0 || K <= 0) return 0;
  return carve(nullptr, T, d, V, R, K, kFwd).head_bytes;
}

size_t aero_distill_bwd_workspace_bytes(int64_t T, int32_t d, int32_t V, int32_t R, int32_t K, int64_t chunk_tokens,
                                        int32_t dw_dtype) {
  return grads_workspace(T, d, V, R, K, chunk_tokens, dw_dtype, kBwd);
}

size_t aero_distill_fwd_bwd_workspace_bytes(int64_t T, int32_t d, int32_t V, int32_t R, int32_t K, int64_t chunk_tokens,
                                            int32_t dw_dtype) {
  return grads_workspace(T, d, V, R, K, chunk_tokens, dw_dtype, kBoth);
}

int aero_distill_fwd(aero_ctx* ctx, const aero_cfg* cfg, int64_t T, int32_t d, int32_t V, int32_t R, int32_t K,
                     const void* H, const void* W, const int32_t* ids, const float* logits, const float* teacher_lse,
                     const int64_t* cs, const float* w, const uint8_t* keep,
                     float* lse, float* kl, float* loss, float* metrics, void* workspace, size_t workspace_bytes) {
  AeroRange nv("aero_distill_fwd");
  if (!loss) return AERO_ERR_INVALID;
  return aero_distill_fwd_listed({}, ctx, cfg, T, d, V, R, K, H, W, ids, logits, teacher_lse, cs, w, keep, lse, kl, loss,
                                 metrics, workspace, workspace_bytes);
}

int aero_distill_bwd(aero_ctx* ctx, const aero_cfg* cfg, int64_t T, int32_t d, int32_t V, int32_t R, int32_t K,
                     const void* H, const void* W, const int32_t* ids, const float* logits, const float* teacher_lse,
                     const int64_t* cs, const float* w, const uint8_t* keep, const float* lse, float grad_scale,
                     void* dH, void* dW, int32_t dw_dtype, int accumulate_dW, void* workspace, size_t workspace_bytes) {
  AeroRange nv("aero_distill_bwd");
  return aero_distill_bwd_listed({}, ctx, cfg, T, d, V, R, K, H, W, ids, logits, teacher_lse, cs, w, keep, lse, grad_scale,
                                 dH, dW, dw_dtype, accumulate_dW, workspace, workspace_bytes);
}

int aero_distill_fwd_bwd(aero_ctx* ctx, const aero_cfg* cfg, int64_t T, int32_t d, int32_t V, int32_t R, int32_t K,
                         const void* H, const void* W, const int32_t* ids, const float* logits, const float* teacher_lse,
                         const int64_t* cs, const float* w, const uint8_t* keep,
                         float* lse, float* kl, float* loss, float* metrics, float grad_scale,
                         void* dH, void* dW, int32_t dw_dtype, int accumulate_dW, void* workspace,
                         size_t workspace_bytes) {
  AeroRange nv("aero_distill_fwd_bwd");
  if (!loss) return AERO_ERR_INVALID;
  return aero_distill_fwd_bwd_listed({}, ctx, cfg, T, d, V, R, K, H, W, ids, logits, teacher_lse, cs, w, keep, lse, kl, loss,
                                     metrics, grad_scale, dH, dW, dw_dtype, accumulate_dW, workspace, workspace_bytes);
}

}  // extern "C"
