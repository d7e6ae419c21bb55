// The preference loss on pairs of rollouts through the lm_head.  With logp_t the log-prob of token t of rollout i,
//   r_i = sum_t (logp_t - ref_t), or its mean over the scored tokens;   m_p = beta (r_c - r_r) - margin
//   loss = sum_p u_p l(m_p),   coef_i = (sum_{p: c = i} - sum_{p: r = i}) u_p beta l'(m_p) [/ scored tokens of i]
//   dz_tv = grad_scale coef_i (1[v = y_t] - p_tv),   dH = dz W,   dW (+)= dz^T H
// Everything between H, W and the log-probs, and between coef and dH, dW, is distillation's with one listed token per row
// (distill.cuh); what is here are the sums over rollouts and pairs.  The products are what a call takes its time for, and
// their row tiles are of 128, so the scored rows of the rollouts in pairs are first gathered into one run (prompts, padding and
// rollouts in no pair cost nothing but that copy): at T = 333 with 253 scored rows two tiles instead of three.
// The gradient of a row needs all rows of all of its rollout's pairs, so the one-call step computes the log-probs of a chunk, then
// coef, then the chunk's gradients; rows that do not fit one chunk of the workspace take the separate passes, which compute the
// logits twice (8 d V FLOP per token instead of 6).  The kernels here read 16 bytes per token, 8 bytes per pair and rollout and
// copy the rows: microseconds beside the products.  All sums are in 64 bits and have a fixed order.
#include "distill.cuh"
#include "entry.cuh"
#include "loss_common.cuh"
#include "vec.cuh"

#include <type_traits>

namespace {

constexpr int kPairBlocks = 148, kThreads = 128, kPlanThreads = 1024;

struct PrefArgs {
  long long T;
  int d, V, R, P;
  int elem;                       // bytes of an element of H
  int backward;                   // the backward alone: rollouts whose coef is not 0, lse given
  int kind, mean;
  double beta, margin, smoothing;
  const void* H;
  const int32_t* y;
  const float* ref;               // NULL: no reference
  const int64_t* cs;
  const int32_t* pairs;           // [P][2]
  const float* weight;            // NULL: 1 / counted pairs
  const float* coef_in;
  const float* lse_in;
  // gathered rows: src[p] is the token row of gathered row p, rollout i owns off[i] .. off[i + 1]
  uint8_t* keep;                  // rollouts in some counted pair
  int* counted;                   // pairs counted
  int64_t* off;                   // [R + 1]
  int64_t* run;                   // [2]: 0 and the number of gathered rows
  uint8_t* one;                   // [1]: 1, the run is kept
  int32_t* src;                   // [T]
  uint8_t* Hg;                    // [T][d]
  int32_t* yg;                    // [T]
  float* lseg;                    // [T]
  float* klg;                     // [T] minus the log-probs
  uint8_t* dHg;                   // [T][d], with gradients
  float* row_weights;             // [T] -grad_scale coef of the row's rollout
  float* ones;                    // [T] 1
  float* zeros;                   // [T] 0: the listed tokens' teacher logits
  float* zg;                      // [T] logits of the rows' targets
  float* gain;                    // [T] forward of bf16 rows: factors of the rows' logits, less one
  float grad_scale;
  const void* W;
  double* r;                      // [R] log ratios
  double* slope;                  // [P] d loss / d r_chosen
  double* partials;               // [kPairBlocks][kPartialStride]
  float* logp;
  float* lse;
  float* ratio;
  float* margins;
  float* coef;
  uint32_t* status;
};

// A pair that counts: both rollouts exist.  (-1, -1) is an empty place.
__device__ __forceinline__ bool pair_of(const PrefArgs& a, int p, int* c, int* r) {
  const int2 q = reinterpret_cast<const int2*>(a.pairs)[p];
  *c = q.x;
  *r = q.y;
  return *c >= 0 && *c < a.R && *r >= 0 && *r < a.R;
}

// Rows t0 .. t1 of a rollout that is used, none where its offsets leave [0, T].
__device__ __forceinline__ bool rows_of(const PrefArgs& a, int i, long long* t0, long long* t1) {
  *t0 = a.cs[i];
  *t1 = a.cs[i + 1];
  return a.keep[i] != 0 && *t0 >= 0 && *t1 >= *t0 && *t1 <= a.T;
}
__device__ __forceinline__ bool scored(const PrefArgs& a, long long t) { return a.y[t] >= 0 && a.y[t] < a.V; }

// f(t, whether the row is scored, scored rows of its group of 32 as a word) by the 32 lanes of a warp, four groups' loads at a time;
// LANES 1: by one thread, row by row.
template <int LANES, typename F>
__device__ __forceinline__ void for_rows(const PrefArgs& a, long long t0, long long t1, int lane, F&& f) {
  if constexpr (LANES == 1) {
    for (long long t = t0; t < t1; ++t) {
      const bool s = scored(a, t);
      f(t, s, s ? 1u : 0u);
    }
  } else {
    for (long long t = t0; t < t1; t += 128) {
      bool s[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) s[q] = t + 32 * q + lane < t1 && scored(a, t + 32 * q + lane);
#pragma unroll
      for (int q = 0; q < 4; ++q) f(t + 32 * q + lane, s[q], __ballot_sync(0xffffffffu, s[q]));
    }
  }
}
// Scored rows of the rollouts i, i + step, ..., to off; with LANES 32 a warp, with 1 a thread for each.
template <int LANES>
__device__ __forceinline__ void count_rows(const PrefArgs& a) {
  const int lane = threadIdx.x % LANES;
  for (int i = threadIdx.x / LANES; i < a.R; i += kPlanThreads / LANES) {
    long long t0, t1, rows = 0;
    if (rows_of(a, i, &t0, &t1)) {
      bool wrong = false;
      for_rows<LANES>(a, t0, t1, lane, [&](long long t, bool s, unsigned word) {
        rows += __popc(word);
        wrong |= t < t1 && !s && a.y[t] != AERO_NO_TOKEN;
      });
      if (wrong) aero_raise(a.status, AERO_ST_BAD_TARGET);
    } else if (lane == 0 && !(t0 >= 0 && t1 >= t0 && t1 <= a.T)) {
      aero_raise(a.status, AERO_ST_BAD_OFFSETS);
    }
    if (lane == 0) a.off[i + 1] = rows;
  }
}
template <int LANES>
__device__ __forceinline__ void list_rows(const PrefArgs& a) {
  const int lane = threadIdx.x % LANES;
  for (int i = threadIdx.x / LANES; i < a.R; i += kPlanThreads / LANES) {
    long long t0, t1, at = a.off[i];
    if (rows_of(a, i, &t0, &t1))
      for_rows<LANES>(a, t0, t1, lane, [&](long long t, bool s, unsigned word) {
        if (s) a.src[at + (LANES == 1 ? 0 : __popc(word & ((1u << lane) - 1u)))] = (int32_t)t;
        at += __popc(word);
      });
  }
}

// One block: which rollouts are used, where their scored rows go, and the list of these rows.  (6 us for a few rollouts of hundreds of
// tokens; a rollout takes far less time here than the products of one token.)
__global__ void __launch_bounds__(kPlanThreads) pref_plan_kernel(PrefArgs a) {
  __shared__ long long sums[32];
  __shared__ int total;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) total = 0;
  for (int i = threadIdx.x; i < a.R; i += kPlanThreads) a.keep[i] = a.backward && a.coef_in[i] != 0.f ? 1 : 0;
  __syncthreads();
  int n = 0;
  bool bad = false;
  for (int p = threadIdx.x; p < a.P; p += kPlanThreads) {
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
  if (lane == 0 && n) atomicAdd(&total, n);
  if (bad) aero_raise(a.status, AERO_ST_BAD_PAIR);
  __syncthreads();
  // scored rows of each rollout (at most T in all where offsets do not overlap), then their running sums
  // (a thread for a rollout where a warp would mostly idle)
  const bool brief = a.T < 32ll * a.R;
  if (brief) count_rows<1>(a);
  else count_rows<32>(a);
  __syncthreads();
  long long carry = 0;
  for (int base = 0; base < a.R; base += kPlanThreads) {
    const int i = base + threadIdx.x;
    long long v = i < a.R ? a.off[i + 1] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long u = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += u;
    }
    if (lane == 31) sums[warp] = v;
    __syncthreads();
    if (warp == 0) {
      long long s = sums[lane];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += u;
      }
      sums[lane] = s;
    }
    __syncthreads();
    v += carry + (warp > 0 ? sums[warp - 1] : 0);
    if (i < a.R) a.off[i + 1] = v;
    carry += sums[31];
    __syncthreads();
  }
  if (carry > a.T) {                                // offsets that overlap: no rollout has tokens
    if (threadIdx.x == 0) aero_raise(a.status, AERO_ST_BAD_OFFSETS);
    for (int i = threadIdx.x; i < a.R; i += kPlanThreads) a.keep[i] = a.off[i + 1] = 0;
    carry = 0;
  }
  if (threadIdx.x == 0) {
    a.off[0] = 0;
    a.run[0] = 0;
    a.run[1] = carry;
    *a.one = 1;
    *a.counted = total;
  }
  __syncthreads();
  if (brief) list_rows<1>(a);
  else list_rows<32>(a);
}

// Each product of 16 terms is added to the accumulator with what does not fit its 24 bits cut off, towards zero.  A dense sum of
// d / 16 of them comes out short by about d / 16 times kCut of itself, on average, and log-sum-exp with it: a token's log-prob has an
// error of 1e-6 to 5e-6 from it, which matters only where the log-probs of a whole rollout are added up.  kCut is a fit to the mean
// error of log-probs of normal H and W (1.60e-8 at d = 1536, 1.53e-8 at d = 3584), not a bound: dense inputs of other
// distributions need 1.48e-8 to 1.72e-8.  Walking d both ways (k_zigzag) makes it hold wherever along d the large columns are; sums of
// fewer or shorter terms lose less (CutOff).
constexpr float kCut = 1.55e-8f;
// How much a sum of these products of 16 loses to the tensor cores' accumulation, against a dense sum: the products of a row of H and
// its target's row of W are added up in steps of 16 as the tensor cores do, with what falls below the 24 bits of each partial sum counted.
// In dense rows that is 2.4e-8 to 4.4e-8 of the partial sums (normal, shifted, heavy-tailed, d = 1536 and 3584); in rows of which one
// column in 16, or 16 in 128, is not zero 2.5e-9 to 3.2e-9, where log-sum-exp loses as much less; of whole numbers 0.  A step that is
// below the accumulator's last two bits is dropped whole, before it is added.  (Mean error of a log-prob in such rows, d = 1536 and 3584:
// as if they were dense 1.7e-6 and 4.4e-6, with no correction -2e-7 to -6e-7, with this one at most 1.2e-7.)
constexpr float kDenseLoss = 1.7e-8f;
struct CutOff {
  float carry = 0.f, lost = 0.f, size = 0.f;
  // s: the sum of 8 neighbouring products, if there are any; a pair of lanes has a step's 16
  __device__ void add(float s, bool any, int lane) {
    s += __shfl_xor_sync(0xffffffffu, s, 1);
    float v = s;
#pragma unroll
    for (int o = 2; o < 32; o <<= 1) {
      const float u = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += u;
    }
    const float up = __shfl_up_sync(0xffffffffu, v, 2);
    const float before = carry + (lane >= 2 ? up : 0.f), sum = __fadd_rz(before, s);
    const bool falls = fabsf(before) >= fabsf(s);
    const float rest = falls ? s - (sum - before) : before - (sum - s);
    if (fabsf(s) > 0x1p-25f * fabsf(before)) lost += fabsf(rest);
    if (any) size += fabsf(sum);
    carry += __shfl_sync(0xffffffffu, v, 31);
  }
  // (a row without products to look at: as dense)
  __device__ float gain(int d) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      lost += __shfl_xor_sync(0xffffffffu, lost, o);
      size += __shfl_xor_sync(0xffffffffu, size, o);
    }
    return kCut * (float)(d / 16) * fminf(lost / (size * kDenseLoss), 1.f);
  }
};

// A warp per row.  GATHER: the row of H into the run, its target with the target's logit and, for the backward alone, lse and
// weight; else the run's row of dH to its own.
template <typename T, bool GATHER>
__global__ void __launch_bounds__(256) pref_rows_kernel(PrefArgs a, T* dH) {
  const int lane = threadIdx.x & 31, d = a.d;
  const long long n = a.run[1];
  if (GATHER && !a.backward) {                      // rows that are not scored keep these
    for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < a.T; t += (long long)gridDim.x * 256) a.logp[t] = a.lse[t] = 0.f;
  }
  for (long long p = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); p < n; p += (long long)gridDim.x * 8) {
    const long long t = a.src[p];
    const T* from = GATHER ? static_cast<const T*>(a.H) + t * d : reinterpret_cast<const T*>(a.dHg) + p * d;
    T* to = GATHER ? reinterpret_cast<T*>(a.Hg) + p * d : dH + t * d;
    const int v = GATHER ? a.y[t] : 0;
    const T* w = static_cast<const T*>(a.W) + (long long)v * d;
    float z = 0.f;
    CutOff cut;
    const bool watch = GATHER && sizeof(T) == 2 && !a.backward;
    const auto part = [&](auto vec) {
      constexpr int VEC = decltype(vec)::value;
#pragma unroll 4
      for (int e0 = 0; e0 < d; e0 += 32 * VEC) {
        const int e = e0 + lane * VEC;
        float s = 0.f;
        if (e < d) {
          float x[VEC], y[VEC];
          rowvec::load<T, VEC>(from + e, x);
          if (GATHER) {
            rowvec::load<T, VEC>(w + e, y);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
              z = fmaf(x[i], y[i], z);
              s = fmaf(x[i], y[i], s);
            }
          }
          rowvec::store<T, VEC>(to + e, x);
        }
        if (watch) cut.add(s, e < d, lane);
      }
    };
    if (d % rowvec::Elem<T>::kVec == 0) part(std::integral_constant<int, rowvec::Elem<T>::kVec>());
    else part(std::integral_constant<int, 1>());
    if (GATHER) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
      const float gain = watch ? cut.gain(d) : 0.f;
      if (lane == 0) {
        if (watch) a.gain[p] = gain;
        a.yg[p] = v;
        a.zg[p] = z;
        a.ones[p] = 1.f;
        a.zeros[p] = 0.f;
        if (a.backward) {
          a.lseg[p] = a.lse_in[t];
          a.row_weights[p] = -a.grad_scale * a.coef_in[aero_owner(a.off, a.R, p)];
        }
      }
    }
  }
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

// A gathered row's outputs (the log-probs arrive negated), and its part of the log ratio.
__device__ __forceinline__ double token_term(const PrefArgs& a, long long p) {
  const long long t = a.src[p];
  const float lp = 0.f - a.klg[p];
  a.logp[t] = lp;
  a.lse[t] = a.lseg[p];
  return (double)lp - (a.ref ? (double)a.ref[t] : 0.0);
}
// What pair p adds to the sum of slopes of rollout i.
__device__ __forceinline__ double slope_of(const PrefArgs& a, int p, int i) {
  const int2 q = reinterpret_cast<const int2*>(a.pairs)[p];
  return (q.x == i ? a.slope[p] : 0.0) - (q.y == i ? a.slope[p] : 0.0);
}

// A block per rollout: its log ratio.
__global__ void __launch_bounds__(kThreads) pref_ratio_kernel(PrefArgs a) {
  __shared__ double sh[kThreads / 32];
  for (int i = blockIdx.x; i < a.R; i += gridDim.x) {
    const long long p0 = a.off[i], p1 = a.off[i + 1];
    double sum = 0.0;
    for (long long p = p0 + threadIdx.x; p < p1; p += kThreads) sum += token_term(a, p);
    sum = block_sum(sum, sh);
    if (threadIdx.x == 0) {
      if (a.mean && p1 > p0) sum /= (double)(p1 - p0);
      a.r[i] = sum;
      a.ratio[i] = (float)sum;
    }
  }
}

// Margin, loss and slope of one pair; its part of the sums.
__device__ __forceinline__ void pair_term(const PrefArgs& a, int p, int n, double (&part)[kPartialStride]) {
  int c, r;
  double slope = 0.0, m = 0.0;
  if (pair_of(a, p, &c, &r)) {
    const double u = a.weight ? (double)a.weight[p] : 1.0 / n, rc = a.r[c], rr = a.r[r];
    m = a.beta * (rc - rr) - a.margin;
    double l;
    if (a.kind == AERO_PREF_LOGISTIC) {
      const double e = exp(-fabs(m)), s = log1p(e);                  // softplus(-|m|)
      const double down = m > 0.0 ? e / (1.0 + e) : 1.0 / (1.0 + e); // sigmoid(-m)
      // (a part without weight counts nothing, also where the margin is infinite)
      l = (a.smoothing < 1.0 ? (1.0 - a.smoothing) * (fmax(-m, 0.0) + s) : 0.0) + (a.smoothing > 0.0 ? a.smoothing * (fmax(m, 0.0) + s) : 0.0);
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

__global__ void __launch_bounds__(kThreads) pref_pairs_kernel(PrefArgs a) {
  __shared__ double sh[kThreads / 32];
  double part[kPartialStride] = {0.0, 0.0, 0.0, 0.0, 0.0};
  const int n = *a.counted;
  for (int p = blockIdx.x * kThreads + threadIdx.x; p < a.P; p += gridDim.x * kThreads) pair_term(a, p, n, part);
  for (int k = 0; k < kPartialStride; ++k) {
    const double s = block_sum(part[k], sh);
    if (threadIdx.x == 0) a.partials[(size_t)blockIdx.x * kPartialStride + k] = s;
  }
}

// A block per rollout walks all pairs in order for its own.  (A rollout is in few of them, but a list per rollout would take a sort
// to have a fixed order.  Of 4000 rollouts 2000 pairs are lost in the noise, 20000 take 75 us, 65536 280 and 262144 1100; the products
// of as many tokens, at 2 us each of the whole GPU for d = 1536, V = 151936, are milliseconds.)
__global__ void __launch_bounds__(kThreads) pref_coef_kernel(PrefArgs a) {
  __shared__ double sh[kThreads / 32];
  for (int i = blockIdx.x; i < a.R; i += gridDim.x) {
    double sum = 0.0;
    if (a.keep[i]) {
#pragma unroll 4
      for (int p = threadIdx.x; p < a.P; p += kThreads) sum += slope_of(a, p, i);
    }
    sum = block_sum(sum, sh);
    const long long p0 = a.off[i], p1 = a.off[i + 1];
    if (a.mean && p1 > p0) sum /= (double)(p1 - p0);
    const float coef = (float)sum;
    if (threadIdx.x == 0) a.coef[i] = coef;
    for (long long p = p0 + threadIdx.x; p < p1; p += kThreads) a.row_weights[p] = -a.grad_scale * coef;
  }
}

// The three kernels above in one block, for calls small enough that it takes no longer than the launches that it saves: a warp per
// rollout, a thread per pair.  (A step of 333 tokens, d = 1536, V = 151936: the three and the sum of the records 16 us and the gaps
// between them, this one 8.)
constexpr int kOneWarps = 32;
__global__ void __launch_bounds__(kOneWarps * 32) pref_loss_kernel(PrefArgs a, float* loss, float* metrics) {
  __shared__ double sh[kOneWarps][kPartialStride];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const auto warp_sum = [](double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
  };
  for (int i = warp; i < a.R; i += kOneWarps) {
    const long long p0 = a.off[i], p1 = a.off[i + 1];
    double sum = 0.0;
#pragma unroll 4
    for (long long p = p0 + lane; p < p1; p += 32) sum += token_term(a, p);
    sum = warp_sum(sum);
    if (lane == 0) {
      if (a.mean && p1 > p0) sum /= (double)(p1 - p0);
      a.r[i] = sum;
      a.ratio[i] = (float)sum;
    }
  }
  __syncthreads();
  double part[kPartialStride] = {0.0, 0.0, 0.0, 0.0, 0.0};
  const int n = *a.counted;
  for (int p = threadIdx.x; p < a.P; p += kOneWarps * 32) pair_term(a, p, n, part);
  for (int k = 0; k < kPartialStride; ++k) {
    part[k] = warp_sum(part[k]);
    if (lane == 0) sh[warp][k] = part[k];
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double tot[kPartialStride] = {0.0, 0.0, 0.0, 0.0, 0.0};
    for (int w = 0; w < kOneWarps; ++w)
      for (int k = 0; k < kPartialStride; ++k) tot[k] += sh[w][k];
    *loss = (float)(-tot[0]);
    if (metrics) {
      const double nk = tot[4] > 0.0 ? tot[4] : 1.0;
      for (int k = 0; k < 3; ++k) metrics[k] = (float)(tot[1 + k] / nk);
      metrics[3] = (float)tot[4];
    }
  }
  for (int i = warp; i < a.R; i += kOneWarps) {
    double sum = 0.0;
    if (a.keep[i])
      for (int p = lane; p < a.P; p += 32) sum += slope_of(a, p, i);
    sum = warp_sum(sum);
    const long long p0 = a.off[i], p1 = a.off[i + 1];
    if (a.mean && p1 > p0) sum /= (double)(p1 - p0);
    const float coef = (float)sum;
    if (lane == 0) a.coef[i] = coef;
    for (long long p = p0 + lane; p < p1; p += 32) a.row_weights[p] = -a.grad_scale * coef;
  }
}
bool small_loss(const PrefArgs& a) { return a.T <= 8192 && a.R <= 1024 && (long long)a.R * a.P <= 1 << 16; }

struct Ws {
  PrefArgs a;                     // its buffers
  char* rest;
  size_t head_bytes;
};

// (elem: bytes of an element of H; 0: whichever needs more)
Ws carve(void* base, int64_t T, int32_t d, int32_t R, int32_t P, int elem, bool grads) {
  Ws s = {};
  char* p = static_cast<char*>(base);
  size_t off = 0;
  auto take = [&](size_t bytes) { char* q = p + off; off += aero_align_up(bytes, 256); return q; };
  const size_t Tn = (size_t)T + 1, rows = Tn * (size_t)d * (elem ? elem : 4);
  s.a.counted = reinterpret_cast<int*>(take(4));
  s.a.one = reinterpret_cast<uint8_t*>(take(1));
  s.a.run = reinterpret_cast<int64_t*>(take(16));
  s.a.keep = reinterpret_cast<uint8_t*>(take((size_t)R + 1));
  s.a.off = reinterpret_cast<int64_t*>(take(((size_t)R + 1) * 8));
  s.a.src = reinterpret_cast<int32_t*>(take(Tn * 4));
  s.a.yg = reinterpret_cast<int32_t*>(take(Tn * 4));
  s.a.lseg = reinterpret_cast<float*>(take(Tn * 4));
  s.a.klg = reinterpret_cast<float*>(take(Tn * 4));
  s.a.row_weights = reinterpret_cast<float*>(take(Tn * 4));
  s.a.zeros = reinterpret_cast<float*>(take(Tn * 4));
  s.a.ones = reinterpret_cast<float*>(take(Tn * 4));
  s.a.zg = reinterpret_cast<float*>(take(Tn * 4));
  s.a.gain = reinterpret_cast<float*>(take(Tn * 4));
  s.a.r = reinterpret_cast<double*>(take(((size_t)R + 1) * 8));
  s.a.slope = reinterpret_cast<double*>(take(((size_t)P + 1) * 8));
  s.a.partials = reinterpret_cast<double*>(take((size_t)kPairBlocks * kPartialStride * 8));
  s.a.Hg = reinterpret_cast<uint8_t*>(take(rows));
  if (grads) s.a.dHg = reinterpret_cast<uint8_t*>(take(rows));
  s.rest = p + off;
  s.head_bytes = off;
  return s;
}

int elem_of(const aero_cfg* cfg) { return cfg && cfg->dtype == AERO_BF16 ? 2 : 4; }

int grid_for(long long n, int per, int most) {
  const long long blocks = (n + per - 1) / per;
  return (int)(blocks < 1 ? 1 : (blocks < most ? blocks : most));
}

constexpr int32_t kMost = 1 << 30;        // pairs, rollouts: the kernels' indexes step past the last one in 32 bits

int check_pref(const aero_pref_cfg* pc, int32_t P, const int32_t* pairs) {
  if (!pc || P < 0 || (P > 0 && !pairs)) return AERO_ERR_INVALID;
  if (P > kMost) return AERO_ERR_UNSUPPORTED;
  if (pc->kind != AERO_PREF_LOGISTIC && pc->kind != AERO_PREF_SQUARE && pc->kind != AERO_PREF_HINGE) return AERO_ERR_UNSUPPORTED;
  if (!(fabsf(pc->beta) < INFINITY) || !(fabsf(pc->margin) < INFINITY) || !(pc->label_smoothing >= 0.f && pc->label_smoothing <= 1.f))
    return AERO_ERR_INVALID;
  if (reinterpret_cast<uintptr_t>(pairs) % 8) return AERO_ERR_INVALID;
  return AERO_OK;
}

// One call: the user's arrays, the workspace, and the pieces that the three entry points put together.
struct Call {
  aero_ctx* ctx;
  const aero_cfg* cfg;
  Ws s;
  const void* W;
  float *loss, *metrics;

  int check(const void* workspace) {
    if (!cfg || !workspace || s.a.R < 0) return AERO_ERR_INVALID;
    if (s.a.R > kMost) return AERO_ERR_UNSUPPORTED;
    // (as the calls below check them; H and y are the caller's, the rest stands for what the workspace holds)
    return aero_distill_check(ctx, cfg, s.a.T, s.a.d, s.a.V, s.a.R, 1, s.a.H, W, s.a.y, reinterpret_cast<const float*>(workspace), s.a.cs,
                              reinterpret_cast<const float*>(workspace), static_cast<const uint8_t*>(workspace), workspace);
  }
  int check_forward(const aero_pref_cfg* pc, const void* workspace) {
    const PrefArgs& p = s.a;
    int rc = check_pref(pc, p.P, p.pairs);
    if (rc) return rc;
    if (!loss || (p.R > 0 && (!p.ratio || !p.coef)) || (p.P > 0 && !p.margins) || (p.T > 0 && (!p.logp || !p.lse))) return AERO_ERR_INVALID;
    return check(workspace);
  }

  int gather() {
    const cudaStream_t stream = ctx->stream;
    pref_plan_kernel<<<1, kPlanThreads, 0, stream>>>(s.a);
    if (s.a.T > 0) {
      const int grid = grid_for(s.a.T, 8, 16 * ctx->sm_count);
      if (cfg->dtype == AERO_BF16) pref_rows_kernel<__nv_bfloat16, true><<<grid, 256, 0, stream>>>(s.a, nullptr);
      else pref_rows_kernel<float, true><<<grid, 256, 0, stream>>>(s.a, nullptr);
    }
    ctx->launches += s.a.T > 0 ? 2 : 1;
    AERO_CUDA_TRY(cudaGetLastError());
    return AERO_OK;
  }

  void given(AeroListed& ex) const {
    ex.z = s.a.zg;
    ex.row_weights = s.a.ones;
  }

  int forward(const AeroListed& ex, size_t room) {
    return aero_distill_fwd_listed(ex, ctx, cfg, s.a.T, s.a.d, s.a.V, 1, 1, s.a.Hg, W, s.a.yg, s.a.zeros, nullptr,
                                   s.a.run, s.a.ones, s.a.one, s.a.lseg, s.a.klg, nullptr, nullptr, s.rest,
                                   room);
  }

  // What stands between the log-probs and the gradients.
  int pairs() {
    if (small_loss(s.a)) {
      pref_loss_kernel<<<1, kOneWarps * 32, 0, ctx->stream>>>(s.a, loss, metrics);
      ctx->launches += 1;
      AERO_CUDA_TRY(cudaGetLastError());
      return AERO_OK;
    }
    const int rollouts = grid_for(s.a.R, 1, 65535);
    if (s.a.R > 0) pref_ratio_kernel<<<rollouts, kThreads, 0, ctx->stream>>>(s.a);
    const int blocks = grid_for(s.a.P, kThreads, kPairBlocks);
    pref_pairs_kernel<<<blocks, kThreads, 0, ctx->stream>>>(s.a);
    if (s.a.R > 0) pref_coef_kernel<<<rollouts, kThreads, 0, ctx->stream>>>(s.a);
    ctx->launches += s.a.R > 0 ? 3 : 1;
    AERO_CUDA_TRY(cudaGetLastError());
    return aero_loss_finalize(ctx, s.a.partials, blocks, kPartialStride, loss, metrics, 0);
  }
  static int between(void* self) { return static_cast<Call*>(self)->pairs(); }

  int backward(void* dW, int32_t dw_dtype, int accumulate_dW, size_t room) {
    AeroListed ex;
    given(ex);
    (cfg->dtype == AERO_BF16 ? ex.row_factor : ex.row_weights) = s.a.row_weights;
    return aero_distill_bwd_listed(ex, ctx, cfg, s.a.T, s.a.d, s.a.V, 1, 1, s.a.Hg, W, s.a.yg, s.a.zeros, nullptr,
                                   s.a.run, s.a.ones, s.a.one, s.a.lseg, 1.f, s.a.dHg, dW, dw_dtype,
                                   accumulate_dW, s.rest, room);
  }

  int scatter(void* dH) {
    if (s.a.T == 0) return AERO_OK;
    AERO_CUDA_TRY(cudaMemsetAsync(dH, 0, (size_t)s.a.T * s.a.d * s.a.elem, ctx->stream));
    const int grid = grid_for(s.a.T, 8, 16 * ctx->sm_count);
    if (cfg->dtype == AERO_BF16) pref_rows_kernel<__nv_bfloat16, false><<<grid, 256, 0, ctx->stream>>>(s.a, static_cast<__nv_bfloat16*>(dH));
    else pref_rows_kernel<float, false><<<grid, 256, 0, ctx->stream>>>(s.a, static_cast<float*>(dH));
    ctx->launches += 1;
    AERO_CUDA_TRY(cudaGetLastError());
    return AERO_OK;
  }
};

Call call_of(aero_ctx* ctx, const aero_cfg* cfg, const aero_pref_cfg* pc, int64_t T, int32_t d, int32_t V, int32_t R, int32_t P,
             const void* H, const void* W, const int32_t* y, const int64_t* cs, void* workspace, bool grads) {
  Call c = {ctx, cfg, carve(workspace, T > 0 ? T : 0, d > 0 ? d : 0, R > 0 ? R : 0, P > 0 ? P : 0, elem_of(cfg), grads), W, nullptr,
            nullptr};
  PrefArgs& a = c.s.a;
  a.T = T; a.d = d; a.V = V; a.R = R; a.P = P; a.elem = elem_of(cfg); a.H = H; a.W = W; a.y = y; a.cs = cs;
  if (ctx) a.status = ctx->d_status;
  if (pc) {
    a.kind = pc->kind; a.mean = pc->mean; a.beta = pc->beta; a.margin = pc->margin; a.smoothing = pc->label_smoothing;
  }
  return c;
}

}  // namespace

extern "C" {

void aero_pref_cfg_default(aero_pref_cfg* pc) {
  if (!pc) return;
  pc->kind = AERO_PREF_LOGISTIC; pc->mean = 0; pc->beta = 0.1f; pc->margin = 0.f; pc->label_smoothing = 0.f;
}

size_t aero_pref_fwd_workspace_bytes(int64_t T, int32_t d, int32_t V, int32_t R, int32_t P) {
  const size_t inner = aero_distill_fwd_workspace_bytes(T, d, V, 1, 1);
  return inner == 0 || R < 0 || P < 0 ? 0 : carve(nullptr, T, d, R, P, 0, false).head_bytes + inner;
}

size_t aero_pref_bwd_workspace_bytes(int64_t T, int32_t d, int32_t V, int32_t R, int64_t chunk_tokens, int32_t dw_dtype) {
  const size_t inner = aero_distill_bwd_workspace_bytes(T, d, V, 1, 1, chunk_tokens, dw_dtype);
  return inner == 0 || R < 0 ? 0 : carve(nullptr, T, d, R, 0, 0, true).head_bytes + inner;
}

size_t aero_pref_fwd_bwd_workspace_bytes(int64_t T, int32_t d, int32_t V, int32_t R, int32_t P, int64_t chunk_tokens, int32_t dw_dtype) {
  size_t inner = aero_distill_fwd_bwd_workspace_bytes(T, d, V, 1, 1, chunk_tokens, dw_dtype);
  if (inner == 0 || R < 0 || P < 0) return 0;
  for (const size_t other : {aero_distill_fwd_workspace_bytes(T, d, V, 1, 1),
                             aero_distill_bwd_workspace_bytes(T, d, V, 1, 1, chunk_tokens, dw_dtype)})
    if (other > inner) inner = other;
  return carve(nullptr, T, d, R, P, 0, true).head_bytes + inner;
}

int aero_pref_fwd(aero_ctx* ctx, const aero_cfg* cfg, const aero_pref_cfg* pc, int64_t T, int32_t d, int32_t V, int32_t R, int32_t P,
                  const void* H, const void* W, const int32_t* y, const float* ref_logp, const int64_t* cs, const int32_t* pairs,
                  const float* pair_weight, float* logp, float* lse, float* ratio, float* margin, float* coef, float* loss,
                  float* metrics, void* workspace, size_t workspace_bytes) {
  AeroRange nv("aero_pref_fwd");
  Call c = call_of(ctx, cfg, pc, T, d, V, R, P, H, W, y, cs, workspace, false);
  PrefArgs& a = c.s.a;
  a.ref = ref_logp; a.pairs = pairs; a.weight = pair_weight; a.logp = logp; a.lse = lse; a.ratio = ratio; a.margins = margin; a.coef = coef;
  c.loss = loss; c.metrics = metrics;
  int rc = c.check_forward(pc, workspace);
  if (rc) return rc;
  const size_t room = workspace_bytes > c.s.head_bytes ? workspace_bytes - c.s.head_bytes : 0;
  if (room < aero_distill_fwd_workspace_bytes(T, d, V, 1, 1)) return AERO_ERR_WORKSPACE;
  if ((rc = aero_check_ctx(ctx)) || (rc = c.gather())) return rc;
  AeroListed ex;
  ex.z_gain = c.s.a.gain;
  c.given(ex);
  if ((rc = c.forward(ex, room))) return rc;
  return c.pairs();
}

int aero_pref_bwd(aero_ctx* ctx, const aero_cfg* cfg, int64_t T, int32_t d, int32_t V, int32_t R, const void* H, const void* W,
                  const int32_t* y, const int64_t* cs, const float* coef, const float* lse, float grad_scale, void* dH, void* dW,
                  int32_t dw_dtype, int accumulate_dW, void* workspace, size_t workspace_bytes) {
  AeroRange nv("aero_pref_bwd");
  Call c = call_of(ctx, cfg, nullptr, T, d, V, R, 0, H, W, y, cs, workspace, true);
  c.s.a.backward = 1; c.s.a.coef_in = coef; c.s.a.lse_in = lse; c.s.a.grad_scale = grad_scale;
  if ((R > 0 && !coef) || (T > 0 && !lse)) return AERO_ERR_INVALID;
  int rc = c.check(workspace);
  if (rc || (rc = aero_distill_check_grads(cfg, T, dH, dW, dw_dtype, accumulate_dW))) return rc;
  const size_t room = workspace_bytes > c.s.head_bytes ? workspace_bytes - c.s.head_bytes : 0;
  if (!aero_distill_bwd_fits(cfg, T, d, V, 1, 1, dw_dtype, room)) return AERO_ERR_WORKSPACE;
  if ((rc = aero_check_ctx(ctx)) || (rc = c.gather())) return rc;
  if ((rc = c.backward(dW, dw_dtype, accumulate_dW, room))) return rc;
  return c.scatter(dH);
}

int aero_pref_fwd_bwd(aero_ctx* ctx, const aero_cfg* cfg, const aero_pref_cfg* pc, int64_t T, int32_t d, int32_t V, int32_t R,
                      int32_t P, const void* H, const void* W, const int32_t* y, const float* ref_logp, const int64_t* cs,
                      const int32_t* pairs, const float* pair_weight, float* logp, float* lse, float* ratio, float* margin,
                      float* coef, float* loss, float* metrics, float grad_scale, void* dH, void* dW, int32_t dw_dtype,
                      int accumulate_dW, void* workspace, size_t workspace_bytes) {
  AeroRange nv("aero_pref_fwd_bwd");
  Call c = call_of(ctx, cfg, pc, T, d, V, R, P, H, W, y, cs, workspace, true);
  PrefArgs& a = c.s.a;
  a.ref = ref_logp; a.pairs = pairs; a.weight = pair_weight; a.logp = logp; a.lse = lse; a.ratio = ratio; a.margins = margin; a.coef = coef;
  a.grad_scale = grad_scale;
  c.loss = loss; c.metrics = metrics;
  int rc = c.check_forward(pc, workspace);
  if (rc || (rc = aero_distill_check_grads(cfg, T, dH, dW, dw_dtype, accumulate_dW))) return rc;
  const size_t room = workspace_bytes > c.s.head_bytes ? workspace_bytes - c.s.head_bytes : 0;
  const bool one_chunk = cfg->dtype == AERO_BF16 && T > 0 && aero_distill_one_chunk(ctx, T, d, V, 1, 1, dw_dtype, room);
  if (!one_chunk && (room < aero_distill_fwd_workspace_bytes(T, d, V, 1, 1) || !aero_distill_bwd_fits(cfg, T, d, V, 1, 1, dw_dtype, room)))
    return AERO_ERR_WORKSPACE;
  if ((rc = aero_check_ctx(ctx)) || (rc = c.gather())) return rc;
  AeroListed ex;
  ex.z_gain = c.s.a.gain;
  c.given(ex);
  if (one_chunk) {
    ex.row_factor = a.row_weights;
    ex.between = Call::between;
    ex.arg = &c;
    rc = aero_distill_fwd_bwd_listed(ex, ctx, cfg, T, d, V, 1, 1, a.Hg, W, a.yg, a.zeros, nullptr, a.run,
                                     a.ones, a.one, a.lseg, a.klg, nullptr, nullptr, 1.f, a.dHg, dW, dw_dtype, accumulate_dW,
                                     c.s.rest, room);
  } else {
    if ((rc = c.forward(ex, room)) || (rc = c.pairs())) return rc;
    rc = c.backward(dW, dw_dtype, accumulate_dW, room);
  }
  return rc ? rc : c.scatter(dH);
}

}  // extern "C"
