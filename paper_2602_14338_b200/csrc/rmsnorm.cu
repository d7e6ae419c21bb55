// The policy model's final RMS norm, which makes the H that stage (b) reads, and its gradient,
// which takes the dH that stage (b) returns:
//   s = x + residual,  rstd = 1 / sqrt(mean(s^2) + eps),  h = s rstd gamma
//   ds = rstd (gamma dh - shat mean(gamma dh shat)) + dsum,   shat = s rstd
//   dgamma (+)= sum_t dh shat
// and the 8-bit form of the rows, q = round(h / scale), scale = max |h| / 127.
//
// Bound by memory: every row is read once and held in registers between the reduction and the outputs (so an
// output may be written over an input row by row).  In the forward, rows of up to 256 vectors of 16 bytes
// belong to a warp, which needs no barrier and has the whole row's loads in flight at once (16384 x 1536 bf16
// with a residual: 43 us against 50 us with a block per row); other rows belong to a block, which has its next
// row's loads in flight while it reduces the current one (16384 x 3584: 79 us, 5.9 TB/s, against 104 us without
// that).  A ring of rows in shared memory filled by bulk copies was tried and is slower (86 us, and 75 us
// instead of 54 us for the backward at 20011 x 1536): bytes in flight are not what is short.
#include "entry.cuh"
#include "vec.cuh"

#include <initializer_list>
#include <type_traits>

namespace {

constexpr int kMaxD = 16384;
constexpr int kBwdBlocks = 1184;      // blocks of the backward at most (their shares of dgamma are workspace)

struct FwdArgs {
  long long T;
  int d;
  const void* x;
  const void* residual;   // or NULL
  const void* gamma;      // NULL: no norm, the rows themselves are brought to 8 bits
  float eps;
  void* sum;              // any output may be NULL
  void* h;
  float* rstd;
  int8_t* q;
  float* q_scale;
};

struct BwdArgs {
  long long T;
  int d;
  const void* dh;
  const void* dsum;       // or NULL
  const void* s;
  const void* gamma;
  const float* rstd;
  void* dx;
  float* part;            // [gridDim.x][d]
};

// Block shapes: at most 256 threads while few vectors per thread suffice, so that several rows are in flight on
// an SM; the largest vector count of a kind goes up to kMaxD.  In the backward that form holds two rows, their next ones and
// dgamma's share and spills 0.7 to 1.5 KB a thread (8192 x 8192 bf16: 202 us, its bytes alone 82).
template <int VEC, int NV>
constexpr int max_threads() {
  return VEC == 1 ? 1024 : (NV * VEC == 32 ? 512 : 256);
}
// Blocks per SM the compiler is to make room for.  Measured (us; 1 / 2 / 3 / 4 / 5 blocks asked for): forward, 16384 x 3584 bf16
// with a residual 89 / 89 / 79 / 110 / 177; backward, 20011 x 1536 bf16 59 / 59 / 57 / 54 / 67, 16384 x 3584 118 / 94 / 143 / 141
// / 223: the registers are worth more than the blocks once rows have to be spilled.  fp32 rows: one block, others not measured.
template <int VEC, int NV>
constexpr int fwd_blocks() { return VEC == 8 && NV == 2 ? 3 : 1; }
template <int VEC, int NV>
constexpr int bwd_blocks() { return VEC == 8 ? (NV == 1 ? 4 : (NV == 2 ? 2 : 1)) : 1; }
constexpr int kWarps = 4;             // rows at a time per block of the warp kernel

// the larger of two, or NaN if either is (fmaxf would drop it)
__device__ __forceinline__ float max_or_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// sum and maximum over a warp, the same value in every lane (fixed order)
__device__ __forceinline__ float2 warp_sum_max(float sum, float mx) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    sum += __shfl_xor_sync(0xffffffffu, sum, o);
    mx = max_or_nan(mx, __shfl_xor_sync(0xffffffffu, mx, o));
  }
  return make_float2(sum, mx);
}

// ... and over the block's threads
__device__ __forceinline__ float2 block_sum_max(float sum, float mx, float2* sh) {
  const int warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
  const float2 v = warp_sum_max(sum, mx);
  if ((threadIdx.x & 31) == 0) sh[warp] = v;
  __syncthreads();
  float2 r = sh[0];
  for (int w = 1; w < nw; ++w) {
    r.x += sh[w].x;
    r.y = max_or_nan(r.y, sh[w].y);
  }
  return r;
}

// What a row's sum of squares and largest |s gamma| make of it.
struct RowScale {
  float rstd, amax, up, inv;
  __device__ RowScale(const FwdArgs& a, float2 red) {
    rstd = a.gamma ? 1.f / sqrtf(red.x / (float)a.d + a.eps) : 1.f;
    amax = red.y * rstd;                                      // (NaN if the row or gamma holds one)
    up = amax < 0x1p-100f ? 0x1p100f : 1.f;                  // keeps 127 / amax finite for the smallest rows
    inv = amax > 0.f ? 127.f / (amax * up) : 0.f;
  }
};

template <int VEC>
__device__ __forceinline__ void store_q(int8_t* p, const float (&f)[VEC], float up, float inv) {
  int8_t b[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const int v = __float2int_rn(f[e] * up * inv);       // (NaN becomes 0; the row's scale is then NaN)
    b[e] = (int8_t)max(-127, min(127, v));
  }
  if constexpr (VEC == 8) *reinterpret_cast<uint2*>(p) = *reinterpret_cast<uint2*>(b);
  else if constexpr (VEC == 4) *reinterpret_cast<uint32_t*>(p) = *reinterpret_cast<uint32_t*>(b);
  else p[0] = b[0];
}

// s and h of VEC elements to the outputs that are asked for.  The sum of two rows is kept in fp32 for the norm and
// rounded once on its way out.
template <typename T, int VEC>
__device__ __forceinline__ void write_outputs(const FwdArgs& a, long long t, int e0, float (&s)[VEC], const float (&g)[VEC],
                                              const RowScale& rs) {
  if (a.sum) rowvec::store<T, VEC>(static_cast<T*>(a.sum) + t * a.d + e0, s);
#pragma unroll
  for (int e = 0; e < VEC; ++e) s[e] = a.gamma ? s[e] * rs.rstd * g[e] : s[e];
  if (a.h) rowvec::store<T, VEC>(static_cast<T*>(a.h) + t * a.d + e0, s);
  if (a.q) store_q<VEC>(a.q + t * a.d + e0, s, rs.up, rs.inv);
}

// ---- a row per warp: lane i holds vectors i, i + 32, ... ---------------------------------------------------
template <typename T, int NV>
__global__ void __launch_bounds__(kWarps * 32) rmsnorm_fwd_warp_kernel(FwdArgs a) {
  constexpr int VEC = rowvec::Elem<T>::kVec;
  const int lane = threadIdx.x & 31;
  const T* gm = static_cast<const T*>(a.gamma);
  for (long long t = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5); t < a.T; t += (long long)gridDim.x * kWarps) {
    uint4 xr[NV], rr[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int e0 = (j * 32 + lane) * VEC;
      if (e0 < a.d) {
        xr[j] = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.x) + t * a.d + e0);
        if (a.residual) rr[j] = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.residual) + t * a.d + e0);
      }
    }
    auto row_sum = [&](int j, float (&s)[VEC], float (&g)[VEC]) {
      const int e0 = (j * 32 + lane) * VEC;
      rowvec::unpack(xr[j], s);
      if (a.residual) {
        float r[VEC];
        rowvec::unpack(rr[j], r);
#pragma unroll
        for (int e = 0; e < VEC; ++e) s[e] += r[e];
      }
      if (gm) rowvec::unpack(__ldg(reinterpret_cast<const uint4*>(gm + e0)), g);
    };
    float ss = 0.f, mx = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if ((j * 32 + lane) * VEC < a.d) {
        float s[VEC], g[VEC];
        row_sum(j, s, g);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          ss = fmaf(s[e], s[e], ss);
          if (a.q) mx = max_or_nan(mx, fabsf(gm ? s[e] * g[e] : s[e]));
        }
      }
    }
    const RowScale rs(a, warp_sum_max(ss, mx));
    if (lane == 0) {
      if (a.rstd) a.rstd[t] = rs.rstd;
      if (a.q_scale) a.q_scale[t] = rs.amax / 127.f;
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int e0 = (j * 32 + lane) * VEC;
      if (e0 < a.d) {
        float s[VEC], g[VEC];
        row_sum(j, s, g);
        write_outputs<T, VEC>(a, t, e0, s, g, rs);
      }
    }
  }
}

// ---- a row per block: thread i holds vectors i, i + blockDim, ... -------------------------------------------
template <typename T, int VEC, int NV>
__global__ void __launch_bounds__(max_threads<VEC, NV>(), fwd_blocks<VEC, NV>()) rmsnorm_fwd_kernel(FwdArgs a) {
  using Raw = typename rowvec::Raw<T, VEC>::type;
  __shared__ float2 sh[2][32];
  const T* gm = static_cast<const T*>(a.gamma);
  Raw gr[NV], xr[NV], rr[NV];
  auto fetch = [&](long long t) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int e0 = (j * blockDim.x + threadIdx.x) * VEC;
      if (e0 < a.d) {
        xr[j] = *reinterpret_cast<const Raw*>(static_cast<const T*>(a.x) + t * a.d + e0);
        if (a.residual) rr[j] = *reinterpret_cast<const Raw*>(static_cast<const T*>(a.residual) + t * a.d + e0);
      }
    }
  };
  fetch(blockIdx.x);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int e0 = (j * blockDim.x + threadIdx.x) * VEC;
    if (e0 < a.d && gm) gr[j] = *reinterpret_cast<const Raw*>(gm + e0);
  }
  int turn = 0;
  for (long long t = blockIdx.x; t < a.T; t += gridDim.x, turn ^= 1) {
    float s[NV][VEC];
    float ss = 0.f, mx = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int e0 = (j * blockDim.x + threadIdx.x) * VEC;
      if (e0 < a.d) {
        rowvec::open<T, VEC>(xr[j], s[j]);
        if (a.residual) {
          float r[VEC];
          rowvec::open<T, VEC>(rr[j], r);
#pragma unroll
          for (int e = 0; e < VEC; ++e) s[j][e] += r[e];
        }
      }
    }
    if (t + gridDim.x < a.T) fetch(t + gridDim.x);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int e0 = (j * blockDim.x + threadIdx.x) * VEC;
      if (e0 < a.d) {
        float g[VEC];
        if (gm) rowvec::open<T, VEC>(gr[j], g);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          ss = fmaf(s[j][e], s[j][e], ss);
          mx = max_or_nan(mx, fabsf(gm ? s[j][e] * g[e] : s[j][e]));
        }
      }
    }
    const RowScale rs(a, block_sum_max(ss, mx, sh[turn]));
    if (threadIdx.x == 0) {
      if (a.rstd) a.rstd[t] = rs.rstd;
      if (a.q_scale) a.q_scale[t] = rs.amax / 127.f;
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int e0 = (j * blockDim.x + threadIdx.x) * VEC;
      if (e0 < a.d) {
        float g[VEC];
        if (gm) rowvec::open<T, VEC>(gr[j], g);
        write_outputs<T, VEC>(a, t, e0, s[j], g, rs);
      }
    }
  }
}

template <typename T, int VEC, int NV>
__global__ void __launch_bounds__(max_threads<VEC, NV>(), bwd_blocks<VEC, NV>()) rmsnorm_bwd_kernel(BwdArgs a) {
  using Raw = typename rowvec::Raw<T, VEC>::type;
  __shared__ float2 sh[2][32];
  Raw gr[NV], sr[NV], hr[NV], ur[NV];
  float dg[NV][VEC], next_rstd = 0.f;
  auto fetch = [&](long long t) {
    next_rstd = a.rstd[t];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int e0 = (j * blockDim.x + threadIdx.x) * VEC;
      if (e0 < a.d) {
        sr[j] = *reinterpret_cast<const Raw*>(static_cast<const T*>(a.s) + t * a.d + e0);
        hr[j] = *reinterpret_cast<const Raw*>(static_cast<const T*>(a.dh) + t * a.d + e0);
        if (a.dsum) ur[j] = *reinterpret_cast<const Raw*>(static_cast<const T*>(a.dsum) + t * a.d + e0);
      }
    }
  };
  fetch(blockIdx.x);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int e0 = (j * blockDim.x + threadIdx.x) * VEC;
    if (e0 < a.d) gr[j] = *reinterpret_cast<const Raw*>(static_cast<const T*>(a.gamma) + e0);
#pragma unroll
    for (int e = 0; e < VEC; ++e) dg[j][e] = 0.f;
  }
  int turn = 0;
  for (long long t = blockIdx.x; t < a.T; t += gridDim.x, turn ^= 1) {
    const float rstd = next_rstd;
    float s[NV][VEC], dh[NV][VEC];
    Raw u[NV];
    float dot = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int e0 = (j * blockDim.x + threadIdx.x) * VEC;
      if (e0 < a.d) {
        rowvec::open<T, VEC>(sr[j], s[j]);
        rowvec::open<T, VEC>(hr[j], dh[j]);
        if (a.dsum) u[j] = ur[j];
      }
    }
    if (t + gridDim.x < a.T) fetch(t + gridDim.x);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int e0 = (j * blockDim.x + threadIdx.x) * VEC;
      if (e0 < a.d) {
        float g[VEC];
        rowvec::open<T, VEC>(gr[j], g);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          s[j][e] *= rstd;                                       // shat
          dg[j][e] = fmaf(dh[j][e], s[j][e], dg[j][e]);
          dh[j][e] *= g[e];
          dot = fmaf(dh[j][e], s[j][e], dot);
        }
      }
    }
    const float c = block_sum_max(dot, 0.f, sh[turn]).x / (float)a.d;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int e0 = (j * blockDim.x + threadIdx.x) * VEC;
      if (e0 < a.d) {
        float o[VEC];
        if (a.dsum) rowvec::open<T, VEC>(u[j], o);
#pragma unroll
        for (int e = 0; e < VEC; ++e) o[e] = fmaf(rstd, dh[j][e] - s[j][e] * c, a.dsum ? o[e] : 0.f);
        rowvec::store<T, VEC>(static_cast<T*>(a.dx) + t * a.d + e0, o);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int e0 = (j * blockDim.x + threadIdx.x) * VEC;
    if (e0 < a.d) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) a.part[(size_t)blockIdx.x * a.d + e0 + e] = dg[j][e];
    }
  }
}

// dgamma (+)= the blocks' shares: 16 columns per block, 64 rows of shares at a time (592 shares of 1536: 6.4 us; 32 columns
// and 32 rows took 8.4)
__global__ void __launch_bounds__(1024) dgamma_kernel(const float* __restrict__ part, int n, int d, float* dgamma,
                                                      int accumulate) {
  __shared__ float sh[64][17];
  const int c = threadIdx.x & 15, col = blockIdx.x * 16 + c, r0 = threadIdx.x >> 4;
  float v = 0.f;
  if (col < d) {
#pragma unroll 8
    for (int r = r0; r < n; r += 64) v += part[(size_t)r * d + col];
  }
  sh[r0][c] = v;
  __syncthreads();
  if (r0 == 0 && col < d) {
    float sum = 0.f;
    for (int r = 0; r < 64; ++r) sum += sh[r][c];
    dgamma[col] = accumulate ? dgamma[col] + sum : sum;
  }
}

// Launches over the blocks that are resident at once: the kernels walk the rows, a second wave of blocks would only be
// uneven.
template <typename K, typename A>
int launch_resident(aero_ctx* ctx, K kernel, const A& a, int threads, long long most, int* grid_out) {
  int per_sm = 0;
  AERO_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, 0));
  if (per_sm < 1) return AERO_ERR_CUDA;
  const long long n = (long long)per_sm * ctx->sm_count;
  const int grid = (int)(n < most ? n : most);
  kernel<<<grid, threads, 0, ctx->stream>>>(a);
  ctx->launches += 1;
  AERO_CUDA_TRY(cudaGetLastError());
  if (grid_out) *grid_out = grid;
  return AERO_OK;
}

// Calls launch(vectors per thread, threads) for a block per row of `nvec` vectors, of which there are more than fit 256 threads
// once where LONG.
template <int VEC, bool LONG, typename F>
int with_block_shape(int nvec, F launch) {
  auto threads = [&](int nv) { return ((nvec + nv - 1) / nv + 31) / 32 * 32; };
  if constexpr (VEC == 1) {
    if (threads(4) <= 1024) return launch(std::integral_constant<int, 4>(), threads(4));
    return launch(std::integral_constant<int, 16>(), threads(16));
  } else {
    constexpr int kMost = 32 / VEC;                     // 32 elements per thread, 512 threads: kMaxD
    if constexpr (!LONG)
      if (threads(1) <= 256) return launch(std::integral_constant<int, 1>(), threads(1));
    if (threads(2) <= 256) return launch(std::integral_constant<int, 2>(), threads(2));
    if (kMost > 4 && threads(4) <= 256) return launch(std::integral_constant<int, 4>(), threads(4));
    return launch(std::integral_constant<int, kMost>(), threads(kMost));
  }
}

// Calls launch(vectors per lane) for a warp per row, in steps of two vectors up to MOST.
template <int MOST, int NV = 2, typename F>
int with_warp_shape(int nvec, F launch) {
  if constexpr (NV >= MOST) return launch(std::integral_constant<int, MOST>());
  else return nvec <= 32 * NV ? launch(std::integral_constant<int, NV>()) : with_warp_shape<MOST, NV + 2>(nvec, launch);
}
constexpr int kFwdLane = 8;                             // most vectors per lane

template <typename T, int VEC>
int launch_fwd(aero_ctx* ctx, const FwdArgs& a) {
  const int nvec = a.d / VEC;
  if constexpr (VEC > 1) {
    if (nvec <= 32 * kFwdLane)
      return with_warp_shape<kFwdLane>(nvec, [&](auto nv) {
        return launch_resident(ctx, rmsnorm_fwd_warp_kernel<T, decltype(nv)::value>, a, kWarps * 32, (a.T + kWarps - 1) / kWarps,
                               nullptr);
      });
  }
  static_assert(kFwdLane * 32 == 256, "rows that are left have more than 256 vectors");
  return with_block_shape<VEC, (VEC > 1)>(nvec, [&](auto nv, int threads) {
    return launch_resident(ctx, rmsnorm_fwd_kernel<T, VEC, decltype(nv)::value>, a, threads, a.T, nullptr);
  });
}

template <typename T, int VEC>
int launch_bwd(aero_ctx* ctx, const BwdArgs& a, float* dgamma, int accumulate) {
  int grid = 1;
  const int rc = with_block_shape<VEC, false>(a.d / VEC, [&](auto nv, int threads) {
    return launch_resident(ctx, rmsnorm_bwd_kernel<T, VEC, decltype(nv)::value>, a, threads, a.T < kBwdBlocks ? a.T : kBwdBlocks,
                           &grid);
  });
  if (rc) return rc;
  dgamma_kernel<<<(a.d + 15) / 16, 1024, 0, ctx->stream>>>(a.part, grid, a.d, dgamma, accumulate);
  ctx->launches += 1;
  AERO_CUDA_TRY(cudaGetLastError());
  return AERO_OK;
}

int run_fwd(aero_ctx* ctx, int32_t dtype, const FwdArgs& a, bool aligned) {
  if (dtype == AERO_FP32) return aligned && a.d % 4 == 0 ? launch_fwd<float, 4>(ctx, a) : launch_fwd<float, 1>(ctx, a);
  return aligned && a.d % 8 == 0 ? launch_fwd<__nv_bfloat16, 8>(ctx, a) : launch_fwd<__nv_bfloat16, 1>(ctx, a);
}

int check_shape(const aero_cfg* cfg, int64_t T, int32_t d) {
  if (!cfg || T < 0 || T >= (int64_t)1 << 31 || d <= 0) return AERO_ERR_INVALID;
  if (cfg->dtype != AERO_BF16 && cfg->dtype != AERO_FP32) return AERO_ERR_UNSUPPORTED;
  if (d > kMaxD) return AERO_ERR_UNSUPPORTED;
  return AERO_OK;
}

bool all_aligned(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (!aero_aligned16(p)) return false;
  return true;
}

}  // namespace

extern "C" {

size_t aero_rmsnorm_workspace_bytes(int64_t T, int32_t d) {
  if (T < 0 || d <= 0) return 0;
  const size_t n = T < kBwdBlocks ? (size_t)(T > 0 ? T : 1) : (size_t)kBwdBlocks;
  return aero_align_up(n * (size_t)d * sizeof(float), 256);
}

int aero_rmsnorm_fwd(aero_ctx* ctx, const aero_cfg* cfg, int64_t T, int32_t d, const void* x, const void* residual,
                     const void* gamma, float eps, void* sum, void* h, float* rstd, int8_t* q, float* q_scale) {
  AeroRange nv("aero_rmsnorm_fwd");
  int rc = check_shape(cfg, T, d);
  if (rc) return rc;
  if (!ctx || !gamma || !(eps > 0.f) || (q == nullptr) != (q_scale == nullptr)) return AERO_ERR_INVALID;
  if (T > 0 && !sum && !h && !rstd && !q) return AERO_ERR_INVALID;
  // (other rows still read gamma when a row's statistics are written; fp32 gives the three one type, and T = d one shape)
  if (cfg->dtype == AERO_FP32 && (gamma == rstd || gamma == q_scale)) return AERO_ERR_INVALID;
  if (T > 0 && !x) return AERO_ERR_INVALID;
  const size_t esz = cfg->dtype == AERO_FP32 ? 4 : 2;
  for (const void* p : {x, residual, gamma, (const void*)sum, (const void*)h})
    if (reinterpret_cast<uintptr_t>(p) % esz) return AERO_ERR_INVALID;
  if ((rc = aero_check_ctx(ctx))) return rc;
  if (T == 0) return AERO_OK;
  const FwdArgs a = {T, d, x, residual, gamma, eps, sum, h, rstd, q, q_scale};
  return run_fwd(ctx, cfg->dtype, a, all_aligned({x, residual, gamma, sum, h, q}));
}

int aero_rmsnorm_bwd(aero_ctx* ctx, const aero_cfg* cfg, int64_t T, int32_t d, const void* dh, const void* dsum,
                     const void* s, const void* gamma, const float* rstd, void* dx, float* dgamma, int accumulate_dgamma,
                     void* workspace, size_t workspace_bytes) {
  AeroRange nv("aero_rmsnorm_bwd");
  int rc = check_shape(cfg, T, d);
  if (rc) return rc;
  if (!ctx || !gamma || !dgamma || !workspace || !aero_aligned256(workspace)) return AERO_ERR_INVALID;
  if (T > 0 && (!dh || !s || !rstd || !dx)) return AERO_ERR_INVALID;
  const size_t esz = cfg->dtype == AERO_FP32 ? 4 : 2;
  for (const void* p : {dh, dsum, s, gamma, (const void*)dx})
    if (reinterpret_cast<uintptr_t>(p) % esz) return AERO_ERR_INVALID;
  if (workspace_bytes < aero_rmsnorm_workspace_bytes(T, d)) return AERO_ERR_WORKSPACE;
  if ((rc = aero_check_ctx(ctx))) return rc;
  if (T == 0) {
    if (!accumulate_dgamma) AERO_CUDA_TRY(cudaMemsetAsync(dgamma, 0, (size_t)d * sizeof(float), ctx->stream));
    return AERO_OK;
  }
  const BwdArgs a = {T, d, dh, dsum, s, gamma, rstd, dx, static_cast<float*>(workspace)};
  const bool al = all_aligned({dh, dsum, s, gamma, dx});
  if (cfg->dtype == AERO_FP32)
    return al && d % 4 == 0 ? launch_bwd<float, 4>(ctx, a, dgamma, accumulate_dgamma)
                            : launch_bwd<float, 1>(ctx, a, dgamma, accumulate_dgamma);
  return al && d % 8 == 0 ? launch_bwd<__nv_bfloat16, 8>(ctx, a, dgamma, accumulate_dgamma)
                          : launch_bwd<__nv_bfloat16, 1>(ctx, a, dgamma, accumulate_dgamma);
}

int aero_quantize_rows(aero_ctx* ctx, const aero_cfg* cfg, int64_t T, int32_t d, const void* x, int8_t* q, float* q_scale) {
  AeroRange nv("aero_quantize_rows");
  int rc = check_shape(cfg, T, d);
  if (rc) return rc;
  if (!ctx || (T > 0 && (!x || !q || !q_scale))) return AERO_ERR_INVALID;
  if (reinterpret_cast<uintptr_t>(x) % (cfg->dtype == AERO_FP32 ? 4 : 2)) return AERO_ERR_INVALID;
  if ((rc = aero_check_ctx(ctx))) return rc;
  if (T == 0) return AERO_OK;
  const FwdArgs a = {T, d, x, nullptr, nullptr, 0.f, nullptr, nullptr, nullptr, q, q_scale};
  return run_fwd(ctx, cfg->dtype, a, all_aligned({x, q}));
}

}  // extern "C"
