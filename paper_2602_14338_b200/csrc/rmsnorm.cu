// The policy model's final RMS norm, which makes the H that stage (b) reads, and its gradient,
// which takes the dH that stage (b) returns:
//   s = x + residual,  rstd = 1 / sqrt(mean(s^2) + eps),  h = s rstd gamma
//   ds = rstd (gamma dh - shat mean(gamma dh shat)) + dsum,   shat = s rstd
//   dgamma (+)= sum_t dh shat
// and the 8-bit form of the rows, q = round(h / scale), scale = max |h| / 127.
//
// Bound by memory: every row is read once and held in registers as fp32 between the reduction and
// the outputs, one block per row (so an output may be written over an input row by row).
#include "entry.cuh"
#include "vec.cuh"

#include <initializer_list>
#include <type_traits>

namespace {

constexpr int kMaxD = 16384;
constexpr int kBwdBlocks = 592;       // blocks of the backward, at most: 4 per SM of a 148-SM device

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

// Launch shapes: at most 256 threads while few vectors per thread suffice, so that several rows are in
// flight on an SM; the largest vector count of a kind goes up to kMaxD.
template <int VEC, int NV>
constexpr int max_threads() {
  return VEC == 1 ? 1024 : (NV * VEC == 32 ? 512 : 256);
}

// sum and maximum over the block's threads, the same value in every thread (fixed order)
__device__ __forceinline__ float2 block_sum_max(float sum, float mx, float2* sh) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    sum += __shfl_xor_sync(0xffffffffu, sum, o);
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
  }
  const int warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
  if ((threadIdx.x & 31) == 0) sh[warp] = make_float2(sum, mx);
  __syncthreads();
  float2 r = sh[0];
  for (int w = 1; w < nw; ++w) {
    r.x += sh[w].x;
    r.y = fmaxf(r.y, sh[w].y);
  }
  return r;
}

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

// One block per row; thread i holds vectors i, i + blockDim, ... of the row.  The sum of two rows is
// kept in fp32 for the norm and rounded once on its way out.
template <typename T, int VEC, int NV>
__global__ void __launch_bounds__(max_threads<VEC, NV>()) rmsnorm_fwd_kernel(FwdArgs a) {
  __shared__ float2 sh[32];
  const long long t = blockIdx.x;
  const T* x = static_cast<const T*>(a.x) + t * a.d;
  const T* res = a.residual ? static_cast<const T*>(a.residual) + t * a.d : nullptr;
  const T* gm = static_cast<const T*>(a.gamma);
  float s[NV][VEC];
  float ss = 0.f, mx = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int e0 = (j * blockDim.x + threadIdx.x) * VEC;
    if (e0 < a.d) {
      rowvec::load<T, VEC>(x + e0, s[j]);
      if (res) {
        float r[VEC];
        rowvec::load<T, VEC>(res + e0, r);
#pragma unroll
        for (int e = 0; e < VEC; ++e) s[j][e] += r[e];
      }
    }
  }
  float g[NV][VEC];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int e0 = (j * blockDim.x + threadIdx.x) * VEC;
    if (e0 < a.d) {
      if (gm) rowvec::load<T, VEC>(gm + e0, g[j]);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        if (!gm) g[j][e] = 1.f;
        ss = fmaf(s[j][e], s[j][e], ss);
        mx = fmaxf(mx, fabsf(s[j][e] * g[j][e]));
      }
    }
  }
  const float2 red = block_sum_max(ss, mx, sh);
  const float rstd = gm ? 1.f / sqrtf(red.x / (float)a.d + a.eps) : 1.f;
  // a NaN drops out of the maximum but not out of the sum of squares: the scale takes it from there
  const float amax = red.x == red.x ? red.y * rstd : red.x;
  const float up = amax < 0x1p-100f ? 0x1p100f : 1.f;      // keeps 127 / amax finite for the smallest rows
  const float inv = amax > 0.f ? 127.f / (amax * up) : 0.f;
  if (threadIdx.x == 0) {
    if (a.rstd) a.rstd[t] = rstd;
    if (a.q_scale) a.q_scale[t] = amax / 127.f;
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int e0 = (j * blockDim.x + threadIdx.x) * VEC;
    if (e0 < a.d) {
      if (a.sum) rowvec::store<T, VEC>(static_cast<T*>(a.sum) + t * a.d + e0, s[j]);
#pragma unroll
      for (int e = 0; e < VEC; ++e) s[j][e] = s[j][e] * rstd * g[j][e];
      if (a.h) rowvec::store<T, VEC>(static_cast<T*>(a.h) + t * a.d + e0, s[j]);
      if (a.q) store_q<VEC>(a.q + t * a.d + e0, s[j], up, inv);
    }
  }
}

// Blocks walk the rows with a stride of the grid; each keeps its share of dgamma in registers and
// leaves it in part[block], which dgamma_kernel adds up in a fixed order.
template <typename T, int VEC, int NV>
__global__ void __launch_bounds__(max_threads<VEC, NV>()) rmsnorm_bwd_kernel(BwdArgs a) {
  __shared__ float2 sh[2][32];
  float g[NV][VEC], dg[NV][VEC];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int e0 = (j * blockDim.x + threadIdx.x) * VEC;
    if (e0 < a.d) rowvec::load<T, VEC>(static_cast<const T*>(a.gamma) + e0, g[j]);
#pragma unroll
    for (int e = 0; e < VEC; ++e) dg[j][e] = 0.f;
  }
  int turn = 0;
  for (long long t = blockIdx.x; t < a.T; t += gridDim.x, turn ^= 1) {
    const float rstd = a.rstd[t];
    float s[NV][VEC], dh[NV][VEC];
    float dot = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int e0 = (j * blockDim.x + threadIdx.x) * VEC;
      if (e0 < a.d) {
        rowvec::load<T, VEC>(static_cast<const T*>(a.s) + t * a.d + e0, s[j]);
        rowvec::load<T, VEC>(static_cast<const T*>(a.dh) + t * a.d + e0, dh[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int e0 = (j * blockDim.x + threadIdx.x) * VEC;
      if (e0 < a.d) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          s[j][e] *= rstd;                                       // shat
          dg[j][e] = fmaf(dh[j][e], s[j][e], dg[j][e]);
          dh[j][e] *= g[j][e];
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
        if (a.dsum) rowvec::load<T, VEC>(static_cast<const T*>(a.dsum) + t * a.d + e0, o);
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

// dgamma (+)= the blocks' shares: 32 columns per block, 32 rows of shares at a time
__global__ void __launch_bounds__(1024) dgamma_kernel(const float* __restrict__ part, int n, int d, float* dgamma,
                                                      int accumulate) {
  __shared__ float sh[32][33];
  const int col = blockIdx.x * 32 + (threadIdx.x & 31), r0 = threadIdx.x >> 5;
  float v = 0.f;
  if (col < d)
    for (int r = r0; r < n; r += 32) v += part[(size_t)r * d + col];
  sh[r0][threadIdx.x & 31] = v;
  __syncthreads();
  if (r0 == 0 && col < d) {
    float sum = 0.f;
    for (int r = 0; r < 32; ++r) sum += sh[r][threadIdx.x];
    dgamma[col] = accumulate ? dgamma[col] + sum : sum;
  }
}

// Calls launch(vectors per thread, threads) for rows of `nvec` vectors.
template <int VEC, typename F>
void with_shape(int nvec, F launch) {
  auto threads = [&](int nv) { return ((nvec + nv - 1) / nv + 31) / 32 * 32; };
  if constexpr (VEC == 1) {
    if (threads(4) <= 1024) launch(std::integral_constant<int, 4>(), threads(4));
    else launch(std::integral_constant<int, 16>(), threads(16));
  } else {
    constexpr int kMost = 32 / VEC;                     // 32 elements per thread, 512 threads: kMaxD
    if (threads(1) <= 256) launch(std::integral_constant<int, 1>(), threads(1));
    else if (threads(2) <= 256) launch(std::integral_constant<int, 2>(), threads(2));
    else if (kMost > 4 && threads(4) <= 256) launch(std::integral_constant<int, 4>(), threads(4));
    else launch(std::integral_constant<int, kMost>(), threads(kMost));
  }
}

template <typename T>
int launch_fwd(aero_ctx* ctx, const FwdArgs& a, bool vec) {
  auto go = [&](auto vec_c) {
    constexpr int VEC = decltype(vec_c)::value;
    with_shape<VEC>(a.d / VEC, [&](auto nv_c, int threads) {
      rmsnorm_fwd_kernel<T, VEC, decltype(nv_c)::value><<<(unsigned)a.T, threads, 0, ctx->stream>>>(a);
    });
  };
  if (vec) go(std::integral_constant<int, rowvec::Elem<T>::kVec>());
  else go(std::integral_constant<int, 1>());
  ctx->launches += 1;
  AERO_CUDA_TRY(cudaGetLastError());
  return AERO_OK;
}

template <typename T>
int launch_bwd(aero_ctx* ctx, const BwdArgs& a, int grid, bool vec, float* dgamma, int accumulate) {
  auto go = [&](auto vec_c) {
    constexpr int VEC = decltype(vec_c)::value;
    with_shape<VEC>(a.d / VEC, [&](auto nv_c, int threads) {
      rmsnorm_bwd_kernel<T, VEC, decltype(nv_c)::value><<<grid, threads, 0, ctx->stream>>>(a);
    });
  };
  if (vec) go(std::integral_constant<int, rowvec::Elem<T>::kVec>());
  else go(std::integral_constant<int, 1>());
  dgamma_kernel<<<(a.d + 31) / 32, 1024, 0, ctx->stream>>>(a.part, grid, a.d, dgamma, accumulate);
  ctx->launches += 2;
  AERO_CUDA_TRY(cudaGetLastError());
  return AERO_OK;
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
  if (T > 0 && !x) return AERO_ERR_INVALID;
  const size_t esz = cfg->dtype == AERO_FP32 ? 4 : 2;
  for (const void* p : {x, residual, gamma, (const void*)sum, (const void*)h})
    if (reinterpret_cast<uintptr_t>(p) % esz) return AERO_ERR_INVALID;
  if ((rc = aero_check_ctx(ctx))) return rc;
  if (T == 0) return AERO_OK;
  const FwdArgs a = {T, d, x, residual, gamma, eps, sum, h, rstd, q, q_scale};
  const bool al = all_aligned({x, residual, gamma, sum, h, q});
  if (cfg->dtype == AERO_FP32) return launch_fwd<float>(ctx, a, al && d % 4 == 0);
  return launch_fwd<__nv_bfloat16>(ctx, a, al && d % 8 == 0);
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
  const int grid = (int)(T < kBwdBlocks ? T : kBwdBlocks);
  const bool al = all_aligned({dh, dsum, s, gamma, dx});
  if (cfg->dtype == AERO_FP32) return launch_bwd<float>(ctx, a, grid, al && d % 4 == 0, dgamma, accumulate_dgamma);
  return launch_bwd<__nv_bfloat16>(ctx, a, grid, al && d % 8 == 0, dgamma, accumulate_dgamma);
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
  const bool al = all_aligned({x, q});
  if (cfg->dtype == AERO_FP32) return launch_fwd<float>(ctx, a, al && d % 4 == 0);
  return launch_fwd<__nv_bfloat16>(ctx, a, al && d % 8 == 0);
}

}  // extern "C"
