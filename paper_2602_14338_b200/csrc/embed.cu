// The tied lm_head weight at the model's other end: X[t, :] = scale W[y_t, :], and its gradient
// dW[v, :] (+)= scale sum_{t: y_t = v} dX[t, :].
//
// The gradient adds the rows of one token in the order of their positions and without atomics on the
// sums, so repeated calls give the same bits.  Up to kSmallT tokens one kernel does it: the block of a
// token's first occurrence finds the others by comparing ids.  Above that the positions are sorted by
// token (stable radix sort of up to 9 bits a pass) and cut into tiles of equal length, so that a token
// that makes up a tenth of the batch costs no more than any other: a warp adds the rows of its tile,
// writes the sums of tokens that lie inside the tile, and leaves those that reach over its ends as
// partial rows, which one more kernel joins.
#include "entry.cuh"
#include "vec.cuh"

#include <initializer_list>

namespace {

constexpr int kSmallT = 2048;
constexpr int kSortTile = 4096, kSortThreads = 256, kSortWarps = kSortThreads / 32;
constexpr int kMaxRadix = 512;
constexpr int kTile = 32;             // sorted positions per warp of the summing kernel

template <typename T, int VEC>
__global__ void __launch_bounds__(256) embed_fwd_kernel(long long T_, int d, int V, const int32_t* __restrict__ y,
                                                        const T* __restrict__ W, float scale, T* __restrict__ X,
                                                        uint32_t* status) {
  constexpr int NV = VEC == 1 ? 8 : 4;                 // vectors per lane: a warp takes NV * 32 * VEC columns of a row
  const int lane = threadIdx.x & 31;
  const int slabs = (d + NV * 32 * VEC - 1) / (NV * 32 * VEC);
  const long long units = T_ * slabs;
  for (long long u = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); u < units; u += (long long)gridDim.x * 8) {
    const long long t = u / slabs;
    const int c0 = (int)(u - t * slabs) * (NV * 32 * VEC) + lane * VEC;
    const int id = y[t];
    const bool ok = id >= 0 && id < V;
    if (!ok && id != AERO_NO_TOKEN && lane == 0) aero_raise(status, AERO_ST_BAD_TARGET);
    float f[NV][VEC];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = c0 + j * 32 * VEC;
      if (c < d && ok) rowvec::load<T, VEC>(W + (long long)id * d + c, f[j]);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = c0 + j * 32 * VEC;
      if (c < d) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[j][e] = ok ? f[j][e] * scale : 0.f;
        rowvec::store<T, VEC>(X + t * d + c, f[j]);
      }
    }
  }
}

// VEC fp32 sums to dW, as 16-byte accesses where the row is made of whole vectors
template <int VEC>
__device__ __forceinline__ void put(float* dst, const float (&s)[VEC], float scale, bool accumulate) {
  if constexpr (VEC == 1) {
    *dst = accumulate ? fmaf(s[0], scale, *dst) : s[0] * scale;
  } else {
#pragma unroll
    for (int q = 0; q < VEC / 4; ++q) {
      float4* p = reinterpret_cast<float4*>(dst) + q;
      float4 o = accumulate ? *p : make_float4(0.f, 0.f, 0.f, 0.f);
      o.x = fmaf(s[4 * q], scale, o.x);
      o.y = fmaf(s[4 * q + 1], scale, o.y);
      o.z = fmaf(s[4 * q + 2], scale, o.z);
      o.w = fmaf(s[4 * q + 3], scale, o.w);
      *p = o;
    }
  }
}

// Block (t, slab): the first occurrence of a token adds the rows of all its occurrences, in order.
template <typename T, int VEC>
__global__ void __launch_bounds__(128) embed_bwd_small_kernel(int T_, int d, int V, const int32_t* __restrict__ y,
                                                              const T* __restrict__ dX, float scale, float* __restrict__ dW,
                                                              int accumulate, uint32_t* status) {
  __shared__ int list[128];
  __shared__ int n_in_warp[4];
  const int t = blockIdx.x, c = (blockIdx.y * 128 + threadIdx.x) * VEC;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int id = y[t];
  if (id < 0 || id >= V) {
    if (id != AERO_NO_TOKEN && blockIdx.y == 0 && threadIdx.x == 0) aero_raise(status, AERO_ST_BAD_TARGET);
    return;
  }
  bool seen = false;
  for (int j = threadIdx.x; j < t; j += 128) seen |= y[j] == id;
  if (__syncthreads_or(seen)) return;                  // an earlier block has this token
  float acc[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
  for (int base = t; base < T_; base += 128) {
    const int j = base + threadIdx.x;
    const bool hit = j < T_ && y[j] == id;
    const unsigned mask = __ballot_sync(0xffffffffu, hit);
    if (lane == 0) n_in_warp[warp] = __popc(mask);
    __syncthreads();
    int off = 0, n = 0;
    for (int w = 0; w < 4; ++w) {
      if (w < warp) off += n_in_warp[w];
      n += n_in_warp[w];
    }
    if (hit) list[off + __popc(mask & ((1u << lane) - 1u))] = j;
    __syncthreads();
    if (c < d) {
      for (int k = 0; k < n; k += 4) {
        float f[4][VEC];
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (k + q < n) rowvec::load<T, VEC>(dX + (long long)list[k + q] * d + c, f[q]);
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (k + q < n)
#pragma unroll
            for (int e = 0; e < VEC; ++e) acc[e] += f[q][e];
      }
    }
    __syncthreads();
  }
  if (c < d) put<VEC>(dW + (long long)id * d + c, acc, scale, accumulate != 0);
}

// ---- stable radix sort of the positions by token -------------------------------------------------
// A pass: digit counts per block of kSortTile keys, laid out [digit][block]; their exclusive prefix;
// the scatter.  The first pass reads the token ids themselves; ids that stand for no token sort last,
// as V.
__device__ __forceinline__ uint32_t key_of(const int32_t* y, const uint32_t* keys, long long i, int V) {
  if (keys) return keys[i];
  const int id = y[i];
  return id >= 0 && id < V ? (uint32_t)id : (uint32_t)V;
}

__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(int n, int V, const int32_t* __restrict__ y,
                                                                  const uint32_t* __restrict__ keys, int shift, int radix,
                                                                  uint32_t* __restrict__ counts, uint32_t* status) {
  __shared__ uint32_t h[kMaxRadix];
  for (int i = threadIdx.x; i < radix; i += kSortThreads) h[i] = 0;
  __syncthreads();
  const int base = blockIdx.x * kSortTile;
  bool bad = false;
  for (int k = threadIdx.x; k < kSortTile && base + k < n; k += kSortThreads) {
    const uint32_t key = key_of(y, keys, base + k, V);
    if (!keys && key == (uint32_t)V) bad |= y[base + k] != AERO_NO_TOKEN;
    atomicAdd(&h[(key >> shift) & (radix - 1)], 1u);
  }
  if (bad) aero_raise(status, AERO_ST_BAD_TARGET);
  __syncthreads();
  for (int i = threadIdx.x; i < radix; i += kSortThreads) counts[(size_t)i * gridDim.x + blockIdx.x] = h[i];
}

// exclusive prefix of n counts in place, one block
__global__ void __launch_bounds__(1024) sort_prefix_kernel(uint32_t* __restrict__ counts, int n) {
  __shared__ uint32_t warp_sum[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t carry = 0;
  for (int base = 0; base < n; base += 4096) {
    const int i = base + threadIdx.x * 4;
    uint32_t v[4], sum = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      v[q] = i + q < n ? counts[i + q] : 0u;
      sum += v[q];
    }
    uint32_t incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t u = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += u;
    }
    if (lane == 31) warp_sum[warp] = incl;
    __syncthreads();
    uint32_t before = 0, total = 0;
    for (int w = 0; w < 32; ++w) {
      if (w < warp) before += warp_sum[w];
      total += warp_sum[w];
    }
    uint32_t run = carry + before + incl - sum;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (i + q < n) counts[i + q] = run;
      run += v[q];
    }
    carry += total;
    __syncthreads();
  }
}

__global__ void __launch_bounds__(kSortThreads) sort_scatter_kernel(int n, int V, const int32_t* __restrict__ y,
                                                                    const uint32_t* __restrict__ keys,
                                                                    const uint32_t* __restrict__ pos, int shift, int radix,
                                                                    const uint32_t* __restrict__ starts,
                                                                    uint32_t* __restrict__ keys_out,
                                                                    uint32_t* __restrict__ pos_out) {
  __shared__ uint32_t h[kSortWarps][kMaxRadix];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < kSortWarps * radix; i += kSortThreads) h[i / radix][i % radix] = 0;
  __syncthreads();
  // each warp takes a contiguous stretch, 32 keys at a time, so that ranks follow the order of the keys
  constexpr int kSteps = kSortTile / kSortThreads;
  const int base = blockIdx.x * kSortTile + warp * (32 * kSteps);
  uint32_t key[kSteps], rank[kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int i = base + s * 32 + lane;
    const bool in = i < n;
    key[s] = in ? key_of(y, keys, i, V) : 0u;
    const uint32_t digit = in ? (key[s] >> shift) & (radix - 1) : 0xffffffffu;
    const unsigned same = __match_any_sync(0xffffffffu, digit);
    uint32_t before = 0;
    if (in) before = h[warp][digit];
    __syncwarp();
    if (in && lane == __ffs(same) - 1) h[warp][digit] = before + __popc(same);
    __syncwarp();
    rank[s] = before + __popc(same & ((1u << lane) - 1u));
  }
  __syncthreads();
  for (int g = threadIdx.x; g < radix; g += kSortThreads) {
    uint32_t run = starts[(size_t)g * gridDim.x + blockIdx.x];
    for (int w = 0; w < kSortWarps; ++w) {
      const uint32_t c = h[w][g];
      h[w][g] = run;
      run += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int i = base + s * 32 + lane;
    if (i < n) {
      const uint32_t dst = h[warp][(key[s] >> shift) & (radix - 1)] + rank[s];
      keys_out[dst] = key[s];
      pos_out[dst] = pos ? pos[i] : (uint32_t)i;
    }
  }
}

// ---- sums over the sorted positions ----------------------------------------------------------------
// Warp (tile, slab): tile = kTile sorted positions, slab = 32 * VEC columns.  A run of equal keys that
// lies inside the tile goes to dW; one that continues from the tile before goes to part[tile][0], one
// that starts here and continues in the tile after to part[tile][1].
template <typename T, int VEC>
__global__ void __launch_bounds__(256) embed_bwd_sum_kernel(int n, int d, int V, const uint32_t* __restrict__ keys,
                                                            const uint32_t* __restrict__ pos, const T* __restrict__ dX,
                                                            float scale, float* __restrict__ dW, int accumulate,
                                                            float* __restrict__ part) {
  const int lane = threadIdx.x & 31;
  const int slabs = (d + 32 * VEC - 1) / (32 * VEC);
  const long long u = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const long long tile = u / slabs;
  const int p0 = (int)(tile * kTile);
  if (tile * kTile >= n) return;
  const int c = ((int)(u - tile * slabs) * 32 + lane) * VEC;
  const int count = min(kTile, n - p0);
  const uint32_t my_key = lane < count ? keys[p0 + lane] : (uint32_t)V;
  const uint32_t my_pos = lane < count ? pos[p0 + lane] : 0u;
  const uint32_t before = p0 > 0 ? keys[p0 - 1] : (uint32_t)V;
  const uint32_t after = p0 + count < n ? keys[p0 + count] : (uint32_t)V;
  float acc[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
  int run0 = 0;                                          // first position of the current run
  constexpr int U = 8;
  for (int k = 0; k < count; k += U) {
    if (__shfl_sync(0xffffffffu, my_key, k) == (uint32_t)V) break;       // only positions without a token follow
    float f[U][VEC];
#pragma unroll
    for (int q = 0; q < U; ++q) {
      const uint32_t row = __shfl_sync(0xffffffffu, my_pos, k + q), key = __shfl_sync(0xffffffffu, my_key, k + q);
      if (key != (uint32_t)V && c < d) rowvec::load<T, VEC>(dX + (long long)row * d + c, f[q]);
    }
#pragma unroll
    for (int q = 0; q < U; ++q) {
      const uint32_t key = __shfl_sync(0xffffffffu, my_key, k + q);
      if (key == (uint32_t)V) break;
#pragma unroll
      for (int e = 0; e < VEC; ++e) acc[e] += f[q][e];
      const bool last = k + q + 1 >= count;
      const uint32_t next = last ? after : __shfl_sync(0xffffffffu, my_key, (k + q + 1) & 31);
      if (next != key || last) {
        const bool head = run0 == 0 && before == key, tail = last && next == key;
        if (c < d) {
          if (head || tail) put<VEC>(part + ((size_t)tile * 2 + (head ? 0 : 1)) * d + c, acc, 1.f, false);
          else put<VEC>(dW + (long long)key * d + c, acc, scale, accumulate != 0);
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
        run0 = k + q + 1;
      }
    }
  }
}

// A run that starts in tile b and reaches into the tiles after it: block (b, 128 columns), eight warps
// take a contiguous eighth of the tiles each, added up in order.
__global__ void __launch_bounds__(256) embed_bwd_join_kernel(int n, int d, int V, const uint32_t* __restrict__ keys,
                                                             const float* __restrict__ part, float scale,
                                                             float* __restrict__ dW, int accumulate) {
  __shared__ float sh[8][128];
  const long long b = blockIdx.x;
  const long long end = (b + 1) * kTile;                 // first position of the next tile
  if (end >= n) return;
  const uint32_t key = keys[end - 1];
  if (key == (uint32_t)V || keys[end] != key) return;
  const bool starts_here = keys[b * kTile] != key || b == 0 || keys[b * kTile - 1] != key;
  if (!starts_here) return;
  // last position of the run by bisection: keys are sorted
  long long lo = end, hi = n;                            // keys[lo] == key, keys[hi] != key
  while (hi - lo > 1) {
    const long long mid = (lo + hi) >> 1;
    if (keys[mid] == key) lo = mid; else hi = mid;
  }
  const long long last = lo / kTile;                     // the run's last tile; tiles b + 1 .. last hold it in slot 0
  const long long count = last - b;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int c0 = blockIdx.y * 128;
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  const long long k0 = b + 1 + count * warp / 8, k1 = b + 1 + count * (warp + 1) / 8;
#pragma unroll 4
  for (long long k = k0; k < k1; ++k) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (c0 + q * 32 + lane < d) acc[q] += part[(size_t)k * 2 * d + c0 + q * 32 + lane];
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) sh[warp][q * 32 + lane] = acc[q];
  __syncthreads();
  if (threadIdx.x < 128 && c0 + (int)threadIdx.x < d) {
    const int c = c0 + threadIdx.x;
    float sum = part[((size_t)b * 2 + 1) * d + c];
    for (int w = 0; w < 8; ++w) sum += sh[w][threadIdx.x];
    float* dst = dW + (long long)key * d + c;
    *dst = accumulate ? fmaf(sum, scale, *dst) : sum * scale;
  }
}

struct Ws {
  uint32_t* keys[2];
  uint32_t* pos[2];
  uint32_t* counts;
  float* part;
  size_t bytes;
};

Ws carve(void* base, int64_t T, int32_t d) {
  Ws w;
  char* p = static_cast<char*>(base);
  size_t off = 0;
  const size_t arr = aero_align_up((size_t)T * sizeof(uint32_t), 256);
  for (int i = 0; i < 2; ++i) {
    w.keys[i] = reinterpret_cast<uint32_t*>(p + off); off += arr;
    w.pos[i] = reinterpret_cast<uint32_t*>(p + off); off += arr;
  }
  const size_t blocks = ((size_t)T + kSortTile - 1) / kSortTile;
  w.counts = reinterpret_cast<uint32_t*>(p + off); off += aero_align_up(blocks * kMaxRadix * sizeof(uint32_t), 256);
  const size_t tiles = ((size_t)T + kTile - 1) / kTile;
  w.part = reinterpret_cast<float*>(p + off); off += aero_align_up(tiles * 2 * (size_t)d * sizeof(float), 256);
  w.bytes = off;
  return w;
}

int sort_positions(aero_ctx* ctx, const Ws& w, int n, int V, const int32_t* y, const uint32_t** keys, const uint32_t** pos) {
  int bits = 1;
  while (bits < 32 && ((uint32_t)V >> bits) != 0) ++bits;          // the keys are 0 .. V
  const int passes = (bits + 8) / 9, per = (bits + passes - 1) / passes;
  const int blocks = (n + kSortTile - 1) / kSortTile;
  const uint32_t *kin = nullptr, *pin = nullptr;
  for (int p = 0; p < passes; ++p) {
    const int radix = 1 << per, shift = p * per;
    sort_count_kernel<<<blocks, kSortThreads, 0, ctx->stream>>>(n, V, y, kin, shift, radix, w.counts, ctx->d_status);
    sort_prefix_kernel<<<1, 1024, 0, ctx->stream>>>(w.counts, radix * blocks);
    sort_scatter_kernel<<<blocks, kSortThreads, 0, ctx->stream>>>(n, V, y, kin, pin, shift, radix, w.counts, w.keys[p & 1],
                                                                  w.pos[p & 1]);
    ctx->launches += 3;
    kin = w.keys[p & 1];
    pin = w.pos[p & 1];
  }
  AERO_CUDA_TRY(cudaGetLastError());
  *keys = kin;
  *pos = pin;
  return AERO_OK;
}

template <typename T, int VEC>
int bwd_launch(aero_ctx* ctx, int64_t T_, int32_t d, int32_t V, const int32_t* y, const T* dX, float scale, float* dW,
               int accumulate, void* ws) {
  if (T_ <= kSmallT) {
    const dim3 grid((unsigned)T_, (unsigned)((d + 128 * VEC - 1) / (128 * VEC)));
    embed_bwd_small_kernel<T, VEC><<<grid, 128, 0, ctx->stream>>>((int)T_, d, V, y, dX, scale, dW, accumulate, ctx->d_status);
    ctx->launches += 1;
    AERO_CUDA_TRY(cudaGetLastError());
    return AERO_OK;
  }
  const Ws w = carve(ws, T_, d);
  const int n = (int)T_;
  const uint32_t *keys, *pos;
  const int rc = sort_positions(ctx, w, n, V, y, &keys, &pos);
  if (rc) return rc;
  const long long tiles = (n + kTile - 1) / kTile, slabs = (d + 32 * VEC - 1) / (32 * VEC);
  embed_bwd_sum_kernel<T, VEC><<<(unsigned)((tiles * slabs + 7) / 8), 256, 0, ctx->stream>>>(n, d, V, keys, pos, dX, scale, dW,
                                                                                             accumulate, w.part);
  const dim3 jgrid((unsigned)tiles, (unsigned)((d + 127) / 128));
  embed_bwd_join_kernel<<<jgrid, 256, 0, ctx->stream>>>(n, d, V, keys, w.part, scale, dW, accumulate);
  ctx->launches += 2;
  AERO_CUDA_TRY(cudaGetLastError());
  return AERO_OK;
}

template <typename T>
int fwd_launch(aero_ctx* ctx, int64_t T_, int32_t d, int32_t V, const int32_t* y, const T* W, float scale, T* X) {
  const bool vec = aero_aligned16(W) && aero_aligned16(X) && d % rowvec::Elem<T>::kVec == 0;
  const int cols = vec ? 4 * 32 * rowvec::Elem<T>::kVec : 8 * 32;
  const long long units = T_ * ((d + cols - 1) / cols), blocks = (units + 7) / 8;
  const unsigned grid = (unsigned)(blocks < (1 << 20) ? blocks : (1 << 20));
  if (vec) embed_fwd_kernel<T, rowvec::Elem<T>::kVec><<<grid, 256, 0, ctx->stream>>>(T_, d, V, y, W, scale, X, ctx->d_status);
  else embed_fwd_kernel<T, 1><<<grid, 256, 0, ctx->stream>>>(T_, d, V, y, W, scale, X, ctx->d_status);
  ctx->launches += 1;
  AERO_CUDA_TRY(cudaGetLastError());
  return AERO_OK;
}

int check_shape(const aero_cfg* cfg, int64_t T, int32_t d, int32_t V) {
  if (!cfg || T < 0 || T >= (int64_t)1 << 31 || d <= 0 || V <= 0) return AERO_ERR_INVALID;
  if (cfg->dtype != AERO_BF16 && cfg->dtype != AERO_FP32) return AERO_ERR_UNSUPPORTED;
  if (d > 65536) return AERO_ERR_UNSUPPORTED;
  return AERO_OK;
}

}  // namespace

extern "C" {

int aero_embed_fwd(aero_ctx* ctx, const aero_cfg* cfg, int64_t T, int32_t d, int32_t V, const int32_t* y, const void* W,
                   float scale, void* X) {
  AeroRange nv("aero_embed_fwd");
  int rc = check_shape(cfg, T, d, V);
  if (rc) return rc;
  if (!ctx || !W || (T > 0 && (!y || !X))) return AERO_ERR_INVALID;
  const size_t esz = cfg->dtype == AERO_FP32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(W) % esz || reinterpret_cast<uintptr_t>(X) % esz) return AERO_ERR_INVALID;
  if ((rc = aero_check_ctx(ctx))) return rc;
  if (T == 0) return AERO_OK;
  if (cfg->dtype == AERO_FP32)
    return fwd_launch<float>(ctx, T, d, V, y, static_cast<const float*>(W), scale, static_cast<float*>(X));
  return fwd_launch<__nv_bfloat16>(ctx, T, d, V, y, static_cast<const __nv_bfloat16*>(W), scale,
                                   static_cast<__nv_bfloat16*>(X));
}

size_t aero_embed_workspace_bytes(int64_t T, int32_t d) {
  if (T < 0 || d <= 0) return 0;
  return T <= kSmallT ? 256 : carve(nullptr, T, d).bytes;
}

int aero_embed_bwd(aero_ctx* ctx, const aero_cfg* cfg, int64_t T, int32_t d, int32_t V, const int32_t* y, const void* dX,
                   float scale, float* dW, int accumulate_dW, void* workspace, size_t workspace_bytes) {
  AeroRange nv("aero_embed_bwd");
  int rc = check_shape(cfg, T, d, V);
  if (rc) return rc;
  if (!ctx || !dW || (T > 0 && (!y || !dX)) || !workspace || !aero_aligned256(workspace)) return AERO_ERR_INVALID;
  if (reinterpret_cast<uintptr_t>(dX) % (cfg->dtype == AERO_FP32 ? 4 : 2)) return AERO_ERR_INVALID;
  if (workspace_bytes < aero_embed_workspace_bytes(T, d)) return AERO_ERR_WORKSPACE;
  if ((rc = aero_check_ctx(ctx))) return rc;
  if (!accumulate_dW) AERO_CUDA_TRY(cudaMemsetAsync(dW, 0, (size_t)V * d * sizeof(float), ctx->stream));
  if (T == 0) return AERO_OK;
  const bool al = aero_aligned16(dX) && aero_aligned16(dW);
  if (cfg->dtype == AERO_FP32) {
    const float* x = static_cast<const float*>(dX);
    if (al && d % 4 == 0) return bwd_launch<float, 4>(ctx, T, d, V, y, x, scale, dW, accumulate_dW, workspace);
    return bwd_launch<float, 1>(ctx, T, d, V, y, x, scale, dW, accumulate_dW, workspace);
  }
  const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(dX);
  if (al && d % 8 == 0) return bwd_launch<__nv_bfloat16, 8>(ctx, T, d, V, y, x, scale, dW, accumulate_dW, workspace);
  return bwd_launch<__nv_bfloat16, 1>(ctx, T, d, V, y, x, scale, dW, accumulate_dW, workspace);
}

}  // extern "C"
