// One AdamW step over many tensors.  Per element, with g' = grad_scale clip g and t the number of this step:
//   m = beta1 m + (1 - beta1) g',   v = beta2 v + (1 - beta2) g'^2
//   p = p - (lr wd p + lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps))
// (1 - lr wd as a factor of p would be rounded to a multiple of 2^-24 first: at lr = 1e-6 a decay of 0.1 would become one of 0.119 and
// one of 0.01 none at all, in every element and step.)
// m and v are fp32, or 8 bits an element with a scale per 256 elements: m as e4m3, the root of v as an unsigned float of
// four exponent and four mantissa bits (v spans twice as many octaves as m; its root fits the same range, and the sign's bit
// goes to the mantissa).  The step itself uses the fp32 values before they are rounded.  Bound by memory: 28 bytes an element
// in fp32, 16 with 8-bit states, a bf16 gradient and a bf16 parameter with its fp32 master; each is read and written once, by one
// launch for up to 128 tensors.  The tensors' addresses travel in the kernel's parameters, so that nothing is copied to the device.
#include "entry.cuh"
#include "vec.cuh"

#include <cuda_fp8.h>

namespace {

constexpr int kSlots = 128;             // tensors per launch
constexpr int kBlock = 256;             // elements per scale of the 8-bit states; a warp's share of a tensor at a time
constexpr int kWarps = 8, kEach = kBlock / 32;
constexpr int kChunk = kWarps * kBlock;  // elements of one span per warp
constexpr int kSpans = 4;                // spans of a warp per chunk of the norm and of the states as numbers
constexpr int kNormBlocks = 148 * 8;     // of the norm's launch: a record each
// Of the others.  (Step with 8-bit states and states as numbers, 233 M elements: 1031 us with 592 blocks, 1023 with 1184, 999 with
// 2368, 966 with 9472, 993 with one per chunk; with fp32 states 1694, 1700, 1599, 1518, 1484.)
constexpr int kMaxBlocks = 148 * 64;
// Chunks at most of a call whose step's blocks add the norm's records up themselves: a record each.  (Without / with, bf16 params with
// fp32 masters, from the host, +-1 us: 60 x 1536 17.4 / 14.3 us, 8 x 98304 21.4 / 18.4, 16 x 98304 25.6 / 22.5, 24 x 98304 = 1152 chunks
// 29.6 / 26.6, 40 x 98304 33.8 / 33.8; 8 x 2^20, with 592 blocks for the step, 53 / 59; calls in a row, fp32, 1 x 1000 17.3 / 14.8,
// 60 x 1536 18.3 / 15.6, 24 x 98304 23.7 / 21.1.)
constexpr int kJoinChunks = kNormBlocks;
constexpr float kTopM = 448.f, kTopV = 496.f;          // largest values of the two 8-bit formats
constexpr float kLeast = 0x1p-100f;     // scales are made of at least this: 448 / it stays finite

enum : uint32_t { kParam16 = 1, kGrad16 = 2, kState8 = 4, kAligned = 8, kOut16 = 16 };

struct Slot {
  long long n;
  void* param;
  const void* grad;
  float* master;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  float weight_decay, lr_scale;
  uint32_t flags;
};
struct Table {
  int count;
  long long chunk0[kSlots + 1];         // first chunk of each tensor among those of the launch
  Slot slot[kSlots];
};

// What the step's kernels share, in the workspace: made of the gradients' norm and the step's number.
struct Scalars {
  float g_factor;                       // grad_scale clip
  float lr, c1, c2;                     // 1 / (1 - beta1^t), the root of 1 / (1 - beta2^t)
  int skip;
  long long t;
};

struct Hyper {
  float beta1, beta2, rest1, rest2, eps;      // rest = 1 - beta
};

// Numbers that the step is made of besides the tensors.
struct PrepareArgs {
  const double* partials;               // NULL: no norm
  int n_partials;
  double beta1, beta2;
  float lr, max_norm, grad_scale;
  int skip_nonfinite;
  const float* lr_dev;
  long long* step;
  float* stats;
  Scalars* out;
};

__device__ __forceinline__ int slot_of(const Table& t, long long chunk) {
  int lo = 0, hi = t.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (t.chunk0[mid] <= chunk) lo = mid; else hi = mid;
  }
  return lo;
}

// A warp's 256 elements from e0 on: eight neighbours a lane where every array of the tensor is made of whole 16-byte vectors,
// else every 32nd element from the lane's own, as far as the tensor goes.
struct Span {
  long long e0;
  int left;                             // elements from e0 to the tensor's end
  bool vec;
  int lane;
  __device__ bool has(int i) const { return vec || i * 32 + lane < left; }
  __device__ long long at(int i) const { return e0 + i * 32 + lane; }
  __device__ long long first() const { return e0 + lane * kEach; }
};

__device__ __forceinline__ void load32(const float* p, const Span& s, float (&x)[kEach]) {
  if (s.vec) {
    const float4 a = reinterpret_cast<const float4*>(p + s.first())[0], b = reinterpret_cast<const float4*>(p + s.first())[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i) x[i] = s.has(i) ? p[s.at(i)] : 0.f;
  }
}
__device__ __forceinline__ void load16(const __nv_bfloat16* p, const Span& s, float (&x)[kEach]) {
  if (s.vec) {
    rowvec::load<__nv_bfloat16, 8>(p + s.first(), x);
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i) x[i] = s.has(i) ? __bfloat162float(p[s.at(i)]) : 0.f;
  }
}
__device__ __forceinline__ void load(const void* p, bool half, const Span& s, float (&x)[kEach]) {
  if (half) load16(static_cast<const __nv_bfloat16*>(p), s, x);
  else load32(static_cast<const float*>(p), s, x);
}
__device__ __forceinline__ void store32(float* p, const Span& s, const float (&x)[kEach]) {
  if (s.vec) {
    reinterpret_cast<float4*>(p + s.first())[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p + s.first())[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (s.has(i)) p[s.at(i)] = x[i];
  }
}
__device__ __forceinline__ void store16(__nv_bfloat16* p, const Span& s, const float (&x)[kEach]) {
  if (s.vec) {
    rowvec::store<__nv_bfloat16, 8>(p + s.first(), x);
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (s.has(i)) p[s.at(i)] = __float2bfloat16_rn(x[i]);
  }
}
__device__ __forceinline__ void store(void* p, bool half, const Span& s, const float (&x)[kEach]) {
  if (half) store16(static_cast<__nv_bfloat16*>(p), s, x);
  else store32(static_cast<float*>(p), s, x);
}
// (a code per register; what is above its 8 bits is not stored)
__device__ __forceinline__ void load_codes(const uint8_t* p, const Span& s, uint32_t (&c)[kEach]) {
  if (s.vec) {
    const uint2 u = *reinterpret_cast<const uint2*>(p + s.first());
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      c[i] = __byte_perm(u.x, 0, 0x4440 + i);
      c[4 + i] = __byte_perm(u.y, 0, 0x4440 + i);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i) c[i] = s.has(i) ? p[s.at(i)] : 0;
  }
}
__device__ __forceinline__ void store_codes(uint8_t* p, const Span& s, const uint32_t (&c)[kEach]) {
  if (s.vec) {
    auto word = [&](int i) {
      return __byte_perm(__byte_perm(c[i], c[i + 1], 0x0040), __byte_perm(c[i + 2], c[i + 3], 0x0040), 0x5410);
    };
    *reinterpret_cast<uint2*>(p + s.first()) = make_uint2(word(0), word(4));
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (s.has(i)) p[s.at(i)] = (uint8_t)c[i];
  }
}

// Largest magnitude of the warp's elements; compared as bits, so that a NaN is larger than all and comes through.
template <bool SIGNED>
__device__ __forceinline__ float warp_top(const float (&x)[kEach]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) top = max(top, SIGNED ? __float_as_uint(x[i]) & 0x7fffffffu : __float_as_uint(x[i]));
  return __uint_as_float(__reduce_max_sync(0xffffffffu, top));
}
// What a block's scale is made of: its largest magnitude, or NaN where that is no finite number.
__device__ __forceinline__ float scale_top(float top) {
  return top < INFINITY ? fmaxf(top, kLeast) : __uint_as_float(0x7fffffffu);
}

__device__ __forceinline__ void open_m(const Slot& t, const Span& s, float (&m)[kEach]) {
  uint32_t c[kEach];
  load_codes(static_cast<const uint8_t*>(t.m), s, c);
  const float scale = t.m_scale[s.e0 / kBlock];
#pragma unroll
  for (int i = 0; i < kEach; i += 2) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(c[i] | c[i + 1] << 8), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    m[i] = __fmul_rn(f.x, scale);
    m[i + 1] = __fmul_rn(f.y, scale);
  }
}
__device__ __forceinline__ void close_m(const Slot& t, const Span& s, const float (&m)[kEach]) {
  const float top = scale_top(warp_top<true>(m)), inv = __fmul_rn(__frcp_rn(top), kTopM);
  uint32_t c[kEach];
#pragma unroll
  for (int i = 0; i < kEach; i += 2) {
    const __nv_fp8x2_storage_t u = __nv_cvt_float2_to_fp8x2(make_float2(__fmul_rn(m[i], inv), __fmul_rn(m[i + 1], inv)), __NV_SATFINITE, __NV_E4M3);
    c[i] = u;
    c[i + 1] = u >> 8;
  }
  store_codes(static_cast<uint8_t*>(t.m), s, c);
  if (s.lane == 0) t.m_scale[s.e0 / kBlock] = top * (1.f / kTopM);
}
// The root's codes are the upper bits of a float whose exponent is moved by 120, so that the smallest normal numbers of the
// two formats fall together and the subnormal ones do too.
__device__ __forceinline__ void open_v(const Slot& t, const Span& s, float (&v)[kEach]) {
  uint32_t c[kEach];
  load_codes(static_cast<const uint8_t*>(t.v), s, c);
  const float scale = t.v_scale[s.e0 / kBlock];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const float r = __fmul_rn(__uint_as_float(c[i] << 19) * 0x1p120f, scale);
    v[i] = __fmul_rn(r, r);
  }
}
// (r: the roots)
__device__ __forceinline__ void close_v(const Slot& t, const Span& s, const float (&r)[kEach]) {
  const float top = scale_top(warp_top<false>(r)), inv = __fmul_rn(__frcp_rn(top), kTopV);
  uint32_t c[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const uint32_t b = __float_as_uint(__fmul_rn(r[i], inv) * 0x1p-120f);
    // to even; a root that is not zero divides the step: it does not become zero
    c[i] = max((b + 0x3ffffu + ((b >> 19) & 1u)) >> 19, min(__float_as_uint(r[i]), 1u));
  }
  store_codes(static_cast<uint8_t*>(t.v), s, c);
  if (s.lane == 0) t.v_scale[s.e0 / kBlock] = top * (1.f / kTopV);
}

// The chunks of a launch, SPANS spans per warp each; neighbouring warps take neighbouring spans, so that a tensor of a few spans
// keeps as many warps busy.  f(tensor, the warp's first element).
template <typename F>
__device__ __forceinline__ void for_chunks(const Table& tab, int spans, F&& f) {
  for (long long c = blockIdx.x; c < tab.chunk0[tab.count]; c += gridDim.x) {
    const int k = slot_of(tab, c);
    f(tab.slot[k], (c - tab.chunk0[k]) * (spans * kChunk) + (threadIdx.x >> 5) * kBlock);
  }
}
__device__ __forceinline__ Span span_at(const Slot& t, long long e0) {
  const long long left = t.n - e0;
  return {e0, (int)(left < kBlock ? left : kBlock), (t.flags & kAligned) && left >= kBlock, (int)(threadIdx.x & 31)};
}

// Sum of the gradients' squares, one record per block: eight squares at a time in fp32, then in 64 bits.  Groups whose sum
// leaves the range in which fp32 holds squares are taken in 64 bits from the start.
__device__ __forceinline__ double squares(const float (&g)[kEach]) {
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < kEach; ++i) q = fmaf(g[i], g[i], q);
  if (q > 0x1p-80f && q < 0x1p120f) return q;
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) sum += (double)g[i] * g[i];
  return sum;
}
__device__ __forceinline__ double correction(double beta, long long t) { return 1.0 / (1.0 - pow(beta, (double)t)); }

// JOIN: one span per chunk, and block 0 also counts the step and leaves all scalars but the gradients' factor, which the step's blocks then make.
template <bool JOIN>
__global__ void __launch_bounds__(kWarps * 32) adamw_norm_kernel(const __grid_constant__ Table tab, double* __restrict__ partials,
                                                                 const PrepareArgs a) {
  constexpr int kEachSpans = JOIN ? 1 : kSpans;
  __shared__ double sh[kWarps], corr[2];
  const bool count = JOIN && blockIdx.x == 0;
  const long long taken = count ? *a.step : 0;
  if (count && (threadIdx.x == 192 || threadIdx.x == 224))
    corr[threadIdx.x == 224] = correction(threadIdx.x == 224 ? a.beta2 : a.beta1, taken + 1);
  double sum = 0.0;
  for_chunks(tab, kEachSpans, [&](const Slot& t, long long e0) {
    if (!JOIN && (t.flags & kAligned) && (t.flags & kGrad16) && t.n - e0 >= (kSpans - 1) * kChunk + kBlock) {
      // all loads of the chunk under way at once (one at a time keeps half of the bytes that the memory needs under way)
      uint4 u[kSpans];
#pragma unroll
      for (int q = 0; q < kSpans; ++q)
        u[q] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(t.grad) + e0 + q * kChunk + (threadIdx.x & 31) * kEach);
#pragma unroll
      for (int q = 0; q < kSpans; ++q) {
        float g[kEach];
        rowvec::unpack(u[q], g);
        sum += squares(g);
      }
    } else {
#pragma unroll 1
      for (int q = 0; q < kEachSpans && e0 < t.n; ++q, e0 += kChunk) {
        float g[kEach];
        load(t.grad, t.flags & kGrad16, span_at(t, e0), g);
        sum += squares(g);
      }
    }
  });
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kWarps; ++w) sum += sh[w];
    partials[blockIdx.x] = sum;
    if (count) {
      *a.step = taken + 1;
      *a.out = {0.f, a.lr_dev ? *a.lr_dev : a.lr, (float)corr[0], (float)sqrt(corr[1]), 0, taken + 1};
    }
  }
}

// Thread 0 of a block gets the norm, from the records in a fixed order, and the factor that clips to max_norm.
__device__ __forceinline__ void norm_and_clip(const PrepareArgs& a, double* sh, double* norm, double* clip) {
  double sum = 0.0;
  if (a.partials)
    for (int i = threadIdx.x; i < a.n_partials; i += kWarps * 32) sum += a.partials[i];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int w = 1; w < kWarps; ++w) sum += sh[w];
  *norm = sqrt(sum) * fabs((double)a.grad_scale);
  *clip = a.max_norm > 0.f ? fmin(1.0, a.max_norm / (*norm + 1e-6)) : 1.0;
  if (*norm != *norm && a.max_norm > 0.f) *clip = *norm;
}
__device__ __forceinline__ void write_stats(const PrepareArgs& a, double norm, double clip, bool skip, long long t) {
  if (!a.stats) return;
  a.stats[0] = (float)norm;
  a.stats[1] = (float)clip;
  a.stats[2] = skip ? 1.f : 0.f;
  a.stats[3] = (float)t;
}

// One block.  Two warps raise the betas to the step's number while the others wait for the norm's records.
__global__ void __launch_bounds__(kWarps * 32) adamw_prepare_kernel(PrepareArgs a) {
  __shared__ double sh[kWarps], corr[2];
  const long long taken = *a.step;
  if (threadIdx.x == 192 || threadIdx.x == 224) corr[threadIdx.x == 224] = correction(threadIdx.x == 224 ? a.beta2 : a.beta1, taken + 1);
  double norm, clip;
  norm_and_clip(a, sh, &norm, &clip);
  if (threadIdx.x != 0) return;
  const bool skip = a.partials && a.skip_nonfinite && !(norm < INFINITY);
  if (!skip) *a.step = taken + 1;
  *a.out = {(float)(clip * (double)a.grad_scale), a.lr_dev ? *a.lr_dev : a.lr, (float)corr[0], (float)sqrt(corr[1]), skip ? 1 : 0, taken + 1};
  write_stats(a, norm, clip, skip, taken + (skip ? 0 : 1));
}

// The root of eight values.  Within 2^-100 .. 2^100: one step of the residual form of Newton's iteration from the hardware's
// reciprocal root (P. Markstein, "Computation of elementary functions on the IBM RISC System/6000 processor", 1990), which gives the
// same bits as sqrtf there: for every v of two binades, and with them of all, any reciprocal root within the instruction's documented
// 2^-22.9 leads to the correctly rounded root, but for two v, for which the device's own does (tests/test_adamw_roots.py carries it
// out; the device is tested on the two at every power of four).  Else, zeros among them, sqrtf.
__device__ __forceinline__ void roots(const float (&v)[kEach], float (&r)[kEach]) {
  bool plain = true;
#pragma unroll
  for (int i = 0; i < kEach; ++i) plain &= v[i] > 0x1p-100f && v[i] < 0x1p100f;
  if (plain) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      float y;
      asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(v[i]));
      const float g = __fmul_rn(v[i], y);
      r[i] = __fmaf_rn(__fmaf_rn(-g, g, v[i]), 0.5f * y, g);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i) r[i] = sqrtf(v[i]);
  }
}

__device__ __forceinline__ void open_m(uint2 u, float scale, float (&m)[kEach]) {
#pragma unroll
  for (int i = 0; i < kEach; i += 2) {
    const uint32_t w = (i < 4 ? u.x : u.y) >> (8 * (i % 4));
    const float2 f = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)w, __NV_E4M3)));
    m[i] = __fmul_rn(f.x, scale);
    m[i + 1] = __fmul_rn(f.y, scale);
  }
}
__device__ __forceinline__ void open_v(uint2 u, float scale, float (&v)[kEach]) {
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const uint32_t c = __byte_perm(i < 4 ? u.x : u.y, 0, 0x4440 + i % 4);
    const float r = __fmul_rn(__uint_as_float(c << 19) * 0x1p120f, scale);
    v[i] = __fmul_rn(r, r);
  }
}

// What a lane loads of a whole span with 8-bit states.
struct Raw {
  uint4 g[2], p[2];
  uint2 m, v;
  float m_scale, v_scale;
};
__device__ __forceinline__ void load_raw(const Slot& t, const Span& s, Raw& r) {
  const long long e = s.first();
  if (t.flags & kGrad16) {
    r.g[0] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(t.grad) + e);
  } else {
    r.g[0] = reinterpret_cast<const uint4*>(static_cast<const float*>(t.grad) + e)[0];
    r.g[1] = reinterpret_cast<const uint4*>(static_cast<const float*>(t.grad) + e)[1];
  }
  if (t.master || !(t.flags & kParam16)) {
    const uint4* p = reinterpret_cast<const uint4*>((t.master ? t.master : static_cast<const float*>(t.param)) + e);
    r.p[0] = p[0];
    r.p[1] = p[1];
  } else {
    r.p[0] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(t.param) + e);
  }
  r.m = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.m) + e);
  r.v = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.v) + e);
  r.m_scale = t.m_scale[s.e0 / kBlock];
  r.v_scale = t.v_scale[s.e0 / kBlock];
}
__device__ __forceinline__ void open(const uint4 (&u)[2], bool half, float (&x)[kEach]) {
  if (half) {
    rowvec::unpack(u[0], x);
  } else {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      x[4 * q] = __uint_as_float(u[q].x); x[4 * q + 1] = __uint_as_float(u[q].y);
      x[4 * q + 2] = __uint_as_float(u[q].z); x[4 * q + 3] = __uint_as_float(u[q].w);
    }
  }
}

// The step of the tensors with states of BITS bits.
// JOIN: each block makes the gradients' factor from the norm's records; else the launch before has left it.
template <int BITS, bool JOIN>
__global__ void __launch_bounds__(kWarps * 32, 4) adamw_step_kernel(const __grid_constant__ Table tab, const Hyper h,
                                                                 const Scalars* __restrict__ scalars, const PrepareArgs a) {
  Scalars sc = *scalars;
  if constexpr (JOIN) {
    __shared__ double sh[kWarps];
    __shared__ float g_factor;
    double norm, clip;
    norm_and_clip(a, sh, &norm, &clip);
    if (threadIdx.x == 0) {
      g_factor = (float)(clip * (double)a.grad_scale);
      if (blockIdx.x == 0) write_stats(a, norm, clip, false, sc.t);
    }
    __syncthreads();
    sc.g_factor = g_factor;
  } else if (sc.skip) {
    return;
  }
  for_chunks(tab, 1, [&](const Slot& t, long long e0) {
    if (e0 >= t.n) return;
    const Span s = span_at(t, e0);
    const bool half = t.flags & kParam16;
    float g[kEach], p[kEach], m[kEach], v[kEach], r[kEach];
    if (BITS == 8 && s.vec) {
      Raw now;
      load_raw(t, s, now);
      open(now.g, t.flags & kGrad16, g);
      open(now.p, half && !t.master, p);
      open_m(now.m, now.m_scale, m);
      open_v(now.v, now.v_scale, v);
    } else {
      load(t.grad, t.flags & kGrad16, s, g);
      if (t.master) load32(t.master, s, p);
      else load(t.param, half, s, p);
      if (BITS == 8) {
        open_m(t, s, m);
        open_v(t, s, v);
      } else {
        load32(static_cast<const float*>(t.m), s, m);
        load32(static_cast<const float*>(t.v), s, v);
      }
    }
    const float lr = sc.lr * t.lr_scale, decay = lr * t.weight_decay, rate = lr * sc.c1;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const float x = __fmul_rn(g[i], sc.g_factor);
      // (each operation rounded by itself: a compiler's choice of which product to fuse would decide, near the border of two codes,
      // which of them an 8-bit state gets)
      m[i] = __fadd_rn(__fmul_rn(h.beta1, m[i]), __fmul_rn(h.rest1, x));
      v[i] = __fadd_rn(__fmul_rn(h.beta2, v[i]), __fmul_rn(__fmul_rn(h.rest2, x), x));
    }
    roots(v, r);
    float top = 0.f, step[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      float inv;
      asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(fmaf(r[i], sc.c2, h.eps)));
      step[i] = fmaf(decay, p[i], rate * m[i] * inv);
      top = fmaxf(top, fabsf(p[i]));
    }
    if (top == INFINITY) {                // infinity less a part of itself would be NaN: only an m that is no number changes it
#pragma unroll
      for (int i = 0; i < kEach; ++i) step[i] = fabsf(p[i]) == INFINITY ? 0.f * m[i] : step[i];
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) p[i] -= step[i];
    if (t.master) store32(t.master, s, p);
    store(t.param, half, s, p);
    if (BITS == 8) {
      close_m(t, s, m);
      close_v(t, s, r);
    } else {
      store32(static_cast<float*>(t.m), s, m);
      store32(static_cast<float*>(t.v), s, v);
    }
  });
}

// The states as numbers: param and master stand for the outputs of m and v.
__global__ void __launch_bounds__(kWarps * 32) adamw_states_kernel(const __grid_constant__ Table tab) {
  for_chunks(tab, kSpans, [&](const Slot& t, long long e0) {
    const bool half = t.flags & kOut16;
    const auto write = [&](long long e, const float (&x)[kEach], void* out) { store(out, half, span_at(t, e), x); };
    if ((t.flags & kAligned) && (t.flags & kState8) && t.n - e0 >= (kSpans - 1) * kChunk + kBlock) {
      const auto codes = [&](const void* from, const float* scales, uint2 (&u)[kSpans], float (&scale)[kSpans]) {
#pragma unroll
        for (int q = 0; q < kSpans; ++q) {
          u[q] = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(from) + e0 + q * kChunk + (threadIdx.x & 31) * kEach);
          scale[q] = scales[(e0 + q * kChunk) / kBlock];
        }
      };
      uint2 m[kSpans], v[kSpans];
      float ms[kSpans], vs[kSpans], x[kEach];
      if (t.param) codes(t.m, t.m_scale, m, ms);
      if (t.master) codes(t.v, t.v_scale, v, vs);
#pragma unroll
      for (int q = 0; q < kSpans; ++q) {
        if (t.param) {
          open_m(m[q], ms[q], x);
          write(e0 + q * kChunk, x, t.param);
        }
        if (t.master) {
          open_v(v[q], vs[q], x);
          write(e0 + q * kChunk, x, t.master);
        }
      }
    } else {
#pragma unroll 1
      for (int q = 0; q < kSpans && e0 < t.n; ++q, e0 += kChunk) {
        const Span s = span_at(t, e0);
        float x[kEach];
        if (t.param) {
          if (t.flags & kState8) open_m(t, s, x);
          else load32(static_cast<const float*>(t.m), s, x);
          write(e0, x, t.param);
        }
        if (t.master) {
          if (t.flags & kState8) open_v(t, s, x);
          else load32(static_cast<const float*>(t.v), s, x);
          write(e0, x, t.master);
        }
      }
    }
  });
}

bool aligned_to(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// The states of one tensor as the calls take them.
int check_states(const aero_adamw_tensor& t) {
  if (t.n < 0) return AERO_ERR_INVALID;
  if (t.state_bits != 8 && t.state_bits != 32) return AERO_ERR_UNSUPPORTED;
  if (t.n == 0) return AERO_OK;
  if (!t.m || !t.v) return AERO_ERR_INVALID;
  if (t.state_bits == 8 ? !t.m_scale || !t.v_scale || !aligned_to(t.m_scale, 4) || !aligned_to(t.v_scale, 4)
                        : !aligned_to(t.m, 4) || !aligned_to(t.v, 4))
    return AERO_ERR_INVALID;
  return AERO_OK;
}
int check_tensor(const aero_adamw_tensor& t) {
  const int rc = check_states(t);
  if (rc) return rc;
  for (const int32_t dt : {t.param_dtype, t.grad_dtype})
    if (dt != AERO_BF16 && dt != AERO_FP32) return AERO_ERR_UNSUPPORTED;
  if (t.master && t.param_dtype != AERO_BF16) return AERO_ERR_INVALID;        // the parameter is its own master
  if (!(t.weight_decay >= 0.f) || !(t.lr_scale >= 0.f)) return AERO_ERR_INVALID;
  if (t.n == 0) return AERO_OK;
  if (!t.param || !t.grad) return AERO_ERR_INVALID;
  if (!aligned_to(t.param, t.param_dtype == AERO_FP32 ? 4 : 2) || !aligned_to(t.grad, t.grad_dtype == AERO_FP32 ? 4 : 2) ||
      !aligned_to(t.master, 4))
    return AERO_ERR_INVALID;
  return AERO_OK;
}

// Fills the table with tensors from *next on that have states of so many bits (0: any), leaving empty ones out, and moves *next on.
void fill(Table& tab, const aero_adamw_tensor* tensors, int32_t n, int32_t* next, int bits, int spans) {
  tab.count = 0;
  tab.chunk0[0] = 0;
  for (; *next < n && tab.count < kSlots; ++*next) {
    const aero_adamw_tensor& t = tensors[*next];
    if (t.n == 0 || (bits && t.state_bits != bits)) continue;
    Slot& s = tab.slot[tab.count];
    s = {t.n, t.param, t.grad, t.master, t.m, t.v, t.m_scale, t.v_scale, t.weight_decay, t.lr_scale, 0};
    bool aligned = true;
    for (const void* p : {(const void*)t.param, t.grad, (const void*)t.master, (const void*)t.m, (const void*)t.v})
      aligned &= aligned_to(p, 16);
    s.flags = (t.param_dtype == AERO_BF16 ? kParam16 : 0) | (t.grad_dtype == AERO_BF16 ? kGrad16 : 0) |
              (t.state_bits == 8 ? kState8 : 0) | (aligned ? kAligned : 0);
    tab.chunk0[tab.count + 1] = tab.chunk0[tab.count] + (t.n + spans * kChunk - 1) / (spans * kChunk);
    ++tab.count;
  }
}

int grid_of(const Table& tab, int most) {
  const long long chunks = tab.chunk0[tab.count];
  return (int)(chunks < most ? chunks : most);
}
int launches_of(int32_t n) { return (n + kSlots - 1) / kSlots; }

}  // namespace

extern "C" {

void aero_adamw_cfg_default(aero_adamw_cfg* ac) {
  if (!ac) return;
  ac->lr = 1e-3f; ac->beta1 = 0.9; ac->beta2 = 0.999; ac->eps = 1e-8f;
  ac->max_norm = 0.f; ac->grad_scale = 1.f; ac->skip_nonfinite = 0;
}

size_t aero_adamw_workspace_bytes(int32_t n_tensors) {
  if (n_tensors < 0) return 0;
  return 256 + aero_align_up((size_t)launches_of(n_tensors) * kNormBlocks * sizeof(double), 256);
}

int aero_adamw_step(aero_ctx* ctx, const aero_adamw_cfg* ac, int32_t n_tensors, const aero_adamw_tensor* tensors,
                    int64_t* step, const float* lr, float* stats, void* workspace, size_t workspace_bytes) {
  AeroRange nv("aero_adamw_step");
  if (!ctx || !ac || n_tensors < 0 || (n_tensors > 0 && !tensors) || !step || !workspace || !aero_aligned256(workspace))
    return AERO_ERR_INVALID;
  if (!(ac->beta1 >= 0.0 && ac->beta1 < 1.0) || !(ac->beta2 >= 0.0 && ac->beta2 < 1.0) || !(ac->eps >= 0.f) ||
      !(ac->lr >= 0.f) || !(ac->max_norm < INFINITY) || !(fabsf(ac->grad_scale) < INFINITY))
    return AERO_ERR_INVALID;
  for (int32_t i = 0; i < n_tensors; ++i)
    if (const int rc = check_tensor(tensors[i])) return rc;
  if (workspace_bytes < aero_adamw_workspace_bytes(n_tensors)) return AERO_ERR_WORKSPACE;
  int rc = aero_check_ctx(ctx);
  if (rc) return rc;
  Scalars* scalars = static_cast<Scalars*>(workspace);
  double* partials = reinterpret_cast<double*>(static_cast<char*>(workspace) + 256);
  const bool norm = ac->max_norm > 0.f || ac->skip_nonfinite;
  Table tab;
  PrepareArgs pa = {norm ? partials : nullptr, 0, ac->beta1, ac->beta2, ac->lr, ac->max_norm, ac->grad_scale, ac->skip_nonfinite, lr,
                    reinterpret_cast<long long*>(step), stats, scalars};
  // Small calls have no launch of their own between norm and step: each block of the step adds the norm's records up itself.
  long long chunks = 0, live = 0;
  bool mixed = false;
  for (int32_t i = 0, bits = 0; i < n_tensors; ++i) {
    if (tensors[i].n == 0) continue;
    chunks += (tensors[i].n + kChunk - 1) / kChunk;
    mixed |= bits && bits != tensors[i].state_bits;
    bits = tensors[i].state_bits;
    ++live;
  }
  const bool join = norm && !ac->skip_nonfinite && !mixed && live > 0 && live <= kSlots && chunks <= kJoinChunks;
  if (norm) {
    for (int32_t next = 0; next < n_tensors;) {
      fill(tab, tensors, n_tensors, &next, 0, join ? 1 : kSpans);
      if (tab.count == 0) break;
      const int grid = grid_of(tab, kNormBlocks);
      if (join) adamw_norm_kernel<true><<<grid, kWarps * 32, 0, ctx->stream>>>(tab, partials, pa);
      else adamw_norm_kernel<false><<<grid, kWarps * 32, 0, ctx->stream>>>(tab, partials + pa.n_partials, pa);
      pa.n_partials += grid;
      ctx->launches += 1;
      if (join) break;                // (all tensors that are not empty: the step runs over the same table)
    }
  }
  if (!join) {
    adamw_prepare_kernel<<<1, kWarps * 32, 0, ctx->stream>>>(pa);
    ctx->launches += 1;
  }
  const Hyper h = {(float)ac->beta1, (float)ac->beta2, (float)(1.0 - ac->beta1), (float)(1.0 - ac->beta2), ac->eps};
  if (join) {
    const int grid = grid_of(tab, kJoinChunks);
    if (tab.slot[0].flags & kState8) adamw_step_kernel<8, true><<<grid, kWarps * 32, 0, ctx->stream>>>(tab, h, scalars, pa);
    else adamw_step_kernel<32, true><<<grid, kWarps * 32, 0, ctx->stream>>>(tab, h, scalars, pa);
    ctx->launches += 1;
  } else {
    for (const int bits : {8, 32}) {
      for (int32_t next = 0; next < n_tensors;) {
        fill(tab, tensors, n_tensors, &next, bits, 1);
        if (tab.count == 0) break;
        const int grid = grid_of(tab, kMaxBlocks);
        if (bits == 8) adamw_step_kernel<8, false><<<grid, kWarps * 32, 0, ctx->stream>>>(tab, h, scalars, pa);
        else adamw_step_kernel<32, false><<<grid, kWarps * 32, 0, ctx->stream>>>(tab, h, scalars, pa);
        ctx->launches += 1;
      }
    }
  }
  AERO_CUDA_TRY(cudaGetLastError());
  return AERO_OK;
}

int aero_adamw_states(aero_ctx* ctx, int32_t n_tensors, const aero_adamw_tensor* tensors, int32_t out_dtype, void* const* m_out,
                      void* const* v_out) {
  AeroRange nv("aero_adamw_states");
  if (!ctx || n_tensors < 0 || (n_tensors > 0 && (!tensors || (!m_out && !v_out)))) return AERO_ERR_INVALID;
  if (out_dtype != AERO_BF16 && out_dtype != AERO_FP32) return AERO_ERR_UNSUPPORTED;
  for (int32_t i = 0; i < n_tensors; ++i) {
    if (const int rc = check_states(tensors[i])) return rc;
    for (void* const* out : {m_out, v_out})
      if (out && tensors[i].n > 0 && (!out[i] || !aligned_to(out[i], out_dtype == AERO_FP32 ? 4 : 2))) return AERO_ERR_INVALID;
  }
  int rc = aero_check_ctx(ctx);
  if (rc) return rc;
  Table tab;
  for (int32_t next = 0; next < n_tensors;) {
    int32_t at = next;
    fill(tab, tensors, n_tensors, &next, 0, kSpans);
    if (tab.count == 0) break;
    for (int k = 0; k < tab.count; ++k, ++at) {
      while (tensors[at].n == 0) ++at;
      Slot& s = tab.slot[k];
      s.param = m_out ? m_out[at] : nullptr;
      s.master = v_out ? static_cast<float*>(v_out[at]) : nullptr;
      bool aligned = true;
      for (const void* p : {(const void*)s.param, (const void*)s.master, (const void*)s.m, (const void*)s.v}) aligned &= aligned_to(p, 16);
      s.flags = (s.flags & kState8) | (aligned ? kAligned : 0) | (out_dtype == AERO_BF16 ? kOut16 : 0);
    }
    adamw_states_kernel<<<grid_of(tab, kMaxBlocks), kWarps * 32, 0, ctx->stream>>>(tab);
    ctx->launches += 1;
  }
  AERO_CUDA_TRY(cudaGetLastError());
  return AERO_OK;
}

}  // extern "C"
