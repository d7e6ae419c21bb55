// Rows in 4-bit floating point and the lm_head product of them.  A value is an e2m1 code (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign)
// times the scale of its block of neighbours in the row:
//   block 16: scale = e4m3 code x the row's scale (a power of two that brings the row's largest block scale into e4m3's range)
//   block 32: scale = a power of two (e8m0)
// Rows are kept in the order in which the tensor cores want them in shared memory, so that the product copies whole contiguous
// pieces: codes in tiles of 128 rows x 256 columns (128 bytes a row, 16-byte chunk c of row r at c xor r mod 8), scales in groups of
// 128 rows x 4 blocks (512 bytes: byte 16 (r mod 32) + 4 (r / 32) + k), tiles and groups of a row tile one after the other.
// Rows and columns that fill up the last tiles are zeros.
//   z_tv = h_row_t w_row_v sum_k (scaled h codes)(scaled w codes),   fp32 accumulators of tcgen05 kinds mxf4nvf4 / mxf4, which take the
// block scales from TMEM.  W is operand A (128 or 256 vocabulary rows), the tokens are operand B, as in the 8-bit product.
//   fp4_rows_kernel   up to 128 tokens: bound by reading W once; each CTA streams a contiguous range of vocabulary rows
//   fp4_pair_kernel   more tokens: CTA pairs, 256 vocabulary rows x up to 384 tokens per unit, in two accumulators of 192
#include "entry.cuh"
#include "tc_ptx.cuh"
#include "tmap.cuh"
#include "vec.cuh"

#include <cuda_fp4.h>
#include <cuda_fp8.h>

namespace {

constexpr int kTile = 128, kSlab = 256;                   // rows and columns of a tile of codes
constexpr uint32_t kRowBytes = kSlab / 2, kTileBytes = kTile * kRowBytes, kGroupBytes = 512;
constexpr int kMaxD = 65536;

__host__ __device__ inline long long tiles_of(long long rows) { return (rows + kTile - 1) / kTile; }
__host__ __device__ inline int slabs_of(int d) { return (d + kSlab - 1) / kSlab; }
__host__ __device__ constexpr int groups_per_slab(int block) { return kSlab / (4 * block); }

// ---- rows to 4 bits and back -------------------------------------------------------------------------------------
// A warp per row; a lane takes 16 neighbouring columns, so a step of the warp is 512 columns, two tiles.
constexpr int kLane = 16, kStep = 32 * kLane;

// Where the bytes of codes, and the byte of the scale, of neighbouring columns from c on of row r stand.
__device__ __forceinline__ size_t code_at(long long r, int c, int slabs) {
  const int in = (c % kSlab) / 2, rr = (int)(r % kTile);
  return ((size_t)(r / kTile) * slabs + c / kSlab) * kTileBytes + rr * kRowBytes + (((in / 16) ^ (rr & 7)) * 16) + in % 16;
}
template <int BLOCK>
__device__ __forceinline__ size_t scale_at(long long r, int c, int slabs) {
  const int k = c / BLOCK, rr = (int)(r % kTile);
  return ((size_t)(r / kTile) * slabs * groups_per_slab(BLOCK) + k / 4) * kGroupBytes + (rr % 32) * 16 + rr / 32 * 4 + k % 4;
}

template <typename T> struct Raw16;       // 16 neighbouring elements as they lie in memory
template <> struct Raw16<__nv_bfloat16> {
  uint4 v[2];
  __device__ void load(const __nv_bfloat16* p) {
    v[0] = reinterpret_cast<const uint4*>(p)[0];
    v[1] = reinterpret_cast<const uint4*>(p)[1];
  }
  __device__ void zero() { v[0] = v[1] = make_uint4(0, 0, 0, 0); }
  __device__ void open(float (&x)[16]) const {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      float f[8];
      rowvec::unpack(v[q], f);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[8 * q + i] = f[i];
    }
  }
  // largest magnitude as the bits of a float: a NaN is larger than all
  __device__ uint32_t top() const {
    uint32_t m = 0;
#pragma unroll
    for (int q = 0; q < 2; ++q)
      for (uint32_t w : {v[q].x, v[q].y, v[q].z, v[q].w}) m = __vmaxu2(m, w & 0x7fff7fffu);
    return max(m >> 16, m & 0xffffu) << 16;
  }
};
template <> struct Raw16<float> {
  uint4 v[4];
  __device__ void load(const float* p) {
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = reinterpret_cast<const uint4*>(p)[q];
  }
  __device__ void zero() { v[0] = v[1] = v[2] = v[3] = make_uint4(0, 0, 0, 0); }
  __device__ void open(float (&x)[16]) const {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      x[4 * q] = __uint_as_float(v[q].x); x[4 * q + 1] = __uint_as_float(v[q].y);
      x[4 * q + 2] = __uint_as_float(v[q].z); x[4 * q + 3] = __uint_as_float(v[q].w);
    }
  }
  __device__ uint32_t top() const {
    uint32_t m = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      for (uint32_t w : {v[q].x, v[q].y, v[q].z, v[q].w}) m = max(m, w & 0x7fffffffu);
    return m;
  }
};

__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }      // -126 .. 127

// Eight values' e2m1 codes in a word, the first lowest.
__device__ __forceinline__ uint32_t e2m1_word(const float (&y)[8]) {
  uint32_t w;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(w)
      : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
  return w;
}

// e2m1 codes of 16 values y_i = x_i f / s: f is a power of two, s the value of an e4m3 code (1 for block 32).
// bf16 rows multiply by an approximate 1 / s.  Where x f / s is half way between two codes, which 8 and 4 significant bits often
// make it, the product may fall to either side; any other quotient is at least 2^-8 of itself from there.  Rounding the product
// to a multiple of 2^-12 (by adding 1.5 2^11, in the product's own fma, and taking it off) puts it back: 2 instructions a value
// instead of a division.
template <typename T>
__device__ __forceinline__ uint2 to_e2m1(const float (&x)[16], float f, float s) {
  uint32_t w[2];
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
  const bool small = f > 0x1p100f;                 // (a row so small that f / s might overflow takes f first)
  if (!small) inv *= f;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float v = x[8 * q + i];
      if constexpr (sizeof(T) == 2) {
        constexpr float kSnap = 0x1.8p11f;
        y[i] = __fadd_rn(__fmaf_rn(small ? v * f : v, inv, kSnap), -kSnap);
      } else {
        y[i] = __fdiv_rn(__fmul_rn(v, f), s);
      }
    }
    w[q] = e2m1_word(y);
  }
  return make_uint2(w[0], w[1]);
}

// The e4m3 code of top / 6, to nearest: for bf16 by the same argument, here with a rounding to 14 bits.
template <typename T>
__device__ __forceinline__ uint32_t e4m3_of_sixth(float top) {
  float y;
  if constexpr (sizeof(T) == 2) y = __uint_as_float((__float_as_uint(top * (1.f / 6.f)) + 0x200u) & ~0x3ffu);
  else y = __fdiv_rn(top, 6.f);
  return __nv_cvt_float_to_fp8(y, __NV_SATFINITE, __NV_E4M3);
}

struct QuantArgs {
  long long T;
  int d, slabs;
  const void* x;
  uint8_t* codes;
  uint8_t* scales;
  float* row_scale;
};

// STEPS: steps of 512 columns that stay in registers between the two passes over a row (block 16 needs the whole row's largest
// magnitude first); 0: the second pass reads the row again.
template <typename T, int BLOCK, int STEPS>
__global__ void __launch_bounds__(256) fp4_quantize_kernel(QuantArgs a) {
  const int lane = threadIdx.x & 31;
  const long long r = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);      // up to whole tiles of 128 rows
  const bool there = r < a.T;
  const T* x = static_cast<const T*>(a.x) + r * a.d;
  const int cols = a.slabs * kSlab;
  constexpr int kHeld = STEPS > 0 ? STEPS : 1;
  Raw16<T> held[kHeld];
  uint32_t tops[kHeld];
  float f = 1.f;
  if constexpr (STEPS > 0) {
#pragma unroll
    for (int q = 0; q < STEPS; ++q) {
      const int c = q * kStep + lane * kLane;
      if (there && c < a.d) held[q].load(x + c);
      else held[q].zero();
    }
  }
  if constexpr (BLOCK == 16) {
    uint32_t top = 0;
    if constexpr (STEPS > 0) {
#pragma unroll
      for (int q = 0; q < STEPS; ++q) top = max(top, tops[q] = held[q].top());
    } else if (there) {
      for (int c = lane * kLane; c < a.d; c += kStep) {
        held[0].load(x + c);
        top = max(top, held[0].top());
      }
    }
    top = __reduce_max_sync(0xffffffffu, top);
    // the smallest power of two that brings the largest of the row's scales, top / 6, to 448 at most
    const float row = __uint_as_float(top);
    float scale = 0.f;
    if (!(row < INFINITY)) scale = __uint_as_float(0x7fffffffu);
    else if (row > 0.f) {
      const int e = max((int)((__float_as_uint(__fdiv_rn(row, 2688.f)) + 0x7fffffu) >> 23) - 127, -126);
      scale = power_of_two(e);
      f = power_of_two(-e);
    }
    if (there && lane == 0) a.row_scale[r] = scale;
  }
  // where the first step's codes and scales go; the next one's are two tiles further
  constexpr int kApart = BLOCK / kLane;                      // lanes from one block to the next
  constexpr int kTilesPerStep = kStep / kSlab;
  uint8_t* codes = a.codes + code_at(r, lane * kLane, a.slabs);
  uint8_t* scales = a.scales + scale_at<BLOCK>(r, lane * kLane, a.slabs);
#pragma unroll (STEPS > 0 ? STEPS : 1)
  for (int q = 0; q < (STEPS > 0 ? STEPS : 1 << 20); ++q) {
    const int c = q * kStep + lane * kLane;
    if (q * kStep >= cols) break;
    if constexpr (STEPS == 0) {
      if (there && c < a.d) held[0].load(x + c);
      else held[0].zero();
    }
    const Raw16<T>& h = held[STEPS > 0 ? q : 0];
    float s = 1.f, factor = f;
    uint32_t byte, top = BLOCK == 16 && STEPS > 0 ? tops[STEPS > 0 ? q : 0] : h.top();
    if constexpr (BLOCK == 16) {
      byte = e4m3_of_sixth<T>(__uint_as_float(top) * f);
      s = __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)byte, __NV_E4M3)));
    } else {
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      // (the exponent that brings the largest into [4, 8); infinity or NaN: the scale's NaN)
      const int e = max((int)(top >> 23) - 129, -127);
      byte = top >= 0x7f800000u ? 255u : (uint32_t)(e + 127);
      factor = power_of_two(min(-e, 127));
    }
    float v[16];
    h.open(v);
    uint2 code = to_e2m1<T>(v, factor, s);
    if (!(s > 0.f)) code = make_uint2(0, 0);
    // four blocks' scales are neighbours: gathered into a word
    uint32_t word = byte;
#pragma unroll
    for (int k = 1; k < 4; ++k) word |= __shfl_down_sync(0xffffffffu, byte, k * kApart) << (8 * k);
    if (c < cols) {
      *reinterpret_cast<uint2*>(codes) = code;
      if (lane % (4 * kApart) == 0) *reinterpret_cast<uint32_t*>(scales) = word;
    }
    codes += kTilesPerStep * kTileBytes;
    scales += kTilesPerStep * groups_per_slab(BLOCK) * kGroupBytes;
  }
}

struct ValueArgs {
  long long T;
  int d, slabs;
  const uint8_t* codes;
  const uint8_t* scales;
  const float* row_scale;
  void* out;
};

// A lane takes 8 neighbouring columns of each tile, so that a warp's stores are whole lines; the loads of kAhead tiles go first.
template <typename O, int BLOCK>
__global__ void __launch_bounds__(256) fp4_values_kernel(ValueArgs a) {
  constexpr int kAhead = 4, kCols = kSlab / 32;
  const int lane = threadIdx.x & 31;
  const long long r = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (r >= a.T) return;
  const float row = BLOCK == 16 ? a.row_scale[r] : 1.f;
  O* out = static_cast<O*>(a.out) + r * a.d + lane * kCols;
  const uint8_t* codes = a.codes + code_at(r, lane * kCols, a.slabs);
  const uint8_t* scales = a.scales + scale_at<BLOCK>(r, lane * kCols, a.slabs);
  for (int t0 = 0; t0 < a.slabs; t0 += kAhead) {
    uint32_t w[kAhead], byte[kAhead];
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      if (t0 + q < a.slabs) {
        w[q] = *reinterpret_cast<const uint32_t*>(codes + (size_t)(t0 + q) * kTileBytes);
        byte[q] = scales[(size_t)(t0 + q) * groups_per_slab(BLOCK) * kGroupBytes];
      }
    }
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      if ((t0 + q) * kSlab + lane * kCols >= a.d) break;
      float s;
      if constexpr (BLOCK == 16) s = row * __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)byte[q], __NV_E4M3)));
      else s = byte[q] == 255 ? __uint_as_float(0x7fffffffu) : (byte[q] == 0 ? 0x1p-127f : __uint_as_float(byte[q] << 23));
      float v[kCols];
#pragma unroll
      for (int i = 0; i < kCols; i += 2) {
        const float2 y = __half22float2(__half2(__nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)(w[q] >> (4 * i)), __NV_E2M1)));
        v[i] = y.x * s;
        v[i + 1] = y.y * s;
      }
      constexpr int VEC = rowvec::Elem<O>::kVec;
#pragma unroll
      for (int i = 0; i < kCols; i += VEC) {
        float part[VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k) part[k] = v[i + k];
        rowvec::store<O, VEC>(out + (size_t)(t0 + q) * kSlab + i, part);
      }
    }
  }
}

// ---- the product ---------------------------------------------------------------------------------------------------
// Warps 0-7 epilogue (one vocabulary row per thread, two warps per quadrant of TMEM), warp 8 copies, warp 9 MMA, warps 10-13 scales:
// each reads the groups of scales that have arrived and stores them to its quadrant's lanes (the tensor cores want all four
// alike).  The asynchronous copy that brings 512 bytes to all quadrants, issued between the products, held these up by 60 cycles
// each, 12 times for 4 products of 150 cycles (2048 tokens, d = 3584, V = 152064: 1008 us with it).
constexpr int EPI_WARPS = 8, kShare = EPI_WARPS / 4, SCALE_WARPS = 4, THREADS = (EPI_WARPS + 2 + SCALE_WARPS) * 32;
constexpr int kRowsN = 128, kPairN = 192, kPairT = 2 * kPairN;         // most tokens per tile
constexpr int kRowBlock = 32;                     // fp4_rows_kernel: ranges of vocabulary rows are multiples of it
constexpr int kMaxStages = 8, kMaxSets = 8;
constexpr uint32_t kScaleCols = 256;              // fp4_rows_kernel: first TMEM column of the scales
constexpr size_t kRing = 204 * 1024;

template <int STAGES>
struct Ctl {
  uint64_t full[STAGES], empty[STAGES], tfull[2], tempty[2];
  uint64_t sfull[STAGES];       // pair kernel: a stage's scales have arrived in this CTA
  uint64_t scales[STAGES];      // scales are in TMEM: of a stage (rows), of a set (pair)
  uint32_t tmem_base;
  int abort;
};
// GROUPS groups of 512 bytes of scales (this thread's 16 bytes of each) to 4 columns each of this warp's quadrant
template <int GROUPS>
__device__ __forceinline__ void scales_to_tmem(uint32_t taddr, const uint8_t* smem, int lane) {
  uint32_t r[4 * GROUPS];
#pragma unroll
  for (int g = 0; g < GROUPS; ++g) {
    const uint4 v = *reinterpret_cast<const uint4*>(smem + g * kGroupBytes + lane * 16);
    r[4 * g] = v.x; r[4 * g + 1] = v.y; r[4 * g + 2] = v.z; r[4 * g + 3] = v.w;
  }
  tc::tmem_st_32x32<4 * GROUPS>(taddr, r);
}
constexpr size_t R_SMEM = 1024 + kRing + sizeof(Ctl<kMaxStages>);

struct Operand {
  const uint8_t* codes;
  const uint8_t* scales;
  const float* row;           // NULL: 1
};
struct Params {
  int T, V, slabs;
  int n;                      // fp4_rows_kernel: tokens in steps of 16 (N of the products)
  int n_tok;                  // fp4_pair_kernel: token tiles
  Operand h, w;
  void* out;
  uint32_t* status;
  int stages, per;            // fp4_rows_kernel: depth of the ring, slabs per stage
};

// Writes the accumulator columns of tokens t0 .. t0 + n of vocabulary row v: a thread has one row, so the 32 lanes of a warp store
// 32 neighbouring logits of a token at a time; the two warps of a quadrant of TMEM take chunks of 32 tokens in turn.  The rows'
// scales are loaded before the accumulator is waited for, a token's by a lane each.
template <typename O, int N>
struct Epilogue {                // of fp4_rows_kernel
  static constexpr int kChunks = (N / 32 + kShare - 1) / kShare;
  float sh[kChunks];
  float sw;
  __device__ void load_scales(const Params& p, int t0, int half, int lane, int v) {
    sw = v < p.V && p.w.row ? p.w.row[v] : 1.f;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      const int t = (kShare * i + half) * 32 + lane;
      sh[i] = t < p.n && t0 + t < p.T ? (p.h.row ? p.h.row[t0 + t] : 1.f) : 0.f;
    }
  }
  __device__ void store(const Params& p, uint32_t taddr, int t0, int half, int v, bool row_ok) const {
    const int n = min(p.n, p.T - t0);
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      const int c = (kShare * i + half) * 32, left = min(32, n - c);
      if (left <= 0) break;
      uint32_t r[32];
      __syncwarp();                                  // the TMEM load is warp-collective
      tc::tmem_ld_32x32(taddr + c, r);
      tc::tmem_ld_wait();
      O* o = static_cast<O*>(p.out) + (size_t)(t0 + c) * p.V + v;
#pragma unroll
      for (int q = 0; q < 32; ++q) {
        const float z = __uint_as_float(r[q]) * __shfl_sync(0xffffffffu, sh[i], q) * sw;
        if (row_ok && q < left) rowvec::Elem<O>::store(o, z);
        o += p.V;
      }
    }
  }
};

template <typename O, int BLOCK>
__global__ void __launch_bounds__(THREADS, 1) fp4_rows_kernel(const Params p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  // a stage is `per` slabs of 256 columns: codes of 128 rows of W, of the n tokens, then the scales of both
  constexpr int kGroups = groups_per_slab(BLOCK);
  constexpr uint32_t kScales = kGroups * kGroupBytes, kSetCols = 2 * 4 * kGroups;
  const int per = p.per, stages = p.stages;
  const uint32_t b_slab = (uint32_t)p.n * kRowBytes, slab_bytes = kTileBytes + b_slab + 2 * kScales;
  auto* ctl = reinterpret_cast<Ctl<kMaxStages>*>(smem + (size_t)stages * per * slab_bytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      tc::mbar_init(&ctl->full[s], 1);
      tc::mbar_init(&ctl->empty[s], 1);
      tc::mbar_init(&ctl->scales[s], SCALE_WARPS);
    }
    for (int b = 0; b < 2; ++b) { tc::mbar_init(&ctl->tfull[b], 1); tc::mbar_init(&ctl->tempty[b], EPI_WARPS); }
    ctl->abort = 0;
    tc::fence_barrier_init();
  }
  if (warp == EPI_WARPS + 1) { tc::tmem_alloc(&ctl->tmem_base, 512); tc::tmem_relinquish(); }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem_base = ctl->tmem_base;
  volatile int* abort_flag = &ctl->abort;
  // this CTA's vocabulary rows, in blocks of 32, cut where tiles of 128 begin
  const int blocks = (p.V + kRowBlock - 1) / kRowBlock;
  const int b0 = (int)((long long)blocks * blockIdx.x / gridDim.x), b1 = (int)((long long)blocks * (blockIdx.x + 1) / gridDim.x);
  constexpr int kPerTile = kTile / kRowBlock;
  auto step = [&](int b) { return min(kPerTile - b % kPerTile, b1 - b); };
  const int nkb = p.slabs;

  if (warp == EPI_WARPS) {
    if (lane == 0) {
      int s = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int b = b0; ok && b < b1; b += step(b)) {
        const int first = b % kPerTile;
        const uint32_t a_bytes = (uint32_t)step(b) * kRowBlock * kRowBytes;
        const size_t tile = b / kPerTile;
        for (int kb = 0; kb < nkb; kb += per) {
          if (!tc::mbar_wait(&ctl->empty[s], ph ^ 1u, abort_flag)) { ok = false; break; }
          const int nk = min(per, nkb - kb);
          uint8_t* at = smem + (size_t)s * per * slab_bytes;
          tc::mbar_arrive_expect_tx(&ctl->full[s], (uint32_t)nk * (a_bytes + b_slab + 2 * kScales));
          for (int k = 0; k < nk; ++k, at += slab_bytes) {
            const size_t slab = kb + k;
            tc::bulk_load(at + first * kRowBlock * kRowBytes,
                          p.w.codes + (tile * nkb + slab) * kTileBytes + first * kRowBlock * kRowBytes, a_bytes, &ctl->full[s]);
            tc::bulk_load(at + kTileBytes, p.h.codes + slab * kTileBytes, b_slab, &ctl->full[s]);
            tc::bulk_load(at + kTileBytes + b_slab, p.w.scales + (tile * nkb + slab) * kScales, kScales, &ctl->full[s]);
            tc::bulk_load(at + kTileBytes + b_slab + kScales, p.h.scales + slab * kScales, kScales, &ctl->full[s]);
          }
          if (++s == stages) { s = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp == EPI_WARPS + 1) {
    if (lane == 0) {
      int s = 0;
      uint32_t ph = 0, at = 0;
      bool ok = true;
      for (int b = b0; ok && b < b1; b += step(b), ++at) {
        const uint32_t buf = at & 1u;
        if (!tc::mbar_wait(&ctl->tempty[buf], ((at >> 1) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
        tc::tc_fence_after();
        for (int kb = 0; kb < nkb; kb += per) {
          // (the scales' warps have waited for the whole stage)
          if (!tc::mbar_wait(&ctl->scales[s], ph, abort_flag)) { ok = false; break; }
          tc::tc_fence_after();
          // (a tile of fewer than 128 rows leaves older codes in the other rows of A: their accumulator rows are not read)
          const int nk = min(per, nkb - kb);
          for (int k = 0; k < nk; ++k) {
            const uint32_t a_addr = tc::smem_u32(smem + (size_t)(s * per + k) * slab_bytes);
            // each place of the ring has scale columns of its own
            const uint32_t sfa = tmem_base + kScaleCols + (uint32_t)(s * per + k) * kSetCols, sfb = sfa + 4 * kGroups;
            const uint64_t adesc = tc::make_smem_desc(a_addr, 16, 1024), bdesc = tc::make_smem_desc(a_addr + kTileBytes, 16, 1024);
#pragma unroll
            for (int kk = 0; kk < kSlab / 64; ++kk) {
              const int g = kk * kGroups / 4;               // block 32: a group holds two instructions' scales
              const uint32_t idesc = tc::make_idesc_fp4(kTile, p.n, BLOCK == 32, BLOCK == 32 ? 2 * (kk & 1) : 0);
              tc::umma_fp4<BLOCK, false>(tmem_base + buf * kRowsN, adesc + 2u * kk, bdesc + 2u * kk, idesc, sfa + 4 * g, sfb + 4 * g,
                                         (kb | k | kk) != 0 ? 1u : 0u);
            }
          }
          tc::umma_commit(&ctl->empty[s]);
          if (++s == stages) { s = 0; ph ^= 1u; }
        }
        if (ok) tc::umma_commit(&ctl->tfull[buf]);
      }
    }
  } else if (warp >= EPI_WARPS + 2) {
    const int quad = warp & 3;                   // (a warp reaches the lanes of its number mod 4)
    int s = 0;
    uint32_t ph = 0;
    bool ok = true;
    for (int b = b0; ok && b < b1; b += step(b)) {
      for (int kb = 0; kb < nkb; kb += per) {
        if (!__all_sync(0xffffffffu, tc::mbar_wait(&ctl->full[s], ph, abort_flag))) { ok = false; break; }
        tc::tc_fence_after();                    // the products of the ring's turn before have read these columns
        const int nk = min(per, nkb - kb);
        for (int k = 0; k < nk; ++k) {
          const uint8_t* from = smem + (size_t)(s * per + k) * slab_bytes + kTileBytes + b_slab;
          const uint32_t to = tmem_base + ((uint32_t)(quad * 32) << 16) + kScaleCols + (uint32_t)(s * per + k) * kSetCols;
          scales_to_tmem<kGroups>(to, from, lane);
          scales_to_tmem<kGroups>(to + 4 * kGroups, from + kScales, lane);
        }
        tc::tmem_st_wait();
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&ctl->scales[s]);
        if (++s == stages) { s = 0; ph ^= 1u; }
      }
    }
  } else {
    uint32_t at = 0;
    const int quad = warp & 3, half = warp >> 2;
    Epilogue<O, kRowsN> epi;
    for (int b = b0; b < b1; b += step(b), ++at) {
      const uint32_t buf = at & 1u;
      const int first = b % kPerTile, v = b / kPerTile * kTile + quad * 32 + lane;
      epi.load_scales(p, 0, half, lane, v);
      if (!__all_sync(0xffffffffu, tc::mbar_wait(&ctl->tfull[buf], (at >> 1) & 1u, abort_flag))) break;
      tc::tc_fence_after();
      if (quad >= first && quad < first + step(b))         // this warp's block of 32 rows is among this CTA's
        epi.store(p, tmem_base + ((uint32_t)(quad * 32) << 16) + buf * kRowsN, 0, half, v, v < p.V);
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&ctl->tempty[buf]);
    }
  }
  __syncwarp();
  if (*abort_flag) {
    const unsigned long long t0 = tc::globaltimer_ns();
    while (tc::globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
  }
  tc::tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) aero_raise(p.status, AERO_ST_TIMEOUT);
  if (warp == EPI_WARPS + 1) {
    tc::tc_fence_after();
    tc::tmem_dealloc(tmem_base, 512);
  }
}

// 32 logits of a vocabulary row in registers: accumulators times the scales of their tokens (in shared memory) and of the row.
__device__ __forceinline__ void scaled(const uint32_t* r, const float* scales, float sw, float (&z)[4]) {
  const float4 s = *reinterpret_cast<const float4*>(scales);
  z[0] = __uint_as_float(r[0]) * s.x * sw; z[1] = __uint_as_float(r[1]) * s.y * sw;
  z[2] = __uint_as_float(r[2]) * s.z * sw; z[3] = __uint_as_float(r[3]) * s.w * sw;
}
template <typename O> struct Held;
template <> struct Held<float> {
  float v[32];
  __device__ void take(int half, const uint32_t (&r)[16], const float* scales, float sw) {
#pragma unroll
    for (int q = 0; q < 16; q += 4) {
      float z[4];
      scaled(r + q, scales + 16 * half + q, sw, z);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[16 * half + q + k] = z[k];
    }
  }
  __device__ float at(int q) const { return v[q]; }
};
template <> struct Held<__nv_bfloat16> {
  __nv_bfloat162 v[16];
  __device__ void take(int half, const uint32_t (&r)[16], const float* scales, float sw) {
#pragma unroll
    for (int q = 0; q < 16; q += 4) {
      float z[4];
      scaled(r + q, scales + 16 * half + q, sw, z);
      v[8 * half + q / 2] = __floats2bfloat162_rn(z[0], z[1]);
      v[8 * half + q / 2 + 1] = __floats2bfloat162_rn(z[2], z[3]);
    }
  }
  __device__ __nv_bfloat16 at(int q) const { return q & 1 ? v[q / 2].y : v[q / 2].x; }
};

// The tokens of a unit are as many as the accumulators hold, 2 x 192 (of 512 columns of TMEM 128 hold scales), and both accumulators
// use the rows of W that were loaded once: with units of 192 tokens the SMs' reads from L2, 10 TB/s, were the bound (2048
// tokens of d = 3584, V = 152064 701 us).  The accumulators are emptied into registers as soon as their products are done, rounded there,
// and stored while the next unit's products run; what is left of the time is the products (96 cycles each, 430 us at the clock that the
// power allows), that emptying, and the round trips of the scales: 690 us in a row at 1.61 GHz under the power cap, 634 alone, 574 in a row
// in one run whose clock was not sampled.  Half the scales (block 32: 657 in a row at 1.66 GHz) save 1.6 % of the cycles, so reading them is
// not what bounds it.
// A stage, per CTA: codes of 128 rows of W and of its half of each accumulator's tokens, scales of these rows of W, and of the three
// groups of 128 token rows (both CTAs' tensor cores multiply all columns).
constexpr int PSTAGES = 4, kPiece = 32, kTokenGroups = kPairT / kTile;
constexpr uint32_t kHalfBytes = kPairN / 2 * kRowBytes;
__host__ __device__ constexpr uint32_t pair_stage(int block) {
  return kTileBytes + 2 * kHalfBytes + (1 + kTokenGroups) * groups_per_slab(block) * kGroupBytes;
}
struct PairCtl : Ctl<PSTAGES> {
  alignas(16) float token_scales[EPI_WARPS * kPairT / kShare];      // each warp's own tokens, of both accumulators
};
constexpr size_t p_smem(int block) { return 1024 + (size_t)PSTAGES * pair_stage(block) + sizeof(PairCtl); }

// Tokens of each accumulator in the unit that begins with token t0: half of what is left, in steps of 64.
__host__ __device__ inline int pair_n(int T, int t0) {
  const int n = ((T - t0 + 1) / 2 + 63) / 64 * 64;
  return n < kPairN ? n : kPairN;
}

template <typename O, int BLOCK>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1)
fp4_pair_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmWs,
                const __grid_constant__ CUtensorMap tmH, const __grid_constant__ CUtensorMap tmHs, const Params p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  constexpr int kGroups = groups_per_slab(BLOCK);
  constexpr uint32_t kStage = pair_stage(BLOCK), kScales = kGroups * kGroupBytes;
  // columns of TMEM: two accumulators, then kSets sets of a slab's scales, W's and for each k step the tokens'.  (Four sets of half a
  // slab were slower, 969 us for 662: a set's way through the scales' warps is longer than the products of half a slab.)
  constexpr int kSets = 2;
  constexpr uint32_t kSetCols = 4 * kGroups * (1 + kTokenGroups), kScaleBase = 2 * kPairN;
  static_assert(kScaleBase + kSets * kSetCols <= 512, "TMEM");
  auto* ctl = reinterpret_cast<PairCtl*>(smem + (size_t)PSTAGES * kStage);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = tc::cluster_ctarank();        // 0 issues the MMAs of the pair
  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
  if (threadIdx.x == 0) {
    for (int s = 0; s < PSTAGES; ++s) {
      tc::mbar_init(&ctl->full[s], 1);
      tc::mbar_init(&ctl->empty[s], 1);
      tc::mbar_init(&ctl->sfull[s], 1);
    }
    for (int k = 0; k < kSets; ++k) tc::mbar_init(&ctl->scales[k], 2 * SCALE_WARPS);
    for (int b = 0; b < 2; ++b) { tc::mbar_init(&ctl->tfull[b], 1); tc::mbar_init(&ctl->tempty[b], 2 * EPI_WARPS); }
    ctl->abort = 0;
    tc::fence_barrier_init();
  }
  if (warp == EPI_WARPS && lane == 0) { tc::prefetch_tmap(&tmW); tc::prefetch_tmap(&tmWs); tc::prefetch_tmap(&tmH); tc::prefetch_tmap(&tmHs); }
  if (warp == EPI_WARPS + 1) { tc::tmem_alloc_pair(&ctl->tmem_base, 512); tc::tmem_relinquish_pair(); }
  tc::tc_fence_before();
  __syncthreads();
  tc::cluster_sync_all();        // the peer's barriers exist before anything signals them
  tc::tc_fence_after();
  const uint32_t tmem_base = ctl->tmem_base;
  volatile int* abort_flag = &ctl->abort;
  // a unit is 256 vocabulary rows x one token tile; the units of one row tile are neighbours, so that
  // pairs running at the same time read the same W rows from L2
  const long long units = (long long)((p.V + 2 * kTile - 1) / (2 * kTile)) * p.n_tok;
  const int nkb = p.slabs;

  if (warp == EPI_WARPS) {
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      for (long long u = pair; ok && u < units; u += npairs) {
        const int tile = (int)(u / p.n_tok) * 2 + (int)rank, t0 = (int)(u % p.n_tok) * kPairT, n = pair_n(p.T, t0);
        const uint32_t bytes = 2 * (kTileBytes + (uint32_t)n * kRowBytes);
        for (int kb = 0; kb < nkb; ++kb, ++it) {
          const int s = it % PSTAGES;
          if (!tc::mbar_wait(&ctl->empty[s], ((it / PSTAGES) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
          uint8_t* at = smem + (size_t)s * kStage;
          const uint32_t full0 = tc::mapa_shared(tc::smem_u32(&ctl->full[s]), 0);
          if (rank == 0) tc::mbar_arrive_expect_tx(&ctl->full[s], bytes);
          // (rows past the last tile of W or of the tokens are filled with zeros by the copies)
          tc::tma_load_2d_pair(at, &tmW, 0, (tile * nkb + kb) * kTile, full0);
          for (int acc = 0; acc < 2; ++acc) {
            for (int i = 0; i < n / 2 / kPiece; ++i) {
              const int t = t0 + acc * n + (int)rank * (n / 2) + i * kPiece;
              tc::tma_load_2d_pair(at + kTileBytes + acc * kHalfBytes + i * kPiece * kRowBytes, &tmH, 0,
                                   (t / kTile * nkb + kb) * kTile + t % kTile, full0);
            }
          }
          at += kTileBytes + 2 * kHalfBytes;
          tc::mbar_arrive_expect_tx(&ctl->sfull[s], (1 + kTokenGroups) * kScales);
          tc::tma_load_2d(at, &tmWs, 0, (tile * nkb + kb) * kGroups, &ctl->sfull[s]);
          for (int i = 0; i < kTokenGroups; ++i)
            tc::tma_load_2d(at + (1 + i) * kScales, &tmHs, 0, ((t0 / kTile + i) * nkb + kb) * kGroups, &ctl->sfull[s]);
        }
      }
    }
  } else if (warp == EPI_WARPS + 1) {
    if (lane == 0 && rank == 0) {
      uint32_t it = 0, at = 0;
      bool ok = true;
      for (long long u = pair; ok && u < units; u += npairs, ++at) {
        const int n = pair_n(p.T, (int)(u % p.n_tok) * kPairT);
        for (int kb = 0; ok && kb < nkb; ++kb, ++it) {
          const int s = it % PSTAGES;
          if (!tc::mbar_wait(&ctl->full[s], (it / PSTAGES) & 1u, abort_flag) ||
              !tc::mbar_wait(&ctl->scales[it % kSets], (it / kSets) & 1u, abort_flag)) { ok = false; break; }
          const uint32_t a_addr = tc::smem_u32(smem + (size_t)s * kStage);
          const uint32_t sfa = tmem_base + kScaleBase + (it % kSets) * kSetCols;
          for (int acc = 0; acc < 2; ++acc) {
            // the accumulator of the unit before has been read
            if (kb == 0 && !tc::mbar_wait(&ctl->tempty[acc], (at & 1u) ^ 1u, abort_flag)) { ok = false; break; }
            tc::tc_fence_after();
            // (a column holds the scales of 32 rows)
            const uint32_t sfb = sfa + 4 * kGroups + (uint32_t)(acc * n) / 32;
            const uint64_t adesc = tc::make_smem_desc(a_addr, 16, 1024);
            const uint64_t bdesc = tc::make_smem_desc(a_addr + kTileBytes + acc * kHalfBytes, 16, 1024);
#pragma unroll
            for (int kk = 0; kk < kSlab / 64; ++kk) {
              const int g = kk * kGroups / 4;                     // block 32: a group holds two instructions' scales
              const uint32_t idesc = tc::make_idesc_fp4(2 * kTile, n, BLOCK == 32, BLOCK == 32 ? 2 * (kk & 1) : 0);
              tc::umma_fp4<BLOCK, true>(tmem_base + acc * kPairN, adesc + 2u * kk, bdesc + 2u * kk, idesc, sfa + 4 * g,
                                        sfb + 4 * kTokenGroups * g, (kb | kk) != 0 ? 1u : 0u);
            }
            if (kb == nkb - 1) tc::umma_commit_pair(&ctl->tfull[acc], 3);
          }
          if (ok) tc::umma_commit_pair(&ctl->empty[s], 3);     // frees the stage in both CTAs when these MMAs retire
        }
      }
    }
  } else if (warp >= EPI_WARPS + 2) {
    const int quad = warp & 3;                   // (a warp reaches the lanes of its number mod 4)
    uint32_t it = 0;
    bool ok = true;
    for (long long u = pair; ok && u < units; u += npairs) {
      for (int kb = 0; kb < nkb; ++kb, ++it) {
        const int s = it % PSTAGES;
        if (!__all_sync(0xffffffffu, tc::mbar_wait(&ctl->sfull[s], (it / PSTAGES) & 1u, abort_flag))) { ok = false; break; }
        const uint8_t* from = smem + (size_t)s * kStage + kTileBytes + 2 * kHalfBytes + lane * 16;
        // W's, then for each k step the tokens' three groups of rows side by side
        uint32_t r[4 * kGroups * (1 + kTokenGroups)];
#pragma unroll
        for (int k = 0; k < kGroups * (1 + kTokenGroups); ++k) {
          const int g = k < kGroups ? k : (k - kGroups) / kTokenGroups, i = k < kGroups ? 0 : 1 + (k - kGroups) % kTokenGroups;
          const uint4 v = *reinterpret_cast<const uint4*>(from + i * kScales + g * kGroupBytes);
          r[4 * k] = v.x; r[4 * k + 1] = v.y; r[4 * k + 2] = v.z; r[4 * k + 3] = v.w;
        }
        // the set's columns are free when the products of kSets slabs ago have retired, which their stage's barrier tells
        const uint32_t old = it - kSets;
        const bool free = it < (uint32_t)kSets || tc::mbar_wait(&ctl->empty[old % PSTAGES], (old / PSTAGES) & 1u, abort_flag);
        if (!__all_sync(0xffffffffu, free)) { ok = false; break; }
        tc::tc_fence_after();
        const uint32_t to = tmem_base + ((uint32_t)(quad * 32) << 16) + kScaleBase + (it % kSets) * kSetCols;
        constexpr int kPart = 8 * kGroups;                       // (32 columns a store at most)
#pragma unroll
        for (int k = 0; k < 4 * kGroups * (1 + kTokenGroups); k += kPart) tc::tmem_st_32x32<kPart>(to + k, r + k);
        tc::tmem_st_wait();
        tc::tc_fence_before();
        __syncwarp();
        // (the stores to this CTA's TMEM, which its own tensor core reads, are complete)
        if (lane == 0) tc::mbar_arrive_cluster_bare(tc::mapa_shared(tc::smem_u32(&ctl->scales[it % kSets]), 0));
      }
    }
  } else {
    // a thread has a vocabulary row, so the 32 lanes of a warp store 32 neighbouring logits of a token at a time; the two warps of a
    // quadrant of TMEM take chunks of 32 tokens in turn.  (The products of the next unit wait for the accumulators to be emptied, so
    // what is between a wait and its release is kept short, and all of it small enough for the instruction cache.)
    constexpr int kChunks = kPairN / 32 / kShare;
    uint32_t at = 0;
    const int quad = warp & 3, half = warp >> 2;
    float* scales = ctl->token_scales + warp * 2 * kChunks * 32;       // of this warp's tokens
    for (long long u = pair; u < units; u += npairs, ++at) {
      const int t0 = (int)(u % p.n_tok) * kPairT, n = pair_n(p.T, t0);
      const int v = (int)(u / p.n_tok) * 2 * kTile + (int)rank * kTile + quad * 32 + lane;
      const bool row_ok = v < p.V;
      const float sw = row_ok && p.w.row ? p.w.row[v] : 1.f;
#pragma unroll
      for (int i = 0; i < 2 * kChunks; ++i) {
        const int t = t0 + (i / kChunks) * n + (kShare * (i % kChunks) + half) * 32 + lane;
        scales[i * 32 + lane] = t < p.T && p.h.row ? p.h.row[t] : 1.f;
      }
      __syncwarp();
      const auto take = [&](int acc, Held<O> (&held)[kChunks]) {
        if (!__all_sync(0xffffffffu, tc::mbar_wait(&ctl->tfull[acc], at & 1u, abort_flag))) return false;
        tc::tc_fence_after();
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
          const int c = (kShare * i + half) * 32;
          if (c < n) {
            // (in halves: the registers left beside the chunks that are held)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              uint32_t r[16];
              __syncwarp();                                // the TMEM load is warp-collective
              tc::tmem_ld_32x16(tmem_base + ((uint32_t)(quad * 32) << 16) + acc * kPairN + c + 16 * k, r);
              tc::tmem_ld_wait();
              held[i].take(k, r, scales + (acc * kChunks + i) * 32, sw);
            }
          }
        }
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive_cluster_bare(tc::mapa_shared(tc::smem_u32(&ctl->tempty[acc]), 0));     // (TMEM has been read)
        return true;
      };
      const auto put = [&](int acc, const Held<O> (&held)[kChunks]) {
        const uint32_t stride = (uint32_t)p.V * (uint32_t)sizeof(O);      // (V <= 2^30)
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
          const int c = t0 + acc * n + (kShare * i + half) * 32, left = row_ok ? min(n - (kShare * i + half) * 32, p.T - c) : 0;
          uint8_t* o = static_cast<uint8_t*>(p.out) + ((long long)c * p.V + v) * (long long)sizeof(O);
          if (__all_sync(0xffffffffu, left >= 32)) {
#pragma unroll
            for (int q = 0; q < 32; ++q, o += stride) *reinterpret_cast<O*>(o) = held[i].at(q);
          } else if (left > 0) {
#pragma unroll
            for (int q = 0; q < 32; ++q, o += stride)
              if (q < left) *reinterpret_cast<O*>(o) = held[i].at(q);
          }
        }
      };
      // both accumulators are emptied before anything is stored where the registers hold them (stored in turn: 690 us for 662)
      Held<O> first[kChunks], second[kChunks];
      if (!take(0, first)) break;
      if (sizeof(O) == 4) put(0, first);
      if (!take(1, second)) break;
      if (sizeof(O) == 2) put(0, first);
      put(1, second);
      __syncwarp();                                        // (before the next unit's scales)
    }
  }
  __syncwarp();
  if (*abort_flag) {
    const unsigned long long t0 = tc::globaltimer_ns();
    while (tc::globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
  }
  tc::tc_fence_before();
  __syncthreads();
  // neither CTA may leave, or free its TMEM, while the other can still signal its barriers,
  // read its shared memory or write its accumulators
  tc::cluster_sync_all();
  if (threadIdx.x == 0 && *abort_flag) aero_raise(p.status, AERO_ST_TIMEOUT);
  if (warp == EPI_WARPS + 1) {
    tc::tc_fence_after();
    tc::tmem_dealloc_pair(tmem_base, 512);
  }
}

template <typename T, int BLOCK>
void launch_quantize(const QuantArgs& a, unsigned grid, cudaStream_t stream) {
  // rows of up to 4096 (bf16) or 2048 (fp32) columns stay in registers between the passes
  constexpr int kMost = sizeof(T) == 2 ? 8 : 4;
  const int steps = (a.slabs * kSlab + kStep - 1) / kStep;
  if (BLOCK == 16 && steps <= 3) fp4_quantize_kernel<T, BLOCK, BLOCK == 16 ? 3 : 0><<<grid, 256, 0, stream>>>(a);
  else if (BLOCK == 16 && steps <= kMost) fp4_quantize_kernel<T, BLOCK, BLOCK == 16 ? kMost : 0><<<grid, 256, 0, stream>>>(a);
  else fp4_quantize_kernel<T, BLOCK, 0><<<grid, 256, 0, stream>>>(a);
}

int check_rows(int64_t T, int32_t d, int32_t block) {
  if (T < 0 || d <= 0) return AERO_ERR_INVALID;
  if (block != 16 && block != 32) return AERO_ERR_UNSUPPORTED;
  if (d % 32 != 0 || d > kMaxD || T > (int64_t)1 << 30) return AERO_ERR_UNSUPPORTED;
  return AERO_OK;
}

template <typename O, int BLOCK>
int product(aero_ctx* ctx, Params p) {
  constexpr uint32_t kScales = groups_per_slab(BLOCK) * kGroupBytes;
  if (p.T > kRowsN) {
    p.n_tok = (p.T + kPairT - 1) / kPairT;
    CUtensorMap tmW, tmWs, tmH, tmHs;
    const uint64_t w_rows = (uint64_t)tiles_of(p.V) * p.slabs, h_rows = (uint64_t)tiles_of(p.T) * p.slabs;
    constexpr uint32_t kGroups = groups_per_slab(BLOCK);
    int rc;
    if ((rc = aero_make_tmap_flat(ctx, &tmW, p.w.codes, w_rows * kTile, kRowBytes / 4, kTile))) return rc;
    if ((rc = aero_make_tmap_flat(ctx, &tmWs, p.w.scales, w_rows * kGroups, kGroupBytes / 4, kGroups))) return rc;
    if ((rc = aero_make_tmap_flat(ctx, &tmH, p.h.codes, h_rows * kTile, kRowBytes / 4, kPiece))) return rc;
    if ((rc = aero_make_tmap_flat(ctx, &tmHs, p.h.scales, h_rows * kGroups, kGroupBytes / 4, kGroups))) return rc;
    auto kernel = fp4_pair_kernel<O, BLOCK>;
    AERO_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)p_smem(BLOCK)));
    const long long units = (long long)((p.V + 2 * kTile - 1) / (2 * kTile)) * p.n_tok;
    const long long max_pairs = ctx->sm_count / 2 > 0 ? ctx->sm_count / 2 : 1;
    kernel<<<2 * (int)(units < max_pairs ? units : max_pairs), THREADS, p_smem(BLOCK), ctx->stream>>>(tmW, tmWs, tmH, tmHs, p);
    ctx->launches += 1;
    AERO_CUDA_TRY(cudaGetLastError());
    return AERO_OK;
  }
  p.n = (p.T + 15) / 16 * 16;
  const size_t slab = kTileBytes + (size_t)p.n * kRowBytes + 2 * kScales;
  const int sets = (int)(kRing / slab) < kMaxSets ? (int)(kRing / slab) : kMaxSets;
  p.per = sets >= 6 ? 2 : 1;
  p.stages = sets / p.per;
  auto kernel = fp4_rows_kernel<O, BLOCK>;
  AERO_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)R_SMEM));
  const int blocks = (p.V + kRowBlock - 1) / kRowBlock;
  kernel<<<blocks < ctx->sm_count ? blocks : ctx->sm_count, THREADS, R_SMEM, ctx->stream>>>(p);
  ctx->launches += 1;
  AERO_CUDA_TRY(cudaGetLastError());
  return AERO_OK;
}

}  // namespace

extern "C" {

size_t aero_fp4_code_bytes(int64_t T, int32_t d) {
  return T < 0 || d <= 0 ? 0 : (size_t)tiles_of(T) * slabs_of(d) * kTileBytes;
}
size_t aero_fp4_scale_bytes(int64_t T, int32_t d, int32_t block) {
  return T < 0 || d <= 0 || (block != 16 && block != 32) ? 0 : (size_t)tiles_of(T) * slabs_of(d) * groups_per_slab(block) * kGroupBytes;
}

int aero_quantize_fp4(aero_ctx* ctx, const aero_cfg* cfg, int64_t T, int32_t d, int32_t block, const void* x, uint8_t* codes,
                      uint8_t* scales, float* row_scale) {
  AeroRange nv("aero_quantize_fp4");
  if (!ctx || !cfg) return AERO_ERR_INVALID;
  int rc = check_rows(T, d, block);
  if (rc) return rc;
  if (cfg->dtype != AERO_BF16 && cfg->dtype != AERO_FP32) return AERO_ERR_UNSUPPORTED;
  if (T > 0 && (!x || !codes || !scales || (block == 16) != (row_scale != nullptr))) return AERO_ERR_INVALID;
  if (!aero_aligned16(x) || !aero_aligned16(codes) || !aero_aligned16(scales) || reinterpret_cast<uintptr_t>(row_scale) % 4)
    return AERO_ERR_INVALID;
  if ((rc = aero_check_ctx(ctx))) return rc;
  if (T == 0) return AERO_OK;
  const QuantArgs a = {T, d, slabs_of(d), x, codes, scales, row_scale};
  const unsigned grid = (unsigned)(tiles_of(T) * (kTile / 8));
  if (cfg->dtype == AERO_BF16) {
    if (block == 16) launch_quantize<__nv_bfloat16, 16>(a, grid, ctx->stream);
    else launch_quantize<__nv_bfloat16, 32>(a, grid, ctx->stream);
  } else {
    if (block == 16) launch_quantize<float, 16>(a, grid, ctx->stream);
    else launch_quantize<float, 32>(a, grid, ctx->stream);
  }
  ctx->launches += 1;
  AERO_CUDA_TRY(cudaGetLastError());
  return AERO_OK;
}

int aero_dequantize_fp4(aero_ctx* ctx, int64_t T, int32_t d, int32_t block, const uint8_t* codes, const uint8_t* scales,
                        const float* row_scale, int32_t out_dtype, void* out) {
  AeroRange nv("aero_dequantize_fp4");
  if (!ctx) return AERO_ERR_INVALID;
  int rc = check_rows(T, d, block);
  if (rc) return rc;
  if (out_dtype != AERO_BF16 && out_dtype != AERO_FP32) return AERO_ERR_UNSUPPORTED;
  if (T > 0 && (!out || !codes || !scales || (block == 16) != (row_scale != nullptr))) return AERO_ERR_INVALID;
  if (!aero_aligned16(out) || !aero_aligned16(codes) || !aero_aligned16(scales) || reinterpret_cast<uintptr_t>(row_scale) % 4)
    return AERO_ERR_INVALID;
  if ((rc = aero_check_ctx(ctx))) return rc;
  if (T == 0) return AERO_OK;
  const ValueArgs a = {T, d, slabs_of(d), codes, scales, row_scale, out};
  const unsigned grid = (unsigned)((T + 7) / 8);
  if (out_dtype == AERO_BF16) {
    if (block == 16) fp4_values_kernel<__nv_bfloat16, 16><<<grid, 256, 0, ctx->stream>>>(a);
    else fp4_values_kernel<__nv_bfloat16, 32><<<grid, 256, 0, ctx->stream>>>(a);
  } else {
    if (block == 16) fp4_values_kernel<float, 16><<<grid, 256, 0, ctx->stream>>>(a);
    else fp4_values_kernel<float, 32><<<grid, 256, 0, ctx->stream>>>(a);
  }
  ctx->launches += 1;
  AERO_CUDA_TRY(cudaGetLastError());
  return AERO_OK;
}

int aero_lmhead_fp4(aero_ctx* ctx, int64_t T, int32_t d, int32_t V, int32_t block, const uint8_t* h_codes, const uint8_t* h_scales,
                    const float* h_row, const uint8_t* w_codes, const uint8_t* w_scales, const float* w_row, int32_t out_dtype,
                    void* out) {
  AeroRange nv("aero_lmhead_fp4");
  if (!ctx || V <= 0 || !w_codes || !w_scales) return AERO_ERR_INVALID;
  int rc = check_rows(T, d, block);
  if (rc) return rc;
  if (V > 1 << 30) return AERO_ERR_UNSUPPORTED;
  if (out_dtype != AERO_BF16 && out_dtype != AERO_FP32) return AERO_ERR_UNSUPPORTED;
  if ((block == 16) != (w_row != nullptr)) return AERO_ERR_INVALID;
  if (T > 0 && (!h_codes || !h_scales || !out || (block == 16) != (h_row != nullptr))) return AERO_ERR_INVALID;
  if (!aero_aligned16(h_codes) || !aero_aligned16(h_scales) || !aero_aligned16(w_codes) || !aero_aligned16(w_scales) ||
      reinterpret_cast<uintptr_t>(h_row) % 4 || reinterpret_cast<uintptr_t>(w_row) % 4 ||
      reinterpret_cast<uintptr_t>(out) % (out_dtype == AERO_FP32 ? 4 : 2))
    return AERO_ERR_INVALID;
  // rows of tiles are counted in 32 bits
  if (tiles_of(T > V ? T : V) * slabs_of(d) * kTile > 0x7fffffffll - kPairT) return AERO_ERR_UNSUPPORTED;
  if ((rc = aero_check_ctx(ctx))) return rc;
  if (T == 0) return AERO_OK;
  const Params p = {(int)T, V, slabs_of(d), 0, 1, {h_codes, h_scales, h_row}, {w_codes, w_scales, w_row}, out, ctx->d_status, 0, 0};
  if (out_dtype == AERO_BF16) return block == 16 ? product<__nv_bfloat16, 16>(ctx, p) : product<__nv_bfloat16, 32>(ctx, p);
  return block == 16 ? product<float, 16>(ctx, p) : product<float, 32>(ctx, p);
}

}  // extern "C"
