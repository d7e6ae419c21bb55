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
//
// Bound by memory: dX is read once and every row of dW written once.  A dW that is overwritten is not
// cleared beforehand: the rows of tokens that do not occur are cleared by blocks of their own, which run
// beside the sort, whose few blocks leave the memory idle.
#include "entry.cuh"
#include "vec.cuh"

#include <initializer_list>

namespace {

// One kernel / sort and tiles, with the clearing of dW: d = 1536, V = 151936 2500 tokens 164 / 189 us, 3500 186 / 190, 4090
// 196 / 189; d = 3584, V = 152064 2500 tokens 353 / 360 us, 4090 398 / 362; d = 1536, V = 3000 2500 tokens 38 / 65 us, 4090
// 59 / 66.  (Positions are listed in 16 bits.)
constexpr int kSmallT = 2816;
constexpr int kSortTile = 2048, kSortThreads = 256, kSortWarps = kSortThreads / 32;
constexpr int kMaxRadix = 512;

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

// Blocks from `first` on clear the rows v0 .. v1 - 1 of dW whose token does not occur.
struct Clear {
  float* dW;               // NULL: nothing to clear
  const uint8_t* occurs;   // [V]
  int d, v0, v1;
  unsigned first;
};

__device__ __forceinline__ bool clear_rows(const Clear& z) {
  if (blockIdx.x < z.first) return false;
  const int lane = threadIdx.x & 31;
  const bool vec = z.d % 4 == 0 && (reinterpret_cast<uintptr_t>(z.dW) & 15u) == 0;
  const long long step = (long long)(gridDim.x - z.first) * (blockDim.x >> 5);
  for (long long v = z.v0 + (long long)(blockIdx.x - z.first) * (blockDim.x >> 5) + (threadIdx.x >> 5); v < z.v1; v += step) {
    if (z.occurs[v]) continue;
    float* row = z.dW + v * z.d;
    if (vec) {
      for (int k = lane; k < z.d / 4; k += 32) reinterpret_cast<float4*>(row)[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    } else {
      for (int k = lane; k < z.d; k += 32) row[k] = 0.f;
    }
  }
  return true;
}

// pieces of 32 vectors per slab, and warps of a block, for whole vectors and for single elements
template <int VEC>
__host__ __device__ constexpr int small_nj() { return VEC == 1 ? 4 : 1; }
template <int VEC>
__host__ __device__ constexpr int small_warps() { return VEC == 1 ? 8 : 4; }

// Block (t, y): the first occurrence of a token adds the rows of all its occurrences, slabs of NJ * 32 * VEC columns y,
// y + gridDim.y, ...  Each warp looks through an equal stretch of the ids and adds the rows it finds, in order; the
// warps' sums are added in order.  A block whose token occurs earlier leaves.  A frequent token is one chain of loads: single
// elements (VEC = 1) are taken four columns of a lane at a time, so that as many rows need no more turns and no more
// blocks look through the ids (2500 fp32 rows, d = 2001, V = 5000: 157 -> 102 us with four columns; whole vectors with
// eight rows in flight instead of four: 2500 bf16 rows, d = 1536, V = 151936 168 -> 164 us).  Four warps or eight: whole
// vectors at d = 3584, V = 152064 352 / 384 us, single elements (1953 bf16 rows, d = 726, V = 1511) 46 / 38 us.
template <typename T, int VEC>
__global__ void __launch_bounds__(small_warps<VEC>() * 32) embed_bwd_small_kernel(int T_, int d, int V, const int32_t* __restrict__ y,
                                                              const T* __restrict__ dX, float scale, float* __restrict__ dW,
                                                              int accumulate, uint32_t* status) {
  using Raw = typename rowvec::Raw<T, VEC>::type;
  constexpr int NW = small_warps<VEC>(), NJ = small_nj<VEC>(), S = 32 * VEC;      // a slab: NJ pieces of S columns
  __shared__ uint16_t list[NW][kSmallT / NW];
  __shared__ int found[NW];
  __shared__ float sums[NW - 1][NJ * S];
  const int t = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int id = y[t];
  if (id < 0 || id >= V) {
    if (id != AERO_NO_TOKEN && blockIdx.y == 0 && threadIdx.x == 0) aero_raise(status, AERO_ST_BAD_TARGET);
    return;
  }
  const int p0 = T_ * warp / NW, p1 = T_ * (warp + 1) / NW;
  int n = 0, first = 0x7fffffff;
#pragma unroll 4
  for (int base = p0; base < p1; base += 32) {
    const int p = base + lane;
    const unsigned hits = __ballot_sync(0xffffffffu, p < p1 && y[p] == id);
    if (hits >> lane & 1u) list[warp][n + __popc(hits & ((1u << lane) - 1u))] = (uint16_t)p;
    if (hits && n == 0) first = base + __ffs(hits) - 1;
    n += __popc(hits);
  }
  if (lane == 0) found[warp] = n;
  if (__syncthreads_or(first < t)) return;             // an earlier block has this token
  int all = 0;
  bool alone = false;
  for (int w = 0; w < NW; ++w) all += found[w];
  for (int w = 0; w < NW; ++w) alone |= found[w] == all;          // (the same answer in all warps)
  for (int s0 = blockIdx.y * NJ * S; s0 < d; s0 += gridDim.y * NJ * S) {
    const int c = s0 + lane * VEC;                       // and c + S, ... c + (NJ - 1) S
    float acc[NJ][VEC];
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < VEC; ++e) acc[j][e] = 0.f;
    constexpr int U = VEC == 1 ? 4 : 8;                  // rows in flight
    for (int k = 0; k < n; k += U) {
      Raw raw[U][NJ];
#pragma unroll
      for (int q = 0; q < U; ++q)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          if (k + q < n && c + j * S < d) raw[q][j] = *reinterpret_cast<const Raw*>(dX + (long long)list[warp][k + q] * d + c + j * S);
#pragma unroll
      for (int q = 0; q < U; ++q)
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          if (k + q < n && c + j * S < d) {
            float f[VEC];
            rowvec::open<T, VEC>(raw[q][j], f);
#pragma unroll
            for (int e = 0; e < VEC; ++e) acc[j][e] += f[e];
          }
        }
    }
    float* dst = dW + (long long)id * d + c;
    if (alone) {                                         // all occurrences in one warp's stretch (often only one): no join
#pragma unroll
      for (int j = 0; j < NJ; ++j)
        if (n > 0 && c + j * S < d) put<VEC>(dst + j * S, acc[j], scale, accumulate != 0);
      continue;
    }
    if (warp < NW - 1) {
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < VEC; ++e) sums[warp][(j * VEC + e) * 32 + lane] = acc[j][e];
    }
    __syncthreads();
    if (warp == NW - 1) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        if (c + j * S >= d) continue;
        float s[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const int i = (j * VEC + e) * 32 + lane;
          s[e] = sums[0][i];
#pragma unroll
          for (int w = 1; w < NW - 1; ++w) s[e] += sums[w][i];
          s[e] += acc[j][e];
        }
        put<VEC>(dst + j * S, s, scale, accumulate != 0);
      }
    }
    __syncthreads();
  }
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
                                                                  int blocks, uint32_t* __restrict__ counts,
                                                                  uint8_t* __restrict__ occurs, Clear z, uint32_t* status) {
  __shared__ uint32_t h[kMaxRadix];
  if (clear_rows(z)) return;
  for (int i = threadIdx.x; i < radix; i += kSortThreads) h[i] = 0;
  __syncthreads();
  const int base = blockIdx.x * kSortTile;
  bool bad = false;
#pragma unroll
  for (int k = threadIdx.x; k < kSortTile; k += kSortThreads) {
    if (base + k >= n) continue;
    const uint32_t key = key_of(y, keys, base + k, V);
    if (!keys && key == (uint32_t)V) bad |= y[base + k] != AERO_NO_TOKEN;
    if (occurs && key != (uint32_t)V) occurs[key] = 1;
    atomicAdd(&h[(key >> shift) & (radix - 1)], 1u);
  }
  if (bad) aero_raise(status, AERO_ST_BAD_TARGET);
  __syncthreads();
  for (int i = threadIdx.x; i < radix; i += kSortThreads) counts[(size_t)i * blocks + blockIdx.x] = h[i];
}

// exclusive sum over the block's threads, and the sum of all; `sh` may be used again after a barrier
__device__ __forceinline__ uint32_t block_before(uint32_t v, uint32_t* sh, uint32_t& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t u = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += u;
  }
  if (lane == 31) sh[warp] = incl;
  __syncthreads();
  uint32_t before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kSortWarps; ++w) {
    if (w < warp) before += sh[w];
    total += sh[w];
  }
  return before + incl - v;
}

// Exclusive prefix of each digit's counts over the blocks, in place, and the digit's total: a block per digit.  (The
// prefix over the totals is left to the blocks of the scatter; 3 us for 204780 keys.)
__global__ void __launch_bounds__(kSortThreads) sort_prefix_kernel(uint32_t* __restrict__ counts, int blocks,
                                                                   uint32_t* __restrict__ totals, Clear z) {
  __shared__ uint32_t sh[2][kSortWarps];
  if (clear_rows(z)) return;
  uint32_t* row = counts + (size_t)blockIdx.x * blocks;
  uint32_t carry = 0;
  for (int base = 0, turn = 0; base < blocks; base += kSortThreads, turn ^= 1) {
    const int i = base + threadIdx.x;
    const uint32_t v = i < blocks ? row[i] : 0u;
    uint32_t total;
    const uint32_t before = block_before(v, sh[turn], total);
    if (i < blocks) row[i] = carry + before;
    carry += total;
  }
  if (threadIdx.x == 0) totals[blockIdx.x] = carry;
}

__global__ void __launch_bounds__(kSortThreads) sort_scatter_kernel(int n, int V, const int32_t* __restrict__ y,
                                                                    const uint32_t* __restrict__ keys,
                                                                    const uint32_t* __restrict__ pos, int shift, int radix,
                                                                    int blocks, const uint32_t* __restrict__ starts,
                                                                    const uint32_t* __restrict__ totals,
                                                                    uint32_t* __restrict__ keys_out,
                                                                    uint32_t* __restrict__ pos_out, Clear z) {
  __shared__ uint32_t h[kSortWarps][kMaxRadix], first[kMaxRadix], sh[kSortWarps];
  if (clear_rows(z)) return;
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
  // where each digit's keys start: thread i has digits 2 i and 2 i + 1
  static_assert(kMaxRadix == 2 * kSortThreads, "two digits per thread");
  const int d0 = 2 * threadIdx.x;
  const uint32_t n0 = d0 < radix ? totals[d0] : 0u, n1 = d0 + 1 < radix ? totals[d0 + 1] : 0u;
  uint32_t all;
  first[d0] = block_before(n0 + n1, sh, all);
  first[d0 + 1] = first[d0] + n0;
  __syncthreads();
  for (int g = threadIdx.x; g < radix; g += kSortThreads) {
    uint32_t run = first[g] + starts[(size_t)g * blocks + blockIdx.x];
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
// Warp (tile, slab): tile = kTile sorted positions, slab = 32 * VEC columns.  A run of equal keys that lies inside the
// tile goes to dW; one that continues from the tile before goes to part[tile][0], one that starts here and continues
// in the tile after to part[tile][1].  Rows are held packed and two are in flight beyond the two being added: more per
// warp costs registers, and it is warps that keep the memory busy (204780 x 1536: 379 us with eight unpacked rows a
// turn, 202 with four packed ones, 173 with two; 277 with tiles of 128 positions).
constexpr int kTile = 32, kInFlight = 2, kShortRun = 8;

// Runs that reach over the end of the tile they start in, for the joining kernel: first and last tile; those of few
// tiles from the front, longer ones from the back.
struct Runs {
  int2* list;              // [tiles]
  int* count;              // [2]: short, long
  int tiles;
};

// The warp that adds up the first slab of such a run's first tile b puts it on the list: tiles b + 1 .. last start with
// its key, those after do not; a search 32 tiles wide, first over the nearest ones.
__device__ __forceinline__ void list_run(const Runs& runs, const uint32_t* __restrict__ keys, uint32_t key, int b, int lane) {
  int lo = b + 1, hi = runs.tiles, step = 1;
  while (hi - lo > 1) {
    const int k = lo + (lane + 1) * step;
    const int ahead = __popc(__ballot_sync(0xffffffffu, k < hi && keys[(long long)k * kTile] == key));
    if (ahead < 32) hi = min(hi, lo + (ahead + 1) * step);
    lo += ahead * step;
    step = ahead == 32 ? max(1, (hi - lo + 31) / 32) : (hi - lo + 31) / 32;
  }
  if (lane == 0) {
    if (lo - b <= kShortRun) runs.list[atomicAdd(&runs.count[0], 1)] = make_int2(b, lo);
    else runs.list[runs.tiles - 1 - atomicAdd(&runs.count[1], 1)] = make_int2(b, lo);
  }
}

template <typename T, int VEC>
__global__ void __launch_bounds__(256) embed_bwd_sum_kernel(int n, int d, int V, const uint32_t* __restrict__ keys,
                                                            const uint32_t* __restrict__ pos, const T* __restrict__ dX,
                                                            float scale, float* __restrict__ dW, int accumulate,
                                                            float* __restrict__ part, Runs runs) {
  using Raw = typename rowvec::Raw<T, VEC>::type;
  constexpr int U = kInFlight;
  const int lane = threadIdx.x & 31;
  const int slabs = (d + 32 * VEC - 1) / (32 * VEC);
  const long long u = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const long long tile = u / slabs;
  if (tile * kTile >= n) return;
  const int p0 = (int)(tile * kTile), count = min(kTile, n - p0);
  const int c = ((int)(u - tile * slabs) * 32 + lane) * VEC;
  const uint32_t none = (uint32_t)V;
  const uint32_t my_key = lane < count ? keys[p0 + lane] : none;
  const uint32_t my_pos = lane < count ? pos[p0 + lane] : 0u;
  const uint32_t before = p0 > 0 ? keys[p0 - 1] : none;
  const uint32_t after = p0 + count < n ? keys[p0 + count] : none;
  // positions without a token are sorted last: the first `live` positions have one
  const int live = __popc(__ballot_sync(0xffffffffu, my_key != none));
  float acc[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
  int run0 = 0;                                          // first position of the current run
  Raw next[U];
  auto fetch = [&](int k) {
#pragma unroll
    for (int q = 0; q < U; ++q) {
      const uint32_t row = __shfl_sync(0xffffffffu, my_pos, (k + q) & 31);
      if (k + q < live && c < d) next[q] = *reinterpret_cast<const Raw*>(dX + (long long)row * d + c);
    }
  };
  fetch(0);
  for (int k = 0; k < live; k += U) {
    Raw cur[U];
#pragma unroll
    for (int q = 0; q < U; ++q) cur[q] = next[q];
    fetch(k + U);
#pragma unroll
    for (int q = 0; q < U; ++q) {
      if (k + q < live) {
        const uint32_t key = __shfl_sync(0xffffffffu, my_key, k + q);
        float f[VEC];
        rowvec::open<T, VEC>(cur[q], f);
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] += f[e];
        const bool last = k + q + 1 >= count;
        const uint32_t following = last ? after : __shfl_sync(0xffffffffu, my_key, (k + q + 1) & 31);
        if (following != key || last) {
          const bool head = run0 == 0 && before == key, tail = last && following == key;
          if (c < d) {
            if (head || tail) put<VEC>(part + ((size_t)tile * 2 + (head ? 0 : 1)) * d + c, acc, 1.f, false);
            else put<VEC>(dW + (long long)key * d + c, acc, scale, accumulate != 0);
          }
          if (tail && !head && c < 32 * VEC) list_run(runs, keys, key, (int)tile, lane);
#pragma unroll
          for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
          run0 = k + q + 1;
        }
      }
    }
  }
}

// Adds up the partial sums of the listed runs, 128 columns at a time: a run of a few tiles by one warp, a longer one by
// the eight warps of a block, a contiguous eighth of its tiles each, in order.  (The order of the list does not matter:
// every run has its own row of dW.)  The list is what makes this short: blocks that each looked through 32 tiles for
// runs took 57 us at 204780 x 1536, most of it waiting for the few that had found some; from the list it is 28 us.
__global__ void __launch_bounds__(256) embed_bwd_join_kernel(int d, const uint32_t* __restrict__ keys,
                                                             const float* __restrict__ part, float scale,
                                                             float* __restrict__ dW, int accumulate, Runs runs) {
  __shared__ float sh[8][128];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, slabs = (d + 127) / 128;
  int c0 = 0, col[4];                                            // (columns past d read the last one and are dropped)
  auto at_slab = [&](int slab) {
    c0 = slab * 128;
#pragma unroll
    for (int q = 0; q < 4; ++q) col[q] = min(c0 + q * 32 + lane, d - 1);
  };
  auto add = [&](int k0, int k1, float (&acc)[4]) {              // slot 0 of tiles k0 .. k1 - 1, 32 loads in flight
    for (int k = k0; k < k1; k += 8) {
      float v[8][4];
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) v[i][q] = part[(size_t)min(k + i, k1 - 1) * 2 * d + col[q]];
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[q] += k + i < k1 ? v[i][q] : 0.f;
    }
  };
  auto finish = [&](int b, int c, float sum) {                   // + the run's share of its first tile (slot 1)
    sum += part[((size_t)b * 2 + 1) * d + c];
    float* dst = dW + (long long)keys[((long long)b + 1) * kTile - 1] * d + c;
    *dst = accumulate ? fmaf(sum, scale, *dst) : sum * scale;
  };
  const long long n_short = (long long)runs.count[0] * slabs, n_long = (long long)runs.count[1] * slabs;
  for (long long i = blockIdx.x; i < n_long; i += gridDim.x) {   // (long ones first: they take longest)
    const int2 run = runs.list[runs.tiles - 1 - i / slabs];
    at_slab((int)(i % slabs));
    const int count = run.y - run.x;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    add(run.x + 1 + (int)((long long)count * warp / 8), run.x + 1 + (int)((long long)count * (warp + 1) / 8), acc);
    __syncthreads();                                             // the previous run's sums have been read
#pragma unroll
    for (int q = 0; q < 4; ++q) sh[warp][q * 32 + lane] = acc[q];
    __syncthreads();
    if (threadIdx.x < 128 && c0 + (int)threadIdx.x < d) {
      float sum = 0.f;
      for (int w = 0; w < 8; ++w) sum += sh[w][threadIdx.x];
      finish(run.x, c0 + threadIdx.x, sum);
    }
  }
  for (long long i = (long long)blockIdx.x * 8 + warp; i < n_short; i += (long long)gridDim.x * 8) {
    const int2 run = runs.list[i / slabs];
    at_slab((int)(i % slabs));
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    add(run.x + 1, run.y + 1, acc);
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (c0 + q * 32 + lane < d) finish(run.x, c0 + q * 32 + lane, acc[q]);
  }
}

struct Ws {
  uint8_t* occurs;
  uint32_t* keys[2];
  uint32_t* pos[2];
  uint32_t* counts;
  uint32_t* totals;
  float* part;
  Runs runs;
  size_t bytes;
};

Ws carve(void* base, int64_t T, int32_t d, int32_t V) {
  Ws w = {};
  char* p = static_cast<char*>(base);
  size_t off = 0;
  auto take = [&](size_t bytes) { char* r = p + off; off += aero_align_up(bytes, 256); return r; };
  if (T > kSmallT) {
    w.occurs = reinterpret_cast<uint8_t*>(take((size_t)V));
    for (int i = 0; i < 2; ++i) {
      w.keys[i] = reinterpret_cast<uint32_t*>(take((size_t)T * sizeof(uint32_t)));
      w.pos[i] = reinterpret_cast<uint32_t*>(take((size_t)T * sizeof(uint32_t)));
    }
    const size_t blocks = ((size_t)T + kSortTile - 1) / kSortTile, tiles = ((size_t)T + kTile - 1) / kTile;
    w.counts = reinterpret_cast<uint32_t*>(take(blocks * kMaxRadix * sizeof(uint32_t)));
    w.totals = reinterpret_cast<uint32_t*>(take(kMaxRadix * sizeof(uint32_t)));
    w.part = reinterpret_cast<float*>(take(tiles * 2 * (size_t)d * sizeof(float)));
    w.runs.list = reinterpret_cast<int2*>(take(tiles * sizeof(int2)));
    w.runs.count = reinterpret_cast<int*>(take(2 * sizeof(int)));
    w.runs.tiles = (int)tiles;
  }
  w.bytes = off > 0 ? off : 256;
  return w;
}

// The sort's launches clear an equal share of the rows of dW each (all but the first, which finds the tokens): a warp per
// row and 32 blocks per SM, so that the stores of all rows are under way at once (204780 x 1536 / 30000 x 3584: 16 blocks
// 357 / 414 us, 32 354 / 405, 128 371 / 412; four blocks whose warps took eight rows each 375 / 469).
int sort_positions(aero_ctx* ctx, const Ws& w, int n, int d, int V, const int32_t* y, float* clear, const uint32_t** keys,
                   const uint32_t** pos) {
  int bits = 1;
  while (bits < 32 && ((uint32_t)V >> bits) != 0) ++bits;          // the keys are 0 .. V
  const int passes = (bits + 8) / 9;
  const int per = (bits + passes - 1) / passes;
  const unsigned blocks = (unsigned)(((long long)n + kSortTile - 1) / kSortTile);
  const unsigned helpers = clear ? 32u * (unsigned)ctx->sm_count : 0u;
  const int shares = 3 * passes - 1;
  int share = 0;
  auto next_share = [&](unsigned first) {
    Clear z = {clear, w.occurs, d, (int)((long long)V * share / shares), (int)((long long)V * (share + 1) / shares), first};
    ++share;
    return z;
  };
  const Clear none = {nullptr, nullptr, 0, 0, 0, 0xffffffffu};
  if (clear) AERO_CUDA_TRY(cudaMemsetAsync(w.occurs, 0, (size_t)V, ctx->stream));
  const uint32_t *kin = nullptr, *pin = nullptr;
  for (int p = 0; p < passes; ++p) {
    const int radix = 1 << per, shift = p * per;
    const bool find = p == 0;
    sort_count_kernel<<<blocks + (find ? 0u : helpers), kSortThreads, 0, ctx->stream>>>(
        n, V, y, kin, shift, radix, (int)blocks, w.counts, find && clear ? w.occurs : nullptr,
        find || !clear ? none : next_share(blocks), ctx->d_status);
    sort_prefix_kernel<<<radix + helpers, kSortThreads, 0, ctx->stream>>>(w.counts, (int)blocks, w.totals,
                                                                          clear ? next_share(radix) : none);
    sort_scatter_kernel<<<blocks + helpers, kSortThreads, 0, ctx->stream>>>(n, V, y, kin, pin, shift, radix, (int)blocks,
                                                                            w.counts, w.totals, w.keys[p & 1], w.pos[p & 1],
                                                                            clear ? next_share(blocks) : none);
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
  const Ws w = carve(ws, T_, d, V);
  const int n = (int)T_;
  if (T_ <= kSmallT) {
    // (the rows of few tokens are written twice at most: clearing all of dW beforehand costs no more)
    if (!accumulate) AERO_CUDA_TRY(cudaMemsetAsync(dW, 0, (size_t)V * d * sizeof(float), ctx->stream));
    const int slabs = (d + small_nj<VEC>() * 32 * VEC - 1) / (small_nj<VEC>() * 32 * VEC);
    embed_bwd_small_kernel<T, VEC><<<dim3((unsigned)T_, (unsigned)((slabs + 2) / 3)), small_warps<VEC>() * 32, 0, ctx->stream>>>(
        n, d, V, y, dX, scale, dW, accumulate, ctx->d_status);
    ctx->launches += 1;
    AERO_CUDA_TRY(cudaGetLastError());
    return AERO_OK;
  }
  const uint32_t *keys, *pos;
  const int rc = sort_positions(ctx, w, n, d, V, y, accumulate ? nullptr : dW, &keys, &pos);
  if (rc) return rc;
  const long long tiles = ((long long)n + kTile - 1) / kTile, slabs = (d + 32 * VEC - 1) / (32 * VEC);
  AERO_CUDA_TRY(cudaMemsetAsync(w.runs.count, 0, 2 * sizeof(int), ctx->stream));
  embed_bwd_sum_kernel<T, VEC><<<(unsigned)((tiles * slabs + 7) / 8), 256, 0, ctx->stream>>>(
      n, d, V, keys, pos, dX, scale, dW, accumulate, w.part, w.runs);
  embed_bwd_join_kernel<<<8 * ctx->sm_count, 256, 0, ctx->stream>>>(d, keys, w.part, scale, dW, accumulate, w.runs);
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

size_t aero_embed_workspace_bytes(int64_t T, int32_t d, int32_t V) {
  return T < 0 || d <= 0 || V <= 0 ? 0 : carve(nullptr, T, d, V).bytes;
}

int aero_embed_bwd(aero_ctx* ctx, const aero_cfg* cfg, int64_t T, int32_t d, int32_t V, const int32_t* y, const void* dX,
                   float scale, float* dW, int accumulate_dW, void* workspace, size_t workspace_bytes) {
  AeroRange nv("aero_embed_bwd");
  int rc = check_shape(cfg, T, d, V);
  if (rc) return rc;
  if (!ctx || !dW || (T > 0 && (!y || !dX)) || !workspace || !aero_aligned256(workspace)) return AERO_ERR_INVALID;
  if (reinterpret_cast<uintptr_t>(dX) % (cfg->dtype == AERO_FP32 ? 4 : 2)) return AERO_ERR_INVALID;
  if (workspace_bytes < aero_embed_workspace_bytes(T, d, V)) return AERO_ERR_WORKSPACE;
  if ((rc = aero_check_ctx(ctx))) return rc;
  if (T == 0) {
    if (!accumulate_dW) AERO_CUDA_TRY(cudaMemsetAsync(dW, 0, (size_t)V * d * sizeof(float), ctx->stream));
    return AERO_OK;
  }
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
