// The lm_head product in 8-bit integers, with a scale for each token and each vocabulary row:
//   z_tv = h_scale_t w_scale_v sum_k h_tk w_vk        (the sum exact in 32-bit integers)
// on tcgen05 kind::i8 with TMEM accumulators and TMA-fed operands.  W is operand A (the 128 or 256
// rows of a tile are vocabulary rows) and the tokens are operand B, so that N follows the number of
// tokens: a single token costs no more tensor time than N = 16, and an accumulator column is one
// token's logits of 128 neighbouring vocabulary rows, which the warps store as whole segments.
//
//   q8_rows_kernel   up to 128 tokens: bound by reading W once.  Each CTA streams a contiguous range
//                    of vocabulary rows, cut in blocks of 32 so that all CTAs get the same bytes.
//   q8_pair_kernel   more tokens: CTA pairs (cta_group::2), 256 vocabulary rows x up to 256 tokens per
//                    unit, both operands shared between the pair as in the lm_head kernel of stage (b).
// Warp roles in both: warps 0-7 epilogue (one vocabulary row per thread, two warps per quadrant of TMEM), warp 8 TMA,
// warp 9 MMA.
#include "entry.cuh"
#include "tc_ptx.cuh"
#include "tmap.cuh"
#include "vec.cuh"

namespace {

constexpr int BM = 128, BK = 128;                 // vocabulary rows per CTA, bytes of K per stage
constexpr int EPI_WARPS = 8, kShare = EPI_WARPS / 4, THREADS = (EPI_WARPS + 2) * 32;
constexpr int kRowsN = 128, kPairN = 256;         // most tokens per tile
constexpr int kRowBlock = 32;                     // q8_rows_kernel: rows per copy of W
constexpr uint32_t A_BYTES = BM * BK;
constexpr int kMaxD = 65536;                      // 128 * 128 * d stays below 2^31

template <int STAGES>
struct Ctl {
  uint64_t full[STAGES], empty[STAGES], tfull[2], tempty[2];
  uint32_t tmem_base;
  int abort;
};
constexpr int kMaxStages = 4, kPairSlabs = 2, PSTAGES = 3;
constexpr uint32_t P_STAGE = kPairSlabs * (A_BYTES + kPairN / 2 * BK);
constexpr size_t kRing = 204 * 1024;              // q8_rows_kernel: as many stages as fit
constexpr size_t R_SMEM = 1024 + kRing + sizeof(Ctl<kMaxStages>);
constexpr size_t P_SMEM = 1024 + (size_t)PSTAGES * P_STAGE + sizeof(Ctl<PSTAGES>);

struct Params {
  int T, d, V;
  int n;                      // tokens per tile (N of the products)
  int n_tok;                  // token tiles
  const float* h_scale;
  const float* w_scale;
  void* out;
  uint32_t* status;
  int stages, slabs;          // q8_rows_kernel: depth of the ring, slabs of 128 bytes of K per stage
};

// Writes the accumulator columns of tokens t0 .. t0 + n of vocabulary row v from TMEM to out: a thread has one row,
// so the 32 lanes of a warp store 32 neighbouring logits of a token at a time; the two warps of a quadrant of TMEM
// take chunks of 32 tokens in turn.  The tokens' scales come from a lane each, loaded before the accumulator is waited
// for.  (Loads between the stores would wait for one another, since the compiler may not move them over the
// stores: a 256 x 256 tile took 31 k cycles that way, 19 k with one warp per quadrant, against the 14 k of its products.)
template <typename O, int N>
struct Epilogue {
  static constexpr int kChunks = (N / 32 + kShare - 1) / kShare;      // chunks of this warp, at most
  float sh[kChunks];
  __device__ void load_scales(const Params& p, int t0, int half, int lane) {
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      const int t = (kShare * i + half) * 32 + lane;
      sh[i] = t < p.n && t0 + t < p.T ? p.h_scale[t0 + t] : 0.f;
    }
  }
  __device__ void store(const Params& p, uint32_t taddr, int t0, int half, int v, bool row_ok) const {
    const float sw = row_ok ? p.w_scale[v] : 0.f;
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
        const float z = (float)(int)r[q] * __shfl_sync(0xffffffffu, sh[i], q) * sw;
        if (row_ok && q < left) rowvec::Elem<O>::store(o, z);
        o += p.V;
      }
    }
  }
};

template <typename O>
__global__ void __launch_bounds__(THREADS, 1)
q8_rows_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmW4,
               const __grid_constant__ CUtensorMap tmH, const Params p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  // a stage is `slabs` slabs of 128 bytes of K: of the 128 rows of W, then of the n tokens
  const int slabs = p.slabs;
  const uint32_t b_slab = (uint32_t)p.n * BK, stage_bytes = slabs * (A_BYTES + b_slab);
  const int stages = p.stages;
  auto* ctl = reinterpret_cast<Ctl<kMaxStages>*>(smem + (size_t)stages * stage_bytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) { tc::mbar_init(&ctl->full[s], 1); tc::mbar_init(&ctl->empty[s], 1); }
    for (int b = 0; b < 2; ++b) { tc::mbar_init(&ctl->tfull[b], 1); tc::mbar_init(&ctl->tempty[b], EPI_WARPS); }
    ctl->abort = 0;
    tc::fence_barrier_init();
  }
  if (warp == EPI_WARPS && lane == 0) { tc::prefetch_tmap(&tmW); tc::prefetch_tmap(&tmH); }
  if (warp == EPI_WARPS + 1) { tc::tmem_alloc(&ctl->tmem_base, 2 * kRowsN); tc::tmem_relinquish(); }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem_base = ctl->tmem_base;
  volatile int* abort_flag = &ctl->abort;
  // this CTA's vocabulary rows, in blocks of 32
  const int blocks = (p.V + kRowBlock - 1) / kRowBlock;
  const int b0 = (int)((long long)blocks * blockIdx.x / gridDim.x), b1 = (int)((long long)blocks * (blockIdx.x + 1) / gridDim.x);
  const int nkb = (p.d + BK - 1) / BK;

  if (warp == EPI_WARPS) {
    if (lane == 0) {
      int s = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int b = b0; ok && b < b1; b += BM / kRowBlock) {
        const int nb = min(BM / kRowBlock, b1 - b);
        for (int kb = 0; kb < nkb; kb += slabs) {
          if (!tc::mbar_wait(&ctl->empty[s], ph ^ 1u, abort_flag)) { ok = false; break; }
          uint8_t* a_s = smem + (size_t)s * stage_bytes;
          const int nk = min(slabs, nkb - kb);
          tc::mbar_arrive_expect_tx(&ctl->full[s], (uint32_t)(nk * (nb * kRowBlock + p.n)) * BK);
          // whole tiles in copies of 128 rows, the last rows of the range in blocks of 32
          if (nb == BM / kRowBlock) {
            for (int k = 0; k < nk; ++k) tc::tma_load_2d(a_s + k * A_BYTES, &tmW4, (kb + k) * BK, b * kRowBlock, &ctl->full[s]);
          } else {
            for (int i = 0; i < nb; ++i)
              for (int k = 0; k < nk; ++k)
                tc::tma_load_2d(a_s + k * A_BYTES + i * kRowBlock * BK, &tmW, (kb + k) * BK, (b + i) * kRowBlock, &ctl->full[s]);
          }
          for (int k = 0; k < nk; ++k)
            tc::tma_load_2d(a_s + slabs * A_BYTES + k * b_slab, &tmH, (kb + k) * BK, 0, &ctl->full[s]);
          if (++s == stages) { s = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp == EPI_WARPS + 1) {
    if (lane == 0) {
      const uint32_t idesc = tc::make_idesc_s8(BM, p.n);
      int s = 0;
      uint32_t ph = 0, at = 0;
      bool ok = true;
      for (int b = b0; ok && b < b1; b += BM / kRowBlock, ++at) {
        const uint32_t buf = at & 1u;
        if (!tc::mbar_wait(&ctl->tempty[buf], ((at >> 1) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
        tc::tc_fence_after();
        for (int kb = 0; kb < nkb; kb += slabs) {
          if (!tc::mbar_wait(&ctl->full[s], ph, abort_flag)) { ok = false; break; }
          tc::tc_fence_after();
          // (a tile of fewer than 128 rows leaves older bytes in the other rows of A: their accumulator
          // rows are not read)
          const uint32_t a_addr = tc::smem_u32(smem + (size_t)s * stage_bytes);
          const int nk = min(slabs, nkb - kb);
          for (int k = 0; k < nk; ++k) {
            const uint64_t adesc = tc::make_smem_desc(a_addr + k * A_BYTES, 16, 1024);
            const uint64_t bdesc = tc::make_smem_desc(a_addr + slabs * A_BYTES + k * b_slab, 16, 1024);
#pragma unroll
            for (int kk = 0; kk < BK / 32; ++kk)
              tc::umma_s8(tmem_base + buf * kRowsN, adesc + 2u * kk, bdesc + 2u * kk, idesc, (kb | k | kk) != 0 ? 1u : 0u);
          }
          tc::umma_commit(&ctl->empty[s]);
          if (++s == stages) { s = 0; ph ^= 1u; }
        }
        if (ok) tc::umma_commit(&ctl->tfull[buf]);
      }
    }
  } else {
    uint32_t at = 0;
    const int quad = warp & 3, half = warp >> 2;
    Epilogue<O, kRowsN> epi;
    epi.load_scales(p, 0, half, lane);
    for (int b = b0; b < b1; b += BM / kRowBlock, ++at) {
      const uint32_t buf = at & 1u;
      if (!__all_sync(0xffffffffu, tc::mbar_wait(&ctl->tfull[buf], (at >> 1) & 1u, abort_flag))) break;
      tc::tc_fence_after();
      const int v = b * kRowBlock + quad * 32 + lane;
      if (b + quad < b1)                           // this warp's block of 32 rows exists
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
    tc::tmem_dealloc(tmem_base, 2 * kRowsN);
  }
}

template <typename O>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1)
q8_pair_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmH, const Params p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  auto* ctl = reinterpret_cast<Ctl<PSTAGES>*>(smem + (size_t)PSTAGES * P_STAGE);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = tc::cluster_ctarank();        // 0 issues the MMAs of the pair
  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
  if (threadIdx.x == 0) {
    for (int s = 0; s < PSTAGES; ++s) { tc::mbar_init(&ctl->full[s], 1); tc::mbar_init(&ctl->empty[s], 1); }
    for (int b = 0; b < 2; ++b) { tc::mbar_init(&ctl->tfull[b], 1); tc::mbar_init(&ctl->tempty[b], 2 * EPI_WARPS); }
    ctl->abort = 0;
    tc::fence_barrier_init();
  }
  if (warp == EPI_WARPS && lane == 0) { tc::prefetch_tmap(&tmW); tc::prefetch_tmap(&tmH); }
  if (warp == EPI_WARPS + 1) { tc::tmem_alloc_pair(&ctl->tmem_base, 2 * kPairN); tc::tmem_relinquish_pair(); }
  tc::tc_fence_before();
  __syncthreads();
  tc::cluster_sync_all();        // the peer's barriers exist before anything signals them
  tc::tc_fence_after();
  const uint32_t tmem_base = ctl->tmem_base;
  volatile int* abort_flag = &ctl->abort;
  // a unit is 256 vocabulary rows x one token tile; the units of one row tile are neighbours, so that
  // pairs running at the same time read the same W rows from L2
  const long long units = (long long)((p.V + 2 * BM - 1) / (2 * BM)) * p.n_tok;
  const int nkb = (p.d + BK - 1) / BK;
  const uint32_t b_slab = (uint32_t)(p.n / 2) * BK;

  if (warp == EPI_WARPS) {
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      for (long long u = pair; ok && u < units; u += npairs) {
        const int vt = (int)(u / p.n_tok), tt = (int)(u % p.n_tok);
        for (int kb = 0; kb < nkb; kb += kPairSlabs, ++it) {
          const int s = it % PSTAGES;
          if (!tc::mbar_wait(&ctl->empty[s], ((it / PSTAGES) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
          uint8_t* a_s = smem + (size_t)s * P_STAGE;
          const uint32_t full0 = tc::mapa_shared(tc::smem_u32(&ctl->full[s]), 0);
          const int nk = min(kPairSlabs, nkb - kb);
          if (rank == 0) tc::mbar_arrive_expect_tx(&ctl->full[s], (uint32_t)nk * (2 * A_BYTES + (uint32_t)p.n * BK));
          for (int k = 0; k < nk; ++k)
            tc::tma_load_2d_pair(a_s + k * A_BYTES, &tmW, (kb + k) * BK, vt * 2 * BM + (int)rank * BM, full0);
          for (int k = 0; k < nk; ++k)
            tc::tma_load_2d_pair(a_s + kPairSlabs * A_BYTES + k * b_slab, &tmH, (kb + k) * BK, tt * p.n + (int)rank * (p.n / 2),
                                 full0);
        }
      }
    }
  } else if (warp == EPI_WARPS + 1) {
    if (lane == 0 && rank == 0) {
      const uint32_t idesc = tc::make_idesc_s8(2 * BM, p.n);
      uint32_t it = 0, at = 0;
      bool ok = true;
      for (long long u = pair; ok && u < units; u += npairs, ++at) {
        const uint32_t buf = at & 1u;
        if (!tc::mbar_wait(&ctl->tempty[buf], ((at >> 1) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
        tc::tc_fence_after();
        for (int kb = 0; kb < nkb; kb += kPairSlabs, ++it) {
          const int s = it % PSTAGES;
          if (!tc::mbar_wait(&ctl->full[s], (it / PSTAGES) & 1u, abort_flag)) { ok = false; break; }
          tc::tc_fence_after();
          const uint32_t a_addr = tc::smem_u32(smem + (size_t)s * P_STAGE);
          const int nk = min(kPairSlabs, nkb - kb);
          for (int k = 0; k < nk; ++k) {
            const uint64_t adesc = tc::make_smem_desc(a_addr + k * A_BYTES, 16, 1024);
            const uint64_t bdesc = tc::make_smem_desc(a_addr + kPairSlabs * A_BYTES + k * b_slab, 16, 1024);
#pragma unroll
            for (int kk = 0; kk < BK / 32; ++kk)
              tc::umma_s8_pair(tmem_base + buf * kPairN, adesc + 2u * kk, bdesc + 2u * kk, idesc, (kb | k | kk) != 0 ? 1u : 0u);
          }
          tc::umma_commit_pair(&ctl->empty[s], 3);     // frees the stage in both CTAs when these MMAs retire
        }
        if (ok) tc::umma_commit_pair(&ctl->tfull[buf], 3);
      }
    }
  } else {
    uint32_t at = 0;
    const int quad = warp & 3, half = warp >> 2;
    Epilogue<O, kPairN> epi;
    for (long long u = pair; u < units; u += npairs, ++at) {
      const int vt = (int)(u / p.n_tok), tt = (int)(u % p.n_tok);
      const uint32_t buf = at & 1u;
      epi.load_scales(p, tt * p.n, half, lane);
      if (!__all_sync(0xffffffffu, tc::mbar_wait(&ctl->tfull[buf], (at >> 1) & 1u, abort_flag))) break;
      tc::tc_fence_after();
      const int v = vt * 2 * BM + (int)rank * BM + quad * 32 + lane;
      epi.store(p, tmem_base + ((uint32_t)(quad * 32) << 16) + buf * kPairN, tt * p.n, half, v, v < p.V);
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive_cluster(tc::mapa_shared(tc::smem_u32(&ctl->tempty[buf]), 0));
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
    tc::tmem_dealloc_pair(tmem_base, 2 * kPairN);
  }
}

}  // namespace

extern "C" int aero_lmhead_q8(aero_ctx* ctx, int64_t T, int32_t d, int32_t V, const int8_t* h8, const float* h_scale,
                              const int8_t* w8, const float* w_scale, int32_t out_dtype, void* out) {
  AeroRange nv("aero_lmhead_q8");
  if (!ctx || T < 0 || T > (int64_t)1 << 30 || d <= 0 || V <= 0 || !w8 || !w_scale) return AERO_ERR_INVALID;
  if (T > 0 && (!h8 || !h_scale || !out)) return AERO_ERR_INVALID;
  if (out_dtype != AERO_BF16 && out_dtype != AERO_FP32) return AERO_ERR_UNSUPPORTED;
  if (d % 16 != 0 || d > kMaxD || V > (1 << 30)) return AERO_ERR_UNSUPPORTED;
  if (!aero_aligned16(h8) || !aero_aligned16(w8)) return AERO_ERR_INVALID;
  if (reinterpret_cast<uintptr_t>(out) % (out_dtype == AERO_FP32 ? 4 : 2)) return AERO_ERR_INVALID;
  int rc = aero_check_ctx(ctx);
  if (rc) return rc;
  if (T == 0) return AERO_OK;
  Params p = {(int)T, d, V, 0, 1, h_scale, w_scale, out, ctx->d_status, 0, 0};
  const CUtensorMapDataType U8 = CU_TENSOR_MAP_DATA_TYPE_UINT8;
  CUtensorMap tmW, tmH;
  // (rows / pair kernel: d = 1536, V = 151936: 65 tokens 51.6 / 54.5 us, 128 tokens 54.1 / 59.0; V = 20000, 128 tokens 15.4
  // / 16.8; d = 3584, V = 152064: 64 tokens 100.5 / 102.8, 128 tokens 109.5 / 107.4.  A pair's units of 256 rows are a
  // coarser cut of the vocabulary.)
  if (T <= kRowsN) {
    p.n = (int)((T + 15) / 16 * 16);
    if ((rc = aero_make_tmap_2d(ctx, &tmW, U8, 1, w8, V, d, d, kRowBlock, BK))) return rc;
    CUtensorMap tmW4;
    if ((rc = aero_make_tmap_2d(ctx, &tmW4, U8, 1, w8, V, d, d, BM, BK))) return rc;
    if ((rc = aero_make_tmap_2d(ctx, &tmH, U8, 1, h8, T, d, d, (uint32_t)p.n, BK))) return rc;
    // W rows are d bytes apart: 128 bytes of each are a poor unit for the memory.  The more of a row is asked for at a
    // time the better, as long as the ring holds three stages (3584 x 152064, one / two / three / five slabs a stage: one
    // token 105 / 94.5 / 93.7 / 92.2 us; 128 tokens 114 / 109 / 116 us, the last with two stages).
    const size_t slab = A_BYTES + (size_t)p.n * BK;
    p.slabs = (int)(kRing / (3 * slab));
    p.stages = (int)(kRing / (p.slabs * slab));            // 3 or 4: at least two slabs fit three times, whatever n
    static_assert(kRing / (3 * (A_BYTES + kRowsN * BK)) >= 2 && kMaxStages == 4, "depth of the ring");
    auto kernel = out_dtype == AERO_FP32 ? q8_rows_kernel<float> : q8_rows_kernel<__nv_bfloat16>;
    AERO_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)R_SMEM));
    const int blocks = (V + kRowBlock - 1) / kRowBlock;
    kernel<<<blocks < ctx->sm_count ? blocks : ctx->sm_count, THREADS, R_SMEM, ctx->stream>>>(tmW, tmW4, tmH, p);
  } else {
    // equal token tiles of at most 256, in steps of 32 (16 tokens from each CTA of the pair)
    p.n_tok = (int)((T + kPairN - 1) / kPairN);
    p.n = (int)(((T + p.n_tok - 1) / p.n_tok + 31) / 32 * 32);
    if ((rc = aero_make_tmap_2d(ctx, &tmW, U8, 1, w8, V, d, d, BM, BK))) return rc;
    if ((rc = aero_make_tmap_2d(ctx, &tmH, U8, 1, h8, T, d, d, (uint32_t)(p.n / 2), BK))) return rc;
    auto kernel = out_dtype == AERO_FP32 ? q8_pair_kernel<float> : q8_pair_kernel<__nv_bfloat16>;
    AERO_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)P_SMEM));
    const long long units = (long long)((V + 2 * BM - 1) / (2 * BM)) * p.n_tok;
    const long long max_pairs = ctx->sm_count / 2 > 0 ? ctx->sm_count / 2 : 1;
    kernel<<<2 * (int)(units < max_pairs ? units : max_pairs), THREADS, P_SMEM, ctx->stream>>>(tmW, tmH, p);
  }
  ctx->launches += 1;
  AERO_CUDA_TRY(cudaGetLastError());
  return AERO_OK;
}
