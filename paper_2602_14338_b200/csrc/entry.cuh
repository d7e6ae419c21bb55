// What every C entry point of the library starts with: an NVTX range, alignment checks, the
// context's device made current.
#pragma once

#include "common.cuh"

#include <nvtx3/nvToolsExt.h>

// NVTX range over one ABI call (visible in Nsight timelines; a no-op without a profiler attached)
struct AeroRange {
  explicit AeroRange(const char* name) { nvtxRangePushA(name); }
  ~AeroRange() { nvtxRangePop(); }
};

static inline bool aero_aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
static inline bool aero_aligned256(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 255u) == 0; }

static inline int aero_check_ctx(aero_ctx* ctx) {
  if (!ctx) return AERO_ERR_INVALID;
  if (cudaSetDevice(ctx->device) != cudaSuccess) return AERO_ERR_CUDA;
  return AERO_OK;
}
