// expert_epilogue.cuh -- the way of bf16 rows from an epilogue group's staging to memory, shared by the products on the
// tensor cores that have features along M and rows along N (expert_gemm.cu, expert_mx.cu).
#pragma once

#include "experts.cuh"
#include "ptx.cuh"

namespace smoes {

constexpr int kGemmGroups = 4;                   // of four epilogue warps

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// The group's staging between its four warps: they fill a chunk's half and arrive; warp 0 of the group waits for them and
// hands the half to the copy engine. Before the next chunk but one goes into the same half, warp 0 has seen it read and
// says so when it begins that chunk itself; so the others run up to a chunk ahead instead of meeting at every chunk.
constexpr int kBarVote = 1, kBarFull = 1 + kGemmGroups, kBarFree = 1 + 2 * kGemmGroups;   // + group
// kHalves = 1: a staging of one chunk, free when its store and all warps have read it.
template <int kHalves = 2>
__device__ __forceinline__ void staging_acquire(int g, bool first_warp, bool issuer) {
  if (first_warp) {
    if (issuer) tma_store_wait_read<kHalves - 1>();   // of two halves: all but the chunk before this one
    __syncwarp();
    if (kHalves == 1) named_bar(kBarFree + g, 128); else named_bar_arrive(kBarFree + g, 128);
  } else {
    named_bar(kBarFree + g, 128);
  }
}
// all: every warp waits (to copy the chunk itself), not just the first.
__device__ __forceinline__ void staging_filled(int g, bool first_warp, bool all) {
  if (first_warp || all)
    named_bar(kBarFull + g, 128);
  else
    named_bar_arrive(kBarFull + g, 128);
}

// Rows [0, rows) of one box to memory, for a chunk that the copy engine would write past: its expert's rows end
// inside, or g's features end inside the box and u's follow. by 128 threads, 16 bytes each. base: row 0, the
// box's first feature; n: features that exist.
__device__ __forceinline__ void copy_box(const uint8_t* box, __nv_bfloat16* base, long long stride, int rows, int n,
                                         int thread) {
  for (int i = thread; i < rows * 8; i += 128) {
    const int r = i >> 3, w = i & 7;
    if (w * 8 < n) *reinterpret_cast<uint4*>(base + r * stride + w * 8) = *reinterpret_cast<const uint4*>(box + r * 128 + ((w ^ (r & 7)) << 4));
  }
}

}  // namespace smoes
