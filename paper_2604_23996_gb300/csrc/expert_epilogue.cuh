// expert_epilogue.cuh -- from the accumulators to bf16 rows in memory, shared by the products on the tensor cores that
// have features along M and rows along N (expert_gemm.cu, expert_mx.cu).
#pragma once

#include "experts.cuh"
#include "ptx.cuh"

namespace smoes {

constexpr int kGemmGroups = 4;                   // of four epilogue warps
constexpr int kChunkCols = 16;                   // columns of D that a group finishes at a time

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// A chunk is 16 columns of D (a feature per lane, an output row per column) by a CTA's 128 features. It leaves
// through shared memory as boxes of 64 features by 16 rows, 128 bytes a row in the copy engine's swizzle:
// out's boxes (two, gated one), then at 4 KB those of pre (two; gated one of g and one of u). A lane rounds two columns
// into one word, exchanges it with its neighbour and picks two neighbouring features of one row out of both; rows 4 (2,
// 6) apart are written at a time, whose swizzled words lie in different banks. Stored from the lanes, 4 bytes
// each, the 32-byte pieces of pre made dsmoe_vlm's gated layer take 557 us instead of 446 without pre.

// Shared addresses of a lane's words: its features f & ~1 and the next in box row 4 odd, with the row's swizzle;
// word i of four rows c + i lies at (at ^ i << 4) + (c + i) * 128 (c a multiple of 8: the swizzle is the row's low
// three bits, and those of i and 4 do not meet).
__device__ __forceinline__ uint32_t pair_address(const uint8_t* boxes, int f) {
  const int odd = f & 1;
  return smem_u32(boxes) + (f >> 6) * 2048 + sw128_offset(4 * odd, (f & 63) - odd);
}
// One lane's values of rows `row` and row + 4 (x0, x4) to the boxes, with its neighbour's.
__device__ __forceinline__ void put_pair(uint32_t at, int row, float x0, float x4, uint32_t pick) {
  const uint32_t own = pack_bf16(x0, x4);
  const uint32_t w = __byte_perm(own, __shfl_xor_sync(0xffffffffu, own, 1), pick);
  asm volatile("st.shared.u32 [%0], %1;" ::"r"((at ^ ((row & 3) << 4)) + row * 128), "r"(w) : "memory");
}
// Even lanes take the low halves (row `row`), odd ones the high halves (row + 4), the lower feature first.
__device__ __forceinline__ uint32_t pair_pick() { return (threadIdx.x & 1) ? 0x3276u : 0x5410u; }

// One column of D a register; f: the lane's feature among the 128 of the boxes.
__device__ __forceinline__ void put_chunk(uint8_t* boxes, int f, const float (&v)[kChunkCols]) {
  const uint32_t at = pair_address(boxes, f), pick = pair_pick();
#pragma unroll
  for (int i = 0; i < kChunkCols / 2; ++i) {
    const int c = (i >> 2) * 8 + (i & 3);
    put_pair(at, c, v[c], v[c + 4], pick);
  }
}

// The residual of a chunk in words of two features, rows as put_pair writes them. res: that of the chunk's first row at
// the lane's even feature, read for `rows` rows (none where the feature does not exist).
template <bool kGated>
__device__ __forceinline__ void load_residual(const ExpertLinearParams& l, const __nv_bfloat16* res, int rows,
                                              uint32_t (&rv)[kChunkCols / 2]) {
  const int odd = threadIdx.x & 1, up = (threadIdx.x >> 4) & 1;
#pragma unroll
  for (int i = 0; i < kChunkCols / (kGated ? 4 : 2); ++i) {
    const int c = kGated ? (i >> 1) * 8 + (i & 1) + 2 * up + 4 * odd : (i >> 2) * 8 + (i & 3) + 4 * odd;
    rv[i] = c < rows ? __ldg(reinterpret_cast<const uint32_t*>(res + c * static_cast<long long>(l.n_out))) : 0u;
  }
}
// Adds one of its words (and the neighbour's) to the lane's values of the two rows. half: 0x3244 in odd lanes, 0x1044
// in even ones (the word's high or low half as the upper half of a float).
__device__ __forceinline__ void add_residual(float& x0, float& x4, uint32_t w, uint32_t half) {
  const bool odd = threadIdx.x & 1;
  const uint32_t got = __shfl_xor_sync(0xffffffffu, w, 1);
  x0 += __uint_as_float(__byte_perm(odd ? got : w, 0u, half));
  x4 += __uint_as_float(__byte_perm(odd ? w : got, 0u, half));
}

// z (bias added) of a chunk to out, in shared memory, by whole warps. f: the lane's feature among the CTA's; rv: its
// residual, when there is one.
template <int kAct, bool kGated>
__device__ __forceinline__ void put_forward(uint8_t* boxes, int f, float (&v)[kChunkCols], bool residual,
                                            const uint32_t (&rv)[kChunkCols / 2]) {
  const uint32_t pick = pair_pick(), half = (threadIdx.x & 1) ? 0x3244u : 0x1044u;
  uint32_t at = pair_address(boxes, f);
  if (!kGated) {
    if (kAct != SMOES_ACT_NONE) {
#pragma unroll
      for (int c = 0; c < kChunkCols; ++c) v[c] = act_value<kAct, true>(v[c]);
    }
    if (residual) {
#pragma unroll
      for (int i = 0; i < kChunkCols / 2; ++i) add_residual(v[(i >> 2) * 8 + (i & 3)], v[(i >> 2) * 8 + (i & 3) + 4], rv[i], half);
    }
    put_chunk(boxes, f, v);
    return;
  }
  // gated: lanes 0-15 hold g, 16-31 u; of columns c and c + 2 each half finishes one
  const int up = (threadIdx.x >> 4) & 1;
  float y[kChunkCols / 2];                       // columns 4 (i / 2) + i % 2 + 2 up
#pragma unroll
  for (int i = 0; i < kChunkCols / 2; ++i) {
    const int c = (i >> 1) * 4 + (i & 1);
    const float got = __shfl_xor_sync(0xffffffffu, up ? v[c] : v[c + 2], 16);
    const float g = up ? got : v[c], u = up ? v[c + 2] : got;
    y[i] = act_value<kAct, true>(g) * u;
  }
  if (residual) {
#pragma unroll
    for (int i = 0; i < kChunkCols / 4; ++i) add_residual(y[(i >> 1) * 4 + (i & 1)], y[(i >> 1) * 4 + (i & 1) + 2], rv[i], half);
  }
  at = (at ^ (up << 5)) + up * 256;              // the half's rows are two further down: the swizzle's bit of 2 with it
#pragma unroll
  for (int i = 0; i < kChunkCols / 4; ++i) {
    const int a = (i >> 1) * 4 + (i & 1);
    put_pair(at, (i >> 1) * 8 + (i & 1), y[a], y[a + 2], pick);
  }
}

// The group's staging between its four warps: they fill a chunk's half and arrive; warp 0 of the group waits for them and
// hands the half to the copy engine. Before the next chunk but one goes into the same half, warp 0 has seen it read and
// says so when it begins that chunk itself; so the others run up to a chunk ahead instead of meeting at every chunk.
constexpr int kBarVote = 1, kBarFull = 1 + kGemmGroups, kBarFree = 1 + 2 * kGemmGroups;   // + group
__device__ __forceinline__ void staging_acquire(int g, bool first_warp, bool issuer) {
  if (first_warp) {
    if (issuer) tma_store_wait_read<1>();        // all but the chunk before this one
    __syncwarp();
    named_bar_arrive(kBarFree + g, 128);
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
