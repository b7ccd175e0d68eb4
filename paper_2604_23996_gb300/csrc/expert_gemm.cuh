// expert_gemm.cuh -- the tiles of the experts' products on the tensor cores, shared by the bf16 and fp32 kernels.
#pragma once

#include <mutex>

#include "experts.cuh"

namespace smoes {

constexpr int kBarBytes = 448;                   // shared memory for a kernel's barriers and counts

// A tile: 256 features (along M) by up to 2^tile_shift rows (along N; for dW n_in by n_z), blocks of kBlock along the depth.
struct GemmTile {
  int e, m;                                      // expert, feature tile
  int row0;                                      // first row (dW: the expert's first row)
  int cols;                                      // rows of the tile (dW: columns of n_z)
  int col0;                                      // dW: first column of n_z
  int blocks;                                    // blocks along the depth
  int last;                                      // dW: rows of the last block
};

// off: the offsets in shared memory (from global memory each tile began with a round trip to L2).
template <int kMode, int kBlock>
__device__ __forceinline__ GemmTile gemm_tile(const ExpertGemmParams& p, const RowTiles& rt, const int32_t* off,
                                              int tile) {
  GemmTile t;
  const int R = static_cast<int>(p.l.R);
  if (kMode == kGemmGradW) {
    const int per = p.m_tiles * p.n_tiles;
    t.e = tile / per;
    const int in = tile - t.e * per;
    const int j = in / p.m_tiles;
    t.m = in - j * p.m_tiles;
    t.col0 = j << p.tile_shift;
    t.cols = min(1 << p.tile_shift, p.l.n_z - t.col0);
    t.row0 = expert_row(off, t.e, R);
    const int rows = max(0, expert_row(off, t.e + 1, R) - t.row0);
    t.blocks = (rows + kBlock - 1) / kBlock;
    t.last = rows - (t.blocks - 1) * kBlock;
    return t;
  }
  const int r = tile / p.m_tiles;
  t.m = tile - r * p.m_tiles;
  const RowTile row = find_row_tile(rt, off, p.l.E, R, ShiftRows{p.tile_shift}, r);
  t.e = row.e;
  t.row0 = row.row0;
  t.cols = min(1 << p.tile_shift, row.row1 - row.row0);
  t.col0 = 0;
  t.last = kBlock;
  t.blocks = ((kMode == kGemmForward ? p.l.n_in : p.l.n_z) + kBlock - 1) / kBlock;
  return t;
}

// N of a tile's products: both CTAs hold half of the rows. dW: whole 64-column boxes in each.
template <int kMode>
__device__ __forceinline__ int gemm_n(int cols) {
  return kMode == kGemmGradW ? (cols + 127) & ~127 : (cols + 31) & ~31;
}

// Chooses tile_shift (between the log2s narrowest and widest) and n_tiles of a launch and returns its pairs of CTAs. Tiles
// have the widest kind of columns, unless all tiles of a narrower kind have a pair each (every tile's products then
// take less time in the one round that there is) or no expert can have more rows (narrower stages, more of them).
// Measured, bf16: 256 x 2048 x 256 takes 14.5 us as one tile of 256 rows and 10.1 us as four of 64.
inline int gemm_split(ExpertGemmParams& p, ExpertGemmMode mode, int widest, int narrowest, int pairs) {
  const ExpertLinearParams& l = p.l;
  long long tiles = 0;
  for (int shift = narrowest; shift <= widest; ++shift) {
    const int cols = 1 << shift;
    p.tile_shift = shift;
    p.n_tiles = (l.n_z + cols - 1) / cols;
    // at most R / cols + min(E, R) row tiles exist, whatever the offsets are
    tiles = mode == kGemmGradW ? static_cast<long long>(l.E) * p.n_tiles : l.R / cols + (l.R < l.E ? l.R : l.E);
    tiles *= p.m_tiles;
    if (tiles <= pairs || (mode != kGemmGradW && l.R <= cols)) break;
  }
  return tiles < 1 ? 1 : tiles < pairs ? static_cast<int>(tiles) : pairs;
}

// Zeros in a CTA's half of a tile of dW, by `warps` warps of which this is number w: a row of 128 features a warp at a
// time, 16 bytes a lane.
__device__ __forceinline__ void zero_weight_tile(const ExpertLinearParams& l, const GemmTile& t, int rank, int w,
                                                 int warps) {
  const int f = t.m * 256 + rank * 128 + (threadIdx.x & 31) * 4;
  if (f >= l.n_in) return;                       // (n_in is a multiple of 4)
  float* row = l.dW + (static_cast<long long>(t.e) * l.n_z + t.col0) * l.n_in + f;
  for (int c = w; c < t.cols; c += warps)
    *reinterpret_cast<float4*>(row + static_cast<long long>(c) * l.n_in) = make_float4(0.f, 0.f, 0.f, 0.f);
}

// Pairs of CTAs of a kernel that the device holds at once, and its shared memory allowed (once per kernel and device).
struct GemmResidency {
  std::mutex mu;
  int pairs[64] = {};
};
template <class K>
cudaError_t gemm_pairs(GemmResidency& r, K kernel, int threads, uint32_t smem, int n_sms, int* out) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(r.mu);
  if (r.pairs[dev] == 0) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(n_sms / 2 * 2);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    int n = 0;
    e = cudaOccupancyMaxActiveClusters(&n, kernel, &cfg);
    if (e != cudaSuccess) return e;
    if (n < 1) return cudaErrorLaunchOutOfResources;
    r.pairs[dev] = n;
  }
  *out = r.pairs[dev];
  return cudaSuccess;
}

}  // namespace smoes
