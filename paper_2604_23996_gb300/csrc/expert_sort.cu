// expert_sort.cu -- the router's selections in expert order: a stable counting sort of T k expert
// indices over at most 256 experts (expert, then selection number).
//
// One cooperative launch. Block b holds a contiguous run of selections, warp w of it a contiguous part:
// 1. every warp counts its experts in shared memory; a block scan over its warps gives each warp's
//    offset inside the block, and the block's counts go to the workspace;
// 2. after one grid barrier every block sums the counts of all blocks (for the experts' first rows) and
//    of the blocks before it;
// 3. every warp walks its selections again, 32 at a time: the rank among equal experts of the 32 is a
//    match and a population count, and the first of them advances the warp's counter.
// The order does not depend on atomics: counts are sums, places are ranks.
//
// Bytes: 4 N read (twice, the second time from L2), 8 N written; a few microseconds of latency (launch,
// barrier, two walks) bound it below some million selections.
#include <algorithm>

#include "experts.cuh"
#include "ptx.cuh"

namespace smoes {
namespace {

constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;

__global__ void __launch_bounds__(kSortThreads, 1) k_expert_sort(const ExpertSortParams p) {
  extern __shared__ int32_t sm[];
  int32_t* wcnt = sm;                              // [kSortWarps][E], then each warp's next row
  int32_t* tot = wcnt + kSortWarps * p.E;          // [E] rows of each expert
  int32_t* pre = tot + p.E;                        // [E] of them in the blocks before this one
  __shared__ int ok_s;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = threadIdx.x; i < (kSortWarps + 2) * p.E; i += kSortThreads) sm[i] = 0;
  pdl_wait();
  pdl_trigger();
  __syncthreads();

  const long long per_warp = p.per / kSortWarps;   // a multiple of 32
  const long long w0 = blockIdx.x * p.per + warp * per_warp;
  const long long w1 = min(w0 + per_warp, p.n);
  int32_t* mine = wcnt + warp * p.E;
  bool bad = false;
  for (long long i0 = w0; i0 < w1; i0 += 128) {    // four independent loads a lane
    int e[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const long long i = i0 + 32 * u + lane;
      e[u] = i < w1 ? __ldg(p.topk_idx + i) : -1;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      bad |= e[u] >= p.E;
      if (e[u] >= 0 && e[u] < p.E) atomicAdd(mine + e[u], 1);
    }
  }
  if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(p.status, kStatusData);
  __syncthreads();
  for (int e = threadIdx.x; e < p.E; e += kSortThreads) {   // exclusive scan over the warps
    int run = 0;
    for (int w = 0; w < kSortWarps; ++w) {
      const int c = wcnt[w * p.E + e];
      wcnt[w * p.E + e] = run;
      run += c;
    }
    if (p.G > 1)
      p.counts[static_cast<long long>(blockIdx.x) * p.E + e] = run;
    else
      tot[e] = run;
  }
  if (p.G > 1) {
    __syncthreads();
    if (threadIdx.x == 0) ok_s = grid_barrier(p.sync, p.G, p.limit_ns, p.status);
    __syncthreads();
    if (!ok_s) return;
    // `parts` threads per expert share the blocks' counts
    const int parts = kSortThreads / p.E;
    const int e = threadIdx.x % p.E, part = threadIdx.x / p.E;
    if (part < parts) {
      int all = 0, before = 0;
#pragma unroll 8
      for (int b = part; b < p.G; b += parts) {
        const int c = __ldcg(p.counts + static_cast<long long>(b) * p.E + e);
        all += c;
        before += b < static_cast<int>(blockIdx.x) ? c : 0;
      }
      atomicAdd(tot + e, all);
      atomicAdd(pre + e, before);
    }
  }
  __syncthreads();
  if (warp == 0) {                                 // first rows: exclusive scan over the experts
    int c[8], sum = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      c[i] = lane * 8 + i < p.E ? tot[lane * 8 + i] : 0;
      sum += c[i];
    }
    int run = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, run, o);
      if (lane >= o) run += v;
    }
    int at = run - sum;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = lane * 8 + i;
      if (e < p.E) {
        pre[e] += at;
        if (blockIdx.x == 0) p.offsets[e] = at;
        at += c[i];
      }
    }
    const int n_rows = __shfl_sync(0xffffffffu, run, 31);
    if (lane == 0) {
      ok_s = n_rows;
      if (blockIdx.x == 0) p.offsets[p.E] = n_rows;
    }
  }
  __syncthreads();
  const int n_rows = ok_s;
  for (int i = threadIdx.x; i < kSortWarps * p.E; i += kSortThreads) wcnt[i] += pre[i % p.E];
  __syncthreads();

  const unsigned lt_mask = (1u << lane) - 1u;
  for (long long i0 = w0; i0 < w1; i0 += 32) {     // the whole warp takes every step
    const long long i = i0 + lane;
    int e = i < w1 ? __ldg(p.topk_idx + i) : -1;
    if (e >= p.E) e = -1;
    const unsigned same = __match_any_sync(0xffffffffu, e);
    const int rank = __popc(same & lt_mask);
    const int row = e >= 0 ? mine[e] + rank : -1;
    __syncwarp();
    if (e >= 0 && rank == 0) mine[e] += __popc(same);
    __syncwarp();
    if (i < w1) {
      p.slot_row[i] = row;
      if (row >= 0) p.row_slot[row] = static_cast<int32_t>(i);
    }
  }
  for (long long r = n_rows + static_cast<long long>(blockIdx.x) * kSortThreads + threadIdx.x; r < p.n;
       r += static_cast<long long>(p.G) * kSortThreads)
    p.row_slot[r] = -1;
}

}  // namespace

cudaError_t launch_expert_sort(const ExpertSortParams& p, cudaStream_t s) {
  const size_t smem = sizeof(int32_t) * (kSortWarps + 2) * p.E;   // at most 34.8 KB
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.G);
  cfg.blockDim = dim3(kSortThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeCooperative;    // every block resident: the barrier is safe
  attr[1].val.cooperative = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.G > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, k_expert_sort, p);
}

}  // namespace smoes
