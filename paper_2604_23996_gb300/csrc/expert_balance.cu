// expert_balance.cu -- expert-level load balance loss of the forward's saved gate values, per sample or over the batch,
// with the selections of every expert and the gradient at the gate values.
//
// Over the n_s tokens of sample s that select anything, with C_se selections of expert e:
//   f_se = E C_se / sum_e' C_se',   P_se = sum_j g_je / n_s,   L = 1/B sum_s sum_e f_se P_se,
//   dL/dg_je = f_se / (B n_s)       (f held constant: it is made of counts), the same for all of the sample's tokens,
// so the gradient leaves as a table [B, E] that the backward reads per sample.
//
// A block takes a run of at most `len` tokens of one sample, a warp a token at a time (lane l holds experts l, l + 32,
// ...), kR tokens with their loads in flight. Runs of a longer sample leave partials, and the block that finishes last
// adds them in order (a ticket per sample); the block that finishes the last sample adds the samples' losses. The sums
// are fp32 in a fixed order, whichever block makes them. Bound by the gate values' bytes; small batches by the latency
// of one launch and the hand-over between the blocks.
#include "device_common.cuh"
#include "ptx.cuh"
#include "smoes_internal.cuh"

namespace smoes {
namespace {

constexpr int kR = 4;
constexpr int kCols = 128;                          // experts at most

// The sum over the block of one value per thread, by thread 0's warp; the same order every time.
__device__ __forceinline__ float block_sum(float v, float* scratch) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  v = warp_sum(v);
  if (lane == 0) scratch[warp] = v;
  __syncthreads();
  v = warp_sum(lane < warps ? scratch[lane] : 0.f);
  __syncthreads();
  return v;
}

template <int PL, int kThreads>
__global__ void __launch_bounds__(kThreads) k_expert_balance(const ExpertBalanceParams p) {
  constexpr int kWarps = kThreads / 32;
  constexpr int kSlices = kThreads / kCols;
  __shared__ float hs[kWarps][PL * 32];
  __shared__ int cs[PL * 32];
  __shared__ int ns;
  __shared__ float h_sl[kSlices][kCols];
  __shared__ int c_sl[kSlices][kCols], n_sl[kSlices];
  __shared__ float scratch[32];
  __shared__ int last;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int E = p.E, k = p.k;
  pdl_wait();                                       // the forward's saved gate values
  pdl_trigger();
  // this block's run: run c of sample s
  int s = 0, c = blockIdx.x, first = 0, end = p.T, runs = gridDim.x;
  if (p.per_sample) {
    int hi = p.B;                                   // base[s] <= block < base[s + 1]
    while (hi - s > 1) {
      const int mid = (s + hi) >> 1;
      if (__ldg(p.base + mid) <= c) s = mid; else hi = mid;
    }
    const int b0 = __ldg(p.base + s);
    runs = __ldg(p.base + s + 1) - b0;
    c -= b0;
    first = __ldg(p.offsets + s);
    end = __ldg(p.offsets + s + 1);
  }
  const int r0 = first + c * p.len, r1 = min(r0 + p.len, end);
  for (int e = tid; e < PL * 32; e += kThreads) cs[e] = 0;
  if (tid == 0) ns = 0;
  __syncthreads();
  float h[PL];
#pragma unroll
  for (int i = 0; i < PL; ++i) h[i] = 0.f;
  int n = 0;
  for (int j0 = r0 + warp; j0 < r1; j0 += kR * kWarps) {
    float g[kR][PL], inv[kR];
    int sel[kR];
#pragma unroll
    for (int r = 0; r < kR; ++r) {
      const int j = j0 + r * kWarps;
      const bool in = j < r1;
#pragma unroll
      for (int i = 0; i < PL; ++i) {
        const int e = lane + 32 * i;
        g[r][i] = in && e < E ? __ldcg(p.gsave + static_cast<size_t>(j) * E + e) : 0.f;
      }
      inv[r] = in ? __ldcg(p.ginv + j) : 0.f;
      sel[r] = in && lane < k ? __ldg(p.topk_idx + static_cast<size_t>(j) * k + lane) : -1;
    }
#pragma unroll
    for (int r = 0; r < kR; ++r) {
      const bool ok = sel[r] >= 0 && sel[r] < E;
      if (ok) atomicAdd(&cs[sel[r]], 1);
      if (__any_sync(0xffffffffu, ok)) {
        ++n;
#pragma unroll
        for (int i = 0; i < PL; ++i) h[i] = fmaf(g[r][i], inv[r], h[i]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < PL; ++i) hs[warp][lane + 32 * i] = h[i];
  if (lane == 0 && n) atomicAdd(&ns, n);
  __syncthreads();
  float H = 0.f;
  int C = 0, N = ns;
  if (tid < E) {
    for (int w = 0; w < kWarps; ++w) H += hs[w][tid];
    C = cs[tid];
  }
  if (runs > 1) {
    // where a run's partials lie: two runs of longer samples begin in a window of `len` tokens at most, and only one of
    // them is its sample's last
    auto row = [&](int run) { return static_cast<size_t>(2 * ((first + run * p.len) / p.len) + (run == runs - 1 ? 1 : 0)); };
    if (tid < E) {
      p.part_h[row(c) * E + tid] = H;
      p.part_c[row(c) * E + tid] = C;
    }
    if (tid == 0) p.part_n[row(c)] = N;
    __threadfence();
    __syncthreads();
    if (tid == 0) last = atomicAdd(p.ticket + s, 1u) == static_cast<uint32_t>(runs - 1);
    __syncthreads();
    if (!last) return;
    __threadfence();
    const int e = tid % kCols, sl = tid / kCols;
    const int a = static_cast<int>(static_cast<long long>(sl) * runs / kSlices);
    const int b = static_cast<int>(static_cast<long long>(sl + 1) * runs / kSlices);
    H = 0.f;
    C = N = 0;
    constexpr int kU = 8;
    for (int q = a; q < b; q += kU) {
      float hv[kU];
      int cv[kU], nv[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const bool in = q + u < b;
        const size_t at = in ? row(q + u) : 0;
        hv[u] = in && e < E ? __ldcg(p.part_h + at * E + e) : 0.f;
        cv[u] = in && e < E ? __ldcg(p.part_c + at * E + e) : 0;
        nv[u] = in ? __ldcg(p.part_n + at) : 0;
      }
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        H += hv[u];
        C += cv[u];
        N += nv[u];
      }
    }
    h_sl[sl][e] = H;
    c_sl[sl][e] = C;
    if (e == 0) n_sl[sl] = N;
    if (tid == 0) p.ticket[s] = 0u;
    __syncthreads();
    H = 0.f;
    C = N = 0;
#pragma unroll
    for (int q = 0; q < kSlices; ++q) {
      if (tid < E) {
        H += h_sl[q][tid];
        C += c_sl[q][tid];
      }
      N += n_sl[q];
    }
  }
  // the sample's loss and gradient (counts stay below 2^24: exact in fp32)
  const float total = block_sum(static_cast<float>(C), scratch);
  const float f = total > 0.f ? static_cast<float>(E) * static_cast<float>(C) / total : 0.f;
  const float inv_n = N > 0 ? 1.f / static_cast<float>(N) : 0.f;
  if (tid < E) {
    const size_t at = static_cast<size_t>(s) * E + tid;
    if (p.counts) p.counts[at] = C;
    if (p.d_gate) p.d_gate[at] = p.scale * f * inv_n / static_cast<float>(p.B);
  }
  const float loss = block_sum(f * (H * inv_n), scratch);
  if (p.B == 1) {
    if (tid == 0) *p.loss = loss;
    return;
  }
  if (tid == 0) {
    p.sample_loss[s] = loss;
    __threadfence();
    last = atomicAdd(p.loss_ticket, 1u) == static_cast<uint32_t>(p.B - 1);
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  float sum = 0.f;
  for (int i = tid; i < p.B; i += kThreads) sum += __ldcg(p.sample_loss + i);
  sum = block_sum(sum, scratch);
  if (tid == 0) {
    *p.loss = sum / static_cast<float>(p.B);
    *p.loss_ticket = 0u;
  }
}

}  // namespace

cudaError_t launch_expert_balance(const ExpertBalanceParams& p, int blocks, cudaStream_t s) {
  if (p.E < 1 || p.E > kCols || blocks < 1) return cudaErrorInvalidValue;
  // short runs leave most warps of a large block without a token
  const bool wide = p.T / blocks >= 64;
  auto run = [&](auto small, auto large) {
    return wide ? launch_pdl(large, dim3(blocks), dim3(1024), 0, s, p) : launch_pdl(small, dim3(blocks), dim3(256), 0, s, p);
  };
  if (p.E <= 32) return run(k_expert_balance<1, 256>, k_expert_balance<1, 1024>);
  if (p.E <= 64) return run(k_expert_balance<2, 256>, k_expert_balance<2, 1024>);
  return run(k_expert_balance<4, 256>, k_expert_balance<4, 1024>);
}

}  // namespace smoes
