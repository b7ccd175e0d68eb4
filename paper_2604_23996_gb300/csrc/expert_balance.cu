// expert_balance.cu -- expert-level load balance loss of the forward's saved gate values, per sample or over the batch,
// with the selections of every expert and the gradient at the gate values.
//
// Over the n_s tokens of sample s that select anything, with C_se selections of expert e:
//   f_se = E C_se / sum_e' C_se',   P_se = sum_j g_je / n_s,   L = 1/B sum_s sum_e f_se P_se,
//   dL/dg_je = f_se / (B n_s)       (f held constant: it is made of counts), the same for all of the sample's tokens,
// so the gradient leaves as a table [B, E] that the backward reads per sample.
//
// A block takes a run of at most `len` tokens of one sample, a warp a token at a time (lane l holds experts l, l + 32,
// ...), kR tokens at work and kR on their way. Runs of a sample that has several leave partials. Up to kFewSamples samples are
// finished by the block that arrives last of all, a warp a sample; with more of them each by the last of its own blocks, and
// the losses are added by the one that finishes the last sample. The sums are fp32 in a fixed order, whichever block makes
// them. Bound by the gate values' bytes (131072 x 128: 20.0 us, of which the tokens take 13 and the hand-over and the last
// block's sums 6; 10.6 us of HBM; for more than 64 experts in blocks of 1024 threads the tokens under way do not fit in 64
// registers, 80 bytes of a thread lie in local memory); small batches by latency: a launch, the search for the block's run (log2 B
// + 1 reads of its table that wait for one another), the tokens, one hand-over between the blocks (16384 x 64: 10.8 us).
#include "device_common.cuh"
#include "ptx.cuh"
#include "smoes_internal.cuh"

namespace smoes {
namespace {

constexpr int kR = 4;
constexpr int kCols = 128;                          // experts at most
constexpr int kFewSamples = 32;                     // (the workspace has a row for each beside those of whole runs)

// An arrival that hands over what the block wrote, and takes what the blocks before it handed over (thread 0, between two
// block barriers).
__device__ __forceinline__ uint32_t arrive(uint32_t* ticket) {
  uint32_t old;
  asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(old) : "l"(ticket) : "memory");
  return old;
}

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
  // the warps' sums, then (behind a barrier) those of the samples or of the slices of one
  union Sums {
    float hs[kWarps][PL * 32];
    struct {
      float h[kFewSamples][kCols];
      int c[kFewSamples][kCols];
    } few;
    struct {
      float h[kSlices][kCols];
      int c[kSlices][kCols];
    } slices;
  };
  __shared__ Sums sums;
  __shared__ int cs[PL * 32];
  __shared__ int ns, N_s[kFewSamples];
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
  struct In {
    float g[kR][PL], inv[kR];
    int sel[kR];
  };
  auto load = [&](int j0, In& in) {
#pragma unroll
    for (int r = 0; r < kR; ++r) {
      const int j = j0 + r * kWarps;
      const bool there = j < r1;
#pragma unroll
      for (int i = 0; i < PL; ++i) {
        const int e = lane + 32 * i;
        in.g[r][i] = there && e < E ? __ldcg(p.gsave + static_cast<size_t>(j) * E + e) : 0.f;
      }
      in.inv[r] = there ? __ldcg(p.ginv + j) : 0.f;
      in.sel[r] = there && lane < k ? __ldg(p.topk_idx + static_cast<size_t>(j) * k + lane) : -1;
    }
  };
  In nx;
  load(r0 + warp, nx);
#pragma unroll 1
  for (int j0 = r0 + warp; j0 < r1; j0 += kR * kWarps) {
    const In in = nx;
    if (j0 + kR * kWarps < r1) load(j0 + kR * kWarps, nx);
#pragma unroll
    for (int r = 0; r < kR; ++r) {
      const bool ok = in.sel[r] >= 0 && in.sel[r] < E;
      if (ok) atomicAdd(&cs[in.sel[r]], 1);
      if (__any_sync(0xffffffffu, ok)) {
        ++n;
#pragma unroll
        for (int i = 0; i < PL; ++i) h[i] = fmaf(in.g[r][i], in.inv[r], h[i]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < PL; ++i) sums.hs[warp][lane + 32 * i] = h[i];
  if (lane == 0 && n) atomicAdd(&ns, n);
  __syncthreads();
  float H = 0.f;
  int C = 0, N = ns;
  if (tid < E) {
    for (int w = 0; w < kWarps; ++w) H += sums.hs[w][tid];
    C = cs[tid];
  }
  // where a run's partials lie: with few samples at its block; otherwise two runs of samples that have several begin in a
  // window of `len` tokens at most, and only one of them is its sample's last
  auto row = [&](int run) { return static_cast<size_t>(2 * ((first + run * p.len) / p.len) + (run == runs - 1 ? 1 : 0)); };
  const bool few = p.few != 0;
  if (few || runs > 1) {
    const size_t at = few ? blockIdx.x : row(c);
    if (tid < E) p.part[at * E + tid] = make_uint2(__float_as_uint(H), static_cast<uint32_t>(C));
    if (tid == 0) p.part_n[at] = N;
    __syncthreads();
    if (tid == 0) last = few ? arrive(p.loss_ticket) == gridDim.x - 1 : arrive(p.ticket + s) == static_cast<uint32_t>(runs - 1);
    __syncthreads();
    if (!last) return;
  }
  if (few) {
    // every sample: columns of its runs added by kCols threads, then a warp a sample
    constexpr int kCol = PL * 32, kSl = kThreads / kCol;
    const int e = tid % kCol, sl = tid / kCol;
    const int per = p.B < kSl ? kSl / p.B : 1;   // slices a sample (then B * per <= kSl <= kFewSamples: a place for each)
    for (int q = sl; q < p.B * per; q += kSl) {
      const int smp = q / per, part = q - smp * per;
      int from = 0, of = gridDim.x;
      if (p.per_sample) {
        from = __ldg(p.base + smp);
        of = __ldg(p.base + smp + 1) - from;
      }
      const int a = from + static_cast<int>(static_cast<long long>(part) * of / per);
      const int b = from + static_cast<int>(static_cast<long long>(part + 1) * of / per);
      float hh = 0.f;
      int cc = 0, nn = 0;
      constexpr int kU = 10;
      for (int u0 = a; u0 < b; u0 += kU) {
        uint2 v[kU];
        int nv[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          const bool in = u0 + u < b;
          v[u] = in && e < E ? __ldcg(p.part + static_cast<size_t>(u0 + u) * E + e) : make_uint2(0u, 0u);
          nv[u] = in && e == 0 ? __ldcg(p.part_n + u0 + u) : 0;
        }
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          hh += __uint_as_float(v[u].x);
          cc += static_cast<int>(v[u].y);
          nn += nv[u];
        }
      }
      sums.few.h[q][e] = hh;
      sums.few.c[q][e] = cc;
      if (e == 0) N_s[q] = nn;
    }
    __syncthreads();
    for (int smp = warp; smp < p.B; smp += kWarps) {
      float hh[PL];
      int cc[PL], nn = 0, total = 0;
#pragma unroll
      for (int i = 0; i < PL; ++i) {
        hh[i] = 0.f;
        cc[i] = 0;
      }
      for (int q = smp * per; q < (smp + 1) * per; ++q) {
        nn += N_s[q];
#pragma unroll
        for (int i = 0; i < PL; ++i) {
          hh[i] += sums.few.h[q][lane + 32 * i];
          cc[i] += sums.few.c[q][lane + 32 * i];
        }
      }
#pragma unroll
      for (int i = 0; i < PL; ++i) total += cc[i];
      total = __reduce_add_sync(0xffffffffu, total);
      const float inv_total = total > 0 ? static_cast<float>(E) / static_cast<float>(total) : 0.f;
      const float inv_n = nn > 0 ? 1.f / static_cast<float>(nn) : 0.f;
      float loss = 0.f;
#pragma unroll
      for (int i = 0; i < PL; ++i) {
        const int x = lane + 32 * i;
        const float f = static_cast<float>(cc[i]) * inv_total;
        loss = fmaf(f, hh[i] * inv_n, loss);
        if (x < E) {
          const size_t at = static_cast<size_t>(smp) * E + x;
          if (p.counts) p.counts[at] = cc[i];
          if (p.d_gate) p.d_gate[at] = p.scale * f * inv_n / static_cast<float>(p.B);
        }
      }
      loss = warp_sum(loss);
      if (lane == 0) scratch[smp] = loss;
    }
    __syncthreads();
    if (warp == 0) {
      const float sum = warp_sum(lane < p.B ? scratch[lane] : 0.f);
      if (lane == 0) {
        *p.loss = sum / static_cast<float>(p.B);
        *p.loss_ticket = 0u;
      }
    }
    return;
  }
  if (runs > 1) {
    const int e = tid % kCols, sl = tid / kCols;
    const int a = static_cast<int>(static_cast<long long>(sl) * runs / kSlices);
    const int b = static_cast<int>(static_cast<long long>(sl + 1) * runs / kSlices);
    H = 0.f;
    C = N = 0;
    constexpr int kU = 8;
    for (int q = a; q < b; q += kU) {
      uint2 v[kU];
      int nv[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const bool in = q + u < b;
        const size_t at = in ? row(q + u) : 0;
        v[u] = in && e < E ? __ldcg(p.part + at * E + e) : make_uint2(0u, 0u);
        nv[u] = in && e == 0 ? __ldcg(p.part_n + at) : 0;
      }
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        H += __uint_as_float(v[u].x);
        C += static_cast<int>(v[u].y);
        N += nv[u];
      }
    }
    sums.slices.h[sl][e] = H;
    sums.slices.c[sl][e] = C;
    if (e == 0) N_s[sl] = N;
    if (tid == 0) p.ticket[s] = 0u;
    __syncthreads();
    H = 0.f;
    C = N = 0;
#pragma unroll
    for (int q = 0; q < kSlices; ++q) {
      if (tid < E) {
        H += sums.slices.h[q][tid];
        C += sums.slices.c[q][tid];
      }
      N += N_s[q];
    }
  }
  // the sample's loss and gradient (counts are at most 2^24, T k: exact in fp32)
  const float total = block_sum(static_cast<float>(C), scratch);
  const float f = total > 0.f ? static_cast<float>(E) * static_cast<float>(C) / total : 0.f;
  const float inv_n = N > 0 ? 1.f / static_cast<float>(N) : 0.f;
  if (tid < E) {
    const size_t at = static_cast<size_t>(s) * E + tid;
    if (p.counts) p.counts[at] = C;
    if (p.d_gate) p.d_gate[at] = p.scale * f * inv_n / static_cast<float>(p.B);
  }
  const float loss = block_sum(f * (H * inv_n), scratch);
  if (tid == 0) {
    p.sample_loss[s] = loss;
    last = arrive(p.loss_ticket) == static_cast<uint32_t>(p.B - 1);
  }
  __syncthreads();
  if (!last) return;
  float sum = 0.f;
  for (int i = tid; i < p.B; i += kThreads) sum += __ldcg(p.sample_loss + i);
  sum = block_sum(sum, scratch);
  if (tid == 0) {
    *p.loss = sum / static_cast<float>(p.B);
    *p.loss_ticket = 0u;
  }
}

}  // namespace

cudaError_t launch_expert_balance(ExpertBalanceParams p, int blocks, cudaStream_t s) {
  p.few = p.B <= kFewSamples;
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
