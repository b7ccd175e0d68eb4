// expert_rows.cu -- tokens into expert order and back, with weights, and the gradients of both:
//   dispatch      Xs[slot_row[t, s]] = X[t]
//   combine       Y[t] = residual[t] + sum_s w[t, s] Ys[slot_row[t, s]]      (w = 1: dispatch's gradient)
//   combine_bwd   dYs[slot_row[t, s]] = w[t, s] dY[t],  dw[t, s] = <dY[t], Ys[slot_row[t, s]]>
//
// All three walk the tokens, not the rows: a token's k rows are read or written by the warp that holds
// the token's own row in registers, so every row crosses HBM once (walking the rows would fetch each
// token k times). Sums are fp32, in slot order: no atomics, the same bits every time. Bound by HBM.
#include <algorithm>

#include "device_common.cuh"
#include "experts.cuh"
#include "ptx.cuh"

namespace smoes {
namespace {

constexpr int kRowThreads = 256;
constexpr int kRowWarps = kRowThreads / 32;

// The rows of a token's selections, one per lane s < k; -1 for none (also for a row out of range).
__device__ __forceinline__ int token_rows(const ExpertRowsParams& p, long long t) {
  const int lane = threadIdx.x & 31;
  const int r = lane < p.k ? __ldg(p.slot_row + t * p.k + lane) : -1;
  return r < static_cast<long long>(p.T) * p.k ? r : -1;
}

// A warp's unit of work: `kWords` words of 16 bytes a lane of one token.
template <int kWords>
__global__ void __launch_bounds__(kRowThreads) k_dispatch(const ExpertRowsParams p, int words, int units) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const long long R = static_cast<long long>(p.T) * p.k;
  const long long unit = static_cast<long long>(blockIdx.x) * kRowWarps + (threadIdx.x >> 5);
  if (unit < static_cast<long long>(p.T) * units) {
    const long long t = unit / units;
    const int w0 = static_cast<int>(unit - t * units) * (32 * kWords) + lane;
    const int rows = token_rows(p, t);
    const uint4* x = static_cast<const uint4*>(p.tokens) + t * words;
    uint4 v[kWords];
#pragma unroll
    for (int u = 0; u < kWords; ++u)
      if (w0 + 32 * u < words) v[u] = __ldg(x + w0 + 32 * u);
    for (int s = 0; s < p.k; ++s) {
      const int r = __shfl_sync(0xffffffffu, rows, s);
      if (r < 0) continue;
      uint4* out = static_cast<uint4*>(p.rows_out) + static_cast<long long>(r) * words;
#pragma unroll
      for (int u = 0; u < kWords; ++u)
        if (w0 + 32 * u < words) out[w0 + 32 * u] = v[u];
    }
  }
  zero_rows(p.rows_out, expert_begin(p.offsets, p.E, R), R, words);
}

template <class T, int KM>
__global__ void __launch_bounds__(kRowThreads) k_combine(const ExpertRowsParams p, int words, int units) {
  pdl_wait();
  pdl_trigger();
  constexpr int N = Pack<T>::N;
  const int lane = threadIdx.x & 31;
  const long long unit = static_cast<long long>(blockIdx.x) * kRowWarps + (threadIdx.x >> 5);
  if (unit >= static_cast<long long>(p.T) * units) return;
  const long long t = unit / units;
  const int word = static_cast<int>(unit - t * units) * 32 + lane;
  const bool in = word < words;
  const int rows = token_rows(p, t);
  float w_lane = 1.f;
  if (p.w && lane < p.k) w_lane = __ldg(p.w + t * p.k + lane);
  uint4 v[KM], base = make_uint4(0u, 0u, 0u, 0u);
  if (p.tokens && in) base = __ldg(static_cast<const uint4*>(p.tokens) + t * words + word);
#pragma unroll
  for (int s = 0; s < KM; ++s) {
    const int r = __shfl_sync(0xffffffffu, rows, s);
    if (r >= 0 && in) v[s] = __ldg(static_cast<const uint4*>(p.rows) + static_cast<long long>(r) * words + word);
  }
  float a[N];
  Pack<T>::unpack(base, a);
#pragma unroll
  for (int s = 0; s < KM; ++s) {
    const int r = __shfl_sync(0xffffffffu, rows, s);
    const float w = __shfl_sync(0xffffffffu, w_lane, s);
    if (r >= 0) {
      float f[N];
      Pack<T>::unpack(v[s], f);
#pragma unroll
      for (int i = 0; i < N; ++i) a[i] = fmaf(w, f[i], a[i]);
    }
  }
  if (in) static_cast<uint4*>(p.tokens_out)[t * words + word] = Pack<T>::pack(a);
}

template <class T, int KM>
__global__ void __launch_bounds__(kRowThreads) k_combine_bwd(const ExpertRowsParams p, int words) {
  pdl_wait();
  pdl_trigger();
  constexpr int N = Pack<T>::N;
  const int lane = threadIdx.x & 31;
  const long long R = static_cast<long long>(p.T) * p.k;
  const long long t = static_cast<long long>(blockIdx.x) * kRowWarps + (threadIdx.x >> 5);
  if (t < p.T) {
    const int rows = token_rows(p, t);
    const float w_lane = lane < p.k ? __ldg(p.w + t * p.k + lane) : 0.f;
    float dot[KM];
#pragma unroll
    for (int s = 0; s < KM; ++s) dot[s] = 0.f;
    const uint4* dy = static_cast<const uint4*>(p.tokens) + t * words;
    for (int w0 = 0; w0 < words; w0 += 32) {
      const int word = w0 + lane;
      const bool in = word < words;
      uint4 g4 = make_uint4(0u, 0u, 0u, 0u), v[KM];
      if (in) g4 = __ldg(dy + word);
#pragma unroll
      for (int s = 0; s < KM; ++s) {
        const int r = __shfl_sync(0xffffffffu, rows, s);
        v[s] = make_uint4(0u, 0u, 0u, 0u);
        if (r >= 0 && in) v[s] = __ldg(static_cast<const uint4*>(p.rows) + static_cast<long long>(r) * words + word);
      }
      float g[N];
      Pack<T>::unpack(g4, g);
#pragma unroll
      for (int s = 0; s < KM; ++s) {
        const int r = __shfl_sync(0xffffffffu, rows, s);
        const float w = __shfl_sync(0xffffffffu, w_lane, s);
        float y[N], o[N];
        Pack<T>::unpack(v[s], y);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          dot[s] = fmaf(g[i], y[i], dot[s]);
          o[i] = w * g[i];
        }
        if (r >= 0 && in)
          static_cast<uint4*>(p.rows_out)[static_cast<long long>(r) * words + word] = Pack<T>::pack(o);
      }
    }
    float mine = 0.f;
#pragma unroll
    for (int s = 0; s < KM; ++s) {
      const float d = warp_sum(dot[s]);
      const int r = __shfl_sync(0xffffffffu, rows, s);
      if (lane == s) mine = r >= 0 ? d : 0.f;
    }
    if (lane < p.k) p.dw[t * p.k + lane] = mine;
  }
  zero_rows(p.rows_out, expert_begin(p.offsets, p.E, R), R, words);
}

// KM: selections the unrolled loops hold, the smallest of 2, 4, 6, 8 and 16 that takes k.
template <class F>
cudaError_t with_k(int k, F&& f) {
  if (k <= 2) return f(std::integral_constant<int, 2>());
  if (k <= 4) return f(std::integral_constant<int, 4>());
  if (k <= 6) return f(std::integral_constant<int, 6>());
  if (k <= 8) return f(std::integral_constant<int, 8>());
  return f(std::integral_constant<int, 16>());
}

int row_words(const ExpertRowsParams& p, bool bf16) { return p.d / (bf16 ? 8 : 4); }
dim3 warps_grid(long long units) { return dim3(static_cast<unsigned>((units + kRowWarps - 1) / kRowWarps)); }

}  // namespace

cudaError_t launch_expert_dispatch(const ExpertRowsParams& p, bool bf16, cudaStream_t s) {
  constexpr int kWords = 4;
  const int words = row_words(p, bf16), units = (words + 32 * kWords - 1) / (32 * kWords);
  return launch_pdl(k_dispatch<kWords>, warps_grid(static_cast<long long>(p.T) * units), dim3(kRowThreads), 0, s, p,
                    words, units);
}

cudaError_t launch_expert_combine(const ExpertRowsParams& p, bool bf16, cudaStream_t s) {
  const int words = row_words(p, bf16), units = (words + 31) / 32;
  const dim3 grid = warps_grid(static_cast<long long>(p.T) * units);
  return with_k(p.k, [&](auto km) {
    constexpr int KM = decltype(km)::value;
    return bf16 ? launch_pdl(k_combine<__nv_bfloat16, KM>, grid, dim3(kRowThreads), 0, s, p, words, units)
                : launch_pdl(k_combine<float, KM>, grid, dim3(kRowThreads), 0, s, p, words, units);
  });
}

cudaError_t launch_expert_combine_bwd(const ExpertRowsParams& p, bool bf16, cudaStream_t s) {
  const int words = row_words(p, bf16);
  const dim3 grid = warps_grid(p.T);
  return with_k(p.k, [&](auto km) {
    constexpr int KM = decltype(km)::value;
    return bf16 ? launch_pdl(k_combine_bwd<__nv_bfloat16, KM>, grid, dim3(kRowThreads), 0, s, p, words)
                : launch_pdl(k_combine_bwd<float, KM>, grid, dim3(kRowThreads), 0, s, p, words);
  });
}

}  // namespace smoes
