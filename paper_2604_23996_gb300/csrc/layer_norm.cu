// layer_norm.cu -- the layer norm in front of the router and the experts, with the residual stream's sum, and its
// gradients.
//
//   s = x + r (rounded to the stream's type; s = x without r),  mean = sum s / d,  var = sum (s - mean)^2 / d,
//   rstd = 1 / sqrt(var + eps),  h = (s - mean) rstd,  y = h w + b
//
//   a = dy w,  dx = rstd (a - mean(a) - h mean(a h)) + ds,  dw = sum_t dy h,  db = sum_t dy
//
// Forward: a row is read once into registers and its variance is taken around the mean that was just formed, so no
// digits cancel where the mean is far from zero. A group of threads holds a row, kWords words of 16 bytes a thread.
//
// Backward: a thread keeps the same columns of every row that its block walks, so the sums of dw and db over the rows
// stay in its registers; they leave once per block and k_norm_sum adds the blocks in order. All sums are fp32 in a
// fixed order. Both are bound by HBM: 131072 x 2048 bf16 forward with the stream's sum 307 us (7.0 TB/s), 16384 x 2048 backward
// with the stream's gradient 44.7 us (6.0 TB/s) and 5 us for the sum over the blocks' partials. Without rows fetched ahead it took
// 118 us; 64 threads a row with four words each spill (225 us); 16 rows of 2048, read by a warp each, 5.1 us.
#include <algorithm>
#include <new>

#include "device_common.cuh"
#include "experts.cuh"
#include "ptx.cuh"

using namespace smoes;

struct smoes_norm_s {
  smoes_norm_desc desc{};
  int n_sms = 148;
  size_t ws_bytes = 0;
};

namespace smoes {
namespace {

constexpr int kNormWordsMax = 2048;              // of 16 bytes a row

struct NormParams {
  int T, words, d;
  float eps, inv_d;
  const void* X;
  const void* residual;      // r, or ds of the backward
  const float* w;
  const float* b;
  void* S;
  void* Y;                   // y, or dx
  float* mean;
  float* rstd;
  const void* dY;
  float* part;               // [blocks][2][d]
  int blocks;
  float* dw;
  float* db;
  int accumulate;
};

// Sums of kN values over the kTpr threads of a row, the same in all of them. Groups of more than a warp meet in shared
// memory: scratch [groups][kTpr / 32][kN]; the caller keeps two and uses them in turn, one block barrier a call.
template <int kTpr, int kN>
__device__ __forceinline__ void row_sums(float (&v)[kN], float* scratch) {
#pragma unroll
  for (int o = 1; o < (kTpr < 32 ? kTpr : 32); o <<= 1) {
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  }
  if constexpr (kTpr > 32) {
    constexpr int kW = kTpr / 32;
    const int warp = threadIdx.x >> 5, first = warp / kW * kW;
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
      for (int i = 0; i < kN; ++i) scratch[warp * kN + i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = 0.f;
#pragma unroll
    for (int q = 0; q < kW; ++q) {
#pragma unroll
      for (int i = 0; i < kN; ++i) v[i] += scratch[(first + q) * kN + i];
    }
  }
}

template <int N>
__device__ __forceinline__ void load_floats(const float* p, float (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const float4 v = __ldg(reinterpret_cast<const float4*>(p + i));
    f[i] = v.x;
    f[i + 1] = v.y;
    f[i + 2] = v.z;
    f[i + 3] = v.w;
  }
}

template <class T, int kTpr, int kWords, int kThreads>
__global__ void __launch_bounds__(kThreads) k_norm_fwd(const NormParams p) {
  constexpr int N = Pack<T>::N;
  __shared__ float scratch[2][kThreads / 32];
  pdl_wait();
  pdl_trigger();
  const int c = threadIdx.x % kTpr;
  const long long t = static_cast<long long>(blockIdx.x) * (kThreads / kTpr) + threadIdx.x / kTpr;
  const bool row = t < p.T;                      // (all threads of a block stay for its barriers)
  uint4 v[kWords], r[kWords];
#pragma unroll
  for (int u = 0; u < kWords; ++u) {
    const int i = c + u * kTpr;
    v[u] = r[u] = make_uint4(0u, 0u, 0u, 0u);
    if (row && i < p.words) {
      v[u] = __ldg(static_cast<const uint4*>(p.X) + t * p.words + i);
      if (p.residual) r[u] = __ldg(static_cast<const uint4*>(p.residual) + t * p.words + i);
    }
  }
  float sum[1] = {0.f};
#pragma unroll
  for (int u = 0; u < kWords; ++u) {
    float f[N];
    Pack<T>::unpack(v[u], f);
    if (p.residual) {
      float g[N];
      Pack<T>::unpack(r[u], g);
#pragma unroll
      for (int i = 0; i < N; ++i) f[i] += g[i];
      v[u] = Pack<T>::pack(f);                   // the norm is of the stream as it is kept
      Pack<T>::unpack(v[u], f);
      const int i = c + u * kTpr;
      if (row && i < p.words) static_cast<uint4*>(p.S)[t * p.words + i] = v[u];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) sum[0] += f[i];
  }
  row_sums<kTpr, 1>(sum, scratch[0]);
  const float mean = sum[0] * p.inv_d;
  float sq[1] = {0.f};
#pragma unroll
  for (int u = 0; u < kWords; ++u) {
    if (c + u * kTpr < p.words) {
      float f[N];
      Pack<T>::unpack(v[u], f);
#pragma unroll
      for (int i = 0; i < N; ++i) sq[0] = fmaf(f[i] - mean, f[i] - mean, sq[0]);
    }
  }
  row_sums<kTpr, 1>(sq, scratch[1]);
  const float rstd = 1.f / sqrtf(fmaf(sq[0], p.inv_d, p.eps));
  if (!row) return;
  if (c == 0 && p.mean) {
    p.mean[t] = mean;
    p.rstd[t] = rstd;
  }
#pragma unroll
  for (int u = 0; u < kWords; ++u) {
    const int i = c + u * kTpr;
    if (i < p.words) {
      float f[N], w[N], b[N];
      Pack<T>::unpack(v[u], f);
      load_floats<N>(p.w + i * N, w);
      if (p.b) {
        load_floats<N>(p.b + i * N, b);
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j) b[j] = 0.f;
      }
#pragma unroll
      for (int j = 0; j < N; ++j) f[j] = fmaf((f[j] - mean) * rstd, w[j], b[j]);
      static_cast<uint4*>(p.Y)[t * p.words + i] = Pack<T>::pack(f);
    }
  }
}

// A round of a block is kRows rows of each of its groups of kTpr threads; the next round's rows are on their way while the
// block works on this one's. Blocks of 1024 threads have 64 registers each and neither fetch ahead nor keep the weight (kLean);
// for bf16 the registers do not suffice all the same (192 bytes of a thread in local memory): 8192 x 16384 with the stream's
// gradient 336 us, of 159 at the copy's rate; 16384 x 8192 in fp32, which fits, 410 of 318; 16384 x 8192 in bf16, by 512 threads
// a row, 184 of 159.
template <class T, int kTpr, int kWords, int kRows, int kThreads, int kBlocks>
__global__ void __launch_bounds__(kThreads, kBlocks) k_norm_bwd(const NormParams p) {
  constexpr int N = Pack<T>::N;
  constexpr int kGroups = kThreads / kTpr;
  constexpr bool kLean = kThreads > 512;
  __shared__ float scratch[2][kThreads / 32 * 2 * kRows];
  extern __shared__ float join[];                // [kGroups][2][kTpr * kWords * N] where there are more groups than one
  pdl_wait();
  pdl_trigger();
  const int c = threadIdx.x % kTpr, grp = threadIdx.x / kTpr;
  const int r0 = static_cast<int>(static_cast<long long>(blockIdx.x) * p.T / gridDim.x);
  const int r1 = static_cast<int>(static_cast<long long>(blockIdx.x + 1) * p.T / gridDim.x);
  float dw[kWords][N], db[kWords][N], held[kWords][N];
  auto weight = [&](int u, float (&w)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = 0.f;
    if (c + u * kTpr < p.words) load_floats<N>(p.w + (c + u * kTpr) * N, w);
  };
#pragma unroll
  for (int u = 0; u < kWords; ++u) {
#pragma unroll
    for (int i = 0; i < N; ++i) dw[u][i] = db[u][i] = 0.f;
    if (!kLean) weight(u, held[u]);
  }
  struct In {
    uint4 dy[kRows][kWords], x[kRows][kWords], ds[kRows][kWords];
    float mean[kRows], rstd[kRows];
  };
  auto load = [&](int base, In& in) {
#pragma unroll
    for (int q = 0; q < kRows; ++q) {
      const int t = base + q * kGroups + grp;
      const bool row = t < r1;
      in.mean[q] = row ? __ldg(p.mean + t) : 0.f;
      in.rstd[q] = row ? __ldg(p.rstd + t) : 0.f;
#pragma unroll
      for (int u = 0; u < kWords; ++u) {
        const int i = c + u * kTpr;
        const long long at = static_cast<long long>(t) * p.words + i;
        in.dy[q][u] = in.x[q][u] = in.ds[q][u] = make_uint4(0u, 0u, 0u, 0u);
        if (row && i < p.words) {
          in.dy[q][u] = __ldg(static_cast<const uint4*>(p.dY) + at);
          in.x[q][u] = __ldg(static_cast<const uint4*>(p.X) + at);
          if (!kLean && p.residual) in.ds[q][u] = __ldg(static_cast<const uint4*>(p.residual) + at);
        }
      }
    }
  };
  constexpr int kStep = kGroups * kRows;
  int turn = 0;
  In nx;
  if (!kLean) load(r0, nx);
#pragma unroll 1
  for (int base = r0; base < r1; base += kStep, turn ^= 1) {
    if (kLean) load(base, nx);
    const In in = nx;
    if (!kLean && base + kStep < r1) load(base + kStep, nx);
    float sums[2 * kRows];
#pragma unroll
    for (int q = 0; q < kRows; ++q) {
      float a0 = 0.f, a1 = 0.f;
#pragma unroll
      for (int u = 0; u < kWords; ++u) {
        float g[N], h[N], w[N];
        if (kLean) weight(u, w);
        Pack<T>::unpack(in.dy[q][u], g);
        Pack<T>::unpack(in.x[q][u], h);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          if (!kLean) w[j] = held[u][j];
          h[j] = (h[j] - in.mean[q]) * in.rstd[q];
          dw[u][j] = fmaf(g[j], h[j], dw[u][j]);
          db[u][j] += g[j];
          const float a = g[j] * w[j];
          a0 += a;
          a1 = fmaf(a, h[j], a1);
        }
      }
      sums[2 * q] = a0;
      sums[2 * q + 1] = a1;
    }
    row_sums<kTpr, 2 * kRows>(sums, scratch[turn]);
#pragma unroll
    for (int q = 0; q < kRows; ++q) {
      const int t = base + q * kGroups + grp;
      if (t >= r1) break;
      const float ma = sums[2 * q] * p.inv_d, mah = sums[2 * q + 1] * p.inv_d;
#pragma unroll
      for (int u = 0; u < kWords; ++u) {
        const int i = c + u * kTpr;
        if (i < p.words) {
          const long long at = static_cast<long long>(t) * p.words + i;
          float g[N], h[N], ds[N], w[N];
          if (kLean) weight(u, w);
          Pack<T>::unpack(in.dy[q][u], g);
          Pack<T>::unpack(in.x[q][u], h);
          Pack<T>::unpack(!kLean ? in.ds[q][u] : p.residual ? __ldg(static_cast<const uint4*>(p.residual) + at) : make_uint4(0u, 0u, 0u, 0u), ds);
#pragma unroll
          for (int j = 0; j < N; ++j) {
            if (!kLean) w[j] = held[u][j];
            const float hj = (h[j] - in.mean[q]) * in.rstd[q];
            g[j] = fmaf(in.rstd[q], fmaf(g[j], w[j], -ma) - hj * mah, ds[j]);
          }
          static_cast<uint4*>(p.Y)[at] = Pack<T>::pack(g);
        }
      }
    }
  }
  if (!p.part) return;
  constexpr int kSpan = kTpr * kWords * N;
  if (kGroups > 1) {                             // the block's groups, in order
#pragma unroll
    for (int u = 0; u < kWords; ++u)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        join[(grp * 2) * kSpan + (c + u * kTpr) * N + j] = dw[u][j];
        join[(grp * 2 + 1) * kSpan + (c + u * kTpr) * N + j] = db[u][j];
      }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * kSpan; i += kThreads) {
      float s = 0.f;
      for (int g = 0; g < kGroups; ++g) s += join[g * 2 * kSpan + i];
      const int col = i % kSpan;
      if (col < p.d) p.part[(static_cast<long long>(blockIdx.x) * 2 + i / kSpan) * p.d + col] = s;
    }
  } else {
#pragma unroll
    for (int u = 0; u < kWords; ++u) {
      const int i = c + u * kTpr;
      if (i < p.words) {
        float* out = p.part + static_cast<long long>(blockIdx.x) * 2 * p.d + i * N;
#pragma unroll
        for (int j = 0; j < N; j += 4) {
          *reinterpret_cast<float4*>(out + j) = make_float4(dw[u][j], dw[u][j + 1], dw[u][j + 2], dw[u][j + 3]);
          *reinterpret_cast<float4*>(out + p.d + j) = make_float4(db[u][j], db[u][j + 1], db[u][j + 2], db[u][j + 3]);
        }
      }
    }
  }
}

// dw and db from the blocks' partials: 32 slices of the blocks, each added in order, then the slices four by eight.
constexpr int kSumSlices = 32, kSumCols = 8;

__device__ __forceinline__ void add4(float4& a, const float4& v) {
  a.x += v.x;
  a.y += v.y;
  a.z += v.z;
  a.w += v.w;
}

__global__ void __launch_bounds__(kSumSlices * kSumCols) k_norm_sum(const NormParams p) {
  __shared__ float4 slice[kSumSlices][kSumCols];
  pdl_wait();
  pdl_trigger();
  const int col = threadIdx.x % kSumCols, sl = threadIdx.x / kSumCols;
  const int n = p.d / 2;                         // float4 columns of [dw | db], a multiple of 4
  const int i = blockIdx.x * kSumCols + col;
  const int b0 = sl * p.blocks / kSumSlices, b1 = (sl + 1) * p.blocks / kSumSlices;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  if (i < n) {
    constexpr int kU = 10;                       // all of a slice in flight (304 blocks)
    for (int b = b0; b < b1; b += kU) {
      float4 v[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (b + u < b1) v[u] = __ldcg(reinterpret_cast<const float4*>(p.part) + static_cast<long long>(b + u) * n + i);
      }
#pragma unroll
      for (int u = 0; u < kU; ++u) add4(a, v[u]);
    }
  }
  slice[sl][col] = a;
  __syncthreads();
  if (sl < 4) {
    a = slice[sl * 8][col];
#pragma unroll
    for (int q = 1; q < 8; ++q) add4(a, slice[sl * 8 + q][col]);
  }
  __syncthreads();
  if (sl < 4) slice[sl][col] = a;
  __syncthreads();
  if (sl != 0 || i >= n) return;
#pragma unroll
  for (int q = 1; q < 4; ++q) add4(a, slice[q][col]);
  float* to = i < p.d / 4 ? p.dw : p.db;
  if (!to) return;
  float4* out = reinterpret_cast<float4*>(to) + (i < p.d / 4 ? i : i - p.d / 4);
  if (p.accumulate) {
    const float4 o = *out;
    a = make_float4(a.x + o.x, a.y + o.y, a.z + o.z, a.w + o.w);
  }
  *out = a;
}

// Blocks of the backward: two per SM, what the device holds at once of rows of at most 512 words (with three or four the second
// round is a short one: 16384 x 2048 53.4 and 47.6 us instead of 44.7), fewer where the partials would weigh against the rows
// (4091 x 512 in fp32 with the sums over the blocks: 8.6 us with one block per SM, 9.7 with two). Of longer rows an SM holds one
// block, so two per SM are two rounds of half the rows each, with twice the partials; the rule was measured at 512 and 2048
// features only.
int norm_blocks(int n_sms, int T) { return T >= 32 * n_sms ? 2 * n_sms : std::max(1, std::min(n_sms, (T + 7) / 8)); }

template <class T, int kTpr, int kWords, int kThreads>
cudaError_t forward(const NormParams& p, cudaStream_t s) {
  const int rows = kThreads / kTpr;
  return launch_pdl(k_norm_fwd<T, kTpr, kWords, kThreads>, dim3((p.T + rows - 1) / rows), dim3(kThreads), 0, s, p);
}

template <class T>
cudaError_t launch_forward(const NormParams& p, cudaStream_t s) {
  if (p.words <= 32) return forward<T, 32, 1, 256>(p, s);
  if (p.words <= 64) return forward<T, 32, 2, 256>(p, s);
  if (p.words <= 128) return forward<T, 32, 4, 256>(p, s);
  if (p.words <= 256) return forward<T, 32, 8, 256>(p, s);
  if (p.words <= 1024) return forward<T, 128, 8, 128>(p, s);
  return forward<T, 256, 8, 256>(p, s);
}

template <class T, int kTpr, int kWords, int kRows, int kThreads, int kBlocks = 2>
cudaError_t backward(NormParams p, cudaStream_t s) {
  const size_t smem = kThreads > kTpr ? sizeof(float) * 2 * (kThreads / kTpr) * kTpr * kWords * Pack<T>::N : 0;
  return launch_pdl(k_norm_bwd<T, kTpr, kWords, kRows, kThreads, kBlocks>, dim3(p.blocks), dim3(kThreads), smem, s, p);
}

template <class T>
cudaError_t launch_backward(const NormParams& p, cudaStream_t s) {
  if (p.words <= 8) return backward<T, 8, 1, 2, 256>(p, s);
  if (p.words <= 32) return backward<T, 32, 1, 2, 256>(p, s);
  if (p.words <= 64) return backward<T, 64, 1, 2, 256>(p, s);
  if (p.words <= 128) return backward<T, 128, 1, 2, 256>(p, s);
  if (p.words <= 256) return backward<T, 128, 2, 1, 256>(p, s);
  if (p.words <= 512) return backward<T, 256, 2, 1, 256>(p, s);
  if (p.words <= 1024) return backward<T, 512, 2, 1, 512, 1>(p, s);
  return backward<T, 1024, 2, 1, 1024, 1>(p, s);
}

bool aligned(const void* a) { return (reinterpret_cast<uintptr_t>(a) & 15u) == 0; }
template <class... Ptrs>
bool all_aligned(Ptrs... ptrs) { return (aligned(ptrs) && ...); }

NormParams params(const smoes_norm_s* P) {
  NormParams p{};
  p.T = P->desc.T;
  p.d = P->desc.d;
  p.words = P->desc.d / (P->desc.dtype == SMOES_BF16 ? 8 : 4);
  p.eps = P->desc.eps;
  p.inv_d = 1.f / static_cast<float>(P->desc.d);
  return p;
}

}  // namespace
}  // namespace smoes

extern "C" {

smoes_status smoes_norm_create(const smoes_norm_desc* desc, smoes_norm* out) {
  if (!desc || !out) return SMOES_ERR_INVALID_ARG;
  *out = nullptr;
  const smoes_norm_desc& d = *desc;
  if (d.dtype != SMOES_F32 && d.dtype != SMOES_BF16) return SMOES_ERR_INVALID_ARG;
  if (d.T < 0 || d.d < 1 || d.d % 8 != 0 || !(d.eps >= 0.f) || !(d.eps < 1e30f)) return SMOES_ERR_INVALID_ARG;
  if (d.T > (1 << 20) || d.d / (d.dtype == SMOES_BF16 ? 8 : 4) > kNormWordsMax) return SMOES_ERR_UNSUPPORTED;
  smoes_norm_s* P = new (std::nothrow) smoes_norm_s();
  if (!P) return SMOES_ERR_INVALID_ARG;
  P->desc = d;
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) == cudaSuccess &&
      cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && n > 0)
    P->n_sms = n;
  P->ws_bytes = sizeof(float) * 2 * static_cast<size_t>(norm_blocks(P->n_sms, d.T)) * d.d;
  *out = P;
  return SMOES_OK;
}

void smoes_norm_destroy(smoes_norm P) { delete P; }

size_t smoes_norm_workspace_bytes(smoes_norm P) { return P ? P->ws_bytes : 0; }

smoes_status smoes_norm_fwd(smoes_norm P, const void* X, const void* residual, const float* w, const float* b, void* S,
                            void* Y, float* mean, float* rstd, cudaStream_t stream) {
  if (!P || (residual != nullptr) != (S != nullptr) || (mean != nullptr) != (rstd != nullptr)) return SMOES_ERR_INVALID_ARG;
  if (P->desc.T == 0) return SMOES_OK;
  if (!X || !w || !Y) return SMOES_ERR_INVALID_ARG;
  if (!all_aligned(X, residual, w, b, S, Y, mean, rstd)) return SMOES_ERR_ALIGNMENT;
  NormParams p = params(P);
  p.X = X;
  p.residual = residual;
  p.w = w;
  p.b = b;
  p.S = S;
  p.Y = Y;
  p.mean = mean;
  p.rstd = rstd;
  const cudaError_t e = P->desc.dtype == SMOES_BF16 ? launch_forward<__nv_bfloat16>(p, stream)
                                                    : launch_forward<float>(p, stream);
  return e == cudaSuccess ? SMOES_OK : SMOES_ERR_CUDA;
}

smoes_status smoes_norm_bwd(smoes_norm P, const void* dY, const void* S, const float* mean, const float* rstd,
                            const float* w, const void* residual, void* dX, float* dw, float* db, int accumulate,
                            void* ws, size_t ws_bytes, cudaStream_t stream) {
  if (!P) return SMOES_ERR_INVALID_ARG;
  if (!all_aligned(dw, db)) return SMOES_ERR_ALIGNMENT;
  const bool sums = dw || db;
  if (P->desc.T == 0) {
    cudaError_t e = cudaSuccess;
    for (float* g : {dw, db})
      if (g && !accumulate && e == cudaSuccess) e = cudaMemsetAsync(g, 0, sizeof(float) * P->desc.d, stream);
    return e == cudaSuccess ? SMOES_OK : SMOES_ERR_CUDA;
  }
  if (!dY || !S || !mean || !rstd || !w || !dX) return SMOES_ERR_INVALID_ARG;
  if (sums && (!ws || ws_bytes < P->ws_bytes)) return SMOES_ERR_WORKSPACE;
  if (!all_aligned(dY, S, mean, rstd, w, residual, dX, ws)) return SMOES_ERR_ALIGNMENT;
  NormParams p = params(P);
  p.dY = dY;
  p.X = S;
  p.mean = const_cast<float*>(mean);
  p.rstd = const_cast<float*>(rstd);
  p.w = w;
  p.residual = residual;
  p.Y = dX;
  p.dw = dw;
  p.db = db;
  p.accumulate = accumulate ? 1 : 0;
  p.part = sums ? static_cast<float*>(ws) : nullptr;
  p.blocks = norm_blocks(P->n_sms, P->desc.T);
  cudaError_t e = P->desc.dtype == SMOES_BF16 ? launch_backward<__nv_bfloat16>(p, stream) : launch_backward<float>(p, stream);
  if (e == cudaSuccess && sums)
    e = launch_pdl(k_norm_sum, dim3((p.d / 2 + kSumCols - 1) / kSumCols), dim3(kSumSlices * kSumCols), 0, stream, p);
  return e == cudaSuccess ? SMOES_OK : SMOES_ERR_CUDA;
}

}  // extern "C"
