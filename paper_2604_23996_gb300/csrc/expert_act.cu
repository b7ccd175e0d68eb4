// expert_act.cu -- gradient of the experts' activation and bias:
//   dz = dout act'(z), or gated dz_g = dout u act'(g), dz_u = dout act(g);   db_e = sum over e's rows of dz
//
// One pass over dOut and pre. A block takes a chunk of at most 64 rows of one expert and 32 x 16 bytes
// of columns, four rows' loads in flight a warp; the eight warps' column sums are added in order into
// one partial per chunk, and a second small kernel adds each expert's partials in a fixed order. Bound by HBM.
// With chunks of 256 rows, CUDA's accurate functions and two exponentials a value, 30035 x 704 gated took
// 116 us.
#include "experts.cuh"
#include "ptx.cuh"

namespace smoes {
namespace {

constexpr int kActThreads = 256;
constexpr int kActWarps = kActThreads / 32;
constexpr int kActRows = 4;                      // rows a warp has in flight

template <class T>
__global__ void __launch_bounds__(kActThreads, 2) k_act_bwd(const ExpertActParams p) {
  constexpr int N = Pack<T>::N;
  constexpr bool kFast = sizeof(T) == 2;
  __shared__ float sum_s[2][kActWarps][32 * N];
  pdl_wait();
  pdl_trigger();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (p.dZ) zero_rows(p.dZ, expert_begin(p.offsets, p.E, p.R), p.R, p.n_z / N);
  const RowTile t = find_row_tile(p.offsets, p.E, p.R, kActChunk, blockIdx.x);
  if (t.e < 0) return;
  const int c0 = (blockIdx.y * 32 + lane) * N;           // column of dOut (and of g or z)
  const bool in = c0 < p.n_out;
  float sg[N], su[N];
#pragma unroll
  for (int i = 0; i < N; ++i) sg[i] = su[i] = 0.f;
  const long long end = min(t.row0 + kActChunk, t.row1);
  if (in) {
    for (long long r0 = t.row0 + warp; r0 < end; r0 += kActWarps * kActRows) {
      uint4 d4[kActRows], z4[kActRows], u4[kActRows];    // every load of the warp's rows before the first use
#pragma unroll
      for (int j = 0; j < kActRows; ++j) {
        const long long r = r0 + j * kActWarps;
        d4[j] = z4[j] = u4[j] = make_uint4(0u, 0u, 0u, 0u);
        if (r >= end) continue;
        d4[j] = __ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(p.dOut) + r * p.n_out + c0));
        if (!p.dZ) continue;
        const T* pre = static_cast<const T*>(p.pre) + r * p.n_z + c0;
        z4[j] = __ldg(reinterpret_cast<const uint4*>(pre));
        if (p.gated) u4[j] = __ldg(reinterpret_cast<const uint4*>(pre + p.n_out));
      }
#pragma unroll
      for (int j = 0; j < kActRows; ++j) {
        const long long r = r0 + j * kActWarps;
        if (r >= end) break;
        float d[N], z[N], u[N], o[N];
        Pack<T>::unpack(d4[j], d);
        if (!p.dZ) {
#pragma unroll
          for (int i = 0; i < N; ++i) sg[i] += d[i];
          continue;
        }
        Pack<T>::unpack(z4[j], z);
        Pack<T>::unpack(u4[j], u);
        T* dz = static_cast<T*>(p.dZ) + r * p.n_z + c0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          float value, slope;
          act_value_slope<kFast>(p.act, z[i], value, slope);
          o[i] = d[i] * value;
          if (p.gated) d[i] *= u[i];
          z[i] = d[i] * slope;
        }
        if (p.gated) {
#pragma unroll
          for (int i = 0; i < N; ++i) su[i] += o[i];
          *reinterpret_cast<uint4*>(dz + p.n_out) = Pack<T>::pack(o);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) sg[i] += z[i];
        *reinterpret_cast<uint4*>(dz) = Pack<T>::pack(z);
      }
    }
  }
  if (!p.db) return;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    sum_s[0][warp][lane * N + i] = sg[i];
    sum_s[1][warp][lane * N + i] = su[i];
  }
  __syncthreads();
  float* part = p.part + static_cast<long long>(blockIdx.x) * p.n_z;
  for (int i = threadIdx.x; i < (p.gated ? 64 * N : 32 * N); i += kActThreads) {
    const int half = i / (32 * N), j = i - half * 32 * N, c = blockIdx.y * 32 * N + j;
    if (c >= p.n_out) continue;
    float a = 0.f;
#pragma unroll
    for (int w = 0; w < kActWarps; ++w) a += sum_s[half][w][j];
    part[half * p.n_out + c] = a;
  }
}

// db_e = the sum of e's partials: 128 columns a block, warp w adds partials w, w + 8, ..., then the warps' sums
// in order.
__global__ void __launch_bounds__(kActThreads) k_act_bias(const ExpertActParams p) {
  __shared__ float4 sum_s[kActWarps][32];
  pdl_wait();
  pdl_trigger();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int e = blockIdx.y, c = (blockIdx.x * 32 + lane) * 4;
  // the expert's first chunk: the chunks of the experts before it, counted by the lanes of every warp
  int before = 0;
  for (int i = lane; i < e; i += 32) {
    const long long rows = expert_begin(p.offsets, i + 1, p.R) - expert_begin(p.offsets, i, p.R);
    if (rows > 0) before += static_cast<int>((rows + kActChunk - 1) / kActChunk);
  }
  const long long first = __reduce_add_sync(0xffffffffu, before);
  const long long rows = expert_begin(p.offsets, e + 1, p.R) - expert_begin(p.offsets, e, p.R);
  long long n = rows > 0 ? (rows + kActChunk - 1) / kActChunk : 0;
  n = min(n, p.R / kActChunk + p.E - first);             // the partials there are room for
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  if (c < p.n_z) {
#pragma unroll 8
    for (long long i = warp; i < n; i += kActWarps) {
      const float4 v = __ldcg(reinterpret_cast<const float4*>(p.part + (first + i) * p.n_z + c));
      a.x += v.x;
      a.y += v.y;
      a.z += v.z;
      a.w += v.w;
    }
  }
  sum_s[warp][lane] = a;
  __syncthreads();
  if (warp == 0 && c < p.n_z) {
    for (int w = 1; w < kActWarps; ++w) {
      const float4 v = sum_s[w][lane];
      a.x += v.x;
      a.y += v.y;
      a.z += v.z;
      a.w += v.w;
    }
    *reinterpret_cast<float4*>(p.db + static_cast<long long>(e) * p.n_z + c) = a;
  }
}

}  // namespace

cudaError_t launch_expert_act_bwd(const ExpertActParams& p, bool bf16, cudaStream_t s) {
  const int per = bf16 ? 256 : 128;
  const long long chunks = p.R / kActChunk + (p.R < p.E ? p.R : p.E);
  const dim3 grid(static_cast<unsigned>(chunks), static_cast<unsigned>((p.n_out + per - 1) / per));
  cudaError_t e = bf16 ? launch_pdl(k_act_bwd<__nv_bfloat16>, grid, dim3(kActThreads), 0, s, p)
                       : launch_pdl(k_act_bwd<float>, grid, dim3(kActThreads), 0, s, p);
  if (e == cudaSuccess && p.db)
    e = launch_pdl(k_act_bias, dim3((p.n_z + 127) / 128, p.E), dim3(kActThreads), 0, s, p);
  return e;
}

}  // namespace smoes
