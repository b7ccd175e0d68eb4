// expert_act.cu -- gradient of the experts' activation and bias:
//   dz = dout act'(z), or gated dz_g = dout u act'(g), dz_u = dout act(g);   db_e = sum over e's rows of dz
//
// One pass over dOut and pre. A block takes a chunk of at most 256 rows of one expert and 32 x 16 bytes
// of columns: a row per warp, then the eight warps' column sums are added in order into one partial
// per chunk; a second small kernel adds each expert's partials in order. Bound by HBM.
#include "experts.cuh"
#include "ptx.cuh"

namespace smoes {
namespace {

constexpr int kActThreads = 256;
constexpr int kActWarps = kActThreads / 32;

template <class T>
__global__ void __launch_bounds__(kActThreads) k_act_bwd(const ExpertActParams p) {
  constexpr int N = Pack<T>::N;
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
    for (long long r = t.row0 + warp; r < end; r += kActWarps) {
      float d[N], z[N], u[N], o[N];
      Pack<T>::unpack(__ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(p.dOut) + r * p.n_out + c0)), d);
      if (!p.dZ) {
#pragma unroll
        for (int i = 0; i < N; ++i) sg[i] += d[i];
        continue;
      }
      const T* pre = static_cast<const T*>(p.pre) + r * p.n_z + c0;
      T* dz = static_cast<T*>(p.dZ) + r * p.n_z + c0;
      Pack<T>::unpack(__ldg(reinterpret_cast<const uint4*>(pre)), z);
      if (p.gated) {
        Pack<T>::unpack(__ldg(reinterpret_cast<const uint4*>(pre + p.n_out)), u);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          o[i] = d[i] * act_value(p.act, z[i]);
          su[i] += o[i];
          d[i] *= u[i];
        }
        *reinterpret_cast<uint4*>(dz + p.n_out) = Pack<T>::pack(o);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        o[i] = d[i] * act_slope(p.act, z[i]);
        sg[i] += o[i];
      }
      *reinterpret_cast<uint4*>(dz) = Pack<T>::pack(o);
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

// db_e = the sum of e's partials, in row order.
__global__ void __launch_bounds__(kActThreads) k_act_bias(const ExpertActParams p) {
  pdl_wait();
  pdl_trigger();
  const int e = blockIdx.y, c = blockIdx.x * kActThreads + threadIdx.x;
  long long first = 0;                                   // the expert's first chunk
  for (int i = 0; i < e; ++i) {
    const long long rows = expert_begin(p.offsets, i + 1, p.R) - expert_begin(p.offsets, i, p.R);
    if (rows > 0) first += (rows + kActChunk - 1) / kActChunk;
  }
  const long long rows = expert_begin(p.offsets, e + 1, p.R) - expert_begin(p.offsets, e, p.R);
  long long n = rows > 0 ? (rows + kActChunk - 1) / kActChunk : 0;
  n = min(n, p.R / kActChunk + p.E - first);             // the partials there are room for
  if (c >= p.n_z) return;
  float a = 0.f;
#pragma unroll 8
  for (long long i = 0; i < n; ++i) a += __ldcg(p.part + (first + i) * p.n_z + c);
  p.db[static_cast<long long>(e) * p.n_z + c] = a;
}

}  // namespace

cudaError_t launch_expert_act_bwd(const ExpertActParams& p, bool bf16, cudaStream_t s) {
  const int per = bf16 ? 256 : 128;
  const long long chunks = p.R / kActChunk + (p.R < p.E ? p.R : p.E);
  const dim3 grid(static_cast<unsigned>(chunks), static_cast<unsigned>((p.n_out + per - 1) / per));
  cudaError_t e = bf16 ? launch_pdl(k_act_bwd<__nv_bfloat16>, grid, dim3(kActThreads), 0, s, p)
                       : launch_pdl(k_act_bwd<float>, grid, dim3(kActThreads), 0, s, p);
  if (e == cudaSuccess && p.db)
    e = launch_pdl(k_act_bias, dim3((p.n_z + kActThreads - 1) / kActThreads, p.E), dim3(kActThreads), 0, s, p);
  return e;
}

}  // namespace smoes
