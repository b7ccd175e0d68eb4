// expert_act.cu -- gradient of the experts' activation and bias:
//   dz = dout act'(z), or gated dz_g = dout u act'(g), dz_u = dout act(g);   db_e = sum over e's rows of dz
//
// One pass over dOut and pre. An item is a chunk of at most 32 rows of one expert by 32 x 16 bytes of columns, four
// rows a warp with all their loads in flight; the eight warps' column sums are added in order into one partial per
// chunk, while the loads of the block's next item are on their way, and a second small kernel adds each expert's
// partials in a fixed order. Bound by HBM. A block per item took 61 us for 30035 x 704 gated (floor 31): most of its
// life went into the launch and the search for its rows.
#include "experts.cuh"
#include "ptx.cuh"

namespace smoes {
namespace {

constexpr int kActThreads = 256;
constexpr int kActWarps = kActThreads / 32;
constexpr int kActRows = 4;                      // rows a warp has in flight

struct ActItem {
  long long row0, end;
  int chunk, c0;             // column of dOut (and of g or z)
  bool in;                   // this thread has columns
};

template <class T>
struct ActLoads {
  uint4 d[kActRows], z[kActRows], u[kActRows];
  __device__ __forceinline__ void load(const ExpertActParams& p, const ActItem& it, int warp) {
#pragma unroll
    for (int j = 0; j < kActRows; ++j) {
      const long long r = it.row0 + warp + j * kActWarps;
      d[j] = z[j] = u[j] = make_uint4(0u, 0u, 0u, 0u);
      if (!it.in || r >= it.end) continue;
      d[j] = __ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(p.dOut) + r * p.n_out + it.c0));
      if (!p.dZ) continue;
      const T* pre = static_cast<const T*>(p.pre) + r * p.n_z + it.c0;
      z[j] = __ldg(reinterpret_cast<const uint4*>(pre));
      if (p.gated) u[j] = __ldg(reinterpret_cast<const uint4*>(pre + p.n_out));
    }
  }
};

template <class T>
__global__ void __launch_bounds__(kActThreads, 2) k_act_bwd(const ExpertActParams p) {
  constexpr int N = Pack<T>::N;
  constexpr bool kFast = sizeof(T) == 2;
  __shared__ float sum_s[2][kActWarps][32 * N];
  pdl_wait();
  pdl_trigger();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const RowTiles tiles = count_row_tiles(p.offsets, p.E, p.R, kActChunk);
  const int segments = (p.n_out + 32 * N - 1) / (32 * N);
  const long long items = static_cast<long long>(tiles.total) * segments;
  auto item_of = [&](long long i) {
    ActItem it{0, 0, 0, 0, false};
    if (i >= items) return it;
    it.chunk = static_cast<int>(i / segments);
    it.c0 = (static_cast<int>(i - static_cast<long long>(it.chunk) * segments) * 32 + lane) * N;
    const RowTile t = find_row_tile(tiles, p.offsets, p.E, p.R, kActChunk, it.chunk);
    it.row0 = t.row0;
    it.end = min(t.row0 + kActChunk, t.row1);
    it.in = it.c0 < p.n_out;
    return it;
  };
  ActItem it = item_of(blockIdx.x);
  ActLoads<T> v;
  v.load(p, it, warp);
  if (p.dZ) zero_rows(p.dZ, expert_begin(p.offsets, p.E, p.R), p.R, p.n_z / N);
  for (long long i = blockIdx.x; i < items; i += gridDim.x) {
    float sg[N], su[N];
#pragma unroll
    for (int x = 0; x < N; ++x) sg[x] = su[x] = 0.f;
#pragma unroll
    for (int j = 0; j < kActRows; ++j) {
      const long long r = it.row0 + warp + j * kActWarps;
      if (!it.in || r >= it.end) continue;
      float d[N], z[N], u[N], o[N];
      Pack<T>::unpack(v.d[j], d);
      if (!p.dZ) {
#pragma unroll
        for (int x = 0; x < N; ++x) sg[x] += d[x];
        continue;
      }
      Pack<T>::unpack(v.z[j], z);
      Pack<T>::unpack(v.u[j], u);
      T* dz = static_cast<T*>(p.dZ) + r * p.n_z + it.c0;
#pragma unroll
      for (int x = 0; x < N; ++x) {
        float value, slope;
        act_value_slope<kFast>(p.act, z[x], value, slope);
        o[x] = d[x] * value;
        if (p.gated) d[x] *= u[x];
        z[x] = d[x] * slope;
      }
      if (p.gated) {
#pragma unroll
        for (int x = 0; x < N; ++x) su[x] += o[x];
        *reinterpret_cast<uint4*>(dz + p.n_out) = Pack<T>::pack(o);
      }
#pragma unroll
      for (int x = 0; x < N; ++x) sg[x] += z[x];
      *reinterpret_cast<uint4*>(dz) = Pack<T>::pack(z);
    }
    const ActItem next = item_of(i + gridDim.x);
    v.load(p, next, warp);
    if (p.db) {
      __syncthreads();                                   // the sums of the item before have been read
#pragma unroll
      for (int x = 0; x < N; ++x) {
        sum_s[0][warp][lane * N + x] = sg[x];
        sum_s[1][warp][lane * N + x] = su[x];
      }
      __syncthreads();
      float* part = p.part + static_cast<long long>(it.chunk) * p.n_z;
      const int col0 = it.c0 - lane * N;
      for (int x = threadIdx.x; x < (p.gated ? 64 * N : 32 * N); x += kActThreads) {
        const int half = x / (32 * N), y = x - half * 32 * N, c = col0 + y;
        if (c >= p.n_out) continue;
        float a = 0.f;
#pragma unroll
        for (int w = 0; w < kActWarps; ++w) a += sum_s[half][w][y];
        part[half * p.n_out + c] = a;
      }
    }
    it = next;
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

cudaError_t launch_expert_act_bwd(const ExpertActParams& p, bool bf16, int n_sms, cudaStream_t s) {
  const int per = bf16 ? 256 : 128;
  // items at most: whole chunks, and one that is not per expert
  const long long items = (p.R / kActChunk + (p.R < p.E ? p.R : p.E)) * ((p.n_out + per - 1) / per);
  const dim3 grid(static_cast<unsigned>(items < 2ll * n_sms ? items : 2ll * n_sms));
  cudaError_t e = bf16 ? launch_pdl(k_act_bwd<__nv_bfloat16>, grid, dim3(kActThreads), 0, s, p)
                       : launch_pdl(k_act_bwd<float>, grid, dim3(kActThreads), 0, s, p);
  if (e == cudaSuccess && p.db)
    e = launch_pdl(k_act_bias, dim3((p.n_z + 127) / 128, p.E), dim3(kActThreads), 0, s, p);
  return e;
}

}  // namespace smoes
