// expert_act.cu -- gradient of the experts' activation and bias:
//   dz = dout act'(z), or gated dz_g = dout u act'(g), dz_u = dout act(g);   db_e = sum over e's rows of dz
//
// One pass over dOut and pre. The rows that there are fall into equal ranges, a block to each range and each
// 32 x 16 bytes of columns, three blocks an SM and all of them resident: a row per warp, three rows' loads in flight.
// Column sums stay in registers until the expert changes; then the eight warps' sums are added in order into the
// partial of (range, expert), and a second small kernel adds each expert's partials in order. Ranges and experts
// both only go up along the rows, so range + expert numbers the partials without gaps to search. No range is empty: the
// second kernel adds every partial between an expert's first range and its last.
//
// Bound by HBM and by issue slots in about equal parts. 30035 x 704 gated: 40 us in bf16 (floor 31; a block per 32 rows, with
// the activation chosen at run time, 57-61), 74 in fp32 with CUDA's accurate functions (floor 62).
#include "experts.cuh"
#include "ptx.cuh"

namespace smoes {
namespace {

constexpr int kActThreads = 256;
constexpr int kActWarps = kActThreads / 32;
constexpr int kActRows = 3;                      // rows a warp has in flight

// Ranges over n rows: the launch's, but a row each at least (its count is of the plan's rows; dropped selections have none).
__device__ __forceinline__ int row_ranges(const ExpertActParams& p, long long n) {
  return n < p.ranges ? static_cast<int>(n) : p.ranges;
}
// First row of range i of `ranges` over n rows.
__device__ __forceinline__ long long range_begin(long long n, int ranges, int i) { return n * i / ranges; }

template <class T, int kAct, bool kGated>
__global__ void __launch_bounds__(kActThreads, kActBlocksPerSm) k_act_bwd(const ExpertActParams p) {
  constexpr int N = Pack<T>::N;
  constexpr bool kFast = sizeof(T) == 2;
  constexpr bool kSumsOnly = kAct == SMOES_ACT_NONE && !kGated;   // dz is dout
  __shared__ float sum_s[kGated ? 2 : 1][kActWarps][32 * N];
  pdl_wait();
  pdl_trigger();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long n = expert_begin(p.offsets, p.E, p.R);
  if (!kSumsOnly) zero_rows(p.dZ, n, p.R, p.n_z / N);
  const int segment = blockIdx.x / p.ranges, range = blockIdx.x - segment * p.ranges, ranges = row_ranges(p, n);
  if (range >= ranges) return;
  const long long end = range_begin(n, ranges, range + 1);
  long long row = range_begin(n, ranges, range);
  const int c0 = (segment * 32 + lane) * N;              // column of dOut (and of g or z)
  const bool in = c0 < p.n_out;
  const T* dout = static_cast<const T*>(p.dOut) + c0;
  const T* pre = static_cast<const T*>(p.pre) + c0;
  T* dz = static_cast<T*>(p.dZ) + c0;
  // the expert of the first row: the last one that begins at or before it
  int e = 0;
  if (p.db) {
    int last = 0;
    for (int i = lane; i < p.E; i += 32)
      if (expert_begin(p.offsets, i, p.R) <= row) last = i;
    e = __reduce_max_sync(0xffffffffu, last);
  }
  while (row < end) {
    // the rows of one expert in this range (without a bias gradient: all of them)
    const long long stop = p.db ? max(row + 1, min(end, expert_begin(p.offsets, e + 1, p.R))) : end;
    float sg[N], su[N];
#pragma unroll
    for (int x = 0; x < N; ++x) sg[x] = su[x] = 0.f;
    if (in) {
      for (long long r0 = row + warp; r0 < stop; r0 += kActWarps * kActRows) {
        uint4 d4[kActRows], z4[kActRows], u4[kActRows];  // every load of the warp's rows before the first use
#pragma unroll
        for (int j = 0; j < kActRows; ++j) {
          const long long r = r0 + j * kActWarps;
          if (r >= stop) break;
          d4[j] = __ldg(reinterpret_cast<const uint4*>(dout + r * p.n_out));
          if (!kSumsOnly) z4[j] = __ldg(reinterpret_cast<const uint4*>(pre + r * p.n_z));
          if (kGated) u4[j] = __ldg(reinterpret_cast<const uint4*>(pre + r * p.n_z + p.n_out));
        }
#pragma unroll
        for (int j = 0; j < kActRows; ++j) {
          const long long r = r0 + j * kActWarps;
          if (r >= stop) break;
          float d[N], z[N], u[N], o[N];
          Pack<T>::unpack(d4[j], d);
          if (!kSumsOnly) Pack<T>::unpack(z4[j], z);
          if (kGated) Pack<T>::unpack(u4[j], u);
#pragma unroll
          for (int x = 0; x < N; ++x) {
            if (!kSumsOnly) {
              float value, slope;
              act_value_slope<kAct, kFast>(z[x], value, slope);
              if (kGated) {
                o[x] = d[x] * value;
                su[x] += o[x];
                d[x] *= u[x];
              }
              d[x] *= slope;
            }
            sg[x] += d[x];
          }
          if (!kSumsOnly) *reinterpret_cast<uint4*>(dz + r * p.n_z) = Pack<T>::pack(d);
          if (kGated) *reinterpret_cast<uint4*>(dz + r * p.n_z + p.n_out) = Pack<T>::pack(o);
        }
      }
    }
    if (p.db) {
#pragma unroll
      for (int x = 0; x < N; ++x) {
        sum_s[0][warp][lane * N + x] = sg[x];
        if (kGated) sum_s[kGated ? 1 : 0][warp][lane * N + x] = su[x];
      }
      __syncthreads();
      float* part = p.part + static_cast<long long>(range + e) * p.n_z;
      for (int x = threadIdx.x; x < (kGated ? 64 * N : 32 * N); x += kActThreads) {
        const int half = x / (32 * N), y = x - half * 32 * N, c = segment * 32 * N + y;
        if (c >= p.n_out) continue;
        float a = 0.f;
#pragma unroll
        for (int w = 0; w < kActWarps; ++w) a += sum_s[half][w][y];
        part[half * p.n_out + c] = a;
      }
      __syncthreads();                                   // sum_s is free again
    }
    row = stop;
    if (p.db)                                            // the next expert that has rows
      while (e + 1 < p.E && expert_begin(p.offsets, e + 1, p.R) <= row) ++e;
  }
}

// db_e = the sum of e's partials: 128 columns a block, warp w adds the partials of the expert's ranges w, w + 8, ...,
// then the warps' sums in order.
__global__ void __launch_bounds__(kActThreads) k_act_bias(const ExpertActParams p) {
  __shared__ float4 sum_s[kActWarps][32];
  pdl_wait();
  pdl_trigger();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int e = blockIdx.y, c = (blockIdx.x * 32 + lane) * 4;
  const long long n = expert_begin(p.offsets, p.E, p.R);
  const long long r0 = expert_begin(p.offsets, e, p.R), r1 = min(n, expert_begin(p.offsets, e + 1, p.R));
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  if (r0 < r1 && c < p.n_z) {
    // the range of row r: the last one that begins at or before it
    const int ranges = row_ranges(p, n);
    int lo = static_cast<int>(r0 * ranges / n), hi = static_cast<int>((r1 - 1) * ranges / n);
    while (lo + 1 < ranges && range_begin(n, ranges, lo + 1) <= r0) ++lo;
    while (hi + 1 < ranges && range_begin(n, ranges, hi + 1) <= r1 - 1) ++hi;
#pragma unroll 8
    for (int i = lo + warp; i <= hi; i += kActWarps) {
      const float4 v = __ldcg(reinterpret_cast<const float4*>(p.part + static_cast<long long>(i + e) * p.n_z + c));
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
    float4* db = reinterpret_cast<float4*>(p.db + static_cast<long long>(e) * p.n_z + c);
    if (p.accumulate) {
      const float4 v = *db;
      a.x += v.x;
      a.y += v.y;
      a.z += v.z;
      a.w += v.w;
    }
    *db = a;
  }
}

template <class T>
cudaError_t launch_act(const ExpertActParams& p, int segments, cudaStream_t s) {
  return with_act(p.act, [&](auto act) {
    constexpr int kAct = decltype(act)::value;
    const dim3 grid(static_cast<unsigned>(p.ranges) * segments);
    return p.gated ? launch_pdl(k_act_bwd<T, kAct, true>, grid, dim3(kActThreads), 0, s, p)
                   : launch_pdl(k_act_bwd<T, kAct, false>, grid, dim3(kActThreads), 0, s, p);
  });
}

}  // namespace

// Ranges at most: what the device holds at once over one segment of columns.
int act_ranges(int n_sms) { return kActBlocksPerSm * n_sms; }

cudaError_t launch_expert_act_bwd(ExpertActParams p, bool bf16, int n_sms, cudaStream_t s) {
  const int per = bf16 ? 256 : 128, segments = (p.n_out + per - 1) / per;
  // as many blocks as are resident at once, but a warp's row each at least
  const long long most = (p.R + kActWarps - 1) / kActWarps;
  p.ranges = act_ranges(n_sms) / segments;
  if (p.ranges > most) p.ranges = static_cast<int>(most);
  if (p.ranges < 1) p.ranges = 1;
  cudaError_t e = bf16 ? launch_act<__nv_bfloat16>(p, segments, s) : launch_act<float>(p, segments, s);
  if (e == cudaSuccess && p.db)
    e = launch_pdl(k_act_bias, dim3((p.n_z + 127) / 128, p.E), dim3(kActThreads), 0, s, p);
  return e;
}

}  // namespace smoes
