// experts.cuh -- the expert layer: plan, kernel parameters and launchers shared by experts_api.cu and
// the kernels (expert_sort.cu, expert_rows.cu, expert_gemm.cu, expert_gemm_f32.cu, expert_act.cu).
#pragma once

#include <cuda_bf16.h>

#include <type_traits>

#include "smoes_internal.cuh"

namespace smoes {

constexpr int kExpertsMax = 256;           // experts of an expert-layer plan
constexpr int kExpertWidthMax = 1 << 20;   // widest row
constexpr int kActBlocksPerSm = 3;         // of the activation gradient, all at once

struct ExpertSortParams {
  long long n;               // selections T * k
  int E, G;                  // blocks
  long long per;             // selections per block, a multiple of 1024
  const int32_t* topk_idx;
  int32_t* offsets;
  int32_t* row_slot;
  int32_t* slot_row;
  int32_t* counts;           // [G][E] (workspace)
  uint32_t* sync;            // [2] grid barrier words (workspace, zero between calls)
  uint32_t* status;
  uint64_t limit_ns;
};

// dispatch, combine and their gradients: rows of `d` elements, T tokens of k selections
struct ExpertRowsParams {
  int T, k, d, E;
  const int32_t* offsets;    // [E+1], or null where no rows are written
  const int32_t* slot_row;   // [T, k]
  const void* tokens;        // X, dY or the residual (or null)
  const void* rows;          // Ys or dXs
  const float* w;            // [T, k] or null (1)
  void* rows_out;            // Xs or dYs
  void* tokens_out;          // Y or dX
  float* dw;                 // [T, k]
};

struct ExpertLinearParams {
  int E, n_in, n_out, n_z, act, gated;
  long long R;
  const int32_t* offsets;
  const void* X;
  const void* W;
  const float* bias;
  const void* residual;
  const void* dZ;
  void* out;                 // out, or dX
  void* pre;
  float* dW;
  int accumulate;
};

struct ExpertActParams {
  int E, n_out, n_z, act, gated;
  long long R;
  const int32_t* offsets;
  const void* dOut;
  const void* pre;
  void* dZ;
  float* db;
  int accumulate;            // db is added to
  int ranges;                // row ranges: one block each and per segment of columns
  float* part;               // [ranges + E][n_z] (workspace)
};

// The products on the tensor cores (expert_gemm.cu, expert_gemm_f32.cu): D[m, n] = sum over the depth of A[m] B[n], with
// the features of an output row along m and the rows along n (the weights' gradient: n_in along m, n_z
// along n, the expert's rows as the depth).
enum ExpertGemmMode { kGemmForward = 0, kGemmGradX = 1, kGemmGradW = 2 };
struct ExpertGemmParams {
  ExpertLinearParams l;
  int n_feat;                // features along m: n_out, or n_in
  int m_tiles;
  int tile_shift;            // log2 of a tile's rows (weights' gradient: its columns of n_z)
  int n_tiles;               // tiles along n_z (weights' gradient)
  uint32_t* status;
  uint64_t limit_ns;
};

cudaError_t launch_expert_gemm(const ExpertLinearParams& p, ExpertGemmMode mode, uint32_t* status, uint64_t limit_ns,
                               int n_sms, cudaStream_t s);
cudaError_t launch_expert_gemm_f32(const ExpertLinearParams& p, ExpertGemmMode mode, uint32_t* status, uint64_t limit_ns,
                                   int n_sms, cudaStream_t s);
cudaError_t launch_expert_sort(const ExpertSortParams& p, cudaStream_t s);
cudaError_t launch_expert_dispatch(const ExpertRowsParams& p, bool bf16, cudaStream_t s);
cudaError_t launch_expert_combine(const ExpertRowsParams& p, bool bf16, cudaStream_t s);
cudaError_t launch_expert_combine_bwd(const ExpertRowsParams& p, bool bf16, cudaStream_t s);
cudaError_t launch_expert_act_bwd(ExpertActParams p, bool bf16, int n_sms, cudaStream_t s);   // fills ranges
int act_ranges(int n_sms);   // most ranges of the activation gradient

// ------------------------------------------------------------------------------ device helpers

// First row of expert e, kept inside [0, R]; expert_rows: its rows (none where offsets run backwards).
__device__ __forceinline__ long long expert_begin(const int32_t* off, int e, long long R) {
  const long long o = off[e];
  return o < 0 ? 0 : o > R ? R : o;
}

// Work over the experts' rows in tiles of 2^shift rows, counted over the experts in order. Every warp that walks
// the tiles keeps the count before every eighth expert in its lanes; `off` is a copy of the offsets in shared memory. (R is
// at most 2^24; with 64-bit rows and a division by the tile the count and the search took some 2000 clocks a kernel and 600
// a tile.)
struct RowTile {
  int e;
  int row0, row1;            // the tile's first row, the expert's end
};
struct RowTiles {
  int before;                // lane l: tiles of the experts before 8 l
  int total;
};
__device__ __forceinline__ int expert_row(const int32_t* off, int e, int R) { return min(max(off[e], 0), R); }
__device__ __forceinline__ int row_tiles_of(const int32_t* off, int e, int E, int R, int shift) {
  if (e >= E) return 0;
  const int rows = expert_row(off, e + 1, R) - expert_row(off, e, R);
  return rows > 0 ? (rows + (1 << shift) - 1) >> shift : 0;
}
// The counts, by one warp from the offsets in global memory: lane l's to before[l], the total to before[32].
__device__ inline void count_row_tiles(const int32_t* offsets, int E, int R, int shift, int* before) {
  const int lane = threadIdx.x & 31;
  int o[9];
#pragma unroll
  for (int i = 0; i < 9; ++i) o[i] = min(max(__ldg(offsets + min(lane * 8 + i, E)), 0), R);   // (past E: no rows)
  int sum = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) sum += o[i + 1] > o[i] ? (o[i + 1] - o[i] + (1 << shift) - 1) >> shift : 0;
  int run = sum;
#pragma unroll
  for (int i = 1; i < 32; i <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, run, i);
    if (lane >= i) run += v;
  }
  before[lane] = run - sum;
  if (lane == 31) before[32] = run;
}
// Tile 0 <= tile < total, by a whole warp.
__device__ __forceinline__ RowTile find_row_tile(const RowTiles& t, const int32_t* off, int E, int R, int shift, int tile) {
  const int lane = threadIdx.x & 31;
  const int q = 31 - __clz(__ballot_sync(0xffffffffu, t.before <= tile));   // the last group that starts at or before it
  const int in = tile - __shfl_sync(0xffffffffu, t.before, q);
  const int n = lane < 8 ? row_tiles_of(off, q * 8 + lane, E, R, shift) : 0;
  int run = n;
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += v;
  }
  const int src = __ffs(__ballot_sync(0xffffffffu, lane < 8 && in < run)) - 1;
  RowTile r;
  r.e = q * 8 + src;
  r.row0 = expert_row(off, r.e, R) + ((in - __shfl_sync(0xffffffffu, run - n, src)) << shift);
  r.row1 = expert_row(off, r.e + 1, R);
  return r;
}

// 16 bytes of T: 8 bf16 or 4 fp32.
template <class T>
struct Pack;
template <>
struct Pack<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <>
struct Pack<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[4]) {
    f[0] = __uint_as_float(v.x);
    f[1] = __uint_as_float(v.y);
    f[2] = __uint_as_float(v.z);
    f[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};

// Zeros in rows [first, R) of an array of rows of `words` 16-byte words, by all threads of the grid.
__device__ __forceinline__ void zero_rows(void* base, long long first, long long R, int words) {
  uint4* out = static_cast<uint4*>(base);
  const long long end = R * words;
  for (long long i = first * words + static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x; i < end;
       i += static_cast<long long>(gridDim.x) * blockDim.x)
    out[i] = make_uint4(0u, 0u, 0u, 0u);
}

// Activations and their slopes. kFast: for results that are rounded to bf16, whose step is 2^-8: the fast
// exponential and reciprocal (a few steps of 2^-22; what underflows is zero), and erfc by the rational form of
// Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26 (absolute error 1.5e-7), which shares its
// e^(-z^2 / 2) with the slope (an epilogue with erfcf takes longer than the products it follows). Otherwise CUDA's
// accurate functions.
__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float fast_reciprocal(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr float kLog2E = 1.4426950408889634f;
template <bool kFast>
__device__ __forceinline__ float sigmoid_of(float z) {
  return kFast ? fast_reciprocal(1.f + fast_exp2(-kLog2E * z)) : 1.f / (1.f + expf(-z));
}
// The fast form's half - erfc(|z| / sqrt 2) / 2 (so that Phi = 0.5 +- it), and e^(-z^2 / 2).
__device__ __forceinline__ float fast_half_erf(float z, float& e) {
  const float w = z * 0.84932180f;                       // sqrt(log2(e) / 2)
  e = fast_exp2(-w * w);
  const float t = fast_reciprocal(fmaf(0.3275911f * 0.70710678f, fabsf(z), 1.f));
  float q = fmaf(0.5f * 1.061405429f, t, 0.5f * -1.453152027f);   // erfc(|z| / sqrt 2) / 2 = t q(t) e^(-z^2 / 2)
  q = fmaf(q, t, 0.5f * 1.421413741f);
  q = fmaf(q, t, 0.5f * -0.284496736f);
  q = fmaf(q, t, 0.5f * 0.254829592f);
  return fmaf(-q, t * e, 0.5f);
}
template <int kAct, bool kFast>
__device__ __forceinline__ float act_value(float z) {
  if (kAct == SMOES_ACT_SILU) return kFast ? z * sigmoid_of<true>(z) : z / (1.f + expf(-z));
  if (kAct == SMOES_ACT_GELU) {
    if (!kFast) return 0.5f * z * erfcf(z * -0.70710678f);
    float e;
    return fmaf(fabsf(z), fast_half_erf(z, e), 0.5f * z);
  }
  return z;
}
template <int kAct, bool kFast>
__device__ __forceinline__ void act_value_slope(float z, float& value, float& slope) {
  if (kAct == SMOES_ACT_SILU) {
    const float s = sigmoid_of<kFast>(z);
    value = z * s;
    slope = fmaf(value, 1.f - s, s);
  } else if (kAct == SMOES_ACT_GELU) {
    float e, n;                                          // e^(-z^2 / 2), Phi(z)
    if (kFast) {
      n = 0.5f + copysignf(fast_half_erf(z, e), z);
    } else {
      e = expf(-0.5f * z * z);
      n = 0.5f * erfcf(z * -0.70710678f);
    }
    value = z * n;
    slope = fmaf(z * 0.39894228f, e, n);
  } else {
    value = z;
    slope = 1.f;
  }
}
// f with the activation as a constant.
template <class F>
auto with_act(int act, F&& f) {
  if (act == SMOES_ACT_SILU) return f(std::integral_constant<int, SMOES_ACT_SILU>());
  if (act == SMOES_ACT_GELU) return f(std::integral_constant<int, SMOES_ACT_GELU>());
  return f(std::integral_constant<int, SMOES_ACT_NONE>());
}

}  // namespace smoes
