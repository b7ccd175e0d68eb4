// mx.cu -- microscaled 4-bit values: quantisation, its inverse, and the quantising copy of tokens into expert order.
//
// A block of 32 consecutive values shares the scale 2^(byte - 127), byte - 127 = max(floor(log2 max|x|) - 2, -127) (the
// largest 4-bit value, 6, is 1.5 x 2^2); a value over the scale is rounded to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to
// the even code), above 6 to 6. The quotient is exact in fp32 but where it is subnormal, far below 0.25: 0 either way. This is
// the microscaling formats' MXFP4, with the scale as their specification gives it. A block that holds a NaN or an infinity becomes NaN: scale byte 255, codes 0.
//
// A thread takes 8 consecutive values, four neighbouring threads a block, whose largest magnitude meets in two shuffles;
// the 4-byte words of a warp's codes are neighbours in memory. Every value is read once. Bound by HBM: 98304 x 1024 bf16
// quantised in 38.3 us (6.6 TB/s), 16384 x 2048 into 98304 rows in 29.4 us (5.9 TB/s, of codes mostly).
#include "experts.cuh"
#include "ptx.cuh"

namespace smoes {
namespace {

constexpr int kMxThreads = 256;
constexpr int kMxWords = 4;                      // of 8 values a thread

// 8 values of T as they lie in memory.
template <class T>
struct Eight;
template <>
struct Eight<__nv_bfloat16> {
  uint4 v;
  __device__ __forceinline__ void load(const void* p, long long i) { v = __ldg(static_cast<const uint4*>(p) + i); }
  __device__ __forceinline__ void zero() { v = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ void get(float (&f)[8]) const { Pack<__nv_bfloat16>::unpack(v, f); }
  static __device__ __forceinline__ void store(void* p, long long i, const float (&f)[8]) {
    static_cast<uint4*>(p)[i] = Pack<__nv_bfloat16>::pack(f);
  }
};
template <>
struct Eight<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const void* p, long long i) {
    a = __ldg(static_cast<const float4*>(p) + 2 * i);
    b = __ldg(static_cast<const float4*>(p) + 2 * i + 1);
  }
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
  static __device__ __forceinline__ void store(void* p, long long i, const float (&f)[8]) {
    static_cast<float4*>(p)[2 * i] = make_float4(f[0], f[1], f[2], f[3]);
    static_cast<float4*>(p)[2 * i + 1] = make_float4(f[4], f[5], f[6], f[7]);
  }
};

// The word of codes of a thread's 8 values and its block's scale byte; whole groups of four threads.
template <class T>
__device__ __forceinline__ uint32_t quantise(const Eight<T>& in, uint32_t& byte) {
  float f[8];
  in.get(f);
  uint32_t most = 0;                             // magnitudes compare as whole numbers, NaN above all
#pragma unroll
  for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(f[i]) & 0x7fffffffu);
  most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
  most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
  const uint32_t e = most >> 23;                 // exponent + 127 (0: below 2^-126)
  if (e == 255u) {
    byte = 255u;
    return 0u;
  }
  byte = e > 2u ? e - 2u : 0u;
  const float inv = __uint_as_float((254u - byte) << 23);   // 1 / scale: 2^-125 .. 2^127
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] *= inv;
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]));
  return r;
}

__device__ __forceinline__ float scale_of(uint32_t byte) {
  return __uint_as_float(byte == 0u ? 0x00400000u : byte == 255u ? 0x7fc00000u : byte << 23);
}

template <class T>
__global__ void __launch_bounds__(kMxThreads) k_mx_quantise(const void* X, long long words, uint32_t* q, uint8_t* scale) {
  pdl_wait();
  pdl_trigger();
  const long long i0 = static_cast<long long>(blockIdx.x) * (kMxThreads * kMxWords) + threadIdx.x;
  Eight<T> v[kMxWords];
#pragma unroll
  for (int u = 0; u < kMxWords; ++u) {
    const long long i = i0 + u * kMxThreads;
    if (i < words) v[u].load(X, i); else v[u].zero();
  }
#pragma unroll
  for (int u = 0; u < kMxWords; ++u) {
    const long long i = i0 + u * kMxThreads;
    uint32_t byte;
    const uint32_t r = quantise(v[u], byte);
    if (i < words) {
      q[i] = r;
      if ((threadIdx.x & 3) == 0) scale[i >> 2] = static_cast<uint8_t>(byte);
    }
  }
}

template <class T>
__global__ void __launch_bounds__(kMxThreads) k_mx_dequantise(const uint32_t* q, const uint8_t* scale, long long words, void* X) {
  pdl_wait();
  pdl_trigger();
  const long long i0 = static_cast<long long>(blockIdx.x) * (kMxThreads * kMxWords) + threadIdx.x;
  uint32_t c[kMxWords], b[kMxWords];
#pragma unroll
  for (int u = 0; u < kMxWords; ++u) {
    const long long i = i0 + u * kMxThreads;
    c[u] = i < words ? __ldg(q + i) : 0u;
    b[u] = i < words ? __ldg(scale + (i >> 2)) : 0u;
  }
#pragma unroll
  for (int u = 0; u < kMxWords; ++u) {
    const long long i = i0 + u * kMxThreads;
    const float s = scale_of(b[u]);
    uint32_t h[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(c[u]));
    float f[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&h[j]));
      f[2 * j] = p.x * s;
      f[2 * j + 1] = p.y * s;
    }
    if (i < words) Eight<T>::store(X, i, f);
  }
}

// A warp's unit of work: kMxWords words of 8 values a lane of one token, quantised once and written to the token's rows.
template <class T>
__global__ void __launch_bounds__(kMxThreads) k_dispatch_mx(const ExpertRowsParams p, int words, int units, uint8_t* scale) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const long long R = static_cast<long long>(p.T) * p.k;
  const long long unit = static_cast<long long>(blockIdx.x) * (kMxThreads / 32) + (threadIdx.x >> 5);
  uint32_t* q = static_cast<uint32_t*>(p.rows_out);
  if (unit < static_cast<long long>(p.T) * units) {
    const long long t = unit / units;
    const int w0 = static_cast<int>(unit - t * units) * (32 * kMxWords) + lane;
    int rows = lane < p.k ? __ldg(p.slot_row + t * p.k + lane) : -1;
    if (rows >= R) rows = -1;
    Eight<T> v[kMxWords];
#pragma unroll
    for (int u = 0; u < kMxWords; ++u)
      if (w0 + 32 * u < words) v[u].load(p.tokens, t * words + w0 + 32 * u); else v[u].zero();
    uint32_t r[kMxWords], byte[kMxWords];
#pragma unroll
    for (int u = 0; u < kMxWords; ++u) r[u] = quantise(v[u], byte[u]);
    for (int s = 0; s < p.k; ++s) {
      const int row = __shfl_sync(0xffffffffu, rows, s);
      if (row < 0) continue;
#pragma unroll
      for (int u = 0; u < kMxWords; ++u) {
        const int w = w0 + 32 * u;
        if (w < words) {
          q[static_cast<long long>(row) * words + w] = r[u];
          if ((lane & 3) == 0) scale[static_cast<long long>(row) * (words >> 2) + (w >> 2)] = static_cast<uint8_t>(byte[u]);
        }
      }
    }
  }
  const long long first = expert_begin(p.offsets, p.E, R);
  if (first >= R) return;
  zero_rows(p.rows_out, first, R, words / 4);
  for (long long i = first * (words >> 2) + static_cast<long long>(blockIdx.x) * kMxThreads + threadIdx.x; i < R * (words >> 2);
       i += static_cast<long long>(gridDim.x) * kMxThreads)
    scale[i] = 0;
}

dim3 mx_grid(long long words) {
  constexpr long long per = kMxThreads * kMxWords;
  return dim3(static_cast<unsigned>((words + per - 1) / per));
}

}  // namespace

cudaError_t launch_mx_quantise(const void* X, bool bf16, long long values, uint8_t* q, uint8_t* scale, cudaStream_t s) {
  const long long words = values / 8;
  return launch_pdl(bf16 ? k_mx_quantise<__nv_bfloat16> : k_mx_quantise<float>, mx_grid(words), dim3(kMxThreads), 0, s, X, words,
                    reinterpret_cast<uint32_t*>(q), scale);
}

cudaError_t launch_mx_dequantise(const uint8_t* q, const uint8_t* scale, long long values, bool bf16, void* X, cudaStream_t s) {
  const long long words = values / 8;
  return launch_pdl(bf16 ? k_mx_dequantise<__nv_bfloat16> : k_mx_dequantise<float>, mx_grid(words), dim3(kMxThreads), 0, s,
                    reinterpret_cast<const uint32_t*>(q), scale, words, X);
}

cudaError_t launch_expert_dispatch_mx(const ExpertRowsParams& p, bool bf16, uint8_t* scale, cudaStream_t s) {
  const int words = p.d / 8, units = (words + 32 * kMxWords - 1) / (32 * kMxWords);
  const long long warps = static_cast<long long>(p.T) * units;
  const dim3 grid(static_cast<unsigned>((warps + kMxThreads / 32 - 1) / (kMxThreads / 32)));
  return launch_pdl(bf16 ? k_dispatch_mx<__nv_bfloat16> : k_dispatch_mx<float>, grid, dim3(kMxThreads), 0, s, p, words, units, scale);
}

}  // namespace smoes
