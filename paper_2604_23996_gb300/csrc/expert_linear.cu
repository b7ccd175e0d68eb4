// expert_linear.cu -- the experts' fp32 products on the FMA units, grouped over ragged row ranges (bf16:
// expert_gemm.cu):
//   forward   z = X W_e^T + b_e, out = act(z) (or act(g) u of z = [g | u]) + residual
//   dX        dZ W_e
//   dW        dZ^T X over the expert's rows
//
// A block forms a 128 x 128 tile, 8 x 8 values a thread, from 16-deep slices of both operands held
// in shared memory as [depth][128]; the next slice is in registers while the present one is multiplied.
// Bound by the FMA rate.
#include "experts.cuh"
#include "ptx.cuh"

namespace smoes {
namespace {

constexpr int kTile = 128;
constexpr int kDepth = 16;
constexpr int kPad = kTile + 4;
constexpr int kLinThreads = 256;

enum LinearMode { kForward = 0, kGradX = 1, kGradW = 2 };

__device__ __forceinline__ float4 load4(const float* p) {
  return __ldg(reinterpret_cast<const float4*>(p));
}
__device__ __forceinline__ void store4(float* p, float a, float b, float c, float d) {
  *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
}

// One operand's slice in registers: along the depth (rows of `ld` elements, 8 of a row a thread) or
// across it (16 rows of the depth, 8 neighbouring columns a thread).
template <bool kAlong>
struct Slice {
  float4 v[2];
  // along: row `outer` (already this thread's; valid when in), depth d0.. < depth_end
  __device__ __forceinline__ void load_along(const float* row, bool in, long long d0, long long depth_end) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const long long d = d0 + (threadIdx.x & 1) * 8 + 4 * h;
      v[h] = in && d < depth_end ? load4(row + d) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }
  // across: base of depth row 0, columns c0 + ... < c_end
  __device__ __forceinline__ void load_across(const float* base, long long ld, long long d0, long long depth_end, int c0,
                                              int c_end) {
    const long long d = d0 + (threadIdx.x >> 4);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int c = c0 + (threadIdx.x & 15) * 4 + 64 * h;
      v[h] = d < depth_end && c < c_end ? load4(base + d * ld + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }
  __device__ __forceinline__ void store(float (*s)[kPad]) const {
    if (kAlong) {
      const int r = threadIdx.x >> 1, d = (threadIdx.x & 1) * 8;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        s[d + 4 * h][r] = v[h].x;
        s[d + 4 * h + 1][r] = v[h].y;
        s[d + 4 * h + 2][r] = v[h].z;
        s[d + 4 * h + 3][r] = v[h].w;
      }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        *reinterpret_cast<float4*>(&s[threadIdx.x >> 4][(threadIdx.x & 15) * 4 + 64 * h]) = v[h];
    }
  }
};

template <int kMode>
__global__ void __launch_bounds__(kLinThreads) k_expert_linear(const ExpertLinearParams p) {
  __shared__ float As[2][kDepth][kPad];
  __shared__ float Bs[2][kDepth][kPad];
  pdl_wait();
  pdl_trigger();
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const float* X = static_cast<const float*>(p.X);
  const float* W = static_cast<const float*>(p.W);
  const float* dZ = static_cast<const float*>(p.dZ);

  // the tile: rows [m0, m_end) of the product, columns from n0; the depth [k0, k_end)
  int e;
  long long m0, m_end, k0 = 0, k_end;
  int n0;
  if (kMode == kGradW) {
    e = blockIdx.z;
    m0 = static_cast<long long>(blockIdx.y) * kTile;
    m_end = p.n_z;
    n0 = blockIdx.x * kTile;
    k0 = expert_begin(p.offsets, e, p.R);
    k_end = max(k0, expert_begin(p.offsets, e + 1, p.R));
  } else {
    zero_rows(p.out, expert_begin(p.offsets, p.E, p.R), p.R,
              static_cast<int>((kMode == kForward ? p.n_out : p.n_in) * sizeof(float) / 16));
    if (kMode == kForward && p.pre)
      zero_rows(p.pre, expert_begin(p.offsets, p.E, p.R), p.R, static_cast<int>(p.n_z * sizeof(float) / 16));
    const RowTiles tiles = count_row_tiles(p.offsets, p.E, p.R, kTile);
    if (static_cast<int>(blockIdx.x) >= tiles.total) return;
    const RowTile t = find_row_tile(tiles, p.offsets, p.E, p.R, kTile, blockIdx.x);
    e = t.e;
    m0 = t.row0;
    m_end = t.row1;
    n0 = blockIdx.y * (kMode == kForward && p.gated ? kTile / 2 : kTile);
    k_end = kMode == kForward ? p.n_in : p.n_z;
  }
  const float* We = W + static_cast<long long>(e) * p.n_z * p.n_in;

  constexpr bool kAlongA = kMode != kGradW, kAlongB = kMode == kForward;
  Slice<kAlongA> a;
  Slice<kAlongB> b;
  const int lr = threadIdx.x >> 1;
  const bool a_in = m0 + lr < m_end;
  const float* a_row = kMode == kForward ? X + (m0 + lr) * p.n_in : dZ + (m0 + lr) * p.n_z;
  // forward: the output feature of B's row lr; gated tiles hold 64 gate rows, then the same 64 of u
  int b_row = n0 + lr;
  bool b_in = b_row < p.n_z;
  if (kMode == kForward && p.gated) {
    const int j = n0 + (lr & 63);
    b_row = lr < 64 ? j : p.n_out + j;
    b_in = j < p.n_out;
  }
  auto load = [&](long long d0) {
    if (kMode == kGradW) {
      a.load_across(dZ, p.n_z, d0, k_end, static_cast<int>(m0), p.n_z);
      b.load_across(X, p.n_in, d0, k_end, n0, p.n_in);
    } else {
      a.load_along(a_row, a_in, d0, k_end);
      if (kMode == kForward)
        b.load_along(We + static_cast<long long>(b_row) * p.n_in, b_in, d0, k_end);
      else
        b.load_across(We, p.n_in, d0, k_end, n0, p.n_in);
    }
  };

  uint64_t acc[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0ull;
  const long long steps = (k_end - k0 + kDepth - 1) / kDepth;
  if (steps > 0) {
    load(k0);
    a.store(As[0]);
    b.store(Bs[0]);
  }
  __syncthreads();
  for (long long st = 0; st < steps; ++st) {
    const int cur = static_cast<int>(st & 1);
    if (st + 1 < steps) load(k0 + (st + 1) * kDepth);
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
      float4 am[2];
      ulonglong2 bn[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        am[h] = *reinterpret_cast<const float4*>(&As[cur][d][ty * 4 + 64 * h]);
        bn[h] = *reinterpret_cast<const ulonglong2*>(&Bs[cur][d][tx * 4 + 64 * h]);
      }
      const float av[8] = {am[0].x, am[0].y, am[0].z, am[0].w, am[1].x, am[1].y, am[1].z, am[1].w};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint64_t aa = pack2(av[i], av[i]);
        acc[i][0] = ffma2(aa, bn[0].x, acc[i][0]);
        acc[i][1] = ffma2(aa, bn[0].y, acc[i][1]);
        acc[i][2] = ffma2(aa, bn[1].x, acc[i][2]);
        acc[i][3] = ffma2(aa, bn[1].y, acc[i][3]);
      }
    }
    if (st + 1 < steps) {
      a.store(As[cur ^ 1]);
      b.store(Bs[cur ^ 1]);
    }
    __syncthreads();
  }

  // thread's rows m0 + ty*4 + i (+64), columns tx*4 + j (+64)
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const long long m = m0 + ty * 4 + (i & 3) + 64 * (i >> 2);
    if (m >= m_end) continue;
    float z[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      z[h][0] = lo2(acc[i][2 * h]);
      z[h][1] = hi2(acc[i][2 * h]);
      z[h][2] = lo2(acc[i][2 * h + 1]);
      z[h][3] = hi2(acc[i][2 * h + 1]);
    }
    if (kMode == kGradW) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int n = n0 + tx * 4 + 64 * h;
        if (n >= p.n_in) continue;
        float4* w = reinterpret_cast<float4*>(p.dW + (static_cast<long long>(e) * p.n_z + m) * p.n_in + n);
        float4 o = make_float4(z[h][0], z[h][1], z[h][2], z[h][3]);
        if (p.accumulate) {
          const float4 old = *w;
          o = make_float4(old.x + o.x, old.y + o.y, old.z + o.z, old.w + o.w);
        }
        *w = o;
      }
    } else if (kMode == kGradX) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int n = n0 + tx * 4 + 64 * h;
        if (n < p.n_in) store4(static_cast<float*>(p.out) + m * p.n_in + n, z[h][0], z[h][1], z[h][2], z[h][3]);
      }
    } else {
      const float* bias = p.bias ? p.bias + static_cast<long long>(e) * p.n_z : nullptr;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int n = p.gated ? n0 + tx * 4 + h * p.n_out : n0 + tx * 4 + 64 * h;   // column of z
        const bool in = p.gated ? n0 + tx * 4 < p.n_out : n < p.n_z;
        if (!in) continue;
        if (bias) {
          const float4 bv = __ldg(reinterpret_cast<const float4*>(bias + n));
          z[h][0] += bv.x;
          z[h][1] += bv.y;
          z[h][2] += bv.z;
          z[h][3] += bv.w;
        }
        if (p.pre) store4(static_cast<float*>(p.pre) + m * p.n_z + n, z[h][0], z[h][1], z[h][2], z[h][3]);
      }
      const int halves = p.gated ? 1 : 2;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int n = n0 + tx * 4 + 64 * h;
        if (h >= halves || n >= p.n_out) continue;
        float y[4];
        float4 res = make_float4(0.f, 0.f, 0.f, 0.f);
        if (p.residual) res = load4(static_cast<const float*>(p.residual) + m * p.n_out + n);
        const float rv[4] = {res.x, res.y, res.z, res.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          y[j] = p.act == SMOES_ACT_SILU ? act_value<SMOES_ACT_SILU, false>(z[h][j])
                 : p.act == SMOES_ACT_GELU ? act_value<SMOES_ACT_GELU, false>(z[h][j]) : z[h][j];
          if (p.gated) y[j] *= z[1][j];
          y[j] += rv[j];
        }
        store4(static_cast<float*>(p.out) + m * p.n_out + n, y[0], y[1], y[2], y[3]);
      }
    }
  }
}

// Row tiles of at most R / 128 + min(E, R) exist whatever the offsets are; the rest return at once.
dim3 row_grid(const ExpertLinearParams& p, int cols, int per) {
  const long long tiles = p.R / kTile + (p.R < p.E ? p.R : p.E);
  return dim3(static_cast<unsigned>(tiles), static_cast<unsigned>((cols + per - 1) / per));
}

}  // namespace

cudaError_t launch_expert_linear(const ExpertLinearParams& p, cudaStream_t s) {
  const dim3 grid = row_grid(p, p.n_out, p.gated ? kTile / 2 : kTile);
  return launch_pdl(k_expert_linear<kForward>, grid, dim3(kLinThreads), 0, s, p);
}
cudaError_t launch_expert_dx(const ExpertLinearParams& p, cudaStream_t s) {
  const dim3 grid = row_grid(p, p.n_in, kTile);
  return launch_pdl(k_expert_linear<kGradX>, grid, dim3(kLinThreads), 0, s, p);
}
cudaError_t launch_expert_dw(const ExpertLinearParams& p, cudaStream_t s) {
  const dim3 grid((p.n_in + kTile - 1) / kTile, (p.n_z + kTile - 1) / kTile, p.E);
  return launch_pdl(k_expert_linear<kGradW>, grid, dim3(kLinThreads), 0, s, p);
}

}  // namespace smoes
