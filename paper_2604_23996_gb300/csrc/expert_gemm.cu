// expert_gemm.cu -- the experts' bf16 products on the tensor cores (tcgen05), grouped over ragged rows:
//   forward   z = W_e x_r + b_e, out = act(z) (or act(g) u of z = [g | u]) + residual
//   dX        W_e^T dz_r
//   dW        sum over the expert's rows of dz_r x_r^T
//
// A pair of CTAs forms a tile of 256 features (along M, 128 in each CTA) by up to 256 rows (along N; for
// dW n_in by n_z). With the rows along N a ragged end costs its own rows rounded up to 32, not a whole
// 128-row tile, and a few decoded tokens stream the weights through the same code; every value that a
// warp reads from one column of tensor memory is one output row, so stores of neighbouring lanes meet in
// memory. Each CTA loads its half of both operands; the first CTA issues the products of both.
//
// Gated: the 128 features of a CTA are 64 of g and the same 64 of u in turns of 16 lanes, so that the two
// halves of a warp hold g and u of the same features and change places with one shuffle per two values.
//
// Ragged edges: rows of the next expert inside a tile are other columns of D and are not stored; features
// past the expert's weights are zeros of the 3-d map (or the rows of u, not stored); a depth that ends
// inside a block is zeros of both maps. For dW the depth is the expert's rows: the last block's products
// stop at the 16 rows that hold the end, and a warp clears the rows behind it in shared memory before
// they are issued (multiplying them by zero would let infinities of the next expert in).
//
// Roles of a CTA's warps: 0 producer, 1 MMA issuer (first CTA), 2 tensor memory and the clearing, 4-11
// epilogue, in two groups that take alternate 32-column chunks. Two accumulators of 256 columns: the epilogue of a
// tile runs under the next tile's products.
#include <algorithm>
#include <mutex>

#include "experts.cuh"
#include "ptx.cuh"

namespace smoes {
namespace {

constexpr int kGemmThreads = 384;
constexpr int kGemmEpiWarps = 8;
constexpr int kGemmStages = 6;
constexpr int kGemmK = 64;                       // depth of a block: 128 bytes of bf16
constexpr uint32_t kGemmHalf = 128 * kGemmK * 2; // one CTA's operand of a block: 16 KB
// dW: rows summed by the tensor cores before the sum moves to fp32 registers. The tensor cores cut each
// addition off towards zero: relative error 4.7e-7 after 512 products, 1.5e-6 after 1536, 9e-6 after 8192.
constexpr int kGemmChunk = 8;                    // blocks of 64 rows

struct GemmSmem {
  uint32_t a[kGemmStages], b[kGemmStages], bars, first, total;
};
constexpr uint32_t gemm_smem_bytes(int E) {
  return 1024 + kGemmStages * 2 * kGemmHalf + 512 + 4 * (E + 1);
}

struct GemmBars {
  uint64_t full[kGemmStages];                    // operands of both CTAs (first CTA's)
  uint64_t empty[kGemmStages];
  uint64_t tail[kGemmStages];                    // this CTA's operands of an expert's last rows, to be cleared
  uint64_t acc_full[2], acc_empty[2];
  uint32_t tmem;
  int abort;
};
static_assert(sizeof(GemmBars) <= 512, "barriers");

// A tile: expert, first feature, the N extent.
struct GemmTile {
  int e, m;                                      // expert, feature tile
  long long row0;                                // first row (dW: the expert's first row)
  int cols;                                      // rows of the tile (dW: columns of n_z)
  int col0;                                      // dW: first column of n_z
  int blocks;                                    // blocks along the depth
  int last;                                      // dW: rows of the last block
};

template <int kMode>
__device__ __forceinline__ GemmTile gemm_tile(const ExpertGemmParams& p, const int* first, int tile) {
  GemmTile t;
  if (kMode == kGemmGradW) {
    const int per = p.m_tiles * p.n_tiles;
    t.e = tile / per;
    const int in = tile - t.e * per;
    const int j = in / p.m_tiles;
    t.m = in - j * p.m_tiles;
    t.col0 = j * 256;
    t.cols = min(256, p.l.n_z - t.col0);
    t.row0 = expert_begin(p.l.offsets, t.e, p.l.R);
    const long long rows = max(0ll, expert_begin(p.l.offsets, t.e + 1, p.l.R) - t.row0);
    t.blocks = static_cast<int>((rows + kGemmK - 1) / kGemmK);
    t.last = static_cast<int>(rows - static_cast<long long>(t.blocks - 1) * kGemmK);
    return t;
  }
  const int lane = threadIdx.x & 31;
  const int rt = tile / p.m_tiles;
  t.m = tile - rt * p.m_tiles;
  // the last expert whose first row tile is at or before rt (empty experts share it with the next)
  const int E = p.l.E;
  const unsigned b0 = __ballot_sync(0xffffffffu, lane * 8 < E && first[min(lane * 8, E)] <= rt);
  const int q = 31 - __clz(b0);
  const int at = q * 8 + (lane & 7);
  const unsigned b1 = __ballot_sync(0xffffffffu, lane < 8 && at < E && first[min(at, E)] <= rt);
  t.e = q * 8 + 31 - __clz(b1);
  const long long begin = expert_begin(p.l.offsets, t.e, p.l.R), end = expert_begin(p.l.offsets, t.e + 1, p.l.R);
  t.row0 = begin + static_cast<long long>(rt - first[t.e]) * 256;
  t.cols = static_cast<int>(min(256ll, end - t.row0));
  t.col0 = 0;
  t.last = kGemmK;
  t.blocks = ((kMode == kGemmForward ? p.l.n_in : p.l.n_z) + kGemmK - 1) / kGemmK;
  return t;
}

// N of the tile's products: both CTAs hold half of the rows. dW: whole 64-column boxes in each.
template <int kMode>
__device__ __forceinline__ int gemm_n(const GemmTile& t) {
  return kMode == kGemmGradW ? (t.cols + 127) & ~127 : (t.cols + 31) & ~31;
}

__device__ __forceinline__ float fast_act(int act, float z) {
  if (act == SMOES_ACT_SILU) return z * __fdividef(1.f, 1.f + __expf(-z));
  if (act == SMOES_ACT_GELU) return 0.5f * z * erfcf(z * -0.70710678f);
  return z;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// One 32-column chunk of D (a feature per lane, an output row per column) to rows of bf16: neighbouring
// lanes exchange every other column, so that each stores two features of one row at once.
// base: row 0's address of the lane's even feature; in: the lane's features exist.
__device__ __forceinline__ void store_chunk(__nv_bfloat16* base, long long stride, const float (&v)[32], int rows,
                                            bool in) {
  const int odd = threadIdx.x & 1;
#pragma unroll
  for (int c = 0; c < 32; c += 2) {
    const float got = __shfl_xor_sync(0xffffffffu, odd ? v[c] : v[c + 1], 1);
    const uint32_t w = odd ? pack_bf16(got, v[c + 1]) : pack_bf16(v[c], got);
    if (in && c + odd < rows) *reinterpret_cast<uint32_t*>(base + (c + odd) * stride) = w;
  }
}

__device__ __forceinline__ void forward_chunk(const ExpertGemmParams& p, float (&v)[32], long long row, int rows,
                                              int f, bool f_in, int zf, float bias) {
  const ExpertLinearParams& l = p.l;
  const int lane = threadIdx.x & 31, odd = lane & 1;
#pragma unroll
  for (int c = 0; c < 32; ++c) v[c] += bias;
  if (l.pre)
    store_chunk(static_cast<__nv_bfloat16*>(l.pre) + row * l.n_z + (zf - odd), l.n_z, v, rows, f_in);
  __nv_bfloat16* out = static_cast<__nv_bfloat16*>(l.out) + row * l.n_out + (f - odd);
  const __nv_bfloat16* res =
      l.residual ? static_cast<const __nv_bfloat16*>(l.residual) + row * l.n_out + (f - odd) : nullptr;
  if (!l.gated) {
    uint32_t rv[16];
    if (res) {
#pragma unroll
      for (int c = 0; c < 32; c += 2)
        rv[c / 2] = f_in && c + odd < rows ? __ldg(reinterpret_cast<const uint32_t*>(res + (c + odd) * static_cast<long long>(l.n_out))) : 0u;
    }
    if (l.act) {
#pragma unroll
      for (int c = 0; c < 32; ++c) v[c] = fast_act(l.act, v[c]);
    }
#pragma unroll
    for (int c = 0; c < 32; c += 2) {
      const float got = __shfl_xor_sync(0xffffffffu, odd ? v[c] : v[c + 1], 1);
      float lo = odd ? got : v[c], hi = odd ? v[c + 1] : got;
      if (res) {
        lo += __uint_as_float(rv[c / 2] << 16);
        hi += __uint_as_float(rv[c / 2] & 0xffff0000u);
      }
      if (f_in && c + odd < rows)
        *reinterpret_cast<uint32_t*>(out + (c + odd) * static_cast<long long>(l.n_out)) = pack_bf16(lo, hi);
    }
    return;
  }
  // gated: lanes 0-15 hold g, 16-31 u; of two columns each half finishes one
  const int up = lane >> 4;
  float y[16];
#pragma unroll
  for (int c = 0; c < 32; c += 2) {
    const float got = __shfl_xor_sync(0xffffffffu, up ? v[c] : v[c + 1], 16);
    const float g = up ? got : v[c], u = up ? v[c + 1] : got;
    y[c / 2] = fast_act(l.act, g) * u;
  }
  uint32_t rv[8];
#pragma unroll
  for (int c = 0; c < 32; c += 4) {
    const int col = c + 2 * odd + up;
    rv[c / 4] = res && f_in && col < rows ? __ldg(reinterpret_cast<const uint32_t*>(res + col * static_cast<long long>(l.n_out))) : 0u;
  }
#pragma unroll
  for (int c = 0; c < 32; c += 4) {
    const float got = __shfl_xor_sync(0xffffffffu, odd ? y[c / 2] : y[c / 2 + 1], 1);
    float lo = odd ? got : y[c / 2], hi = odd ? y[c / 2 + 1] : got;
    const int col = c + 2 * odd + up;
    if (res) {
      lo += __uint_as_float(rv[c / 4] << 16);
      hi += __uint_as_float(rv[c / 4] & 0xffff0000u);
    }
    if (f_in && col < rows) *reinterpret_cast<uint32_t*>(out + col * static_cast<long long>(l.n_out)) = pack_bf16(lo, hi);
  }
}

template <int kMode>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kGemmThreads, 1)
k_expert_gemm(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
              const __grid_constant__ CUtensorMap tmB16, const ExpertGemmParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t* sa = smem;
  uint8_t* sb = smem + kGemmStages * kGemmHalf;
  GemmBars& bars = *reinterpret_cast<GemmBars*>(smem + 2 * kGemmStages * kGemmHalf);
  int* first = reinterpret_cast<int*>(smem + 2 * kGemmStages * kGemmHalf + 512);   // [E + 1] row tiles before e
  const ExpertLinearParams& l = p.l;
  const int warp = warp_index(), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kGemmStages; ++i) {
      mbar_init(&bars.full[i], 2);
      mbar_init(&bars.empty[i], 1);
      mbar_init(&bars.tail[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars.acc_full[i], 1);
      mbar_init(&bars.acc_empty[i], 2 * kGemmEpiWarps);
    }
    bars.abort = 0;
    fence_mbar_init();
    tma_prefetch_desc(&tmA);
    tma_prefetch_desc(&tmB);
  }
  if (warp == 2) tmem_alloc_pair(&bars.tmem, 512);
  pdl_wait();
  pdl_trigger();
  int n_total;                                   // tiles
  if (kMode == kGemmGradW) {
    n_total = l.E * p.m_tiles * p.n_tiles;
  } else if (warp == 0) {
    int n[8], sum = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = lane * 8 + i;
      const long long rows = e < l.E ? expert_begin(l.offsets, e + 1, l.R) - expert_begin(l.offsets, e, l.R) : 0;
      n[i] = rows > 0 ? static_cast<int>((rows + 255) / 256) : 0;
      sum += n[i];
    }
    int run = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, run, o);
      if (lane >= o) run += v;
    }
    int at = run - sum;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (lane * 8 + i <= l.E) first[lane * 8 + i] = at;
      at += n[i];
    }
    if (l.E == 256 && lane == 31) first[256] = at;
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();                                // both CTAs' barriers are ready before anything arrives on them
  tc_fence_after();
  if (kMode != kGemmGradW) n_total = first[l.E] * p.m_tiles;
  const uint32_t tmem = bars.tmem;
  const WaitCtx wc{&bars.abort, p.status, p.limit_ns};

  if (warp == 0) {
    // ------------------------------------------------------------------------------- producer
    int st = 0;
    uint32_t ph = 0;
    bool ok = true;
    for (int tile = pair; ok && tile < n_total; tile += n_pairs) {
      const GemmTile t = gemm_tile<kMode>(p, first, tile);
      const int half_n = gemm_n<kMode>(t) / 2;
      for (int kb = 0; kb < t.blocks; ++kb) {
        if (!warp_wait(&bars.empty[st], ph ^ 1, wc)) { ok = false; break; }
        if (elect_one()) {
          uint8_t* a = sa + st * kGemmHalf;
          uint8_t* b = sb + st * kGemmHalf;
          if (kMode == kGemmGradW) {
            const int boxes = half_n / 64;
            const uint32_t bytes = kGemmHalf + boxes * 8192u;
            const int r0 = static_cast<int>(t.row0) + kb * kGemmK;
            uint32_t bar;
            if (kb == t.blocks - 1 && (t.last & 15)) {
              bar = smem_u32(&bars.tail[st]);
              mbar_arrive_expect_tx(&bars.tail[st], bytes);
            } else {
              bar = peer_smem(&bars.full[st], 0);
              mbar_arrive_expect_tx_peer(bar, bytes);
            }
            const int i0 = t.m * 256 + static_cast<int>(rank) * 128;
            tma_load_2d_pair(a, &tmA, bar, i0, r0);
            tma_load_2d_pair(a + 8192, &tmA, bar, i0 + 64, r0);
            const int c0 = t.col0 + static_cast<int>(rank) * half_n;
            for (int i = 0; i < boxes; ++i) tma_load_2d_pair(b + i * 8192, &tmB, bar, c0 + 64 * i, r0);
          } else {
            const uint32_t bar = peer_smem(&bars.full[st], 0);
            mbar_arrive_expect_tx_peer(bar, kGemmHalf + half_n * 128u);
            const int k0 = kb * kGemmK;
            if (kMode == kGemmForward) {
              if (l.gated) {
                const int f0 = t.m * 128 + static_cast<int>(rank) * 64;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                  tma_load_3d_pair(a + i * 2048, &tmA, bar, k0, (i & 1) * l.n_out + f0 + (i >> 1) * 16, t.e);
              } else {
                tma_load_3d_pair(a, &tmA, bar, k0, t.m * 256 + static_cast<int>(rank) * 128, t.e);
              }
            } else {
              const int i0 = t.m * 256 + static_cast<int>(rank) * 128;
              tma_load_3d_pair(a, &tmA, bar, i0, k0, t.e);
              tma_load_3d_pair(a + 8192, &tmA, bar, i0 + 64, k0, t.e);
            }
            const int r0 = static_cast<int>(t.row0) + static_cast<int>(rank) * half_n;
            if (half_n == 128) {
              tma_load_2d_pair(b, &tmB, bar, k0, r0);
            } else {
              for (int i = 0; i < half_n; i += 16) tma_load_2d_pair(b + i * 128, &tmB16, bar, k0, r0 + i);
            }
          }
        }
        __syncwarp();
        if (++st == kGemmStages) { st = 0; ph ^= 1; }
      }
    }
    // every stage given back: no commit of the first CTA is still on its way to this one when it ends
    for (int i = 0; ok && i < kGemmStages; ++i) {
      ok = warp_wait(&bars.empty[st], ph ^ 1, wc);
      if (++st == kGemmStages) { st = 0; ph ^= 1; }
    }
  } else if (warp == 1 && rank == 0) {
    // ----------------------------------------------------------------------------- MMA issuer
    int st = 0, acc = 0;
    uint32_t ph = 0, aph = 0;
    bool ok = true;
    constexpr bool kMajorA = kMode != kGemmForward, kMajorB = kMode == kGemmGradW;   // along M / N in memory
    for (int tile = pair; ok && tile < n_total; tile += n_pairs) {
      const GemmTile t = gemm_tile<kMode>(p, first, tile);
      const uint32_t idesc = idesc_bf16(256, gemm_n<kMode>(t), kMajorA, kMajorB);
      const int chunk = kMode == kGemmGradW ? kGemmChunk : t.blocks;
      for (int k0 = 0; ok && k0 < t.blocks; k0 += chunk) {
        if (!warp_wait(&bars.acc_empty[acc], aph ^ 1, wc)) { ok = false; break; }
        tc_fence_after();
        const uint32_t d = tmem + acc * 256;
        const int k1 = min(k0 + chunk, t.blocks);
        for (int kb = k0; kb < k1; ++kb) {
          if (!warp_wait(&bars.full[st], ph, wc)) { ok = false; break; }
          tc_fence_after();
          if (elect_one()) {
            const uint32_t a = smem_u32(sa + st * kGemmHalf), b = smem_u32(sb + st * kGemmHalf);
            const int steps = kMode == kGemmGradW && kb == t.blocks - 1 ? (t.last + 15) >> 4 : 4;
            for (int s = 0; s < steps; ++s) {
              const uint64_t da = kMajorA ? sdesc_sw128(a + s * 2048, 8192, 1024) : sdesc_sw128(a + s * 32, 16, 1024);
              const uint64_t db = kMajorB ? sdesc_sw128(b + s * 2048, 8192, 1024) : sdesc_sw128(b + s * 32, 16, 1024);
              umma_bf16_pair(d, da, db, idesc, kb > k0 || s > 0);
            }
            umma_commit_pair(&bars.empty[st]);
            if (kb == k1 - 1) umma_commit_pair(&bars.acc_full[acc]);
          }
          __syncwarp();
          if (++st == kGemmStages) { st = 0; ph ^= 1; }
        }
        if (++acc == 2) { acc = 0; aph ^= 1; }
      }
    }
  } else if (warp == 2 && kMode == kGemmGradW) {
    // ------------------------------------------------- dW: clears what follows an expert's last row
    int st = 0;
    uint32_t phases = 0;                         // bit s: parity of tail[s]
    for (int tile = pair; tile < n_total; tile += n_pairs) {
      const GemmTile t = gemm_tile<kMode>(p, first, tile);
      if (t.blocks == 0) continue;
      const int s = (st + t.blocks - 1) % kGemmStages;
      st = (st + t.blocks) % kGemmStages;
      if (!(t.last & 15)) continue;
      if (!warp_wait(&bars.tail[s], (phases >> s) & 1, wc)) break;
      phases ^= 1u << s;
      // rows [last, round_up(last, 16)) of every 64-column box: 8 words of 16 bytes a row
      const int boxes = gemm_n<kMode>(t) / 128, words = (16 - (t.last & 15)) * 8;
      for (int x = 0; x < 2 + boxes; ++x) {
        uint8_t* box = x < 2 ? sa + s * kGemmHalf + x * 8192 : sb + s * kGemmHalf + (x - 2) * 8192;
        for (int i = lane; i < words; i += 32) *reinterpret_cast<uint4*>(box + t.last * 128 + i * 16) = make_uint4(0u, 0u, 0u, 0u);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive_peer_release(peer_smem(&bars.full[s], 0));
      __syncwarp();
    }
  } else if (warp >= 4) {
    // ------------------------------------------------------------------------------- epilogue
    const int q = warp & 3, g = (warp - 4) >> 2;
    const uint32_t lanes = static_cast<uint32_t>(32 * q) << 16;
    if (kMode != kGemmGradW) {
      const long long end = expert_begin(l.offsets, l.E, l.R);
      if (end < l.R) {                           // rows of no expert
        const int threads = 32 * kGemmEpiWarps;
        for (int which = 0; which < (l.pre ? 2 : 1); ++which) {
          uint4* o = static_cast<uint4*>(which ? l.pre : l.out);
          const int words = (which ? l.n_z : p.n_feat) / 8;
          for (long long i = end * words + static_cast<long long>(blockIdx.x) * threads + (threadIdx.x - 128);
               i < l.R * words; i += static_cast<long long>(gridDim.x) * threads)
            o[i] = make_uint4(0u, 0u, 0u, 0u);
        }
      }
    }
    int acc = 0;
    uint32_t aph = 0;
    bool ok = true;
    for (int tile = pair; ok && tile < n_total; tile += n_pairs) {
      const GemmTile t = gemm_tile<kMode>(p, first, tile);
      if constexpr (kMode == kGemmGradW) {
        float sum[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 32; ++i) sum[c][i] = 0.f;
        for (int k0 = 0; k0 < t.blocks; k0 += kGemmChunk) {
          if (!warp_wait(&bars.acc_full[acc], aph, wc)) { ok = false; break; }
          tc_fence_after();
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int col = g * 128 + c * 32;
            if (col < t.cols) {
              float v[32];
              tmem_ld32(tmem + acc * 256 + col + lanes, v);
#pragma unroll
              for (int i = 0; i < 32; ++i) sum[c][i] += v[i];
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_peer(peer_smem(&bars.acc_empty[acc], 0));
          if (++acc == 2) { acc = 0; aph ^= 1; }
        }
        const int i = t.m * 256 + static_cast<int>(rank) * 128 + 32 * q + lane;
        if (ok && i < l.n_in && !(l.accumulate && t.blocks == 0)) {
          float* w = l.dW + (static_cast<long long>(t.e) * l.n_z + t.col0 + g * 128) * l.n_in + i;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              if (g * 128 + c * 32 + j < t.cols) {
                float* at = w + static_cast<long long>(c * 32 + j) * l.n_in;
                *at = l.accumulate ? *at + sum[c][j] : sum[c][j];
              }
            }
          }
        }
      } else {
        // the lane's feature: of the output (f) and, forward, of z
        int f = t.m * 256 + static_cast<int>(rank) * 128 + 32 * q + lane, zf = f;
        if (kMode == kGemmForward && l.gated) {
          f = t.m * 128 + static_cast<int>(rank) * 64 + 16 * q + (lane & 15);
          zf = f + (lane >> 4) * l.n_out;
        }
        const bool f_in = f < p.n_feat;
        float bias = 0.f;
        if (kMode == kGemmForward && l.bias && f_in) bias = __ldg(l.bias + static_cast<long long>(t.e) * l.n_z + zf);
        if (!warp_wait(&bars.acc_full[acc], aph, wc)) { ok = false; break; }
        tc_fence_after();
        const int chunks = (t.cols + 31) / 32;
        for (int c = g; c < chunks; c += 2) {
          float v[32];
          tmem_ld32(tmem + acc * 256 + c * 32 + lanes, v);
          const long long row = t.row0 + c * 32;
          const int rows = min(32, t.cols - c * 32);
          if (kMode == kGemmForward)
            forward_chunk(p, v, row, rows, f, f_in, zf, bias);
          else
            store_chunk(static_cast<__nv_bfloat16*>(l.out) + row * l.n_in + (f - (lane & 1)), l.n_in, v, rows, f_in);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_peer(peer_smem(&bars.acc_empty[acc], 0));
        if (++acc == 2) { acc = 0; aph ^= 1; }
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (bars.abort && threadIdx.x == 0)            // copies and products in flight end long before this does
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  if (warp == 2) tmem_dealloc_pair(tmem, 512);
}

// Pairs of CTAs that the device holds at once.
template <int kMode>
cudaError_t max_pairs(int n_sms, uint32_t smem, int* out) {
  static std::mutex mu;
  static int cached[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(mu);
  if (cached[dev] == 0) {
    e = cudaFuncSetAttribute(k_expert_gemm<kMode>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             static_cast<int>(gemm_smem_bytes(kExpertsMax)));
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(n_sms / 2 * 2);
    cfg.blockDim = dim3(kGemmThreads);
    cfg.dynamicSmemBytes = smem;
    int n = 0;
    e = cudaOccupancyMaxActiveClusters(&n, k_expert_gemm<kMode>, &cfg);
    if (e != cudaSuccess) return e;
    if (n < 1) return cudaErrorLaunchOutOfResources;
    cached[dev] = n;
  }
  *out = cached[dev];
  return cudaSuccess;
}

template <int kMode>
cudaError_t launch(const ExpertGemmParams& p, const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& b16,
                   long long tiles, int n_sms, cudaStream_t s) {
  const uint32_t smem = gemm_smem_bytes(kExpertsMax);
  int pairs = 0;
  const cudaError_t e = max_pairs<kMode>(n_sms, smem, &pairs);
  if (e != cudaSuccess) return e;
  pairs = static_cast<int>(std::min<long long>(pairs, std::max(1ll, tiles)));
  return launch_pdl(k_expert_gemm<kMode>, dim3(2 * pairs), dim3(kGemmThreads), smem, s, a, b, b16, p);
}

}  // namespace

cudaError_t launch_expert_gemm(const ExpertLinearParams& l, ExpertGemmMode mode, uint32_t* status, uint64_t limit_ns,
                               int n_sms, cudaStream_t s) {
  ExpertGemmParams p{};
  p.l = l;
  p.status = status;
  p.limit_ns = limit_ns;
  p.n_feat = mode == kGemmForward ? l.n_out : l.n_in;
  const int per = mode == kGemmForward && l.gated ? 128 : 256;
  p.m_tiles = (p.n_feat + per - 1) / per;
  p.n_tiles = (l.n_z + 255) / 256;
  const uint64_t R = static_cast<uint64_t>(l.R), ni = l.n_in, nz = l.n_z, E = l.E;
  CUtensorMap a, b, b16;
  bool ok;
  if (mode == kGemmGradW) {
    const uint64_t da[2] = {ni, R}, sta[1] = {ni * 2}, db[2] = {nz, R}, stb[1] = {nz * 2};
    const uint32_t box[2] = {64, 64};
    ok = encode_bf16(&a, l.X, 2, da, sta, box) && encode_bf16(&b, l.dZ, 2, db, stb, box);
    b16 = b;
  } else {
    const uint64_t da[3] = {ni, nz, E}, sta[2] = {ni * 2, ni * nz * 2};
    const uint32_t boxa[3] = {64, mode == kGemmGradX ? 64u : l.gated ? 16u : 128u, 1};
    const uint64_t depth = mode == kGemmForward ? ni : nz;
    const uint64_t db[2] = {depth, R}, stb[1] = {depth * 2};
    const uint32_t box[2] = {64, 128}, box16[2] = {64, 16};
    const void* rows = mode == kGemmForward ? l.X : l.dZ;
    ok = encode_bf16(&a, l.W, 3, da, sta, boxa) && encode_bf16(&b, rows, 2, db, stb, box) &&
         encode_bf16(&b16, rows, 2, db, stb, box16);
  }
  if (!ok) return cudaErrorInvalidValue;
  // at most R / 256 + min(E, R) row tiles
  const long long row_tiles = l.R / 256 + std::min<long long>(l.E, l.R);
  if (mode == kGemmForward) return launch<kGemmForward>(p, a, b, b16, row_tiles * p.m_tiles, n_sms, s);
  if (mode == kGemmGradX) return launch<kGemmGradX>(p, a, b, b16, row_tiles * p.m_tiles, n_sms, s);
  return launch<kGemmGradW>(p, a, b, b16, static_cast<long long>(l.E) * p.m_tiles * p.n_tiles, n_sms, s);
}

}  // namespace smoes
