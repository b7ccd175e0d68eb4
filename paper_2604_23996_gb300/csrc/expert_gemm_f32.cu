// expert_gemm_f32.cu -- the experts' fp32 products on the bf16 tensor cores (tcgen05), grouped over ragged rows
// (formulas: expert_linear's in include/smoes.h; tiles: expert_gemm.cuh).
//
// Each fp32 value is the sum of three bf16 values, x = h + m + l to 2^-27 of x, each the rounding of what the ones
// before it leave. Of the nine products of two such sums the six that reach 2^-18 are formed, l h, h l, m m, m h,
// h m and h h; the other three are below 2^-26 of |x y| (with cut instead of rounded parts they reach 2^-22 and
// all have one sign). The tensor cores sum them in fp32 but cut each addition off, so h h has an accumulator of its
// own, the five small products another, whose cuts are 2^-8 smaller, and after every 256 of the depth both move
// to fp32 sums in registers (relative error 2.4e-7 from sixteen additions). Infinities and magnitudes above
// 3.38e38, which round to one, give NaN.
//
// A pair of CTAs forms 256 features by up to 128 rows, as in expert_gemm.cu. Roles of a CTA's warps: 0 copies fp32
// blocks of 32 of the depth to shared memory, 1 issues the products (first CTA), 2 and 3 hand the second CTA's planes to
// the first, 4-19 split the blocks, eight of them every other one, and, one 256-deep chunk behind, all move the sums and
// store finished tiles. (2 holds tensor memory as well.)
// A block's planes: along the depth 128-byte rows of [h | m], and of [l | l] for two blocks; across it one box of 32 depth
// rows per plane and 64 features. Rows behind an expert's last one are cleared where they are split.
//
// The first CTA's products read planes that the second CTA's threads wrote. That order holds between CTAs only with a
// release and an acquire at cluster scope, and each takes about as long as a block's products. Warps 2 and 3 make them,
// for every other block each: in the second CTA they see the planes finished and release them to the first, there they
// acquire them and arrive for the issuer. Made by the splitting warps and the issuer: 364 us for 8192 x 2048 x 2048 forward
// instead of 300; by one warp of the second CTA and the issuer: 361. Without them (arrivals of a CTA's scope across the
// pair, no promise that the products see the planes) 257.
//
// Bound by shared memory (a block's 24 KB arrive, are read and written as 36 KB, and the products read 72 KB, 1220
// clocks at 128 bytes each against 770 of the products) and by a block's way through splitting, handing over and products,
// four at a time. Measured: 32768 x 2048 x 2048 of 16 experts 243 TFLOP/s forward, 253 dX, 250 dW; 8192 x 512 x 256 of 16
// experts 21 us dX and 20 us dW, on the FMA units (128 x 128 a block of threads) 187 for both.
#include "expert_gemm.cuh"
#include "experts.cuh"
#include "ptx.cuh"

namespace smoes {
namespace {

constexpr int kF32Threads = 640;
constexpr int kF32Warps = 16;                    // splitting, and epilogue in groups of four
constexpr int kF32K = 32;                        // depth of a block
constexpr int kF32Chunk = 8;                     // blocks between moves of the sums
// Blocks go to two halves of the splitting warps in turn: while one waits for its block's bytes and fences what it
// wrote, the other splits (8192 x 2048 x 2048: 300 instead of 311 us forward, 289 instead of 290 dX, 295 instead of
// 308 dW).
constexpr int kTurns = 2, kSplitThreads = 32 * kF32Warps / kTurns;      // threads that split a block
// A half sees every other use of a raw stage only, and by its parity could not tell a barrier's phase from the one two
// before. Barriers are therefore kept for six blocks, two uses of each of the three stages: every use of one of them has
// the same half of the warps behind it, and the same in front. Planes have four stages, each of them one half's.
constexpr int kRawStages = 3, kRawBars = kTurns * kRawStages, kPlaneStages = 4;
static_assert(kPlaneStages % kTurns == 0, "a stage of planes has the same half of the warps behind every use");
constexpr uint32_t kRawA = 128 * kF32K * 4, kRawB = 64 * kF32K * 4;     // one CTA's fp32 operands of a block
constexpr uint32_t kPlanesA = kPlaneStages * 3 * 128 * kF32K * 2, kPlanesB = kPlanesA / 2;   // all stages of their planes
constexpr uint32_t kF32Smem =
    1024 + kPlanesA + kPlanesB + kRawStages * (kRawA + kRawB) + kBarBytes + 4 * (kExpertsMax + 1);
static_assert(kF32Smem <= 227 * 1024, "shared memory of a CTA");

struct F32Bars {
  uint64_t raw_full[kRawBars], raw_empty[kRawBars];
  uint64_t split_full[kPlaneStages];             // planes of both CTAs (in the first)
  uint64_t split_mine[kPlaneStages];             // the second CTA's planes (in the second)
  uint64_t split_peer[kPlaneStages];             // the second CTA's planes (in the first)
  uint64_t split_empty[kPlaneStages];
  uint64_t acc_full[2], acc_empty[2];
  uint32_t tmem;
  int abort;
  int before[33];                                // row tiles (count_row_tiles)
};
static_assert(sizeof(F32Bars) <= kBarBytes, "barriers");

// A block's place in the ring of raw stages: its barriers, and those of the block that had its stage before it.
struct RawPlace {
  int bar = 0;
  uint32_t ph = 0;
  __device__ __forceinline__ int stage() const { return bar < kRawStages ? bar : bar - kRawStages; }
  __device__ __forceinline__ int before() const { return bar < kRawStages ? bar + kRawStages : bar - kRawStages; }
  __device__ __forceinline__ uint32_t before_ph() const { return bar < kRawStages ? ph ^ 1 : ph; }
  __device__ __forceinline__ void next() {
    if (++bar == kRawBars) { bar = 0; ph ^= 1; }
  }
};
// And in that of the planes.
struct PlanePlace {
  int st = 0;
  uint32_t ph = 0;
  __device__ __forceinline__ void next() {
    if (++st == kPlaneStages) { st = 0; ph ^= 1; }
  }
};

// Where plane x (0 h, 1 m, 2 l) of a stage begins among an operand's planes of kRows rows or columns. kAcross: one after
// the other. Along the depth two planes share rows of 128 bytes: h and m of a stage, l of two stages.
template <bool kAcross, int kRows>
__device__ __forceinline__ uint32_t plane_offset(int st, int x) {
  if (kAcross) return static_cast<uint32_t>(st * 3 + x) * (kRows * kF32K * 2);
  return x < 2 ? st * (kRows * 128) + x * 64 : (kPlaneStages + (st >> 1)) * (kRows * 128) + (st & 1) * 64;
}

// Four values, split, to their places in the planes.
__device__ __forceinline__ uint2 split_off(float (&x)[4]) {             // x becomes what is left
  uint2 w;
  uint32_t* half[2] = {&w.x, &w.y};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    const uint32_t u = *reinterpret_cast<const uint32_t*>(&b);
    x[2 * i] -= __uint_as_float(u << 16);
    x[2 * i + 1] -= __uint_as_float(u & 0xffff0000u);
    *half[i] = u;
  }
  return w;
}
__device__ __forceinline__ void split_store(const float4& v, uint8_t* h, uint8_t* m, uint8_t* l) {
  float x[4] = {v.x, v.y, v.z, v.w};
  *reinterpret_cast<uint2*>(h) = split_off(x);
  *reinterpret_cast<uint2*>(m) = split_off(x);
  *reinterpret_cast<uint2*>(l) = split_off(x);
}

// Word `u` (16 bytes) of a raw operand of kRows rows or columns, split into its planes of stage st. kAcross: the depth
// runs over the rows of the block, of which `depth` exist.
template <bool kAcross, int kRows>
__device__ __forceinline__ void split_word(const uint8_t* raw, uint8_t* planes, int st, int u, int depth) {
  float4 v;
  if (kAcross) {
    v = *reinterpret_cast<const float4*>(raw + u * 16);
    const int k = u / (kRows / 4), c = u % (kRows / 4) * 4;
    if (k >= depth) v = make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr uint32_t kPlane = kRows * kF32K * 2;
    uint8_t* at = planes + plane_offset<true, kRows>(st, 0) + (c >> 6) * (kF32K * 128) + sw128_offset(k, c & 63);
    split_store(v, at, at + kPlane, at + 2 * kPlane);
  } else {
    // a warp's 4 rows are 0, 4, 1, 5 (or 2, 6, 3, 7) of eight: the words of a half warp's two rows lie in different banks
    const int w = u >> 5, x = (u >> 3) & 3, k = (u & 7) * 4;
    const int r = (w >> 1) * 8 + (w & 1) * 2 + (x & 1) * 4 + (x >> 1);
    v = *reinterpret_cast<const float4*>(raw + r * (kF32K * 4) + k * 4);
    // (a plane of a row's second 64 bytes: the swizzled word's place with that bit the other way round)
    uint8_t* rows = planes + sw128_offset(r, k);
    const int m = (sw128_offset(r, k) & 64) ? -64 : 64;
    const uint32_t l = plane_offset<false, kRows>(st, 2);
    uint8_t* h = rows + plane_offset<false, kRows>(st, 0);
    split_store(v, h, h + m, rows + (l & ~64u) + ((l & 64) ? m : 0));
  }
}

template <int kMode, int kAct, bool kGated>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kF32Threads, 1)
k_expert_gemm_f32(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                  const __grid_constant__ CUtensorMap tmB16, const ExpertGemmParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t* planes_a = smem;
  uint8_t* planes_b = planes_a + kPlanesA;
  uint8_t* raw_a = planes_b + kPlanesB;          // [stage] each
  uint8_t* raw_b = raw_a + kRawStages * kRawA;
  F32Bars& bars = *reinterpret_cast<F32Bars*>(raw_b + kRawStages * kRawB);
  int32_t* off = reinterpret_cast<int32_t*>(reinterpret_cast<uint8_t*>(&bars) + kBarBytes);   // [E + 1] offsets
  const ExpertLinearParams& l = p.l;
  const int warp = warp_index(), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
  constexpr bool kAcrossA = kMode != kGemmForward, kAcrossB = kMode == kGemmGradW;   // the depth is not contiguous

  if (threadIdx.x == 0) {
    for (int i = 0; i < kRawBars; ++i) {
      mbar_init(&bars.raw_full[i], 1);
      mbar_init(&bars.raw_empty[i], kF32Warps / kTurns);
    }
    for (int i = 0; i < kPlaneStages; ++i) {
      mbar_init(&bars.split_full[i], kF32Warps / kTurns + 1);   // (this CTA's warps, and the other's through split_peer)
      mbar_init(&bars.split_mine[i], kF32Warps / kTurns);
      mbar_init(&bars.split_peer[i], 1);
      mbar_init(&bars.split_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars.acc_full[i], 1);
      mbar_init(&bars.acc_empty[i], 2 * kF32Warps);
    }
    bars.abort = 0;
    fence_mbar_init();
    tma_prefetch_desc(&tmA);
    tma_prefetch_desc(&tmB);
    tma_prefetch_desc(&tmB16);
  }
  if (warp == 2) tmem_alloc_pair(&bars.tmem, 512);
  pdl_wait();
  pdl_trigger();
  if (kMode != kGemmGradW && warp == 3) count_row_tiles(l.offsets, l.E, static_cast<int>(l.R), ShiftRows{p.tile_shift}, bars.before);
  for (int e = threadIdx.x; e <= l.E; e += kF32Threads) off[e] = __ldg(l.offsets + e);
  tc_fence_before();
  __syncthreads();
  cluster_sync();                                // both CTAs' barriers are ready before anything arrives on them
  tc_fence_after();
  RowTiles rt{};
  if (kMode != kGemmGradW) rt = RowTiles{bars.before[lane], bars.before[32]};
  const int n_total = kMode == kGemmGradW ? l.E * p.m_tiles * p.n_tiles : rt.total * p.m_tiles;   // tiles
  const uint32_t tmem = bars.tmem;               // accumulator b: h h at columns 256 b, the small products at 256 b + 128
  const WaitCtx wc{&bars.abort, p.status, p.limit_ns};
  // the producer and the MMA issuer look a tile up once the first block of the one before it is on its way: at the
  // tile's own beginning the tensor cores stood still meanwhile
  auto tile_at = [&](int tile) {
    return tile < n_total ? gemm_tile<kMode, kF32K>(p, rt, off, tile) : GemmTile{};
  };

  if (warp == 0) {
    // ------------------------------------------------------------------------------- producer
    RawPlace at;
    bool ok = true;
    GemmTile next = tile_at(pair);
    for (int tile = pair; ok && tile < n_total; tile += n_pairs) {
      const GemmTile t = next;
      const int half_n = gemm_n<kMode>(t.cols) / 2;
      if (t.blocks == 0) next = tile_at(tile + n_pairs);
      for (int kb = 0; kb < t.blocks; ++kb) {
        if (!warp_wait(&bars.raw_empty[at.before()], at.before_ph(), wc)) { ok = false; break; }
        if (elect_one()) {
          uint8_t* a = raw_a + at.stage() * kRawA;
          uint8_t* b = raw_b + at.stage() * kRawB;
          const uint32_t bar = smem_u32(&bars.raw_full[at.bar]);
          // few rows: boxes of 16
          const bool few = kMode != kGemmGradW && half_n < 64;
          mbar_arrive_expect_tx(&bars.raw_full[at.bar], kRawA + (few ? half_n * (kF32K * 4) : kRawB));
          const int k0 = kb * kF32K, r = static_cast<int>(rank);
          if (kMode == kGemmGradW) {
            const int r0 = t.row0 + k0;
            tma_load_2d_pair(a, &tmA, bar, t.m * 256 + r * 128, r0);
            tma_load_2d_pair(b, &tmB, bar, t.col0 + r * half_n, r0);
          } else {
            if (kMode == kGemmGradX) {
              tma_load_3d_pair(a, &tmA, bar, t.m * 256 + r * 128, k0, t.e);
            } else if (kGated) {
              const int f0 = t.m * 128 + r * 64;
#pragma unroll
              for (int i = 0; i < 8; ++i)
                tma_load_3d_pair(a + i * 2048, &tmA, bar, k0, (i & 1) * l.n_out + f0 + (i >> 1) * 16, t.e);
            } else {
              tma_load_3d_pair(a, &tmA, bar, k0, t.m * 256 + r * 128, t.e);
            }
            const int r0 = t.row0 + r * half_n;
            if (!few) {
              tma_load_2d_pair(b, &tmB, bar, k0, r0);
            } else {
              for (int i = 0; i < half_n; i += 16) tma_load_2d_pair(b + i * (kF32K * 4), &tmB16, bar, k0, r0 + i);
            }
          }
        }
        __syncwarp();
        if (kb == 0) next = tile_at(tile + n_pairs);
        at.next();
      }
    }
  } else if (warp == 1 && rank == 0) {
    // ----------------------------------------------------------------------------- MMA issuer
    PlanePlace at;
    int acc = 0;
    uint32_t aph = 0;
    bool ok = true;
    GemmTile next = tile_at(pair);
    for (int tile = pair; ok && tile < n_total; tile += n_pairs) {
      const GemmTile t = next;
      if (t.blocks == 0) next = tile_at(tile + n_pairs);
      const uint32_t idesc = idesc_bf16(256, gemm_n<kMode>(t.cols), kAcrossA, kAcrossB);
      for (int k0 = 0; ok && k0 < t.blocks; k0 += kF32Chunk) {
        if (!warp_wait<true>(&bars.acc_empty[acc], aph ^ 1, wc)) { ok = false; break; }
        tc_fence_after();
        const uint32_t d = tmem + acc * 256;
        const int k1 = min(k0 + kF32Chunk, t.blocks);
        for (int kb = k0; kb < k1; ++kb) {
          if (!warp_wait(&bars.split_full[at.st], at.ph, wc)) { ok = false; break; }
          tc_fence_after();
          if (elect_one()) {
            const uint32_t a = smem_u32(planes_a), b = smem_u32(planes_b);
            // plane 0 h, 1 m, 2 l; the products of planes (x, y) with x + y <= 2, small ones first
            constexpr int kX[6] = {2, 0, 1, 1, 0, 0}, kY[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
            for (int c = 0; c < 6; ++c) {
#pragma unroll
              for (int s = 0; s < 2; ++s) {
                const uint32_t pa = a + plane_offset<kAcrossA, 128>(at.st, kX[c]) + s * (kAcrossA ? 2048 : 32);
                const uint32_t pb = b + plane_offset<kAcrossB, 64>(at.st, kY[c]) + s * (kAcrossB ? 2048 : 32);
                const uint64_t da = sdesc_sw128(pa, kAcrossA ? kF32K * 128 : 16, 1024);
                const uint64_t db = sdesc_sw128(pb, kAcrossB ? kF32K * 128 : 16, 1024);
                umma_bf16_pair(c == 5 ? d : d + 128, da, db, idesc, kb > k0 || s > 0 || (c > 0 && c < 5));
              }
            }
            umma_commit_pair(&bars.split_empty[at.st]);
            if (kb == k1 - 1) umma_commit_pair(&bars.acc_full[acc]);
          }
          __syncwarp();
          if (kb == 0) next = tile_at(tile + n_pairs);
          at.next();
        }
        if (++acc == 2) { acc = 0; aph ^= 1; }
      }
    }
  } else if (warp == 2 || warp == 3) {
    // ------------------- the second CTA's planes handed to the first, every other block by each of two warps
    PlanePlace at;
    bool ok = true;
    for (int tile = pair; ok && tile < n_total; tile += n_pairs) {
      const int blocks = gemm_tile<kMode, kF32K>(p, rt, off, tile).blocks;
      for (int kb = 0; kb < blocks; ++kb, at.next()) {
        if ((at.st & 1) != (warp & 1)) continue;
        ok = rank == 0 ? warp_wait<true>(&bars.split_peer[at.st], at.ph, wc) : warp_wait(&bars.split_mine[at.st], at.ph, wc);
        if (!ok) break;
        if (lane == 0) {
          if (rank == 0)
            mbar_arrive(&bars.split_full[at.st]);
          else
            mbar_arrive_peer_release(peer_smem(&bars.split_peer[at.st], 0));
        }
        __syncwarp();
      }
    }
  } else if (warp >= 4) {
    // ------------------------------------------------- splitting, and the sums one chunk behind
    const int q = warp & 3, g = (warp - 4) >> 2, tid = threadIdx.x - 128;
    const uint32_t lanes = static_cast<uint32_t>(32 * q) << 16;
    if (kMode != kGemmGradW) {
      const long long end = expert_begin(off, l.E, l.R);
      if (end < l.R) {                           // rows of no expert
        for (int which = 0; which < (l.pre ? 2 : 1); ++which) {
          uint4* o = static_cast<uint4*>(which ? l.pre : l.out);
          const int words = (which ? l.n_z : p.n_feat) / 4;
          for (long long i = end * words + static_cast<long long>(blockIdx.x) * (32 * kF32Warps) + tid;
               i < l.R * words; i += static_cast<long long>(gridDim.x) * (32 * kF32Warps))
            o[i] = make_uint4(0u, 0u, 0u, 0u);
        }
      }
    }
    float sum[32];                               // columns 32 g + j
#pragma unroll
    for (int j = 0; j < 32; ++j) sum[j] = 0.f;

    // the finished tile's sums to memory: lanes hold neighbouring features, a column is an output row (dW: a row of dW)
    auto store = [&](const GemmTile& t) {
      const int cols = t.cols - g * 32;          // of this group's columns
      if constexpr (kMode == kGemmForward) {
        const int fl = kGated ? 16 * q + (lane & 15) : 32 * q + lane;
        const int f = (t.m * 2 + static_cast<int>(rank)) * (kGated ? 64 : 128) + fl;
        const int up = lane >> 4;
        const int zf = f + (kGated ? up * l.n_out : 0);
        const bool in = f < p.n_feat;
        const float bias = l.bias && in ? __ldg(l.bias + static_cast<long long>(t.e) * l.n_z + zf) : 0.f;
        const long long row = t.row0 + g * 32;
        float* out = static_cast<float*>(l.out) + row * l.n_out + f;
        float* pre = static_cast<float*>(l.pre) + row * l.n_z + zf;
        const float* res = static_cast<const float*>(l.residual) + row * l.n_out + f;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          sum[j] += bias;
          if (l.pre && in && j < cols) pre[static_cast<long long>(j) * l.n_z] = sum[j];
        }
        if (kGated) {                            // of two columns each half of the warp finishes one
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            const float got = __shfl_xor_sync(0xffffffffu, up ? sum[j] : sum[j + 1], 16);
            const float y = act_value<kAct, false>(up ? got : sum[j]) * (up ? sum[j + 1] : got);
            if (in && j + up < cols) {
              const long long at = static_cast<long long>(j + up) * l.n_out;
              out[at] = l.residual ? y + __ldg(res + at) : y;
            }
          }
        } else {
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            if (in && j < cols) {
              const long long at = static_cast<long long>(j) * l.n_out;
              const float y = act_value<kAct, false>(sum[j]);
              out[at] = l.residual ? y + __ldg(res + at) : y;
            }
          }
        }
      } else {
        const int f = t.m * 256 + static_cast<int>(rank) * 128 + 32 * q + lane;
        const long long row = kMode == kGemmGradW ? static_cast<long long>(t.e) * l.n_z + t.col0 : t.row0;
        float* out = (kMode == kGemmGradW ? l.dW : static_cast<float*>(l.out)) + (row + g * 32) * l.n_in + f;
        const bool add = kMode == kGemmGradW && l.accumulate;
        if (f < l.n_in) {
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            if (j < cols) *out = add ? *out + sum[j] : sum[j];
            out += l.n_in;
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 32; ++j) sum[j] = 0.f;
    };

    // a chunk is split, then the one before it drained (one place each: inlined twice the sums do not fit the registers)
    const int turn = (warp - 4) / (kF32Warps / kTurns), part = tid & (kSplitThreads - 1);
    RawPlace at;
    PlanePlace to;
    int acc = 0;
    uint32_t aph = 0;
    bool ok = true;
    int tile = pair, k0 = 0;
    bool more = tile < n_total;
    GemmTile t{}, done{};                        // the chunk's tile; that of the chunk before
    if (more) t = gemm_tile<kMode, kF32K>(p, rt, off, tile);
    bool pending = false, pending_last = false;
    while (more || pending) {
      const int k1 = more ? min(k0 + kF32Chunk, t.blocks) : k0;
      for (int kb = k0; kb < k1; ++kb, at.next(), to.next()) {
        if (at.bar % kTurns != turn) continue;
        if (!warp_wait(&bars.raw_full[at.bar], at.ph, wc) ||
            !warp_wait(&bars.split_empty[to.st], to.ph ^ 1, wc)) { ok = false; break; }
        const int st = at.stage();
        const int depth = kMode == kGemmGradW && kb == t.blocks - 1 ? t.last : kF32K;
        const uint8_t* ra = raw_a + st * kRawA;
        const uint8_t* rb = raw_b + st * kRawB;
#pragma unroll
        for (int i = 0; i < 2 * kTurns; ++i)
          split_word<kAcrossA, 128>(ra, planes_a, to.st, part + i * kSplitThreads, depth);
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
          const int u = part + i * kSplitThreads;
          if (kAcrossB || (u >> 6) * 8 < gemm_n<kMode>(t.cols) / 2)     // (two warps split eight rows)
            split_word<kAcrossB, 64>(rb, planes_b, to.st, u, depth);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&bars.raw_empty[at.bar]);
          mbar_arrive(rank == 0 ? &bars.split_full[to.st] : &bars.split_mine[to.st]);
        }
      }
      if (!ok) break;
      if (pending && done.blocks > 0) {
        ok = warp_wait(&bars.acc_full[acc], aph, wc);
        if (!ok) break;
        tc_fence_after();
        if (g * 32 < done.cols) {
          float v[32];
          tmem_ld32(tmem + acc * 256 + 128 + g * 32 + lanes, v);
#pragma unroll
          for (int j = 0; j < 32; ++j) sum[j] += v[j];
          tmem_ld32(tmem + acc * 256 + g * 32 + lanes, v);
#pragma unroll
          for (int j = 0; j < 32; ++j) sum[j] += v[j];
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_peer(peer_smem(&bars.acc_empty[acc], 0));
        if (++acc == 2) { acc = 0; aph ^= 1; }
      }
      if (pending && pending_last && done.blocks > 0) store(done);
      if (kMode == kGemmGradW && pending && done.blocks == 0 && !l.accumulate)   // an expert without rows
        zero_weight_tile(l, done, static_cast<int>(rank), warp - 4, kF32Warps);
      pending = more;
      pending_last = k1 == t.blocks;
      done = t;
      k0 = k1;
      if (more && pending_last) {
        tile += n_pairs;
        k0 = 0;
        more = tile < n_total;
        if (more) t = gemm_tile<kMode, kF32K>(p, rt, off, tile);
      }
    }
    // every plane given back: no commit of the first CTA is still on its way to this one when it ends
    // (each half those that it would wait for next)
    for (int i = 0; ok && i < kPlaneStages; ++i, to.next())
      if (to.st % kTurns == turn) ok = warp_wait(&bars.split_empty[to.st], to.ph ^ 1, wc);
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

template <int kMode, int kAct, bool kGated>
cudaError_t launch(ExpertGemmParams& p, const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& b16, int n_sms,
                   cudaStream_t s) {
  static GemmResidency held;
  int pairs = 0;
  const cudaError_t e = gemm_pairs(held, k_expert_gemm_f32<kMode, kAct, kGated>, kF32Threads, kF32Smem, n_sms, &pairs);
  if (e != cudaSuccess) return e;
  pairs = gemm_split(p, static_cast<ExpertGemmMode>(kMode), 7, kMode == kGemmGradW ? 7 : 5, pairs);
  return launch_pdl(k_expert_gemm_f32<kMode, kAct, kGated>, dim3(2 * pairs), dim3(kF32Threads), kF32Smem, s, a, b, b16, p);
}

}  // namespace

cudaError_t launch_expert_gemm_f32(const ExpertLinearParams& l, ExpertGemmMode mode, uint32_t* status,
                                   uint64_t limit_ns, int n_sms, cudaStream_t s) {
  ExpertGemmParams p{};
  p.l = l;
  p.status = status;
  p.limit_ns = limit_ns;
  p.n_feat = mode == kGemmForward ? l.n_out : l.n_in;
  const int per = mode == kGemmForward && l.gated ? 128 : 256;
  p.m_tiles = (p.n_feat + per - 1) / per;
  const uint64_t R = static_cast<uint64_t>(l.R), ni = l.n_in, nz = l.n_z, E = l.E;
  CUtensorMap a, b, b16;
  bool ok;
  if (mode == kGemmGradW) {
    const uint64_t da[2] = {ni, R}, sta[1] = {ni * 4}, db[2] = {nz, R}, stb[1] = {nz * 4};
    const uint32_t boxa[2] = {128, kF32K}, boxb[2] = {64, kF32K};
    ok = encode_f32(&a, l.X, 2, da, sta, boxa) && encode_f32(&b, l.dZ, 2, db, stb, boxb);
    b16 = b;
  } else {
    const uint64_t da[3] = {ni, nz, E}, sta[2] = {ni * 4, ni * nz * 4};
    const uint32_t across[3] = {128, kF32K, 1}, along[3] = {kF32K, l.gated ? 16u : 128u, 1};
    const uint64_t depth = mode == kGemmForward ? ni : nz;
    const uint64_t db[2] = {depth, R}, stb[1] = {depth * 4};
    const uint32_t boxb[2] = {kF32K, 64}, box16[2] = {kF32K, 16};
    const void* rows = mode == kGemmForward ? l.X : l.dZ;
    ok = encode_f32(&a, l.W, 3, da, sta, mode == kGemmGradX ? across : along) &&
         encode_f32(&b, rows, 2, db, stb, boxb) && encode_f32(&b16, rows, 2, db, stb, box16);
  }
  if (!ok) return cudaErrorInvalidValue;
  if (mode == kGemmForward)
    return with_act(l.act, [&](auto act) {
      constexpr int kAct = decltype(act)::value;
      return l.gated ? launch<kGemmForward, kAct, true>(p, a, b, b16, n_sms, s)
                     : launch<kGemmForward, kAct, false>(p, a, b, b16, n_sms, s);
    });
  if (mode == kGemmGradX) return launch<kGemmGradX, SMOES_ACT_NONE, false>(p, a, b, b16, n_sms, s);
  return launch<kGemmGradW, SMOES_ACT_NONE, false>(p, a, b, b16, n_sms, s);
}

}  // namespace smoes
