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
// stop at the 16 rows that hold the end, and a warp of each CTA clears the rows behind it in shared memory before
// they are issued (multiplying them by zero would let infinities of the next expert in). The products of the first CTA
// read what the second cleared: handed over at cluster scope, which takes about 1 us, and the tile's first block, so that
// it passes under the products of the tile before.
//
// Roles of a CTA's warps: 0 producer, 1 MMA issuer (first CTA), 2 tensor memory and the clearing, 4-19
// epilogue, in four groups that take 16-column chunks in turn (two groups on 32 columns: 131072 x 144 x 1024 of 64
// experts with silu and pre 134 instead of 107 us). Two accumulators of 256 columns: the epilogue of a tile runs
// under the next tile's products.
//
// Measured, equal experts, before the power limit sets in: 98304 x 2048 x 2048 of 64 experts 447 us forward and dX
// (1.84 PFLOP/s), 520 dW (which writes 1.07 GB), 16384 x 8192 x 2048 282 us (1.95 PFLOP/s). A layer of this size runs
// at the power limit: the same calls back to back take 10 to 15% longer. Otherwise bound by the products; small depths
// (n_in below 500 or so) by the epilogue, few rows by the weights' bytes.
#include "expert_gemm.cuh"
#include "experts.cuh"
#include "ptx.cuh"

namespace smoes {
namespace {

constexpr int kGemmThreads = 640;
constexpr int kGemmEpiWarps = 16;
constexpr int kGemmGroups = 4;                   // of four epilogue warps
constexpr int kChunkCols = 16;                   // columns of D that a group finishes at a time
constexpr int kGemmStagesMost = 8;
constexpr uint32_t kGemmRing = 5 * 32768;        // operand stages: five of 256 columns, eight of 64
constexpr int kGemmK = 64;                       // depth of a block: 128 bytes of bf16
constexpr uint32_t kGemmHalf = 128 * kGemmK * 2; // one CTA's operand of a block: 16 KB
// dW: rows summed by the tensor cores before the sum moves to fp32 registers. The tensor cores cut each
// addition off towards zero: relative error 4.7e-7 after 512 products, 1.5e-6 after 1536, 9e-6 after 8192.
constexpr int kGemmChunk = 8;                    // blocks of 64 rows

constexpr uint32_t kGemmStaging = 16384;         // one epilogue group's output boxes: two chunks of 8 KB
// alignment, operands, output boxes, barriers, [E + 1] offsets
constexpr uint32_t kGemmSmem = 1024 + kGemmRing + kGemmGroups * kGemmStaging + kBarBytes + 4 * (kExpertsMax + 1);
static_assert(kGemmSmem <= 227 * 1024, "shared memory of a CTA");

struct GemmBars {
  uint64_t full[kGemmStagesMost];                    // operands of both CTAs (first CTA's)
  uint64_t empty[kGemmStagesMost];
  uint64_t tail[kGemmStagesMost];                    // this CTA's operands of an expert's last rows, to be cleared
  uint64_t acc_full[2], acc_empty[2];
  uint32_t tmem;
  int abort;
  int before[33];                                // row tiles (count_row_tiles)
};
static_assert(sizeof(GemmBars) <= kBarBytes, "barriers");

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// A chunk is 16 columns of D (a feature per lane, an output row per column) by a CTA's 128 features. It leaves
// through shared memory as boxes of 64 features by 16 rows, 128 bytes a row in the copy engine's swizzle:
// out's boxes (two, gated one), then at 4 KB those of pre (two; gated one of g and one of u). A lane rounds two columns
// into one word, exchanges it with its neighbour and picks two neighbouring features of one row out of both; rows 4 (2,
// 6) apart are written at a time, whose swizzled words lie in different banks. Stored from the lanes, 4 bytes
// each, the 32-byte pieces of pre made dsmoe_vlm's gated layer take 557 us instead of 446 without pre.

// Shared addresses of a lane's words: its features f & ~1 and the next in box row 4 odd, with the row's swizzle;
// word i of four rows c + i lies at (at ^ i << 4) + (c + i) * 128 (c a multiple of 8: the swizzle is the row's low
// three bits, and those of i and 4 do not meet).
__device__ __forceinline__ uint32_t pair_address(const uint8_t* boxes, int f) {
  const int odd = f & 1;
  return smem_u32(boxes) + (f >> 6) * 2048 + sw128_offset(4 * odd, (f & 63) - odd);
}
// One lane's values of rows `row` and row + 4 (x0, x4) to the boxes, with its neighbour's.
__device__ __forceinline__ void put_pair(uint32_t at, int row, float x0, float x4, uint32_t pick) {
  const uint32_t own = pack_bf16(x0, x4);
  const uint32_t w = __byte_perm(own, __shfl_xor_sync(0xffffffffu, own, 1), pick);
  asm volatile("st.shared.u32 [%0], %1;" ::"r"((at ^ ((row & 3) << 4)) + row * 128), "r"(w) : "memory");
}
// Even lanes take the low halves (row `row`), odd ones the high halves (row + 4), the lower feature first.
__device__ __forceinline__ uint32_t pair_pick() { return (threadIdx.x & 1) ? 0x3276u : 0x5410u; }

// One column of D a register; f: the lane's feature among the 128 of the boxes.
__device__ __forceinline__ void put_chunk(uint8_t* boxes, int f, const float (&v)[kChunkCols]) {
  const uint32_t at = pair_address(boxes, f), pick = pair_pick();
#pragma unroll
  for (int i = 0; i < kChunkCols / 2; ++i) {
    const int c = (i >> 2) * 8 + (i & 3);
    put_pair(at, c, v[c], v[c + 4], pick);
  }
}

// The residual of a chunk in words of two features, rows as put_pair writes them. res: that of the chunk's first row at
// the lane's even feature, read for `rows` rows (none where the feature does not exist).
template <bool kGated>
__device__ __forceinline__ void load_residual(const ExpertLinearParams& l, const __nv_bfloat16* res, int rows,
                                              uint32_t (&rv)[kChunkCols / 2]) {
  const int odd = threadIdx.x & 1, up = (threadIdx.x >> 4) & 1;
#pragma unroll
  for (int i = 0; i < kChunkCols / (kGated ? 4 : 2); ++i) {
    const int c = kGated ? (i >> 1) * 8 + (i & 1) + 2 * up + 4 * odd : (i >> 2) * 8 + (i & 3) + 4 * odd;
    rv[i] = c < rows ? __ldg(reinterpret_cast<const uint32_t*>(res + c * static_cast<long long>(l.n_out))) : 0u;
  }
}
// Adds one of its words (and the neighbour's) to the lane's values of the two rows. half: 0x3244 in odd lanes, 0x1044
// in even ones (the word's high or low half as the upper half of a float).
__device__ __forceinline__ void add_residual(float& x0, float& x4, uint32_t w, uint32_t half) {
  const bool odd = threadIdx.x & 1;
  const uint32_t got = __shfl_xor_sync(0xffffffffu, w, 1);
  x0 += __uint_as_float(__byte_perm(odd ? got : w, 0u, half));
  x4 += __uint_as_float(__byte_perm(odd ? w : got, 0u, half));
}

// z (bias added) of a chunk to out, in shared memory, by whole warps. f: the lane's feature among the CTA's; rv: its
// residual, when there is one.
template <int kAct, bool kGated>
__device__ __forceinline__ void put_forward(uint8_t* boxes, int f, float (&v)[kChunkCols], bool residual,
                                            const uint32_t (&rv)[kChunkCols / 2]) {
  const uint32_t pick = pair_pick(), half = (threadIdx.x & 1) ? 0x3244u : 0x1044u;
  uint32_t at = pair_address(boxes, f);
  if (!kGated) {
    if (kAct != SMOES_ACT_NONE) {
#pragma unroll
      for (int c = 0; c < kChunkCols; ++c) v[c] = act_value<kAct, true>(v[c]);
    }
    if (residual) {
#pragma unroll
      for (int i = 0; i < kChunkCols / 2; ++i) add_residual(v[(i >> 2) * 8 + (i & 3)], v[(i >> 2) * 8 + (i & 3) + 4], rv[i], half);
    }
    put_chunk(boxes, f, v);
    return;
  }
  // gated: lanes 0-15 hold g, 16-31 u; of columns c and c + 2 each half finishes one
  const int up = (threadIdx.x >> 4) & 1;
  float y[kChunkCols / 2];                       // columns 4 (i / 2) + i % 2 + 2 up
#pragma unroll
  for (int i = 0; i < kChunkCols / 2; ++i) {
    const int c = (i >> 1) * 4 + (i & 1);
    const float got = __shfl_xor_sync(0xffffffffu, up ? v[c] : v[c + 2], 16);
    const float g = up ? got : v[c], u = up ? v[c + 2] : got;
    y[i] = act_value<kAct, true>(g) * u;
  }
  if (residual) {
#pragma unroll
    for (int i = 0; i < kChunkCols / 4; ++i) add_residual(y[(i >> 1) * 4 + (i & 1)], y[(i >> 1) * 4 + (i & 1) + 2], rv[i], half);
  }
  at = (at ^ (up << 5)) + up * 256;              // the half's rows are two further down: the swizzle's bit of 2 with it
#pragma unroll
  for (int i = 0; i < kChunkCols / 4; ++i) {
    const int a = (i >> 1) * 4 + (i & 1);
    put_pair(at, (i >> 1) * 8 + (i & 1), y[a], y[a + 2], pick);
  }
}

// The group's staging between its four warps: they fill a chunk's half and arrive; warp 0 of the group waits for them and
// hands the half to the copy engine. Before the next chunk but one goes into the same half, warp 0 has seen it read and
// says so when it begins that chunk itself; so the others run up to a chunk ahead instead of meeting at every chunk.
constexpr int kBarVote = 1, kBarFull = 1 + kGemmGroups, kBarFree = 1 + 2 * kGemmGroups;   // + group
__device__ __forceinline__ void staging_acquire(int g, bool first_warp, bool issuer) {
  if (first_warp) {
    if (issuer) tma_store_wait_read<1>();        // all but the chunk before this one
    __syncwarp();
    named_bar_arrive(kBarFree + g, 128);
  } else {
    named_bar(kBarFree + g, 128);
  }
}
// all: every warp waits (to copy the chunk itself), not just the first.
__device__ __forceinline__ void staging_filled(int g, bool first_warp, bool all) {
  if (first_warp || all)
    named_bar(kBarFull + g, 128);
  else
    named_bar_arrive(kBarFull + g, 128);
}

// Rows [0, rows) of one box to memory, for a chunk that the copy engine would write past: its expert's rows end
// inside, or g's features end inside the box and u's follow. by 128 threads, 16 bytes each. base: row 0, the
// box's first feature; n: features that exist.
__device__ __forceinline__ void copy_box(const uint8_t* box, __nv_bfloat16* base, long long stride, int rows, int n) {
  for (int i = threadIdx.x & 127; i < rows * 8; i += 128) {
    const int r = i >> 3, w = i & 7;
    if (w * 8 < n) *reinterpret_cast<uint4*>(base + r * stride + w * 8) = *reinterpret_cast<const uint4*>(box + r * 128 + ((w ^ (r & 7)) << 4));
  }
}

template <int kMode, int kAct, bool kGated>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kGemmThreads, 1)
k_expert_gemm(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
              const __grid_constant__ CUtensorMap tmB16, const __grid_constant__ CUtensorMap tmOut,
              const __grid_constant__ CUtensorMap tmPre, const ExpertGemmParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t* staging = smem + kGemmRing;
  GemmBars& bars = *reinterpret_cast<GemmBars*>(staging + kGemmGroups * kGemmStaging);
  int32_t* off = reinterpret_cast<int32_t*>(staging + kGemmGroups * kGemmStaging + kBarBytes);   // [E + 1] offsets
  const ExpertLinearParams& l = p.l;
  const int warp = warp_index(), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;

  // a stage: A's 128 features, then B's half of the widest tile; as many as fit
  const uint32_t stage_bytes = kGemmHalf + (64u << p.tile_shift);
  const int n_stages = min(kGemmStagesMost, static_cast<int>(kGemmRing / stage_bytes));
  auto stage_a = [&](int s) { return smem + s * stage_bytes; };
  auto stage_b = [&](int s) { return smem + s * stage_bytes + kGemmHalf; };

  if (threadIdx.x == 0) {
    for (int i = 0; i < n_stages; ++i) {
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
    tma_prefetch_desc(&tmB16);
    tma_prefetch_desc(&tmOut);
    if (kMode == kGemmForward) tma_prefetch_desc(&tmPre);
  }
  if (warp == 2) tmem_alloc_pair(&bars.tmem, 512);
  pdl_wait();
  pdl_trigger();
  if (kMode != kGemmGradW && warp == 3) count_row_tiles(l.offsets, l.E, static_cast<int>(l.R), p.tile_shift, bars.before);
  for (int e = threadIdx.x; e <= l.E; e += kGemmThreads) off[e] = __ldg(l.offsets + e);
  tc_fence_before();
  __syncthreads();
  cluster_sync();                                // both CTAs' barriers are ready before anything arrives on them
  tc_fence_after();
  RowTiles rt{};
  if (kMode != kGemmGradW) rt = RowTiles{bars.before[lane], bars.before[32]};
  const int n_total = kMode == kGemmGradW ? l.E * p.m_tiles * p.n_tiles : rt.total * p.m_tiles;   // tiles
  const uint32_t tmem = bars.tmem;
  const WaitCtx wc{&bars.abort, p.status, p.limit_ns};
  // the producer and the MMA issuer look a tile up once the first block of the one before it is on its way: at the
  // tile's own beginning the tensor cores stood still meanwhile
  auto tile_at = [&](int tile) {
    return tile < n_total ? gemm_tile<kMode, kGemmK>(p, rt, off, tile) : GemmTile{};
  };

  if (warp == 0) {
    // ------------------------------------------------------------------------------- producer
    int st = 0;
    uint32_t ph = 0;
    bool ok = true;
    GemmTile next = tile_at(pair);
    for (int tile = pair; ok && tile < n_total; tile += n_pairs) {
      const GemmTile t = next;
      const int half_n = gemm_n<kMode>(t.cols) / 2;
      if (t.blocks == 0) next = tile_at(tile + n_pairs);
      for (int kb = 0; kb < t.blocks; ++kb) {
        if (!warp_wait(&bars.empty[st], ph ^ 1, wc)) { ok = false; break; }
        if (elect_one()) {
          uint8_t* a = stage_a(st);
          uint8_t* b = stage_b(st);
          if (kMode == kGemmGradW) {
            const int boxes = half_n / 64;
            const uint32_t bytes = kGemmHalf + boxes * 8192u;
            const int r0 = t.row0 + (kb == 0 ? t.blocks - 1 : kb - 1) * kGemmK;   // the last rows first
            uint32_t bar;
            if (kb == 0 && (t.last & 15)) {
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
              if (kGated) {
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
            const int r0 = t.row0 + static_cast<int>(rank) * half_n;
            if (half_n == 128) {
              tma_load_2d_pair(b, &tmB, bar, k0, r0);
            } else {
              for (int i = 0; i < half_n; i += 16) tma_load_2d_pair(b + i * 128, &tmB16, bar, k0, r0 + i);
            }
          }
        }
        __syncwarp();
        if (kb == 0) next = tile_at(tile + n_pairs);
        if (++st == n_stages) { st = 0; ph ^= 1; }
      }
    }
    // every stage given back: no commit of the first CTA is still on its way to this one when it ends
    for (int i = 0; ok && i < n_stages; ++i) {
      ok = warp_wait(&bars.empty[st], ph ^ 1, wc);
      if (++st == n_stages) { st = 0; ph ^= 1; }
    }
  } else if (warp == 1 && rank == 0) {
    // ----------------------------------------------------------------------------- MMA issuer
    int st = 0, acc = 0;
    uint32_t ph = 0, aph = 0;
    bool ok = true;
    constexpr bool kMajorA = kMode != kGemmForward, kMajorB = kMode == kGemmGradW;   // along M / N in memory
    GemmTile next = tile_at(pair);
    for (int tile = pair; ok && tile < n_total; tile += n_pairs) {
      const GemmTile t = next;
      if (t.blocks == 0) next = tile_at(tile + n_pairs);
      const uint32_t idesc = idesc_bf16(256, gemm_n<kMode>(t.cols), kMajorA, kMajorB);
      const int chunk = kMode == kGemmGradW ? kGemmChunk : t.blocks;
      for (int k0 = 0; ok && k0 < t.blocks; k0 += chunk) {
        if (!warp_wait(&bars.acc_empty[acc], aph ^ 1, wc)) { ok = false; break; }
        tc_fence_after();
        const uint32_t d = tmem + acc * 256;
        const int k1 = min(k0 + chunk, t.blocks);
        for (int kb = k0; kb < k1; ++kb) {
          // an expert's last rows: warps of both CTAs have cleared what follows them
          const bool cleared = kMode == kGemmGradW && kb == 0 && (t.last & 15);
          if (!(cleared ? warp_wait<true>(&bars.full[st], ph, wc) : warp_wait(&bars.full[st], ph, wc))) { ok = false; break; }
          tc_fence_after();
          if (elect_one()) {
            const uint32_t a = smem_u32(stage_a(st)), b = smem_u32(stage_b(st));
            const int steps = kMode == kGemmGradW && kb == 0 ? (t.last + 15) >> 4 : 4;
            for (int s = 0; s < steps; ++s) {
              const uint64_t da = kMajorA ? sdesc_sw128(a + s * 2048, 8192, 1024) : sdesc_sw128(a + s * 32, 16, 1024);
              const uint64_t db = kMajorB ? sdesc_sw128(b + s * 2048, 8192, 1024) : sdesc_sw128(b + s * 32, 16, 1024);
              umma_bf16_pair(d, da, db, idesc, kb > k0 || s > 0);
            }
            umma_commit_pair(&bars.empty[st]);
            if (kb == k1 - 1) umma_commit_pair(&bars.acc_full[acc]);
          }
          __syncwarp();
          if (kb == 0) next = tile_at(tile + n_pairs);
          if (++st == n_stages) { st = 0; ph ^= 1; }
        }
        if (++acc == 2) { acc = 0; aph ^= 1; }
      }
    }
  } else if (warp == 2 && kMode == kGemmGradW) {
    // ------------------------------------------------- dW: clears what follows an expert's last row
    int st = 0;
    uint32_t phases = 0;                         // bit s: parity of tail[s]
    for (int tile = pair; tile < n_total; tile += n_pairs) {
      const GemmTile t = gemm_tile<kMode, kGemmK>(p, rt, off, tile);
      if (t.blocks == 0) continue;
      const int s = st;
      st = (st + t.blocks) % n_stages;
      if (!(t.last & 15)) continue;
      if (!warp_wait(&bars.tail[s], (phases >> s) & 1, wc)) break;
      phases ^= 1u << s;
      // rows [last, round_up(last, 16)) of every 64-column box, 8 lanes a row of 128 bytes
      const int boxes = 2 + gemm_n<kMode>(t.cols) / 128;
      uint8_t* box = lane < 16 ? stage_a(s) + (lane >> 3) * 8192 : stage_b(s) + ((lane >> 3) - 2) * 8192;
      if ((lane >> 3) < boxes)
        for (int r = t.last; r & 15; ++r) *reinterpret_cast<uint4*>(box + r * 128 + (lane & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
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
      const long long end = expert_begin(off, l.E, l.R);
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
    int buf = 0;                                 // the chunk's half of the group's staging
    const bool issuer = q == 0 && elect_one();   // issues the group's stores
    int acc = 0;
    uint32_t aph = 0;
    bool ok = true;
    for (int tile = pair; ok && tile < n_total; tile += n_pairs) {
      const GemmTile t = gemm_tile<kMode, kGemmK>(p, rt, off, tile);
      if constexpr (kMode == kGemmGradW) {
        if (t.blocks == 0) {                     // an expert without rows
          if (!l.accumulate) zero_weight_tile(l, t, static_cast<int>(rank), warp - 4, kGemmEpiWarps);
          continue;
        }
        float sum[4][16];                        // columns 64 g + 16 c + i
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 16; ++i) sum[c][i] = 0.f;
        for (int k0 = 0; k0 < t.blocks; k0 += kGemmChunk) {
          ok = named_bar_all(kBarVote + g, 128, q != 0 || warp_wait(&bars.acc_full[acc], aph, wc));
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int col = g * 64 + c * 16;
            if (col < t.cols) {
              float v[16];
              tmem_ld16(tmem + acc * 256 + col + lanes, v);
#pragma unroll
              for (int i = 0; i < 16; ++i) sum[c][i] += v[i];
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_peer(peer_smem(&bars.acc_empty[acc], 0));
          if (++acc == 2) { acc = 0; aph ^= 1; }
        }
        // [16 rows of n_z][128 features] a chunk, to the copy engine, which leaves out what lies past n_z and n_in
        if (!ok) break;
        const int i0 = t.m * 256 + static_cast<int>(rank) * 128;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int col = g * 64 + c * 16;
          if (col >= t.cols) break;
          float* box = reinterpret_cast<float*>(staging + g * kGemmStaging + buf * (kGemmStaging / 2));
          staging_acquire(g, q == 0, issuer);
#pragma unroll
          for (int j = 0; j < 16; ++j) box[j * 128 + 32 * q + lane] = sum[c][j];
          fence_proxy_async_smem();
          staging_filled(g, q == 0, false);
          if (issuer && i0 < l.n_in) {
            if (l.accumulate)
              tma_add_3d(&tmOut, box, i0, t.col0 + col, t.e);
            else
              tma_store_3d(&tmOut, box, i0, t.col0 + col, t.e);
          }
          if (issuer) tma_store_commit();        // (every chunk is a group, an empty one too: staging_acquire counts them)
          buf ^= 1;
        }
      } else {
        // the CTA's first feature (f0) and its width, the lane's among them (fl), and of z forward (zf)
        constexpr bool gated = kGated;
        const int width = gated ? 64 : 128;
        const int f0 = (t.m * 2 + static_cast<int>(rank)) * width;
        const int fl = gated ? 16 * q + (lane & 15) : 32 * q + lane;
        const int zf = f0 + fl + (gated ? (lane >> 4) * l.n_out : 0);
        const bool f_in = f0 + fl < p.n_feat;
        const bool whole = f0 + width <= p.n_feat;
        const long long ld = p.n_feat;
        float bias = 0.f;
        const __nv_bfloat16* res = static_cast<const __nv_bfloat16*>(l.residual) + f0 + (fl & ~1);
        uint32_t rv[kChunkCols / 2];
        if (kMode == kGemmForward && l.bias && f_in) bias = __ldg(l.bias + static_cast<long long>(t.e) * l.n_z + zf);
        // one warp of the group waits for the products, the others for it; one answer for all four
        ok = named_bar_all(kBarVote + g, 128, q != 0 || warp_wait(&bars.acc_full[acc], aph, wc));
        if (!ok) break;
        tc_fence_after();
        const int chunks = (t.cols + kChunkCols - 1) / kChunkCols;
        for (int c = g; c < chunks; c += kGemmGroups) {
          const long long row = t.row0 + c * kChunkCols;
          const int rows = min(kChunkCols, t.cols - c * kChunkCols);
          if (kMode == kGemmForward && l.residual) load_residual<kGated>(l, res + row * ld, f_in ? rows : 0, rv);
          uint8_t* boxes = staging + g * kGemmStaging + buf * (kGemmStaging / 2);
          float v[kChunkCols];
          tmem_ld16(tmem + acc * 256 + c * kChunkCols + lanes, v);
          if (c + kGemmGroups >= chunks) {                 // the accumulator's last use
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_peer(peer_smem(&bars.acc_empty[acc], 0));
          }
          staging_acquire(g, q == 0, issuer);
          if (kMode == kGemmForward) {
#pragma unroll
            for (int j = 0; j < kChunkCols; ++j) v[j] += bias;
            if (l.pre) put_chunk(boxes + 4096, gated ? fl + (lane >> 4) * 64 : fl, v);
            put_forward<kAct, kGated>(boxes, fl, v, l.residual != nullptr, rv);
          } else {
            put_chunk(boxes, fl, v);
          }
          fence_proxy_async_smem();
          const int n_out_boxes = width / 64;
          const bool engine = rows == kChunkCols && (whole || !gated);
          staging_filled(g, q == 0, !engine);
          if (engine) {
            if (issuer) {
              for (int i = 0; i < n_out_boxes; ++i)
                if (f0 + 64 * i < p.n_feat) tma_store_2d(&tmOut, boxes + i * 2048, f0 + 64 * i, static_cast<int>(row));
              if (kMode == kGemmForward && l.pre)
                for (int i = 0; i < 2; ++i) {
                  const int x = gated ? f0 + i * l.n_out : f0 + 64 * i;
                  if (x < l.n_z) tma_store_2d(&tmPre, boxes + 4096 + i * 2048, x, static_cast<int>(row));
                }
            }
          } else {
            for (int i = 0; i < n_out_boxes; ++i)
              copy_box(boxes + i * 2048, static_cast<__nv_bfloat16*>(l.out) + row * ld + f0 + 64 * i, ld, rows,
                       p.n_feat - f0 - 64 * i);
            if (kMode == kGemmForward && l.pre)
              for (int i = 0; i < 2; ++i) {
                const int f = gated ? f0 : f0 + 64 * i;
                copy_box(boxes + 4096 + i * 2048, static_cast<__nv_bfloat16*>(l.pre) + row * l.n_z + f + (gated ? i * l.n_out : 0),
                         l.n_z, rows, p.n_feat - f);
              }
          }
          if (issuer) tma_store_commit();        // (every chunk is a group, an empty one too: staging_acquire counts them)
          buf ^= 1;
        }
        if (chunks <= g && lane == 0) mbar_arrive_peer(peer_smem(&bars.acc_empty[acc], 0));
        if (++acc == 2) { acc = 0; aph ^= 1; }
      }
    }
    if (issuer) tma_store_wait_all<0>();
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
cudaError_t launch(ExpertGemmParams& p, const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& b16,
                   const CUtensorMap& out, const CUtensorMap& pre, int n_sms, cudaStream_t s) {
  static GemmResidency held;
  int pairs = 0;
  const cudaError_t e = gemm_pairs(held, k_expert_gemm<kMode, kAct, kGated>, kGemmThreads, kGemmSmem, n_sms, &pairs);
  if (e != cudaSuccess) return e;
  pairs = gemm_split(p, static_cast<ExpertGemmMode>(kMode), 8, kMode == kGemmGradW ? 7 : 6, pairs);
  return launch_pdl(k_expert_gemm<kMode, kAct, kGated>, dim3(2 * pairs), dim3(kGemmThreads), kGemmSmem, s, a, b, b16, out, pre, p);
}

}  // namespace

cudaError_t launch_expert_gemm(const ExpertLinearParams& l, ExpertGemmMode mode, uint32_t* status,
                               uint64_t limit_ns, int n_sms, cudaStream_t s) {
  ExpertGemmParams p{};
  p.l = l;
  p.status = status;
  p.limit_ns = limit_ns;
  p.n_feat = mode == kGemmForward ? l.n_out : l.n_in;
  const int per = mode == kGemmForward && l.gated ? 128 : 256;
  p.m_tiles = (p.n_feat + per - 1) / per;
  const uint64_t R = static_cast<uint64_t>(l.R), ni = l.n_in, nz = l.n_z, E = l.E;
  CUtensorMap a, b, b16, out, pre;
  bool ok;
  if (mode == kGemmGradW) {
    const uint64_t da[2] = {ni, R}, sta[1] = {ni * 2}, db[2] = {nz, R}, stb[1] = {nz * 2};
    const uint32_t box[2] = {64, 64};
    ok = encode_bf16(&a, l.X, 2, da, sta, box) && encode_bf16(&b, l.dZ, 2, db, stb, box);
    const uint64_t dout[3] = {ni, nz, E}, stout[2] = {ni * 4, ni * nz * 4};
    const uint32_t boxout[3] = {128, 16, 1};
    ok = ok && encode_f32(&out, l.dW, 3, dout, stout, boxout);
    b16 = pre = b;
  } else {
    const uint64_t da[3] = {ni, nz, E}, sta[2] = {ni * 2, ni * nz * 2};
    const uint32_t boxa[3] = {64, mode == kGemmGradX ? 64u : l.gated ? 16u : 128u, 1};
    const uint64_t depth = mode == kGemmForward ? ni : nz;
    const uint64_t db[2] = {depth, R}, stb[1] = {depth * 2};
    const uint32_t box[2] = {64, 128}, box16[2] = {64, 16};
    const void* rows = mode == kGemmForward ? l.X : l.dZ;
    ok = encode_bf16(&a, l.W, 3, da, sta, boxa) && encode_bf16(&b, rows, 2, db, stb, box) &&
         encode_bf16(&b16, rows, 2, db, stb, box16);
    const uint64_t nf = p.n_feat, dout[2] = {nf, R}, stout[1] = {nf * 2}, dpre[2] = {nz, R}, stpre[1] = {nz * 2};
    const uint32_t box_out[2] = {64, kChunkCols};
    ok = ok && encode_bf16(&out, l.out, 2, dout, stout, box_out);
    pre = out;
    if (l.pre) ok = ok && encode_bf16(&pre, l.pre, 2, dpre, stpre, box_out);
  }
  if (!ok) return cudaErrorInvalidValue;
  if (mode == kGemmForward)
    return with_act(l.act, [&](auto act) {
      constexpr int kAct = decltype(act)::value;
      return l.gated ? launch<kGemmForward, kAct, true>(p, a, b, b16, out, pre, n_sms, s)
                     : launch<kGemmForward, kAct, false>(p, a, b, b16, out, pre, n_sms, s);
    });
  if (mode == kGemmGradX) return launch<kGemmGradX, SMOES_ACT_NONE, false>(p, a, b, b16, out, pre, n_sms, s);
  return launch<kGemmGradW, SMOES_ACT_NONE, false>(p, a, b, b16, out, pre, n_sms, s);
}

}  // namespace smoes
