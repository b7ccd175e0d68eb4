// expert_mx.cu -- the experts' products of microscaled 4-bit values on the tensor cores (tcgen05), grouped over ragged
// rows:  z = W_e x_r + b_e,  out = act(z) (or act(g) u of z = [g | u]) + residual, out in bf16.
//
// Both operands hold pairs of e2m1 codes along the depth and a power-of-two scale for every 32 of it; the tensor cores
// multiply by both scales. A pair of CTAs forms a tile of 256 features (along M, 128 in each CTA) by up to kRowsMost rows (along
// N), in blocks of 256 of the depth: 128 bytes a row, in the copy engine's swizzle, as for 64 bf16 values. Each CTA loads its half
// of both operands; the first CTA issues the products of both. (One CTA a tile of 128 x 192 reads every operand byte of the
// tile for itself: 98304 x 2048 x 2048 took 190 us without an epilogue, at 15.5 TB/s from L2.)
//
// Scales lie in memory as they are given, [rows][n_in / 32] bytes. The tensor cores want them in tensor memory: of a CTA's own
// features, and of all of the tile's rows in both CTAs. The 32 bytes of four blocks of every row (a round) come to shared memory
// by the copy engine, or where rows are not whole 16-byte words by two copying warps; four warps of each CTA, one for each
// quarter of its tensor memory's lanes, read four rows 32 apart a lane and store a block's words to one of four sets of
// columns. A set is free once the block four before is done, and the stores arrive where the block's operands do, so the MMA
// issuer waits for one barrier a block and commits to one. (Not kept, 98304 x 2048 x 2048 gated: words through shared memory
// and the tensor cores' own copy, the second CTA's released at cluster scope, 1 us a block: 237 us; the storing warps copying
// for themselves, 1000 clocks a round: 231 us; barriers and commits of the scales' own: 162 against 145.)
//
// What the second CTA's warps store to its tensor memory is complete when they arrive (tcgen05.wait::st, then the fence for a
// thread's arrival), as the accumulators' loads are in the epilogue; the arrivals and the waits for them have cluster scope. The
// first CTA's products read no shared memory that threads wrote, so the arrivals need not release it. (If they do: 378 us instead
// of 144.)
//
// Ragged edges and gated layers are those of expert_gemm.cu: rows of the next expert inside a tile are other columns of
// D and are not stored; features past the expert's weights and a depth that ends inside a block are zeros of the maps (their scales
// are set to 2^-127, so no NaN scale meets a zero).
//
// Roles of a CTA's warps: 0 and 8 producers of the features and of the rows (one for both issued for 610 clocks a block, whose
// products take 416), 1 MMA issuer (first CTA), 2-5 scales to tensor memory, 6-7 scales to shared memory, 9-24 epilogue, four
// for each quarter of the lanes that take 32-row chunks in turn.
//
// Measured: 98304 x 2048 x 2048 of 64 experts gated with silu 142-145 us (5.8 PFLOP/s; the products alone, without waiting for
// operands, 95 us: products of 64 of the depth an instruction, four times the bf16 rate at most), 98304 x 1024 x 2048 99 us (402 MB
// of output at 4 TB/s), 16384 x 4096 x 4096 84 us (6.5 PFLOP/s), 16 tokens of 6 of 64 experts, 2048 x 2048, 18 us (6.4 TB/s). Bound
// by the warps' turns: 47% of the issue slots are used, and each of scales, math, matrix stores and copies taken out gains 3 to 14
// us of 142; not by L2 (all tiles reading the same operands: 142) nor by the ring (six stages: 147). Few rows are bound by the
// weights' bytes.
#include <cmath>
#include <type_traits>

#include "expert_gemm.cuh"
#include "experts.cuh"
#include "ptx.cuh"

namespace smoes {
namespace {

constexpr int kMxScaleWarps = 4;
constexpr int kMxCopyWarps = 2;
constexpr int kMxCopy = 2 + kMxScaleWarps;       // 0 producer of the features, 1 MMA issuer, then the scales' warps
constexpr int kMxRows = kMxCopy + kMxCopyWarps;  // producer of the rows
constexpr int kMxEpi = kMxRows + 1;              // first epilogue warp
constexpr int kMxTurns = 4;                      // epilogue warps of each quarter of the lanes, on chunks in turn
constexpr int kMxEpiWarps = 4 * kMxTurns;
constexpr int kMxGemmThreads = 32 * (kMxEpi + kMxEpiWarps);
constexpr int kMxBlock = 256;                    // depth of a block: 128 bytes
constexpr int kMxA = 128 * 128;                  // a block's bytes of the features
constexpr int kRowsMost = 208;                   // (two accumulators and the scales fill the 512 columns)
constexpr int kMxStagesMost = 8;
constexpr uint32_t kMxRing = 5 * (kMxA + kRowsMost * 64);
constexpr int kMxSets = 4;                       // blocks' scales in tensor memory
constexpr uint32_t kMxSetCols = 24;              // two words of 4 columns of the features and 8 of the rows
constexpr uint32_t kMxScaleCols = 2 * kRowsMost; // behind the accumulators
constexpr int kMxGroups = 4 + (kRowsMost + 31) / 32;     // of 32 features or rows
constexpr int kMxRound = 4;                      // blocks whose scales are copied at a time: 32 bytes a row
constexpr int kMxSlots = 3;
constexpr uint32_t kMxSlot = kMxGroups * 32 * 32;
constexpr int kMxChunk = 32;                     // rows that an epilogue warp finishes at a time
constexpr uint32_t kMxStaging = 2048;            // its box of 32 features by 32 rows, or gated two of 16 features
constexpr uint32_t kMxBarBytes = 1024;
constexpr uint32_t kMxSmem = 1024 + kMxRing + kMxSlots * kMxSlot + kMxEpiWarps * kMxStaging + kMxBarBytes + 4 * (kExpertsMax + 1);
static_assert(kMxScaleCols + kMxSets * kMxSetCols <= 512, "tensor memory");
static_assert(kMxSmem <= 227 * 1024, "shared memory of a CTA");
// The pair's tiles for the epilogue, written by the rows' producer. It is at most the stages, two accumulators and the tile it
// looks up ahead of the epilogue: fewer than kMxNotes tiles, so no note is written over before it is read.
constexpr int kMxNotes = 16;
struct alignas(16) MxNote {
  int e, m, row0, rows;
};

struct MxBars {
  uint64_t full[kMxStagesMost];                  // operands and scales of both CTAs (first CTA's)
  uint64_t empty[kMxStagesMost];
  uint64_t slot_full[kMxSlots], slot_empty[kMxSlots];
  uint64_t acc_full[2], acc_empty[2];
  uint64_t note_full[kMxNotes];
  uint32_t tmem;
  int abort;
  int before[33];
  MxNote notes[kMxNotes];
};
static_assert(sizeof(MxBars) <= kMxBarBytes && kMxStagesMost + 4 < kMxNotes, "barriers");
static_assert(kMxRing / (kMxA + kRowsMost * 64) > kMxSets, "a block's scales arrive after the stage's block before is done");

// 16 scale bytes of each of kUnits rows, `step` bytes apart, to shared memory 1024 bytes apart; the first there[i] of them, zeros
// behind. Whole words of kBytes are copied; with kBytes = 0 (rows of no whole 4-byte words) they are put together from the aligned
// words that hold them. any: an aligned address that may be read. kTail: the array may end inside a word, end: where, tail: its bytes
// of that word (nothing is read behind the array).
template <int kBytes, bool kTail, int kUnits>
__device__ __forceinline__ void fetch_scales(uint32_t dst, const uint8_t* src, long long step, const int (&there)[kUnits],
                                             const uint8_t* any, const uint8_t* end, uint32_t tail) {
  if constexpr (kBytes > 0) {
#pragma unroll
    for (int i = 0; i < kUnits; ++i)
#pragma unroll
      for (int j = 0; j < 16; j += kBytes)
        cp_async<kBytes>(dst + 1024 * i + j, there[i] > j ? src + i * step + j : any, min(max(there[i] - j, 0), kBytes));
  } else {
    uint32_t w[kUnits][5];
    int skew[kUnits];
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const uint8_t* p = src + i * step;
      skew[i] = static_cast<int>(reinterpret_cast<uintptr_t>(p) & 3u);
      const uint32_t* words = reinterpret_cast<const uint32_t*>(p - skew[i]);
#pragma unroll
      for (int j = 0; j < 5; ++j) {
        w[i][j] = 0u;
        if (there[i] > 0 && 4 * j < skew[i] + there[i])
          w[i][j] = kTail && reinterpret_cast<const uint8_t*>(words + j + 1) > end ? tail : __ldg(words + j);
      }
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      uint32_t out[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int left = there[i] - 4 * j;       // bytes of this word that the row has
        out[j] = __funnelshift_r(w[i][j], w[i][j + 1], 8 * skew[i]);
        if (left < 4) out[j] &= left > 0 ? (1u << (8 * left)) - 1u : 0u;
      }
      asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};"
                   ::"r"(dst + 1024 * i), "r"(out[0]), "r"(out[1]), "r"(out[2]), "r"(out[3]) : "memory");
    }
  }
}
// Shared address of half h (16 bytes) of row r in a slot; the halves of every other four rows change places (bank conflicts).
__device__ __forceinline__ uint32_t scale_at(uint32_t slot, int r, int h) {
  return slot + static_cast<uint32_t>(r) * 32u + static_cast<uint32_t>((h ^ (r >> 2)) & 1) * 16u;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// The epilogue's sums and products go two at a time (f32x2): of the instructions that an SM issues under dsmoe_vlm's gated layer
// half were its epilogue's.
__device__ __forceinline__ void add_bias(float (&v)[16], const float (&bias)[2]) {
#pragma unroll
  for (int j = 0; j < 16; j += 2) {
    const float b = bias[(j >> 1) & 1];
    const uint64_t s = fadd2(pack2(v[j], v[j + 1]), pack2(b, b));
    v[j] = lo2(s);
    v[j + 1] = hi2(s);
  }
}
// act(v) in place.
template <int kAct>
__device__ __forceinline__ void activate(float (&v)[16]) {
#pragma unroll
  for (int j = 0; j < 16; j += 2) {
    if (kAct == SMOES_ACT_SILU) {
      const uint64_t z = pack2(v[j], v[j + 1]);
      const uint64_t w = fmul2(z, pack2(-kLog2E, -kLog2E));
      const uint64_t e = fadd2(pack2(fast_exp2(lo2(w)), fast_exp2(hi2(w))), pack2(1.f, 1.f));
      const uint64_t y = fmul2(z, pack2(fast_reciprocal(lo2(e)), fast_reciprocal(hi2(e))));
      v[j] = lo2(y);
      v[j + 1] = hi2(y);
    } else {
      v[j] = act_value<kAct, true>(v[j]);
      v[j + 1] = act_value<kAct, true>(v[j + 1]);
    }
  }
}
// act(v) u in place.
template <int kAct>
__device__ __forceinline__ void gate(float (&v)[16], const float (&u)[16]) {
  if (kAct != SMOES_ACT_NONE) activate<kAct>(v);
#pragma unroll
  for (int j = 0; j < 16; j += 2) {
    const uint64_t y = fmul2(pack2(v[j], v[j + 1]), pack2(u[j], u[j + 1]));
    v[j] = lo2(y);
    v[j + 1] = hi2(y);
  }
}

template <int kAct, bool kGated>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kMxGemmThreads, 1)
k_expert_mx(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
            const __grid_constant__ CUtensorMap tmB16, const __grid_constant__ CUtensorMap tmScaleA,
            const __grid_constant__ CUtensorMap tmScaleB, const __grid_constant__ CUtensorMap tmOut,
            const __grid_constant__ CUtensorMap tmOut16, const ExpertMxParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t* scale_ring = smem + kMxRing;
  uint8_t* staging = scale_ring + kMxSlots * kMxSlot;
  MxBars& bars = *reinterpret_cast<MxBars*>(staging + kMxEpiWarps * kMxStaging);
  int32_t* off = reinterpret_cast<int32_t*>(staging + kMxEpiWarps * kMxStaging + kMxBarBytes);   // [E + 1] offsets
  const ExpertLinearParams& l = p.l;
  const int warp = warp_index(), lane = threadIdx.x & 31;
  const int R = static_cast<int>(l.R);
  const uint32_t rank = cluster_rank();
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
  const AnyRows rows_of = p.rows_of;
  // a stage: the CTA's 128 features, then its half of the widest tile
  const uint32_t stage_bytes = kMxA + static_cast<uint32_t>(p.tile_rows) * 64u;
  const int n_stages = min(kMxStagesMost, static_cast<int>(kMxRing / stage_bytes));
  auto stage_a = [&](int s) { return smem + s * stage_bytes; };
  auto stage_b = [&](int s) { return smem + s * stage_bytes + kMxA; };

  if (threadIdx.x == 0) {
    for (int i = 0; i < n_stages; ++i) {
      mbar_init(&bars.full[i], 1 + 2 * kMxScaleWarps);
      mbar_init(&bars.empty[i], 1);
    }
    for (int i = 0; i < kMxSlots; ++i) {
      mbar_init(&bars.slot_full[i], p.scale_maps ? 1 : 32 * kMxCopyWarps);
      mbar_init(&bars.slot_empty[i], kMxScaleWarps);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars.acc_full[i], 1);
      mbar_init(&bars.acc_empty[i], 2 * kMxEpiWarps);
    }
    for (int i = 0; i < kMxNotes; ++i) mbar_init(&bars.note_full[i], 1);
    bars.abort = 0;
    fence_mbar_init();
    tma_prefetch_desc(&tmA);
    tma_prefetch_desc(&tmB);
    tma_prefetch_desc(&tmB16);
    tma_prefetch_desc(&tmScaleA);
    tma_prefetch_desc(&tmScaleB);
    tma_prefetch_desc(&tmOut);
    tma_prefetch_desc(&tmOut16);
  }
  if (warp == 2) tmem_alloc_pair(&bars.tmem, 512);
  pdl_wait();
  pdl_trigger();
  if (warp == 3) count_row_tiles(l.offsets, l.E, R, rows_of, bars.before);
  for (int e = threadIdx.x; e <= l.E; e += kMxGemmThreads) off[e] = __ldg(l.offsets + e);
  tc_fence_before();
  __syncthreads();
  cluster_sync();                                // both CTAs' barriers are ready before anything arrives on them
  tc_fence_after();
  const RowTiles rt{bars.before[lane], bars.before[32]};
  const int n_total = rt.total * p.m_tiles;
  const int blocks = (l.n_in + kMxBlock - 1) / kMxBlock;
  const uint32_t tmem = bars.tmem;
  const WaitCtx wc{&bars.abort, p.status, p.limit_ns};
  // The pair's tiles in turn, looked up by a whole warp: most are of the same expert as the one before or of one of the
  // next few; only farther ones are searched for.
  struct Tile {
    int e, m, row0, rows;
    int r, before, tiles;                        // row tile; those of the experts before e, and of e
  };
  auto settle = [&](Tile& t) {
    const int start = expert_row(off, t.e, R);
    t.row0 = start + rows_of.first(t.r - t.before);
    t.rows = min(p.tile_rows, expert_row(off, t.e + 1, R) - t.row0);
  };
  auto search = [&](Tile& t) {
    const RowTile row = find_row_tile<true>(rt, off, l.E, R, rows_of, t.r);
    t.e = row.e;
    t.before = row.before;
    t.tiles = row.tiles;
  };
  auto first_tile = [&] {
    Tile t{};
    if (pair < n_total) {
      t.r = pair / p.m_tiles;
      t.m = pair - t.r * p.m_tiles;
      search(t);
      settle(t);
    }
    return t;
  };
  const int step_r = n_pairs / p.m_tiles, step_m = n_pairs - step_r * p.m_tiles;
  auto tile_after = [&](Tile t) {
    t.r += step_r;
    t.m += step_m;
    if (t.m >= p.m_tiles) {
      t.m -= p.m_tiles;
      ++t.r;
    }
    if (t.r >= rt.total) return t;
    for (int i = 0; t.r >= t.before + t.tiles; ++i) {
      if (i == 3) {
        search(t);
        break;
      }
      t.before += t.tiles;
      ++t.e;
      t.tiles = rows_of.tiles(expert_row(off, t.e + 1, R) - expert_row(off, t.e, R));
    }
    settle(t);
    return t;
  };

  if (warp == 0 || warp == kMxRows) {
    // ------------------------------------------------------------------------------- producers
    const bool rows = warp == kMxRows;
    int st = 0, note = 0;
    uint32_t ph = 0;
    bool ok = true;
    Tile next = first_tile();
    for (int tile = pair; ok && tile < n_total; tile += n_pairs) {
      const Tile t = next;
      if (rows && lane == 0) {
        bars.notes[note] = MxNote{t.e, t.m, t.row0, t.rows};
        mbar_arrive(&bars.note_full[note]);
      }
      note = (note + 1) % kMxNotes;
      const int half = min((t.rows + 31) & ~31, p.tile_rows) / 2;
      const int r0 = t.row0 + static_cast<int>(rank) * half;
      const int f0 = t.m * (kGated ? 128 : 256) + static_cast<int>(rank) * (kGated ? 64 : 128);
      for (int kb = 0; kb < blocks; ++kb) {
        if (!warp_wait(&bars.empty[st], ph ^ 1, wc)) { ok = false; break; }
        if (elect_one()) {
          const uint32_t bar = peer_smem(&bars.full[st], 0);
          const int x = kb * 128;
          if (!rows) {
            uint8_t* a = stage_a(st);
            // the first CTA expects the bytes of both (the second one's may come before: the phase waits for this arrival)
            if (rank == 0) mbar_arrive_expect_tx(&bars.full[st], 2 * kMxA + half * 256u);
            if (kGated) {                        // 16 features of g, the same of u, the next 16 ...
#pragma unroll
              for (int i = 0; i < 4; ++i) tma_load_4d_pair(a + i * 4096, &tmA, bar, x, f0 + 16 * i, 0, t.e);
            } else {
              tma_load_4d_pair(a, &tmA, bar, x, f0, 0, t.e);
            }
          } else {
            uint8_t* b = stage_b(st);
            if (2 * half == p.tile_rows) {
              tma_load_2d_pair(b, &tmB, bar, x, r0);
            } else {
              for (int i = 0; i < half; i += 16) tma_load_2d_pair(b + i * 128, &tmB16, bar, x, r0 + i);
            }
          }
        }
        __syncwarp();
        if (kb == 0) next = tile_after(t);
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
    int st = 0, acc = 0, set = 0;
    uint32_t ph = 0, aph = 0;
    bool ok = true;
    const uint64_t a0 = sdesc_sw128(smem_u32(stage_a(0)), 16, 1024), b0 = sdesc_sw128(smem_u32(stage_b(0)), 16, 1024);
    Tile next = first_tile();
    for (int tile = pair; ok && tile < n_total; tile += n_pairs) {
      const Tile t = next;
      const int n = min((t.rows + 31) & ~31, p.tile_rows);
      const uint32_t id0 = idesc_mx4(256, n, 0), id1 = idesc_mx4(256, n, 1);
      if (!warp_wait<true>(&bars.acc_empty[acc], aph ^ 1, wc)) break;
      tc_fence_after();
      const uint32_t d = tmem + acc * kRowsMost;
      for (int kb = 0; kb < blocks; ++kb) {
        if (!warp_wait<true>(&bars.full[st], ph, wc)) { ok = false; break; }
        tc_fence_after();
        if (elect_one()) {
          const uint64_t at = (st * stage_bytes) >> 4, da = a0 + at, db = b0 + at;
          const uint32_t sa = tmem + kMxScaleCols + set * kMxSetCols;
          // 64 of the depth an instruction: 32 bytes of each row, one half of a scale word
          umma_mx4_pair(d, da, db, id0, sa, sa + 4, kb > 0);
          umma_mx4_pair(d, da + 2, db + 2, id1, sa, sa + 4, 1u);
          umma_mx4_pair(d, da + 4, db + 4, id0, sa + 12, sa + 16, 1u);
          umma_mx4_pair(d, da + 6, db + 6, id1, sa + 12, sa + 16, 1u);
          umma_commit_pair(&bars.empty[st]);
          if (kb == blocks - 1) umma_commit_pair(&bars.acc_full[acc]);
        }
        __syncwarp();
        if (kb == 0) next = tile_after(t);
        set = (set + 1) % kMxSets;
        if (++st == n_stages) { st = 0; ph ^= 1; }
      }
      if (++acc == 2) { acc = 0; aph ^= 1; }
    }
  } else if (warp >= 2 && warp < kMxCopy) {
    // ------------------------------------------------------------------- scales to tensor memory
    const uint32_t slots = smem_u32(scale_ring);
    const uint32_t cols = tmem + (static_cast<uint32_t>(32 * (warp & 3)) << 16) + kMxScaleCols;
    // A set is stored to once the products of the block kMxSets before are done (its stage's `empty`), and the store arrives at
    // the `full` of the block's own stage: with more stages than sets its phase before is over.
    int slot = 0, set = 0, st = 0, old = 0, stored = 0;
    uint32_t lph = 0, oph = 0;
    bool ok = true;
    for (int tile = pair; ok && tile < n_total; tile += n_pairs) {
      for (int k0 = 0; ok && k0 < blocks; k0 += kMxRound) {
        ok = warp_wait(&bars.slot_full[slot], lph, wc);
        const uint32_t from = slots + slot * kMxSlot;
        const int n_blocks = min(kMxRound, blocks - k0);
        uint32_t v[kMxGroups][2];                // lane's row of each group, a block's words
        auto read = [&](int b) {
#pragma unroll
          for (int g = 0; g < kMxGroups; ++g)
            asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v[g][0]), "=r"(v[g][1])
                         : "r"(scale_at(from, g * 32 + lane, b >> 1) + 8 * (b & 1)));
        };
        if (ok) read(0);
        for (int b = 0; ok && b < n_blocks; ++b) {
          if (stored < kMxSets) {
            ++stored;
          } else {
            ok = warp_wait(&bars.empty[old], oph, wc);
            if (!ok) break;
            tc_fence_after();
            if (++old == n_stages) { old = 0; oph ^= 1; }
          }
          const uint32_t to = cols + set * kMxSetCols;
          tmem_st16(to, {v[0][0], v[1][0], v[2][0], v[3][0], v[4][0], v[5][0], v[6][0], v[7][0], v[8][0], v[9][0], v[10][0], 0u,
                         v[0][1], v[1][1], v[2][1], v[3][1]});
          tmem_st8(to + 16, v[4][1], v[5][1], v[6][1], v[7][1], v[8][1], v[9][1], v[10][1], 0u);
          if (b + 1 < n_blocks) read(b + 1);     // (under the stores)
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_peer(peer_smem(&bars.full[st], 0));
          __syncwarp();
          set = (set + 1) % kMxSets;
          if (++st == n_stages) st = 0;
        }
        if (lane == 0) mbar_arrive(&bars.slot_empty[slot]);   // (every lane's words have arrived: the warp stored them)
        if (++slot == kMxSlots) { slot = 0; lph ^= 1; }
      }
    }
  } else if (warp >= kMxCopy && warp < kMxRows && (warp == kMxCopy || !p.scale_maps)) {
    // ------------------------------------------------------------------- scales to shared memory
    const int n_scales = l.n_in / 32;
    const uint8_t* x_end = p.x_scale + static_cast<long long>(R) * n_scales;
    const int x_tail = R * (n_scales & 3) & 3;   // (the weights' rows are multiples of 8: they end with a word)
    uint32_t tail = 0;
    for (int i = 0; i < x_tail; ++i) tail |= static_cast<uint32_t>(__ldg(x_end - x_tail + i)) << (8 * i);
    int slot = 0;
    uint32_t lph = 0;
    bool ok = true;
    Tile next = first_tile();
    for (int tile = pair; ok && tile < n_total; tile += n_pairs) {
      const Tile t = next;
      const int f0 = t.m * (kGated ? 128 : 256) + static_cast<int>(rank) * (kGated ? 64 : 128);
      for (int k0 = 0; k0 < blocks; k0 += kMxRound) {
        if (!warp_wait(&bars.slot_empty[slot], lph ^ 1, wc)) { ok = false; break; }
        uint8_t* to = scale_ring + slot * kMxSlot;
        if (p.scale_maps) {
          if (elect_one()) {
            uint64_t* bar = &bars.slot_full[slot];
            mbar_arrive_expect_tx(bar, (128 + p.tile_rows) * 32u);
            if (kGated) {
#pragma unroll
              for (int i = 0; i < 4; ++i) tma_load_4d(to + i * 1024, &tmScaleA, bar, k0 * 8, f0 + 16 * i, 0, t.e);
            } else {
              tma_load_4d(to, &tmScaleA, bar, k0 * 8, f0, 0, t.e);
            }
            tma_load_2d(to + 4096, &tmScaleB, bar, k0 * 8, t.row0);
          }
        } else {
          // sixteen rows at a time, two lanes a row, the warps in turn: the features' (gated: one warp g's, the other
          // u's, as the operand has them), then the rows'
          const int w = warp - kMxCopy, r = 16 * w + (lane >> 1);
          const int at = k0 * 8 + (lane & 1) * 16, there = min(max(n_scales - at, 0), 16);
          const int f = kGated ? w * l.n_out + f0 + (lane >> 1) : f0 + r, f_step = kGated ? 16 : 32;
          const uint32_t dst = scale_at(smem_u32(to), r, lane & 1);
          int have_a[4], have_b[4], have_c[3];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            have_a[i] = f + i * f_step < l.n_z ? there : 0;
            have_b[i] = 16 * w + 32 * i < t.rows && t.row0 + r + 32 * i < R ? there : 0;
            if (i < 3) have_c[i] = 16 * w + 32 * (i + 4) < t.rows && t.row0 + r + 32 * (i + 4) < R ? there : 0;
          }
          const uint8_t* a = p.w_scale + (static_cast<long long>(t.e) * l.n_z + f) * n_scales + at;
          const uint8_t* b = p.x_scale + static_cast<long long>(t.row0 + r) * n_scales + at;
          const long long n = n_scales;
          auto fetch = [&](auto bytes, auto last) {
            constexpr int kB = decltype(bytes)::value;
            constexpr bool kTail = decltype(last)::value;
            fetch_scales<kB, false>(dst, a, f_step * n, have_a, p.w_scale, nullptr, 0u);
            fetch_scales<kB, kTail>(dst + 4096, b, 32 * n, have_b, p.w_scale, x_end, tail);
            if (t.rows > 128) fetch_scales<kB, kTail>(dst + 8192, b + 128 * n, 32 * n, have_c, p.w_scale, x_end, tail);
          };
          // Words of the tile's rows (in 32s) lie past the array only where fewer than three rows follow; only there are they
          // looked at one by one (in every tile: 6007 x 1440 -> 1416 38 us with its dispatch instead of 32.5).
          const bool inside = x_tail == 0 || t.row0 + ((t.rows + 31) & ~31) + 3 <= R;
          if ((n_scales & 7) == 0) fetch(std::integral_constant<int, 8>(), std::false_type());
          else if ((n_scales & 3) == 0) fetch(std::integral_constant<int, 4>(), std::false_type());
          else if (inside) fetch(std::integral_constant<int, 0>(), std::false_type());
          else fetch(std::integral_constant<int, 0>(), std::true_type());
          if ((n_scales & 3) == 0) cp_async_arrive(&bars.slot_full[slot]); else mbar_arrive(&bars.slot_full[slot]);
        }
        __syncwarp();
        if (k0 == 0) next = tile_after(t);
        if (++slot == kMxSlots) { slot = 0; lph ^= 1; }
      }
    }
    cp_async_wait_all();
    if (p.scale_maps)                            // no copy is in flight at the end
      for (int i = 0; ok && i < kMxSlots; ++i) {
        ok = warp_wait(&bars.slot_empty[slot], lph ^ 1, wc);
        if (++slot == kMxSlots) { slot = 0; lph ^= 1; }
      }
  } else if (warp >= kMxEpi) {
    // ------------------------------------------------------------------------------- epilogue
    // Warps work alone. A warp's features are two times 16 (gated: 16, as g and as u). A 16-lane load gives a thread two
    // neighbouring rows of features lane / 4 and 8 further on; rounded and packed they are stored transposed, 8 features
    // (16 bytes) of a row at a time, to the warp's box, which the copy engine takes to memory (boxes of 64 features by four warps,
    // that met at two barriers a chunk: 6007 x 1024 -> 1416 17.5 us instead of 16.8.)
    constexpr int kHalves = kGated ? 1 : 2;
    constexpr uint32_t kRow = 32 * kHalves;      // bytes of a row of a box
    const int q = warp & 3, g = (warp - kMxEpi) >> 2;
    const uint32_t lanes = static_cast<uint32_t>(32 * q) << 16;
    const int et = threadIdx.x - 32 * kMxEpi;
    const long long end = expert_begin(off, l.E, l.R);
    if (end < l.R) {                             // rows of no expert
      const int words = l.n_out / 8;
      uint4* o = static_cast<uint4*>(l.out);
      for (long long i = end * words + static_cast<long long>(blockIdx.x) * (32 * kMxEpiWarps) + et; i < l.R * words;
           i += static_cast<long long>(gridDim.x) * (32 * kMxEpiWarps))
        o[i] = make_uint4(0u, 0u, 0u, 0u);
    }
    const int width = kGated ? 64 : 128;
    const int fw = kGated ? 16 * q : 32 * q;     // the warp's first feature among the CTA's
    uint8_t* mine = staging + (warp - kMxEpi) * kMxStaging;
    // byte of 16-byte word w of row r in a box, in the copy engine's swizzle
    auto box_at = [](int r, int w) {
      return static_cast<uint32_t>(r) * kRow + static_cast<uint32_t>((w ^ (kGated ? r >> 2 : r >> 1)) & (2 * kHalves - 1)) * 16u;
    };
    const int st_row = (lane >> 4) * 8 + (lane & 7), st_word = (lane >> 3) & 1;
    const bool issuer = elect_one();
    int buf = 0, acc = 0;
    uint32_t aph = 0;
    for (int tile = pair, i = 0; tile < n_total; tile += n_pairs, ++i) {
      if (!warp_wait(&bars.note_full[i % kMxNotes], (i / kMxNotes) & 1, wc)) break;
      const MxNote t = bars.notes[i % kMxNotes];
      const int f0 = (t.m * 2 + static_cast<int>(rank)) * width + fw;
      const long long ld = l.n_out;
      float bias[2][2] = {{0.f, 0.f}, {0.f, 0.f}};   // non-gated: of the halves; gated: of g and of u
      if (l.bias) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int f = f0 + (kGated ? 0 : 16 * h) + 8 * j + (lane >> 2);
            if (f < l.n_out) bias[h][j] = __ldg(l.bias + static_cast<long long>(t.e) * l.n_z + f + (kGated ? h * l.n_out : 0));
          }
      }
      if (!warp_wait(&bars.acc_full[acc], aph, wc)) break;
      tc_fence_after();
      const int chunks = (t.rows + kMxChunk - 1) / kMxChunk;
      for (int c = g; c < chunks; c += kMxTurns) {
        const long long row = t.row0 + c * kMxChunk;
        const int rows = min(kMxChunk, t.rows - c * kMxChunk);
        uint8_t* box = mine + (kGated ? buf * 1024 : 0);
        const uint32_t from = tmem + acc * kRowsMost + c * kMxChunk + lanes;
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
          uint32_t raw[kGated ? 2 : 1][16];      // gated: g and u; [rows 8 n][features 8 i][two rows]
          tmem_ld_16x256b_x4(from + (static_cast<uint32_t>(16 * h) << 16), raw[0]);
          if constexpr (kGated) tmem_ld_16x256b_x4(from + (16u << 16), raw[1]);
          // the residual's words, transposed as the accumulators are: [rows 8 n][features 8 i]
          uint32_t rv[4][2];
          if (l.residual) {
            const int f = f0 + 16 * h + 2 * (lane & 3);
            const __nv_bfloat16* res = static_cast<const __nv_bfloat16*>(l.residual) + (row + (lane >> 2)) * ld + f;
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
              for (int j = 0; j < 2; ++j)
                rv[n][j] = 8 * n + (lane >> 2) < rows && f + 8 * j < l.n_out
                               ? __ldg(reinterpret_cast<const uint32_t*>(res + 8 * n * ld + 8 * j)) : 0u;
          }
          tmem_ld_ready(raw[0]);
          if constexpr (kGated) tmem_ld_ready(raw[1]);
          if (h == kHalves - 1 && c + kMxTurns >= chunks) {   // the accumulator's last use
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_peer(peer_smem(&bars.acc_empty[acc], 0));
          }
          float v[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) v[j] = __uint_as_float(raw[0][j]);
          if (l.bias) add_bias(v, bias[h]);
          if constexpr (kGated) {
            float u[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) u[j] = __uint_as_float(raw[1][j]);
            if (l.bias) add_bias(u, bias[1]);
            gate<kAct>(v, u);
          } else if (kAct != SMOES_ACT_NONE) {
            activate<kAct>(v);
          }
          if (h == 0 && issuer) tma_store_wait_read<kGated ? 1 : 0>();   // the box is free again
          __syncwarp();
          if (l.residual) {
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                const uint32_t w = transpose_8x8(rv[n][j]);
                v[4 * n + 2 * j] += __uint_as_float(w << 16);
                v[4 * n + 2 * j + 1] += __uint_as_float(w & 0xffff0000u);
              }
          }
          const uint32_t at = smem_u32(box);
#pragma unroll
          for (int n = 0; n < 2; ++n)            // 16 rows
            stmatrix_x4_trans(at + box_at(16 * n + st_row, 2 * h + st_word), pack_bf16(v[8 * n], v[8 * n + 1]),
                              pack_bf16(v[8 * n + 2], v[8 * n + 3]), pack_bf16(v[8 * n + 4], v[8 * n + 5]),
                              pack_bf16(v[8 * n + 6], v[8 * n + 7]));
        }
        if (rows == kMxChunk || rows == 16) {      // the engine leaves out what lies past n_out
          fence_proxy_async_smem();
          __syncwarp();
          if (issuer && f0 < l.n_out) tma_store_2d(rows == 16 ? &tmOut16 : &tmOut, box, f0, static_cast<int>(row));
        } else {                                   // its expert's rows end inside: 16 bytes a lane
          __syncwarp();
          constexpr int kWords = 2 * kHalves;
          for (int j = lane; j < rows * kWords; j += 32) {
            const int r = j / kWords, w = j % kWords;
            if (f0 + 8 * w < l.n_out)
              *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(l.out) + (row + r) * ld + f0 + 8 * w) =
                  *reinterpret_cast<const uint4*>(box + box_at(r, w));
          }
          __syncwarp();
        }
        if (issuer) tma_store_commit();            // (every chunk is a group, an empty one too)
        if (kGated) buf ^= 1;
      }
      if (chunks <= g && lane == 0) mbar_arrive_peer(peer_smem(&bars.acc_empty[acc], 0));
      if (++acc == 2) { acc = 0; aph ^= 1; }
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

template <int kAct, bool kGated>
cudaError_t launch(ExpertMxParams& p, const CUtensorMap& a, const CUtensorMap& b16, const CUtensorMap& scale_a,
                   const CUtensorMap& out, const CUtensorMap& out16, int n_sms, cudaStream_t s) {
  static GemmResidency held;
  int pairs = 0;
  const cudaError_t e = gemm_pairs(held, k_expert_mx<kAct, kGated>, kMxGemmThreads, kMxSmem, n_sms, &pairs);
  if (e != cudaSuccess) return e;
  // Rows of a tile: the widest, unless all tiles of a narrower kind have a pair each or no expert has more rows (narrower
  // stages, more of them), as for the bf16 products.
  const ExpertLinearParams& l = p.l;
  long long tiles = 0;
  for (int rows : {32, 64, 128, kRowsMost}) {
    p.tile_rows = rows;
    tiles = (l.R / rows + (l.R < l.E ? l.R : l.E)) * p.m_tiles;   // at most, whatever the offsets are
    if (tiles <= pairs || l.R <= rows) break;
  }
  // A few rounds of the widest tiles: the width whose rounds take least, a tile counted as its rows and 64 more (measured, 6007
  // x 1024 -> 1416 with GELU and residual: 208 rows 21.3 us in 2.3 rounds, 192 21.0, 160 19.3 in 3.0, 128 19.0 in 3.7). Several
  // experts have half an unfilled tile each. (At this shape it takes 160, not 128: the cost knows rounds, not how many of a
  // tile's 32-row chunks the four epilogue warps of a quarter share out evenly.)
  if (p.tile_rows == kRowsMost && tiles < 8ll * pairs) {
    long long least = 0;
    for (int rows : {kRowsMost, 192, 160, 128, 96}) {
      const double row_tiles = l.E == 1 ? static_cast<double>((l.R + rows - 1) / rows) : static_cast<double>(l.R) / rows + 0.5 * l.E;
      const long long cost = static_cast<long long>(std::ceil(row_tiles * p.m_tiles / pairs)) * (rows + 64);
      if (least == 0 || cost < least) {
        least = cost;
        p.tile_rows = rows;
      }
    }
    tiles = (l.R / p.tile_rows + (l.R < l.E ? l.R : l.E)) * p.m_tiles;
  }
  p.rows_of = AnyRows::of(p.tile_rows);
  const uint64_t bytes = l.n_in / 2, db[2] = {bytes, static_cast<uint64_t>(l.R)}, stb[1] = {bytes};
  const uint32_t box[2] = {128, static_cast<uint32_t>(p.tile_rows) / 2};
  CUtensorMap b, scale_b;
  if (!encode_u8(&b, l.X, 2, db, stb, box)) return cudaErrorInvalidValue;
  scale_b = b;
  if (p.scale_maps) {
    const uint64_t n = l.n_in / 32, ds[2] = {n, static_cast<uint64_t>(l.R)}, sts[1] = {n};
    const uint32_t boxs[2] = {32, static_cast<uint32_t>(p.tile_rows)};
    if (!encode_u8(&scale_b, p.x_scale, 2, ds, sts, boxs)) return cudaErrorInvalidValue;
  }
  pairs = tiles < 1 ? 1 : tiles < pairs ? static_cast<int>(tiles) : pairs;
  return launch_pdl(k_expert_mx<kAct, kGated>, dim3(2 * pairs), dim3(kMxGemmThreads), kMxSmem, s, a, b, b16, scale_a, scale_b, out,
                    out16, p);
}

}  // namespace

cudaError_t launch_expert_mx(ExpertMxParams p, int n_sms, cudaStream_t s) {
  const ExpertLinearParams& l = p.l;
  const int per = l.gated ? 128 : 256;
  p.m_tiles = (l.n_out + per - 1) / per;
  const uint64_t R = static_cast<uint64_t>(l.R), bytes = l.n_in / 2, nz = l.n_z, E = l.E, no = l.n_out;
  // the weights as [E][g, u][n_out] (one of the two where there is no gate)
  const uint64_t parts = l.gated ? 2 : 1, da[4] = {bytes, no, parts, E}, sta[3] = {bytes, bytes * no, bytes * nz}, db[2] = {bytes, R}, stb[1] = {bytes};
  const uint32_t rows_a = l.gated ? 16 : 128, boxa[4] = {128, rows_a, static_cast<uint32_t>(parts), 1}, box16[2] = {128, 16}, width = l.gated ? 16u : 32u, box_out[2] = {width, kMxChunk},
                 box_out16[2] = {width, 16};
  const uint64_t dout[2] = {no, R}, stout[1] = {no * 2};
  CUtensorMap a, b16, out, out16;
  if (!encode_u8(&a, l.W, 4, da, sta, boxa) || !encode_u8(&b16, l.X, 2, db, stb, box16) ||
      !encode_bf16(&out, l.out, 2, dout, stout, box_out) || !encode_bf16(&out16, l.out, 2, dout, stout, box_out16))
    return cudaErrorInvalidValue;
  // rows of scales of whole 16-byte words: the copy engine's
  p.scale_maps = l.n_in % 512 == 0;
  CUtensorMap scale_a = a;
  if (p.scale_maps) {
    const uint64_t n = l.n_in / 32, ds[4] = {n, no, parts, E}, sts[3] = {n, n * no, n * nz};
    const uint32_t boxs[4] = {32, rows_a, static_cast<uint32_t>(parts), 1};
    if (!encode_u8(&scale_a, p.w_scale, 4, ds, sts, boxs)) return cudaErrorInvalidValue;
  }
  return with_act(l.act, [&](auto act) {
    constexpr int kAct = decltype(act)::value;
    return l.gated ? launch<kAct, true>(p, a, b16, scale_a, out, out16, n_sms, s)
                   : launch<kAct, false>(p, a, b16, scale_a, out, out16, n_sms, s);
  });
}

}  // namespace smoes
