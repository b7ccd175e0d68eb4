// expert_mx.cu -- the experts' products of microscaled 4-bit values on the tensor cores (tcgen05), grouped over ragged
// rows:  z = W_e x_r + b_e,  out = act(z) (or act(g) u of z = [g | u]) + residual, out in bf16.
//
// Both operands hold pairs of e2m1 codes along the depth and a power-of-two scale for every 32 of it; the tensor cores
// multiply by both scales. A CTA forms a tile of 128 features (along M) by up to kRowsMost rows (along N), in blocks of
// 256 of the depth: 128 bytes a row, in the copy engine's swizzle, as for 64 bf16 values.
//
// Scales lie in memory as they are given, [rows][n_in / 32] bytes. The tensor cores want them in tensor memory, in lane
// r % 32 and column r / 32 of row r, with four blocks' bytes in a word. A warp loads the 8 bytes of a block of 256 of four rows
// 32 apart a lane, writes their words side by side (16 bytes a lane: no bank conflicts) and hands them to the MMA issuer, which
// copies them to tensor memory ahead of the products.
//
// Ragged edges and gated layers are those of expert_gemm.cu: rows of the next expert inside a tile are other columns of
// D and are not stored; features past the expert's weights and a depth that ends inside a block are zeros of the maps (their scales
// are set to 2^-127, so no NaN scale meets a zero).
#include "expert_epilogue.cuh"
#include "expert_gemm.cuh"
#include "experts.cuh"
#include "ptx.cuh"

namespace smoes {
namespace {

constexpr int kMxScaleWarps = 4;
constexpr int kMxEpi = 2 + kMxScaleWarps;        // first epilogue warp; 0 producer, 1 MMA issuer, then the scales' warps
constexpr int kMxEpiWarps = 4 * kGemmGroups;
constexpr int kMxGemmThreads = 32 * (kMxEpi + kMxEpiWarps);
constexpr int kMxBlock = 256;                    // depth of a block: 128 bytes
constexpr int kMxA = 128 * 128;                  // a block's bytes of the features
constexpr int kRowsMost = 192;
constexpr int kMxStagesMost = 8;
constexpr uint32_t kMxRing = 4 * (kMxA + kRowsMost * 128);
constexpr uint32_t kMxScaleStage = 2 * 512 + 2 * 1024;   // of the features and of up to 256 rows: two words each
constexpr uint32_t kMxStaging = 8192;            // one epilogue group's output boxes: two chunks
constexpr uint32_t kMxSmem = 1024 + kMxRing + kMxStagesMost * kMxScaleStage + kGemmGroups * kMxStaging + kBarBytes + 4 * (kExpertsMax + 1);
static_assert(kMxSmem <= 227 * 1024, "shared memory of a CTA");
constexpr uint32_t kMxScaleCols = 2 * kRowsMost;  // tensor memory: two accumulators, then two blocks' scales
constexpr uint32_t kMxScaleSet = 24;             // 2 words x 4 columns of the features, 2 x 8 of the rows

struct MxBars {
  uint64_t full[kMxStagesMost];                  // the operands
  uint64_t scales[kMxStagesMost];                // their scales
  uint64_t empty[kMxStagesMost];
  uint64_t acc_full[2], acc_empty[2];
  uint32_t tmem;
  int abort;
  int before[33];
};
static_assert(sizeof(MxBars) <= kBarBytes, "barriers");

// Bytes [at, at + 8) of a row of n scales; what lies past the row is 0.
__device__ __forceinline__ uint2 load_scales(const uint8_t* row, int at, int n) {
  if (row == nullptr || at >= n) return make_uint2(0u, 0u);
  if ((n & 7) == 0) return __ldg(reinterpret_cast<const uint2*>(row + at));
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (at + i < n) w[i >> 2] |= static_cast<uint32_t>(__ldg(row + at + i)) << (8 * (i & 3));
  return make_uint2(w[0], w[1]);
}

template <int kAct, bool kGated>
__global__ void __launch_bounds__(kMxGemmThreads, 1)
k_expert_mx(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
            const __grid_constant__ CUtensorMap tmOut, const ExpertMxParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t* scale_ring = smem + kMxRing;
  uint8_t* staging = scale_ring + kMxStagesMost * kMxScaleStage;
  MxBars& bars = *reinterpret_cast<MxBars*>(staging + kGemmGroups * kMxStaging);
  int32_t* off = reinterpret_cast<int32_t*>(staging + kGemmGroups * kMxStaging + kBarBytes);   // [E + 1] offsets
  const ExpertLinearParams& l = p.l;
  const int warp = warp_index(), lane = threadIdx.x & 31;
  const int R = static_cast<int>(l.R);
  const AnyRows rows_of{p.tile_rows};
  const uint32_t stage_bytes = kMxA + static_cast<uint32_t>(p.tile_rows) * 128u;
  const int n_stages = min(kMxStagesMost, static_cast<int>(kMxRing / stage_bytes));
  auto stage_a = [&](int s) { return smem + s * stage_bytes; };
  auto stage_b = [&](int s) { return smem + s * stage_bytes + kMxA; };
  auto stage_scales = [&](int s) { return scale_ring + s * kMxScaleStage; };

  if (threadIdx.x == 0) {
    for (int i = 0; i < n_stages; ++i) {
      mbar_init(&bars.full[i], 1);
      mbar_init(&bars.scales[i], 1);
      mbar_init(&bars.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars.acc_full[i], 1);
      mbar_init(&bars.acc_empty[i], kMxEpiWarps);
    }
    bars.abort = 0;
    fence_mbar_init();
    tma_prefetch_desc(&tmA);
    tma_prefetch_desc(&tmB);
    tma_prefetch_desc(&tmOut);
  }
  if (warp == 2) tmem_alloc(&bars.tmem, 512);
  pdl_wait();
  pdl_trigger();
  if (warp == 3) count_row_tiles(l.offsets, l.E, R, rows_of, bars.before);
  for (int e = threadIdx.x; e <= l.E; e += kMxGemmThreads) off[e] = __ldg(l.offsets + e);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const RowTiles rt{bars.before[lane], bars.before[32]};
  const int n_total = rt.total * p.m_tiles;
  const int blocks = (l.n_in + kMxBlock - 1) / kMxBlock;
  const uint32_t tmem = bars.tmem;
  const WaitCtx wc{&bars.abort, p.status, p.limit_ns};
  struct Tile {
    int e, m, row0, rows;
  };
  auto tile_at = [&](int tile) {
    Tile t{0, 0, 0, 0};
    if (tile < n_total) {
      const int r = tile / p.m_tiles;
      t.m = tile - r * p.m_tiles;
      const RowTile row = find_row_tile(rt, off, l.E, R, rows_of, r);
      t.e = row.e;
      t.row0 = row.row0;
      t.rows = min(p.tile_rows, row.row1 - row.row0);
    }
    return t;
  };

  if (warp == 0) {
    // ------------------------------------------------------------------------------- producer
    int st = 0;
    uint32_t ph = 0;
    bool ok = true;
    Tile next = tile_at(blockIdx.x);
    for (int tile = blockIdx.x; ok && tile < n_total; tile += gridDim.x) {
      const Tile t = next;
      const int n = (t.rows + 31) & ~31;
      for (int kb = 0; kb < blocks; ++kb) {
        if (!warp_wait(&bars.empty[st], ph ^ 1, wc)) { ok = false; break; }
        if (elect_one()) {
          uint8_t* a = stage_a(st);
          uint8_t* b = stage_b(st);
          mbar_arrive_expect_tx(&bars.full[st], kMxA + n * 128u);
          const int x = kb * 128;
          if (kGated) {
            const int f0 = t.m * 64;
#pragma unroll
            for (int i = 0; i < 8; ++i)
              tma_load_3d(a + i * 2048, &tmA, &bars.full[st], x, (i & 1) * l.n_out + f0 + (i >> 1) * 16, t.e);
          } else {
            tma_load_3d(a, &tmA, &bars.full[st], x, t.m * 128, t.e);
          }
          for (int i = 0; i < n; i += 32) tma_load_2d(b + i * 128, &tmB, &bars.full[st], x, t.row0 + i);
        }
        __syncwarp();
        if (kb == 0) next = tile_at(tile + gridDim.x);
        if (++st == n_stages) { st = 0; ph ^= 1; }
      }
    }
    for (int i = 0; ok && i < n_stages; ++i) {   // every stage given back: no copy or product is in flight at the end
      ok = warp_wait(&bars.empty[st], ph ^ 1, wc);
      if (++st == n_stages) { st = 0; ph ^= 1; }
    }
  } else if (warp == 1) {
    // ----------------------------------------------------------------------------- MMA issuer
    int st = 0, acc = 0, set = 0;
    uint32_t ph = 0, aph = 0;
    bool ok = true;
    Tile next = tile_at(blockIdx.x);
    for (int tile = blockIdx.x; ok && tile < n_total; tile += gridDim.x) {
      const Tile t = next;
      const int n = (t.rows + 31) & ~31;
      if (!warp_wait(&bars.acc_empty[acc], aph ^ 1, wc)) break;
      tc_fence_after();
      const uint32_t d = tmem + acc * kRowsMost;
      for (int kb = 0; kb < blocks; ++kb) {
        if (!warp_wait(&bars.full[st], ph, wc) || !warp_wait(&bars.scales[st], ph, wc)) { ok = false; break; }
        tc_fence_after();
        if (elect_one()) {
          const uint32_t a = smem_u32(stage_a(st)), b = smem_u32(stage_b(st)), sc = smem_u32(stage_scales(st));
          const uint32_t sa = tmem + kMxScaleCols + set * kMxScaleSet, sb = sa + 8;
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            tmem_copy_scales(sa + 4 * w, sdesc_scales(sc + 512 * w));
            tmem_copy_scales(sb + 8 * w, sdesc_scales(sc + 1024 + 1024 * w));
            if (n > 128) tmem_copy_scales(sb + 8 * w + 4, sdesc_scales(sc + 1024 + 1024 * w + 512));
          }
#pragma unroll
          for (int s = 0; s < 4; ++s)              // 64 of the depth an instruction
            umma_mx4(d, sdesc_sw128(a + s * 32, 16, 1024), sdesc_sw128(b + s * 32, 16, 1024), idesc_mx4(128, n, s & 1),
                     sa + 4 * (s >> 1), sb + 8 * (s >> 1), kb > 0 || s > 0);
          umma_commit(&bars.empty[st]);
          if (kb == blocks - 1) umma_commit(&bars.acc_full[acc]);
        }
        __syncwarp();
        if (kb == 0) next = tile_at(tile + gridDim.x);
        set ^= 1;
        if (++st == n_stages) { st = 0; ph ^= 1; }
      }
      if (++acc == 2) { acc = 0; aph ^= 1; }
    }
  } else if (warp < kMxEpi) {
    // ------------------------------------------------------------------------------- scales
    const int n_scales = l.n_in / 32;
    int st = 0, turn = warp - 2;                 // blocks until this warp's next one
    uint32_t ph = 0;
    bool ok = true;
    for (int tile = blockIdx.x; ok && tile < n_total; tile += gridDim.x) {
      const Tile t = tile_at(tile);
      const int groups = (t.rows + 31) >> 5;
      const uint8_t* row[4 + kRowsMost / 32];    // of the lane's features and rows
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int r = g * 32 + lane;
        const int f = kGated ? ((r >> 4) & 1) * l.n_out + t.m * 64 + (r >> 5) * 16 + (r & 15) : t.m * 128 + r;
        row[g] = f < l.n_z ? p.w_scale + (static_cast<long long>(t.e) * l.n_z + f) * n_scales : nullptr;
      }
#pragma unroll
      for (int g = 0; g < kRowsMost / 32; ++g) {
        const int r = t.row0 + g * 32 + lane;
        row[4 + g] = g < groups && r < R ? p.x_scale + static_cast<long long>(r) * n_scales : nullptr;
      }
      for (int kb = 0; kb < blocks; ++kb) {
        if (turn == 0) {
          uint2 v[4 + kRowsMost / 32];
#pragma unroll
          for (int g = 0; g < 4 + kRowsMost / 32; ++g) v[g] = load_scales(row[g], kb * 8, n_scales);
          if (!warp_wait(&bars.empty[st], ph ^ 1, wc)) { ok = false; break; }
          uint4* out = reinterpret_cast<uint4*>(stage_scales(st)) + lane;   // 512 bytes a word of 128 rows
          out[0] = make_uint4(v[0].x, v[1].x, v[2].x, v[3].x);
          out[32] = make_uint4(v[0].y, v[1].y, v[2].y, v[3].y);
          out[64] = make_uint4(v[4].x, v[5].x, v[6].x, v[7].x);
          out[128] = make_uint4(v[4].y, v[5].y, v[6].y, v[7].y);
          if (groups > 4) {
            out[96] = make_uint4(v[8].x, v[9].x, 0u, 0u);
            out[160] = make_uint4(v[8].y, v[9].y, 0u, 0u);
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars.scales[st]);
          turn = kMxScaleWarps;
        }
        --turn;
        if (++st == n_stages) { st = 0; ph ^= 1; }
      }
    }
  } else {
    // ------------------------------------------------------------------------------- epilogue
    const int q = warp & 3, g = (warp - kMxEpi) >> 2;
    const uint32_t lanes = static_cast<uint32_t>(32 * q) << 16;
    const bool lead = (warp - kMxEpi) % 4 == 0;  // the group's warp that waits and stores
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
    const int fl = kGated ? 16 * q + (lane & 15) : 32 * q + lane;
    const bool issuer = lead && elect_one();
    int buf = 0, acc = 0;
    uint32_t aph = 0;
    for (int tile = blockIdx.x; tile < n_total; tile += gridDim.x) {
      const Tile t = tile_at(tile);
      const int f0 = t.m * width;
      const int zf = f0 + fl + (kGated ? (lane >> 4) * l.n_out : 0);
      const bool f_in = f0 + fl < l.n_out;
      const bool whole = f0 + width <= l.n_out;
      const long long ld = l.n_out;
      float bias = 0.f;
      const __nv_bfloat16* res = static_cast<const __nv_bfloat16*>(l.residual) + f0 + (fl & ~1);
      uint32_t rv[kChunkCols / 2];
      if (l.bias && f_in) bias = __ldg(l.bias + static_cast<long long>(t.e) * l.n_z + zf);
      if (!named_bar_all(kBarVote + g, 128, !lead || warp_wait(&bars.acc_full[acc], aph, wc))) break;
      tc_fence_after();
      const int chunks = (t.rows + kChunkCols - 1) / kChunkCols;
      for (int c = g; c < chunks; c += kGemmGroups) {
        const long long row = t.row0 + c * kChunkCols;
        const int rows = min(kChunkCols, t.rows - c * kChunkCols);
        if (l.residual) load_residual<kGated>(l, res + row * ld, f_in ? rows : 0, rv);
        uint8_t* boxes = staging + g * kMxStaging + buf * (kMxStaging / 2);
        float v[kChunkCols];
        tmem_ld16(tmem + acc * kRowsMost + c * kChunkCols + lanes, v);
        if (c + kGemmGroups >= chunks) {           // the accumulator's last use
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars.acc_empty[acc]);
        }
        staging_acquire(g, lead, issuer);
#pragma unroll
        for (int j = 0; j < kChunkCols; ++j) v[j] += bias;
        put_forward<kAct, kGated>(boxes, fl, v, l.residual != nullptr, rv);
        fence_proxy_async_smem();
        const bool engine = rows == kChunkCols && (whole || !kGated);
        staging_filled(g, lead, !engine);
        if (engine) {
          if (issuer)
            for (int i = 0; i < width / 64; ++i)
              if (f0 + 64 * i < l.n_out) tma_store_2d(&tmOut, boxes + i * 2048, f0 + 64 * i, static_cast<int>(row));
        } else {
          for (int i = 0; i < width / 64; ++i)
            copy_box(boxes + i * 2048, static_cast<__nv_bfloat16*>(l.out) + row * ld + f0 + 64 * i, ld, rows, l.n_out - f0 - 64 * i,
                     et & 127);
        }
        if (issuer) tma_store_commit();            // (every chunk is a group, an empty one too: staging_acquire counts them)
        buf ^= 1;
      }
      if (chunks <= g && lane == 0) mbar_arrive(&bars.acc_empty[acc]);
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
  tc_fence_after();
  if (warp == 2) tmem_dealloc(tmem, 512);
}

template <int kAct, bool kGated>
cudaError_t launch(const ExpertMxParams& p, const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& out, int n_sms,
                   cudaStream_t s) {
  auto kernel = k_expert_mx<kAct, kGated>;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kMxSmem));
  if (e != cudaSuccess) return e;
  const ExpertLinearParams& l = p.l;
  long long tiles = (l.R / p.tile_rows + (l.R < l.E ? l.R : l.E)) * p.m_tiles;   // at most, whatever the offsets are
  const int grid = tiles < 1 ? 1 : tiles < n_sms ? static_cast<int>(tiles) : n_sms;
  return launch_pdl(kernel, dim3(grid), dim3(kMxGemmThreads), kMxSmem, s, a, b, out, p);
}

}  // namespace

cudaError_t launch_expert_mx(ExpertMxParams p, int n_sms, cudaStream_t s) {
  const ExpertLinearParams& l = p.l;
  const int per = l.gated ? 64 : 128;
  p.m_tiles = (l.n_out + per - 1) / per;
  p.tile_rows = l.R <= 32 * static_cast<long long>(l.E) ? 32 : l.R <= 96 * static_cast<long long>(l.E) ? 96 : kRowsMost;
  const uint64_t R = static_cast<uint64_t>(l.R), bytes = l.n_in / 2, nz = l.n_z, E = l.E, no = l.n_out;
  const uint64_t da[3] = {bytes, nz, E}, sta[2] = {bytes, bytes * nz}, db[2] = {bytes, R}, stb[1] = {bytes};
  const uint32_t boxa[3] = {128, l.gated ? 16u : 128u, 1}, boxb[2] = {128, 32}, box_out[2] = {64, kChunkCols};
  const uint64_t dout[2] = {no, R}, stout[1] = {no * 2};
  CUtensorMap a, b, out;
  if (!encode_u8(&a, l.W, 3, da, sta, boxa) || !encode_u8(&b, l.X, 2, db, stb, boxb) || !encode_bf16(&out, l.out, 2, dout, stout, box_out))
    return cudaErrorInvalidValue;
  return with_act(l.act, [&](auto act) {
    constexpr int kAct = decltype(act)::value;
    return l.gated ? launch<kAct, true>(p, a, b, out, n_sms, s) : launch<kAct, false>(p, a, b, out, n_sms, s);
  });
}

}  // namespace smoes
