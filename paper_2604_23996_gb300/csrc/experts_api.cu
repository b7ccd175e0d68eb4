// experts_api.cu -- host side of the expert layer's calls in include/smoes.h: plan, workspace layout,
// argument checks and launches.
#include <algorithm>
#include <new>

#include "experts.cuh"

using namespace smoes;

struct smoes_experts_s {
  smoes_experts_desc desc{};
  long long R = 0;
  int n_sms = 148;
  int sort_blocks = 1;
  long long sort_per = 0;
  uint64_t limit_ns = kWaitLimitNs;
  size_t sync = 0, header_bytes = 0, counts = 0, part = 0, total = 0;   // workspace: [status | sync | ...]
};

namespace {

constexpr size_t kWsAlign = 256;
size_t align_ws(size_t x) { return (x + kWsAlign - 1) / kWsAlign * kWsAlign; }
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
smoes_status cuda_status(cudaError_t e) { return e == cudaSuccess ? SMOES_OK : SMOES_ERR_CUDA; }

smoes_status check_ws(const smoes_experts_s* P, const void* ws, size_t ws_bytes) {
  if (!ws || ws_bytes < P->total) return SMOES_ERR_WORKSPACE;
  return (reinterpret_cast<uintptr_t>(ws) & (kWsAlign - 1)) != 0 ? SMOES_ERR_ALIGNMENT : SMOES_OK;
}

// A row of `width` elements: whole 16-byte words.
smoes_status check_width(const smoes_experts_s* P, long long width) {
  if (width < 1 || width % (P->desc.dtype == SMOES_BF16 ? 8 : 4) != 0) return SMOES_ERR_INVALID_ARG;
  return width > kExpertWidthMax ? SMOES_ERR_UNSUPPORTED : SMOES_OK;
}

template <class... Ptrs>
smoes_status check_given(Ptrs... ptrs) {
  return ((ptrs == nullptr) || ...) ? SMOES_ERR_INVALID_ARG : SMOES_OK;
}
template <class... Ptrs>
smoes_status check_aligned(Ptrs... ptrs) {
  return (!aligned16(ptrs) || ...) ? SMOES_ERR_ALIGNMENT : SMOES_OK;
}

bool known_act(int act) { return act == SMOES_ACT_NONE || act == SMOES_ACT_SILU || act == SMOES_ACT_GELU; }

cudaError_t launch_product(const smoes_experts_s* P, const ExpertLinearParams& p, ExpertGemmMode mode, void* ws,
                           cudaStream_t stream) {
  uint32_t* status = static_cast<uint32_t*>(ws);
  return P->desc.dtype == SMOES_BF16 ? launch_expert_gemm(p, mode, status, P->limit_ns, P->n_sms, stream)
                                     : launch_expert_gemm_f32(p, mode, status, P->limit_ns, P->n_sms, stream);
}

ExpertRowsParams rows_params(const smoes_experts_s* P, int d) {
  ExpertRowsParams p{};
  p.T = P->desc.T;
  p.k = P->desc.k;
  p.E = P->desc.E;
  p.d = d;
  return p;
}

}  // namespace

extern "C" {

smoes_status smoes_experts_create(const smoes_experts_desc* desc, smoes_experts* out) {
  if (!desc || !out) return SMOES_ERR_INVALID_ARG;
  *out = nullptr;
  const smoes_experts_desc& d = *desc;
  if (d.T < 0 || d.E < 1 || d.k < 1 || d.max_width < 0) return SMOES_ERR_INVALID_ARG;
  if (d.dtype != SMOES_F32 && d.dtype != SMOES_BF16) return SMOES_ERR_INVALID_ARG;
  if (d.T > (1 << 20) || d.E > kExpertsMax || d.k > kMaxTopK || d.max_width > kExpertWidthMax)
    return SMOES_ERR_UNSUPPORTED;
  smoes_experts_s* P = new (std::nothrow) smoes_experts_s();
  if (!P) return SMOES_ERR_INVALID_ARG;
  P->desc = d;
  P->R = static_cast<long long>(d.T) * d.k;
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) == cudaSuccess &&
      cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && n > 0)
    P->n_sms = n;
  // sort: one block up to 8192 selections (no grid barrier), otherwise 2048 and more a block
  P->sort_blocks = P->R <= 8192 ? 1 : static_cast<int>(std::min<long long>(P->n_sms, (P->R + 2047) / 2048));
  P->sort_per = ((P->R + P->sort_blocks - 1) / P->sort_blocks + 1023) / 1024 * 1024;
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t at = o; o = align_ws(o + std::max<size_t>(bytes, 1)); return at; };
  take(16);                                        // status
  P->sync = take(16);
  P->header_bytes = o;
  P->counts = take(sizeof(int32_t) * static_cast<size_t>(P->sort_blocks) * d.E);
  P->part = take(sizeof(float) * static_cast<size_t>(act_ranges(P->n_sms) + d.E) * d.max_width);
  P->total = o;
  *out = P;
  return SMOES_OK;
}

void smoes_experts_destroy(smoes_experts P) { delete P; }

size_t smoes_experts_workspace_bytes(smoes_experts P) { return P ? P->total : 0; }

smoes_status smoes_experts_workspace_init(smoes_experts P, void* ws, size_t ws_bytes, cudaStream_t stream) {
  if (!P) return SMOES_ERR_INVALID_ARG;
  const smoes_status st = check_ws(P, ws, ws_bytes);
  if (st != SMOES_OK) return st;
  return cuda_status(cudaMemsetAsync(ws, 0, P->header_bytes, stream));
}

smoes_status smoes_experts_set_wait_limit(smoes_experts P, uint64_t limit_ns) {
  if (!P) return SMOES_ERR_INVALID_ARG;
  P->limit_ns = limit_ns ? limit_ns : kWaitLimitNs;
  return SMOES_OK;
}

smoes_status smoes_experts_read_status(smoes_experts P, const void* ws, cudaStream_t stream) {
  if (!P || !ws) return SMOES_ERR_INVALID_ARG;
  uint32_t word = 0;
  cudaError_t e = cudaStreamSynchronize(stream);
  if (e == cudaSuccess) e = cudaMemcpy(&word, ws, sizeof(word), cudaMemcpyDeviceToHost);
  if (e != cudaSuccess) return SMOES_ERR_CUDA;
  if (word & kStatusTimeout) return SMOES_ERR_DEVICE_TIMEOUT;
  return word & kStatusData ? SMOES_ERR_DATA : SMOES_OK;
}

smoes_status smoes_expert_sort(smoes_experts P, const int32_t* topk_idx, int32_t* expert_offsets, int32_t* row_slot,
                               int32_t* slot_row, void* ws, size_t ws_bytes, cudaStream_t stream) {
  if (!P) return SMOES_ERR_INVALID_ARG;
  smoes_status st = check_ws(P, ws, ws_bytes);
  if (st == SMOES_OK) st = check_given(expert_offsets);
  if (st != SMOES_OK) return st;
  if (P->R == 0) return cuda_status(cudaMemsetAsync(expert_offsets, 0, sizeof(int32_t) * (P->desc.E + 1), stream));
  st = check_given(topk_idx, row_slot, slot_row);
  if (st == SMOES_OK) st = check_aligned(topk_idx, expert_offsets, row_slot, slot_row);
  if (st != SMOES_OK) return st;
  uint8_t* b = static_cast<uint8_t*>(ws);
  ExpertSortParams p{};
  p.n = P->R;
  p.E = P->desc.E;
  p.G = P->sort_blocks;
  p.per = P->sort_per;
  p.topk_idx = topk_idx;
  p.offsets = expert_offsets;
  p.row_slot = row_slot;
  p.slot_row = slot_row;
  p.counts = reinterpret_cast<int32_t*>(b + P->counts);
  p.sync = reinterpret_cast<uint32_t*>(b + P->sync);
  p.status = reinterpret_cast<uint32_t*>(b);
  p.limit_ns = P->limit_ns;
  return cuda_status(launch_expert_sort(p, stream));
}

smoes_status smoes_expert_dispatch(smoes_experts P, const void* X, int d, const int32_t* expert_offsets,
                                   const int32_t* slot_row, void* Xs, cudaStream_t stream) {
  if (!P) return SMOES_ERR_INVALID_ARG;
  smoes_status st = check_width(P, d);
  if (st != SMOES_OK) return st;
  if (P->R == 0) return SMOES_OK;
  st = check_given(X, expert_offsets, slot_row, Xs);
  if (st == SMOES_OK) st = check_aligned(X, expert_offsets, slot_row, Xs);
  if (st != SMOES_OK) return st;
  ExpertRowsParams p = rows_params(P, d);
  p.offsets = expert_offsets;
  p.slot_row = slot_row;
  p.tokens = X;
  p.rows_out = Xs;
  return cuda_status(launch_expert_dispatch(p, P->desc.dtype == SMOES_BF16, stream));
}

static smoes_status rows_back(smoes_experts P, const void* rows, int d, const float* w, const int32_t* slot_row,
                              const void* residual, void* out, cudaStream_t stream) {
  ExpertRowsParams p = rows_params(P, d);
  p.slot_row = slot_row;
  p.rows = rows;
  p.w = w;
  p.tokens = residual;
  p.tokens_out = out;
  return cuda_status(launch_expert_combine(p, P->desc.dtype == SMOES_BF16, stream));
}

smoes_status smoes_expert_dispatch_bwd(smoes_experts P, const void* dXs, int d, const int32_t* slot_row,
                                       const void* residual, void* dX, cudaStream_t stream) {
  if (!P) return SMOES_ERR_INVALID_ARG;
  smoes_status st = check_width(P, d);
  if (st != SMOES_OK) return st;
  if (P->R == 0) return SMOES_OK;
  st = check_given(dXs, slot_row, dX);
  if (st == SMOES_OK) st = check_aligned(dXs, slot_row, residual, dX);
  return st != SMOES_OK ? st : rows_back(P, dXs, d, nullptr, slot_row, residual, dX, stream);
}

smoes_status smoes_expert_combine(smoes_experts P, const void* Ys, int d, const float* topk_w,
                                  const int32_t* slot_row, const void* residual, void* Y, cudaStream_t stream) {
  if (!P) return SMOES_ERR_INVALID_ARG;
  smoes_status st = check_width(P, d);
  if (st != SMOES_OK) return st;
  if (P->R == 0) return SMOES_OK;
  st = check_given(Ys, topk_w, slot_row, Y);
  if (st == SMOES_OK) st = check_aligned(Ys, topk_w, slot_row, residual, Y);
  return st != SMOES_OK ? st : rows_back(P, Ys, d, topk_w, slot_row, residual, Y, stream);
}

smoes_status smoes_expert_combine_bwd(smoes_experts P, const void* dY, const void* Ys, int d, const float* topk_w,
                                      const int32_t* expert_offsets, const int32_t* slot_row, void* dYs,
                                      float* d_topk_w, cudaStream_t stream) {
  if (!P) return SMOES_ERR_INVALID_ARG;
  smoes_status st = check_width(P, d);
  if (st != SMOES_OK) return st;
  if (P->R == 0) return SMOES_OK;
  st = check_given(dY, Ys, topk_w, expert_offsets, slot_row, dYs, d_topk_w);
  if (st == SMOES_OK) st = check_aligned(dY, Ys, topk_w, expert_offsets, slot_row, dYs, d_topk_w);
  if (st != SMOES_OK) return st;
  ExpertRowsParams p = rows_params(P, d);
  p.offsets = expert_offsets;
  p.slot_row = slot_row;
  p.tokens = dY;
  p.rows = Ys;
  p.w = topk_w;
  p.rows_out = dYs;
  p.dw = d_topk_w;
  return cuda_status(launch_expert_combine_bwd(p, P->desc.dtype == SMOES_BF16, stream));
}

smoes_status smoes_expert_linear(smoes_experts P, const smoes_linear_args* args, const int32_t* expert_offsets,
                                 void* out, void* pre, void* ws, size_t ws_bytes, cudaStream_t stream) {
  if (!P || !args) return SMOES_ERR_INVALID_ARG;
  const smoes_linear_args& a = *args;
  if (!known_act(a.act) || (a.gated != 0 && a.gated != 1)) return SMOES_ERR_INVALID_ARG;
  smoes_status st = check_ws(P, ws, ws_bytes);
  if (st == SMOES_OK) st = check_width(P, a.n_in);
  if (st == SMOES_OK) st = check_width(P, a.n_out);
  if (st == SMOES_OK) st = check_width(P, static_cast<long long>(a.n_out) * (a.gated ? 2 : 1));
  if (st != SMOES_OK) return st;
  if (P->R == 0) return SMOES_OK;
  st = check_given(a.X, a.W, expert_offsets, out);
  if (st == SMOES_OK) st = check_aligned(a.X, a.W, a.bias, a.residual, expert_offsets, out, pre);
  if (st != SMOES_OK) return st;
  ExpertLinearParams p{};
  p.E = P->desc.E;
  p.n_in = a.n_in;
  p.n_out = a.n_out;
  p.n_z = a.n_out * (a.gated ? 2 : 1);
  p.act = a.act;
  p.gated = a.gated;
  p.R = P->R;
  p.offsets = expert_offsets;
  p.X = a.X;
  p.W = a.W;
  p.bias = a.bias;
  p.residual = a.residual;
  p.out = out;
  p.pre = pre;
  return cuda_status(launch_product(P, p, kGemmForward, ws, stream));
}

static smoes_status act_bwd(smoes_experts P, const void* dOut, const void* pre, int n_out, int act, int gated,
                            const int32_t* expert_offsets, void* dZ, float* db, bool accumulate, void* ws,
                            size_t ws_bytes, cudaStream_t stream) {
  if (!P) return SMOES_ERR_INVALID_ARG;
  if (!known_act(act) || (gated != 0 && gated != 1)) return SMOES_ERR_INVALID_ARG;
  smoes_status st = check_ws(P, ws, ws_bytes);
  if (st == SMOES_OK) st = check_width(P, n_out);
  const long long n_z = static_cast<long long>(n_out) * (gated ? 2 : 1);
  if (st == SMOES_OK) st = check_width(P, n_z);
  if (st != SMOES_OK) return st;
  if (db && n_z > P->desc.max_width) return SMOES_ERR_WORKSPACE;
  const bool plain = act == SMOES_ACT_NONE && !gated;   // dZ is dOut
  if (plain ? (pre || dZ || !db) : false) return SMOES_ERR_INVALID_ARG;
  if (!aligned16(db)) return SMOES_ERR_ALIGNMENT;
  if (P->R == 0)
    return db && !accumulate ? cuda_status(cudaMemsetAsync(db, 0, sizeof(float) * P->desc.E * n_z, stream)) : SMOES_OK;
  st = check_given(dOut, expert_offsets);
  if (st == SMOES_OK && !plain) st = check_given(pre, dZ);
  if (st == SMOES_OK) st = check_aligned(dOut, pre, expert_offsets, dZ);
  if (st != SMOES_OK) return st;
  ExpertActParams p{};
  p.E = P->desc.E;
  p.n_out = n_out;
  p.n_z = static_cast<int>(n_z);
  p.act = act;
  p.gated = gated;
  p.R = P->R;
  p.offsets = expert_offsets;
  p.dOut = dOut;
  p.pre = pre;
  p.dZ = dZ;
  p.db = db;
  p.accumulate = accumulate ? 1 : 0;
  p.part = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + P->part);
  return cuda_status(launch_expert_act_bwd(p, P->desc.dtype == SMOES_BF16, P->n_sms, stream));
}

smoes_status smoes_expert_act_bwd(smoes_experts P, const void* dOut, const void* pre, int n_out, int act, int gated,
                                  const int32_t* expert_offsets, void* dZ, float* db, void* ws, size_t ws_bytes,
                                  cudaStream_t stream) {
  return act_bwd(P, dOut, pre, n_out, act, gated, expert_offsets, dZ, db, false, ws, ws_bytes, stream);
}

smoes_status smoes_expert_act_bwd_accumulate(smoes_experts P, const void* dOut, const void* pre, int n_out, int act,
                                             int gated, const int32_t* expert_offsets, void* dZ, float* db, void* ws,
                                             size_t ws_bytes, cudaStream_t stream) {
  if (!db) return SMOES_ERR_INVALID_ARG;
  return act_bwd(P, dOut, pre, n_out, act, gated, expert_offsets, dZ, db, true, ws, ws_bytes, stream);
}

smoes_status smoes_expert_linear_bwd(smoes_experts P, const void* dZ, const void* X, const void* W, int n_in, int n_z,
                                     const int32_t* expert_offsets, void* dX, float* dW, int accumulate_dW, void* ws,
                                     size_t ws_bytes, cudaStream_t stream) {
  if (!P || (!dX && !dW)) return SMOES_ERR_INVALID_ARG;
  smoes_status st = check_ws(P, ws, ws_bytes);
  if (st == SMOES_OK) st = check_width(P, n_in);
  if (st == SMOES_OK) st = check_width(P, n_z);
  if (st != SMOES_OK) return st;
  if (!aligned16(dW)) return SMOES_ERR_ALIGNMENT;
  if (P->R == 0) {
    if (!dW || accumulate_dW) return SMOES_OK;
    return cuda_status(cudaMemsetAsync(dW, 0, sizeof(float) * P->desc.E * static_cast<size_t>(n_z) * n_in, stream));
  }
  st = check_given(dZ, expert_offsets);
  if (st == SMOES_OK && dX) st = check_given(W);
  if (st == SMOES_OK && dW) st = check_given(X);
  if (st == SMOES_OK) st = check_aligned(dZ, X, W, expert_offsets, dX);
  if (st != SMOES_OK) return st;
  ExpertLinearParams p{};
  p.E = P->desc.E;
  p.n_in = n_in;
  p.n_out = n_z;
  p.n_z = n_z;
  p.R = P->R;
  p.offsets = expert_offsets;
  p.X = X;
  p.W = W;
  p.dZ = dZ;
  p.out = dX;
  p.dW = dW;
  p.accumulate = accumulate_dW ? 1 : 0;
  cudaError_t e = cudaSuccess;
  // (8192 x 512 x 256 in fp32 of 16 unequal experts: the two would take 41 us side by side instead of 45. A kernel that
  // begins beside the one before it has no promise of seeing what the kernels before both wrote: only its own wait on the
  // launch before gives that, and the wait takes the overlap.)
  if (dW) e = launch_product(P, p, kGemmGradW, ws, stream);
  if (e == cudaSuccess && dX) e = launch_product(P, p, kGemmGradX, ws, stream);
  return cuda_status(e);
}

static smoes_status check_mx(smoes_dtype dtype, long long rows, int n) {
  if ((dtype != SMOES_F32 && dtype != SMOES_BF16) || rows < 0 || n < 32 || n % 32 != 0) return SMOES_ERR_INVALID_ARG;
  return rows > (1ll << 31) || n > kExpertWidthMax ? SMOES_ERR_UNSUPPORTED : SMOES_OK;
}

smoes_status smoes_mx_quantise(const void* X, smoes_dtype dtype, long long rows, int n, uint8_t* codes, uint8_t* scales,
                               cudaStream_t stream) {
  smoes_status st = check_mx(dtype, rows, n);
  if (st != SMOES_OK || rows == 0) return st;
  st = check_given(X, codes, scales);
  if (st == SMOES_OK) st = check_aligned(X, codes, scales);
  return st != SMOES_OK ? st : cuda_status(launch_mx_quantise(X, dtype == SMOES_BF16, rows * n, codes, scales, stream));
}

smoes_status smoes_mx_dequantise(const uint8_t* codes, const uint8_t* scales, long long rows, int n, smoes_dtype dtype,
                                 void* X, cudaStream_t stream) {
  smoes_status st = check_mx(dtype, rows, n);
  if (st != SMOES_OK || rows == 0) return st;
  st = check_given(codes, scales, X);
  if (st == SMOES_OK) st = check_aligned(codes, scales, X);
  return st != SMOES_OK ? st : cuda_status(launch_mx_dequantise(codes, scales, rows * n, dtype == SMOES_BF16, X, stream));
}

smoes_status smoes_expert_dispatch_mx(smoes_experts P, const void* X, int d, const int32_t* expert_offsets,
                                      const int32_t* slot_row, uint8_t* codes, uint8_t* scales, cudaStream_t stream) {
  if (!P) return SMOES_ERR_INVALID_ARG;
  smoes_status st = check_mx(P->desc.dtype, P->R, d);
  if (st != SMOES_OK || P->R == 0) return st;
  st = check_given(X, expert_offsets, slot_row, codes, scales);
  if (st == SMOES_OK) st = check_aligned(X, expert_offsets, slot_row, codes, scales);
  if (st != SMOES_OK) return st;
  ExpertRowsParams p = rows_params(P, d);
  p.offsets = expert_offsets;
  p.slot_row = slot_row;
  p.tokens = X;
  p.rows_out = codes;
  return cuda_status(launch_expert_dispatch_mx(p, P->desc.dtype == SMOES_BF16, scales, stream));
}

smoes_status smoes_expert_linear_mx(smoes_experts P, const smoes_linear_mx_args* args, const int32_t* expert_offsets,
                                    void* out, void* ws, size_t ws_bytes, cudaStream_t stream) {
  if (!P || !args) return SMOES_ERR_INVALID_ARG;
  const smoes_linear_mx_args& a = *args;
  if (!known_act(a.act) || (a.gated != 0 && a.gated != 1)) return SMOES_ERR_INVALID_ARG;
  if (P->desc.dtype != SMOES_BF16) return SMOES_ERR_UNSUPPORTED;
  smoes_status st = check_ws(P, ws, ws_bytes);
  if (st == SMOES_OK) st = check_mx(P->desc.dtype, P->R, a.n_in);
  if (st == SMOES_OK) st = check_width(P, a.n_out);
  if (st == SMOES_OK) st = check_width(P, static_cast<long long>(a.n_out) * (a.gated ? 2 : 1));
  if (st != SMOES_OK || P->R == 0) return st;
  st = check_given(a.X, a.X_scales, a.W, a.W_scales, expert_offsets, out);
  if (st == SMOES_OK) st = check_aligned(a.X, a.X_scales, a.W, a.W_scales, a.bias, a.residual, expert_offsets, out);
  if (st != SMOES_OK) return st;
  ExpertMxParams p{};
  p.l.E = P->desc.E;
  p.l.n_in = a.n_in;
  p.l.n_out = a.n_out;
  p.l.n_z = a.n_out * (a.gated ? 2 : 1);
  p.l.act = a.act;
  p.l.gated = a.gated;
  p.l.R = P->R;
  p.l.offsets = expert_offsets;
  p.l.X = a.X;
  p.l.W = a.W;
  p.l.bias = a.bias;
  p.l.residual = a.residual;
  p.l.out = out;
  p.x_scale = a.X_scales;
  p.w_scale = a.W_scales;
  p.status = static_cast<uint32_t*>(ws);
  p.limit_ns = P->limit_ns;
  return cuda_status(launch_expert_mx(p, P->n_sms, stream));
}

}  // extern "C"
