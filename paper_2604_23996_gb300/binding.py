"""ctypes binding of the SMoES C ABI (include/smoes.h).

Argument marshalling only: every computation runs in ``lib/libsmoes.so``. Functions carry the
C names; tensors are passed as torch CUDA tensors (their data pointers) or None. Importing this
module fails loudly when the library has not been built: there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import numpy as np
import torch

from .build import LIB

if not os.path.exists(LIB):
    raise ImportError(f"SMoES CUDA library not built ({LIB}); run __graft_entry__.build()")
_lib = C.CDLL(LIB)

SMOES_OK = 0
STATUS_NAMES = {0: "SMOES_OK", -1: "SMOES_ERR_INVALID_ARG", -2: "SMOES_ERR_UNSUPPORTED",
                -3: "SMOES_ERR_ALIGNMENT", -4: "SMOES_ERR_WORKSPACE", -5: "SMOES_ERR_CUDA",
                -6: "SMOES_ERR_DEVICE_TIMEOUT", -7: "SMOES_ERR_DATA"}
SMOES_F32, SMOES_BF16 = 0, 1
SMOES_GATE_SOFTMAX, SMOES_GATE_SIGMOID = 0, 1
SMOES_ACT_NONE, SMOES_ACT_SILU, SMOES_ACT_GELU = 0, 1, 2
SMOES_SCORE_PROVIDED, SMOES_SCORE_GAUSS, SMOES_SCORE_ATTN, SMOES_SCORE_GMM = 0, 1, 2, 3
(SMOES_CALL_ROUTER_FWD, SMOES_CALL_ROUTER_FWD_PERMUTE, SMOES_CALL_ROUTER_BWD, SMOES_CALL_BIN_PERMUTE,
 SMOES_CALL_ATTN_SCORE) = 0, 1, 2, 3, 4


class SmoesError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {STATUS_NAMES.get(code, code)} ({smoes_status_string(code)})")
        self.code = code


class RouterDesc(C.Structure):
    _fields_ = [("T", C.c_int), ("d", C.c_int), ("E", C.c_int), ("k", C.c_int),
                ("n_bins", C.c_int), ("n_samples", C.c_int), ("dtype", C.c_int),
                ("sample_offsets_host", C.POINTER(C.c_int32)),
                ("expert_bin_host", C.POINTER(C.c_int32)), ("renorm_topk", C.c_int),
                ("attn_max_heads", C.c_int), ("gate", C.c_int), ("score_bias", C.c_void_p),
                ("mi_topk_mask", C.c_int)]


class GaussArgs(C.Structure):
    _fields_ = [("X", C.c_void_p), ("mu", C.c_void_p), ("var", C.c_void_p), ("tau", C.c_float)]


class AttnArgs(C.Structure):
    _fields_ = [("Q", C.c_void_p), ("K", C.c_void_p), ("B", C.c_int), ("H", C.c_int),
                ("S", C.c_int), ("hd", C.c_int), ("is_vision", C.c_void_p), ("m_prev", C.c_void_p),
                ("key_bias", C.c_void_p), ("sm_scale", C.c_float), ("causal", C.c_int),
                ("xattn_norm", C.c_void_p), ("x_norm", C.c_void_p)]


class GmmArgs(C.Structure):
    _fields_ = [("X", C.c_void_p), ("n_components", C.c_int), ("log_pi", C.c_void_p),
                ("mu", C.c_void_p), ("var", C.c_void_p), ("tau", C.c_float)]


class ScoreArgs(C.Structure):
    _fields_ = [("gauss", GaussArgs), ("attn", AttnArgs), ("gmm", GmmArgs)]


class ExpertsDesc(C.Structure):
    _fields_ = [("T", C.c_int), ("E", C.c_int), ("k", C.c_int), ("dtype", C.c_int), ("max_width", C.c_int)]


class LinearArgs(C.Structure):
    _fields_ = [("X", C.c_void_p), ("W", C.c_void_p), ("bias", C.c_void_p), ("residual", C.c_void_p),
                ("n_in", C.c_int), ("n_out", C.c_int), ("act", C.c_int), ("gated", C.c_int)]


_vp, _i, _f, _sz = C.c_void_p, C.c_int, C.c_float, C.c_size_t
_sig = {
    "smoes_plan_create": (_i, [C.POINTER(RouterDesc), C.POINTER(_vp)]),
    "smoes_plan_destroy": (None, [_vp]),
    "smoes_workspace_bytes": (_sz, [_vp]),
    "smoes_workspace_init": (_i, [_vp, _vp, _sz, _vp]),
    "smoes_status_string": (C.c_char_p, [_i]),
    "smoes_plan_set_wait_limit": (_i, [_vp, C.c_uint64]),
    "smoes_call_launches": (_i, [_vp, _i]),
    "smoes_read_device_status": (_i, [_vp, _vp, _vp, C.POINTER(C.c_int32)]),
    "smoes_modality_score": (_i, [_vp, _i, C.POINTER(ScoreArgs), _vp, _vp, _sz, _vp]),
    "smoes_router_fwd": (_i, [_vp, _vp, _vp, _vp, C.POINTER(GaussArgs), _vp, _vp, _vp, _vp, _vp,
                              _vp, _vp, _vp, _sz, _vp]),
    "smoes_router_fwd_permute": (_i, [_vp, _vp, _vp, _vp, C.POINTER(GaussArgs), _vp, _vp, _vp, _vp,
                                      _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz,
                                      _vp]),
    "smoes_router_bwd": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _f, _vp, _i, _vp, _vp, _vp, _sz, _vp]),
    "smoes_bin_permute": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "smoes_bin_permute_noalloc": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "smoes_gaussian_stats_update": (_i, [_vp, _vp, _vp, C.c_double, _vp, _vp, _vp, _vp, _vp, _vp,
                                         _sz, _vp]),
    "smoes_adaptive_bins": (_i, [_vp, _vp, C.c_double, _vp, _vp, _vp, _vp]),
    "smoes_bin_balance": (_i, [_vp, _vp, _f, _vp, _vp, _vp, _vp, _sz, _vp]),
    "smoes_experts_create": (_i, [C.POINTER(ExpertsDesc), C.POINTER(_vp)]),
    "smoes_experts_destroy": (None, [_vp]),
    "smoes_experts_workspace_bytes": (_sz, [_vp]),
    "smoes_experts_workspace_init": (_i, [_vp, _vp, _sz, _vp]),
    "smoes_experts_set_wait_limit": (_i, [_vp, C.c_uint64]),
    "smoes_experts_read_status": (_i, [_vp, _vp, _vp]),
    "smoes_expert_sort": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "smoes_expert_dispatch": (_i, [_vp, _vp, _i, _vp, _vp, _vp, _vp]),
    "smoes_expert_dispatch_bwd": (_i, [_vp, _vp, _i, _vp, _vp, _vp, _vp]),
    "smoes_expert_combine": (_i, [_vp, _vp, _i, _vp, _vp, _vp, _vp, _vp]),
    "smoes_expert_combine_bwd": (_i, [_vp, _vp, _vp, _i, _vp, _vp, _vp, _vp, _vp, _vp]),
    "smoes_expert_linear": (_i, [_vp, C.POINTER(LinearArgs), _vp, _vp, _vp, _vp, _sz, _vp]),
    "smoes_expert_act_bwd": (_i, [_vp, _vp, _vp, _i, _i, _i, _vp, _vp, _vp, _vp, _sz, _vp]),
    "smoes_expert_act_bwd_accumulate": (_i, [_vp, _vp, _vp, _i, _i, _i, _vp, _vp, _vp, _vp, _sz, _vp]),
    "smoes_expert_linear_bwd": (_i, [_vp, _vp, _vp, _vp, _i, _i, _vp, _vp, _vp, _i, _vp, _sz, _vp]),
    "smoes_attention_fwd": (_i, [_vp, C.POINTER(AttnArgs), _vp, _i, _vp, _vp, _vp, _sz, _vp]),
}
for _name, (_res, _args) in _sig.items():
    _fn = getattr(_lib, _name)
    _fn.restype = _res
    _fn.argtypes = _args


def exported_symbols():
    return list(_sig)


def _p(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream=None):
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


def _check(code: int, what: str):
    if code != SMOES_OK:
        raise SmoesError(code, what)


def smoes_status_string(code: int) -> str:
    return _lib.smoes_status_string(code).decode()


def smoes_plan_create(T, d, E, k, n_bins, sample_offsets, expert_bin, dtype, renorm_topk=0,
                      attn_max_heads=0, gate=0, score_bias=None, mi_topk_mask=0):
    """Returns (status, plan handle). sample_offsets [B+1] and expert_bin [E] are host arrays."""
    offs = np.ascontiguousarray(np.asarray(sample_offsets, dtype=np.int32))
    eb = np.ascontiguousarray(np.asarray(expert_bin, dtype=np.int32))
    desc = RouterDesc(T, d, E, k, n_bins, max(len(offs) - 1, 0), dtype,
                      offs.ctypes.data_as(C.POINTER(C.c_int32)),
                      eb.ctypes.data_as(C.POINTER(C.c_int32)), renorm_topk, attn_max_heads,
                      int(gate), _p(score_bias), int(mi_topk_mask))
    h = C.c_void_p()
    code = _lib.smoes_plan_create(C.byref(desc), C.byref(h))
    return code, h


def smoes_plan_set_wait_limit(plan, limit_ns: int) -> int:
    return _lib.smoes_plan_set_wait_limit(plan, int(limit_ns))


def smoes_call_launches(plan, call: int) -> int:
    """Kernel launches one call makes on this plan (host query)."""
    return _lib.smoes_call_launches(plan, int(call))


def smoes_plan_destroy(plan):
    _lib.smoes_plan_destroy(plan)


def smoes_workspace_bytes(plan) -> int:
    return int(_lib.smoes_workspace_bytes(plan))


def smoes_workspace_init(plan, ws: torch.Tensor, stream=None) -> int:
    return _lib.smoes_workspace_init(plan, _p(ws), ws.numel() * ws.element_size(), _stream(stream))


def smoes_read_device_status(plan, ws: torch.Tensor, stream=None):
    n = C.c_int32(0)
    code = _lib.smoes_read_device_status(plan, _p(ws), _stream(stream), C.byref(n))
    return code, int(n.value)


def smoes_modality_score(plan, mode, M, ws, X=None, mu=None, var=None, tau=0.0, attn=None,
                         gmm=None, stream=None) -> int:
    """attn: dict with Q, K, B, H, S, hd, is_vision | m_prev, key_bias, sm_scale, causal,
    xattn_norm, x_norm (tensors or scalars)."""
    args = ScoreArgs()
    args.gauss = GaussArgs(_p(X), _p(mu), _p(var), float(tau))
    if attn is not None:
        a = attn
        args.attn = AttnArgs(_p(a["Q"]), _p(a["K"]), a["B"], a["H"], a["S"], a["hd"],
                             _p(a.get("is_vision")), _p(a.get("m_prev")), _p(a.get("key_bias")),
                             float(a["sm_scale"]), int(a.get("causal", 1)),
                             _p(a.get("xattn_norm")), _p(a.get("x_norm")))
    if gmm is not None:
        args.gmm = GmmArgs(_p(gmm["X"]), int(gmm["n_components"]), _p(gmm["log_pi"]), _p(gmm["mu"]),
                           _p(gmm["var"]), float(gmm.get("tau", 0.0)))
    return _lib.smoes_modality_score(plan, mode, C.byref(args), _p(M), _p(ws),
                                     ws.numel() * ws.element_size(), _stream(stream))


def smoes_router_fwd(plan, X, W, M_in, gauss, M_out, topk_idx, topk_w, bin_prob, joint, mi, loss,
                     ws, stream=None) -> int:
    """gauss: None (M_in given) or dict(mu=..., var=..., tau=...)."""
    g = None
    if gauss is not None:
        g = GaussArgs(None, _p(gauss["mu"]), _p(gauss["var"]), float(gauss.get("tau", 0.0)))
    return _lib.smoes_router_fwd(plan, _p(X), _p(W), _p(M_in), None if g is None else C.byref(g),
                                 _p(M_out), _p(topk_idx), _p(topk_w), _p(bin_prob), _p(joint),
                                 _p(mi), _p(loss), _p(ws), ws.numel() * ws.element_size(),
                                 _stream(stream))


def smoes_router_fwd_permute(plan, X, W, M_in, gauss, M_out, topk_idx, topk_w, bin_prob, joint, mi,
                             loss, home, is_vision, bin_offsets, perm_token, perm_mask, dispatch,
                             expert_counts, ws, stream=None) -> int:
    """smoes_router_fwd and smoes_bin_permute of its top-k in one call (one launch on bf16)."""
    g = None
    if gauss is not None:
        g = GaussArgs(None, _p(gauss["mu"]), _p(gauss["var"]), float(gauss.get("tau", 0.0)))
    return _lib.smoes_router_fwd_permute(plan, _p(X), _p(W), _p(M_in),
                                         None if g is None else C.byref(g), _p(M_out),
                                         _p(topk_idx), _p(topk_w), _p(bin_prob), _p(joint),
                                         _p(mi), _p(loss), _p(home), _p(is_vision),
                                         _p(bin_offsets), _p(perm_token), _p(perm_mask),
                                         _p(dispatch), _p(expert_counts), _p(ws),
                                         ws.numel() * ws.element_size(), _stream(stream))


def smoes_router_bwd(plan, X, W, M, topk_idx, d_topk_w, loss_scale, dW, accumulate_dW, dX,
                     dlogits, ws, stream=None) -> int:
    return _lib.smoes_router_bwd(plan, _p(X), _p(W), _p(M), _p(topk_idx), _p(d_topk_w),
                                 float(loss_scale), _p(dW), int(accumulate_dW), _p(dX),
                                 _p(dlogits), _p(ws), ws.numel() * ws.element_size(),
                                 _stream(stream))


def smoes_bin_permute(plan, topk_idx, home, is_vision, bin_offsets, perm_token, perm_mask,
                      dispatch, expert_counts, ws, stream=None) -> int:
    return _lib.smoes_bin_permute(plan, _p(topk_idx), _p(home), _p(is_vision), _p(bin_offsets),
                                  _p(perm_token), _p(perm_mask), _p(dispatch), _p(expert_counts),
                                  _p(ws), ws.numel() * ws.element_size(), _stream(stream))


def smoes_bin_permute_noalloc(plan, topk_idx, home, is_vision, bin_offsets, perm_token, perm_mask,
                              dispatch, expert_counts, stream=None) -> int:
    """The permutation without a workspace (scratch inside the library), for callers that cannot
    allocate device memory; see include/smoes.h for its limits and sharing rules."""
    return _lib.smoes_bin_permute_noalloc(plan, _p(topk_idx), _p(home), _p(is_vision),
                                          _p(bin_offsets), _p(perm_token), _p(perm_mask),
                                          _p(dispatch), _p(expert_counts), _stream(stream))


def smoes_gaussian_stats_update(plan, X, is_vision, beta, N, S_mu, S_var, mu, var, ws,
                                stream=None) -> int:
    return _lib.smoes_gaussian_stats_update(plan, _p(X), _p(is_vision), float(beta), _p(N), _p(S_mu),
                                            _p(S_var), _p(mu), _p(var), _p(ws),
                                            ws.numel() * ws.element_size(), _stream(stream))


def _attn_args(a):
    return AttnArgs(_p(a["Q"]), _p(a["K"]), a["B"], a["H"], a["S"], a["hd"], _p(a.get("is_vision")),
                    _p(a.get("m_prev")), _p(a.get("key_bias")), float(a["sm_scale"]),
                    int(a.get("causal", 1)), _p(a.get("xattn_norm")), _p(a.get("x_norm")))


def smoes_attention_fwd(plan, attn, V, n_kv_heads, O, M, ws, stream=None) -> int:
    """Attention forward with the vision score (O and M); attn as for smoes_modality_score."""
    args = _attn_args(attn)
    return _lib.smoes_attention_fwd(plan, C.byref(args), _p(V), int(n_kv_heads), _p(O), _p(M), _p(ws),
                                    ws.numel() * ws.element_size(), _stream(stream))


def smoes_bin_balance(plan, topk_idx, loss_scale, loss_bal, ws, f_e=None, P_e=None, stream=None) -> int:
    return _lib.smoes_bin_balance(plan, _p(topk_idx), float(loss_scale), _p(loss_bal), _p(f_e),
                                  _p(P_e), _p(ws), ws.numel() * ws.element_size(), _stream(stream))


def smoes_adaptive_bins(plan, expert_counts, beta, C_bar, expert_bin, f_spec=None, stream=None) -> int:
    return _lib.smoes_adaptive_bins(plan, _p(expert_counts), float(beta), _p(C_bar), _p(expert_bin),
                                    _p(f_spec), _stream(stream))


# The expert layer's calls are made by ``Experts``, with addresses as plain integers (a layer of a few tokens takes less
# time on the GPU than the marshalling of its arguments). What a plan needs besides:

def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _raw(stream):
    return (torch.cuda.current_stream() if stream is None else stream).cuda_stream


def smoes_experts_create(T, E, k, dtype, max_width=0):
    """Returns (status, plan handle) of an expert layer."""
    desc = ExpertsDesc(T, E, k, dtype, max_width)
    h = C.c_void_p()
    code = _lib.smoes_experts_create(C.byref(desc), C.byref(h))
    return code, h


def smoes_experts_destroy(plan):
    _lib.smoes_experts_destroy(plan)


def smoes_experts_workspace_bytes(plan) -> int:
    return int(_lib.smoes_experts_workspace_bytes(plan))


def smoes_experts_workspace_init(plan, ws, stream=None) -> int:
    return _lib.smoes_experts_workspace_init(plan, _ptr(ws), ws.numel() * ws.element_size(), _raw(stream))


def smoes_experts_set_wait_limit(plan, limit_ns: int) -> int:
    return _lib.smoes_experts_set_wait_limit(plan, int(limit_ns))


# ----------------------------------------------------------------------------- convenience

class Router:
    """Owns one plan and its workspace (torch-allocated) and the output buffers of one layer.

    Pure plumbing around the C calls above: allocation with torch, status checks, and the
    fwd -> bwd -> permute sequence.
    """

    def __init__(self, T, d, E, k, n_bins, sample_offsets, expert_bin, dtype=SMOES_BF16,
                 renorm_topk=0, attn_max_heads=0, device="cuda", gate=0, score_bias=None,
                 mi_topk_mask=0):
        code, self.plan = smoes_plan_create(T, d, E, k, n_bins, sample_offsets, expert_bin, dtype,
                                            renorm_topk, attn_max_heads, gate, score_bias,
                                            mi_topk_mask)
        _check(code, "smoes_plan_create")
        self.T, self.d, self.E, self.k, self.K = T, d, E, k, n_bins
        self.B = len(sample_offsets) - 1
        self.device = device
        nbytes = smoes_workspace_bytes(self.plan)
        self.ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
        _check(smoes_workspace_init(self.plan, self.ws), "smoes_workspace_init")
        dev = device
        self.topk_idx = torch.empty((T, k), dtype=torch.int32, device=dev)
        self.topk_w = torch.empty((T, k), dtype=torch.float32, device=dev)
        self.bin_prob = torch.empty((T, n_bins), dtype=torch.float32, device=dev)
        self.joint = torch.empty((max(self.B, 1), 2, n_bins), dtype=torch.float32, device=dev)
        self.mi = torch.empty(max(self.B, 1), dtype=torch.float32, device=dev)
        self.loss = torch.empty(1, dtype=torch.float32, device=dev)
        self.M = torch.empty((T, 2), dtype=torch.float32, device=dev)
        cap = T * min(k, n_bins)
        self.bin_offsets = torch.empty(n_bins + 1, dtype=torch.int32, device=dev)
        self.perm_token = torch.empty(max(cap, 1), dtype=torch.int32, device=dev)
        self.perm_mask = torch.empty(max(cap, 1), dtype=torch.int32, device=dev)
        self.dispatch = torch.empty((n_bins, n_bins), dtype=torch.int32, device=dev)
        self.expert_counts = torch.empty((2, E), dtype=torch.int32, device=dev)

    def __del__(self):
        try:
            smoes_plan_destroy(self.plan)
        except Exception:
            pass

    def forward(self, X, W, M_in=None, mu=None, var=None, tau=0.0, bin_prob=True, stream=None):
        gauss = None if M_in is not None else dict(mu=mu, var=var, tau=tau)
        code = smoes_router_fwd(self.plan, X, W, M_in, gauss, None if M_in is not None else self.M,
                                self.topk_idx, self.topk_w, self.bin_prob if bin_prob else None,
                                self.joint, self.mi, self.loss, self.ws, stream)
        _check(code, "smoes_router_fwd")

    def forward_permute(self, X, W, M_in=None, mu=None, var=None, tau=0.0, bin_prob=True,
                        is_vision=None, home=None, stream=None):
        """forward() then permute() of its top-k, fused into one launch on bf16 plans."""
        gauss = None if M_in is not None else dict(mu=mu, var=var, tau=tau)
        code = smoes_router_fwd_permute(
            self.plan, X, W, M_in, gauss, None if M_in is not None else self.M, self.topk_idx,
            self.topk_w, self.bin_prob if bin_prob else None, self.joint, self.mi, self.loss, home,
            is_vision, self.bin_offsets, self.perm_token, self.perm_mask, self.dispatch,
            self.expert_counts if is_vision is not None else None, self.ws, stream)
        _check(code, "smoes_router_fwd_permute")

    def backward(self, X, W, M, dW, dX=None, dlogits=None, loss_scale=1.0, d_topk_w=None,
                 accumulate=False, stream=None):
        code = smoes_router_bwd(self.plan, X, W, M, self.topk_idx, d_topk_w, loss_scale, dW,
                                accumulate, dX, dlogits, self.ws, stream)
        _check(code, "smoes_router_bwd")

    def permute(self, is_vision=None, home=None, topk_idx=None, stream=None):
        code = smoes_bin_permute(self.plan, self.topk_idx if topk_idx is None else topk_idx, home,
                                 is_vision, self.bin_offsets, self.perm_token, self.perm_mask,
                                 self.dispatch, self.expert_counts if is_vision is not None else None,
                                 self.ws, stream)
        _check(code, "smoes_bin_permute")

    def modality_score(self, mode, M, **kw):
        code = smoes_modality_score(self.plan, mode, M, self.ws, **kw)
        _check(code, "smoes_modality_score")

    def device_status(self, stream=None):
        code, n_absent = smoes_read_device_status(self.plan, self.ws, stream)
        return code, n_absent


class Experts:
    """The expert layer behind a router: one plan, its workspace and the maps of its last ``sort``.

    ``T`` tokens of ``k`` selections over ``E`` experts give ``R = T * k`` rows in expert order. A layer of one
    expert and one selection (``E = k = 1``) is a dense layer and needs no sort. Tensors are contiguous, of the
    plan's type (weights of the top-k, biases and their gradients float32) and on the plan's device; a tensor
    that is not raises a ValueError before anything is launched. Results are new tensors unless an output is given.
    The plan's device is the current one when the layer is made, and has to be the current one at every call (a
    ValueError otherwise: the library's launches go to the current device). Calls run on the stream given, or the
    current one; calls of one layer share its workspace, so those on different streams are the caller's to order. The
    methods call the library themselves: a decoding step's calls are bound by their time on the host.
    """

    def __init__(self, T, E, k, dtype=SMOES_BF16, max_width=0, device="cuda"):
        self.plan = None
        device = torch.device(device)
        if device.type != "cuda":
            raise ValueError(f"device: a GPU is wanted, got {device}")
        self._index = torch.cuda.current_device() if device.index is None else device.index
        self.check_device()
        code, self.plan = smoes_experts_create(T, E, k, dtype, max_width)
        _check(code, "smoes_experts_create")
        self.T, self.E, self.k, self.R = T, E, k, T * k
        self.dtype = torch.bfloat16 if dtype == SMOES_BF16 else torch.float32
        self.ws = torch.empty(smoes_experts_workspace_bytes(self.plan), dtype=torch.uint8, device=device)
        self.device = self.ws.device
        _check(smoes_experts_workspace_init(self.plan, self.ws), "smoes_experts_workspace_init")
        self.expert_offsets = torch.zeros(E + 1, dtype=torch.int32, device=device)
        self.row_slot = torch.full((self.R,), -1, dtype=torch.int32, device=device)
        self.slot_row = torch.full((T, k), -1, dtype=torch.int32, device=device)
        if E == 1 and k == 1:                          # every token is a row of the one expert
            self.expert_offsets[1:].fill_(T)
            torch.arange(T, out=self.row_slot)
            torch.arange(T, out=self.slot_row.view(-1))

    def __del__(self):
        try:
            smoes_experts_destroy(self.plan)
        except Exception:
            pass

    def check_device(self):
        """A ValueError if the plan's device is not the current one."""
        current = torch._C._cuda_getDevice()
        if current != self._index:
            raise ValueError(f"device: the layer is on cuda:{self._index}, the current device is cuda:{current}")

    def _stream(self, stream):
        """The handle of the stream that a call is about to be launched on."""
        self.check_device()
        if stream is None:
            return torch._C._cuda_getCurrentRawStream(self._index)
        if stream.device_index != self._index:
            raise ValueError(f"stream: one of cuda:{self._index} is wanted, got one of cuda:{stream.device_index}")
        return stream.cuda_stream

    def _in(self, name, t, shape, dtype):
        """Address of one checked argument; None stays None."""
        if t is None:
            return None
        if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != self._index:
            raise ValueError(f"{name}: a contiguous {dtype} tensor of shape {tuple(shape)} on {self.device} is "
                             f"wanted, got {t.dtype} {tuple(t.shape)} on {t.device}")
        return t.data_ptr()

    def _new(self, t, shape, dtype, stream):
        """The output given, checked, or a new one from the memory of the stream that the call runs on."""
        if t is None:
            if stream is None:
                return torch.empty(shape, dtype=dtype, device=self.device)
            with torch.cuda.stream(stream):
                return torch.empty(shape, dtype=dtype, device=self.device)
        self._in("output", t, shape, dtype)
        return t

    def sort(self, topk_idx, stream=None):
        """Selections [T, k] int32 (negative: takes no part) into expert order; fills and returns
        expert_offsets, row_slot, slot_row."""
        idx = self._in("topk_idx", topk_idx, (self.T, self.k), torch.int32)
        ws = self.ws
        _check(_lib.smoes_expert_sort(self.plan, idx, self.expert_offsets.data_ptr(), self.row_slot.data_ptr(),
                                      self.slot_row.data_ptr(), ws.data_ptr(), ws.numel(), self._stream(stream)),
               "smoes_expert_sort")
        return self.expert_offsets, self.row_slot, self.slot_row

    def dispatch(self, X, out=None, stream=None):
        """Tokens [T, d] into expert order: [R, d]."""
        d = X.shape[-1]
        x = self._in("X", X, (self.T, d), self.dtype)
        out = self._new(out, (self.R, d), self.dtype, stream)
        _check(_lib.smoes_expert_dispatch(self.plan, x, d, self.expert_offsets.data_ptr(), self.slot_row.data_ptr(),
                                          out.data_ptr(), self._stream(stream)), "smoes_expert_dispatch")
        return out

    def dispatch_bwd(self, dXs, residual=None, out=None, stream=None):
        """Gradient of the tokens from that of their rows, plus ``residual`` [T, d]."""
        d = dXs.shape[-1]
        dx = self._in("dXs", dXs, (self.R, d), self.dtype)
        res = self._in("residual", residual, (self.T, d), self.dtype)
        out = self._new(out, (self.T, d), self.dtype, stream)
        _check(_lib.smoes_expert_dispatch_bwd(self.plan, dx, d, self.slot_row.data_ptr(), res, out.data_ptr(),
                                              self._stream(stream)), "smoes_expert_dispatch_bwd")
        return out

    def combine(self, Ys, topk_w, residual=None, out=None, stream=None):
        """Rows [R, d] back to their tokens, weighted by topk_w [T, k] float32, plus ``residual``."""
        d = Ys.shape[-1]
        ys = self._in("Ys", Ys, (self.R, d), self.dtype)
        w = self._in("topk_w", topk_w, (self.T, self.k), torch.float32)
        res = self._in("residual", residual, (self.T, d), self.dtype)
        out = self._new(out, (self.T, d), self.dtype, stream)
        _check(_lib.smoes_expert_combine(self.plan, ys, d, w, self.slot_row.data_ptr(), res, out.data_ptr(),
                                         self._stream(stream)), "smoes_expert_combine")
        return out

    def combine_bwd(self, dY, Ys, topk_w, dYs=None, d_topk_w=None, stream=None):
        """Gradients of the rows and of the weights (the d_topk_w of ``Router.backward``)."""
        d = dY.shape[-1]
        dy = self._in("dY", dY, (self.T, d), self.dtype)
        ys = self._in("Ys", Ys, (self.R, d), self.dtype)
        w = self._in("topk_w", topk_w, (self.T, self.k), torch.float32)
        dYs = self._new(dYs, (self.R, d), self.dtype, stream)
        d_topk_w = self._new(d_topk_w, (self.T, self.k), torch.float32, stream)
        _check(_lib.smoes_expert_combine_bwd(self.plan, dy, ys, d, w, self.expert_offsets.data_ptr(),
                                             self.slot_row.data_ptr(), dYs.data_ptr(), d_topk_w.data_ptr(),
                                             self._stream(stream)), "smoes_expert_combine_bwd")
        return dYs, d_topk_w

    def linear(self, X, W, bias=None, act=SMOES_ACT_NONE, gated=False, residual=None, save_pre=False, out=None,
               pre=None, stream=None):
        """act(x W_e^T + b_e) + residual of rows [R, n_in] in expert order, W [E, n_z, n_in]; gated: z = [g | u],
        act(g) u. Returns (out, pre); pre is None unless save_pre (or a tensor to write) asks for it."""
        n_z, n_in = W.shape[-2:]
        n_out = n_z // 2 if gated else n_z
        if gated and n_z % 2:
            raise ValueError(f"W: a gated layer has an even number of rows, got {n_z}")
        dt, ws = self.dtype, self.ws
        args = LinearArgs(self._in("X", X, (self.R, n_in), dt), self._in("W", W, (self.E, n_z, n_in), dt),
                          self._in("bias", bias, (self.E, n_z), torch.float32),
                          self._in("residual", residual, (self.R, n_out), dt), n_in, n_out, act, gated)
        out = self._new(out, (self.R, n_out), dt, stream)
        if save_pre or pre is not None:
            pre = self._new(pre, (self.R, n_z), dt, stream)
        _check(_lib.smoes_expert_linear(self.plan, args, self.expert_offsets.data_ptr(), out.data_ptr(), _ptr(pre),
                                        ws.data_ptr(), ws.numel(), self._stream(stream)), "smoes_expert_linear")
        return out, pre

    def act_bwd(self, dOut, pre=None, act=SMOES_ACT_NONE, gated=False, bias_grad=False, dZ=None, db=None,
                stream=None, accumulate=False):
        """Gradients of the pre-activations and of the bias: (dZ, db). Without an activation and not gated dZ is
        dOut itself (and not given). db is None unless bias_grad (or a tensor to write) asks for it; accumulate adds to
        the given db."""
        n_out = dOut.shape[-1]
        n_z = 2 * n_out if gated else n_out
        dout = self._in("dOut", dOut, (self.R, n_out), self.dtype)
        if dZ is not None and act == SMOES_ACT_NONE and not gated:
            raise ValueError("dZ: without an activation and not gated it is dOut, and none is written")
        if accumulate and db is None:
            raise ValueError("db: a tensor to accumulate into is wanted")
        if bias_grad or db is not None:
            db = self._new(db, (self.E, n_z), torch.float32, stream)
        if act == SMOES_ACT_NONE and not gated:
            z, dz, dZ = None, None, dOut
            if db is None:
                return dZ, None
        elif pre is None:
            raise ValueError("pre: the pre-activations that linear saved are wanted")
        else:
            z = self._in("pre", pre, (self.R, n_z), self.dtype)
            dZ = self._new(dZ, (self.R, n_z), self.dtype, stream)
            dz = dZ.data_ptr()
        ws = self.ws
        call = _lib.smoes_expert_act_bwd_accumulate if accumulate else _lib.smoes_expert_act_bwd
        _check(call(self.plan, dout, z, n_out, act, gated, self.expert_offsets.data_ptr(), dz, _ptr(db), ws.data_ptr(),
                    ws.numel(), self._stream(stream)), "smoes_expert_act_bwd")
        return dZ, db

    def linear_bwd(self, dZ, X, W, need_dX=True, need_dW=True, dX=None, dW=None, accumulate=False, stream=None):
        """Gradients of the rows [R, n_in] and of the weights (float32; accumulate adds to the given dW)."""
        n_z, n_in = W.shape[-2:]
        dz = self._in("dZ", dZ, (self.R, n_z), self.dtype)
        x = self._in("X", X, (self.R, n_in), self.dtype)
        w = self._in("W", W, (self.E, n_z, n_in), self.dtype)
        if accumulate and dW is None:
            raise ValueError("dW: a tensor to accumulate into is wanted")
        dX = self._new(dX, (self.R, n_in), self.dtype, stream) if need_dX else None
        dW = self._new(dW, (self.E, n_z, n_in), torch.float32, stream) if need_dW else None
        ws = self.ws
        _check(_lib.smoes_expert_linear_bwd(self.plan, dz, x, w, n_in, n_z, self.expert_offsets.data_ptr(), _ptr(dX),
                                            _ptr(dW), accumulate, ws.data_ptr(), ws.numel(), self._stream(stream)),
               "smoes_expert_linear_bwd")
        return dX, dW

    def device_status(self, stream=None):
        return _lib.smoes_experts_read_status(self.plan, self.ws.data_ptr(), self._stream(stream))
