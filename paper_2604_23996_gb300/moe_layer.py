"""One whole MoE layer on the router and the expert calls: a training step's forward and backward, and the
forward alone for serving.

    forward   (layer norm ->) top-k of the router (with the MI regulariser, and the experts' balance loss) -> rows in
              expert order -> gated up-projection silu(g) * u -> down-projection -> weighted rows back to the tokens,
              plus the residual stream; for serving also with the experts' weights and rows in 4 bits
    backward  the same way back; the gradient of the top-k weights and the one of the tokens that comes
              through the experts meet the router's own gradient in ``Router.backward`` and ``dispatch_bwd``

``python -m paper_2604_23996_gb300.moe_layer`` runs a training step and a decoding step of a workload's layer on
the GPU and prints their times.
"""
from __future__ import annotations

import torch

from . import binding as bd


class MoELayer:
    """Router and experts of one layer for batches of ``T`` tokens.

    ``W_gate`` [E, d], ``W_up`` [E, 2 f, d] (g's rows, then u's) and ``W_down`` [E, d, f] are the caller's, of the
    plan's type; ``b_up`` [E, 2 f] and ``b_down`` [E, d] float32 are optional (``biases``: their gradients are formed).
    The gradients' buffers are kept (float32), written by every backward or accumulated into.

    ``router`` and ``experts`` hold the results of the last forward. A backward belongs to the last forward in training,
    whatever was evaluated since, and can be repeated.

    ``norm_eps``: the layer's tokens are the layer norm of the residual stream X, with weight and bias ``norm`` = (w, b)
    [d] float32 (b may be None) given to every forward; their gradients are dnorm_w and dnorm_b. ``balance``: "sample" or
    "batch": a forward in training forms the experts' balance loss (balance_loss [1], expert_counts) and its backward adds the
    gradient of ``balance_scale`` times it.
    """

    # what the backward reads of the router's and the experts' own buffers, which the next forward writes again
    _STATE = (("router", "ws"), ("router", "topk_idx"), ("router", "topk_w"), ("router", "M"),
              ("experts", "expert_offsets"), ("experts", "row_slot"), ("experts", "slot_row"))

    def __init__(self, T, d, f, E, k, n_bins, sample_offsets, expert_bin, dtype=bd.SMOES_BF16, device="cuda", biases=False,
                 norm_eps=None, balance=None):
        if balance not in (None, "sample", "batch"):
            raise ValueError(f'balance: "sample", "batch" or None is wanted, got {balance!r}')
        self.experts = bd.Experts(T, E, k, dtype, max_width=max(2 * f, d) if biases else 0, device=device)
        self.router = bd.Router(T, d, E, k, n_bins, sample_offsets, expert_bin, dtype, device=device)
        self.biases = biases
        self.saved = None                              # tensors of the last forward in training
        self.kept = None                               # and copies of _STATE, once another forward has followed it
        new = lambda *shape: torch.zeros(shape, dtype=torch.float32, device=device)  # noqa: E731
        self.dW_gate, self.dW_up, self.dW_down = new(E, d), new(E, 2 * f, d), new(E, d, f)
        self.db_up, self.db_down = (new(E, 2 * f), new(E, d)) if biases else (None, None)
        self.norm = None if norm_eps is None else bd.LayerNorm(T, d, dtype, eps=norm_eps, device=device)
        self.dnorm_w, self.dnorm_b = (None, None) if norm_eps is None else (new(d), new(d))
        self.balance, self.balance_loss, self.expert_counts = balance, None, None

    def forward(self, X, W_gate, W_up, W_down, M_in=None, mu=None, var=None, tau=0.0, b_up=None, b_down=None, training=True,
                norm=None, balance_scale=1.0):
        """X [T, d] -> Y [T, d] = X + sum over the chosen experts. ``training`` keeps what the backward reads. The MI
        loss is in ``router.loss``. For serving (bf16, d and f multiples of 32) W_up and W_down may be both in 4 bits
        (``binding.mx_quantise``)."""
        r, ex = self.router, self.experts
        ex.check_device()
        mx = isinstance(W_up, bd.Mx)
        if mx != isinstance(W_down, bd.Mx) or (mx and training):
            raise ValueError("W_up, W_down: both in 4 bits, and not in training")
        if mx and ex.dtype is not torch.bfloat16:
            raise ValueError("W_up, W_down: 4 bits are for layers in bf16")
        if (norm is None) != (self.norm is None):
            raise ValueError("norm: a weight and a bias are wanted where the layer was made with norm_eps, and nowhere else")
        if training:
            self.saved = self.kept = None
        elif self.saved is not None and self.kept is None:
            self.kept = [getattr(getattr(self, owner), name).clone() for owner, name in self._STATE]
        stream, mean, rstd = X, None, None             # X: the tokens that router and experts see
        if self.norm is not None:
            X, _, mean, rstd = self.norm.forward(stream, *norm, stats=training)
        r.forward(X, W_gate, M_in=M_in, mu=mu, var=var, tau=tau, bin_prob=False)
        ex.sort(r.topk_idx)
        if mx:
            H = ex.linear_mx(ex.dispatch_mx(X), W_up, bias=b_up, act=bd.SMOES_ACT_SILU, gated=True)
            return ex.combine(ex.linear_mx(bd.mx_quantise(H), W_down, bias=b_down), r.topk_w, residual=stream)
        d_gate = None
        if training and self.balance is not None:
            self.balance_loss, self.expert_counts, d_gate = r.expert_balance(per_sample=self.balance == "sample",
                                                                             loss_scale=balance_scale)
        Xs = ex.dispatch(X)
        H, pre = ex.linear(Xs, W_up, bias=b_up, act=bd.SMOES_ACT_SILU, gated=True, save_pre=training)
        Ys, _ = ex.linear(H, W_down, bias=b_down)
        if training:
            self.saved = (X, W_gate, W_up, W_down, M_in, Xs, pre, H, Ys, d_gate, (stream, mean, rstd, norm))
        return ex.combine(Ys, r.topk_w, residual=stream)

    def backward(self, dY, loss_scale=1.0, accumulate=False):
        """Gradient of <dY, Y> + loss_scale * L_MI (+ balance_scale * L_balance) of the last forward in training: returns
        dX [T, d], fills dW_gate, dW_up, dW_down (and db_up, db_down, dnorm_w, dnorm_b), or adds to all of them."""
        if self.saved is None:
            raise RuntimeError("backward: no forward in training to go back through")
        if self.kept is None:
            return self._backward(dY, loss_scale, accumulate)
        self._exchange()
        try:
            return self._backward(dY, loss_scale, accumulate)
        finally:
            self._exchange()

    def _exchange(self):
        """The kept buffers in the place of the present ones, or back."""
        for i, (owner, name) in enumerate(self._STATE):
            owner = getattr(self, owner)
            present = getattr(owner, name)
            setattr(owner, name, self.kept[i])
            self.kept[i] = present

    def _backward(self, dY, loss_scale, accumulate):
        r, ex = self.router, self.experts
        X, W_gate, W_up, W_down, M_in, Xs, pre, H, Ys, d_gate, (stream, mean, rstd, norm) = self.saved
        dYs, d_topk_w = ex.combine_bwd(dY, Ys, r.topk_w)
        if self.biases:
            ex.act_bwd(dYs, db=self.db_down, accumulate=accumulate)
        dH, _ = ex.linear_bwd(dYs, H, W_down, dW=self.dW_down, accumulate=accumulate)
        dZ, _ = ex.act_bwd(dH, pre, act=bd.SMOES_ACT_SILU, gated=True, db=self.db_up,
                           accumulate=accumulate and self.biases)
        dXs, _ = ex.linear_bwd(dZ, Xs, W_up, dW=self.dW_up, accumulate=accumulate)
        dX = torch.empty_like(X)
        r.backward(X, W_gate, M_in if M_in is not None else r.M, self.dW_gate, dX=dX, loss_scale=loss_scale,
                   d_topk_w=d_topk_w, accumulate=accumulate, d_gate=d_gate)
        if self.norm is not None:
            dn = ex.dispatch_bwd(dXs, residual=dX)
            dX, _, _ = self.norm.backward(dn, stream, mean, rstd, norm[0], residual=dY, need_db=norm[1] is not None,
                                          dw=self.dnorm_w, db=self.dnorm_b, accumulate=accumulate)
            return dX
        # the router's part and the residual stream's join the experts'
        dX += dY
        return ex.dispatch_bwd(dXs, residual=dX)


def _step_times(config, f, decode_tokens, steps=10, norm=False, balance=None, mx=False):
    from .workloads import config_workload, CONFIGS
    wl = config_workload(config)
    g = torch.Generator(device="cuda").manual_seed(0)
    dt = CONFIGS[config]["dtype"]
    code = bd.SMOES_BF16 if dt is torch.bfloat16 else bd.SMOES_F32

    def normal(*shape, std):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(dt)

    X, W_gate = wl.X.cuda(), wl.W.cuda()
    stats = dict(mu=wl.mu.cuda(), var=wl.var.cuda(), tau=wl.tau)
    W_up, W_down = normal(wl.E, 2 * f, wl.d, std=wl.d ** -0.5), normal(wl.E, wl.d, f, std=f ** -0.5)
    dY = normal(wl.T, wl.d, std=1.0)

    def timed(fn):
        for _ in range(3):
            fn()
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        torch.cuda.synchronize()
        a.record()
        for _ in range(steps):
            fn()
        b.record()
        torch.cuda.synchronize()
        return a.elapsed_time(b) / steps

    made = dict(dtype=code, norm_eps=1e-5 if norm else None)
    if norm:
        stats["norm"] = (torch.ones(wl.d, device="cuda"), torch.zeros(wl.d, device="cuda"))
    layer = MoELayer(wl.T, wl.d, f, wl.E, wl.k, wl.n_bins, wl.sample_offsets, wl.expert_bin, balance=balance, **made)

    def train():
        layer.forward(X, W_gate, W_up, W_down, **stats)
        layer.backward(dY)

    ms = timed(train)
    n = decode_tokens
    serve = MoELayer(n, wl.d, f, wl.E, wl.k, wl.n_bins, [0, n], wl.expert_bin, **made)
    Xd = X[:n].contiguous()
    us = 1e3 * timed(lambda: serve.forward(Xd, W_gate, W_up, W_down, training=False, **stats))
    us4 = ""
    if mx:
        q_up, q_down = bd.mx_quantise(W_up), bd.mx_quantise(W_down)
        us4 = f", {1e3 * timed(lambda: serve.forward(Xd, W_gate, q_up, q_down, training=False, **stats)):.1f} us in 4 bits"
    assert layer.router.device_status()[0] == layer.experts.device_status() == serve.experts.device_status() == bd.SMOES_OK
    flops = 18.0 * wl.T * wl.k * wl.d * f
    print(f"{config}: T={wl.T} d={wl.d} f={f} E={wl.E} k={wl.k}: training step {ms:.3f} ms "
          f"({flops / ms / 1e9:.0f} TFLOP/s of the experts' products), decoding step of {n} tokens {us:.1f} us{us4}")


if __name__ == "__main__":
    import argparse
    ap = argparse.ArgumentParser(description="Times one MoE layer on a synthetic workload.")
    ap.add_argument("--config", default="dsmoe_vlm")
    ap.add_argument("--expert-width", type=int, default=1024)
    ap.add_argument("--decode-tokens", type=int, default=16)
    ap.add_argument("--norm", action="store_true", help="a layer norm in front of the router and the experts")
    ap.add_argument("--balance", choices=["sample", "batch"], help="the experts' balance loss in training")
    ap.add_argument("--mx", action="store_true", help="the decoding step with the experts in 4 bits as well")
    a = ap.parse_args()
    _step_times(a.config, a.expert_width, a.decode_tokens, norm=a.norm, balance=a.balance, mx=a.mx)
