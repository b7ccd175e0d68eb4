"""One whole MoE layer on the router and the expert calls: a training step's forward and backward, and the
forward alone for serving.

    forward   top-k of the router (with the MI regulariser) -> rows in expert order -> gated up-projection
              silu(g) * u -> down-projection -> weighted rows back to the tokens, plus the residual stream
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
    """

    # what the backward reads of the router's and the experts' own buffers, which the next forward writes again
    _STATE = (("router", "ws"), ("router", "topk_idx"), ("router", "topk_w"), ("router", "M"),
              ("experts", "expert_offsets"), ("experts", "row_slot"), ("experts", "slot_row"))

    def __init__(self, T, d, f, E, k, n_bins, sample_offsets, expert_bin, dtype=bd.SMOES_BF16, device="cuda", biases=False):
        self.experts = bd.Experts(T, E, k, dtype, max_width=max(2 * f, d) if biases else 0, device=device)
        self.router = bd.Router(T, d, E, k, n_bins, sample_offsets, expert_bin, dtype, device=device)
        self.biases = biases
        self.saved = None                              # tensors of the last forward in training
        self.kept = None                               # and copies of _STATE, once another forward has followed it
        new = lambda *shape: torch.zeros(shape, dtype=torch.float32, device=device)  # noqa: E731
        self.dW_gate, self.dW_up, self.dW_down = new(E, d), new(E, 2 * f, d), new(E, d, f)
        self.db_up, self.db_down = (new(E, 2 * f), new(E, d)) if biases else (None, None)

    def forward(self, X, W_gate, W_up, W_down, M_in=None, mu=None, var=None, tau=0.0, b_up=None, b_down=None, training=True):
        """X [T, d] -> Y [T, d] = X + sum over the chosen experts. ``training`` keeps what the backward reads. The MI
        loss is in ``router.loss``."""
        r, ex = self.router, self.experts
        ex.check_device()
        if training:
            self.saved = self.kept = None
        elif self.saved is not None and self.kept is None:
            self.kept = [getattr(getattr(self, owner), name).clone() for owner, name in self._STATE]
        r.forward(X, W_gate, M_in=M_in, mu=mu, var=var, tau=tau, bin_prob=False)
        ex.sort(r.topk_idx)
        Xs = ex.dispatch(X)
        H, pre = ex.linear(Xs, W_up, bias=b_up, act=bd.SMOES_ACT_SILU, gated=True, save_pre=training)
        Ys, _ = ex.linear(H, W_down, bias=b_down)
        if training:
            self.saved = (X, W_gate, W_up, W_down, M_in, Xs, pre, H, Ys)
        return ex.combine(Ys, r.topk_w, residual=X)

    def backward(self, dY, loss_scale=1.0, accumulate=False):
        """Gradient of <dY, Y> + loss_scale * L_MI of the last forward in training: returns dX [T, d], fills dW_gate,
        dW_up, dW_down (and db_up, db_down), or adds to all of them."""
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
        X, W_gate, W_up, W_down, M_in, Xs, pre, H, Ys = self.saved
        dYs, d_topk_w = ex.combine_bwd(dY, Ys, r.topk_w)
        if self.biases:
            ex.act_bwd(dYs, db=self.db_down, accumulate=accumulate)
        dH, _ = ex.linear_bwd(dYs, H, W_down, dW=self.dW_down, accumulate=accumulate)
        dZ, _ = ex.act_bwd(dH, pre, act=bd.SMOES_ACT_SILU, gated=True, db=self.db_up,
                           accumulate=accumulate and self.biases)
        dXs, _ = ex.linear_bwd(dZ, Xs, W_up, dW=self.dW_up, accumulate=accumulate)
        dX = torch.empty_like(X)
        r.backward(X, W_gate, M_in if M_in is not None else r.M, self.dW_gate, dX=dX, loss_scale=loss_scale,
                   d_topk_w=d_topk_w, accumulate=accumulate)
        # the router's part and the residual stream's join the experts'
        dX += dY
        return ex.dispatch_bwd(dXs, residual=dX)


def _step_times(config, f, decode_tokens, steps=10):
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

    layer = MoELayer(wl.T, wl.d, f, wl.E, wl.k, wl.n_bins, wl.sample_offsets, wl.expert_bin, code)

    def train():
        layer.forward(X, W_gate, W_up, W_down, **stats)
        layer.backward(dY)

    ms = timed(train)
    n = decode_tokens
    serve = MoELayer(n, wl.d, f, wl.E, wl.k, wl.n_bins, [0, n], wl.expert_bin, code)
    Xd = X[:n].contiguous()
    us = 1e3 * timed(lambda: serve.forward(Xd, W_gate, W_up, W_down, training=False, **stats))
    assert layer.router.device_status()[0] == layer.experts.device_status() == serve.experts.device_status() == bd.SMOES_OK
    flops = 18.0 * wl.T * wl.k * wl.d * f
    print(f"{config}: T={wl.T} d={wl.d} f={f} E={wl.E} k={wl.k}: training step {ms:.3f} ms "
          f"({flops / ms / 1e9:.0f} TFLOP/s of the experts' products), decoding step of {n} tokens {us:.1f} us")


if __name__ == "__main__":
    import argparse
    ap = argparse.ArgumentParser(description="Times one MoE layer on a synthetic workload.")
    ap.add_argument("--config", default="dsmoe_vlm")
    ap.add_argument("--expert-width", type=int, default=1024)
    ap.add_argument("--decode-tokens", type=int, default=16)
    a = ap.parse_args()
    _step_times(a.config, a.expert_width, a.decode_tokens)
