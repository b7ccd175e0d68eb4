"""The whole MoE layer (router, experts, and the way back) against the fp64 oracles of both, on the GPU's own top-k
and the stored inputs. In fp32 every step's own error is near 2^-20, so the layer's results meet the oracle's within the
2e-3 that the router's tests commit to; the bf16 layer rounds the rows between its steps six times on the longest way (2^-9 each
in the mean, independent), 2^-9 * sqrt(6) = 4.8e-3 of the norm: 1e-2 is allowed."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as OE
from oracle import smoes_oracle as O
from paper_2604_23996_gb300.workloads import random_router_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def layer_module():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2604_23996_gb300 import moe_layer
    return moe_layer


def rel(a, b):
    a = a.detach().double().cpu().numpy()
    return float(np.linalg.norm(a - b) / np.linalg.norm(b))


@pytest.mark.parametrize("dt,biases", [(torch.float32, True), (torch.bfloat16, False), (torch.bfloat16, True)],
                         ids=["fp32_biases", "bf16", "bf16_biases"])
def test_layer_forward_and_backward(layer_module, dt, biases):
    bd = layer_module.bd
    T, d, f, E, k, n_bins = 333, 136, 72, 16, 3, 4
    wl = random_router_case(41, T=T, d=d, E=E, k=k, n_bins=n_bins, sample_lengths=[100, 150, 83], dtype=dt, aligned=True)
    code = bd.SMOES_BF16 if dt is torch.bfloat16 else bd.SMOES_F32
    rng = np.random.default_rng(2)

    def normal(*shape, std=1.0, dtype=dt):
        return torch.from_numpy(rng.standard_normal(shape) * std).to(dtype).cuda()

    X, W_gate = wl.X.cuda(), wl.W.cuda()
    W_up, W_down, dY = normal(E, 2 * f, d, std=d ** -0.5), normal(E, d, f, std=f ** -0.5), normal(T, d)
    b_up = normal(E, 2 * f, std=0.1, dtype=torch.float32) if biases else None
    b_down = normal(E, d, std=0.1, dtype=torch.float32) if biases else None
    layer = layer_module.MoELayer(T, d, f, E, k, n_bins, wl.sample_offsets, wl.expert_bin, code, biases=biases)
    Y = layer.forward(X, W_gate, W_up, W_down, mu=wl.mu.cuda(), var=wl.var.cuda(), tau=wl.tau, b_up=b_up, b_down=b_down)
    served = layer.forward(X, W_gate, W_up, W_down, mu=wl.mu.cuda(), var=wl.var.cuda(), tau=wl.tau, b_up=b_up,
                           b_down=b_down, training=False)
    assert torch.equal(Y, served)
    dX = layer.backward(dY, loss_scale=0.5)
    assert layer.router.device_status()[0] == layer.experts.device_status() == bd.SMOES_OK

    h = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
    Xh, Wg, Wu, Wd, dYh = h(X), h(W_gate), h(W_up), h(W_down), h(dY)
    M = O.gaussian_score(Xh, wl.mu.double().numpy(), wl.var.double().numpy(), wl.tau)
    idx = layer.router.topk_idx.cpu().numpy()
    fwd = O.router_forward_variant(Xh, Wg, M, wl.expert_bin, n_bins, wl.sample_offsets, k, topk_idx=idx)
    off, row_slot, slot_row = OE.sort(idx, E)
    Xs = OE.dispatch(Xh, row_slot, k)
    H, z = OE.linear(Xs, Wu, off, h(b_up), OE.SILU, True)
    Ys, _ = OE.linear(H, Wd, off, h(b_down))
    tol = 2e-3 if dt is torch.float32 else 1e-2
    assert rel(Y, OE.back(Ys, slot_row, fwd["topk_w"], Xh)) < tol

    dYs, dw = OE.combine_bwd(dYh, Ys, fwd["topk_w"], slot_row)
    dH, dW_down = OE.linear_bwd(dYs, H, Wd, off)
    dZ, db_up = OE.act_bwd(dH, z, off, OE.SILU, True)
    dXs, dW_up = OE.linear_bwd(dZ, Xs, Wu, off)
    _, dW_gate, dX_router = O.router_backward(Xh, Wg, M, fwd, wl.expert_bin, wl.sample_offsets, 0.5, d_topk_w=dw)
    assert rel(dX, OE.back(dXs, slot_row, None, dX_router + dYh)) < tol
    assert rel(layer.dW_up, dW_up) < tol and rel(layer.dW_down, dW_down) < tol
    assert rel(layer.dW_gate, dW_gate) < tol
    if biases:
        assert rel(layer.db_up, db_up) < tol
        assert rel(layer.db_down, np.stack([dYs[off[e]:off[e + 1]].sum(0) for e in range(E)])) < tol
    before = layer.dW_up.clone()
    layer.backward(dY, loss_scale=0.5, accumulate=True)
    assert torch.equal(layer.dW_up, 2 * before)          # the same sums, added once
