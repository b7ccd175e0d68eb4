"""Selections that are dropped for the experts' balance loss leave the other gradients as the forward made them: the weights of the
top-k are normalised over all that it chose, the masked gate of the MI loss too.

Tolerances, from the arithmetic: gradients of one backward are added in fp32, 16 steps of 2^-24 of the parts' magnitudes. The
upstream gradient against the oracle: a product of at most four gate values and their sums, each off by e_g relatively, and
fewer than E + k + 20 roundings, of the sum of magnitudes."""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as L
from oracle import smoes_oracle as O
from tests.test_gpu_expert_balance import BF16, F32, U, bd, host  # noqa: F401  (bd: the fixture)
from paper_2604_23996_gb300.workloads import random_router_case

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, bd, dt, gate="softmax", renorm=0, mask=0, T=400, d=96, E=40, k=4, K=5, lens=(150, 249, 1)):
        self.wl = wl = random_router_case(7 + renorm + mask, T, d, E, k, K, list(lens), dtype=dt, aligned=True)
        rng = np.random.default_rng(E + mask)
        sigmoid = gate == "sigmoid"
        self.r = bd.Router(T, d, E, k, K, wl.sample_offsets, wl.expert_bin, bd.SMOES_BF16 if dt is BF16 else bd.SMOES_F32,
                           renorm_topk=renorm, mi_topk_mask=mask, gate=bd.SMOES_GATE_SIGMOID if sigmoid else bd.SMOES_GATE_SOFTMAX)
        self.X, self.W = wl.X.cuda(), wl.W.cuda()
        m = rng.random((T, 1)).astype(np.float32)
        self.M = torch.from_numpy(np.concatenate([m, 1 - m], 1)).cuda()
        self.r.forward(self.X, self.W, M_in=self.M)
        self.fwd = self.r.topk_idx.cpu().numpy()
        self.idx = self.fwd.copy()
        self.idx[rng.random(T) < 0.1] = -1              # padding tokens
        self.idx[rng.random(self.idx.shape) < 0.25] = -3    # selections over an expert's capacity
        self.didx = torch.from_numpy(self.idx).cuda()
        up = rng.standard_normal(self.idx.shape).astype(np.float32)
        up[self.idx < 0] = 0                            # as the gradient of the combination leaves them
        self.up_host, self.up = up, torch.from_numpy(up).cuda()
        x, w = host(self.X), host(self.W)
        z = x @ w.T
        self.raw = 1 / (1 + np.exp(-z)) if sigmoid else O.softmax_gate(z)
        self.g = self.raw / self.raw.sum(1, keepdims=True)
        self.slope = 1 - self.raw if sigmoid else np.ones_like(z)
        self.e_g = 2 * d * 2 * U * (np.abs(x) @ np.abs(w).T).max() + 32 * U
        self.T, self.d, self.E, self.k = T, d, E, k

    def logits(self, scale=0.0, up=None, d_gate=None, topk_idx=None):
        dz, dW = torch.empty(self.T, self.E, device="cuda"), torch.empty(self.E, self.d, device="cuda")
        self.r.backward(self.X, self.W, self.M, dW, dlogits=dz, loss_scale=scale, d_topk_w=up, d_gate=d_gate, topk_idx=topk_idx)
        return dz


PLANS = [dict(), dict(renorm=1), dict(mask=1), dict(gate="sigmoid"), dict(gate="sigmoid", mask=1), dict(renorm=1, mask=1)]
IDS = ["plain", "renorm", "mask", "sigmoid", "sigmoid_mask", "renorm_mask"]


@pytest.mark.parametrize("plan", PLANS, ids=IDS)
@pytest.mark.parametrize("dt", [BF16, F32], ids=["bf16", "fp32"])
def test_the_other_gradients_keep_the_forwards_selections(bd, dt, plan):  # noqa: F811
    c = Case(bd, dt, **plan)
    _, _, d_gate = c.r.expert_balance(topk_idx=c.didx)
    others, gates = c.logits(0.7, c.up), c.logits(0.0, d_gate=d_gate, topk_idx=c.didx)
    assert torch.equal(c.logits(0.7, c.up, topk_idx=c.didx), others)
    both = host(c.logits(0.7, c.up, d_gate, c.didx))
    mi, top = host(c.logits(0.7)), host(c.logits(0.0, c.up))
    assert (np.abs(both - (mi + top + host(gates))) <= 16 * U * (np.abs(mi) + np.abs(top) + np.abs(host(gates))) + 1e-30).all()
    # and with the bin-level balance loss besides
    loss = torch.empty(1, device="cuda")
    assert bd.smoes_bin_balance(c.r.plan, c.r.topk_idx, 1.3, loss, c.r.ws) == bd.SMOES_OK
    bins, everything = host(c.logits()), host(c.logits(0.7, c.up, d_gate, c.didx))
    size = sum(np.abs(a) for a in (mi, top, host(gates), bins))
    assert (np.abs(everything - (mi + top + host(gates) + bins)) <= 16 * U * size + 1e-30).all()
    # tokens without a selection left get nothing of the balance loss
    assert not gates[torch.from_numpy(~(c.idx >= 0).any(1)).cuda()].any()


@pytest.mark.parametrize("dt", [BF16, F32], ids=["bf16", "fp32"])
def test_renormalised_weights_against_the_oracle(bd, dt):  # noqa: F811
    c = Case(bd, dt, renorm=1)
    _, _, d_gate = c.r.expert_balance(topk_idx=c.didx, loss_scale=0.5)
    got = host(c.logits(0.0, c.up, d_gate, c.didx))
    t = L.expert_balance(c.g, c.idx, c.wl.sample_offsets, 0.5)[3]
    want = O.topk_weight_grad_logits(c.g, c.fwd, c.up_host.astype(np.float64), True) + L.gate_grad_logits(c.g, t, 1.0)
    a, n = np.zeros_like(c.g), np.zeros_like(c.g)
    np.put_along_axis(a, c.fwd.astype(np.int64), np.abs(c.up_host).astype(np.float64), 1)
    np.put_along_axis(n, c.fwd.astype(np.int64), 1.0, 1)
    G = (n * c.g).sum(1, keepdims=True)
    A = (a + n * (c.g * a).sum(1, keepdims=True) / G) / G + t
    size = c.g * (A + (c.g * A).sum(1, keepdims=True))
    assert (np.abs(got - want) <= size * (8 * c.e_g + (c.E + c.k + 20) * U)).all()
