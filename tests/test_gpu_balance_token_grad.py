"""The tokens' gradient of a bf16 router's backward with a gradient of the gate values (the experts' balance loss), against the
fp64 oracle: it takes all of dz's bits that the weights' gradient takes.

Tolerance, from the arithmetic: dz leaves as two bf16 parts, the second one's rounding is 2^-16 of dz; a product with a bf16
weight is exact in fp32; each of the additions (two parts of E padded to a multiple of 64) is off by a step of 2^-23 of the sum
of magnitudes at most; then one rounding to bf16, 2^-8 of the value. dz itself is off by what the logits' test grants it."""
import numpy as np
import pytest
import torch

from tests.test_gpu_expert_balance import CASES, U, Case, L, bd, host  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("per_sample", [True, False])
@pytest.mark.parametrize("name", [n for n, c in CASES.items() if c[6] is torch.bfloat16])
def test_dx_takes_both_parts_of_dz(bd, name, per_sample):  # noqa: F811
    c = Case(bd, name)
    out, t = c.check(per_sample)
    dW, dX = torch.empty(c.E, c.d, device="cuda"), torch.empty_like(c.X)
    c.r.backward(c.X, c.W, c.M, dW, dX=dX, loss_scale=0.0, d_gate=out[2], topk_idx=c.didx)
    dz = L.gate_grad_logits(c.g, t, c.slope)
    e_z = c.g * (t + (c.g * t).sum(1, keepdims=True)) * (3 * c.e_g + (c.E + 10) * U)
    w = np.abs(host(c.W))
    terms = 2 * (-(-c.E // 64) * 64)
    want = dz @ host(c.W)
    before = (2.0 ** -16 + 1.01 * terms * 2.0 ** -23) * (np.abs(dz) @ w) + 1.01 * e_z @ w
    assert (np.abs(host(dX) - want) <= 2.0 ** -8 * np.abs(want) + 1.01 * before + 1e-30).all()
    again = torch.empty_like(dX)
    c.r.backward(c.X, c.W, c.M, dW, dX=again, loss_scale=0.0, d_gate=out[2], topk_idx=c.didx)
    assert torch.equal(again, dX)
