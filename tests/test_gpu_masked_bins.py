"""MI and its gradients where a bin has no mass in a sample, or none of one modality: with the gate masked to the chosen experts a
sample's tokens may all pass a bin by, and with hard scores a bin may be chosen by one modality alone. Such a term of eq. (14) is 0 and
its logarithm counts as 0 in the gradient. Against the fp64 oracle on the GPU's own choice, with the tolerances of the other
variants."""
import numpy as np
import pytest
import torch

from oracle import smoes_oracle as O
from paper_2604_23996_gb300.workloads import random_router_case
from tests.parity import assert_scalar_close, assert_tensor_close
from tests.test_gpu_variants import bd  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
CASES = {
    # T, d, E, k, K, lengths, type, gate, hard scores
    "one_token": (1, 64, 16, 2, 8, [1], BF16, 0, False),
    "one_token_fp32": (1, 64, 16, 2, 8, [1], F32, 0, False),
    "few_tokens": (40, 96, 40, 4, 10, [1, 2, 3, 34], BF16, 0, False),
    "few_tokens_sigmoid": (40, 96, 40, 4, 10, [1, 2, 3, 34], BF16, 1, False),
    "few_tokens_fp32": (40, 96, 40, 4, 10, [1, 2, 3, 34], F32, 1, False),
    "hard": (60, 96, 64, 2, 16, [4, 16, 40], BF16, 0, True),
    "hard_fp32": (60, 96, 64, 2, 16, [4, 16, 40], F32, 0, True),
    "hard_e128": (300, 64, 128, 2, 32, [30, 70, 200], BF16, 1, True),
}


@pytest.mark.parametrize("name", list(CASES))
def test_bins_without_mass(bd, name):  # noqa: F811
    T, d, E, k, K, lens, dt, gate, hard = CASES[name]
    wl = random_router_case(300 + T, T, d, E, k, K, lens, dtype=dt, aligned=True)
    r = bd.Router(T, d, E, k, K, wl.sample_offsets, wl.expert_bin, bd.SMOES_BF16 if dt is BF16 else bd.SMOES_F32, gate=gate, mi_topk_mask=1)
    rng = np.random.default_rng(T + E)
    m = (rng.random(T) < 0.4) if hard else 0.2 + 0.6 * rng.random(T)
    M = np.stack([m, 1 - m], 1).astype(np.float32)
    X, W, Md = wl.X.cuda(), wl.W.cuda(), torch.from_numpy(M).cuda()
    r.forward(X, W, M_in=Md)
    dl, dW = torch.empty(T, E, device="cuda"), torch.empty(E, d, device="cuda")
    r.backward(X, W, Md, dW, dlogits=dl, loss_scale=0.9)
    assert r.device_status()[0] == bd.SMOES_OK
    idx = r.topk_idx.cpu().numpy()
    Xd, Wd = wl.X.double().numpy(), wl.W.double().numpy()
    f = O.router_forward_variant(Xd, Wd, M.astype(np.float64), wl.expert_bin, K, wl.sample_offsets, k, gate="sigmoid" if gate else "softmax",
                                 mask=True, topk_idx=idx)
    empty = [(f["joint"][i] == 0).sum() for i in range(len(lens))]
    assert sum(empty) > 0                               # there are such bins
    assert_tensor_close(r.joint.cpu().numpy(), f["joint"], "joint")
    assert_scalar_close(r.mi.cpu().numpy()[:wl.B], f["mi"], "mi")
    assert_scalar_close(r.loss.item(), f["loss"], "loss")
    dz, _, _ = O.router_backward_variant(Xd, Wd, M.astype(np.float64), f, wl.expert_bin, wl.sample_offsets, 0.9)
    got = dl.cpu().numpy()
    assert np.isfinite(got).all()
    # a sample of one token has no information: fp32 coefficients of rounding size, of gate values of at most 1
    assert np.abs(got - dz).max() <= 2e-3 * np.abs(dz).max() + 1e-6
    assert np.abs(dW.cpu().numpy() - dz.T @ Xd).max() <= 2e-3 * np.abs(dz.T @ Xd).max() + 1e-6 * T * np.abs(Xd).max()
