"""GPU parity of the expert-level load-balance loss, its counts and its gradient through the router's backward against the
fp64 oracle, on the GPU's own (or edited) selections.

Tolerances, from the arithmetic. The logits are sums of d products in fp32, each addition off by a step of 2^-23 of the sum of
magnitudes at most: e_z = d 2^-23 max_je sum |x w|. A gate value is e^z (or sigmoid(z)) over a sum of them: off by 2 e_z and
16 steps, relatively. The loss is a sum of positive terms over fewer than 400 additions in a row. The table d_gate is four
operations on whole numbers: 5 roundings. dW keeps the tolerance that the router's own tests commit to (2e-3 of the norm)."""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as L
from oracle import smoes_oracle as O
from paper_2604_23996_gb300.workloads import random_router_case

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def bd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2604_23996_gb300 import binding
    return binding


def host(t):
    return t.detach().double().cpu().numpy()


def rel(a, b):
    return float(np.linalg.norm(host(a) - b) / np.linalg.norm(b))


CASES = {
    # T, d, E, k, n_bins, lengths, type, gate, dropped
    "bf16_e64": (1300, 256, 64, 6, 8, [600, 700], BF16, "softmax", 0.0),
    "bf16_one_token": (1, 64, 8, 2, 2, [1], BF16, "softmax", 0.0),
    "bf16_e128_ragged": (777, 192, 128, 8, 16, [1, 300, 33, 2, 441], BF16, "softmax", 0.0),
    "bf16_e48_dropped": (900, 128, 48, 5, 6, [450, 64, 386], BF16, "softmax", 0.3),
    "bf16_many_samples": (400, 64, 16, 2, 4, [1, 2, 3, 4] * 40, BF16, "softmax", 0.1),
    "bf16_e72_sigmoid": (513, 128, 72, 4, 9, [512, 1], BF16, "sigmoid", 0.0),
    "bf16_e9": (130, 64, 9, 3, 3, [65, 65], BF16, "softmax", 0.0),
    "bf16_long": (20000, 64, 64, 6, 8, [7001, 12999], BF16, "softmax", 0.05),
    "fp32_e16": (640, 136, 16, 3, 4, [640], F32, "softmax", 0.0),
    "fp32_e40_dropped": (700, 96, 40, 4, 5, [300, 399, 1], F32, "softmax", 0.2),
    "fp32_e64_sigmoid": (333, 64, 64, 8, 8, [100, 233], F32, "sigmoid", 0.1),
}


class Case:
    def __init__(self, bd, name, all_dropped=None):
        T, d, E, k, K, lens, dt, gate, dropped = CASES[name]
        self.wl = wl = random_router_case(len(name) + T, T, d, E, k, K, lens, dtype=dt, aligned=True)
        rng = np.random.default_rng(T)
        self.bias = torch.from_numpy((0.1 * rng.standard_normal(E)).astype(np.float32)).cuda() if gate == "sigmoid" else None
        self.r = bd.Router(T, d, E, k, K, wl.sample_offsets, wl.expert_bin, bd.SMOES_BF16 if dt is BF16 else bd.SMOES_F32,
                           gate=bd.SMOES_GATE_SIGMOID if gate == "sigmoid" else bd.SMOES_GATE_SOFTMAX, score_bias=self.bias)
        self.X, self.W = wl.X.cuda(), wl.W.cuda()
        m = rng.random((T, 1)).astype(np.float32)
        self.M = torch.from_numpy(np.concatenate([m, 1 - m], 1)).cuda()
        self.r.forward(self.X, self.W, M_in=self.M)
        idx = self.r.topk_idx.cpu().numpy()
        if dropped:
            idx[rng.random(T) < dropped] = -1           # padding tokens
            idx[rng.random(idx.shape) < dropped / 2] = -5
        if all_dropped is not None:
            idx[wl.sample_offsets[all_dropped]:wl.sample_offsets[all_dropped + 1]] = -1
        self.idx, self.didx = idx, torch.from_numpy(idx).cuda()
        x, w = host(self.X), host(self.W)
        z = x @ w.T
        self.raw = 1 / (1 + np.exp(-z)) if gate == "sigmoid" else O.softmax_gate(z)
        self.g = self.raw / self.raw.sum(1, keepdims=True)
        self.slope = 1 - self.raw if gate == "sigmoid" else np.ones_like(z)
        self.e_z = d * 2 * U * (np.abs(x) @ np.abs(w).T).max()
        self.e_g = 2 * self.e_z + 32 * U
        self.T, self.d, self.E = T, d, E

    def check(self, per_sample, scale=0.5):
        off = self.wl.sample_offsets if per_sample else [0, self.T]
        out = self.r.expert_balance(topk_idx=self.didx, per_sample=per_sample, loss_scale=scale)
        loss, counts, d_gate, t = L.expert_balance(self.g, self.idx, off, scale)
        assert np.array_equal(out[1].cpu().numpy(), counts)
        assert abs(float(out[0]) - loss) <= loss * (self.e_g + 400 * U)
        assert (np.abs(host(out[2]) - d_gate) <= 5 * U * d_gate).all()
        return out, t


@pytest.mark.parametrize("per_sample", [True, False])
@pytest.mark.parametrize("name", list(CASES))
def test_loss_counts_and_gradient(bd, name, per_sample):
    c = Case(bd, name)
    out, t = c.check(per_sample)
    again, _ = c.check(per_sample)
    assert all(torch.equal(a, b) for a, b in zip(out, again))                # the tickets are back, the bits the same
    new = lambda *shape, dt=F32: torch.full(shape, float("nan"), dtype=dt, device="cuda")  # noqa: E731
    dW, dX, dz = new(c.E, c.d), new(c.T, c.d, dt=c.X.dtype), new(c.T, c.E)
    c.r.backward(c.X, c.W, c.M, dW, dX=dX, dlogits=dz, loss_scale=0.0, d_gate=out[2], topk_idx=c.didx)
    assert c.r.device_status()[0] == bd.SMOES_OK
    want = L.gate_grad_logits(c.g, t, c.slope)
    size = c.g * (t + (c.g * t).sum(1, keepdims=True))
    assert (np.abs(host(dz) - want) <= size * (3 * c.e_g + (c.E + 10) * U)).all()
    assert not dz[torch.from_numpy(~((c.idx >= 0) & (c.idx < c.E)).any(1)).cuda()].any()
    if c.T > 1:
        assert rel(dW, want.T @ host(c.X)) < 2e-3
        # dX is formed from dz rounded to bf16 (half a step, 2^-8 of each dz) and rounded once more; W's experts share a
        # component here that the sum over experts cancels, so the first bound is of the magnitudes
        dx, w = want @ host(c.W), np.abs(host(c.W))
        half = 2.0 ** -8 if c.X.dtype is BF16 else 2 * U
        assert (np.abs(host(dX) - dx) <= half * (np.abs(want) @ w + np.abs(dx)) + 2 * c.E * U * (np.abs(want) @ w)
                + (size * (3 * c.e_g + (c.E + 10) * U)) @ w + 1e-30).all()


@pytest.mark.parametrize("name", ["bf16_e64", "bf16_e72_sigmoid", "fp32_e40_dropped"])
def test_joins_the_other_gradients(bd, name):
    """MI, top-k weights, bin-level balance and expert-level balance in one backward: the sum of what they give alone."""
    c = Case(bd, name)
    up = torch.from_numpy(np.random.default_rng(1).standard_normal(c.idx.shape).astype(np.float32)).cuda()
    _, _, d_gate = c.r.expert_balance(topk_idx=c.didx)
    dW, loss = torch.empty(c.E, c.d, device="cuda"), torch.empty(1, device="cuda")

    def logits(scale, up=None, d_gate=None):
        dz = torch.empty(c.T, c.E, device="cuda")
        c.r.backward(c.X, c.W, c.M, dW, dlogits=dz, loss_scale=scale, d_topk_w=up, d_gate=d_gate, topk_idx=c.didx)
        return host(dz)

    mi, top, gates = logits(0.7), logits(0.0, up), logits(0.0, d_gate=d_gate)
    both = logits(0.7, up, d_gate)
    assert bd.smoes_bin_balance(c.r.plan, c.r.topk_idx, 1.3, loss, c.r.ws) == bd.SMOES_OK
    bins, everything, no_up = logits(0.0), logits(0.7, up, d_gate), logits(0.7, None, d_gate)
    # one fp32 addition for each further gradient
    for got, parts in ((both, (mi, top, gates)), (everything, (mi, top, gates, bins)), (no_up, (mi, gates, bins))):
        assert (np.abs(got - sum(parts)) <= 16 * U * sum(np.abs(a) for a in parts) + 1e-30).all()


def test_gradient_against_differences(bd):
    """The loss (counts held) along directions of W, by central differences of the oracle's."""
    c = Case(bd, "fp32_e16")
    _, _, d_gate = c.r.expert_balance(topk_idx=c.didx)
    dW = torch.empty(c.E, c.d, device="cuda")
    c.r.backward(c.X, c.W, c.M, dW, loss_scale=0.0, d_gate=d_gate, topk_idx=c.didx)
    x, w = host(c.X), host(c.W)
    f = lambda w: L.expert_balance(O.softmax_gate(x @ w.T), c.idx, c.wl.sample_offsets)[0]  # noqa: E731
    rng = np.random.default_rng(0)
    for _ in range(5):
        v = rng.standard_normal(w.shape)
        slope = (f(w + 1e-5 * v) - f(w - 1e-5 * v)) / 2e-5
        assert abs((host(dW) * v).sum() - slope) <= 2e-3 * np.linalg.norm(host(dW)) * np.linalg.norm(v) / np.sqrt(w.size)


def test_a_sample_without_selections_and_none_at_all(bd):
    c = Case(bd, "bf16_e48_dropped", all_dropped=1)
    out, _ = c.check(True)
    assert not out[1][1].any() and not out[2][1].any()
    c.idx[:] = -1
    c.didx.fill_(-1)
    for per_sample in (True, False):
        loss, counts, d_gate = c.r.expert_balance(topk_idx=c.didx, per_sample=per_sample)
        assert float(loss) == 0 and not counts.any() and not d_gate.any()


def test_selections_out_of_range_and_repeated(bd):
    c = Case(bd, "bf16_e9")
    c.idx[3] = [9, 1 << 30, -7]                         # nothing that exists
    c.idx[4] = [8, 8, 8]                                # the same one three times
    c.didx.copy_(torch.from_numpy(c.idx))
    out, t = c.check(True)
    assert not t[3].any() and t[4].any()
    dW, dz = torch.empty(c.E, c.d, device="cuda"), torch.empty(c.T, c.E, device="cuda")
    c.r.backward(c.X, c.W, c.M, dW, dlogits=dz, loss_scale=0.0, d_gate=out[2], topk_idx=c.didx)
    assert not dz[3].any() and dz[4].any()


def test_graph_and_stream(bd):
    c = Case(bd, "bf16_e64")
    want, _ = c.check(True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = c.r.expert_balance(topk_idx=c.didx, loss_scale=0.5, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    dW, dz = torch.empty(c.E, c.d, device="cuda"), torch.empty(c.T, c.E, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.r.forward(c.X, c.W, M_in=c.M)
        got = c.r.expert_balance(loss_scale=0.5)
        c.r.backward(c.X, c.W, c.M, dW, dlogits=dz, d_gate=got[2])
    c.X.mul_(1.5)
    for _ in range(2):
        graph.replay()
    c.r.forward(c.X, c.W, M_in=c.M)
    want, dz2 = c.r.expert_balance(loss_scale=0.5), torch.empty_like(dz)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    c.r.backward(c.X, c.W, c.M, dW, dlogits=dz2, d_gate=want[2])
    assert torch.equal(dz, dz2)


def test_no_tokens_and_refusals(bd):
    r = bd.Router(0, 64, 8, 2, 2, [0], [0] * 4 + [1] * 4)
    loss, counts, d_gate = r.expert_balance()
    assert float(loss) == 0 and counts.shape == d_gate.shape == (0, 8)
    loss, counts, d_gate = r.expert_balance(per_sample=False)
    assert float(loss) == 0 and not counts.any() and not d_gate.any()
    c = Case(bd, "bf16_e64")
    with pytest.raises(ValueError, match="topk_idx"):
        c.r.expert_balance(topk_idx=c.didx.long())
    with pytest.raises(ValueError, match="counts"):
        c.r.expert_balance(counts=torch.empty(3, 64, dtype=torch.int32, device="cuda"))
    dW = torch.empty(c.E, c.d, device="cuda")
    for bad in (torch.zeros(64, device="cuda"), torch.zeros(3, 64, device="cuda"), torch.zeros(2, 64)):
        with pytest.raises(ValueError, match="d_gate"):
            c.r.backward(c.X, c.W, c.M, dW, d_gate=bad)
