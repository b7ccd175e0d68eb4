"""The MoE layer with a layer norm in front, the experts' balance loss, and its experts in 4 bits for serving: against the fp64
oracles on the GPU's own top-k and the stored inputs, with the tolerances of the layer's own test (fp32 2e-3 of the norm,
bf16 1e-2: one more rounding of the rows, of the normed tokens, 2^-9 sqrt(7) in the mean)."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as OE
from oracle import layer_oracle as OL
from oracle import smoes_oracle as O
from paper_2604_23996_gb300.workloads import random_router_case

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def layer_module():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2604_23996_gb300 import moe_layer
    return moe_layer


def host(t):
    return t.detach().double().cpu().numpy()


def rel(a, b):
    return float(np.linalg.norm(host(a) - b) / np.linalg.norm(b))


class Case:
    def __init__(self, module, dt, T=333, d=160, f=96, E=16, k=3, lengths=(100, 150, 83)):
        self.bd = module.bd
        rng = np.random.default_rng(2)
        self.wl = wl = random_router_case(41, T=T, d=d, E=E, k=k, n_bins=4, sample_lengths=list(lengths), dtype=dt, aligned=True)
        self.code = self.bd.SMOES_BF16 if dt is BF16 else self.bd.SMOES_F32
        new = lambda *shape, std=1.0, to=dt: torch.from_numpy(rng.standard_normal(shape) * std).to(to).cuda()  # noqa: E731
        self.X, self.W_gate = wl.X.cuda(), wl.W.cuda()
        self.W_up, self.W_down, self.dY = new(E, 2 * f, d, std=d ** -0.5), new(E, d, f, std=f ** -0.5), new(T, d)
        self.norm = (1 + new(d, std=0.2, to=F32), new(d, std=0.2, to=F32))
        self.M = torch.from_numpy(np.stack([a := rng.random(T), 1 - a], 1).astype(np.float32)).cuda()
        self.layer = lambda **kw: module.MoELayer(T, d, f, E, k, 4, wl.sample_offsets, wl.expert_bin, self.code, **kw)
        self.T, self.E, self.k = T, E, k

    def oracle(self, idx, balance_scale, mi_scale, norm):
        """(Y, dX, dW_gate, dW_up, dW_down, dnorm_w, dnorm_b, balance loss, counts)."""
        wl, X, dY = self.wl, host(self.X), host(self.dY)
        Wg, Wu, Wd, M = host(self.W_gate), host(self.W_up), host(self.W_down), host(self.M)
        N, mean, rstd = OL.norm(X, host(self.norm[0]), host(self.norm[1]), 1e-5) if norm else (X, None, None)
        fwd = O.router_forward_variant(N, Wg, M, wl.expert_bin, 4, wl.sample_offsets, self.k, topk_idx=idx)
        off, row_slot, slot_row = OE.sort(idx, self.E)
        Ns = OE.dispatch(N, row_slot, self.k)
        H, z = OE.linear(Ns, Wu, off, None, OE.SILU, True)
        Ys, _ = OE.linear(H, Wd, off)
        Y = OE.back(Ys, slot_row, fwd["topk_w"], X)
        loss, counts, _, t = OL.expert_balance(fwd["g"], idx, wl.sample_offsets, balance_scale)
        dYs, dw = OE.combine_bwd(dY, Ys, fwd["topk_w"], slot_row)
        dH, dWd = OE.linear_bwd(dYs, H, Wd, off)
        dZ, _ = OE.act_bwd(dH, z, off, OE.SILU, True)
        dNs, dWu = OE.linear_bwd(dZ, Ns, Wu, off)
        dz, _, _ = O.router_backward(N, Wg, M, fwd, wl.expert_bin, wl.sample_offsets, mi_scale, d_topk_w=dw)
        dz = dz + OL.gate_grad_logits(fwd["g"], t, 1.0)
        dN = OE.back(dNs, slot_row, None, dz @ Wg)
        if not norm:
            return Y, dN + dY, dz.T @ N, dWu, dWd, None, None, loss, counts
        dX, dnw, dnb = OL.norm_bwd(dN, X, mean, rstd, host(self.norm[0]), dY)
        return Y, dX, dz.T @ N, dWu, dWd, dnw, dnb, loss, counts


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("dt", [F32, BF16], ids=["fp32", "bf16"])
def test_training_with_norm_and_balance(layer_module, dt, norm):
    c = Case(layer_module, dt)
    layer = c.layer(norm_eps=1e-5 if norm else None, balance="sample")
    kw = dict(M_in=c.M, norm=c.norm if norm else None)
    Y = layer.forward(c.X, c.W_gate, c.W_up, c.W_down, balance_scale=20.0, **kw)
    served = layer.forward(c.X, c.W_gate, c.W_up, c.W_down, training=False, **kw)
    assert torch.equal(Y, served)
    dX = layer.backward(c.dY, loss_scale=0.5)
    assert layer.router.device_status()[0] == layer.experts.device_status() == c.bd.SMOES_OK
    want = c.oracle(layer.router.topk_idx.cpu().numpy(), 20.0, 0.5, norm)
    tol = 2e-3 if dt is F32 else 1e-2
    got = (Y, dX, layer.dW_gate, layer.dW_up, layer.dW_down, layer.dnorm_w, layer.dnorm_b)
    for name, a, b in zip(("Y", "dX", "dW_gate", "dW_up", "dW_down", "dnorm_w", "dnorm_b"), got, want):
        assert (a is None) == (b is None) and (a is None or rel(a, b) < tol), (name, rel(a, b))
    assert abs(float(layer.balance_loss) - want[7]) <= 1e-3 * want[7]
    assert np.array_equal(layer.expert_counts.cpu().numpy(), want[8])
    kept = [t.clone() for t in got[2:] if t is not None]
    again = layer.backward(c.dY, loss_scale=0.5, accumulate=True)
    assert torch.equal(again, dX) and all(torch.equal(t, 2 * b) for t, b in zip([t for t in got[2:] if t is not None], kept))
    # and the balance loss does move the gradient
    plain = c.layer(norm_eps=1e-5 if norm else None)
    plain.forward(c.X, c.W_gate, c.W_up, c.W_down, **kw)
    plain.backward(c.dY, loss_scale=0.5)
    assert not torch.equal(plain.dW_gate, kept[0]) and torch.equal(plain.dW_up, kept[1])


def test_balance_over_the_batch(layer_module):
    c = Case(layer_module, BF16)
    layer = c.layer(balance="batch")
    layer.forward(c.X, c.W_gate, c.W_up, c.W_down, M_in=c.M)
    layer.backward(c.dY)
    assert layer.expert_counts.shape == (1, c.E) and int(layer.expert_counts.sum()) == c.T * c.k


@pytest.mark.parametrize("norm", [True, False])
def test_serving_in_4_bits(layer_module, norm):
    """The steps of the layer one by one, each by the oracle from the stored result of the one before; the products keep the
    bf16 layer's tolerance, of each element: one rounding (2^-8) and n_in steps of 2^-23 of the sum of magnitudes."""
    c = Case(layer_module, BF16)
    bd = c.bd
    layer = c.layer(norm_eps=1e-5 if norm else None)
    kw = dict(M_in=c.M, norm=c.norm if norm else None, training=False)
    Qu, Qd = bd.mx_quantise(c.W_up), bd.mx_quantise(c.W_down)
    Y = layer.forward(c.X, c.W_gate, Qu, Qd, **kw)
    r, ex = layer.router, layer.experts
    assert r.device_status()[0] == ex.device_status() == bd.SMOES_OK
    N = layer.norm.forward(c.X, *c.norm)[0] if norm else c.X
    off, row_slot, slot_row = OE.sort(r.topk_idx.cpu().numpy(), c.E)
    values = lambda q: OL.mx_values(*(t.cpu().numpy() for t in q))  # noqa: E731
    H = ex.linear_mx(ex.dispatch_mx(N), Qu, act=bd.SMOES_ACT_SILU, gated=True)
    x = OE.dispatch(OL.mx_values(*OL.mx_quantise(host(N))), row_slot, c.k)
    want, z = OE.linear(x, values(Qu), off, None, OE.SILU, True)
    assert rel(H, want) < 2.0 ** -8
    h = OL.mx_values(*OL.mx_quantise(host(H)))
    Ys, _ = OE.linear(h, values(Qd), off)
    w = host(r.topk_w)
    size = np.concatenate([np.abs(h[off[e]:off[e + 1]]) @ np.abs(values(Qd)[e]).T for e in range(c.E)])
    want = OE.back(Ys, slot_row, w, host(c.X))
    tol = OE.back(2.0 ** -8 * np.abs(Ys) + h.shape[1] * 2.0 ** -23 * size, slot_row, w) + 2.0 ** -8 * np.abs(want) + 2.0 ** -21 * (
        np.abs(host(c.X)) + OE.back(np.abs(Ys), slot_row, w))
    assert (np.abs(host(Y) - want) <= tol).all()
    # a training forward and its backward are not disturbed by serving in between
    kw.pop("training")
    layer.forward(c.X, c.W_gate, c.W_up, c.W_down, **kw)
    dX = layer.backward(c.dY)
    layer.forward(c.X.flip(0), c.W_gate, Qu, Qd, training=False, **kw)
    assert torch.equal(layer.backward(c.dY), dX)


def test_arguments_are_refused(layer_module):
    c = Case(layer_module, BF16)
    bd, layer = c.bd, c.layer()
    Qu, Qd = bd.mx_quantise(c.W_up), bd.mx_quantise(c.W_down)
    for args, kw in (((Qu, Qd), dict()), ((Qu, c.W_down), dict(training=False)), ((c.W_up, Qd), dict(training=False))):
        with pytest.raises(ValueError, match="4 bits"):
            layer.forward(c.X, c.W_gate, *args, M_in=c.M, **kw)
    with pytest.raises(ValueError, match="norm"):
        layer.forward(c.X, c.W_gate, c.W_up, c.W_down, M_in=c.M, norm=c.norm)
    with pytest.raises(ValueError, match="norm"):
        c.layer(norm_eps=1e-5).forward(c.X, c.W_gate, c.W_up, c.W_down, M_in=c.M)
    with pytest.raises(ValueError, match="balance"):
        c.layer(balance="layer")


def test_the_command_times_a_step(layer_module, capsys):
    layer_module._step_times("tiny_fp32", 64, 4, steps=1, norm=True, balance="sample")
    assert "training step" in capsys.readouterr().out
