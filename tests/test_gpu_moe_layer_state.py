"""What the MoE layer keeps between its calls: gradients of several batches added up, and the forward that a backward belongs
to."""
import pytest
import torch

from paper_2604_23996_gb300.workloads import random_router_case

pytestmark = pytest.mark.gpu

T, d, f, E, k, N_BINS = 300, 136, 72, 16, 3, 4
BUFFERS = ("dW_gate", "dW_up", "dW_down", "db_up", "db_down")


class Case:
    """A layer with biases, its weights, and batches."""

    def __init__(self, dt, biases=True):
        if not torch.cuda.is_available():
            pytest.skip("no GPU")
        from paper_2604_23996_gb300 import moe_layer
        self.bd = moe_layer.bd
        self.wl = random_router_case(7, T=T, d=d, E=E, k=k, n_bins=N_BINS, sample_lengths=[100, 150, 50], dtype=dt, aligned=True)
        self.g = torch.Generator(device="cuda").manual_seed(3)
        self.dt = dt
        self.W = (self.wl.W.cuda(), self.normal(E, 2 * f, d, std=d ** -0.5), self.normal(E, d, f, std=f ** -0.5))
        self.b = dict(b_up=self.normal(E, 2 * f, std=0.1, dtype=torch.float32),
                      b_down=self.normal(E, d, std=0.1, dtype=torch.float32)) if biases else {}
        self.stats = dict(mu=self.wl.mu.cuda(), var=self.wl.var.cuda(), tau=self.wl.tau)
        code = self.bd.SMOES_BF16 if dt is torch.bfloat16 else self.bd.SMOES_F32
        self.layer = moe_layer.MoELayer(T, d, f, E, k, N_BINS, self.wl.sample_offsets, self.wl.expert_bin, code, biases=biases)

    def normal(self, *shape, std=1.0, dtype=None):
        return (torch.randn(shape, generator=self.g, device="cuda") * std).to(dtype or self.dt)

    def forward(self, X, **kw):
        return self.layer.forward(X, *self.W, **self.stats, **self.b, **kw)

    def gradients(self):
        return {n: getattr(self.layer, n).clone() for n in BUFFERS if getattr(self.layer, n) is not None}


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
def test_gradients_of_two_batches_add_up(dt):
    c = Case(dt)
    batches = [(c.normal(T, d), c.normal(T, d)) for _ in range(2)]
    alone = []
    for X, dY in batches:
        c.forward(X)
        c.layer.backward(dY)
        alone.append(c.gradients())
    c.forward(batches[0][0])
    c.layer.backward(batches[0][1])
    c.forward(batches[1][0])
    c.layer.backward(batches[1][1], accumulate=True)
    for name, got in c.gradients().items():
        assert torch.equal(got, alone[0][name] + alone[1][name]), name


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("between", [1, 3])
def test_a_forward_between_leaves_the_backward_as_it_is(dt, between):
    """Other tokens evaluated between a training forward and its backward: the gradients are the same bits as without."""
    c = Case(dt)
    X, dY = c.normal(T, d), c.normal(T, d)
    c.forward(X)
    want_x = c.layer.backward(dY, loss_scale=0.5)
    want = c.gradients()
    Y = c.forward(X)
    for _ in range(between):
        other = c.normal(T, d)
        got = c.forward(other, training=False)
        assert torch.isfinite(got).all() and not torch.equal(got, Y)
    evaluated = c.layer.router.topk_idx.clone(), c.layer.router.loss.clone()
    assert torch.equal(c.layer.backward(dY, loss_scale=0.5), want_x)
    for name, got in c.gradients().items():
        assert torch.equal(got, want[name]), name
    # the router's results stay those of the last forward; a backward can be repeated; the next step is its own
    assert torch.equal(c.layer.router.topk_idx, evaluated[0]) and torch.equal(c.layer.router.loss, evaluated[1])
    assert torch.equal(c.layer.backward(dY, loss_scale=0.5), want_x)
    again = c.forward(X)
    assert torch.equal(again, Y) and torch.equal(c.layer.backward(dY, loss_scale=0.5), want_x)
    assert c.layer.router.device_status()[0] == c.layer.experts.device_status() == c.bd.SMOES_OK


def test_an_evaluation_gives_what_it_gives_alone():
    c = Case(torch.bfloat16)
    X, other = c.normal(T, d), c.normal(T, d)
    want = c.forward(other, training=False)
    c.forward(X)
    assert torch.equal(c.forward(other, training=False), want)


def test_the_backward_is_that_of_the_last_training_forward():
    c = Case(torch.float32)
    X1, X2, dY = c.normal(T, d), c.normal(T, d), c.normal(T, d)
    c.forward(X2)
    want = c.layer.backward(dY)
    c.forward(X1)
    c.forward(X1, training=False)
    c.forward(X2)
    assert torch.equal(c.layer.backward(dY), want)


def test_a_backward_without_a_training_forward_is_refused():
    c = Case(torch.bfloat16)
    dY = c.normal(T, d)
    with pytest.raises(RuntimeError):
        c.layer.backward(dY)
    c.forward(c.normal(T, d), training=False)
    with pytest.raises(RuntimeError):
        c.layer.backward(dY)
    with pytest.raises(c.bd.SmoesError):
        c.forward(None)
    with pytest.raises(RuntimeError):
        c.layer.backward(dY)
