"""GPU parity of the layer norm and its gradients against the fp64 oracle on the same stored inputs.

Tolerances, from the arithmetic: a result of type t is rounded once, half a step of t at most (bf16 2^-8, fp32 2^-24 of the
value). In fp32 every operation is off by 2^-24 of its result at most; a row's sum is at most 64 additions in a row in a
thread, 5 across a warp and 32 across warps: n = 101 roundings of the sum of magnitudes. The sums over the rows: a thread
adds the rows of its block (at most T / 100 and 16 more), then at most 32 groups,
the blocks of a slice and the slices (fewer than 32 + 12) are added."""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as O

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
N_ROW = 101
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def bd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2604_23996_gb300 import binding
    return binding


def host(t):
    return t.detach().double().cpu().numpy()


def code(bd, dt):
    return bd.SMOES_BF16 if dt is BF16 else bd.SMOES_F32


def assert_close(got, want, tol, what):
    got = host(got)
    bad = ~(np.abs(got - want) <= tol)
    assert got.shape == want.shape and not bad.any(), (
        f"{what}: {bad.sum()} of {bad.size} out of tolerance, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}")


class Case:
    def __init__(self, bd, T, d, dt, shift=0.0, seed=0, eps=1e-5):
        g = torch.Generator().manual_seed(1000 * T + d + seed)
        new = lambda *shape, std=1.0, to=dt: (torch.randn(shape, generator=g) * std).to(to).cuda()  # noqa: E731
        self.X, self.r, self.dY, self.ds = new(T, d) + shift, new(T, d), new(T, d), new(T, d)
        self.w, self.b = 1 + new(d, std=0.3, to=F32), new(d, to=F32)
        self.norm = bd.LayerNorm(T, d, code(bd, dt), eps=eps)
        self.dt, self.eps = dt, eps


def check_forward(c, residual, bias):
    Y, S, mean, rstd = c.norm.forward(c.X, c.w, c.b if bias else None, residual=c.r if residual else None)
    if residual:                                        # one rounding of an exact sum: the same bits
        assert torch.equal(S, (c.X.double() + c.r.double()).to(c.dt))
    else:
        assert S is c.X
    s, w = host(S), host(c.w)
    want, m, q = O.norm(s, w, host(c.b) if bias else None, c.eps)
    e_mean = N_ROW * U * np.abs(s).mean(1) + U * np.abs(m)
    # the variance around a mean that is off by e is larger by e^2; its sum and the root: (n + 4) / 2 + 3 roundings
    e_rstd = q * (((N_ROW + 4) / 2 + 3) * U) + q ** 3 * e_mean ** 2
    assert_close(mean, m, e_mean, "mean")
    assert_close(rstd, q, e_rstd, "rstd")
    h = np.abs(s - m[:, None])
    e_h = q[:, None] * (e_mean[:, None] + U * h) + h * e_rstd[:, None] + 2 * U * h * q[:, None]
    tol = np.abs(w) * e_h + 2 * U * (h * q[:, None] * np.abs(w) + np.abs(want)) + HALF[c.dt] * np.abs(want)
    assert_close(Y, want, tol, "Y")
    return S, mean, rstd


def check_backward(c, S, mean, rstd, residual):
    T, d = c.X.shape
    dX, dw, db = c.norm.backward(c.dY, S, mean, rstd, c.w, residual=c.ds if residual else None)
    s, dy, w, m, q = host(S), host(c.dY), host(c.w), host(mean)[:, None], host(rstd)[:, None]
    want = O.norm_bwd(dy, s, host(mean), host(rstd), w, host(c.ds) if residual else None)
    h, a = (s - m) * q, dy * w
    e_h = 2 * U * np.abs(h)
    e_ma = (N_ROW + 2) * U * np.abs(a).mean(1, keepdims=True)
    e_mah = (N_ROW + 5) * U * np.abs(a * h).mean(1, keepdims=True)
    ma, mah = np.abs(a.mean(1, keepdims=True)), np.abs((a * h).mean(1, keepdims=True))
    tol = q * (e_ma + np.abs(h) * e_mah + e_h * mah + 4 * U * (np.abs(a) + ma + np.abs(h) * mah)) + 3 * U * np.abs(want[0])
    assert_close(dX, want[0], tol + HALF[c.dt] * np.abs(want[0]), "dX")
    n = -(-T // 100) + 16 + 32 + 44
    assert_close(dw, want[1], (n * U * np.abs(dy * h) + np.abs(dy) * e_h + U * np.abs(dy * h)).sum(0), "dw")
    assert_close(db, want[2], n * U * np.abs(dy).sum(0), "db")
    return dX, dw, db


SHAPES = [(1, 8, BF16), (3, 16, F32), (5, 64, BF16), (7, 72, F32), (130, 104, BF16), (33, 264, BF16), (129, 520, F32),
          (17, 1032, BF16), (40, 2048, BF16), (6, 2056, BF16), (5, 2056, F32), (9, 4104, BF16), (5, 8192, F32), (3, 16384, BF16),
          (4099, 512, F32), (3001, 256, BF16), (1, 2048, BF16)]


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("T,d,dt", SHAPES)
def test_forward_and_backward(bd, T, d, dt, residual):
    c = Case(bd, T, d, dt)
    S, mean, rstd = check_forward(c, residual, bias=True)
    check_backward(c, S, mean, rstd, residual)


@pytest.mark.parametrize("dt,shift", [(F32, 1000.0), (F32, -3e5), (BF16, 100.0)])
def test_a_mean_far_from_zero(bd, dt, shift):
    c = Case(bd, 37, 512, dt, shift=shift)
    S, mean, rstd = check_forward(c, False, bias=False)
    check_backward(c, S, mean, rstd, False)


def test_gradients_against_differences(bd):
    """<dY, Y> in fp64 from the oracle's forward, by central differences along X, w and b."""
    c = Case(bd, 5, 24, F32)
    _, S, mean, rstd = c.norm.forward(c.X, c.w, c.b)
    dX, dw, db = (host(t) for t in c.norm.backward(c.dY, S, mean, rstd, c.w))
    x, w, b, dy = host(c.X), host(c.w), host(c.b), host(c.dY)
    f = lambda x, w, b: (dy * O.norm(x, w, b, c.eps)[0]).sum()  # noqa: E731
    rng, h = np.random.default_rng(0), 1e-5
    for _ in range(8):
        vx, vw, vb = rng.standard_normal(x.shape), rng.standard_normal(w.shape), rng.standard_normal(b.shape)
        slope = (f(x + h * vx, w + h * vw, b + h * vb) - f(x - h * vx, w - h * vw, b - h * vb)) / (2 * h)
        got = (dX * vx).sum() + (dw * vw).sum() + (db * vb).sum()
        # the differences' own error is h^2 times third derivatives (1e-10 here); fp32 gradients of 300 terms: 1e-5 of their size
        assert abs(got - slope) <= 1e-5 * (np.abs(dX * vx).sum() + np.abs(dw * vw).sum() + np.abs(db * vb).sum())


def test_rows_do_not_meet(bd):
    """A row of NaN and one of infinities leave the others' results as they are, the bits too."""
    c = Case(bd, 50, 136, BF16)
    Y, _, mean, rstd = c.norm.forward(c.X, c.w, c.b)
    dX, _, _ = c.norm.backward(c.dY, c.X, mean, rstd, c.w)
    X = c.X.clone()
    X[7], X[21, 3] = float("nan"), float("inf")
    keep = torch.ones(50, dtype=torch.bool)
    keep[7] = keep[21] = False
    Y2, _, mean2, rstd2 = c.norm.forward(X, c.w, c.b)
    dX2, _, _ = c.norm.backward(c.dY, X, mean2, rstd2, c.w)
    assert torch.equal(Y2[keep], Y[keep]) and torch.equal(dX2[keep], dX[keep])
    assert Y2[7].isnan().all() and Y2[21].isnan().any()


def test_accumulation_and_parts(bd):
    c = Case(bd, 700, 264, BF16)
    _, S, mean, rstd = c.norm.forward(c.X, c.w, c.b)
    dX, dw, db = c.norm.backward(c.dY, S, mean, rstd, c.w)
    again = c.norm.backward(c.dY, S, mean, rstd, c.w)
    assert all(torch.equal(a, b) for a, b in zip((dX, dw, db), again))       # the same bits
    aw, ab = dw.clone(), db.clone()
    c.norm.backward(c.dY, S, mean, rstd, c.w, dw=aw, db=ab, accumulate=True)
    assert torch.equal(aw, 2 * dw) and torch.equal(ab, 2 * db)
    only, none, b2 = c.norm.backward(c.dY, S, mean, rstd, c.w, need_dw=False)
    assert none is None and torch.equal(only, dX) and torch.equal(b2, db)
    only, none, none2 = c.norm.backward(c.dY, S, mean, rstd, c.w, need_dw=False, need_db=False)
    assert none is None and none2 is None and torch.equal(only, dX)
    Y, _, m, r = c.norm.forward(c.X, c.w, c.b, stats=False)
    assert m is None and r is None


def test_no_tokens(bd):
    n = bd.LayerNorm(0, 64)
    X, w = torch.empty(0, 64, dtype=BF16, device="cuda"), torch.ones(64, device="cuda")
    Y, S, mean, rstd = n.forward(X, w)
    assert Y.shape == (0, 64) and mean.shape == (0,)
    dw = torch.full((64,), 3.0, device="cuda")
    dX, _, db = n.backward(X, S, mean, rstd, w, dw=dw)
    assert not dw.any() and not db.any()
    dw.fill_(3.0)
    n.backward(X, S, mean, rstd, w, dw=dw, db=db, accumulate=True)
    assert (dw == 3).all()


def test_streams_and_graphs(bd):
    c = Case(bd, 300, 512, BF16)
    Y, S, mean, rstd = c.norm.forward(c.X, c.w, c.b, residual=c.r)
    want = c.norm.backward(c.dY, S, mean, rstd, c.w, residual=c.ds)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = c.norm.forward(c.X, c.w, c.b, residual=c.r, stream=side)
    got = c.norm.backward(c.dY, out[1], out[2], out[3], c.w, residual=c.ds, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out[0], Y) and all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = c.norm.forward(c.X, c.w, c.b, residual=c.r)
        got = c.norm.backward(c.dY, out[1], out[2], out[3], c.w, residual=c.ds)
    c.X.mul_(0.5)
    c.dY.neg_()
    graph.replay()
    Y2, S2, mean2, rstd2 = c.norm.forward(c.X, c.w, c.b, residual=c.r)
    want = c.norm.backward(c.dY, S2, mean2, rstd2, c.w, residual=c.ds)
    assert torch.equal(out[0], Y2) and all(torch.equal(a, b) for a, b in zip(got, want))


def test_arguments_are_refused(bd):
    c = Case(bd, 8, 64, BF16)
    n = c.norm
    for bad in (c.X[:4], c.X.float(), c.X.cpu(), c.X.t().contiguous().t()):
        with pytest.raises(ValueError, match="X"):
            n.forward(bad, c.w)
    with pytest.raises(ValueError, match="w"):
        n.forward(c.X, c.w.to(BF16))
    with pytest.raises(ValueError, match="sum_out"):
        n.forward(c.X, c.w, sum_out=torch.empty_like(c.X))
    with pytest.raises(ValueError, match="accumulate"):
        n.backward(c.dY, c.X, c.w[:8], c.w[:8], c.w, accumulate=True)
    with pytest.raises(bd.SmoesError):                  # a view that does not begin on 16 bytes
        n.forward(torch.empty(8 * 64 + 1, dtype=BF16, device="cuda")[1:].view(8, 64), c.w)
