"""GPU parity of the microscaled 4-bit calls: quantisation and its inverse bit for bit, and the experts' products against
the fp64 oracle on the same codes.

Tolerance of the products, from the arithmetic: a product of two 4-bit values with their scales is exact; each of the n_in
additions in fp32 is off by a step of 2^-23 of the sum of magnitudes at most (the tensor cores cut off); bias, activation (slopes
at most 1.13, the functions good to 2^-18 of |z| + 1), gate and residual as in the bf16 layer; one rounding to bf16, 2^-8."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as E_
from oracle import layer_oracle as O

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
U_BF16, U_F32 = 2.0 ** -8, 2.0 ** -23


@pytest.fixture(scope="module")
def bd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2604_23996_gb300 import binding
    return binding


def host(t):
    return t.detach().double().cpu().numpy()


def assert_close(got, want, tol, what):
    got = host(got)
    bad = ~(np.abs(got - want) <= tol)
    assert got.shape == want.shape and not bad.any(), (
        f"{what}: {bad.sum()} of {bad.size} out of tolerance, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}")


def hard_values(rng, rows, n, dt):
    """Every size and the middles between them at many exponents, zeros, the ends of the type's range."""
    edges = np.array([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7, 7.5])
    x = rng.choice(edges, (rows, n)) * rng.choice([-1.0, 1.0], (rows, n))
    x *= 2.0 ** rng.integers(-149, 122, (rows, n // 32)).repeat(32, 1)
    plain = rng.random((rows, n // 32)).repeat(32, 1) < 0.5
    x = np.where(plain, rng.standard_normal((rows, n)), x)
    x[0, :32] = 0
    return torch.from_numpy(x.astype(np.float32)).to(dt)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("rows,n", [(1, 32), (3, 96), (64, 32), (33, 1440), (700, 2048), (5, 32 * 129)])
def test_quantise_and_back(bd, rows, n, dt):
    X = hard_values(np.random.default_rng(rows + n), rows, n, dt)
    q, s = O.mx_quantise(host(X))
    got = bd.mx_quantise(X.cuda())
    assert np.array_equal(got.codes.cpu().numpy(), q) and np.array_equal(got.scales.cpu().numpy(), s)
    values = O.mx_values(q, s)
    assert np.array_equal(host(bd.mx_dequantise(got, F32)), values)
    assert np.array_equal(host(bd.mx_dequantise(got)), values)               # exact in bf16 too
    again = bd.mx_quantise(bd.mx_dequantise(got))       # what is a 4-bit value already stays it
    assert np.array_equal(host(bd.mx_dequantise(again)), values)


def test_every_code_with_every_scale(bd):
    codes = torch.arange(256, dtype=torch.uint8).repeat(256).view(256, 256)             # 16 blocks of 16 pairs a row
    scales = torch.arange(256, dtype=torch.uint8).view(256, 1).repeat(1, 16).contiguous()
    want = O.mx_values(codes.numpy(), scales.numpy())
    for dt in (BF16, F32):
        got = bd.mx_dequantise(bd.Mx(codes.cuda(), scales.cuda()), dt)
        assert torch.equal(got.cpu().float().nan_to_num(7e30), torch.from_numpy(want).to(dt).float().nan_to_num(7e30))


def test_blocks_that_are_not_finite(bd):
    X = torch.randn(4, 96)
    X[0, 5], X[1, 40], X[2, 95] = float("nan"), float("inf"), -float("inf")
    for dt in (BF16, F32):
        x = X.to(dt)
        q, s = O.mx_quantise(host(x))
        got = bd.mx_quantise(x.cuda())
        assert np.array_equal(got.codes.cpu().numpy(), q) and np.array_equal(got.scales.cpu().numpy(), s)
        assert got.scales[0, 0] == got.scales[1, 1] == got.scales[2, 2] == 255
        back = bd.mx_dequantise(got)
        assert back[0, :32].isnan().all() and int(back.isnan().sum()) == 96


class Layer:
    def __init__(self, bd, T, E, k, seed=0, dropped=0.0, route=None):
        rng = np.random.default_rng(seed)
        self.g = torch.Generator().manual_seed(seed)
        if route is not None:
            idx = rng.permutation(np.repeat(np.arange(E), route)).reshape(T, k).astype(np.int32)
        else:
            idx = np.argsort(-(rng.standard_normal((T, E)) + rng.standard_normal(E)), axis=1)[:, :k].astype(np.int32)
        if dropped:
            idx[rng.random((T, k)) < dropped] = -1
        self.off, self.row_slot, self.slot_row = E_.sort(idx, E)
        self.bd, self.ex, self.n, self.k = bd, bd.Experts(T, E, k), int(self.off[-1]), k
        self.ex.sort(torch.from_numpy(idx).cuda())

    def normal(self, *shape, std=1.0, dt=BF16):
        return (torch.randn(shape, generator=self.g) * std).to(dt).cuda()


@pytest.mark.parametrize("T,E,k,d,dropped", [(1, 8, 2, 32, 0.0), (7, 16, 3, 96, 0.3), (16, 64, 6, 2048, 0.0), (333, 48, 5, 1440, 0.1),
                                             (50, 256, 16, 64, 1.0), (6007, 1, 1, 160, 0.0)])
def test_dispatch(bd, T, E, k, d, dropped):
    lay = Layer(bd, T, E, k, seed=T, dropped=dropped)
    for dt in (BF16, F32):
        ex = lay.ex
        if dt is F32:
            ex = bd.Experts(T, E, k, bd.SMOES_F32)
            ex.expert_offsets, ex.slot_row = lay.ex.expert_offsets, lay.ex.slot_row
        X = lay.normal(T, d, dt=dt)
        q, s = O.mx_quantise(host(X))
        there = lay.row_slot >= 0
        want_q, want_s = np.zeros((T * k, d // 2), np.uint8), np.zeros((T * k, d // 32), np.uint8)
        want_q[there], want_s[there] = q[lay.row_slot[there] // k], s[lay.row_slot[there] // k]
        out = bd.Mx(torch.full((T * k, d // 2), 9, dtype=torch.uint8, device="cuda"),
                    torch.full((T * k, d // 32), 9, dtype=torch.uint8, device="cuda"))
        for got in (ex.dispatch_mx(X), ex.dispatch_mx(X, out=out)):
            assert np.array_equal(got.codes.cpu().numpy(), want_q) and np.array_equal(got.scales.cpu().numpy(), want_s)


def check_linear(lay, n_in, n_out, act=0, gated=False, bias=False, residual=False, spread=False):
    bd, ex = lay.bd, lay.ex
    n_z = n_out * (2 if gated else 1)
    X, W = lay.normal(ex.R, n_in, dt=F32), lay.normal(ex.E, n_z, n_in, std=n_in ** -0.5, dt=F32)
    if spread:                                          # every block with a scale of its own
        for t in (X, W):
            t.view(-1, 32).mul_(torch.exp2(torch.randint(-6, 7, (t.numel() // 32, 1), generator=lay.g).float()).cuda())
    qx, qw = bd.mx_quantise(X), bd.mx_quantise(W)
    qx.scales[lay.n:] = 255                             # rows of no expert hold NaN
    x, w = O.mx_values(*(t.cpu().numpy() for t in qx)), O.mx_values(*(t.cpu().numpy() for t in qw))
    x[lay.n:] = 0
    b = lay.normal(ex.E, n_z, std=0.3, dt=F32) if bias else None
    r = lay.normal(ex.R, n_out) if residual else None
    out = ex.linear_mx(qx, qw, bias=b, act=act, gated=gated, residual=r, out=torch.full((ex.R, n_out), float("nan"), dtype=BF16, device="cuda"))
    again = ex.linear_mx(qx, qw, bias=b, act=act, gated=gated, residual=r)
    assert ex.device_status() == bd.SMOES_OK and torch.equal(out, again)
    rh = None if r is None else host(r)
    if rh is not None:
        rh[lay.n:] = 0
    want, z = E_.linear(x, w, lay.off, None if b is None else host(b), act, gated, rh)
    size = np.zeros((ex.R, n_z))                        # sums of magnitudes
    for e in range(ex.E):
        a, c = lay.off[e], lay.off[e + 1]
        size[a:c] = np.abs(x[a:c]) @ np.abs(w[e]).T + (0 if b is None else np.abs(host(b)[e]))
    e_z = (n_in + 1) * U_F32 * size
    if gated:
        g, u = z[:, :n_out], z[:, n_out:]
        e_a = 1.13 * e_z[:, :n_out] + (0 if act == 0 else 2.0 ** -18 * (np.abs(g) + 1))
        tol = e_a * (np.abs(u) + e_z[:, n_out:]) + np.abs(E_.act(act, g)) * e_z[:, n_out:]
    else:
        tol = 1.13 * e_z + (0 if act == 0 else 2.0 ** -18 * (np.abs(z) + 1))
    tol = tol + 4 * U_F32 * (np.abs(want) + (0 if rh is None else np.abs(rh)))
    assert_close(out, want, tol + U_BF16 * np.abs(want), "out")


@pytest.mark.parametrize("n_in", [32, 64, 96, 128, 256, 288, 512, 1440, 2048])
def test_linear_depths(bd, n_in):
    check_linear(Layer(bd, 40, 4, 2, seed=n_in), n_in, 136, spread=True)


@pytest.mark.parametrize("n_out", [8, 24, 64, 72, 128, 136, 256, 520])
@pytest.mark.parametrize("gated", [False, True])
def test_linear_widths(bd, n_out, gated):
    check_linear(Layer(bd, 60, 3, 2, seed=n_out), 160, n_out, act=1 if gated else 0, gated=gated, bias=True, residual=True, spread=True)


@pytest.mark.parametrize("act,gated", [(0, False), (1, False), (2, False), (0, True), (1, True), (2, True)])
@pytest.mark.parametrize("bias,residual", [(False, False), (True, False), (False, True), (True, True)])
def test_linear_epilogues(bd, act, gated, bias, residual):
    check_linear(Layer(bd, 90, 5, 2, seed=3, dropped=0.2), 224, 88, act, gated, bias, residual)


ROUTES = [(1, 1, 1, None, 0.0), (1, 64, 6, None, 0.0), (16, 64, 6, None, 0.0), (31, 1, 1, None, 0.0), (33, 1, 1, None, 0.0), (193, 1, 1, None, 0.0),
          (1000, 1, 1, None, 0.0), (128, 8, 2, (0, 1, 31, 32, 33, 95, 64, 0), 0.0), (480, 6, 2, (191, 192, 193, 0, 383, 1), 0.0),
          (300, 256, 4, None, 0.1), (64, 16, 4, None, 1.0), (5000, 24, 4, None, 0.05)]


@pytest.mark.parametrize("T,E,k,route,dropped", ROUTES)
def test_linear_rows(bd, T, E, k, route, dropped):
    lay = Layer(bd, T, E, k, seed=T + E, dropped=dropped, route=route)
    check_linear(lay, 320, 144, spread=True)
    check_linear(lay, 544, 72, act=1, gated=True, residual=True)


def test_linear_large(bd):
    check_linear(Layer(bd, 4000, 16, 4, seed=9), 2048, 1024, act=1, gated=True)


def test_other_experts_do_not_reach_a_row(bd):
    """NaN in the weights and rows of one expert: the others' results keep their bits, its own become NaN."""
    lay = Layer(bd, 200, 4, 2, seed=5, route=(90, 100, 110, 100))
    ex = lay.ex
    X, W = bd.mx_quantise(lay.normal(ex.R, 128)), bd.mx_quantise(lay.normal(4, 136, 128))
    want = ex.linear_mx(X, W)
    a, b = int(lay.off[1]), int(lay.off[2])
    W.scales[1], X.scales[a:b] = 255, 255
    got = ex.linear_mx(X, W)
    assert got[a:b].isnan().all() and torch.equal(got[:a], want[:a]) and torch.equal(got[b:], want[b:])
    assert not want.isnan().any()


def test_one_nan_block_reaches_its_row_alone(bd):
    lay = Layer(bd, 70, 1, 1, seed=6)
    X, W = bd.mx_quantise(lay.normal(70, 352)), bd.mx_quantise(lay.normal(1, 40, 352))
    want = lay.ex.linear_mx(X, W)
    X.scales[13, 10] = 255
    got = lay.ex.linear_mx(X, W)
    assert got[13].isnan().all()
    got[13] = want[13]
    assert torch.equal(got, want)


def test_serving_step_and_graph(bd):
    """Dispatch, gated up-projection, quantisation, down-projection and combine as a decoding step makes them, captured and
    replayed on other tokens, against the steps one by one."""
    T, E, k, d, f = 16, 8, 2, 256, 160
    lay = Layer(bd, T, E, k, seed=1)
    ex = lay.ex
    Wu, Wd = bd.mx_quantise(lay.normal(E, 2 * f, d, std=d ** -0.5)), bd.mx_quantise(lay.normal(E, d, f, std=f ** -0.5))
    w = torch.rand(T, k, generator=lay.g).cuda()
    X = lay.normal(T, d)

    def step():
        H = ex.linear_mx(ex.dispatch_mx(X), Wu, act=bd.SMOES_ACT_SILU, gated=True)
        return ex.combine(ex.linear_mx(bd.mx_quantise(H), Wd), w, residual=X)

    # step by step, each from the stored result of the one before
    Y, Xq = step(), ex.dispatch_mx(X)
    H = ex.linear_mx(Xq, Wu, act=bd.SMOES_ACT_SILU, gated=True)
    wd = O.mx_values(*(t.cpu().numpy() for t in Wd))
    h = O.mx_values(*O.mx_quantise(host(H)))
    Ys, _ = E_.linear(h, wd, lay.off)
    size = sum(np.abs(h) @ np.abs(wd[e]).T for e in range(E)) * f * U_F32
    want = E_.back(Ys, lay.slot_row, host(w), host(X))
    tol = E_.back(U_BF16 * np.abs(Ys) + size, lay.slot_row, host(w)) + 4 * U_F32 * (np.abs(host(X)) + E_.back(np.abs(Ys), lay.slot_row, host(w)))
    assert_close(Y, want, tol + U_BF16 * np.abs(want), "Y")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    X.copy_(lay.normal(T, d))
    graph.replay()
    assert torch.equal(out, step())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    q = bd.mx_quantise(X, stream=side)
    values = bd.mx_dequantise(q, stream=side)
    H = ex.linear_mx(ex.dispatch_mx(X, stream=side), Wu, act=1, gated=True, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(values, bd.mx_dequantise(bd.mx_quantise(X)))
    assert torch.equal(H, ex.linear_mx(ex.dispatch_mx(X), Wu, act=1, gated=True))


def test_nothing_to_do(bd):
    ex = bd.Experts(0, 4, 2)
    X = bd.Mx(torch.empty(0, 32, dtype=torch.uint8, device="cuda"), torch.empty(0, 2, dtype=torch.uint8, device="cuda"))
    W = bd.mx_quantise(torch.randn(4, 8, 64, device="cuda"))
    assert ex.linear_mx(X, W).shape == (0, 8)
    assert ex.dispatch_mx(torch.empty(0, 64, dtype=BF16, device="cuda")).codes.shape == (0, 32)
    assert bd.mx_dequantise(bd.mx_quantise(torch.empty(0, 64, device="cuda"))).shape == (0, 64)


def test_arguments_are_refused(bd):
    lay = Layer(bd, 8, 2, 1, seed=0)
    ex = lay.ex
    X, W = bd.mx_quantise(lay.normal(8, 64)), bd.mx_quantise(lay.normal(2, 16, 64))
    for bad in (torch.zeros(8, 40), torch.zeros(8, 64, dtype=torch.float16), torch.zeros(8, 64).t()):
        with pytest.raises(ValueError, match="X"):
            bd.mx_quantise(bad.cuda())
    with pytest.raises(ValueError, match="device"):
        bd.mx_quantise(torch.zeros(8, 64))
    with pytest.raises(ValueError, match="X"):
        ex.linear_mx(bd.Mx(X.codes[:4], X.scales[:4]), W)
    with pytest.raises(ValueError, match="X"):
        ex.linear_mx(bd.Mx(X.codes, X.scales[:, :1].contiguous()), W)
    with pytest.raises(ValueError, match="W"):
        ex.linear_mx(X, bd.Mx(W.codes, W.scales.int()))
    with pytest.raises(ValueError, match="W"):
        ex.linear_mx(X, bd.mx_quantise(lay.normal(2, 17, 64)), gated=True)
    with pytest.raises(bd.SmoesError):
        ex.linear_mx(X, W, act=5)
    f32 = bd.Experts(8, 2, 1, bd.SMOES_F32)
    with pytest.raises(bd.SmoesError) as e:
        f32.linear_mx(X, W)
    assert e.value.code == -2


def test_two_streams_at_once(bd):
    """Two layers' products and quantisations on two streams, many at a time: each its own result."""
    lays = [Layer(bd, 500, 8, 2, seed=s) for s in (1, 2)]
    data = [(bd.mx_quantise(lay.normal(lay.ex.R, 512)), bd.mx_quantise(lay.normal(8, 256, 512)), lay.normal(500, 512)) for lay in lays]
    want = [(lay.ex.linear_mx(x, w, act=1, gated=True), lay.ex.dispatch_mx(t)) for lay, (x, w, t) in zip(lays, data)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(25):
        for i, (lay, (x, w, t)) in enumerate(zip(lays, data)):
            got[i].append((lay.ex.linear_mx(x, w, act=1, gated=True, stream=streams[i]), lay.ex.dispatch_mx(t, stream=streams[i])))
    torch.cuda.synchronize()
    for i in range(2):
        assert lays[i].ex.device_status() == bd.SMOES_OK
        for out, q in got[i]:
            assert torch.equal(out, want[i][0]) and torch.equal(q.codes, want[i][1].codes) and torch.equal(q.scales, want[i][1].scales)


def test_graphs_that_share_a_workspace(bd):
    """Two captured graphs of one layer, replayed in turn on one stream."""
    lay = Layer(bd, 300, 8, 2, seed=4)
    ex = lay.ex
    X, Wa, Wb = lay.normal(300, 256), bd.mx_quantise(lay.normal(8, 128, 256)), bd.mx_quantise(lay.normal(8, 64, 256))
    graphs, outs = [], []
    for W in (Wa, Wb):
        ex.linear_mx(ex.dispatch_mx(X), W)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(ex.linear_mx(ex.dispatch_mx(X), W))
        graphs.append(g)
    for seed in range(3):
        X.copy_(lay.normal(300, 256))
        for g in graphs:
            g.replay()
        for out, W in zip(outs, (Wa, Wb)):
            assert torch.equal(out, ex.linear_mx(ex.dispatch_mx(X), W))
