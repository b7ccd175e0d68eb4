"""GPU parity of the expert layer (sort, dispatch, combine, the experts' products and the gradients)
against the plain fp64 oracle on the same stored inputs.

Maps are compared exactly, dispatch bitwise. Tolerances, fixed from the arithmetic before any run:
* a result in bf16 is rounded once: half a step, 2^-8 of the value at most (fp32: 2^-24, taken as 2^-23);
* a sum of n products in fp32 is off by at most n steps of 2^-23 of the sum of their magnitudes (the
  tensor cores cut each addition off where the FMA units round it: a whole step, not half);
* activations: slopes are at most 1.13 in magnitude (silu 1.10, gelu 1.13), so an error of z passes with
  that factor, and the functions themselves are good to 2^-18 of |z| + 1 (fast exponentials: a few
  steps of 2^-22 times an argument that stays below 16 where the result matters).
"""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as O

pytestmark = pytest.mark.gpu

U_BF16, U_F32 = 2.0 ** -8, 2.0 ** -23


@pytest.fixture(scope="module")
def bd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2604_23996_gb300 import binding
    return binding


def unit(dt):
    return U_BF16 if dt is torch.bfloat16 else U_F32


def host(t):
    return t.detach().double().cpu().numpy()


def assert_close(got, want, tol, what):
    got = host(got)
    assert got.shape == want.shape, what
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (f"{what}: {bad.sum()} of {bad.size} out of tolerance, first at {np.argwhere(bad)[0]}: "
                           f"{got[bad][0]} for {want[bad][0]}")


class Layer:
    """Seeded selections and inputs; every row past the last selection holds NaN in the inputs."""

    def __init__(self, bd, T, E, k, dt, seed=0, route="mixed", dropped=0.0, max_width=0):
        self.bd, self.T, self.E, self.k, self.dt = bd, T, E, k, dt
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        rng = np.random.default_rng(seed)
        if route == "mixed":                            # distinct experts, some liked better
            score = rng.standard_normal((T, E)) + rng.standard_normal(E)
            idx = np.argsort(-score, axis=1)[:, :k]
        elif route == "one":                            # every selection the same expert
            idx = np.full((T, k), E // 2)
        elif route == "ends":                           # the first and the last expert alone
            idx = rng.choice([0, E - 1], size=(T, k))
        else:                                           # counts given: route = rows of each expert
            idx = rng.permutation(np.repeat(np.arange(E), route)).reshape(T, k)
        idx = idx.astype(np.int32)
        if dropped:
            idx[rng.random((T, k)) < dropped] = -1
        self.idx = idx
        self.ex = bd.Experts(T, E, k, dtype=bd.SMOES_BF16 if dt is torch.bfloat16 else bd.SMOES_F32,
                             max_width=max_width)
        self.off, self.row_slot, self.slot_row = O.sort(idx, E)
        self.ex.sort(torch.from_numpy(idx).cuda())
        self.n = int(self.off[-1])
        w = rng.random((T, k)).astype(np.float32)
        self.w = torch.from_numpy(w).cuda()

    def normal(self, *shape, std=1.0, dtype=None):
        return (torch.randn(shape, generator=self.g, device="cuda") * std).to(dtype or self.dt)

    def rows(self, width, std=1.0):
        x = self.normal(self.ex.R, width, std=std)
        x[self.n:] = float("nan")
        return x

    def host_rows(self, x):
        x = host(x)
        x[self.n:] = 0.0
        return x


SORTS = [(1, 1, 1, "mixed", 0.0), (1, 8, 2, "mixed", 0.0), (7, 256, 16, "mixed", 0.2), (16, 64, 6, "mixed", 0.0),
         (333, 48, 5, "mixed", 0.1), (1000, 16, 2, "one", 0.0), (1365, 3, 6, "one", 0.5), (1366, 3, 6, "ends", 0.0),
         (5000, 128, 8, "mixed", 0.0), (9001, 7, 3, "mixed", 1.0), (60000, 128, 8, "mixed", 0.05),
         (20011, 256, 16, "mixed", 0.0)]


@pytest.mark.parametrize("T,E,k,route,dropped", SORTS)
def test_sort(bd, T, E, k, route, dropped):
    if route == "mixed" and k > E:
        route = "ends"
    lay = Layer(bd, T, E, k, torch.bfloat16, seed=T, route=route, dropped=dropped)
    for _ in range(2):                                  # the workspace is left as it was found
        lay.ex.row_slot.fill_(-7)
        lay.ex.slot_row.fill_(-7)
        off, row_slot, slot_row = lay.ex.sort(torch.from_numpy(lay.idx).cuda())
        assert np.array_equal(off.cpu().numpy(), lay.off)
        assert np.array_equal(row_slot.cpu().numpy(), lay.row_slot)
        assert np.array_equal(slot_row.cpu().numpy(), lay.slot_row)
    assert lay.ex.device_status() == bd.SMOES_OK


def test_sort_drops_and_reports_experts_that_do_not_exist(bd):
    ex = bd.Experts(3, 4, 2)
    off, row_slot, slot_row = ex.sort(torch.tensor([[3, 4], [0, 2 ** 31 - 1], [-2 ** 31, 3]], dtype=torch.int32,
                                                   device="cuda"))
    assert off.tolist() == [0, 1, 1, 1, 3]
    assert row_slot.tolist() == [2, 0, 5, -1, -1, -1]
    assert slot_row.tolist() == [[1, -1], [0, -1], [-1, 2]]
    assert ex.device_status() == -7                     # SMOES_ERR_DATA


TOKENS = [(1, 1, 1, 8, "mixed", 0.0), (1, 64, 6, 2048, "mixed", 0.0), (333, 48, 5, 1416, "mixed", 0.1),
          (130, 16, 2, 256, "one", 0.0), (77, 32, 4, 264, "mixed", 1.0), (65, 32, 16, 520, "mixed", 0.3),
          (200, 12, 3, 8, "ends", 0.0), (50, 20, 7, 1032, "mixed", 0.0)]


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("T,E,k,d,route,dropped", TOKENS)
def test_rows_there_and_back(bd, T, E, k, d, route, dropped, dt):
    if dt is torch.float32:
        d = d // 2                                      # odd counts of 16-byte words for both
    lay = Layer(bd, T, E, k, dt, seed=d + T, route=route, dropped=dropped)
    X = lay.normal(T, d)
    Xs = lay.ex.dispatch(X, out=torch.full((T * k, d), float("nan"), dtype=dt, device="cuda"))
    assert np.array_equal(host(Xs), O.dispatch(host(X), lay.row_slot, k))

    rows, res = lay.rows(d), lay.normal(T, d)
    w = host(lay.w)
    mag = O.back(np.abs(lay.host_rows(rows)), lay.slot_row, np.abs(w), np.abs(host(res)))
    for residual in (None, res):
        r = None if residual is None else host(residual)
        want = O.back(lay.host_rows(rows), lay.slot_row, w, r)
        assert_close(lay.ex.combine(rows, lay.w, residual=residual), want, unit(dt) * np.abs(want) + (k + 1) * U_F32 * mag,
                     "combine")
        want = O.back(lay.host_rows(rows), lay.slot_row, None, r)
        m1 = O.back(np.abs(lay.host_rows(rows)), lay.slot_row, None, np.abs(host(res)))
        assert_close(lay.ex.dispatch_bwd(rows, residual=residual), want, unit(dt) * np.abs(want) + (k + 1) * U_F32 * m1,
                     "dispatch_bwd")

    dY = lay.normal(T, d)
    dYs, dw = lay.ex.combine_bwd(dY, rows, lay.w, dYs=torch.full_like(rows, float("nan")))
    want_s, want_w = O.combine_bwd(host(dY), lay.host_rows(rows), w, lay.slot_row)
    assert_close(dYs, want_s, unit(dt) * np.abs(want_s), "dYs")
    _, mag_w = O.combine_bwd(np.abs(host(dY)), np.abs(lay.host_rows(rows)), w, lay.slot_row)
    assert_close(dw, want_w, d * U_F32 * mag_w, "dw")


def test_combine_is_the_transpose_of_its_gradient(bd):
    """<combine(Ys), dY> changes with Ys and w as combine_bwd says: exact differences, the map is bilinear."""
    lay = Layer(bd, 40, 8, 3, torch.float32, seed=5, dropped=0.2)
    Ys, dY = lay.normal(120, 64), lay.normal(40, 64)
    Ys[lay.n:] = 0
    dYs, dw = lay.ex.combine_bwd(dY, Ys, lay.w)
    vY, vw = lay.normal(120, 64), lay.normal(40, 3)
    L = lambda y, w: float((host(lay.ex.combine(y, w)) * host(dY)).sum())  # noqa: E731
    eps = 0.5                                           # linear in each: no truncation error
    mag = float((O.back(np.abs(host(Ys)) + np.abs(host(vY)), lay.slot_row, np.abs(host(lay.w)) + np.abs(host(vw)))
                 * np.abs(host(dY))).sum())
    tol = 64 * U_F32 * mag / eps
    dY_fd = (L(Ys + eps * vY, lay.w) - L(Ys - eps * vY, lay.w)) / (2 * eps)
    dw_fd = (L(Ys, lay.w + eps * vw) - L(Ys, lay.w - eps * vw)) / (2 * eps)
    vY[lay.n:] = 0
    assert abs(dY_fd - float((host(dYs) * host(vY)).sum())) <= tol
    assert abs(dw_fd - float((host(dw) * host(vw)).sum())) <= tol


# T, E, k, n_in, n_out, act, gated, bias, residual, pre, route, dropped
PRODUCTS = [
    (1, 1, 1, 8, 8, 0, False, False, False, False, "mixed", 0.0),
    (1, 8, 2, 64, 64, 1, True, False, False, True, "mixed", 0.0),
    (16, 64, 6, 256, 128, 1, True, True, False, False, "mixed", 0.0),
    (129, 1, 1, 136, 264, 2, False, True, True, True, "mixed", 0.0),
    (333, 12, 5, 200, 88, 1, True, True, True, True, "mixed", 0.1),
    (500, 6, 2, 512, 256, 0, False, False, True, False, "ends", 0.0),
    (300, 4, 1, 72, 520, 2, True, True, False, True, (0, 1, 298, 1), 0.0),
    (515, 5, 1, 320, 304, 1, False, False, False, True, (127, 128, 129, 131, 0), 0.0),
    (1030, 5, 1, 128, 256, 0, False, True, False, False, (255, 256, 257, 0, 262), 0.0),
    (64, 256, 16, 40, 24, 2, False, True, True, False, "mixed", 0.5),
    (70, 9, 3, 1032, 40, 1, False, True, False, False, "mixed", 1.0),
    (700, 3, 1, 1416, 712, 1, True, True, True, False, (13, 680, 7), 0.0),
]


def z_bound(X, W, off, bias):
    mag, _ = O.linear(np.abs(X), np.abs(W), off, None if bias is None else np.abs(bias))
    return (X.shape[1] + 2) * U_F32 * mag


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("case", PRODUCTS, ids=[str(i) for i in range(len(PRODUCTS))])
def test_linear(bd, case, dt):
    T, E, k, n_in, n_out, act, gated, bias, residual, pre, route, dropped = case
    lay = Layer(bd, T, E, k, dt, seed=n_in + T, route=list(route) if isinstance(route, tuple) else route, dropped=dropped)
    n_z = n_out * (2 if gated else 1)
    X, W = lay.rows(n_in), lay.normal(E, n_z, n_in, std=n_in ** -0.5)
    b = lay.normal(E, n_z, std=0.3, dtype=torch.float32) if bias else None
    res = lay.rows(n_out) if residual else None
    nan = lambda *s: torch.full(s, float("nan"), dtype=dt, device="cuda")  # noqa: E731
    out, z = lay.ex.linear(X, W, bias=b, act=act, gated=gated, residual=res, out=nan(T * k, n_out),
                           pre=nan(T * k, n_z) if pre else None)
    Xh, Wh, bh = lay.host_rows(X), host(W), None if b is None else host(b)
    want, want_z = O.linear(Xh, Wh, lay.off, bh, act, gated, None if res is None else lay.host_rows(res))
    tol_z = z_bound(Xh, Wh, lay.off, bh)
    if pre:
        assert_close(z, want_z, unit(dt) * np.abs(want_z) + tol_z, "pre")
    else:
        assert z is None
    g, tol_g = want_z[:, :n_out], tol_z[:, :n_out]
    tol = 1.13 * tol_g + (2.0 ** -18 * (np.abs(g) + 1) if act else 0.0)
    if gated:
        u, tol_u = want_z[:, n_out:], tol_z[:, n_out:]
        tol = tol * (np.abs(u) + tol_u) + np.abs(O.act(act, g)) * tol_u
    tol = tol + unit(dt) * np.abs(want) + 4 * U_F32 * (0.0 if res is None else np.abs(lay.host_rows(res)))
    tol[lay.n:] = 0.0
    assert_close(out, want, tol, "out")
    again, _ = lay.ex.linear(X, W, bias=b, act=act, gated=gated, residual=res)
    assert torch.equal(out, again)
    assert lay.ex.device_status() == bd.SMOES_OK


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("case", PRODUCTS, ids=[str(i) for i in range(len(PRODUCTS))])
def test_act_bwd(bd, case, dt):
    T, E, k, _, n_out, act, gated, bias, _, _, route, dropped = case
    n_z = n_out * (2 if gated else 1)
    lay = Layer(bd, T, E, k, dt, seed=n_out + T, route=list(route) if isinstance(route, tuple) else route,
                dropped=dropped, max_width=n_z)
    dOut, z = lay.rows(n_out), lay.rows(n_z, std=2.0)
    dZ, db = lay.ex.act_bwd(dOut, z, act=act, gated=gated, bias_grad=bias)
    dh, zh = lay.host_rows(dOut), lay.host_rows(z)
    want, want_b = O.act_bwd(dh, zh, lay.off, act, gated)
    g = zh[:, :n_out]
    near = 2.0 ** -18 * np.abs(dh) * (np.abs(g) + 1)
    if gated:
        near = np.concatenate([near * np.abs(zh[:, n_out:]), near], 1)
    if act == 0 and not gated:
        assert dZ is dOut
    else:
        assert_close(dZ, want, unit(dt) * np.abs(want) + near, "dZ")
    if bias:
        mag = np.stack([(np.abs(want) * (lay.n + 2) * U_F32 + near)[lay.off[e]:lay.off[e + 1]].sum(0) for e in range(E)])
        assert_close(db, want_b, mag, "db")
        _, db2 = lay.ex.act_bwd(dOut, z, act=act, gated=gated, bias_grad=True)
        assert torch.equal(db, db2)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("case", PRODUCTS, ids=[str(i) for i in range(len(PRODUCTS))])
def test_linear_bwd(bd, case, dt):
    T, E, k, n_in, n_out, _, gated, _, _, _, route, dropped = case
    n_z = n_out * (2 if gated else 1)
    lay = Layer(bd, T, E, k, dt, seed=n_in + n_z, route=list(route) if isinstance(route, tuple) else route,
                dropped=dropped)
    dZ, X, W = lay.rows(n_z), lay.rows(n_in), lay.normal(E, n_z, n_in, std=n_in ** -0.5)
    dX, dW = lay.ex.linear_bwd(dZ, X, W, dX=torch.full((T * k, n_in), float("nan"), dtype=dt, device="cuda"),
                               dW=torch.full((E, n_z, n_in), float("nan"), device="cuda"))
    zh, xh, wh = lay.host_rows(dZ), lay.host_rows(X), host(W)
    want_x, want_w = O.linear_bwd(zh, xh, wh, lay.off)
    mag_x, mag_w = O.linear_bwd(np.abs(zh), np.abs(xh), np.abs(wh), lay.off)
    assert_close(dX, want_x, unit(dt) * np.abs(want_x) + n_z * U_F32 * mag_x, "dX")
    rows = np.diff(lay.off)[:, None, None]
    assert_close(dW, want_w, rows * U_F32 * mag_w, "dW")
    # one at a time, and accumulated: the same products
    only_x, none = lay.ex.linear_bwd(dZ, X, W, need_dW=False)
    assert none is None and torch.equal(only_x, dX)
    base = lay.normal(E, n_z, n_in, dtype=torch.float32)
    acc = base.clone()
    none, acc2 = lay.ex.linear_bwd(dZ, X, W, need_dX=False, dW=acc, accumulate=True)
    assert none is None and acc2 is acc
    assert_close(acc, want_w + host(base), rows * U_F32 * mag_w + U_F32 * (np.abs(want_w) + np.abs(host(base))), "dW +=")
    empty = torch.from_numpy(np.diff(lay.off) == 0).cuda()
    assert torch.equal(acc[empty], base[empty]) and not dW[empty].any()


@pytest.mark.parametrize("act,gated", [(1, True), (2, True), (2, False), (1, False)])
def test_gradients_against_differences(bd, act, gated):
    """Central differences of <linear(X, W, b), G> along a random direction of all three at once, in fp32, against
    act_bwd and linear_bwd. Truncation: eps^2 / 6 times the third derivative, bounded with the activations'
    derivatives (at most 1.13, 1.0, 2.0) and z's exact change; rounding: the sums' own bound over eps."""
    T, E, k, n_in, n_out = 24, 4, 2, 32, 16
    lay = Layer(bd, T, E, k, torch.float32, seed=act + 10 * gated, dropped=0.1, max_width=64)
    n_z = n_out * (2 if gated else 1)
    X, W, b = lay.normal(T * k, n_in), lay.normal(E, n_z, n_in, std=n_in ** -0.5), lay.normal(E, n_z, std=0.3)
    vX, vW, vb = lay.normal(T * k, n_in, std=0.3), lay.normal(E, n_z, n_in, std=0.05), lay.normal(E, n_z, std=0.1)
    G = lay.normal(T * k, n_out)
    for t in (X, vX, G):
        t[lay.n:] = 0
    _, pre = lay.ex.linear(X, W, bias=b, act=act, gated=gated, save_pre=True)
    dZ, db = lay.ex.act_bwd(G, pre, act=act, gated=gated, bias_grad=True)
    dX, dW = lay.ex.linear_bwd(dZ, X, W)
    slope = float((host(dX) * host(vX)).sum() + (host(dW) * host(vW)).sum() + (host(db) * host(vb)).sum())
    eps = 2.0 ** -8
    L = lambda s: float((host(lay.ex.linear(X + s * vX, W + s * vW, bias=b + s * vb, act=act, gated=gated)[0])  # noqa: E731
                         * host(G)).sum())
    fd = (L(eps) - L(-eps)) / (2 * eps)
    # z(s) = z + s z1 + s^2 z2: magnitudes of z1 and z2 over |s| <= eps
    h = [host(t) for t in (X, W, b, vX, vW, vb)]
    _, zx = O.linear(np.abs(h[3]), np.abs(h[1]) + eps * np.abs(h[4]), lay.off)
    _, zw = O.linear(np.abs(h[0]) + eps * np.abs(h[3]), np.abs(h[4]), lay.off, np.abs(h[5]))
    _, z2 = O.linear(np.abs(h[3]), np.abs(h[4]), lay.off)
    _, z0 = O.linear(np.abs(h[0]), np.abs(h[1]), lay.off, np.abs(h[2]))
    z1, z2 = zx + zw, 2 * z2                            # first and second derivative of z
    a1, a2 = z1[:, :n_out], z2[:, :n_out]
    d1, d2, d3 = 1.13 * a1, a1 ** 2 + 1.13 * a2, 2.0 * a1 ** 3 + 3 * a1 * a2
    f, f0 = d3, z0[:, :n_out]
    if gated:
        u0, u1, u2 = z0[:, n_out:] + eps * z1[:, n_out:], z1[:, n_out:], z2[:, n_out:]
        f = d3 * u0 + 3 * d2 * u1 + 3 * d1 * u2
        f0 = f0 * u0
    Gh = np.abs(host(G))
    trunc = eps ** 2 / 6 * float((Gh * f).sum())
    rounding = 4 * (n_in + 8) * U_F32 * float((Gh * (f0 + 1)).sum()) / eps
    assert abs(fd - slope) <= trunc + rounding + 1e-5 * abs(slope)
    assert trunc + rounding < 0.25 * float((Gh * d1).sum())     # the bound says something


def test_other_experts_nonfinite_rows_and_weights_stay_theirs(bd):
    """An expert whose rows or weights hold infinities and NaN leaves the others' results as they are, also where its
    rows share a tile's memory with theirs."""
    for dt in (torch.bfloat16, torch.float32):
        lay = Layer(bd, 300, 4, 1, dt, seed=3, route=[37, 100, 83, 80])
        n_in, n_z = 136, 72
        X, dZ, W = lay.rows(n_in), lay.rows(n_z), lay.normal(4, n_z, n_in, std=0.1)
        a, b = 37, 137
        out, _ = lay.ex.linear(X, W)
        dX, dW = lay.ex.linear_bwd(dZ, X, W)
        X2, dZ2, W2 = X.clone(), dZ.clone(), W.clone()
        X2[a:b], dZ2[a:b], W2[1] = float("nan"), float("inf"), float("inf")
        out2, _ = lay.ex.linear(X2, W2)
        dX2, dW2 = lay.ex.linear_bwd(dZ2, X2, W2)
        rest = torch.ones(300, dtype=torch.bool, device="cuda")
        rest[a:b] = False
        assert torch.equal(out[rest], out2[rest]) and torch.equal(dX[rest], dX2[rest])
        assert torch.equal(dW[[0, 2, 3]], dW2[[0, 2, 3]])
        assert not torch.isfinite(out2[a:b]).any() and not torch.isfinite(dW2[1]).any()


def test_nonfinite_values_pass_as_in_the_formula(bd):
    ex = bd.Experts(4, 1, 1)
    X = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    X[0, 0], X[1, 0], X[2, 0] = float("inf"), float("nan"), -3e38
    W = torch.ones(1, 64, 64, dtype=torch.bfloat16, device="cuda")
    out, pre = ex.linear(X, W, act=bd.SMOES_ACT_GELU, save_pre=True)
    assert torch.isposinf(out[0]).all() and torch.isnan(out[1]).all()
    assert (out[2] == 0).all() and (out[3] == 0).all() and torch.isposinf(pre[0]).all()


def test_on_another_stream(bd):
    lay = Layer(bd, 600, 16, 4, torch.bfloat16, seed=9, max_width=256)
    X, W = lay.normal(600, 256), lay.normal(16, 256, 256, std=0.06)
    torch.cuda.synchronize()

    def steps():
        lay.ex.sort(idx)
        Xs = lay.ex.dispatch(X)
        h, pre = lay.ex.linear(Xs, W, act=1, gated=True, save_pre=True)
        dZ, db = lay.ex.act_bwd(h, pre, act=1, gated=True, bias_grad=True)
        return [Xs, h, pre, dZ, db, *lay.ex.linear_bwd(dZ, Xs, W)]

    idx = torch.from_numpy(lay.idx).cuda()
    want = steps()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = steps()
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_on_a_stream_given_by_argument(bd):
    """Outputs made by a call on another stream than the current one are not handed out again before it is done."""
    lay = Layer(bd, 4096, 16, 4, torch.bfloat16, seed=10, max_width=512)
    X, W = lay.normal(4096, 256), lay.normal(16, 512, 256, std=0.06)
    idx = torch.from_numpy(lay.idx).cuda()
    lay.ex.sort(idx)
    want, _ = lay.ex.linear(lay.ex.dispatch(X), W, act=1, gated=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(5):
        lay.ex.sort(idx, stream=side)
        Xs = lay.ex.dispatch(X, stream=side)
        got, _ = lay.ex.linear(Xs, W, act=1, gated=True, stream=side)
        del Xs                                          # its memory is the side stream's until linear has read it
        torch.full((16384, 256), 7.0, dtype=torch.bfloat16, device="cuda")
        side.synchronize()
        assert torch.equal(got, want)


def test_offsets_past_32_bits(bd):
    """More than 2^31 elements in the rows: the last rows are the right ones."""
    T, E, k, d = 131072, 128, 8, 2056
    g = torch.Generator(device="cuda").manual_seed(1)
    ex = bd.Experts(T, E, k)
    idx = torch.randn((T, E), generator=g, device="cuda").topk(k, dim=1).indices.to(torch.int32)
    off, row_slot, slot_row = ex.sort(idx)
    X = torch.randn((T, d), generator=g, device="cuda").to(torch.bfloat16)
    Xs = ex.dispatch(X)
    for lo in (0, T * k // 2, T * k - 4096):
        part = row_slot[lo:lo + 4096].long() // k
        assert torch.equal(Xs[lo:lo + 4096], X[part])
    W = (torch.randn((E, 16, d), generator=g, device="cuda") * d ** -0.5).to(torch.bfloat16)
    out, _ = ex.linear(Xs, W)
    want = Xs[-4096:].double() @ W[-1].double().T
    assert int(off[-2]) <= T * k - 4096
    assert ((out[-4096:].double() - want).abs() <= U_BF16 * want.abs() + 1e-3).all()
    dX, _ = ex.linear_bwd(out, Xs, W, need_dW=False)
    want = out[-4096:].double() @ W[-1].double()
    assert ((dX[-4096:].double() - want).abs() <= U_BF16 * want.abs() + 1e-3).all()
    w = torch.rand((T, k), generator=g, device="cuda")
    Y = ex.combine(Xs, w)
    want = X[-4096:].double() * w[-4096:].double().sum(1, keepdim=True)
    assert ((Y[-4096:].double() - want).abs() <= U_BF16 * want.abs() + 1e-5).all()


def test_offsets_and_maps_of_another_make_stay_inside(bd):
    """Offsets that run backwards or leave [0, R], rows out of range: every call keeps to its buffers (guard rows on both
    sides of every output stay as they were) and returns."""
    T, E, k, d = 300, 6, 2, 64
    R = T * k
    for dt, code in ((torch.bfloat16, bd.SMOES_BF16), (torch.float32, bd.SMOES_F32)):
        ex = bd.Experts(T, E, k, dtype=code, max_width=128)
        ex.expert_offsets.copy_(torch.tensor([40, -7, 2 ** 31 - 1, 3, 590, 100, 550], dtype=torch.int32))
        ex.slot_row.copy_(torch.randint(-2 ** 31, 2 ** 31 - 1, (T, k), dtype=torch.int64).to(torch.int32))
        ex.slot_row[:5] = torch.tensor([[0, R - 1], [R, -1], [R + 1, 7], [2 ** 31 - 1, -2 ** 31], [1, 2]], dtype=torch.int32)

        def guarded(rows, width, dtype=dt):
            whole = torch.full((rows + 64, width), 3.0, dtype=dtype, device="cuda")
            return whole, whole[32:32 + rows]

        x = lambda rows, width: torch.ones((rows, width), dtype=dt, device="cuda")  # noqa: E731
        W = torch.ones((E, 128, d), dtype=dt, device="cuda")
        w = torch.ones((T, k), device="cuda")
        outs = [guarded(R, d), guarded(T, d), guarded(T, d), guarded(R, d), guarded(T, k * 2, torch.float32), guarded(R, 64),
                guarded(R, 128), guarded(R, 128), guarded(E, 128, torch.float32), guarded(R, d), guarded(E * 128, d, torch.float32)]
        o = [v for _, v in outs]
        ex.dispatch(x(T, d), out=o[0])
        ex.combine(x(R, d), w, out=o[1])
        ex.dispatch_bwd(x(R, d), out=o[2])
        dw = torch.empty((T, k), device="cuda")
        ex.combine_bwd(x(T, d), x(R, d), w, dYs=o[3], d_topk_w=dw)
        ex.linear(x(R, d), W, act=1, gated=True, out=o[5], pre=o[6])
        ex.act_bwd(x(R, 64), x(R, 128), act=1, gated=True, dZ=o[7], db=o[8])
        ex.linear_bwd(x(R, 128), x(R, d), W, dX=o[9], dW=o[10].view(E, 128, d))
        torch.cuda.synchronize()
        for whole, _ in outs:
            assert (whole[:32] == 3).all() and (whole[-32:] == 3).all()
        assert torch.isfinite(dw).all() and ex.device_status() == bd.SMOES_OK


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_both_gradients_at_once_are_complete_when_the_call_is(bd, dt):
    """The two products of linear_bwd overlap on the GPU. What ran before is done when they write, and both are done when the
    next kernel reads: one expert holds nearly all rows, so that dW takes far longer than dX; the outputs are poisoned right
    before and read right after."""
    lay = Layer(bd, 6000, 4, 1, dt, seed=12, route=[20, 5900, 0, 80])
    dZ, X, W = lay.rows(128), lay.rows(64), lay.normal(4, 128, 64, std=0.1)
    dX, dW = lay.ex.linear_bwd(dZ, X, W)
    alone_x, _ = lay.ex.linear_bwd(dZ, X, W, need_dW=False)
    _, alone_w = lay.ex.linear_bwd(dZ, X, W, need_dX=False)
    torch.cuda.synchronize()
    assert torch.equal(dX, alone_x) and torch.equal(dW, alone_w)
    for _ in range(40):
        dX.fill_(float("nan"))
        dW.fill_(float("nan"))
        lay.ex.linear_bwd(dZ, X, W, dX=dX, dW=dW)
        got_w, got_x = dW.clone(), dX.clone()
        assert torch.equal(got_w, alone_w) and torch.equal(got_x, alone_x)
    # the activation's gradient and the sort before it, the layer below behind it, without a wait between
    lay = Layer(bd, 3000, 16, 2, dt, seed=13, max_width=256)
    X, W, idx = lay.normal(3000, 128), lay.normal(16, 256, 128, std=0.1), torch.from_numpy(lay.idx).cuda()

    def steps():
        lay.ex.sort(idx)
        Xs = lay.ex.dispatch(X)
        h, pre = lay.ex.linear(Xs, W, act=1, gated=True, save_pre=True)
        dZ, db = lay.ex.act_bwd(h, pre, act=1, gated=True, bias_grad=True)
        dX, dW = lay.ex.linear_bwd(dZ, Xs, W)
        return lay.ex.dispatch_bwd(dX), dW, db

    want = [t.clone() for t in steps()]
    for _ in range(30):
        for a, b in zip(steps(), want):
            assert torch.equal(a, b)


def test_whole_numbers_come_out_exactly_call_after_call(bd):
    """fp32 products of many short tiles: 72 experts with none to a few rows, a few hundred blocks of the ring each call. Whole
    numbers up to 8 and sums below 2^17, so that every order of the sums gives the same bits; a block split too early or used
    twice shows."""
    for T, E, k, n_in, n_z, seed in ((4, 72, 4, 1024, 2048, 31), (45, 72, 4, 264, 520, 32), (1, 72, 1, 32, 8, 33)):
        lay = Layer(bd, T, E, k, torch.float32, seed=seed, dropped=0.1)
        whole = lambda *shape: torch.randint(-8, 9, shape, generator=lay.g, device="cuda").float()
        X, W, dZ = whole(lay.ex.R, n_in), whole(E, n_z, n_in), whole(lay.ex.R, n_z)
        want = torch.zeros(lay.ex.R, n_z, device="cuda", dtype=torch.float64)
        want_x = torch.zeros(lay.ex.R, n_in, device="cuda", dtype=torch.float64)
        want_w = torch.zeros(E, n_z, n_in, device="cuda", dtype=torch.float64)
        for e in range(E):
            a, b = int(lay.off[e]), int(lay.off[e + 1])
            want[a:b] = X[a:b].double() @ W[e].double().T
            want_x[a:b] = dZ[a:b].double() @ W[e].double()
            want_w[e] = dZ[a:b].double().T @ X[a:b].double()
        for _ in range(20):
            out, _ = lay.ex.linear(X, W)
            dX, dW = lay.ex.linear_bwd(dZ, X, W)
            assert torch.equal(out.double(), want) and torch.equal(dX.double(), want_x)
            assert torch.equal(dW.double(), want_w)


def test_captured_in_a_graph(bd):
    """A layer's calls replayed as a CUDA graph on new tokens and selections give what the calls give."""
    lay = Layer(bd, 700, 16, 4, torch.bfloat16, seed=11, max_width=256)
    X, W = lay.normal(700, 256), lay.normal(16, 256, 256, std=0.06)
    idx = torch.from_numpy(lay.idx).cuda()

    def steps():
        lay.ex.sort(idx)
        Xs = lay.ex.dispatch(X)
        h, pre = lay.ex.linear(Xs, W, act=2, gated=True, save_pre=True)
        dZ, db = lay.ex.act_bwd(h, pre, act=2, gated=True, bias_grad=True)
        dX, dW = lay.ex.linear_bwd(dZ, Xs, W)
        return [lay.ex.dispatch_bwd(dX, residual=X), db, dW]

    steps()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = steps()
    X.copy_(lay.normal(700, 256))
    idx.copy_((idx + 3) % 16)
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in got]
    for a, b in zip(got, steps()):
        assert torch.equal(a, b)


def test_no_tokens(bd):
    ex = bd.Experts(0, 8, 2, max_width=64)
    off, _, _ = ex.sort(torch.empty((0, 2), dtype=torch.int32, device="cuda"))
    assert off.tolist() == [0] * 9
    X = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    W = torch.ones((8, 32, 64), dtype=torch.bfloat16, device="cuda")
    assert ex.dispatch(X).shape == (0, 64)
    assert ex.linear(X, W)[0].shape == (0, 32)
    dZ, db = ex.act_bwd(X[:, :32].contiguous(), X[:, :32].contiguous(), act=1, bias_grad=True)
    assert not db.any()
    dX, dW = ex.linear_bwd(dZ, X, W)
    assert dX.shape == (0, 64) and not dW.any()
    assert ex.combine(X, torch.empty((0, 2), device="cuda")).shape == (0, 64)


def test_refused_arguments(bd):
    ex = bd.Experts(10, 4, 2)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    W = bf(4, 32, 64)
    for call in (lambda: ex.sort(torch.zeros((10, 2), dtype=torch.int64, device="cuda")),
                 lambda: ex.sort(torch.zeros((9, 2), dtype=torch.int32, device="cuda")),
                 lambda: ex.sort(torch.zeros((10, 2), dtype=torch.int32)),
                 lambda: ex.dispatch(bf(11, 64)),
                 lambda: ex.dispatch(bf(10, 64).float()),
                 lambda: ex.dispatch(bf(64, 10).t()),
                 lambda: ex.dispatch(bf(10, 64), out=bf(10, 64)),
                 lambda: ex.combine(bf(20, 64), torch.zeros(10, 2, dtype=torch.bfloat16, device="cuda")),
                 lambda: ex.combine(bf(20, 64), torch.zeros(10, 2, device="cuda"), residual=bf(20, 64)),
                 lambda: ex.linear(bf(20, 32), W),
                 lambda: ex.linear(bf(20, 64), W, bias=bf(4, 32)),
                 lambda: ex.linear(bf(20, 64), bf(4, 33, 64), gated=True),
                 lambda: ex.linear(bf(20, 64), bf(3, 32, 64)),
                 lambda: ex.act_bwd(bf(20, 32), act=1),
                 lambda: ex.act_bwd(bf(20, 32), bf(20, 32), act=1, gated=True),
                 lambda: ex.linear_bwd(bf(20, 32), bf(20, 64), W, accumulate=True),
                 lambda: ex.linear_bwd(bf(20, 32), bf(20, 64), W, dW=bf(4, 32, 64))):
        with pytest.raises(ValueError):
            call()
    for call, code in ((lambda: ex.dispatch(bf(10, 60)), -1),                      # rows of whole 16-byte words
                       (lambda: ex.linear(bf(20, 64), bf(4, 36, 64)), -1),
                       (lambda: ex.linear(bf(20, 64), W, act=3), -1),
                       (lambda: ex.act_bwd(bf(20, 32), bf(20, 32), act=1, bias_grad=True), -4),   # no max_width
                       (lambda: ex.linear_bwd(bf(20, 32), bf(20, 64), W, need_dX=False, need_dW=False), -1)):
        with pytest.raises(bd.SmoesError) as err:
            call()
        assert err.value.code == code
    moved = torch.zeros(10 * 64 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(10, 64)   # 8 bytes off
    with pytest.raises(bd.SmoesError) as err:
        ex.dispatch(moved)
    assert err.value.code == -3
    assert ex.device_status() == bd.SMOES_OK
