"""The expert products where a pair of CTAs works through several full tiles, and their accuracy at real depths.

Element-wise tolerances are those of the layer's other tests. The relative norms, fixed before any run: the tensor cores cut each
addition of 16 products off, half a step of 2^-23 in the mean, all to one side.
* fp32 products: sums move after 256 of the depth, 16 additions, 16 * 2^-24 = 9.5e-7 of what they sum to: 1e-6. Without the third
  part of the values each product is off by 2^-18 / sqrt 3 for either factor, 3.1e-6.
* the weights' gradient in bf16: sums move after 512 rows, 32 additions, 1.9e-6: 2e-6. Left in the tensor cores for 8192 rows a sum
  is off by 9e-6."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as O
from tests.test_gpu_experts import U_F32, Layer, assert_close, bd, host, unit, z_bound  # noqa: F401  (bd: the fixture)

pytestmark = pytest.mark.gpu

DTYPES = pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])

# T, E, k, n_in, n_out, act, gated: at 76 pairs of CTAs three to six row tiles of 256 (fp32: 128) for each
MANY = [(20011, 8, 1, 256, 264, 1, True), (20011, 8, 1, 264, 256, 2, False), (6007, 8, 4, 136, 520, 2, True)]


@DTYPES
@pytest.mark.parametrize("T,E,k,n_in,n_out,act,gated", MANY)
def test_several_full_tiles_a_pair(bd, T, E, k, n_in, n_out, act, gated, dt):  # noqa: F811
    lay = Layer(bd, T, E, k, dt, seed=n_in + n_out, dropped=0.05)
    n_z = n_out * (2 if gated else 1)
    X, W = lay.rows(n_in), lay.normal(E, n_z, n_in, std=n_in ** -0.5)
    b, res = lay.normal(E, n_z, std=0.3, dtype=torch.float32), lay.rows(n_out)
    out, z = lay.ex.linear(X, W, bias=b, act=act, gated=gated, residual=res, save_pre=True)
    Xh, Wh, bh, rh = lay.host_rows(X), host(W), host(b), lay.host_rows(res)
    want, want_z = O.linear(Xh, Wh, lay.off, bh, act, gated, rh)
    tol_z = z_bound(Xh, Wh, lay.off, bh)
    assert_close(z, want_z, unit(dt) * np.abs(want_z) + tol_z, "pre")
    g = want_z[:, :n_out]
    tol = 1.13 * tol_z[:, :n_out] + 2.0 ** -18 * (np.abs(g) + 1)
    if gated:
        u, tol_u = want_z[:, n_out:], tol_z[:, n_out:]
        tol = tol * (np.abs(u) + tol_u) + np.abs(O.act(act, g)) * tol_u
    tol = tol + unit(dt) * np.abs(want) + 4 * U_F32 * np.abs(rh)
    tol[lay.n:] = 0.0
    assert_close(out, want, tol, "out")
    dZ = lay.rows(n_z)
    dX, dW = lay.ex.linear_bwd(dZ, X, W)
    zh = lay.host_rows(dZ)
    want_x, want_w = O.linear_bwd(zh, Xh, Wh, lay.off)
    mag_x, mag_w = O.linear_bwd(np.abs(zh), np.abs(Xh), np.abs(Wh), lay.off)
    assert_close(dX, want_x, unit(dt) * np.abs(want_x) + n_z * U_F32 * mag_x, "dX")
    assert_close(dW, want_w, np.diff(lay.off)[:, None, None] * U_F32 * mag_w, "dW")
    assert lay.ex.device_status() == bd.SMOES_OK


def rel(got, want):
    return float((got.double() - want).norm() / want.norm())


def test_fp32_products_at_a_depth_of_2048(bd):  # noqa: F811
    rows = [1500, 548]
    lay = Layer(bd, 2048, 2, 1, torch.float32, seed=21, route=rows)
    X, W, dZ = lay.normal(2048, 2048), lay.normal(2, 512, 2048), lay.normal(2048, 512)
    W2, dZ2 = lay.normal(2, 2048, 512), lay.normal(2048, 2048)
    a = rows[0]
    both = lambda f: torch.cat([f(slice(0, a), 0), f(slice(a, None), 1)])  # noqa: E731
    out, _ = lay.ex.linear(X, W)
    assert rel(out, both(lambda r, e: X[r].double() @ W[e].double().T)) <= 1e-6
    dX, _ = lay.ex.linear_bwd(dZ2, dZ, W2, need_dW=False)
    assert rel(dX, both(lambda r, e: dZ2[r].double() @ W2[e].double())) <= 1e-6
    _, dW = lay.ex.linear_bwd(dZ, X, W, need_dX=False)
    assert rel(dW, torch.stack([dZ[:a].double().T @ X[:a].double(), dZ[a:].double().T @ X[a:].double()])) <= 1e-6


def test_weights_gradient_over_8192_rows(bd):  # noqa: F811
    """Rows of one sign, so that every addition cuts the same way."""
    T = 8201
    ex = bd.Experts(T, 1, 1)
    g = torch.Generator(device="cuda").manual_seed(22)
    X, dZ = (torch.rand((T, 256), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    W = torch.zeros((1, 256, 256), dtype=torch.bfloat16, device="cuda")
    _, dW = ex.linear_bwd(dZ, X, W, need_dX=False)
    assert rel(dW[0], dZ.double().T @ X.double()) <= 2e-6
