"""Arrays of more than 2^31 elements: the last rows of a long call have the bits that a call of their own gives them."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def bd():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("40 GB of device memory are wanted")
    from paper_2604_23996_gb300 import binding
    return binding


def test_layer_norm(bd):
    T, d, n = (1 << 17) + 3, 16384, 5                   # 2^31 elements in all but the last three rows
    g = torch.Generator(device="cuda").manual_seed(0)
    X = torch.zeros(T, d, dtype=BF16, device="cuda")
    X[-n:] = torch.randn(n, d, generator=g, device="cuda").to(BF16)
    w, b = torch.randn(d, generator=g, device="cuda"), torch.randn(d, generator=g, device="cuda")
    long, short = bd.LayerNorm(T, d), bd.LayerNorm(n, d)
    Y, _, mean, rstd = long.forward(X, w, b)
    y, _, m, r = short.forward(X[-n:], w, b)
    assert torch.equal(Y[-n:], y) and torch.equal(mean[-n:], m) and torch.equal(rstd[-n:], r)
    assert torch.equal(Y[7], b.to(BF16))                # a row of zeros
    dX, _, _ = long.backward(Y, X, mean, rstd, w, need_dw=False, need_db=False, dX=torch.empty_like(X))
    assert torch.equal(dX[-n:], short.backward(y, X[-n:], m, r, w)[0])


def test_quantise_and_back(bd):
    rows, n = (1 << 16) + 2, 32768
    X = torch.zeros(rows, n, dtype=BF16, device="cuda")
    X[-3:] = torch.randn(3, n, device="cuda").to(BF16)
    q = bd.mx_quantise(X)
    last = bd.mx_quantise(X[-3:])
    assert torch.equal(q.codes[-3:], last.codes) and torch.equal(q.scales[-3:], last.scales) and not q.codes[:-3].any()
    assert torch.equal(bd.mx_dequantise(q, out=X)[-3:], bd.mx_dequantise(last))


def test_products(bd):
    R, n_in, n_out, n = (1 << 17) + 40, 64, 16384, 40
    X, W = bd.mx_quantise(torch.randn(R, n_in, device="cuda")), bd.mx_quantise(torch.randn(1, n_out, n_in, device="cuda"))
    res = torch.randn(n, n_out, device="cuda").to(BF16)
    residual = torch.zeros(R, n_out, dtype=BF16, device="cuda")
    residual[-n:] = res
    out = bd.Experts(R, 1, 1).linear_mx(X, W, residual=residual)
    want = bd.Experts(n, 1, 1).linear_mx(bd.Mx(X.codes[-n:], X.scales[-n:]), W, residual=res)
    assert torch.equal(out[-n:], want)
    first = bd.Experts(n, 1, 1).linear_mx(bd.Mx(X.codes[:n], X.scales[:n]), W)
    assert torch.equal(out[:n], first)
