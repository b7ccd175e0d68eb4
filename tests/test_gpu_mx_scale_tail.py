"""4-bit products of rows whose scales end inside a word: the bits are those of the same rows in a longer array."""
import pytest
import torch

from tests.test_gpu_mx import BF16, bd  # noqa: F401  (bd: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R", [1, 2, 3, 5, 33, 67, 131, 201])
@pytest.mark.parametrize("n_in", [32, 96, 544, 1440, 2016])
def test_the_last_rows(bd, R, n_in):  # noqa: F811
    g = torch.Generator().manual_seed(R + n_in)
    X = bd.mx_quantise(torch.randn(R + 3, n_in, generator=g).to(BF16).cuda())
    W = bd.mx_quantise(torch.randn(1, 72, n_in, generator=g).to(BF16).cuda())
    rows = bd.Mx(X.codes[:R].contiguous(), X.scales[:R].contiguous())
    behind = bd.Mx(X.codes[:R], X.scales[:R])           # the same, other rows' scales behind them
    want = bd.Experts(R + 3, 1, 1).linear_mx(X, W)[:R]
    ex = bd.Experts(R, 1, 1)
    assert torch.equal(ex.linear_mx(rows, W), want) and torch.equal(ex.linear_mx(behind, W), want)
    assert ex.device_status() == bd.SMOES_OK and bool(want.isfinite().all()) and bool(want.any())
