"""Host-side checks of the 4-bit calls (no GPU needed)."""
import ctypes as C

import numpy as np
import pytest

from oracle import layer_oracle as O


@pytest.fixture(scope="module")
def bd():
    from paper_2604_23996_gb300.build import build_library
    build_library()
    from paper_2604_23996_gb300 import binding
    return binding


A, ODD = 1 << 12, (1 << 12) + 8                         # addresses that are never read


@pytest.mark.parametrize("args,code", [((A, 1, -1, 64, A, A), -1), ((A, 1, 4, 0, A, A), -1), ((A, 1, 4, 40, A, A), -1), ((A, 2, 4, 64, A, A), -1),
                                       ((A, 1, (1 << 31) + 1, 64, A, A), -2), ((A, 1, 4, (1 << 20) + 32, A, A), -2), ((None, 1, 4, 64, A, A), -1),
                                       ((A, 1, 4, 64, None, A), -1), ((A, 1, 4, 64, A, None), -1), ((ODD, 1, 4, 64, A, A), -3),
                                       ((A, 1, 4, 64, ODD, A), -3), ((A, 1, 4, 64, A, ODD), -3), ((None, 1, 0, 64, None, None), 0)])
def test_quantise(bd, args, code):
    X, dtype, rows, n, q, s = args
    assert bd._lib.smoes_mx_quantise(X, dtype, rows, n, q, s, None) == code
    assert bd._lib.smoes_mx_dequantise(q, s, rows, n, dtype, X, None) == code


def test_tensors_of_the_host_and_of_another_device_are_refused(bd, monkeypatch):
    import torch
    X = torch.zeros(4, 64)
    x = bd.Mx(torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8))
    for current in (-1, 0):
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current, raising=False)
        with pytest.raises(ValueError, match="device"):
            bd.mx_quantise(X)
        with pytest.raises(ValueError, match="device"):
            bd.mx_dequantise(x)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 1)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    with pytest.raises(ValueError, match="device"):
        bd.mx_quantise(X)

    class Stream:
        device_index, cuda_stream = 0, 5

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    with pytest.raises(ValueError, match="device"):
        bd.mx_dequantise(x, stream=Stream())


def test_expert_calls(bd):
    code, plan = bd.smoes_experts_create(8, 2, 1, bd.SMOES_BF16)
    need = bd.smoes_experts_workspace_bytes(plan)
    assert code == 0
    d = lambda *a: bd._lib.smoes_expert_dispatch_mx(*a, None)  # noqa: E731
    assert d(None, A, 64, A, A, A, A) == -1 and d(plan, A, 40, A, A, A, A) == -1 and d(plan, None, 64, A, A, A, A) == -1
    assert d(plan, A, 64, A, A, ODD, A) == -3 and d(plan, A, 64, A, A, A, ODD) == -3

    def linear(plan=plan, ws=A, ws_bytes=need, out=A, off=A, **kw):
        a = dict(X=A, X_scales=A, W=A, W_scales=A, bias=None, residual=None, n_in=64, n_out=16, act=0, gated=0) | kw
        return bd._lib.smoes_expert_linear_mx(plan, C.byref(bd.LinearMxArgs(**a)), off, out, ws, ws_bytes, None)

    assert linear(plan=None) == -1 and linear(act=3) == -1 and linear(gated=2) == -1 and linear(n_in=40) == -1 and linear(n_out=12) == -1
    assert linear(ws=None) == -4 and linear(ws_bytes=need - 1) == -4 and linear(ws=ODD) == -3
    for name in ("X", "X_scales", "W", "W_scales"):
        assert linear(**{name: None}) == -1 and linear(**{name: ODD}) == -3
    assert linear(out=None) == -1 and linear(off=None) == -1 and linear(bias=ODD) == -3 and linear(residual=ODD) == -3
    assert linear(n_out=1 << 20, gated=1) == -2
    bd.smoes_experts_destroy(plan)
    code, plan = bd.smoes_experts_create(8, 2, 1, bd.SMOES_F32)
    assert linear(plan=plan) == -2
    bd.smoes_experts_destroy(plan)


def test_the_oracle_rounds_as_the_format_says():
    x = np.zeros((1, 32))
    x[0, :12] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7.9, -0.25, -0.7500001, 0.2500001]
    q, s = O.mx_quantise(x)
    assert s[0, 0] == 127
    assert list(O.mx_values(q, s)[0, :12]) == [0, 1, 1, 2, 2, 4, 4, 6, 6, 0, -1, 0.5]
    q, s = O.mx_quantise(np.full((1, 32), 2.0 ** -149))
    assert s[0, 0] == 0 and not O.mx_values(q, s).any()


@pytest.mark.parametrize("n", [32, 64, 96, 128, 160, 192, 208])
def test_division_by_a_tiles_rows_is_exact(n):
    """The product's tiles are counted with the upper half of a product by ceil(2^32 / n)."""
    x = np.arange((1 << 24) + n, dtype=np.uint64)
    assert (((x * np.uint64(-(-(1 << 32) // n))) >> np.uint64(32)) == x // np.uint64(n)).all()
