"""Host-side checks of the layer norm's calls (no GPU needed)."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def bd():
    from paper_2604_23996_gb300.build import build_library
    build_library()
    from paper_2604_23996_gb300 import binding
    return binding


def create(bd, T=100, d=64, dtype=1, eps=1e-5):
    plan = C.c_void_p()
    return bd._lib.smoes_norm_create(bd.NormDesc(T, d, dtype, eps), plan), plan


@pytest.mark.parametrize("kw,code", [(dict(), 0), (dict(T=0), 0), (dict(d=8), 0), (dict(d=16384), 0), (dict(d=8192, dtype=0), 0),
                                     (dict(T=1 << 20), 0), (dict(eps=0.0), 0), (dict(T=-1), -1), (dict(d=0), -1), (dict(d=12), -1),
                                     (dict(dtype=2), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1),
                                     (dict(eps=float("inf")), -1), (dict(d=16392), -2), (dict(d=8200, dtype=0), -2),
                                     (dict(T=(1 << 20) + 1), -2)])
def test_create(bd, kw, code):
    got, plan = create(bd, **kw)
    assert got == code
    assert (bd._lib.smoes_norm_workspace_bytes(plan) > 0) == (code == 0)
    bd._lib.smoes_norm_destroy(plan)


def test_arguments_are_refused_before_anything_is_launched(bd):
    _, plan = create(bd)
    a, odd = 256, 264                                   # addresses that are never read
    fwd = lambda *p: bd._lib.smoes_norm_fwd(plan, *p, None)  # noqa: E731
    assert fwd(None, None, a, a, None, a, a, a) == -1   # no X
    assert fwd(a, None, None, a, None, a, a, a) == -1   # no weight
    assert fwd(a, a, a, a, None, a, a, a) == -1         # a residual without a place for the sum
    assert fwd(a, None, a, a, a, a, a, a) == -1         # and the other way round
    assert fwd(a, None, a, a, None, a, a, None) == -1   # one of the statistics
    assert fwd(odd, None, a, a, None, a, a, a) == -3
    assert fwd(a, None, a, odd, None, a, a, a) == -3
    need = bd._lib.smoes_norm_workspace_bytes(plan)
    bwd = lambda *p: bd._lib.smoes_norm_bwd(plan, *p, None)  # noqa: E731
    assert bwd(None, a, a, a, a, None, a, a, a, 0, a, need) == -1
    assert bwd(a, a, a, a, a, None, None, a, a, 0, a, need) == -1
    assert bwd(a, a, a, a, a, None, a, a, a, 0, None, need) == -4
    assert bwd(a, a, a, a, a, None, a, a, a, 0, a, need - 1) == -4
    assert bwd(a, a, a, a, a, odd, a, a, a, 0, a, need) == -3
    assert bwd(a, a, a, a, a, None, a, a, odd, 0, a, need) == -3
    bd._lib.smoes_norm_destroy(plan)
    assert bd._lib.smoes_norm_fwd(None, a, None, a, a, None, a, a, a, None) == -1
