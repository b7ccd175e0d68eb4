"""Selections given to a router's backward are checked, with a gradient of the gate values and without one (no GPU needed: nothing
gets as far as the library)."""
import pytest
import torch

from tests.test_mx_host import bd  # noqa: F401  (the fixture: builds the library)


@pytest.fixture
def router(bd, monkeypatch):  # noqa: F811
    def reached(*_):
        raise AssertionError("the library was called")

    monkeypatch.setattr(bd, "smoes_router_bwd", reached)
    monkeypatch.setattr(bd, "smoes_router_bwd_gates", reached)
    r = object.__new__(bd.Router)
    r.plan, r.T, r.E, r.k, r.B = None, 6, 4, 2, 2
    r.ws, r.topk_idx = torch.zeros(16, dtype=torch.uint8), torch.zeros(6, 2, dtype=torch.int32)
    return r


BAD = [torch.zeros(6, 2, dtype=torch.int64), torch.zeros(5, 2, dtype=torch.int32), torch.zeros(2, 6, dtype=torch.int32).t(),
       torch.zeros(6, 2)]


@pytest.mark.parametrize("gates", [False, True])
@pytest.mark.parametrize("bad", BAD, ids=["int64", "short", "strided", "float"])
def test_selections_of_another_make(router, bad, gates):
    with pytest.raises(ValueError, match="topk_idx"):
        router.backward(None, None, None, None, topk_idx=bad, d_gate=torch.zeros(2, 4) if gates else None)


@pytest.mark.parametrize("topk_idx", [None, torch.zeros(6, 2, dtype=torch.int32)], ids=["the forward's", "given"])
def test_good_ones_reach_the_library(router, topk_idx):
    for d_gate in (None, torch.zeros(2, 4), torch.zeros(1, 4)):
        with pytest.raises(AssertionError, match="the library"):
            router.backward(None, None, None, None, topk_idx=topk_idx, d_gate=d_gate)
