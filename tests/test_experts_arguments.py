"""Arguments that an expert layer would not use as they are given are refused (on the host, with the library faked)."""
import pytest
import torch

from tests.test_experts_device import bd, layer  # noqa: F401  (fixtures)


def test_a_gradient_that_would_stay_unwritten_is_refused(bd, layer, monkeypatch):  # noqa: F811
    """Without an activation and not gated the activation's gradient is its input: a tensor given for it stays as it was."""
    ex, lib = layer
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    dOut = torch.zeros(4, 16, dtype=torch.bfloat16)
    for kw in (dict(), dict(bias_grad=True), dict(db=torch.zeros(2, 16))):
        with pytest.raises(ValueError, match="dZ"):
            ex.act_bwd(dOut, dZ=torch.empty_like(dOut), **kw)
    assert not lib.calls
    dZ, db = ex.act_bwd(dOut, bias_grad=True)
    assert dZ is dOut and db.shape == (2, 16) and len(lib.calls) == 1
    assert ex.act_bwd(dOut, dOut, act=1, dZ=(given := torch.empty_like(dOut)))[0] is given
