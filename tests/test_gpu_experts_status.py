"""Bounded waits of the expert layer: one that runs out is reported through the status word and the kernel returns; the context
stays usable, and the workspace works again once it has been cleared.

With a limit of 1 ns a block that reaches the sort's grid barrier before the last one gives up at its first poll (the blocks of
2^20 tokens reach it microseconds apart); the last one resets the barrier on its way through. The products' waits are over within
their first polls, which the hardware holds for longer than 1 ns each, whatever the limit.
"""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as O
from tests.test_gpu_experts import bd  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def test_sort_timeout_is_reported_and_recoverable(bd):  # noqa: F811
    T, E, k = 1 << 20, 16, 8
    idx = np.argsort(np.random.default_rng(5).random((T, E)), axis=1)[:, :k].astype(np.int32)
    top = torch.from_numpy(idx).cuda()
    ex = bd.Experts(T, E, k)
    assert bd.smoes_experts_set_wait_limit(ex.plan, 1) == 0
    ex.sort(top)
    assert ex.device_status() == -6                     # SMOES_ERR_DEVICE_TIMEOUT
    assert bd.smoes_experts_set_wait_limit(ex.plan, 0) == 0
    assert bd.smoes_experts_workspace_init(ex.plan, ex.ws) == 0
    assert ex.device_status() == bd.SMOES_OK
    for got, want in zip(ex.sort(top), O.sort(idx, E)):
        assert np.array_equal(got.cpu().numpy(), want)
    assert ex.device_status() == bd.SMOES_OK
    assert bd.smoes_experts_set_wait_limit(None, 5) == -1
