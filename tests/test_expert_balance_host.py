"""Host-side checks of the expert-level balance calls (no GPU needed)."""
import numpy as np
import pytest


@pytest.fixture(scope="module")
def plan():
    from paper_2604_23996_gb300.build import build_library
    build_library()
    from paper_2604_23996_gb300 import binding as bd
    code, p = bd.smoes_plan_create(100, 64, 16, 2, 4, [0, 40, 100], np.arange(16) // 4, bd.SMOES_BF16)
    assert code == 0
    yield bd, p, bd.smoes_workspace_bytes(p)
    bd.smoes_plan_destroy(p)


def test_balance_arguments(plan):
    bd, p, need = plan
    a, odd = 1 << 12, (1 << 12) + 4                     # addresses that are never read
    call = lambda *v: bd._lib.smoes_expert_balance(*v, None)  # noqa: E731
    assert call(None, a, 1, 1.0, a, a, a, a, need) == -1
    assert call(p, a, 1, 1.0, None, a, a, a, need) == -1
    assert call(p, a, 2, 1.0, a, a, a, a, need) == -1
    assert call(p, None, 1, 1.0, a, a, a, a, need) == -1
    assert call(p, a, 1, 1.0, a, a, a, None, need) == -4
    assert call(p, a, 1, 1.0, a, a, a, a, need - 1) == -4
    assert call(p, odd, 1, 1.0, a, a, a, a, need) == -3
    assert call(p, a, 1, 1.0, a, odd, a, a, need) == -3
    assert call(p, a, 1, 1.0, a, a, odd, a, need) == -3
    assert call(p, a, 1, 1.0, a, a, a, odd, need) == -3


def test_backward_arguments(plan):
    bd, p, need = plan
    a, odd = 1 << 12, (1 << 12) + 4
    call = lambda idx, d_gate: bd._lib.smoes_router_bwd_gates(p, a, a, a, idx, None, d_gate, 1, 1.0, a, 0, None, None, a, need, None)  # noqa: E731
    assert call(None, a) == -1
    assert call(a, odd) == -3


@pytest.mark.parametrize("T,lengths", [(1, [1]), (100, [1] * 100), (70000, [3, 69997]), (70000, [35000, 35000]), (4865, [33, 32, 4800])])
def test_partials_of_different_runs_lie_apart(T, lengths):
    """Runs of `len` tokens of samples that have several: 2 (begin / len) + (last of its sample) is a place of its own."""
    for sms in (148, 152):
        length = max(32, -(-T // sms))
        taken, begin = set(), 0
        for n in lengths:
            runs = -(-n // length)
            for r in range(runs if runs > 1 else 0):
                at = 2 * ((begin + r * length) // length) + (r == runs - 1)
                assert at not in taken and at < 2 * (T // length + 1)
                taken.add(at)
            begin += n
