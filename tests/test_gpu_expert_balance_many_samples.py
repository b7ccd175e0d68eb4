"""The expert-level balance loss of more than 32 samples of which some have several runs of tokens: partials of their runs, tickets
of their own, sums by the last of their own blocks. Oracle and tolerances of the call's other tests."""
import pytest
import torch

from tests import test_gpu_expert_balance as B
from tests.test_gpu_expert_balance import BF16, F32, Case, bd  # noqa: F401  (bd: the fixture)

pytestmark = pytest.mark.gpu

SHORT = [1, 33, 200, 7] * 12                            # runs of 32 tokens: 1, 2, 7 and 1 of them; blocks of 256 threads
LONG = [500, 1, 133, 1366] * 10                         # runs of 132 or 136 tokens: 4, 1, 1 or 2, 11; blocks of 1024 threads
CASES = {
    # T, d, E, k, n_bins, lengths, type, gate, dropped
    "short_e16": (sum(SHORT), 64, 16, 2, 4, SHORT, BF16, "softmax", 0.0),
    "short_e64_dropped": (sum(SHORT), 64, 64, 6, 8, SHORT, BF16, "softmax", 0.2),
    "short_e128": (sum(SHORT), 64, 128, 8, 16, SHORT, BF16, "softmax", 0.0),
    "short_fp32_e40_sigmoid": (sum(SHORT), 64, 40, 4, 5, SHORT, F32, "sigmoid", 0.1),
    "long_e16_dropped": (sum(LONG), 64, 16, 2, 4, LONG, BF16, "softmax", 0.1),
    "long_e64": (sum(LONG), 64, 64, 6, 8, LONG, BF16, "softmax", 0.0),
    "long_e128_dropped": (sum(LONG), 64, 128, 8, 16, LONG, BF16, "softmax", 0.1),
    "33_samples": (33 * 200, 64, 32, 4, 4, [200] * 33, BF16, "softmax", 0.0),
    "one_long_among_many": (6000 + 49, 64, 64, 6, 8, [1] * 20 + [6000] + [1] * 29, BF16, "softmax", 0.0),
}


@pytest.mark.parametrize("name", list(CASES))
def test_samples_of_several_runs(bd, name, monkeypatch):  # noqa: F811
    monkeypatch.setitem(B.CASES, name, CASES[name])
    c = Case(bd, name)
    out, _ = c.check(True)
    for per_sample in (True, False, True):              # the tickets are back, whichever call comes next
        again, _ = c.check(per_sample)
        if per_sample:
            assert all(torch.equal(a, b) for a, b in zip(out, again))
    assert c.r.device_status()[0] == bd.SMOES_OK


@pytest.mark.parametrize("sample", [0, 1, 2])
def test_a_sample_without_selections_among_them(bd, sample, monkeypatch):  # noqa: F811
    name = "short_e64_dropped"
    monkeypatch.setitem(B.CASES, name, CASES[name])
    c = Case(bd, name, all_dropped=sample)
    out, _ = c.check(True)
    assert not out[1][sample].any() and not out[2][sample].any()
    assert out[1][6].any()                              # one of 200 tokens (those of one token may be dropped as a whole)


def test_a_graph_of_them(bd, monkeypatch):  # noqa: F811
    name = "short_e128"
    monkeypatch.setitem(B.CASES, name, CASES[name])
    c = Case(bd, name)
    want, _ = c.check(True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = c.r.expert_balance(topk_idx=c.didx, loss_scale=0.5)
    for _ in range(3):
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
