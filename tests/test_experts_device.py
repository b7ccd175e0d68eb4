"""An expert layer belongs to the device that was current when it was made, and refuses calls while another one is: launches go to
the current device, whatever the device of the tensors. On the host, with the current device and the library faked."""
import pytest
import torch


@pytest.fixture(scope="module")
def bd():
    from paper_2604_23996_gb300.build import build_library
    build_library()
    from paper_2604_23996_gb300 import binding
    return binding


class Lib:
    """Notes every call; nothing runs."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or 0


@pytest.fixture
def layer(bd, monkeypatch):
    """A layer of cuda:1 whose tensors pass for ones of cuda:1."""
    lib = Lib()
    monkeypatch.setattr(bd, "_lib", lib)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 100 + index, raising=False)
    monkeypatch.setattr(bd.Experts, "_in", lambda self, name, t, shape, dtype: None if t is None else t.data_ptr())
    monkeypatch.setattr(bd.Experts, "_new", lambda self, t, shape, dtype, stream: torch.empty(shape, dtype=dtype) if t is None else t)
    ex = bd.Experts.__new__(bd.Experts)
    ex.plan, ex.T, ex.E, ex.k, ex.R, ex.dtype, ex._index = None, 4, 2, 1, 4, torch.bfloat16, 1
    ex.device, ex.ws = torch.device("cpu"), torch.zeros(1024, dtype=torch.uint8)
    ex.expert_offsets, ex.row_slot, ex.slot_row = (torch.zeros(n, dtype=torch.int32) for n in (3, 4, 4))
    return ex, lib


def calls(bd, ex, stream=None):
    rows, W = torch.zeros(4, 16, dtype=torch.bfloat16), torch.zeros(2, 16, 16, dtype=torch.bfloat16)
    w, idx = torch.zeros(4, 1), torch.zeros(4, 1, dtype=torch.int32)
    return [lambda: ex.sort(idx, stream=stream), lambda: ex.dispatch(rows, stream=stream),
            lambda: ex.dispatch_bwd(rows, stream=stream), lambda: ex.combine(rows, w, stream=stream),
            lambda: ex.combine_bwd(rows, rows, w, stream=stream), lambda: ex.linear(rows, W, stream=stream),
            lambda: ex.act_bwd(rows, rows, act=1, stream=stream), lambda: ex.linear_bwd(rows, rows, W, stream=stream),
            lambda: ex.device_status(stream=stream)]


def test_calls_are_refused_while_another_device_is_current(bd, layer, monkeypatch):
    ex, lib = layer
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)

    class Stream:
        device_index, cuda_stream = 1, 55

    for stream in (None, Stream()):
        for call in calls(bd, ex, stream):
            with pytest.raises(ValueError, match="cuda:1.*cuda:0"):
                call()
    assert not lib.calls


def test_a_stream_of_another_device_is_refused(bd, layer, monkeypatch):
    ex, lib = layer
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)

    class Stream:
        device_index, cuda_stream = 0, 55

    for call in calls(bd, ex, Stream()):
        with pytest.raises(ValueError, match="stream"):
            call()
    assert not lib.calls


def test_calls_on_its_own_device_run_on_its_stream(bd, layer, monkeypatch):
    ex, lib = layer
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)

    class Stream:
        device_index, cuda_stream = 1, 55

    for stream, handle in ((None, 101), (Stream(), 55)):
        for call in calls(bd, ex, stream):
            call()
            assert lib.calls.pop()[1][-1] == handle


@pytest.mark.parametrize("device", ["cuda:1", "cpu"])
def test_a_layer_of_another_device_is_not_made(bd, monkeypatch, device):
    monkeypatch.setattr(bd, "_lib", Lib())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="device"):
        bd.Experts(4, 2, 1, device=device)
    assert all(name == "smoes_experts_destroy" for name, _ in bd._lib.calls)
