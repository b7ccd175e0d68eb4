"""Calls of the MoE layer that are refused before the router or the experts are touched (no GPU needed: both are stand-ins)."""
import pytest
import torch

from tests.test_mx_host import bd  # noqa: F401  (the fixture: builds the library)


class Untouched:
    def __getattr__(self, name):
        raise AssertionError(f"{name} was used")


class Experts(Untouched):
    def __init__(self, dtype):
        self.dtype = dtype

    def check_device(self):
        pass


def layer(dtype):
    from paper_2604_23996_gb300.moe_layer import MoELayer
    it = object.__new__(MoELayer)
    it.router, it.experts, it.norm, it.saved, it.kept, it.balance = Untouched(), Experts(dtype), None, "the forward's", None, None
    return it


def weights(bd):  # noqa: F811
    q = bd.Mx(torch.zeros(2, 64, 16, dtype=torch.uint8), torch.zeros(2, 64, 1, dtype=torch.uint8))
    return q, q


def test_4_bit_weights_of_an_fp32_layer(bd):  # noqa: F811
    it = layer(torch.float32)
    with pytest.raises(ValueError, match="bf16"):
        it.forward(torch.zeros(4, 32), None, *weights(bd), training=False)
    assert it.saved == "the forward's" and it.kept is None


def test_4_bit_weights_in_training_or_mixed(bd):  # noqa: F811
    it = layer(torch.bfloat16)
    q, _ = weights(bd)
    for args, training in (((q, q), True), ((q, torch.zeros(2)), False), ((torch.zeros(2), q), False)):
        with pytest.raises(ValueError, match="4 bits"):
            it.forward(torch.zeros(4, 32), None, *args, training=training)
    assert it.saved == "the forward's"
