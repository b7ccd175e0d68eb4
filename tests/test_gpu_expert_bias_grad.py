"""The experts' bias gradient where few of the plan's rows take part, against the fp64 oracle. Rows are summed in ranges that
are sized by the plan; with fewer rows than ranges some ranges have none, and nothing of the workspace that this call did not
write may reach the sums: the workspace behind its header is filled with NaN first.

Tolerances as in the activation gradient's own test: the functions' 2^-18 of |z| + 1 a row, and a sum of n values in fp32."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as O
from tests.test_gpu_experts import U_F32, Layer, assert_close, bd  # noqa: F401  (bd: the fixture)

pytestmark = pytest.mark.gpu

HEADER = 512                                            # status and barrier words, cleared by workspace_init


def gradient(lay, dOut, z, act, gated, byte):
    lay.ex.ws[HEADER:] = byte
    return lay.ex.act_bwd(dOut, z if act or gated else None, act=act, gated=gated, bias_grad=True)[1]


def check(lay, n_out, act, gated):
    n_z = n_out * (2 if gated else 1)
    dOut, z = lay.rows(n_out), lay.rows(n_z, std=2.0)
    db = gradient(lay, dOut, z, act, gated, 255)        # four bytes of 255: NaN
    dh, zh = lay.host_rows(dOut), lay.host_rows(z)
    dZ, want = O.act_bwd(dh, zh, lay.off, act, gated)
    near = 2.0 ** -18 * np.abs(dh) * (np.abs(zh[:, :n_out]) + 1) if act else np.zeros_like(dh)
    if gated:
        near = np.concatenate([near * np.abs(zh[:, n_out:]), near], 1)
    mag = np.abs(dZ) * (lay.n + 2) * U_F32 + near
    assert_close(db, want, np.stack([mag[lay.off[e]:lay.off[e + 1]].sum(0) for e in range(lay.E)]), "db")
    assert torch.equal(db, gradient(lay, dOut, z, act, gated, 0))


# T, E, k, n_out, act, gated, dropped
FEW = [(4096, 4, 1, 40, 1, False, 0.98), (4096, 4, 1, 40, 2, True, 0.95), (1366, 48, 6, 264, 1, True, 0.99),
       (8000, 1, 1, 520, 0, False, 0.97), (300, 16, 4, 72, 0, True, 0.9), (20000, 256, 8, 16, 2, False, 0.999)]


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("T,E,k,n_out,act,gated,dropped", FEW)
def test_bias_gradient_of_mostly_dropped_selections(bd, T, E, k, n_out, act, gated, dropped, dt):  # noqa: F811
    lay = Layer(bd, T, E, k, dt, seed=T + n_out, dropped=dropped, max_width=n_out * (2 if gated else 1))
    assert 0 < lay.n < T * k // 8                       # fewer rows than a range of eight each would take
    check(lay, n_out, act, gated)


@pytest.mark.parametrize("n", [1, 2, 3, 5, 31, 32])
def test_bias_gradient_of_a_few_rows_of_one_expert(bd, n):  # noqa: F811
    lay = Layer(bd, 32, 1, 1, torch.float32, seed=n, max_width=8)
    idx = np.full((32, 1), -1, dtype=np.int32)
    idx[np.random.default_rng(n).permutation(32)[:n]] = 0
    lay.off, lay.row_slot, lay.slot_row = O.sort(idx, 1)
    lay.n = n
    lay.ex.sort(torch.from_numpy(idx).cuda())
    check(lay, 8, 1, False)


@pytest.mark.parametrize("act,gated", [(0, False), (1, True), (2, False)])
def test_bias_gradient_accumulated(bd, act, gated):  # noqa: F811
    """What db held, plus the gradient in one addition: the same bits as that addition by itself."""
    lay = Layer(bd, 500, 12, 4, torch.bfloat16, seed=act, dropped=0.2, max_width=144)
    n_z = 144 if gated else 72
    dOut, z = lay.rows(72), lay.rows(n_z) if act or gated else None
    dZ, db = lay.ex.act_bwd(dOut, z, act=act, gated=gated, bias_grad=True)
    base = lay.normal(12, n_z, dtype=torch.float32)
    acc = base.clone()
    dZ2, got = lay.ex.act_bwd(dOut, z, act=act, gated=gated, db=acc, accumulate=True)
    assert got is acc and torch.equal(acc, base + db) and torch.equal(dZ2[:lay.n], dZ[:lay.n])
    with pytest.raises(ValueError):
        lay.ex.act_bwd(dOut, z, act=act, gated=gated, bias_grad=True, accumulate=True)


def test_bias_gradient_accumulated_without_tokens(bd):  # noqa: F811
    ex = bd.Experts(0, 3, 2, max_width=64)
    db = torch.full((3, 64), 5.0, device="cuda")
    ex.act_bwd(torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"), db=db, accumulate=True)
    assert (db == 5).all()
