"""Host side of the expert layer (no GPU needed): plan limits, workspace sizes, and refusals that come before any
launch; the oracle's own identities."""
import ctypes as C

import numpy as np
import pytest

from oracle import experts_oracle as O


@pytest.fixture(scope="module")
def bd():
    from paper_2604_23996_gb300.build import build_library
    build_library()
    from paper_2604_23996_gb300 import binding
    return binding


@pytest.mark.parametrize("kw,code", [
    (dict(), 0), (dict(T=0), 0), (dict(T=1 << 20, k=16), 0), (dict(E=1, k=1), 0), (dict(E=256), 0), (dict(k=6, E=2), 0),
    (dict(T=-1), -1), (dict(E=0), -1), (dict(k=0), -1), (dict(max_width=-8), -1), (dict(dtype=2), -1),
    (dict(T=(1 << 20) + 1), -2), (dict(E=257), -2), (dict(k=17), -2), (dict(max_width=(1 << 20) + 1), -2),
])
def test_plan_limits(bd, kw, code):
    got, plan = bd.smoes_experts_create(**{**dict(T=100, E=16, k=2, dtype=bd.SMOES_BF16, max_width=64), **kw})
    assert got == code
    if code == 0:
        assert bd.smoes_experts_workspace_bytes(plan) >= 512
        bd.smoes_experts_destroy(plan)
    else:
        assert not plan.value


def test_calls_refuse_before_any_launch(bd):
    """Fake device addresses: every one of these returns on the host."""
    lib = C.CDLL(bd.LIB)
    code, plan = bd.smoes_experts_create(10, 4, 2, bd.SMOES_BF16, 64)
    assert code == 0
    n = bd.smoes_experts_workspace_bytes(plan)
    ok, odd, ws = C.c_void_p(0x10000), C.c_void_p(0x10008), C.c_void_p(0x20000)
    z = C.c_size_t(n)
    lib.smoes_expert_sort.argtypes = None
    assert lib.smoes_expert_sort(None, ok, ok, ok, ok, ws, z, None) == -1
    assert lib.smoes_expert_sort(plan, ok, ok, ok, ok, None, z, None) == -4
    assert lib.smoes_expert_sort(plan, ok, ok, ok, ok, ws, C.c_size_t(n - 1), None) == -4
    assert lib.smoes_expert_sort(plan, ok, ok, ok, ok, ok.__class__(0x20010), z, None) == -3
    assert lib.smoes_expert_sort(plan, None, ok, ok, ok, ws, z, None) == -1
    assert lib.smoes_expert_sort(plan, ok, ok, odd, ok, ws, z, None) == -3
    assert lib.smoes_expert_dispatch(plan, ok, 12, ok, ok, ok, None) == -1
    assert lib.smoes_expert_dispatch(plan, ok, (1 << 20) + 8, ok, ok, ok, None) == -2
    assert lib.smoes_expert_dispatch(plan, odd, 16, ok, ok, ok, None) == -3
    assert lib.smoes_expert_dispatch(plan, ok, 16, None, ok, ok, None) == -1
    assert lib.smoes_expert_dispatch_bwd(plan, ok, 16, ok, odd, ok, None) == -3
    assert lib.smoes_expert_combine(plan, ok, 16, None, ok, None, ok, None) == -1
    assert lib.smoes_expert_combine_bwd(plan, ok, ok, 16, ok, ok, ok, ok, None, None) == -1

    def linear(n_in=16, n_out=16, act=0, gated=0, X=ok, out=ok):
        a = bd.LinearArgs(X, ok, None, None, n_in, n_out, act, gated)
        return lib.smoes_expert_linear(plan, C.byref(a), ok, out, None, ws, z, None)

    assert linear(act=3) == -1 and linear(act=-1) == -1 and linear(gated=2) == -1
    assert linear(n_in=0) == -1 and linear(n_out=12) == -1 and linear(n_in=(1 << 20) + 8) == -2
    assert linear(n_out=1 << 20, gated=1) == -2 and linear(X=None) == -1 and linear(out=odd) == -3
    act = lib.smoes_expert_act_bwd
    assert act(plan, ok, ok, 64, 1, 1, ok, ok, ok, ws, z, None) == -4      # 128 > max_width
    assert act(plan, ok, ok, 16, 0, 0, ok, ok, ok, ws, z, None) == -1      # dZ is dOut
    assert act(plan, ok, None, 16, 0, 0, ok, None, None, ws, z, None) == -1
    assert act(plan, ok, None, 16, 1, 0, ok, ok, None, ws, z, None) == -1
    bwd = lib.smoes_expert_linear_bwd
    assert bwd(plan, ok, ok, ok, 16, 16, ok, None, None, 0, ws, z, None) == -1
    assert bwd(plan, ok, None, ok, 16, 16, ok, None, ok, 0, ws, z, None) == -1
    assert bwd(plan, ok, ok, None, 16, 16, ok, ok, None, 0, ws, z, None) == -1
    assert bwd(plan, ok, ok, ok, 16, 16, ok, ok, odd, 0, ws, z, None) == -3
    bd.smoes_experts_destroy(plan)


def test_oracle_slopes_are_the_differences_of_the_activations():
    z = np.linspace(-9, 9, 2001)
    h = 1e-5
    for kind in (O.NONE, O.SILU, O.GELU):
        fd = (O.act(kind, z + h) - O.act(kind, z - h)) / (2 * h)
        assert np.abs(fd - O.act_slope(kind, z)).max() < 1e-9      # h^2/6 f''' + 2^-53 * 9 / h


def test_oracle_layer_is_the_dense_layer_token_by_token():
    rng = np.random.default_rng(0)
    T, E, k, d, f = 30, 5, 2, 7, 3
    idx = np.argsort(rng.random((T, E)), 1)[:, :k].astype(np.int32)
    idx[4, 1] = -1
    w, X = rng.random((T, k)), rng.standard_normal((T, d))
    W1, W2 = rng.standard_normal((E, 2 * f, d)), rng.standard_normal((E, d, f))
    off, row_slot, slot_row = O.sort(idx, E)
    h, _ = O.linear(O.dispatch(X, row_slot, k), W1, off, None, O.SILU, True)
    y, _ = O.linear(h, W2, off)
    got = O.back(y, slot_row, w, X)
    for t in range(T):
        want = X[t].copy()
        for s in range(k):
            if idx[t, s] >= 0:
                zz = W1[idx[t, s]] @ X[t]
                want += w[t, s] * (W2[idx[t, s]] @ (zz[:f] / (1 + np.exp(-zz[:f])) * zz[f:]))
        assert np.allclose(got[t], want, rtol=1e-12, atol=1e-12)
