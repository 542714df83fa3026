"""The 64-bit reference of the router's losses, against the losses' own
properties and differences of the forward (CPU)."""
import numpy as np
import pytest

from tests import router_loss_ref as R


def test_equal_loads_have_balance_one():
    E, k = 8, 2
    y = np.zeros((E, E))
    idx = np.stack([np.arange(E), (np.arange(E) + 1) % E], 1)
    bal, z, counts, psum, n = R.forward(y, idx)
    assert bal[0] == pytest.approx(1.0) and (counts == k).all() and n[0] == E
    assert z[0] == pytest.approx(np.log(E) ** 2)


def test_one_expert_for_all_has_balance_e_over_k():
    E, k, T = 6, 2, 5
    y = np.full((T, E), -1000.0)
    y[:, 3] = 0.0
    bal = R.forward(y, np.tile([3, 1], (T, 1)))[0]
    assert bal[0] == pytest.approx(E / k)


@pytest.mark.parametrize("masked", [False, True])
def test_gradient_against_differences(masked):
    rng = np.random.default_rng(3)
    T, E, k = 9, 5, 2
    y = rng.standard_normal((T, E))
    idx = np.argsort(-y, 1)[:, :k]
    off = [1, 4, 4, 8]
    mask = rng.random(T) < 0.7 if masked else None
    db, dz = rng.standard_normal(3), rng.standard_normal(3)
    _, _, counts, _, n = R.forward(y, idx, off, mask)
    got = R.backward(y, counts, n, db, dz, k, off, mask)

    def loss(v):
        b, z = R.forward(v, idx, off, mask)[:2]
        return (b * db).sum() + (z * dz).sum()

    h = 1e-6
    for t in range(T):
        for e in range(E):
            up, dn = y.copy(), y.copy()
            up[t, e] += h
            dn[t, e] -= h
            assert got[t, e] == pytest.approx((loss(up) - loss(dn)) / (2 * h), abs=1e-8)
