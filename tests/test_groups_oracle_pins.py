"""Pins of the oracle of row groups, experts and adapters (CPU): hand-worked values, and gradients against differences."""
import numpy as np
import pytest

from oracle import groups_oracle as O


def test_plan_by_hand():
    order, groups, offsets = O.group_rows([2, 0, -1, 2, 5, 0], 3)
    assert order.tolist() == [1, 5, 0, 3, 2, 4] and groups.tolist() == [0, 0, 2, 2, -1, -1] and offsets.tolist() == [0, 2, 2, 4]


def test_experts_by_hand():
    x, w = np.array([[1.0, 2.0], [3.0, 4.0]]), np.array([[[1.0, 0.0]], [[0.0, -1.0]]])
    y, size = O.grouped(x, w, [1, 0, 7, 1], 2)
    assert y.tolist() == [[-2.0], [1.0], [0.0], [-4.0]] and size.tolist() == [[2.0], [1.0], [0.0], [4.0]]


def test_adapters_by_hand():
    x, a, b = np.array([[1.0, 2.0], [3.0, 4.0]]), np.array([[[1.0, -1.0]]]), np.array([[[2.0], [0.5], [1.0]]])
    y, t, *_ = O.adapters(x, a, b, [0, -1], base=np.ones((2, 3)), scale=[3.0])
    assert t.tolist() == [[-1.0], [0.0]] and y.tolist() == [[-5.0, -0.5, -2.0], [1.0, 1.0, 1.0]]


@pytest.mark.parametrize("seed", range(3))
def test_gradients_against_differences(seed):
    rng = np.random.default_rng(seed)
    M, G, r, K, N = 5, 3, 2, 4, 3
    x, a, b, w = rng.normal(size=(M, K)), rng.normal(size=(G, r, K)), rng.normal(size=(G, N, r)), rng.normal(size=(M, N))
    group, scale = rng.integers(-1, G, size=M), rng.normal(size=G)

    def loss(x, a, b):
        return (w * O.adapters(x, a, b, group, scale=scale)[0]).sum()

    t = O.adapters(x, a, b, group, scale=scale)[1]
    (dx, *_), (da, *_), (db, _) = O.adapters_grad(w, x, a, b, t, group, scale=scale)
    for i, (value, grad) in enumerate(((x, dx), (a, da), (b, db))):
        for at in np.ndindex(*value.shape):
            up, down = [x.copy(), a.copy(), b.copy()], [x.copy(), a.copy(), b.copy()]
            up[i][at] += 1e-6
            down[i][at] -= 1e-6
            assert abs((loss(*up) - loss(*down)) / 2e-6 - grad[at]) < 1e-7
