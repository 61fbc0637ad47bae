"""Pins of the base losses' oracle that do not depend on it: differences of the
loss, the closed forms of small rows, the cross entropy as a distillation."""
import numpy as np
import pytest

from oracle import losses as lo

RNG = np.random.default_rng(5)


def _members(kind, R, V, K):
    if kind == "labels":
        labels = RNG.integers(0, V, R)
        labels[0] = -1
        return lo.label_members(labels)
    idx = RNG.integers(0, V, (R, K))          # (columns may repeat)
    idx[0, 1:] = -1
    t = RNG.normal(size=(R, K))
    return lo.teacher_members(idx, t, None if kind == "own" else lo._lse(t) + 0.3, 1.3)


@pytest.mark.parametrize("kind", ("labels", "own", "teacher"))
def test_gradient_against_differences(kind):
    R, V, T = 5, 11, 0.7
    x, w = RNG.normal(size=(R, V)), RNG.uniform(0.5, 2.0, R)
    mem = _members(kind, R, V, 4)
    g = lo.losses(x, *mem, w, T, 1.5)["grad"]
    for r in range(R):
        for v in range(V):
            up, down = x.copy(), x.copy()
            up[r, v] += 1e-5
            down[r, v] -= 1e-5
            d = (lo.losses(up, *mem, w, T, 1.5)["total"] - lo.losses(down, *mem, w, T, 1.5)["total"]) / 2e-5
            assert abs(d - g[r, v]) < 1e-8


def test_head_gradients_against_differences():
    R, V, H = 4, 7, 3
    h, w = RNG.normal(size=(R, H)), RNG.normal(size=(V, H))
    mem = _members("teacher", R, V, 3)
    out = lo.head(h, w, mem, None, 0.9, 0.5)
    for arr, g in ((h, out["grad_hidden"]), (w, out["grad_weight"])):
        for at in np.ndindex(arr.shape):
            old = arr[at]
            arr[at] = old + 1e-5
            up = lo.head(h, w, mem, None, 0.9, 0.5)["total"]
            arr[at] = old - 1e-5
            down = lo.head(h, w, mem, None, 0.9, 0.5)["total"]
            arr[at] = old
            assert abs((up - down) / 2e-5 - g[at]) < 1e-8


def test_closed_forms():
    # two equal logits: log 2, gradient +-1/2
    out = lo.losses(np.zeros((1, 2)), *lo.label_members([1]))
    assert np.isclose(out["loss"][0], np.log(2)) and np.allclose(out["grad"], [[0.5, -0.5]])
    # the distillation of a distribution into itself: no loss, no gradient
    x = RNG.normal(size=(3, 6))
    idx = np.tile(np.arange(6), (3, 1))
    out = lo.losses(x, *lo.teacher_members(idx, x))
    assert np.allclose(out["loss"], 0) and np.allclose(out["grad"], 0)
    # one member: the cross entropy
    a = lo.losses(x, *lo.teacher_members([[2], [-1], [5]], np.full((3, 1), 7.0)))
    b = lo.losses(x, *lo.label_members([2, -1, 5]))
    assert np.allclose(a["loss"], b["loss"]) and np.allclose(a["grad"], b["grad"])
    # the gradient of a live row sums to zero at any temperature
    assert np.allclose(lo.losses(x, *lo.label_members([0, 1, 2]), None, 0.3)["grad"].sum(1), 0)


def test_rows_out_of_play():
    x = RNG.normal(size=(4, 5))
    x[1] = np.nan
    x[2] = -np.inf
    out = lo.losses(x, *lo.label_members([0, -1, 3, 2]), np.array([1.0, 1.0, 1.0, 0.0]))
    assert np.array_equal(out["live"], [True, False, False, False])
    assert np.isneginf(out["lse"][2]) and np.all(out["grad"][1:] == 0) and np.all(out["loss"][1:] == 0)


def test_top_orders_ties_by_index():
    y = np.array([[1.0, 3.0, 3.0, -np.inf, 0.0, 3.0]])
    idx, val, _ = lo.top(y, 4)
    assert idx.tolist() == [[1, 2, 5, 0]] and val.tolist() == [[3.0, 3.0, 3.0, 1.0]]
    idx, val, _ = lo.top(y, 4, d2t=[5, 3, 1])
    assert idx.tolist() == [[0, 2, -1, -1]] and val[0, :2].tolist() == [3.0, 3.0]
