"""Pins of the oracle of microscaled numbers and of distillation: closed forms, brute force and differences (CPU)."""
import numpy as np
import pytest

from oracle import train_oracle as O


def test_every_element_and_every_border():
    # magnitudes up to 6 in a block whose scale is 2^0 (its largest value is 4 to 6: exponent 2)
    a = np.zeros((1, 32))
    a[0, :16] = [0, 0.5, 1, 1.5, 2, 3, 4, 6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5]
    a[0, 16:24] = [0.2500001, 0.7499999, 1.2500001, 1.7499999, 2.5000001, 3.4999999, 5.0000001, -0.1]
    codes, scales = O.mx_quantize(a)
    assert scales[0, 0] == 127
    v = O.mx_values(O.mx_codes(codes), scales)[0]
    assert list(v[:16]) == [0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, 1, 1, 2, 2, 4, 4, -4]
    assert list(v[16:24]) == [0.5, 0.5, 1.5, 1.5, 3, 3, 6, 0] and codes[0, 23] == 8


def test_nearest_element_by_brute_force():
    rng = np.random.default_rng(3)
    a = rng.uniform(0, 8, size=(50, 32))
    a[:, 0] = rng.uniform(4, 8, size=50)                   # scale 2^0 in every block
    v = O.mx_values(O.mx_codes(O.mx_quantize(a)[0]), O.mx_quantize(a)[1])
    best = np.abs(a[:, :, None] - O.ELEMENTS).min(axis=2)
    assert np.array_equal(np.abs(a - v), best)


@pytest.mark.parametrize("top,byte", [(1.0, 125), (0.75, 124), (6.0, 127), (8.0, 128), (3.4028234663852886e38, 252), (2.0 ** -126, 0),
                                      (2.0 ** -149, 0), (2.0 ** -124, 1), (0.0, 127), (np.inf, 255), (np.nan, 255)])
def test_scale_of_a_block(top, byte):
    x = np.zeros((1, 32))
    x[0, 7] = top
    codes, scales = O.mx_quantize(x)
    assert scales[0, 0] == byte
    if byte == 255:
        assert np.isnan(O.mx_values(O.mx_codes(codes), scales)).all() and not codes.any()


def test_product_of_hand_made_blocks():
    x, w = np.zeros((1, 64)), np.zeros((2, 64))
    x[0, 0], x[0, 33] = 6.0, -12.0
    w[0, 0], w[1, 33] = 0.5, 3.0
    cx, cw = O.mx_quantize(x), O.mx_quantize(w)
    y, size = O.mx_linear(O.mx_codes(cw[0]), cw[1], O.mx_codes(cx[0]), cx[1])
    assert y.tolist() == [[3.0, -36.0]] and size.tolist() == [[3.0, 36.0]]


def test_loss_closed_forms():
    # the student equals the teacher and the teacher's set is the whole vocabulary: no loss, no gradient
    rng = np.random.default_rng(5)
    z = rng.normal(size=(3, 9))
    idx = np.tile(np.arange(9), (3, 1))
    loss, grad, _, _, _ = O.distill(z, idx, z, tau=1.7)
    assert np.abs(loss).max() < 1e-14 and np.abs(grad).max() < 1e-15
    # one entry: cross entropy against its index
    loss, grad, _, _, _ = O.distill(z, idx[:, 4:5], z[:, 4:5])
    q = np.exp(z) / np.exp(z).sum(axis=1, keepdims=True)
    assert np.allclose(loss, -np.log(q[:, 4]), rtol=1e-14)
    assert np.allclose(grad, q - (np.arange(9) == 4), atol=1e-15)
    # uniform logits
    loss, _, stats, _, _ = O.distill(np.zeros((1, 8)), np.array([[2, -1, 99]]), np.array([[1.0, 5.0, 5.0]]))
    assert np.isclose(loss[0], np.log(8)) and stats.tolist() == [[0.0, 8.0]]


@pytest.mark.parametrize("tau", [1.0, 2.0, 0.7])
@pytest.mark.parametrize("whole", [False, True])
def test_gradient_by_differences(tau, whole):
    rng = np.random.default_rng(11)
    z, teacher = rng.normal(size=(2, 12)), rng.normal(size=(2, 12))
    idx = np.array([[3, 3, 7, -1], [0, 11, 5, 40]])          # an index twice, absent entries
    top = np.take_along_axis(teacher, np.clip(idx, 0, 11), axis=1)
    lse = np.log(np.exp(teacher / tau).sum(axis=1)) if whole else None
    weight = np.array([0.5, 2.0])
    _, grad, _, _, _ = O.distill(z, idx, top, tau, lse, weight)
    h = 1e-5
    for t in range(2):
        for v in range(12):
            d = np.zeros_like(z)
            d[t, v] = h
            up, down = O.distill(z + d, idx, top, tau, lse, weight)[0].sum(), O.distill(z - d, idx, top, tau, lse, weight)[0].sum()
            assert abs((up - down) / (2 * h) - grad[t, v]) < 1e-8


def test_tokens_without_entries_or_weight():
    z = np.ones((3, 5))
    idx = np.array([[-1, -1], [1, 2], [1, 2]])
    top = np.array([[1.0, 2.0], [-np.inf, -np.inf], [1.0, 2.0]])
    loss, grad, stats, _, _ = O.distill(z, idx, top, weight=np.array([1.0, 1.0, 0.0]))
    assert not loss.any() and not grad.any() and np.isnan(stats[2]).all()


def test_distill_entries_without_probability_add_nothing():
    # the teacher rules out (p underflows to 0) what the student rules out too
    z = np.array([[0.5, -np.inf, 1.0]])
    loss, grad, *_ = O.distill(z, np.array([[0, 1, 2]]), np.array([[1.0, -65504.0, 2.0]]), 0.7)
    short = O.distill(z[:, [0, 2]], np.array([[0, 1]]), np.array([[1.0, 2.0]]), 0.7)
    assert np.array_equal(loss, short[0]) and np.array_equal(grad[:, [0, 2]], short[1]) and grad[0, 1] == 0
