"""Pins of the oracle of a training step's head: gradients against differences, the generator against known values."""
import numpy as np
import pytest

from oracle import head_oracle as O


def _differences(f, x, step=1e-6):
    out = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        up, down = x.copy(), x.copy()
        up[i] += step
        down[i] -= step
        out[i] = (f(up) - f(down)) / (2 * step)
    return out


def test_mix64_is_the_output_function_of_splitmix64():
    # the first three outputs of SplitMix64 from state 0
    assert [O.mix64(k * O.GOLDEN & O.MASK) for k in (1, 2, 3)] == [0xE220A8397B1DCDAF, 0x6E789E6AA1B965F4, 0x06C45D188009454F]


def test_dropout_keeps_the_share_it_should():
    n = 20000
    for p in (0.0, 0.1, 0.5, 0.9, 1.0):
        share = O.kept(n, p, 12345, 7).mean()
        assert abs(share - (1 - p)) <= 5 * np.sqrt(p * (1 - p) / n)
    assert np.array_equal(O.kept(100, 0.5, 3, 8), O.kept(116, 0.5, 3, 0)[16:])      # word 8 is the 16th element's
    assert not np.array_equal(O.kept(100, 0.5, 3, 0), O.kept(100, 0.5, 4, 0))
    x = np.array([[np.inf, np.nan, 1.0, -2.0]])
    assert np.all(O.dropout(x, 1.0, 1, 0) == 0)


def test_layernorm_gradients_are_the_differences():
    rng = np.random.default_rng(0)
    x, gamma, beta, gy = rng.standard_normal((3, 5)), rng.standard_normal(5), rng.standard_normal(5), rng.standard_normal((3, 5))
    value = lambda x_, g_, b_: float((O.layernorm(x_, g_, b_, 1e-5)[0] * gy).sum())
    dx, dgamma, dbeta = O.layernorm_backward(x, gamma, gy, 1e-5)
    # central differences: an error of step^2 times the third derivative, and 1e-16 / step of rounding
    assert np.abs(dx - _differences(lambda v: value(v, gamma, beta), x)).max() < 1e-7
    assert np.abs(dgamma - _differences(lambda v: value(x, v, beta), gamma)).max() < 1e-7
    assert np.abs(dbeta - _differences(lambda v: value(x, gamma, v), beta)).max() < 1e-7


@pytest.mark.parametrize("with_bias", [False, True])
def test_loss_gradients_are_the_differences(with_bias):
    rng = np.random.default_rng(1)
    h, V, b = rng.standard_normal((4, 3)), rng.standard_normal((6, 3)), rng.standard_normal(6)
    label, gloss = np.array([2, -1, 5, 0]), rng.random(4)
    bias = b if with_bias else None
    value = lambda h_, V_, b_: float((O.softmax_xent(h_, V_, b_, label)[0] * gloss).sum())
    dh, dV, db, g, p = O.softmax_xent_backward(h, V, bias, label, gloss)
    assert np.abs(dh - _differences(lambda v: value(v, V, bias), h)).max() < 1e-8
    assert np.abs(dV - _differences(lambda v: value(h, v, bias), V)).max() < 1e-8
    if with_bias:
        assert np.abs(db - _differences(lambda v: value(h, V, v), b)).max() < 1e-8
    assert np.all(dh[1] == 0) and np.allclose(p.sum(1), [1, 0, 1, 1]) and np.abs(g.sum(1)).max() < 1e-15


def test_a_class_behind_a_bias_of_minus_infinity_takes_no_part():
    rng = np.random.default_rng(2)
    h, V, b = rng.standard_normal((2, 3)), rng.standard_normal((4, 3)), np.array([0.1, -np.inf, 0.2, 0.3])
    label = np.array([0, 3])
    loss, lse = O.softmax_xent(h, V, b, label)
    keep = [0, 2, 3]
    loss3, lse3 = O.softmax_xent(h, V[keep], b[keep], np.array([0, 2]))
    assert np.allclose(loss, loss3) and np.allclose(lse, lse3)
    dV = O.softmax_xent_backward(h, V, b, label, np.ones(2))[1]
    assert np.all(dV[1] == 0)
