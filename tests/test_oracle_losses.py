"""Pins of oracle/losses.py: every gradient against differences of its loss, and the closed forms of special cases."""
import numpy as np
import pytest

from oracle import losses as ol


def rows(seed, n, v):
    r = np.random.RandomState(seed)
    return r.randn(n, v) * 2.0, r


def differences(f, z, h=1e-6):
    g = np.zeros_like(z)
    for i in range(len(z)):
        a, b = z.copy(), z.copy()
        a[i] += h
        b[i] -= h
        g[i] = (f(a) - f(b)) / (2 * h)
    return g


@pytest.mark.parametrize("tau,soft,hard", [(1.0, 1.0, 0.0), (2.0, 0.7, 0.3), (0.5, 0.0, 1.0), (4.0, 1.0, 0.5)])
def test_distillation_gradient_is_that_of_the_loss(tau, soft, hard):
    z, r = rows(1, 4, 13)
    for zz in z:
        ids, t = [3, 7, -1, 3, 12], r.randn(5)                     # an empty slot, and one word twice
        loss, grad, _, _ = ol.distill_row(zz, ids, t, 7, tau, soft, hard)
        want = differences(lambda x: ol.distill_row(x, ids, t, 7, tau, soft, hard)[0], zz)
        assert np.allclose(grad, want, atol=2e-8)
        assert abs(grad.sum()) < 1e-12                               # the losses do not change when a row is shifted


def test_distillation_of_the_student_itself_is_zero_and_without_slots_is_cross_entropy():
    z, _ = rows(2, 1, 9)
    loss, grad, _, _ = ol.distill_row(z[0], list(range(9)), z[0], 0, 2.0, 1.0, 0.0)
    assert abs(loss) < 1e-14 and np.abs(grad).max() < 1e-14
    loss, grad, _, lse = ol.distill_row(z[0], [-1, -1], [0.0, 1.0], 4, 2.0, 1.0, 1.0)
    assert loss == pytest.approx(lse - z[0][4]) and np.allclose(grad, ol.softmax(z[0]) - (np.arange(9) == 4))


@pytest.mark.parametrize("advantage", [1.3, -0.8, 0.0])
@pytest.mark.parametrize("old", [-2.0, -1.5, -0.9, -1.1])
def test_policy_derivative_is_that_of_the_loss(advantage, old):
    f = lambda x: ol.policy_of_logp(x, old, -1.3, advantage, 0.2, 0.25, 0.1)      # noqa: E731
    x = -1.45                                                                      # ratios e^0.55, e^0.05, e^-0.55, e^-0.35: on both sides of the limits
    assert (f(x + 1e-6)[0] - f(x - 1e-6)[0]) / 2e-6 == pytest.approx(f(x)[1], abs=1e-8)
    z, _ = rows(3, 1, 11)
    logp, lse, grad = ol.token_logp(z[0], 5)
    assert np.allclose(grad, differences(lambda v: ol.token_logp(v, 5)[0], z[0]), atol=1e-8) and logp == pytest.approx(z[0][5] - lse)


@pytest.mark.parametrize("kind,smoothing", [("sigmoid", 0.0), ("sigmoid", 0.1), ("hinge", 0.0), ("squared", 0.0)])
def test_preference_derivative_is_that_of_the_loss(kind, smoothing):
    for margin in (-30.0, -2.0, 0.3, 4.0, 25.0):
        f = lambda x: ol.preference_of_margin(x, kind, 0.3, smoothing)             # noqa: E731
        assert (f(margin + 1e-5)[0] - f(margin - 1e-5)[0]) / 2e-5 == pytest.approx(f(margin)[1], abs=1e-7)
    assert ol.preference_of_margin(0.0, "sigmoid", 1.0, 0.0)[0] == pytest.approx(np.log(2.0))
