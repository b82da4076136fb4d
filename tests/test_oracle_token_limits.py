"""Pins of oracle/tokens.py at the limits of its ranges: hand cases, identities and differences."""
import math

import numpy as np
import pytest

from oracle import tokens as ot


@pytest.mark.parametrize("gap", [10.0, 90.0, 1000.0, 1e9])
def test_a_tail_far_below_the_list(gap):
    """2 listed tokens at `gap`, 6 others at 0: p_T = 6 e^-gap / (2 + 6 e^-gap), and the tail's pull is shared evenly."""
    z = np.zeros(8)
    z[:2] = gap
    loss, grad = ot.distill_row(z, [0, 1], [math.log(0.45)] * 2)
    s = 2 + 6 * math.exp(-gap)
    ln_pt = math.log(6) - gap - math.log(s)
    want = 0.9 * (math.log(0.45) + math.log(s)) + 0.1 * (math.log(0.1) - ln_pt)
    np.testing.assert_allclose(loss, want, rtol=1e-13)
    np.testing.assert_allclose(grad[:2], 1 / s - 0.45, rtol=1e-12)
    np.testing.assert_allclose(grad[2:], math.exp(-gap) / s - 0.1 / 6, rtol=1e-12)
    assert abs(grad.sum()) < 1e-15


def _difference(z, ids, lq, j, **kw):
    h = np.zeros(len(z))
    h[j] = 1e-5
    return (ot.distill_row(z + h, ids, lq, **kw)[0] - ot.distill_row(z - h, ids, lq, **kw)[0]) / 2e-5


@pytest.mark.parametrize("scale", [1.0, 0.7])
def test_gradient_where_the_tail_is_masked_altogether(scale):
    """The second term is left out, and what is left has the weight Q."""
    z = np.array([0.3, -math.inf, 1.2, -math.inf, -0.5, -math.inf])
    ids, lq = [4, 0, 2], np.log([0.2, 0.3, 0.1])
    loss, grad = ot.distill_row(z, ids, lq, scale=scale, weight=1.3)
    for j in (0, 2, 4):
        assert abs(_difference(z, ids, lq, j, scale=scale, weight=1.3) - grad[j]) < 1e-8
    assert abs(grad.sum()) < 1e-15 and (grad[[1, 3, 5]] == 0).all() and abs(grad[2]) > 0.1


def test_gradient_of_a_list_that_is_no_distribution():
    z = np.random.default_rng(3).standard_normal(9)
    lp = ot.log_softmax(z[None])[0]
    _, grad = ot.distill_row(z, [2, 5], np.log([0.9, 0.5]))
    want = np.exp(lp)
    want[[2, 5]] -= [0.9, 0.5]
    np.testing.assert_allclose(grad, want, rtol=1e-14)


@pytest.mark.parametrize("by", [-700.0, -100.0, 100.0, 1e5])
def test_only_differences_of_a_renormalised_list_count(by):
    z = np.random.default_rng(4).standard_normal(9)
    lq = np.array([-0.5, -1.25, -3.0])
    a = ot.distill_row(z, [2, 5, 7], lq, bucket=False)
    b = ot.distill_row(z, [2, 5, 7], lq + by, bucket=False)
    np.testing.assert_allclose(a[0], b[0], rtol=1e-9)
    np.testing.assert_allclose(a[1], b[1], rtol=1e-9)
    loss, grad = ot.distill_row(z, [2, 5], [-math.inf] * 2, bucket=False)
    assert loss == 0 and not grad.any()
