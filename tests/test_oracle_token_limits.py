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
