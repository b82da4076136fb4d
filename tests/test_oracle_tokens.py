"""Pins of oracle/tokens.py: identities, hand cases and differences."""
import math

import numpy as np
import pytest

from oracle import tokens as ot


def test_log_softmax_hand_case_and_masks():
    lp = ot.log_softmax([[math.log(1.0), math.log(2.0), math.log(5.0), -math.inf]])
    np.testing.assert_allclose(np.exp(lp[0]), [1 / 8, 2 / 8, 5 / 8, 0])
    assert np.all(ot.log_softmax([[-math.inf] * 3]) == -math.inf)
    assert np.isnan(ot.log_softmax([[0.0, math.inf], [math.nan, 1.0]])).all()


def test_entropy_of_uniform_and_certain_rows():
    np.testing.assert_allclose(ot.entropy(ot.log_softmax(np.zeros((1, 37)))), math.log(37))
    assert ot.entropy(ot.log_softmax([[5.0, -math.inf]]))[0] == 0
    # -d/dscale of the normaliser: H = lse - scale * E[z]
    z = np.random.default_rng(0).standard_normal((1, 50))
    lse = lambda s: np.log(np.exp(s * z).sum())  # noqa: E731
    want = lse(1.3) - 1.3 * (lse(1.3 + 1e-6) - lse(1.3 - 1e-6)) / 2e-6
    np.testing.assert_allclose(ot.entropy(ot.log_softmax(z, 1.3)), want, rtol=1e-7)


def test_top_breaks_ties_by_index_and_ranks_nan_last():
    assert ot.top([[1.0, 3.0, 3.0, -0.0, 0.0, math.nan, -math.inf]], 7).tolist() == [[1, 2, 0, 3, 4, 5, 6]]


@pytest.mark.parametrize("bucket", [True, False])
@pytest.mark.parametrize("scale", [1.0, 0.7])
def test_distill_gradient_is_the_difference_quotient(bucket, scale):
    rng = np.random.default_rng(1)
    z = rng.standard_normal(12)
    t = np.sort(ot.log_softmax(rng.standard_normal((1, 12)))[0])[::-1][:4]
    ids = [7, 2, 9, 0]
    loss, grad = ot.distill_row(z, ids, t, scale, bucket, 1.7)
    for j in range(12):
        h = np.zeros(12)
        h[j] = 1e-5
        a, _ = ot.distill_row(z + h, ids, t, scale, bucket, 1.7)
        b, _ = ot.distill_row(z - h, ids, t, scale, bucket, 1.7)
        assert abs((a - b) / 2e-5 - grad[j]) < 1e-8
    assert abs(grad.sum()) < 1e-12 and loss > 0


def test_distill_identities():
    rng = np.random.default_rng(2)
    z = rng.standard_normal(20)
    lp = ot.log_softmax(z[None])[0]
    # the model itself as its teacher: nothing to learn
    loss, grad = ot.distill_row(z, [3, 8, 1], lp[[3, 8, 1]])
    assert abs(loss) < 1e-15 and np.abs(grad).max() < 1e-15
    # a list of every token is the whole divergence, with or without the bucket
    t = ot.log_softmax(rng.standard_normal((1, 20)))[0]
    whole = float((np.exp(t) * (t - lp)).sum())
    for bucket in (True, False):
        loss, grad = ot.distill_row(z, np.arange(20), t, bucket=bucket)
        assert abs(loss - whole) < 1e-12
        np.testing.assert_allclose(grad, np.exp(lp) - np.exp(t), atol=1e-12)
    # one certain token: cross entropy
    loss, grad = ot.distill_row(z, [4], [0.0], bucket=False)
    assert abs(loss + lp[4]) < 1e-14
    # padding, repeats and weight 0
    a = ot.distill_row(z, [4, -1, 4, 99], [-0.3, -1.0, -0.1, 0.0])
    b = ot.distill_row(z, [4], [-0.3])
    assert a[0] == b[0] and np.array_equal(a[1], b[1])
    assert ot.distill_row(z, [4], [0.0], weight=0.0)[0] == 0 and ot.distill_row(z, [-1], [0.0])[0] == 0


def test_reveal_hand_case():
    ids = np.array([[9, 0, 0, 5, 0, 0]])
    cand = np.array([[11, 12, 13, 14, 15, 16]])
    score = np.array([[9.0, 0.5, 0.7, 8.0, 0.7, math.nan]])
    out, left = ot.reveal(ids, cand, score, [2], 0)
    assert out.tolist() == [[9, 0, 13, 5, 15, 0]] and left.tolist() == [2]
    out, left = ot.reveal(ids, cand, score, [1], 0, lowest=True)
    assert out.tolist() == [[9, 12, 0, 5, 0, 0]]
    out, left = ot.reveal(ids, cand, score, [9], 0, window=[[4, 99]])
    assert out.tolist() == [[9, 0, 0, 5, 15, 16]] and left.tolist() == [2]
