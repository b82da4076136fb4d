"""oracle/ends.py against itself: draws against the distribution that they are draws from, gradients against differences."""
import numpy as np
import pytest

from oracle import ends as oe


def _logits(n, seed=0):
    rng = np.random.default_rng(seed)
    return np.round(2 * rng.standard_normal(n), 1)  # (with ties)


@pytest.mark.parametrize("kw", [dict(), dict(top_k=7), dict(top_p=0.6), dict(min_p=0.1), dict(top_k=40, top_p=0.8, min_p=0.02, scale=1.5)])
def test_a_grid_of_numbers_draws_each_token_by_its_weight(kw):
    z = _logits(1300)
    w = oe.weights(z, kw.get("scale", 1.0)) * oe.kept(z, **kw)[0]
    # the share of the unit square that draws a token: its block's share of u0 times its share of the block
    n = 200
    count = np.zeros(len(z))
    mass = np.add.reduceat(w, [0, 512, 1024])
    for i in range(n):
        u0 = (i + 0.5) / n
        for j in range(n):
            if j == 0:
                t, lp, _ = oe.sample(z, (u0, 0.0), **kw)
                b = t // 512
                cum = np.cumsum(w[512 * b:512 * b + 512])
            # (inside a block by the definition at once: the draw of the block is the same)
            count[512 * b + int((cum <= (j + 0.5) / n * cum[-1]).sum())] += 1
    share = count / n ** 2
    want = w / w.sum()
    # a border inside the grid moves a share by at most one cell of either side
    assert np.abs(np.add.reduceat(share, [0, 512, 1024]) - mass / w.sum()).max() <= 1.0 / n
    assert np.abs(share - want).max() <= 2.0 / n and (share[w == 0] == 0).all()


def test_cuts():
    z = np.array([0.0, 3.0, 1.0, 3.0, -np.inf, 2.0])
    assert oe.kept(z, top_k=1)[0].nonzero()[0].tolist() == [1]
    assert oe.kept(z, top_k=2)[0].nonzero()[0].tolist() == [1, 3]
    assert oe.kept(z, top_p=0.3)[0].nonzero()[0].tolist() == [1]
    assert oe.kept(z, top_p=0.5)[0].nonzero()[0].tolist() == [1, 3]
    assert oe.kept(z, min_p=1.0)[0].nonzero()[0].tolist() == [1, 3]
    assert oe.kept(z, min_p=0.2)[0].nonzero()[0].tolist() == [1, 3, 5]
    assert oe.sample(z, (0.0, 0.0))[0] == 0 and oe.sample(z, (1.0, 1.0))[0] == 5
    assert oe.sample(np.full(3, -np.inf), (0.5, 0.5))[:2] == (0, -np.inf)
    t, lp, _ = oe.sample(np.array([1.0, np.nan, 2.0]), (0.5, 0.5))
    assert t == 2 and np.isnan(lp)


def _difference(f, x, e=1e-5):
    out = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += e
        b[i] -= e
        out[i] = (f(a) - f(b)) / (2 * e)
    return out


@pytest.mark.parametrize("kind", ["rms", "ln", "ln_plain"])
@pytest.mark.parametrize("affine", ["", "g", "gb"])
@pytest.mark.parametrize("per", [0, 2])
def test_norm_gradient_against_differences(kind, affine, per):
    rng = np.random.default_rng(1)
    rows, d = 5, 8
    h, dout = rng.standard_normal((rows, d)) + 0.3, rng.standard_normal((rows, d))
    g = 1 + 0.2 * rng.standard_normal(d) if "g" in affine else None
    b = 0.2 * rng.standard_normal(d) if "b" in affine else None
    sc = 0.3 * rng.standard_normal((3, d)) if per else None
    sh = 0.3 * rng.standard_normal((3, d)) if per else None

    def loss(h=h, g=g, b=b, sh=sh, sc=sc):
        return float((oe.norm(h, kind, g, b, sh, sc, max(per, 1)) * dout).sum())
    got = oe.norm_grad(dout, h, kind, g, b, sc, max(per, 1), residual=np.ones((rows, d)))
    near = dict(rtol=1e-6, atol=1e-8)
    assert np.allclose(got["dh"] - 1, _difference(lambda x: loss(h=x), h), **near)
    if g is not None:
        assert np.allclose(got["dg"], _difference(lambda x: loss(g=x), g), **near)
    if b is not None:
        assert np.allclose(got["db"], _difference(lambda x: loss(b=x), b), **near)
    if per:
        assert np.allclose(got["dshift"], _difference(lambda x: loss(sh=x), sh), **near)
        assert np.allclose(got["dscale"], _difference(lambda x: loss(sc=x), sc), **near)


def test_embedding_gradient_against_differences():
    rng = np.random.default_rng(2)
    table, ids, dout = rng.standard_normal((6, 3)), np.array([1, 4, 1, -1, 5, 6, 1]), rng.standard_normal((7, 3))
    f = lambda t: float((oe.embedding(t, ids, 2.0) * dout).sum())  # noqa: E731
    got, size, n = oe.embedding_grad(dout, ids, 6, 2.0)
    assert np.allclose(got, _difference(f, table), rtol=1e-8, atol=1e-8) and n.tolist() == [0, 3, 0, 0, 1, 1]
    assert (size + 1e-12 >= np.abs(got)).all()
