"""sgd_kernel_sample on the GPU where its arithmetic is at its limits: logits as far apart as their type has them, at scales that bring
them together, against oracle/ends.py in float64 (bounds as in test_gpu_sample.py)."""
import numpy as np
import pytest
import torch

from oracle import ends as oe
from test_gpu_sample import B, FILTERS, _check, _draw, _numbers, _put  # noqa: F401
from test_sample_weights_host import UNIT, bound, weight

pytestmark = pytest.mark.gpu


def _wide(rows, vocab, scale, dtype, seed):
    """Logits whose scaled values lie some units apart, or as far as the type has them; the last row a few far below all others."""
    top = min(8.0 / scale, 3.3e38 if dtype != "f16" else 6e4)
    z = np.random.default_rng(seed).uniform(-top, top, (rows, vocab))
    z[-1, ::3] = -top
    z[-1, 1::3] = top
    return z


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [2.0 ** -63, 2.0 ** -64, 2.0 ** -65, 2.0 ** -100, 2.0 ** -118, 1e-38, 1.5e-39, 1e-41, 1e-45])
def test_differences_beyond_the_type(B, scale, dtype):
    """Differences of up to 6.6e38, which fp32 does not hold, at scales down to the smallest."""
    scale = float(np.float32(scale))
    for rows, vocab in ((5, 3), (9, 700), (5, 5000), (3, 40001)):
        z = _put(_wide(rows, vocab, scale, dtype, vocab), dtype)
        for i, kw in enumerate(FILTERS):
            u = _numbers(rows, i)
            _check(_draw(B, z, u, scale=scale, **kw), z, u, some=False, scale=scale, **kw)


def test_few_and_many_long_rows_at_a_small_scale(B):
    """By clusters, and by CTAs of their own."""
    scale = float(np.float32(1e-38))
    for rows in (1, 12, 300):
        z = _put(_wide(rows, 60001, scale, "f32", rows), "f32")
        few = slice(0, min(rows, 6))
        for i, kw in enumerate(FILTERS):
            u = _numbers(rows, i)
            ids, lp = _draw(B, z, u, scale=scale, **kw)
            _check((ids[few], lp[few]), z[few], u[few], some=False, scale=scale, **kw)


@pytest.mark.parametrize("scale", [1e9, 1e37, 2e38])
@pytest.mark.parametrize("rows", [3, 200])
def test_large_scales_of_long_rows(B, scale, rows):
    """All of the mass on the likeliest, or on those that equal it."""
    rng = np.random.default_rng(rows)
    z1 = rng.standard_normal((rows, 30011))
    z1[1::2] = np.round(z1[1::2])
    z = _put(z1, "f32")
    few = slice(0, min(rows, 6))
    for i, kw in enumerate(FILTERS):
        u = _numbers(rows, i)
        ids, lp = _draw(B, z, u, scale=scale, **kw)
        zn = z[few].double().cpu().numpy()
        for r in range(len(zn)):
            want, want_lp, near = oe.sample(zn[r], u[r].double().numpy(), scale=scale, **kw)
            assert 0 <= ids[r] < 30011 and (near <= 9e-9 or ids[r] == want), (i, r)
            assert near <= 9e-9 or abs(lp[r] - want_lp) <= 1e-4


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("vocab", [2, 1500, 20000])
def test_smallest_masses(B, vocab, dtype):
    """Beside one token of weight 1, all others at 2^-43.9 (rounded to the unit 2^-43) or 2^-44.1 (none): at the number 1 the last token of
    positive mass is drawn."""
    for power, want in ((-43.1, vocab - 1), (-43.5, vocab - 1), (-43.9, vocab - 1), (-44.1, 0), (-44.5, 0), (-47.0, 0), (-60.0, 0)):
        z1 = np.full((1, vocab), power * np.log(2.0))  # (fp16 has steps of 2^-6 there, 0.02 in base 2)
        z1[0, 0] = 0.0
        z = _put(z1, dtype)
        u = torch.ones(1, 2)
        for kw in (dict(), dict(min_p=1e-14), dict(top_k=vocab - 1) if vocab > 2 else dict()):
            ids, _ = _draw(B, z, u, **kw)
            assert ids[0] == (min(want, vocab - 2) if "top_k" in kw else want), (power, kw)


@pytest.mark.parametrize("third", [False, True])
@pytest.mark.parametrize("scale", [1.0, 1e-38])
def test_masses_are_within_the_headers_bound(B, scale, third):
    """Two tokens of weights 1 and w: at a share of 1 / (1 + w') the second is kept for a mass above w', so that shares on both sides of
    the bound show whether the mass lies within it.  Half of the logits are those whose restated mass is off by the most."""
    scale = float(np.float32(scale))
    rng = np.random.default_rng(4)
    x = (-rng.uniform(0.01, min(10.0, 3.3e38 * scale), 200000) / scale).astype(np.float32)
    exact, _, _ = weight(x, 0.0, scale)
    w = np.exp(x.astype(np.longdouble) * np.longdouble(scale))
    off = np.abs(exact * np.longdouble(UNIT) / w - 1)
    worst = np.argsort(-off.astype(np.float64))[:60]
    u = torch.tensor([[0.0, 1.0 - 2.0 ** -24]]).cuda()
    ids = torch.empty(1, dtype=torch.int32, device="cuda")
    for i in [*worst, *range(60)]:
        z = torch.tensor([[0.0, x[i], -np.inf][:3 if third else 2]], device="cuda")
        for sign, kept in ((1, 0), (-1, 1)):
            edge = w[i] * (1 + sign * np.longdouble(bound())) + sign * UNIT / 2
            p = float(1 / (1 + edge)) * (1 - sign * 2.0 ** -51)
            B.sgd_kernel_sample(z, u, ids, top_k=2 if third else 0, top_p=p, scale=scale)
            assert int(ids) == kept, (float(x[i]), sign)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("vocab", [700, 5000, 40000])
def test_cuts_among_equal_logits(B, vocab, dtype):
    """Shares that fall between two tokens of equal weight: the cut goes by the token."""
    z = np.zeros((8, vocab))
    z[4:] = -2.5
    z = _put(z, dtype)
    for i, kw in enumerate([dict(top_p=0.37), dict(top_p=0.9), dict(min_p=1.0, top_p=0.7), dict(top_k=600, top_p=0.61),
                            dict(min_p=0.3, top_p=0.93, top_k=499)]):
        k = min(kw.get("top_k", vocab), vocab)
        n = round(kw["top_p"] * k)  # the share of n tokens and 0.4 of another: n + 1 are kept
        kw["top_p"] = (n + 0.4) / k
        mask, near = oe.kept(z[0].double().cpu().numpy(), **kw)
        assert mask.sum() == n + 1 and mask[:n + 1].all() and near > 9e-9
        u = _numbers(8, i)
        u[0] = u[4] = 1.0 - 2.0 ** -24  # the last one that is kept
        ids, lp = _draw(B, z, u, **kw)
        assert ids[0] == n and ids[4] == n
        far = 0
        for r in range(8):
            want, _, near = oe.sample(z[r].double().cpu().numpy(), u[r].double().numpy(), **kw)
            if near > 9e-9:
                far += 1
                assert ids[r] == want
        assert far >= 7
