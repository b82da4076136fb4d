"""The masses that sgd_kernel_sample compares, restated in fp32 from the kernel's source: within the bound that the public header gives
(no GPU needed)."""
import os
import re

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, F64, F80 = np.float32, np.float64, np.longdouble
UNIT = 2.0 ** -43  # of the largest weight


def bound():
    """The header's: a mass is within 2^-n of its value and half a unit."""
    text = open(os.path.join(ROOT, "include", "sgd_kernels.h")).read()
    assert "multiples of 2^-43 of the largest weight" in " ".join(text.replace(" * ", " ").split())
    return 2.0 ** -int(re.search(r"each within 2\^-(\d+) of its\s+(?:\* )?value", text).group(1))


def table():
    src = open(os.path.join(ROOT, "paper_2609_29505_gb300", "csrc", "sample_kernel.cuh")).read()
    return np.array([int(x, 16) for x in re.findall(r"0x([0-9A-F]{16})ull", src)], np.uint64)


def _fma(a, b, c):
    # (the product is exact in float64; two roundings of the sum differ from one by a bit of float64 near a tie)
    return (a.astype(F64) * F64(b) + np.asarray(c, F64)).astype(F32)


def weight(z, m, scale):
    """As weight() of sample_kernel.cuh: the exact multiple of the unit before it is rounded to a whole one, and that."""
    f = F32(2.0 ** -64 if scale < 2.0 ** -64 else 1.0)
    c64 = F64(F32(scale) / f) * 1.4426950408889634
    c = F32(c64)
    c_lo = F32(c64 - F64(c))
    z, m = z.astype(F32), F32(m)
    mf = F32(m * f)
    d = _fma(z, f, -mf)
    t = d * c
    back = _fma(-z, f, d)
    dl = _fma(z, f, back - d) + (-mf - back)
    tl = _fma(d, c, -t) + (d.astype(F64) * F64(c_lo) + (dl * c).astype(F64)).astype(F32)
    magic = F32(393216.0)
    y = t + magic
    k = y.view(np.int32) - magic.view(np.int32)
    g = (t - (y - magic)) + tl
    p = F32(0.009618129)
    for a in (0.05550411, 0.24022651, 0.6931472):
        p = (g.astype(F64) * np.asarray(p, F64) + F64(F32(a))).astype(F32)
    none = ~(t > -48.0)
    e = np.where(none, F32(0), g * p)
    base = table()[k & 31]
    w = base + ((base >> np.uint64(32)).astype(np.int64) * np.rint(e.astype(F64) * 2.0 ** 32).astype(np.int64)).astype(np.uint64)
    shift = 19 - (k >> 5)
    none |= shift > 63
    exact = np.where(none, 0, w.astype(F80) * np.exp2(-shift.astype(F80)))
    half = np.uint64(1) << np.clip(shift - 1, 0, 62).astype(np.uint64)
    return exact, np.where(none, np.uint64(0), (w + half) >> np.clip(shift, 0, 63).astype(np.uint64)), t


def test_table_is_the_powers_of_two():
    want = np.exp2(np.arange(32).astype(F80) / 32 + 62)
    assert len(table()) == 32 and (np.abs(table().astype(F80) - want) <= 1).all()


@pytest.mark.parametrize("scale", [1.0, 1.25, 0.3, 3.0, 1e-3, 64.0, 2.0 ** -65, 1e-38, 1e-41])
def test_masses_are_within_the_headers_bound(scale):
    """Four roundings of the fraction's order (g, the polynomial's last sum and product, the exponent's two parts): the largest error is some
    3.8 2^-31, of one logit in some hundred thousand."""
    scale = float(F32(scale))
    rng = np.random.default_rng(1)
    spread = min(2.0 / scale, 1e37)
    z = (spread * rng.standard_normal(400000)).astype(F32)
    z[:200000] = np.where(rng.random(200000) < 0.5, z[:200000], (-spread * 30 * rng.random(200000)).astype(F32))
    m = z.max()
    exact, whole, t = weight(z, m, scale)
    true = np.exp((z.astype(F80) - F80(m)) * F80(F32(scale)))
    units = true / F80(UNIT)
    big = units > 0.5
    assert (np.abs(exact - units)[big] <= bound() * units[big]).all()
    assert (np.abs(whole.astype(F80) - units)[big] <= bound() * units[big] + 0.5).all()
    assert (whole[units < 0.4999] == 0).all() and whole.max() == 2 ** 43
