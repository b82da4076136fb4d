"""sgd_kernel_sample on the GPU, against oracle/ends.py in float64 on the same logits and numbers.

The drawn token has to be the oracle's, unless the oracle's draw is within NEAR of another token: a weight is off by the
error of its exponent's fraction e (at most 0.011, off by 4 roundings of 2^-24 / 2: 2^-29.5) and half a unit of 2^-43, so
that masses of up to 2^17 tokens, compared relative to a mass of at least 1, are off by 2^-29.5 + 2^17 2^-44 = 9e-9.

ln p: the sum's tolerance of test_gpu_tokens.py (186 u; u = 2^-24) and 4 u of |x - m| and of ln s.
"""
import math

import numpy as np
import pytest
import torch

from oracle import ends as oe

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
NEAR = 9e-9
DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
INF = math.inf


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2609_29505_gb300 import binding, build
    build.build()
    binding.lib()
    return binding


def _put(z, dtype, pad=0, offset=0):
    """A [rows, vocab] view on the device: `pad` columns between rows, `offset` elements into its buffer, and what lies
    around the rows larger than all of them."""
    rows, vocab = z.shape
    buf = torch.full((offset + rows * (vocab + pad) + 16,), 3e4, dtype=DT[dtype], device="cuda")
    v = buf[offset:offset + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]
    v.copy_(torch.from_numpy(z))
    return v


def _logits(rows, vocab, seed, peaks=True):
    rng = np.random.default_rng(seed)
    z = 2.0 * rng.standard_normal((rows, vocab))
    if peaks:
        for _ in range(min(20, vocab)):
            z[np.arange(rows), rng.integers(0, vocab, rows)] = 4 + 8 * rng.random(rows)
    return z


def _numbers(rows, seed):
    u = torch.rand(rows, 2, generator=torch.Generator().manual_seed(seed))
    return u


def _draw(B, z, u, **kw):
    rows = z.shape[0]
    ids = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    lp = torch.full((rows,), 77.0, device="cuda")
    B.sgd_kernel_sample(z, u.cuda(), ids, logprobs=lp, **kw)
    assert B.sgd_kernel_status() == 0
    return ids.cpu().numpy(), lp.cpu().numpy()


def _check(got, z, u, some=True, **kw):
    """Every row's token and ln p; of several rows most must be far from a border (`some`): with top_p 0.999 the tokens at the cut have
    about 1e-7 of the mass each, so that a border is within NEAR of one row in five (2 NEAR / 1e-7); half of the rows, and none
    of fewer than eight, leaves room for that."""
    ids, lp = got
    z, u = z.double().cpu().numpy(), u.double().numpy()
    far = 0
    for r in range(len(z)):
        want, want_lp, near = oe.sample(z[r], u[r], **kw)
        if near > NEAR:
            assert ids[r] == want, (r, ids[r], want, near)
            far += 1
        assert 0 <= ids[r] < z.shape[1]
        x = z[r] * float(np.float32(kw.get("scale", 1.0)))
        if not np.isfinite(want_lp):
            assert np.array_equal(lp[r], want_lp, equal_nan=True)
            continue
        m = x.max()
        ln_s = np.log(np.exp(x - m).sum())
        want_lp = x[ids[r]] - m - ln_s
        assert abs(lp[r] - want_lp) <= 186 * U + 4 * U * (abs(x[ids[r]] - m) + abs(ln_s)), (r, lp[r], want_lp)
    assert not some or len(z) < 8 or far * 2 >= len(z)


SIZES = [(1, 1), (3, 2), (5, 8), (4, 65), (3, 511), (3, 512), (3, 513), (9, 1000), (3, 1024), (2, 1025), (200, 1000), (9, 2047), (700, 900), (5, 8192), (5, 8193), (1, 4099),
         (7, 16385), (3, 32003), (1, 126464), (3, 126464), (20, 126464), (160, 20011)]
FILTERS = [dict(), dict(top_k=1), dict(top_k=50), dict(top_p=0.9), dict(min_p=0.05), dict(top_k=40, top_p=0.8, min_p=0.01),
           dict(top_p=0.95, min_p=0.002), dict(top_k=700), dict(top_k=700, top_p=0.97), dict(top_k=3000, top_p=0.99), dict(min_p=1e-4),
           dict(top_p=0.999)]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_draws(B, rows, vocab, dtype):
    z = _put(_logits(rows, vocab, rows + vocab), dtype)
    for i, kw in enumerate(FILTERS if vocab < 100000 or rows == 3 else FILTERS[:6]):
        u = _numbers(rows, i)
        _check(_draw(B, z, u, **kw), z, u, **kw)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("scale", [0.3, 1.25, 3.0])
def test_broad_rows(B, scale, dtype):
    """No peaks: a cut by mass leaves tens of thousands of tokens."""
    z = _put(_logits(6, 60001, 3, peaks=False), dtype)
    for i, kw in enumerate(FILTERS):
        u = _numbers(6, 10 + i)
        _check(_draw(B, z, u, scale=scale, **kw), z, u, scale=scale, **kw)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (3, 5), (8, 8), (13, 2)])
@pytest.mark.parametrize("vocab", [5, 1000, 20011])
def test_rows_at_any_address(B, vocab, pad, offset, dtype):
    z = _put(_logits(6, vocab, 5), dtype, pad, offset)
    for i, kw in enumerate(FILTERS[:7]):
        u = _numbers(6, i)
        _check(_draw(B, z, u, **kw), z, u, **kw)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("vocab", [700, 5000, 40000])
def test_equal_logits(B, vocab, dtype):
    """All equal, two values, few values: what is cut among equal ones goes by the token."""
    rng = np.random.default_rng(vocab)
    z = np.zeros((6, vocab))
    z[2] = z[3] = rng.integers(0, 2, vocab)
    z[4] = z[5] = rng.integers(-3, 4, vocab) * 0.5
    z = _put(z, dtype)
    for i, kw in enumerate([dict(), dict(top_k=3), dict(top_k=600), dict(top_k=4321), dict(top_p=0.37), dict(top_p=0.9), dict(min_p=0.5),
                            dict(min_p=1.0, top_p=0.7), dict(top_k=2500, top_p=0.61), dict(min_p=0.3, top_p=0.93, top_k=1900)]):
        u = _numbers(6, i)
        # (equal weights: cumulative masses are multiples of one number, and a border may be hit on the spot)
        _check(_draw(B, z, u, **kw), z, u, some=False, **kw)


def test_every_token_of_a_cut_can_be_drawn(B):
    """A grid of numbers over one row: the tokens that come out are those that may be drawn, each by its share."""
    vocab, n = 1300, 64
    z1 = np.round(_logits(1, vocab, 8, peaks=False), 1)
    grid = (torch.arange(n) + 0.5) / n
    u = torch.stack([grid.repeat_interleave(n), grid.repeat(n)], 1)
    for kw in (dict(), dict(top_k=9), dict(top_p=0.4), dict(min_p=0.2)):
        z = _put(z1, "f32").expand(n * n, vocab).contiguous()
        ids, _ = _draw(B, z, u, **kw)
        row = z[0].double().cpu().numpy()
        w = oe.weights(row) * oe.kept(row, **kw)[0]
        count = np.bincount(ids, minlength=vocab) / n ** 2
        assert (count[w == 0] == 0).all()
        assert np.abs(count - w / w.sum()).max() <= 2.0 / n


@pytest.mark.parametrize("vocab", [3000, 20000, 100000])
@pytest.mark.parametrize("rows", [1, 9, 200])
def test_filters_that_leave_many_tokens(B, rows, vocab):
    """A min-p that leaves more than the list holds, with a top-k and without; a top-k of most of the tokens; flat rows, whose cut
    by mass is among tens of thousands of nearly equal tokens."""
    rng = np.random.default_rng(vocab + rows)
    z1 = np.where(np.arange(rows)[:, None] % 2 == 0, 0.3, 1.0) * rng.standard_normal((rows, vocab))
    for dtype in ("bf16", "f32"):
        z = _put(z1, dtype)
        few = slice(0, min(rows, 9))
        for i, kw in enumerate([dict(min_p=0.02), dict(min_p=0.01, top_k=40), dict(min_p=0.01, top_k=2000, top_p=0.8), dict(min_p=0.001, top_p=0.9),
                                dict(top_k=vocab - 7), dict(top_k=vocab // 2, top_p=0.7), dict(top_p=0.3), dict(top_p=0.97), dict(top_k=5000)]):
            u = _numbers(rows, 20 + i)
            ids, lp = _draw(B, z, u, **kw)
            _check((ids[few], lp[few]), z[few], u[few], **kw)


@pytest.mark.parametrize("kw", [dict(), dict(top_k=50), dict(top_p=0.9), dict(min_p=0.05)])
def test_numbers_at_the_ends_and_outside(B, kw):
    z = _put(_logits(8, 3001, 4), "f16")
    u = torch.tensor([[0.0, 0.0], [1.0 - 2.0 ** -24] * 2, [1.0, 1.0], [-3.0, 0.5], [0.5, 7.0], [math.nan, math.nan], [INF, -INF], [1e-45, 1e-45]])
    ids, lp = _draw(B, z, u, **kw)
    zn = z.double().cpu().numpy()
    for r in range(8):
        want, _, near = oe.sample(zn[r], u[r].double().numpy(), **kw)
        assert ids[r] == want or near <= NEAR


def test_numbers_at_a_border_of_blocks(B):
    """u0 as near as fp32 has it to the border of two blocks: there the masses are taken anew."""
    rows, vocab = 12, 30000
    z = _put(_logits(rows, vocab, 6, peaks=False), "f32")
    zn = z.double().cpu().numpy()
    u = _numbers(rows, 1)
    for r in range(rows):
        w = np.pad(oe.weights(zn[r]), (0, -vocab % 512)).reshape(-1, 512).sum(1)
        u[r, 0] = float(np.float32((np.cumsum(w) / w.sum())[3 + 4 * r]))
    _check(_draw(B, z, u), z, u, some=False)
    # (fp32 numbers above 1/2 are 6e-8 apart: two thirds of those that are nearest to a border are farther from it than NEAR; half of the
    # rows' borders are above 1/2)
    assert sum(oe.sample(zn[r], u[r].double().numpy())[2] > NEAR for r in range(rows)) >= rows // 4


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("vocab", [3, 1000, 40001])
def test_masks_and_rows_without_a_distribution(B, vocab, dtype):
    z1 = _logits(9, vocab, 7)
    low = float(torch.finfo(DT[dtype]).min)
    z1[0] = -INF
    z1[1] = -INF
    z1[1, vocab // 2] = -3.0           # one token is left
    z1[2, ::2] = -INF
    z1[3, vocab // 2] = math.nan
    z1[4, vocab - 1] = INF
    z1[5, :] = low                     # masked by the type's lowest value, all of them
    z1[6, 1:] = low
    z1[7, : vocab // 2] = low
    z1[8] = -INF
    z1[8, vocab // 3] = math.nan
    z = _put(z1, dtype)
    for i, kw in enumerate([dict(), dict(top_k=2), dict(top_p=0.9), dict(min_p=0.1), dict(top_k=2000, top_p=0.5, min_p=0.0001)]):
        u = _numbers(9, i)
        ids, lp = _draw(B, z, u, **kw)
        _check((ids, lp), z, u, some=False, **kw)
        assert ids[0] == 0 and lp[0] == -INF and ids[1] == vocab // 2 and lp[1] == 0.0
        assert np.isnan(lp[3]) and np.isnan(lp[4]) and np.isnan(lp[8]) and ids[4] == vocab - 1 and ids[8] == 0
        assert ids[6] == 0


@pytest.mark.parametrize("scale", [1e-38, 1e-6, 1e6, 2e38])
def test_scales(B, scale):
    z = _put(_logits(5, 5000, 9), "f32")
    for i, kw in enumerate([dict(), dict(top_k=5), dict(top_p=0.7), dict(min_p=0.5)]):
        u = _numbers(5, i)
        ids, _ = _draw(B, z, u, scale=scale, **kw)
        zn = z.double().cpu().numpy()
        for r in range(5):
            want, _, near = oe.sample(zn[r], u[r].double().numpy(), scale=scale, **kw)
            # (equal weights at the smallest scales: borders are hit on the spot)
            assert ids[r] == want or near <= NEAR


def test_magnitudes(B):
    """Logits far from 0, where a difference of two is not exact in fp32, and of the largest values."""
    rng = np.random.default_rng(1)
    z1 = rng.standard_normal((4, 4000))
    z1[0] += 1e4
    z1[1] *= 1e30
    z1[2] = np.where(rng.random(4000) < 0.5, 3.4e38, -3.4e38)
    z1[3] -= 3e5
    z = _put(z1, "f32")
    for i, kw in enumerate([dict(), dict(top_k=30), dict(top_p=0.8), dict(min_p=0.01)]):
        u = _numbers(4, i)
        _check(_draw(B, z, u, **kw), z, u, some=False, **kw)


def test_rows_that_are_not_asked_for(B):
    z = _put(_logits(40, 9000, 2), "f16")
    u = _numbers(40, 3)
    row_ids = torch.arange(40, dtype=torch.int32, device="cuda") % 3
    for kw in (dict(), dict(top_p=0.9)):
        ids, lp = _draw(B, z, u, row_ids=row_ids, row_id=1, **kw)
        all_ids, all_lp = _draw(B, z, u, **kw)
        on = (row_ids == 1).cpu().numpy()
        assert np.array_equal(ids[on], all_ids[on]) and np.array_equal(lp[on], all_lp[on])
        assert (ids[~on] == -7).all() and (lp[~on] == 77).all()


def test_without_logprobs_the_token_is_the_same(B):
    z = _put(_logits(30, 50000, 12), "bf16")
    for i, kw in enumerate(FILTERS):
        u = _numbers(30, i).cuda()
        ids, other = torch.empty(30, dtype=torch.int32, device="cuda"), torch.empty(30, dtype=torch.int32, device="cuda")
        B.sgd_kernel_sample(z, u, ids, logprobs=torch.empty(30, device="cuda"), **kw)
        B.sgd_kernel_sample(z, u, other, **kw)
        assert torch.equal(ids, other)


def test_streams_and_graphs(B):
    z = _put(_logits(300, 30000, 4), "f16")
    u = _numbers(300, 2).cuda()
    kw = dict(top_p=0.9, scale=1.25)
    want, want_lp = torch.empty(300, dtype=torch.int32, device="cuda"), torch.empty(300, device="cuda")
    B.sgd_kernel_sample(z, u, want, logprobs=want_lp, **kw)
    torch.cuda.synchronize()
    outs = [(torch.empty_like(want), torch.empty_like(want_lp)) for _ in range(4)]
    streams = [torch.cuda.Stream() for _ in outs]
    for s, (i, p) in zip(streams, outs):
        B.sgd_kernel_sample(z, u, i, logprobs=p, stream=s, **kw)
    torch.cuda.synchronize()
    assert all(torch.equal(i, want) and torch.equal(p, want_lp) for i, p in outs)
    ids = torch.empty_like(want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.sgd_kernel_sample(z, u, ids, **kw)
    for seed in (5, 6):
        u.copy_(_numbers(300, seed))
        g.replay()
        B.sgd_kernel_sample(z, u, want, **kw)
        assert torch.equal(ids, want)


def test_binding_refuses(B):
    z, u = torch.zeros(3, 8, device="cuda"), torch.rand(3, 2, device="cuda")
    ids = torch.zeros(3, dtype=torch.int32, device="cuda")
    for kw in (dict(uniforms=u.double()), dict(ids=ids.long()), dict(logprobs=torch.zeros(3, device="cuda").half())):
        with pytest.raises(TypeError):
            B.sgd_kernel_sample(z, **{**dict(uniforms=u, ids=ids), **kw})
    for kw in (dict(uniforms=u[:2]), dict(uniforms=u.t().contiguous().t()), dict(ids=ids[:2]), dict(uniforms=u.cpu()), dict(top_k=2 ** 31)):
        with pytest.raises(ValueError):
            B.sgd_kernel_sample(z, **{**dict(uniforms=u, ids=ids), **kw})
    for kw in (dict(top_k=-1), dict(top_p=0.0), dict(top_p=1.5), dict(min_p=-1.0), dict(min_p=2.0), dict(scale=0.0)):
        with pytest.raises(B.SgdError):
            B.sgd_kernel_sample(z, u, ids, **kw)


@pytest.mark.parametrize("dtype,rows,vocab,pad", [("f16", 280, 126464, 0), ("bf16", 281, 126461, 3), ("f32", 141, 126464, 0), ("bf16", 700, 50000, 8),
                                                  ("f32", 300, 60000, 4), ("f16", 400, 100003, 5)])
def test_many_long_rows(B, dtype, rows, vocab, pad):
    """More of them than run at once; some without a distribution, some numbers next to a block's border, rows that are not asked for."""
    rng = np.random.default_rng(rows)
    z1 = (1.0 + np.arange(rows) % 3)[:, None] * rng.standard_normal((rows, vocab), dtype=np.float32)
    z1[np.arange(rows), rng.integers(0, vocab, rows)] = 9.0
    z1[3] = -INF
    z1[5, 77] = math.nan
    z1[6, vocab - 1] = INF
    z1[7, 1:] = -INF
    z = _put(z1, dtype, pad)
    u = _numbers(rows, 1)
    zn = z.float().cpu().numpy()
    for r in range(8, 20):  # next to a border: masses are taken anew
        w = oe.weights(zn[r])
        u[r, 0] = float(np.float32((np.cumsum(np.pad(w, (0, -vocab % 512)).reshape(-1, 512).sum(1)) / w.sum())[r * 4]))
    on = torch.ones(rows, dtype=torch.int32, device="cuda")
    on[::5] = 0
    for ids in (None, on):
        got, lp = _draw(B, z, u, **({} if ids is None else dict(row_ids=ids, row_id=1)))
        keep = np.ones(rows, bool) if ids is None else on.cpu().numpy() == 1
        assert (got[~keep] == -7).all() and (lp[~keep] == 77).all()
        look = [r for r in range(rows) if keep[r] and (r < 24 or r % 9 == 0)]
        _check((got[look], lp[look]), z[look], u[look], some=False)
        # the log-probability of every token is that of the scoring kernel
        want = torch.empty(rows, 1, device="cuda")
        B.sgd_kernel_logprobs(z, tokens=torch.from_numpy(got).cuda()[:, None], token_logprobs=want)
        want = want[:, 0].cpu().numpy()
        fine = keep & np.isfinite(lp) & np.isfinite(want)
        assert np.abs(lp[fine] - want[fine]).max() <= 2 * (186 * U + 4 * U * 80) and fine.sum() >= keep.sum() - 3


def test_many_long_rows_without_a_distribution(B):
    """Each takes the first token of its order."""
    rows, vocab = 3000, 50000
    z = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    z[:, 100] = 1.0
    z[:, 4] = math.nan
    ids = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    lp = torch.zeros(rows, device="cuda")
    B.sgd_kernel_sample(z, torch.rand(rows, 2, device="cuda"), ids, logprobs=lp)
    assert (ids == 100).all() and lp.isnan().all() and B.sgd_kernel_status() == 0


def test_many_long_rows_streams_and_graphs(B):
    z = _put(_logits(300, 126464, 3).astype(np.float32), "f16")
    u = _numbers(300, 4).cuda()
    want, want_lp = torch.empty(300, dtype=torch.int32, device="cuda"), torch.empty(300, device="cuda")
    B.sgd_kernel_sample(z, u, want, logprobs=want_lp)
    torch.cuda.synchronize()
    outs = [(torch.empty_like(want), torch.empty_like(want_lp)) for _ in range(3)]
    for s, (i, p) in zip([torch.cuda.Stream() for _ in outs], outs):
        B.sgd_kernel_sample(z, u, i, logprobs=p, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(i, want) and torch.equal(p, want_lp) for i, p in outs)
    ids = torch.empty_like(want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.sgd_kernel_sample(z, u, ids)
    g.replay()
    assert torch.equal(ids, want)


@pytest.mark.parametrize("dtype,vocab", [("f16", 3 << 19), ("f32", 3 << 18), ("bf16", 1000003)])
def test_longest_rows(B, dtype, vocab):
    """Rows of 3 MiB, by a cluster and by CTAs of their own; the same rows at odd addresses."""
    rng = np.random.default_rng(2)
    z1 = (2.0 * rng.standard_normal((3, vocab), dtype=np.float32))
    z1[:, rng.integers(0, vocab, 30)] = 10.0 + 4.0 * rng.random(30, dtype=np.float32)
    z1[2] *= 0.1
    u = _numbers(3, 8)
    for offset in (0, 1):
        z = _put(z1, dtype, offset=offset)
        for kw in (dict(), dict(top_k=50), dict(top_k=3000), dict(top_p=0.9), dict(min_p=0.01), dict(top_k=40, top_p=0.9, min_p=0.02)):
            # (NEAR is for 2^17 tokens; half a unit of 2^-43 each, 1.6 million are off by 9e-8)
            ids, _ = _draw(B, z, u, **kw)
            for r in range(3):
                want, _, near = oe.sample(z[r].double().cpu().numpy(), u[r].double().numpy(), **kw)
                assert ids[r] == want or near <= 12 * NEAR, (kw, r, ids[r], want, near)
    many = z[:1].expand(700, vocab).contiguous()
    got, _ = _draw(B, many, u[:1].expand(700, 2).contiguous(), top_p=0.5)
    assert (got == got[0]).all()


@pytest.mark.parametrize("kw", [dict(top_p=1e-300), dict(top_p=1e-12), dict(top_p=1 - 2 ** -53), dict(top_p=1 - 1e-9), dict(min_p=1e-300), dict(min_p=1e-12, top_p=0.5),
                                dict(top_k=2 ** 31 - 1), dict(top_k=1, top_p=0.5, min_p=1.0)])
@pytest.mark.parametrize("rows,vocab", [(3, 900), (3, 9000), (2, 50000), (200, 50000)])
def test_filters_at_their_ends(B, rows, vocab, kw):
    z = _put(_logits(rows, vocab, 17), "f32")
    u = _numbers(rows, 5)
    few = slice(0, min(rows, 9))
    ids, lp = _draw(B, z, u, **kw)
    _check((ids[few], lp[few]), z[few], u[few], some=False, **kw)
