"""Operators on a token model's logits on the GPU, against oracle/tokens.py in float64 on the same inputs.

Tolerances, from the kernels' arithmetic (u = 2^-24, the rounding of fp32):
  exponent y = c x - R in base 2, |y| ln 2 = scale (m - x): c = scale log2(e) is off by 2 u, y by u, and
    ex2.approx by 2^-22 = 4 u, so that a term 2^y is off by (4 + 3 |y| ln 2) u; terms with |y| ln 2 > 12 add
    less than e^-12 each to a sum of at least 1, so that a sum of up to 2^20 terms of any sizes is off by
    (4 + 3 * 14) u from that, and by 140 u from being added up (at most 128 in a row in a thread, then
    a tree): 186 u < 1.2e-5 relative, SUM below.
  ln p = (x - m) scale - ln s: SUM, and 4 u of |x - m| scale and of ln s.
  gradient: p is off by SUM + (4 + 3 |ln p|) u; the tail's p (1 - q_T / p_T) by twice SUM of each part, and by what
    q_T = 1 - Q is off: expf is within one step, 2 u q_i, the sum is in fp64, so that q_T is off by 2 u Q and
    the token's gradient by (p / p_T) 2 u Q;  then half a step of the output's type (and half of its
    smallest subnormal).
  loss: sum of q (ln q - ln p) with ln p off by SUM and q by 2 u (expf), which moves L by 2 u q |ln q - ln p|;
    q_T (ln q_T - ln p_T) by 2 SUM q_T, and q_T itself by Q 2 u.
"""
import math

import numpy as np
import pytest
import torch

from oracle import tokens as ot

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
SUM = 186 * U
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


def _logits(rows, vocab, dtype, seed, pad=0, offset=0, peaks=True):
    """A [rows, vocab] view on the device: `pad` columns between rows, `offset` elements into its buffer.
    What lies around the rows is larger than all of them."""
    rng = np.random.default_rng(seed)
    z = 2.0 * rng.standard_normal((rows, vocab))
    if peaks:
        for _ in range(min(20, vocab)):
            z[np.arange(rows), rng.integers(0, vocab, rows)] = 4 + 8 * rng.random(rows)
    buf = torch.full((offset + rows * (vocab + pad) + 16,), 3e4, dtype=DT[dtype], device="cuda")
    v = buf[offset:offset + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]
    v.copy_(torch.from_numpy(z))
    return v


def _np(t):
    return t.detach().double().cpu().numpy()


def _score(B, z, k=4, n=2, scale=1.0, seed=0, tokens=None, **kw):
    rows, vocab = z.shape
    k = min(k, vocab)
    g = torch.Generator().manual_seed(seed)
    if tokens is None:
        tokens = torch.randint(0, vocab, (rows, n), generator=g, dtype=torch.int32)
    tokens = tokens.cuda()
    out = dict(token_logprobs=torch.full(tokens.shape, 77.0, device="cuda"), entropy=torch.full((rows,), 77.0, device="cuda"))
    if k:
        out["top_ids"] = torch.full((rows, k), -7, dtype=torch.int32, device="cuda")
        out["top_logprobs"] = torch.full((rows, k), 77.0, device="cuda")
    B.sgd_kernel_logprobs(z, tokens=tokens, scale=scale, **out, **kw)
    assert B.sgd_kernel_status() == 0
    return {n: v.cpu().numpy() for n, v in out.items()}, tokens.cpu().numpy()


def _near(got, want, tol):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf])
    ok = np.isfinite(want)
    assert np.isfinite(got[ok]).all()
    err = np.abs(got[ok] - want[ok])
    tol = np.broadcast_to(tol, want.shape)[ok]
    assert (err <= tol).all(), f"worst error {np.max(err / tol):.2f} of its tolerance"


def _check_score(got, tokens, z, k, scale=1.0):
    z = _np(z)
    lp = ot.log_softmax(z, scale)
    with np.errstate(invalid="ignore"):
        big = np.nanmax(np.where(np.isfinite(lp), lp, -INF), axis=1, keepdims=True)  # ln of the largest p = -ln s
    big = np.where(np.isfinite(big), big, 0.0)
    tol = lambda v: SUM + 4 * U * (np.abs(np.where(np.isfinite(v), v, 0)) + 2 * np.abs(big))  # noqa: E731
    want = ot.token_logprobs(lp, tokens)
    _near(got["token_logprobs"], want, tol(want))
    # H = ln s - ln 2 t / s: SUM in s, in t (whose terms |y| 2^y add up to |t|) and the roundings
    H = ot.entropy(lp)
    _near(got["entropy"], H, SUM * (1 + 2 * (np.abs(H) + np.abs(big[:, 0]))))
    if k:
        k = min(k, z.shape[1])
        ids = ot.top(z, k)
        assert np.array_equal(got["top_ids"], ids)
        want = np.take_along_axis(lp, ids, 1)
        _near(got["top_logprobs"], want, tol(want))


# one row and few (large clusters), and more; 16-byte boundaries and every tail; slices without an element
SIZES = [(1, 1), (3, 2), (2, 7), (5, 8), (3, 9), (2, 63), (4, 65), (3, 255), (2, 1000), (200, 1000), (3, 1001), (1, 4099),
         (2, 8191), (7, 16385), (3, 32003), (1, 126464), (3, 126464), (40, 126464)]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", SIZES)
@pytest.mark.parametrize("k", [0, 1, 8])
def test_logprobs(B, rows, vocab, dtype, k):
    z = _logits(rows, vocab, dtype, rows + vocab)
    got, tokens = _score(B, z, k=k, n=3)
    _check_score(got, tokens, z, k)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (3, 5), (8, 8), (13, 2), (5, 7)])
@pytest.mark.parametrize("vocab", [5, 1000, 20011])
def test_logprobs_of_rows_at_any_address(B, vocab, pad, offset, dtype):
    z = _logits(6, vocab, dtype, 5, pad=pad, offset=offset)
    for k in (1, 5):
        got, tokens = _score(B, z, k=k, scale=1.25)
        _check_score(got, tokens, z, k, 1.25)


@pytest.mark.parametrize("k", [2, 17, 32, 33, 63, 64])
@pytest.mark.parametrize("vocab", [64, 999, 70001])
def test_long_lists(B, vocab, k):
    z = _logits(9, vocab, "f16", k)
    got, tokens = _score(B, z, k=k)
    _check_score(got, tokens, z, k)


def _rows_that_are_hard(vocab):
    """Orders, ties and masks: one row each."""
    rng = np.random.default_rng(3)
    up = np.linspace(-3, 12, vocab)
    rows = [up, up[::-1], np.zeros(vocab), np.full(vocab, -65504.0), np.full(vocab, -INF)]
    z = np.full(vocab, -INF)
    z[vocab // 2] = -3.0
    rows.append(z)  # one token left
    z = np.full(vocab, -INF)
    z[rng.permutation(vocab)[:max(1, vocab // 40)]] = 1.5
    rows.append(z)  # a few, all equal
    rows.append(np.where(rng.random(vocab) < 0.5, 0.0, -0.0))  # zeros of both signs
    rows.append(rng.integers(-2, 3, vocab).astype(float))  # five values
    rows.append(np.where(rng.random(vocab) < 0.7, -INF, rng.standard_normal(vocab)))
    z = rng.standard_normal(vocab)
    z[:min(vocab, 64)] = 9.0 + np.arange(min(vocab, 64)) / 64.0  # the largest side by side
    rows.append(z)
    z = rng.standard_normal(vocab)
    z[-1], z[0] = 60000.0, 59968.0  # far above the rest
    rows.append(z)
    rows.append(np.where(np.arange(vocab) % 2 == 0, 65504.0, -65504.0))
    z = np.full(vocab, 2.0)
    z[rng.permutation(vocab)[:min(vocab, 30)]] = 5.0 + np.arange(min(vocab, 30)) // 3  # a few above many equal ones
    rows.append(z)
    z = np.full(vocab, -INF)
    z[rng.permutation(vocab)[:min(vocab, 30)]] = rng.standard_normal(min(vocab, 30))  # a few tokens allowed
    rows.append(z)
    return np.stack(rows)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("vocab", [3, 300, 5003, 126464])
@pytest.mark.parametrize("k", [1, 3, 40, 64])
def test_hard_rows(B, vocab, k, dtype):
    z = torch.from_numpy(_rows_that_are_hard(vocab)).to(DT[dtype]).cuda()
    got, tokens = _score(B, z, k=k)
    _check_score(got, tokens, z, k)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("vocab", [9, 3001, 126464])
def test_rows_with_nan_or_infinity(B, vocab, dtype):
    z = _logits(6, vocab, dtype, 9)
    z[0, 4] = math.nan
    z[1, vocab - 1] = INF
    z[2, 0] = -INF
    z[3, :] = math.nan
    z[4, :] = -INF
    z[4, 1] = math.nan
    for k in (1, 5):
        got, tokens = _score(B, z, k=k)
        lp = ot.log_softmax(_np(z))
        for r in (0, 1, 3, 4):
            assert np.isnan(got["token_logprobs"][r]).all() and np.isnan(got["entropy"][r])
            assert np.isnan(got["top_logprobs"][r]).all()
        assert np.array_equal(got["top_ids"], ot.top(_np(z), k))
        rest = [2, 5]
        _check_score({n: v[rest] for n, v in got.items()}, tokens[rest], z[rest], k)
        assert np.isfinite(lp[5]).all()


def test_given_tokens_in_number_and_out_of_range(B):
    vocab, n = 5000, 700  # more than a CTA has threads
    z = _logits(4, vocab, "f16", 11)
    t = torch.randint(0, vocab, (4, n), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    t[:, 0], t[:, 1], t[:, 2], t[:, 3], t[:, 400] = -1, vocab, -100, 2 ** 31 - 1, t[:, 401]
    got, tokens = _score(B, z, k=0, tokens=t)
    _check_score(got, tokens, z, 0)
    assert (got["token_logprobs"][:, [0, 2]] == 0).all() and np.isnan(got["token_logprobs"][:, [1, 3]]).all()


@pytest.mark.parametrize("vocab", [700, 126464])
def test_rows_that_are_not_asked_for_stay(B, vocab):
    z = _logits(50, vocab, "f16", 12)
    ids = torch.randint(0, 3, (50,), generator=torch.Generator().manual_seed(2), dtype=torch.int32).cuda()
    z[ids != 1] = math.nan
    for k in (1, 6):
        got, tokens = _score(B, z, k=k, row_ids=ids, row_id=1)
        on = (ids == 1).cpu().numpy()
        for v in got.values():
            assert (v[~on] == (-7 if v.dtype == np.int32 else 77.0)).all()
        _check_score({n: v[on] for n, v in got.items()}, tokens[on], z[ids == 1], k)


def test_single_outputs(B):
    z = _logits(5, 3001, "bf16", 13)
    want, _ = _score(B, z, k=4)
    for name in ("entropy", "top_ids", "top_logprobs"):
        out = torch.full_like(torch.from_numpy(want[name]), 5).cuda()
        B.sgd_kernel_logprobs(z, **{name: out})
        if name == "entropy":  # no list asked for: the same numbers all the same
            assert torch.equal(out.cpu(), torch.from_numpy(want[name]))
        else:
            assert np.array_equal(out.cpu().numpy(), want[name])


@pytest.mark.parametrize("dtype,vocab", [("f16", 3 << 19), ("f32", 3 << 18), ("bf16", 1000003)])
def test_the_largest_rows(B, dtype, vocab):
    z = _logits(2, vocab, dtype, 14)
    got, tokens = _score(B, z, k=9)
    _check_score(got, tokens, z, 9)
    ids, logq = _lists(z, 9, 14)
    _distill(B, z, ids, logq)


@pytest.mark.parametrize("rows,vocab", [(70000, 49200), (70000, 8200)])
def test_more_rows_than_a_cluster_lists(B, rows, vocab):
    """Above 448 rows of a cluster, rows that are asked for or have a weight are not listed beforehand.  A block of
    rows again and again: the same outputs."""
    n = 500
    block = torch.empty(n, vocab, dtype=torch.float16, device="cuda").normal_(0, 2, generator=torch.Generator("cuda").manual_seed(3))
    z = block.repeat(rows // n, 1)
    g = torch.Generator("cuda").manual_seed(4)
    on = torch.rand(rows, device="cuda", generator=g) < 0.5
    on[1234:1234 + 7000] = False
    tokens = torch.arange(n, device="cuda").int()[:, None].repeat(rows // n, 1)
    few, _ = _score(B, block, k=3, tokens=tokens[:n])
    got, _ = _score(B, z, k=3, tokens=tokens, row_ids=on.int(), row_id=1)
    on_ = on.cpu().numpy()
    for name, v in got.items():
        want = np.tile(few[name].reshape(n, -1), (rows // n, 1))[on_]
        v = v.reshape(rows, -1)
        assert (v[~on_] == (-7 if v.dtype == np.int32 else 77.0)).all()
        if v.dtype == np.int32:
            assert np.array_equal(v[on_], want)
        else:  # (another kernel: both are off by less than SUM and the roundings)
            _near(v[on_], want, 2 * (SUM * (1 + 2 * np.abs(want)) + 64 * U))
    if vocab > 10000:
        return
    ids, logq = _lists(block, 4, 5)
    ids, logq = ids.repeat(rows // n, 1), logq.repeat(rows // n, 1)
    w = on.float() * 0.5
    loss, grad = _distill(B, z, ids, logq, weight=w, grad="bf16", check=False)
    assert (loss[~on] == 0).all() and not grad[~on].any()
    some = torch.nonzero(on)[:, 0][::1777]
    _check_rows(loss[some], grad[some], z[some], ids[some], logq[some], True, w[some])
    first = {}
    for r in torch.nonzero(on)[:, 0][:4000].tolist():  # rows of one kind agree bit for bit
        if r % n in first:
            assert torch.equal(grad[r], grad[first[r % n]]) and loss[r] == loss[first[r % n]]
        first.setdefault(r % n, r)


def test_offsets_past_32_bits(B):
    """Rows whose offset in elements, and in bytes, is above 2^32."""
    vocab, ld, rows = 1000, 1 << 29, 10
    buf = torch.empty(ld * (rows - 1) + vocab, dtype=torch.float16, device="cuda")
    z = torch.as_strided(buf, (rows, vocab), (ld, 1))
    z.copy_(_logits(rows, vocab, "f16", 15))
    got, tokens = _score(B, z, k=3)
    _check_score(got, tokens, z, 3)
    ids, logq = torch.tensor([[5, 7]] * rows, dtype=torch.int32).cuda(), torch.full((rows, 2), -1.5).cuda()
    z0 = z.clone()
    loss = torch.empty(rows, device="cuda")
    B.sgd_kernel_distill(z, ids, logq, loss, grad=z)
    _check_distill(loss, z, z0, ids, logq, 1.0, True, None)


# many long rows: they stream, and the CTAs of a cluster share a row where that fills the SMs better (152: one
# each; 153, 301: one round more); the last two are too short for that
@pytest.mark.parametrize("rows,vocab,dtype,pad,offset", [
    (152, 126464, "f16", 0, 0), (153, 126464, "f16", 0, 0), (301, 126464, "f16", 0, 0), (1100, 60001, "bf16", 0, 1),
    (400, 100003, "f16", 13, 0), (230, 50021, "f32", 0, 3), (300, 126461, "f16", 5, 2), (70, 300007, "bf16", 1, 0),
    (12, 3 << 19, "f16", 0, 0), (14, 700001, "f32", 2, 1), (1100, 16387, "f16", 5, 2), (700, 32003, "bf16", 0, 1)])
@pytest.mark.parametrize("k", [0, 1, 9, 64])
def test_logprobs_of_many_rows(B, rows, vocab, dtype, pad, offset, k):
    z = torch.empty(rows, vocab + pad, dtype=DT[dtype], device="cuda").normal_(0, 2, generator=torch.Generator("cuda").manual_seed(rows))
    buf = torch.full((offset + rows * (vocab + pad),), 3e4, dtype=DT[dtype], device="cuda")
    v = buf[offset:].view(rows, vocab + pad)
    v[:, :vocab] = z[:, :vocab]
    z = v[:, :vocab]
    z[rows // 2, vocab // 3:] = -INF
    got, tokens = _score(B, z, k=k, n=2)
    some = sorted({0, 1, rows // 2, rows - 1, *range(3, rows, max(1, rows // 5))})
    _check_score({n: x[some] for n, x in got.items()}, tokens[some], z[some], k)
    # every row, against the kernel for few rows: the same list, and statistics within the tolerance of both
    for a in range(0, rows, 8):
        few, _ = _score(B, z[a:a + 8], k=k, tokens=torch.from_numpy(tokens[a:a + 8]))
        for n in few:
            if n == "top_ids":
                assert np.array_equal(few[n], got[n][a:a + 8])
            else:
                _near(got[n][a:a + 8], few[n], 2 * (SUM * (1 + 2 * np.abs(np.where(np.isfinite(few[n]), few[n], 0))) + 64 * U))


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("k", [1, 3, 64])
def test_hard_rows_among_many(B, k, dtype):
    hard = torch.from_numpy(_rows_that_are_hard(126464)).to(DT[dtype])
    n = len(hard)
    z = hard.repeat(13, 1).cuda()
    assert z.numel() * z.element_size() >= 32 << 20
    got, tokens = _score(B, z, k=k, tokens=torch.arange(2 * n).view(n, 2).int().repeat(13, 1))
    _check_score({m: x[:n] for m, x in got.items()}, tokens[:n], hard, k)
    for x in got.values():
        x = x.reshape(13, n, -1)
        assert np.array_equal(x, np.broadcast_to(x[:1], x.shape), equal_nan=True)


@pytest.mark.parametrize("share", [0.0, 0.004, 0.5, 1.0])
@pytest.mark.parametrize("k", [1, 6])
def test_rows_that_are_not_asked_for_stay_among_many(B, k, share):
    rows, vocab = 900, 70001
    g = torch.Generator("cuda").manual_seed(4)
    z = torch.empty(rows, vocab, dtype=torch.float16, device="cuda").normal_(0, 2, generator=g)
    on = torch.rand(rows, device="cuda", generator=g) < share
    ids = torch.where(on, 5, 4).int()
    want, tokens = _score(B, z, k=k)
    z[~on] = math.nan
    got, _ = _score(B, z, k=k, row_ids=ids, row_id=5)
    on = on.cpu().numpy()
    for n, v in got.items():
        assert (v[~on] == (-7 if v.dtype == np.int32 else 77.0)).all()
        assert np.array_equal(v[on], want[n][on])


# ---------------------------------------------------------------------------
# distillation
# ---------------------------------------------------------------------------

def _lists(z, k, seed, noise=0.7, scale=1.0):
    """The k likeliest tokens of a teacher that is near the rows of z: ids and their log-probabilities."""
    x = _np(z) * scale
    x = x + noise * np.random.default_rng(seed).standard_normal(x.shape)
    lp = ot.log_softmax(x)
    ids = ot.top(x, k)
    return (torch.from_numpy(ids.astype(np.int32)).cuda(),
            torch.from_numpy(np.take_along_axis(lp, ids, 1).astype(np.float32)).cuda())


def _check_distill(loss, grad, z, ids, logq, scale, bucket, weight):
    z, ids, logq = _np(z), ids.cpu().numpy(), _np(logq)
    w = np.ones(len(z)) if weight is None else _np(weight)
    loss = _np(loss)
    for r in range(len(z)):
        L, g = ot.distill_row(z[r], ids[r], logq[r], scale, bucket, w[r])
        if w[r] == 0 or not ((ids[r] >= 0) & (ids[r] < z.shape[1])).any():
            assert loss[r] == 0 and (grad is None or not grad[r].any())
            continue
        lp = ot.log_softmax(z[r][None], scale)[0]
        p = np.exp(lp)
        q = np.zeros(len(p))
        for i, lq in zip(ids[r][::-1], logq[r][::-1]):
            if 0 <= i < len(p):
                q[i] = np.exp(lq)
        Q = q.sum()
        S = q > 0
        qt = max(0.0, 1 - Q) if bucket else 0.0
        if not bucket:
            q /= Q
        with np.errstate(divide="ignore", invalid="ignore"):
            pull = np.where(S, q * np.abs(np.log(q) - lp), 0.0).sum()
            pt = np.where(S, 0.0, p).sum()
            ratio = qt / pt if pt > 0 else 0.0
        tol = SUM * (q.sum() + 2 * qt) + 2 * U * pull
        if qt > 0 and pt > 0:  # 1 - Q: its rounding moves q_T
            tol += 4 * U * Q * abs(np.log(qt) - np.log(pt) + 1)
        _near(loss[r], L, abs(w[r]) * tol + U * abs(L))
        if grad is not None:
            G = grad.dtype
            half, least = torch.finfo(G).eps / 2, torch.finfo(G).smallest_normal * torch.finfo(G).eps / 2
            far = np.where(np.isfinite(lp), np.abs(np.where(np.isfinite(lp), lp, 0)), 0)
            ep = SUM + (4 + 3 * far) * U
            tol = abs(w[r]) * scale * (p * ep + np.where(S, q * (SUM if not bucket else 4 * U), p * ratio * (2 * SUM + ep)))
            if qt > 0 and pt > 0:
                tol += abs(w[r]) * scale * np.where(S, 0.0, p / pt * 2 * U * Q)
            _near(_np(grad[r]), g, tol + half * (np.abs(g) + tol) + least)


def _distill(B, z, ids, logq, scale=1.0, bucket=True, weight=None, grad="f32", check=True):
    rows, vocab = z.shape
    loss = torch.full((rows,), 55.0, device="cuda")
    g = torch.full((rows, vocab), 55.0, dtype=DT[grad], device="cuda") if grad else None
    B.sgd_kernel_distill(z, ids, logq, loss, grad=g, row_weight=weight, tail=B.TAIL_BUCKET if bucket else B.TAIL_RENORM,
                         scale=scale)
    assert B.sgd_kernel_status() == 0
    if check:
        _check_distill(loss, g, z, ids, logq, scale, bucket, weight)
    return loss, g


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,vocab", SIZES)
@pytest.mark.parametrize("bucket", [True, False])
def test_distill(B, rows, vocab, dtype, bucket):
    rows = min(rows, 40)
    z = _logits(rows, vocab, dtype, rows * vocab)
    ids, logq = _lists(z, min(vocab, 8), 1)
    w = torch.linspace(-1.0, 2.0, rows).cuda()
    _distill(B, z, ids, logq, bucket=bucket, weight=w)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("grad", ["", "f16", "bf16", "f32"])
@pytest.mark.parametrize("bucket", [True, False])
def test_distill_types(B, dtype, grad, bucket):
    z = _logits(5, 20011, dtype, 2)
    ids, logq = _lists(z, 32, 2, scale=1.25)
    _distill(B, z, ids, logq, scale=1.25, bucket=bucket, grad=grad)


@pytest.mark.parametrize("k", [1, 31, 32, 33, 64])
@pytest.mark.parametrize("vocab", [64, 1000, 126464])
def test_distill_list_lengths(B, vocab, k):
    z = _logits(4, vocab, "f16", k)
    ids, logq = _lists(z, k, 3)
    for bucket in (True, False):
        _distill(B, z, ids, logq, bucket=bucket)


@pytest.mark.parametrize("dtype,grad", [("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("pad,offset,gpad,goffset", [(0, 1, 0, 1), (3, 0, 3, 0), (1, 2, 0, 0), (0, 0, 7, 3), (8, 8, 5, 0)])
def test_distill_rows_at_any_address(B, dtype, grad, pad, offset, gpad, goffset):
    rows, vocab = 5, 3001
    z = _logits(rows, vocab, dtype, 4, pad=pad, offset=offset)
    ids, logq = _lists(z, 7, 4)
    buf = torch.full((goffset + rows * (vocab + gpad) + 9,), 55.0, dtype=DT[grad], device="cuda")
    g = buf[goffset:goffset + rows * (vocab + gpad)].view(rows, vocab + gpad)[:, :vocab]
    loss = torch.empty(rows, device="cuda")
    B.sgd_kernel_distill(z, ids, logq, loss, grad=g)
    _check_distill(loss, g, z, ids, logq, 1.0, True, None)
    around = torch.ones_like(buf, dtype=torch.bool)
    around[goffset:goffset + rows * (vocab + gpad)].view(rows, vocab + gpad)[:, :vocab] = False
    assert (buf[around] == 55.0).all()


@pytest.mark.parametrize("vocab", [1000, 126464])
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_gradient_in_the_place_of_the_logits(B, vocab, dtype):
    z = _logits(9, vocab, dtype, 6, pad=3, offset=1)
    ids, logq = _lists(z, 16, 6)
    w = torch.ones(9).cuda()
    w[4] = 0
    want = _distill(B, z, ids, logq, weight=w, grad=dtype)
    loss = torch.empty(9, device="cuda")
    B.sgd_kernel_distill(z, ids, logq, loss, grad=z, row_weight=w)
    assert torch.equal(loss, want[0]) and torch.equal(z, want[1])


@pytest.mark.parametrize("bucket", [True, False])
@pytest.mark.parametrize("vocab", [40, 5003])
def test_lists_that_are_hard(B, vocab, bucket):
    """Padding, repeats, empty lists, certain and impossible tokens, all of them, weights of 0."""
    z = _logits(9, vocab, "f32", 7)
    k = 12
    ids, logq = _lists(z, k, 7)
    ids[0, 3:] = -1
    ids[1, 5] = ids[1, 2]
    ids[1, 11] = ids[1, 0]
    ids[2, :] = -1
    ids[3, 0], ids[3, 1] = vocab, 2 ** 31 - 1
    logq[4, 0], logq[4, 1:] = 0.0, -INF
    logq[5, :] = logq[5, :] - 8.0  # nearly all of it in the tail
    logq[6, :] = math.log(1.0 / k)  # nothing in the tail
    ids[7, :] = ids[7, 0]
    w = torch.ones(9).cuda()
    w[8] = 0
    z[8] = math.nan
    _distill(B, z, ids, logq, bucket=bucket, weight=w)


@pytest.mark.parametrize("bucket", [True, False])
def test_masked_logits(B, bucket):
    """-inf inside and outside the list, a row of -inf alone, a list of all that is left."""
    z = _logits(5, 3000, "f16", 8)
    ids, logq = _lists(z, 10, 8)
    z[0, 100:2000] = -INF
    z[0, ids[0].long()] = 3.0
    z[1, ids[1, 3].long()] = -INF  # impossible for the model, likely for the teacher
    keep = z[2, ids[2].long()].clone()
    z[2] = -INF
    z[2, ids[2].long()] = keep  # no tail: p_T = 0
    z[3] = -INF
    loss, g = _distill(B, z, ids, logq, bucket=bucket)
    assert loss[1] == INF and loss[3] == INF and torch.isfinite(g).all()
    out = ~torch.isin(torch.arange(100, 2000, device="cuda"), ids[0].long())
    assert (g[0, 100:2000][out] == 0).all()


def test_nan_rows_stay_their_own(B):
    z = _logits(4, 9001, "bf16", 9)
    ids, logq = _lists(z, 5, 9)
    z[1, 7000] = math.nan
    z[2, 3] = INF
    loss, g = _distill(B, z, ids, logq, check=False)
    assert torch.isnan(loss[1:3]).all() and torch.isnan(g[1:3]).all(1).all()
    rest = [0, 3]
    _check_distill(loss[rest], g[rest], z[rest], ids[rest], logq[rest], 1.0, True, None)


def test_a_small_tail_is_not_lost(B):
    """p_T of 1e-9 against q_T of 0.1: 1 - sum_S p in fp32 would be 0."""
    z = torch.zeros(2, 4000, device="cuda")
    z[:, :4] = 30.0
    z[1, :4] = 60.0
    ids = torch.arange(4, dtype=torch.int32, device="cuda").repeat(2, 1)
    logq = torch.full((2, 4), math.log(0.225), device="cuda")
    _distill(B, z, ids, logq)


def _check_rows(loss, grad, z, ids, logq, bucket, w):
    """_check_distill at scale 1 in float64 on the device, for rows of which there are many."""
    rows, vocab = z.shape
    lp = torch.log_softmax(z.double(), 1)
    p = lp.exp()
    here = (ids >= 0) & (ids < vocab)
    here &= ~torch.tril(ids[:, :, None] == ids[:, None, :], -1).any(2)
    at = torch.where(here, ids.long(), vocab)
    lq = logq.double()
    q = torch.where(here, lq.exp(), 0.0)
    Q = q.sum(1, keepdim=True)
    live = (w[:, None] != 0) & here.any(1, keepdim=True)
    scatter = lambda v: torch.zeros(rows, vocab + 1, dtype=torch.float64, device=z.device).scatter_(1, at, v)[:, :vocab]  # noqa: E731
    S = scatter(torch.ones_like(q)) > 0
    lps = torch.gather(lp, 1, at.clamp(max=vocab - 1))
    if bucket:
        qt, pt = (1 - Q).clamp(min=0), torch.where(S, 0.0, p).sum(1, keepdim=True)
    else:
        q, lq, qt, pt = q / Q, lq - Q.log(), torch.zeros_like(Q), torch.ones_like(Q)
    terms = torch.where(q > 0, q * (lq - lps), 0.0)
    L = terms.sum(1, keepdim=True) + torch.where(qt > 0, qt * (qt.log() - pt.log()), 0.0)
    tol = SUM * (q.sum(1, keepdim=True) + 2 * qt) + 2 * U * terms.abs().sum(1, keepdim=True)
    tol = tol + torch.where(qt > 0, 4 * U * Q * (qt.log() - pt.log() + 1).abs(), 0.0)
    w = torch.where(live, w[:, None].double(), 0.0)
    L = torch.where(live, w * L, 0.0)
    assert ((loss[:, None].double() - L).abs() <= w.abs() * torch.where(live, tol, 0.0) + U * L.abs()).all()
    if grad is None:
        return
    G = grad.dtype
    half, least = torch.finfo(G).eps / 2, torch.finfo(G).smallest_normal * torch.finfo(G).eps / 2
    qs, ratio = scatter(q), qt / pt
    g = torch.where(live, w * torch.where(S, p - qs, p * (1 - ratio)), 0.0)
    ep = SUM + (4 + 3 * torch.where(p > 0, lp.abs(), 0.0)) * U
    tol = p * ep + torch.where(S, qs * (4 * U if bucket else SUM), p * ratio * (2 * SUM + ep))
    if bucket:
        tol = tol + torch.where(S, 0.0, p / pt * 2 * U * Q)
    tol = torch.where(live, w.abs() * tol, 0.0)
    err = (grad.double() - g).abs()
    assert (err <= tol + half * (g.abs() + tol) + least).all(), (err / (tol + half * (g.abs() + tol) + least)).max()


# many long rows (48 MiB and more of them): they stream through clusters of 1 to 8 CTAs
@pytest.mark.parametrize("rows,vocab,dtype,grad,pad,offset", [
    (200, 126464, "f16", "bf16", 0, 0), (301, 126464, "f16", "f16", 0, 0), (210, 126464, "f16", "", 0, 0),
    (800, 32003, "bf16", "bf16", 0, 1), (801, 32003, "f16", "f32", 13, 0), (260, 50021, "f32", "f32", 0, 3),
    (1600, 16387, "f16", "f16", 5, 2), (1600, 16387, "bf16", "", 1, 0), (100, 266176, "f16", "bf16", 0, 0),
    (98, 133081, "f32", "bf16", 2, 1), (102, 126464, "f32", "f32", 0, 0), (5000, 8209, "f16", "bf16", 0, 0),
    (6100, 4177, "f16", "bf16", 3, 0), (6100, 4177, "f16", "", 3, 0), (3000, 4409, "f32", "", 0, 1), (1600, 8190, "f32", "f32", 0, 1),
    (1700, 16384, "bf16", "bf16", 0, 0)])
@pytest.mark.parametrize("bucket,k", [(True, 32), (False, 64), (True, 1)])
def test_distill_of_many_rows(B, rows, vocab, dtype, grad, pad, offset, bucket, k):
    assert rows * vocab * torch.finfo(DT[dtype]).bits // 8 >= 48 << 20
    g = torch.Generator("cuda").manual_seed(rows)
    buf = torch.full((offset + rows * (vocab + pad),), 3e4, dtype=DT[dtype], device="cuda")
    z = buf[offset:].view(rows, vocab + pad)[:, :vocab]
    z.copy_(torch.empty(rows, vocab, device="cuda").normal_(0, 2, generator=g))
    z[rows // 3, vocab // 2:] = -INF
    top = torch.topk(z.float() + torch.empty(rows, vocab, device="cuda").normal_(0, 1, generator=g), k, dim=1)
    ids = top.indices.int()
    logq = top.values - math.log(vocab) - 2.0
    ids[3, k // 2:] = -1
    ids[4, :] = -1
    ids[5, k - 1] = ids[5, 0]
    w = 0.5 + torch.rand(rows, device="cuda", generator=g)
    w[torch.rand(rows, device="cuda", generator=g) < 0.3] = 0
    loss, out = _distill(B, z, ids, logq, bucket=bucket, weight=w, grad=grad, check=False)
    some = sorted({0, 1, 3, 4, 5, rows // 3, rows - 1, *range(7, rows, max(1, rows // 5))})
    _check_distill(loss[some], None if out is None else out[some], z[some], ids[some], logq[some], 1.0, bucket, w[some])
    for a in range(0, rows, 16):
        b = slice(a, a + 16)
        _check_rows(loss[b], out[b] if grad else None, z[b], ids[b], logq[b], bucket, w[b])
    if dtype == grad:  # in the place of the logits
        l2 = torch.empty_like(loss)
        B.sgd_kernel_distill(z, ids, logq, l2, grad=z, row_weight=w, tail=B.TAIL_BUCKET if bucket else B.TAIL_RENORM)
        assert torch.equal(l2, loss) and torch.equal(z, out)
        assert (buf[:offset] == 3e4).all() and (buf[offset:].view(rows, vocab + pad)[:, vocab:] == 3e4).all()


@pytest.mark.parametrize("weights", ["none", "zero", "one left", "none given"])
def test_weights_of_many_rows(B, weights):
    rows, vocab = 1400, 20000
    z = torch.empty(rows, vocab, dtype=torch.float16, device="cuda").normal_(0, 2, generator=torch.Generator("cuda").manual_seed(1))
    ids, logq = torch.randint(0, vocab, (rows, 3), dtype=torch.int32).cuda(), torch.full((rows, 3), -1.2).cuda()
    w = None if weights == "none given" else torch.zeros(rows, device="cuda") if weights != "none" else torch.ones(rows, device="cuda")
    if weights == "one left":
        w[777] = 2.0
    loss, g = _distill(B, z, ids, logq, weight=w, grad="bf16", check=False)
    some = [0, 5, 776, 777, 778, rows - 1]
    _check_distill(loss[some], g[some], z[some], ids[some], logq[some], 1.0, True, None if w is None else w[some])
    if weights in ("zero", "one left"):
        assert int((loss != 0).sum()) == (weights == "one left") and int((g != 0).any(1).sum()) == (weights == "one left")


@pytest.mark.parametrize("bucket", [True, False])
def test_gradient_is_the_difference_of_the_loss(B, bucket):
    """(L(z + h v) - L(z - h v)) / 2 h against <gradient, v>, through the kernel alone: fp32 losses off by
    3 SUM each and a third derivative of at most 1 in a direction of length 1: h = 0.05 leaves
    3 SUM / 0.05 + 0.05^2 / 6 < 2e-3."""
    z = _logits(8, 500, "f32", 10)
    ids, logq = _lists(z, 9, 10)
    v = torch.randn(8, 500, generator=torch.Generator().manual_seed(3)).cuda()
    v[:, :] = 0.2 * v
    v.scatter_(1, ids.long(), torch.randn(8, 9, generator=torch.Generator().manual_seed(4)).cuda())
    v /= v.norm(dim=1, keepdim=True)
    loss, g = _distill(B, z, ids, logq, bucket=bucket)
    a, _ = _distill(B, z + 0.05 * v, ids, logq, bucket=bucket, grad="")
    b, _ = _distill(B, z - 0.05 * v, ids, logq, bucket=bucket, grad="")
    assert ((a - b) / 0.1 - (g * v).sum(1)).abs().max() < 2e-3


def test_own_top_list_pulls_at_nothing(B):
    """A teacher that is the model: loss and gradient vanish against their parts' rounding."""
    z = _logits(6, 126464, "f16", 11)
    ids = torch.empty(6, 32, dtype=torch.int32, device="cuda")
    lp = torch.empty(6, 32, device="cuda")
    B.sgd_kernel_logprobs(z, top_ids=ids, top_logprobs=lp)
    loss, g = _distill(B, z, ids, lp)
    assert loss.abs().max() < 4 * SUM and g.abs().max() < 4 * SUM


# ---------------------------------------------------------------------------
# reveal
# ---------------------------------------------------------------------------

def _check_reveal(B, ids, cand, score, n, mask, lowest=False, window=None, **kw):
    ids, cand, score = torch.as_tensor(ids).int(), torch.as_tensor(cand).int(), torch.as_tensor(score).float()
    n = torch.as_tensor(n).int()
    win = None if window is None else torch.as_tensor(window).int()
    out, left = torch.full_like(ids, -9).cuda(), torch.full((len(ids),), -9, dtype=torch.int32).cuda()
    B.sgd_sampler_reveal(ids.cuda(), cand.cuda(), score.cuda(), n.cuda(), out, mask, lowest=lowest,
                         window=None if win is None else win.cuda(), n_left=left)
    want, wleft = ot.reveal(ids.numpy(), cand.numpy(), score.numpy(), n.numpy(), mask, lowest,
                            None if win is None else win.numpy())
    assert np.array_equal(out.cpu().numpy(), want)
    assert np.array_equal(left.cpu().numpy(), wleft)


@pytest.mark.parametrize("batch,tokens", [(1, 1), (3, 2), (2, 31), (1, 32), (5, 33), (2, 192), (4, 1024), (3, 1025), (2, 4096),
                                          (1, 10007), (1, 49152)])
@pytest.mark.parametrize("coarse", [False, True])
@pytest.mark.parametrize("lowest", [False, True])
def test_reveal(B, batch, tokens, coarse, lowest):
    rng = np.random.default_rng(tokens)
    ids = np.where(rng.random((batch, tokens)) < 0.6, 7, rng.integers(8, 99, (batch, tokens)))
    score = rng.standard_normal((batch, tokens))
    if coarse:
        score = np.round(2 * score) / 2
    cand = rng.integers(100, 200, (batch, tokens))
    for n in (0, 1, max(1, tokens // 16), tokens // 2, tokens + 5, -3):
        _check_reveal(B, ids, cand, score, np.full(batch, n), 7, lowest)
    lo = rng.integers(-2, tokens + 1, batch)
    _check_reveal(B, ids, cand, score, rng.integers(0, 9, batch), 7, lowest,
                  np.stack([lo, lo + rng.integers(0, tokens + 4, batch)], 1))


def test_reveal_scores_that_are_hard(B):
    N = 300
    s = np.zeros((7, N))
    s[1] = -INF
    s[2, ::3], s[2, 1::3] = math.nan, -INF
    s[3] = np.where(np.arange(N) % 2, 0.0, -0.0)
    s[4] = math.nan
    s[5, 10:20] = INF
    s[6] = -3.4e38
    s[6, 5] = -INF
    ids = np.full((7, N), 7)
    ids[:, ::7] = 1
    cand = np.arange(7 * N).reshape(7, N) + 100
    for n in (1, 9, 100, 257, 258):
        for lowest in (False, True):
            _check_reveal(B, ids, cand, s, np.full(7, n), 7, lowest)
    _check_reveal(B, ids, cand, s, np.full(7, 5), 12345)  # nothing is masked
    _check_reveal(B, ids, cand, s, np.full(7, 5), 7, window=np.array([[9, 3]] * 7))  # an empty window


def test_reveal_in_place_and_of_columns(B):
    rng = np.random.default_rng(5)
    ids = torch.from_numpy(np.where(rng.random((3, 500)) < 0.5, 7, 1)).int().cuda()
    cand, score = torch.randint(10, 99, (3, 500, 5), dtype=torch.int32).cuda(), torch.randn(3, 500, 4).cuda()
    n = torch.tensor([3, 40, 0], dtype=torch.int32).cuda()
    want, _ = ot.reveal(ids.cpu().numpy(), cand[:, :, 2].cpu().numpy(), score[:, :, 1].cpu().numpy(), n.cpu().numpy(), 7)
    B.sgd_sampler_reveal(ids, cand[:, :, 2], score[:, :, 1], n, ids, 7)
    assert np.array_equal(ids.cpu().numpy(), want)


# ---------------------------------------------------------------------------
# streams, graphs, repeated and concurrent calls
# ---------------------------------------------------------------------------

def _everything(B, z, ids, logq, seq, stream=None):
    rows = z.shape[0]
    o = dict(e=torch.zeros(rows, device="cuda"), i=torch.zeros(rows, 5, dtype=torch.int32, device="cuda"),
             p=torch.zeros(rows, 5, device="cuda"), l=torch.zeros(rows, device="cuda"), g=torch.zeros_like(z),
             s=torch.zeros_like(seq), n=torch.full((1,), 2, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()

    def call():
        B.sgd_kernel_logprobs(z, entropy=o["e"], top_ids=o["i"], top_logprobs=o["p"], stream=stream)
        B.sgd_kernel_distill(z, ids, logq, o["l"], grad=o["g"], stream=stream)
        B.sgd_sampler_reveal(seq, o["i"][None, :, 0], o["e"][None], o["n"], o["s"], 0, lowest=True, stream=stream)
    return o, call


def _inputs(seed, rows=24, vocab=40000):
    z = _logits(rows, vocab, "f16", seed)
    ids, logq = _lists(z, 8, seed)
    return z, ids, logq, torch.zeros(1, rows, dtype=torch.int32, device="cuda")


def _same(a, b):
    return all(torch.equal(a[n], b[n]) for n in a)


def test_two_streams_at_once_and_runs_repeat_bit_for_bit(B):
    sets = [_inputs(s) for s in (20, 21)]
    want = []
    for x in sets:
        o, call = _everything(B, *x)
        call()
        want.append(o)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    both = [_everything(B, *x, stream=s) for x, s in zip(sets, streams)]
    for _ in range(20):
        for _, call in both:
            call()
    torch.cuda.synchronize()
    for w, (o, _) in zip(want, both):
        assert _same(w, o)


def test_captured_calls_replay_on_new_inputs(B):
    """Two graphs, replayed at the same time on two streams, after their inputs changed."""
    sets = [_inputs(s) for s in (30, 31)]
    new = [_inputs(s) for s in (32, 33)]
    want = []
    for x in new:
        o, call = _everything(B, *x)
        call()
        want.append(o)
    graphs, outs = [], []
    for x in sets:
        o, call = _everything(B, *x)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        graphs.append(g)
        outs.append(o)
    for x, y in zip(sets, new):
        for a, b in zip(x, y):
            a.copy_(b)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        assert _same(w, o)
    assert B.sgd_kernel_status() == 0


def test_binding_checks_tensors(B):
    z = torch.zeros(4, 100, dtype=torch.float16, device="cuda")
    f, i = torch.zeros(4, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    p = torch.zeros(4, 2, device="cuda")
    with pytest.raises(ValueError, match="shape"):
        B.sgd_kernel_logprobs(z, entropy=f[:3])
    with pytest.raises(ValueError, match="is on"):
        B.sgd_kernel_logprobs(z, entropy=f.cpu())
    with pytest.raises(TypeError):
        B.sgd_kernel_logprobs(z, top_ids=i.long())
    with pytest.raises(ValueError, match="dense"):
        B.sgd_kernel_logprobs(z.t(), entropy=torch.zeros(100, device="cuda"))
    with pytest.raises(ValueError, match="together"):
        B.sgd_kernel_logprobs(z, tokens=i)
    with pytest.raises(B.SgdError):
        B.sgd_kernel_logprobs(z[:1].expand(4, 100), entropy=f)  # all rows are one
    with pytest.raises(ValueError, match="shape"):
        B.sgd_kernel_distill(z, i, p, f, grad=z[:, :50])
    with pytest.raises(B.SgdError, match="overlaps"):
        B.sgd_kernel_distill(z[:3], i[:3], p[:3], f[:3], grad=z[1:])
    with pytest.raises(ValueError, match="evenly"):
        B.sgd_sampler_reveal(torch.zeros(2, 4, dtype=torch.int32, device="cuda"),
                             torch.zeros(2, 9, dtype=torch.int32, device="cuda")[:, :4], torch.zeros(2, 4, device="cuda"),
                             torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, 4, dtype=torch.int32, device="cuda"), 0)
