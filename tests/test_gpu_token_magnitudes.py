"""Finite logits of any magnitude (masks of the type's lowest value, of -1e10 and others, large scales) on the GPU,
scored and distilled, against oracle/tokens.py in float64: only NaN and +inf in a row make NaN.  Tolerances
as derived in test_gpu_tokens.py; an exponent that is taken as (x - m) c instead of c x - R has the same
bound, two roundings and c's.  Rows here have probabilities of any smallness: ex2.approx gives 0 for those
below 2^-126, which moves a gradient by less than FLUSH times its factors of at most 1."""
import numpy as np
import pytest
import torch

from oracle import tokens as ot
from test_gpu_tokens import B, DT, SUM, U, _check_score, _near, _np, _score  # noqa: F401

FLUSH = 2.0 ** -126

pytestmark = pytest.mark.gpu

MASKS = {"f32": [-1e9, -1e10, -1e20, -1e30, -1e37, float(torch.finfo(torch.float32).min)],
         "bf16": [-1e9, -1e10, -1e20, -1e30, -1e37, float(torch.finfo(torch.bfloat16).min)],
         "f16": [-65504.0]}


def _rows(vocab, mask, seed):
    """Ways in which a mask lies in a row: one token, every other, ranges of whole slices at either end, all but one
    or a few, all; and logits that are large themselves."""
    rng = np.random.default_rng(seed)
    z = 2.0 * rng.standard_normal((13, vocab))
    z[0, vocab // 3] = mask
    z[1, rng.random(vocab) < 0.5] = mask
    z[2, :vocab // 2] = mask
    z[3, vocab // 2:] = mask
    z[4, : vocab - 3] = mask
    z[5, 3:] = mask
    z[6, :] = mask
    z[6, vocab // 2] = 1.0
    z[7, :] = mask
    z[8, :] = -mask
    z[8, 1::3] = 0.0
    z[9, vocab // 5] = -mask
    z[10, :] = np.where(np.arange(vocab) % 2 == 0, mask, -mask)
    z[11, :] = mask * (1.0 - rng.random(vocab) / 64)
    z[12, vocab // 4:] = mask / 2
    z[12, vocab // 2:] = mask
    return z


CASES = [(d, m) for d in MASKS for m in MASKS[d]]


@pytest.mark.parametrize("dtype,mask", CASES)
@pytest.mark.parametrize("vocab", [70, 1000, 20011, 126464])
@pytest.mark.parametrize("scale", [1.0, 0.75, 0.25, 3.0])
def test_scores_of_masked_rows(B, vocab, dtype, mask, scale):
    z = torch.from_numpy(_rows(vocab, mask, 1)).to(DT[dtype]).cuda()
    for k in (1, 5):
        got, tokens = _score(B, z, k=k, n=3, scale=scale)
        # (what fp32 does not hold is infinite: log-probabilities below -3.4e38)
        _check(got, tokens, z, k, scale)


def _check(got, tokens, z, k, scale):
    for n in ("token_logprobs", "top_logprobs"):
        got[n] = np.where(np.isneginf(got[n]), -np.inf, got[n].astype(np.float64))
    real = ot.log_softmax

    def in_range(x, s=1.0):
        lp = real(x, s)
        return np.where(lp < -3.4028235e38, -np.inf, lp)
    ot.log_softmax = in_range
    try:
        _check_score(got, tokens, z, k, scale)
    finally:
        ot.log_softmax = real


@pytest.mark.parametrize("scale", [1e8, 3e30, 1e-30])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("vocab", [70, 20011])
def test_scores_at_extreme_scales(B, vocab, dtype, scale):
    z = torch.from_numpy(_rows(vocab, -60.0, 2)).to(DT[dtype]).cuda()
    scale = float(np.float32(scale))
    for k in (1, 5):
        got, tokens = _score(B, z, k=k, n=3, scale=scale)
        _check(got, tokens, z, k, scale)


@pytest.mark.parametrize("dtype,mask", [("f32", -1e10), ("f32", MASKS["f32"][-1]), ("bf16", MASKS["bf16"][-1]), ("f16", -65504.0)])
@pytest.mark.parametrize("k", [0, 1, 9])
def test_scores_of_masked_rows_among_many(B, dtype, mask, k):
    vocab, n = 126464, 13
    hard = torch.from_numpy(_rows(vocab, mask, 3)).to(DT[dtype])
    z = hard.repeat(16, 1).cuda()
    got, tokens = _score(B, z, k=k, tokens=torch.arange(2 * n).view(n, 2).int().repeat(16, 1))
    _check({m: x[:n] for m, x in got.items()} if k else
           {**{m: x[:n] for m, x in got.items()}, "top_logprobs": np.zeros(1)}, tokens[:n], hard, k, 1.0)
    for x in got.values():
        x = x.reshape(16, n, -1)
        assert np.array_equal(x, np.broadcast_to(x[:1], x.shape))


def _check_distill(loss, grad, z, ids, logq, scale, bucket):
    """Lists of distinct tokens, every one of them weighted."""
    z, ids, logq, loss = _np(z), ids.cpu().numpy(), _np(logq), _np(loss)
    for r in range(len(z)):
        L, g = ot.distill_row(z[r], ids[r], logq[r], scale, bucket)
        lp = ot.log_softmax(z[r][None], scale)[0]
        p = np.exp(lp)
        S = np.zeros(len(p), bool)
        S[ids[r]] = True
        q = np.zeros(len(p))
        q[ids[r]] = np.exp(logq[r])
        Q = q.sum()
        qt = max(0.0, 1 - Q) if bucket else 0.0
        q /= 1.0 if bucket else Q
        pt = np.where(S, 0.0, p).sum()
        assert pt > 0
        pull = (q[ids[r]] * np.abs(np.log(q[ids[r]]) - lp[ids[r]])).sum()
        # (4 U of it: ln p of a token far below the maximum is a product and a difference)
        tol = SUM * (q.sum() + 2 * qt) + 4 * U * pull
        if qt > 0:
            tol += 4 * U * Q * abs(np.log(qt) - np.log(pt) + 1)
        _near(loss[r], L, tol + U * abs(L))
        if grad is not None:
            G = grad.dtype
            half, least = torch.finfo(G).eps / 2, torch.finfo(G).smallest_normal * torch.finfo(G).eps / 2
            ep = np.where(p > 0, SUM + (4 + 3 * np.abs(np.where(p > 0, lp, 0.0))) * U, 0.0)
            tol = p * ep + np.where(S, q * (SUM if not bucket else 4 * U), p * (qt / pt) * (2 * SUM + ep) + p / pt * 2 * U * Q)
            tol = scale * (tol + FLUSH)
            _near(_np(grad[r]), g, tol + half * (np.abs(g) + tol) + least)


def _lists(z, mask, k):
    """A list of k tokens a row, some of them masked ones, as the row has them; some of what counts stays outside."""
    rng = np.random.default_rng(5)
    z = z.double().cpu().numpy()
    ids = np.stack([rng.permutation(z.shape[1])[:k] for _ in range(len(z))])
    for r in range(len(z)):  # the largest but one, and not the largest
        order = np.argsort(-z[r], kind="stable")
        ids[r][ids[r] == order[0]] = order[1]
        if order[1] not in ids[r]:
            ids[r][0] = order[1]
    lq = np.log(rng.dirichlet(np.ones(k + 1), len(z))[:, :k] * 0.98 + 1e-3)
    return torch.from_numpy(ids.astype(np.int32)).cuda(), torch.from_numpy(lq.astype(np.float32)).cuda()


@pytest.mark.parametrize("dtype,mask", CASES)
@pytest.mark.parametrize("vocab", [70, 1000, 126464])
@pytest.mark.parametrize("bucket", [True, False])
def test_distillation_of_masked_rows(B, vocab, dtype, mask, bucket):
    z = torch.from_numpy(_rows(vocab, mask, 4)).to(DT[dtype]).cuda()
    keep = [0, 1, 2, 3, 4, 5, 7, 8, 11, 12]  # (the others are one token's alone: nothing is left outside a list, or in it)
    z = z[keep].contiguous()
    ids, logq = _lists(z, mask, 7)
    loss = torch.empty(len(z), device="cuda")
    for grad in ("", "f32", "bf16"):
        g = torch.empty(z.shape, dtype=DT[grad], device="cuda") if grad else None
        B.sgd_kernel_distill(z, ids, logq, loss, grad=g, tail=B.TAIL_BUCKET if bucket else B.TAIL_RENORM)
        _check_distill(loss, g, z, ids, logq, 1.0, bucket)


@pytest.mark.parametrize("dtype,mask", [("f32", -1e10), ("f32", MASKS["f32"][-1]), ("bf16", MASKS["bf16"][-1]), ("f16", -65504.0)])
@pytest.mark.parametrize("grad", ["", "f32"])
def test_distillation_of_masked_rows_among_many(B, dtype, mask, grad):
    vocab, n = 126464, 10
    hard = torch.from_numpy(_rows(vocab, mask, 6)).to(DT[dtype])[[0, 1, 2, 3, 4, 5, 7, 8, 11, 12]].contiguous()
    ids, logq = _lists(hard, mask, 7)
    z, ids, logq = hard.repeat(25, 1).cuda(), ids.repeat(25, 1), logq.repeat(25, 1)
    assert z.numel() * z.element_size() >= 48 << 20
    for bucket in (True, False):
        loss = torch.empty(len(z), device="cuda")
        g = torch.empty(z.shape, dtype=DT[grad], device="cuda") if grad else None
        B.sgd_kernel_distill(z, ids, logq, loss, grad=g, tail=B.TAIL_BUCKET if bucket else B.TAIL_RENORM)
        _check_distill(loss[:n], None if g is None else g[:n], hard, ids[:n], logq[:n], 1.0, bucket)
        assert torch.equal(loss.view(25, n), loss[:n].expand(25, n))
        assert g is None or torch.equal(g.view(25, n, vocab), g[:n].expand(25, n, vocab))


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_distillation_at_a_large_scale(B, dtype):
    z = torch.from_numpy(_rows(3001, -60.0, 7)).to(DT[dtype])[[0, 1, 2, 3, 7, 8]].contiguous().cuda()
    ids, logq = _lists(z, -60.0, 7)
    loss, g = torch.empty(len(z), device="cuda"), torch.empty(z.shape, device="cuda")
    B.sgd_kernel_distill(z, ids, logq, loss, grad=g, tail=B.TAIL_RENORM, scale=1e8)
    _check_distill(loss, g, z, ids, logq, 1e8, False)


@pytest.mark.parametrize("scale", [10.0, 0.25, 1.0])
def test_rows_whose_scaled_logits_are_out_of_range(B, scale):
    """Largest logits of -1e38 and 3e38: scaled ones, their differences or both are out of fp32's range; what is below that
    has -inf for ln p, and a listed one an infinite loss."""
    vocab = 300
    rng = np.random.default_rng(8)
    z = np.full((4, vocab), -3.2e38)
    z[0, ::3] = -1e38
    z[1, ::3] = 3e38
    z[2, :] = -3e38 + 1e37 * rng.random(vocab)
    z[3, ::3], z[3, 1::3] = -1e38, -1e38 * (1 + 2.0 ** -20)
    z = torch.from_numpy(z).float().cuda()
    got, tokens = _score(B, z, k=5, n=3, scale=scale, tokens=torch.tensor([[0, 1, 2]] * 4, dtype=torch.int32))
    _check(got, tokens, z, 5, scale)
    ids = torch.tensor([[0, 1]] * 4, dtype=torch.int32, device="cuda")
    logq = torch.log(torch.tensor([[0.5, 0.25]] * 4, device="cuda"))
    for tail in (B.TAIL_BUCKET, B.TAIL_RENORM):
        loss, g = torch.empty(4, device="cuda"), torch.empty(z.shape, device="cuda")
        B.sgd_kernel_distill(z, ids, logq, loss, grad=g, tail=tail, scale=scale)
        for r in range(4):
            L, want = ot.distill_row(_np(z[r]), [0, 1], _np(logq[r]), scale, tail == B.TAIL_BUCKET)
            L = np.inf if L > 3.4028235e38 else L
            assert loss[r].item() == L or abs(loss[r].item() - L) <= 16 * U * L, (r, loss[r].item(), L)
            assert np.abs(_np(g[r]) - want).max() <= scale * 8 * SUM
