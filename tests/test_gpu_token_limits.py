"""The operators on a token model's logits at the limits of their ranges, against float64 on the same inputs.
Tolerances as in test_gpu_tokens.py: SUM for a row's sum, U for a rounding."""
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


def _normal(rows, vocab, dtype, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.empty(rows, vocab, dtype=DT[dtype], device="cuda").normal_(0, 2, generator=g)


@pytest.mark.parametrize("rows,vocab,dtype,grad", [(420, 126464, "f16", "bf16"), (420, 126464, "f16", ""), (900, 40000, "f16", "f16"),
                                                   (900, 40000, "bf16", ""), (5, 3001, "f32", "f32")])
def test_lists_without_weight_between_others(B, rows, vocab, dtype, grad):
    """Renormalised lists whose log-probabilities are all -inf (a teacher's row that was masked altogether), in runs of
    many lengths between others: nothing of them in the others' losses.  The loss is off by what its terms
    are: ln p by SUM, q (and its share of the list) by 4 U."""
    k = 6
    z = _normal(rows, vocab, dtype, 1)
    rng = np.random.default_rng(2)
    ids = torch.from_numpy(np.stack([rng.permutation(vocab)[:k] for _ in range(rows)]).astype(np.int32)).cuda()
    z.scatter_(1, ids.long(), torch.from_numpy(20.0 * rng.random((rows, k))).to(z))  # (another list's logits would show)
    logq = torch.from_numpy(-1.0 - 2.0 * rng.random((rows, k))).float().cuda()
    dead = torch.from_numpy(np.concatenate([[i % 2 == 1] * n for i, n in enumerate(rng.integers(1, 30, rows))])[:rows]).cuda()
    logq[dead] = -INF
    loss = torch.full((rows,), 55.0, device="cuda")
    g = torch.full((rows, vocab), 55.0, dtype=DT[grad], device="cuda") if grad else None
    B.sgd_kernel_distill(z, ids, logq, loss, grad=g, tail=B.TAIL_RENORM)
    assert B.sgd_kernel_status() == 0
    assert (loss[dead] == 0).all() and (g is None or not g[dead].any())
    live = ~dead
    lp = torch.cat([torch.gather(torch.log_softmax(a.double(), 1), 1, i.long()) for a, i in zip(z.split(64), ids.split(64))])[live]
    lq = torch.log_softmax(logq[live].double(), 1)
    q = lq.exp()
    want = (q * (lq - lp)).sum(1)
    tol = 2 * SUM + 4 * U * (q * (lq - lp).abs()).sum(1)
    assert ((loss[live].double() - want).abs() <= tol + U * want.abs()).all()
    again = torch.empty_like(loss)
    for _ in range(5):
        B.sgd_kernel_distill(z, ids, logq, again, tail=B.TAIL_RENORM)
        assert torch.equal(again, loss) or g is not None
        assert ((again[live].double() - want).abs() <= tol + U * want.abs()).all()


@pytest.mark.parametrize("rows,vocab,dtype", [(12, 700, "f16"), (12, 9001, "f32"), (420, 126464, "f16")])
@pytest.mark.parametrize("bucket", [True, False])
@pytest.mark.parametrize("bad", [math.nan, INF])
def test_what_is_no_number_shows_wherever_it_stands(B, rows, vocab, dtype, bucket, bad):
    """NaN or +inf at a token that the list gives no weight, at one that it does, outside the list beside a masked token
    that has weight, and alone in a row of -inf."""
    z = _normal(rows, vocab, dtype, 3)
    ids = torch.arange(4, dtype=torch.int32, device="cuda").repeat(rows, 1) * 5
    logq = torch.tensor([-1.0, -2.0, -INF, -3.0], device="cuda").repeat(rows, 1)
    z[0, 10], z[1, 5] = bad, bad
    z[2, 0], z[2, vocab - 1] = -INF, bad
    z[3, :] = -INF
    z[3, 7] = bad
    z[4, :], ids[4, 1:] = -INF, -1
    z[4, 10] = bad
    z[5, 10] = -INF  # a number, as it has no weight
    for grad in ("", "f32"):
        loss = torch.empty(rows, device="cuda")
        g = torch.empty(rows, vocab, dtype=DT[grad], device="cuda") if grad else None
        B.sgd_kernel_distill(z, ids, logq, loss, grad=g, tail=B.TAIL_BUCKET if bucket else B.TAIL_RENORM)
        assert torch.isnan(loss[:5]).all() and torch.isfinite(loss[5:]).all()
        assert g is None or torch.isnan(g[:5]).all() and torch.isfinite(g[5:]).all()


def _check_tails(loss, grad, z, ids, logq, rows):
    """Rows of lists with distinct tokens and a bucket, as derived in test_gpu_tokens.py, with the tail's share of its
    tokens in the place of p / p_T.  ln p_T is off by SUM and, as a sum of its parts, by 4 U of their size."""
    loss, ids, logq = loss.double().cpu().numpy(), ids.cpu().numpy(), logq.double().cpu().numpy()
    for r in rows:
        x = z[r].double().cpu().numpy()
        L, g = ot.distill_row(x, ids[r], logq[r])
        lp = ot.log_softmax(x[None])[0]
        p, q = np.exp(lp), np.exp(logq[r])
        out = np.ones(len(p), bool)
        out[ids[r]] = False
        of_tail = np.exp(np.where(out, x - x[out].max(), -np.inf))
        lpt = x[out].max() - x.max() + np.log(of_tail.sum()) - np.log(np.exp(x - x.max()).sum())
        Q = q.sum()
        qt = max(0.0, 1 - Q)
        assert qt > 0
        tol = SUM * (Q + 2 * qt) + 4 * U * ((q * np.abs(logq[r] - lp[ids[r]])).sum() + qt * abs(np.log(qt) - lpt))
        tol += 4 * U * Q * abs(np.log(qt) - lpt + 1)
        assert abs(loss[r] - L) <= tol + U * abs(L), (r, loss[r], L)
        if grad is not None:
            half, least = torch.finfo(grad.dtype).eps / 2, torch.finfo(grad.dtype).smallest_normal * torch.finfo(grad.dtype).eps / 2
            ep = np.where(p > 0, SUM + (4 + 3 * np.abs(lp)) * U, 0.0)
            share = of_tail / of_tail.sum()  # off by the exponent's distance from the tail's maximum
            es = 2 * SUM + (4 + 3 * np.abs(np.log(np.where(share > 0, share, 1.0)))) * U
            qs = np.zeros(len(p))
            qs[ids[r]] = q
            tol = p * ep + np.where(out, share * (qt * es + 2 * U * Q), qs * 4 * U) + 2.0 ** -126  # (ex2 is 0 below)
            err = np.abs(grad[r].double().cpu().numpy() - g)
            assert (err <= tol + half * (np.abs(g) + tol) + least).all(), (r, (err / tol).max())


@pytest.mark.parametrize("gap", [30.0, 80.0, 90.0, 120.0, 1000.0, 60000.0, 1e10, 3e38])
@pytest.mark.parametrize("rows,vocab,dtype,grad", [(6, 70, "f32", "f32"), (6, 4001, "f32", "f32"), (6, 4001, "f16", "bf16"), (3, 126464, "bf16", "f32"),
                                                   (420, 126464, "f16", "f32"), (210, 126464, "f32", "bf16"), (420, 126464, "bf16", "")])
def test_a_tail_far_below_the_list(B, rows, vocab, dtype, grad, gap):
    """A student that is certain of the listed tokens alone, while the teacher leaves the others a tenth, a half or a
    thousandth."""
    if gap > torch.finfo(DT[dtype]).max / 2:
        pytest.skip("out of the type's range")
    k = 4
    z = _normal(rows, vocab, dtype, 5)
    rng = np.random.default_rng(6)
    ids = torch.from_numpy(np.stack([rng.permutation(vocab)[:k] for _ in range(rows)]).astype(np.int32)).cuda()
    top = gap + 2.0 * torch.from_numpy(rng.random((rows, k))).cuda()
    z.scatter_(1, ids.long(), top.to(z))
    part = torch.tensor([0.9, 0.5, 0.999], device="cuda").repeat((rows + 2) // 3)[:rows, None]
    logq = torch.log(part * torch.softmax(torch.from_numpy(rng.standard_normal((rows, k))).float().cuda(), 1))
    loss = torch.empty(rows, device="cuda")
    g = torch.empty(rows, vocab, dtype=DT[grad], device="cuda") if grad else None
    B.sgd_kernel_distill(z, ids, logq, loss, grad=g)
    assert B.sgd_kernel_status() == 0
    _check_tails(loss, g, z, ids, logq, sorted({0, 1, 2, *range(3, rows, max(1, rows // 9))}))
    if g is not None:  # (off by what each of the tail's tokens and of the list's is)
        assert (g.double().sum(1).abs() <= 1e-2 if grad == "bf16" else g.double().sum(1).abs() <= 1e-4).all()


@pytest.mark.parametrize("rows,vocab,dtype,grad", [(8, 60, "f32", "f32"), (8, 5003, "f16", "bf16"), (420, 126464, "f16", "f32"), (210, 126464, "f32", "f32")])
def test_a_tail_that_is_masked_altogether(B, rows, vocab, dtype, grad):
    """Every token outside the list at -inf, the list's mass below 1: against the formula's derivative, which sums to 0
    (p is off by SUM and its exponent's bound, q by 4 U), and against differences of the kernel's own losses, off by
    3 SUM each: h = 0.05 leaves 3 SUM / 0.05 + 0.05^2 < 4e-3 in a direction of length 1."""
    k = 6
    rng = np.random.default_rng(8)
    ids = torch.from_numpy(np.stack([rng.permutation(vocab)[:k] for _ in range(rows)]).astype(np.int32)).cuda()
    z = torch.full((rows, vocab), -INF, dtype=DT[dtype], device="cuda")
    z.scatter_(1, ids.long(), torch.from_numpy(2 * rng.standard_normal((rows, k))).to(z))
    logq = torch.from_numpy(np.log(rng.dirichlet(np.ones(k), rows) * rng.uniform(0.2, 0.95, (rows, 1)) + 1e-3)).float().cuda()
    loss, g = torch.empty(rows, device="cuda"), torch.empty(rows, vocab, dtype=DT[grad], device="cuda")
    B.sgd_kernel_distill(z, ids, logq, loss, grad=g)
    for r in sorted({0, 1, 2, rows - 1, *range(3, rows, max(1, rows // 9))}):
        at, lq = ids[r].cpu().numpy(), logq[r].double().cpu().numpy()
        L, want = ot.distill_row(z[r].double().cpu().numpy(), at, lq)
        lp = ot.log_softmax(z[r].double().cpu().numpy()[None])[0][at]
        assert abs(want.sum()) < 1e-14
        q = np.exp(lq)
        assert abs(loss[r].item() - L) <= SUM * q.sum() + 4 * U * (q * np.abs(lq - lp)).sum() + U * abs(L)
        got = g[r].double().cpu().numpy()
        tol = np.exp(lp) * (SUM + (4 + 3 * np.abs(lp)) * U) + 4 * U * q
        assert (np.abs(got[at] - want[at]) <= tol + torch.finfo(DT[grad]).eps / 2 * (np.abs(want[at]) + tol)).all()
        got[at] = 0
        assert not got.any()
    if dtype == "f32":
        v = torch.randn(rows, k, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
        v /= v.norm(dim=1, keepdim=True)
        d = []
        for h in (0.05, -0.05):
            loss2 = torch.empty(rows, device="cuda")
            B.sgd_kernel_distill(z.scatter_add(1, ids.long(), h * v), ids, logq, loss2)
            d.append(loss2)
        assert ((d[0] - d[1]) / 0.1 - (torch.gather(g, 1, ids.long()) * v).sum(1)).abs().max() < 4e-3


@pytest.mark.parametrize("rows,vocab,dtype,grad", [(9, 60, "f32", "f32"), (9, 5003, "f16", "f32"), (420, 126464, "f16", "f32"), (420, 126464, "bf16", "")])
@pytest.mark.parametrize("k", [1, 5, 40])
def test_renormalised_lists_of_any_scale(B, rows, vocab, dtype, grad, k):
    """Scores that are shifted by up to 1000, so that their exponentials are out of fp32's range, or are spread over
    more than it.  q / Q is off by 4 U and by its exponent's rounding, U of |score| and of |score - largest|."""
    z = _normal(rows, vocab, dtype, 9)
    rng = np.random.default_rng(10)
    ids = torch.from_numpy(np.stack([rng.permutation(vocab)[:k] for _ in range(rows)]).astype(np.int32)).cuda()
    by = np.array([-1000.0, -104.0, -95.0, -88.0, -60.0, 0.0, 60.0, 89.0, 1000.0])
    spread = np.where(rng.random((rows, 1)) < 0.3, 100.0, 2.0)
    logq = torch.from_numpy(by[np.arange(rows) % 9][:, None] - spread * rng.random((rows, k))).float().cuda()
    loss = torch.empty(rows, device="cuda")
    g = torch.empty(rows, vocab, dtype=DT[grad], device="cuda") if grad else None
    B.sgd_kernel_distill(z, ids, logq, loss, grad=g, tail=B.TAIL_RENORM)
    assert B.sgd_kernel_status() == 0
    for r in sorted({*range(min(rows, 27)), rows - 1, *range(27, rows, max(1, rows // 9))}):
        at, lq = ids[r].cpu().numpy(), logq[r].double().cpu().numpy()
        x = z[r].double().cpu().numpy()
        L, want = ot.distill_row(x, at, lq, bucket=False)
        lp = ot.log_softmax(x[None])[0]
        lh = lq - lq.max()
        lh = lh - np.log(np.exp(lh).sum())
        q = np.exp(lh)
        eq = (8 + 2 * np.abs(lh) + np.abs(lh).max()) * U  # (expf, its rounded exponent, the sum, the quotient)
        terms = np.where(q > 0, np.abs(lh - lp[at]), 0.0)
        tol = 2 * SUM + (q * (eq * (terms + 1) + 4 * U * (terms + np.abs(lh)))).sum()
        assert abs(loss[r].item() - L) <= tol + U * abs(L), (r, loss[r].item(), L)
        if g is not None:
            tol = np.exp(lp) * (SUM + (4 + 3 * np.abs(lp)) * U)
            tol[at] += q * eq + 2.0 ** -126  # (an entry below 2^-126 of the largest may be 0)
            assert (np.abs(g[r].double().cpu().numpy() - want) <= tol + U * np.abs(want) + 2.0 ** -149).all(), r


@pytest.mark.parametrize("rows,vocab", [(0, 64), (0, 126464)])
def test_empty_tensors(B, rows, vocab):
    z = torch.empty(rows, vocab, dtype=torch.float16, device="cuda")
    ids, lq = torch.empty(rows, 4, dtype=torch.int32, device="cuda"), torch.empty(rows, 4, device="cuda")
    one = torch.empty(rows, device="cuda")
    B.sgd_kernel_logprobs(z, tokens=ids, token_logprobs=lq, entropy=one, top_ids=ids, top_logprobs=lq)
    B.sgd_kernel_logprobs(z, entropy=one, row_ids=torch.empty(rows, dtype=torch.int32, device="cuda"))
    B.sgd_kernel_distill(z, ids, lq, one, grad=torch.empty_like(z), row_weight=one)


@pytest.mark.parametrize("batch,n", [(0, 5), (3, 0), (0, 0)])
def test_reveal_of_empty_tensors(B, batch, n):
    ids, n_reveal = torch.empty(batch, n, dtype=torch.int32, device="cuda"), torch.ones(batch, dtype=torch.int32, device="cuda")
    left = torch.full((batch,), 9, dtype=torch.int32, device="cuda")
    window = torch.zeros(batch, 2, dtype=torch.int32, device="cuda")
    B.sgd_sampler_reveal(ids, ids, torch.empty(batch, n, device="cuda"), n_reveal, ids, 0)
    B.sgd_sampler_reveal(ids, ids, torch.empty(batch, n, device="cuda"), n_reveal, ids, 0, window=window, n_left=left)
    assert (left == 0).all()


def test_tokens_of_no_number_beside_another_output(B):
    z = _normal(3, 100, "f16", 1)
    e, none = torch.empty(3, device="cuda"), torch.empty(3, 0, device="cuda")
    B.sgd_kernel_logprobs(z, tokens=none.int(), token_logprobs=none, entropy=e, top_ids=none.int(), top_logprobs=none)
    want = torch.distributions.Categorical(logits=z.double()).entropy()
    assert ((e.double() - want).abs() < 4 * SUM * (1 + want)).all()


@pytest.mark.parametrize("rows,vocab", [(700, 49152), (600, 49151), (500, 70001), (400, 90001), (330, 100003)])
@pytest.mark.parametrize("k", [2, 64])
def test_lists_of_slices_of_few_tiles(B, rows, vocab, k):
    """3, 5, 6 and 7 tiles a row, after a call that leaves the largest values in every place of shared memory."""
    high = torch.full((320, 126464), 60000.0, dtype=torch.float16, device="cuda")
    ids, lp = torch.empty(320, 64, dtype=torch.int32, device="cuda"), torch.empty(320, 64, device="cuda")
    z = _normal(rows, vocab, "f16", 11)
    top, want = torch.empty(rows, k, dtype=torch.int32, device="cuda"), torch.empty(rows, k, device="cuda")
    for _ in range(3):
        B.sgd_kernel_logprobs(high, top_ids=ids, top_logprobs=lp)
        B.sgd_kernel_logprobs(z, top_ids=top, top_logprobs=want)
        order = torch.sort(z.float(), dim=1, descending=True, stable=True).indices[:, :k]
        assert torch.equal(top.long(), order)
    assert torch.equal(ids.long(), torch.arange(64, device="cuda").expand(320, 64))


def test_ids_of_more_than_32_bits_are_refused(B):
    """2^32 would be cut down to token 0."""
    z, e = _normal(2, 100, "f16", 1), torch.empty(2, device="cuda")
    ids = torch.zeros(2, dtype=torch.int32, device="cuda")
    for bad in (2 ** 32, 2 ** 31, -2 ** 31 - 1):
        with pytest.raises(ValueError, match="row_id"):
            B.sgd_kernel_logprobs(z, entropy=e, row_ids=ids, row_id=bad)
        with pytest.raises(ValueError, match="mask_id"):
            B.sgd_sampler_reveal(ids[None], ids[None], e[None], ids[:1], ids[None].clone(), bad)
