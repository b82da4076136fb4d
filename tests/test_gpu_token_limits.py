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
