"""The operators at a token model's two ends in a run together, as they are used: a masked-token trajectory whose candidates are drawn
from the scheduled model's own logits, each step checked against oracle/ends.py on the logits that the step wrote; and training
steps of an embedding, a norm and a head on the distillation loss, whose gradients are checked against automatic differentiation in
float64."""
import math

import numpy as np
import pytest
import torch

from oracle import ends as oe
from oracle import tokens as ot
from paper_2609_29505_gb300 import synth

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
NEAR = 9e-9  # of a draw to another token (test_gpu_sample.py)


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2609_29505_gb300 import binding, build
    build.build()
    binding.lib()
    return binding


@pytest.mark.parametrize("by", ["confidence", "entropy"])
@pytest.mark.parametrize("kw", [dict(), dict(top_p=0.8, scale=1.25), dict(top_k=20, min_p=0.01)])
def test_trajectory_draws_from_the_logits(B, by, kw):
    from paper_2609_29505_gb300 import schedule
    cfg = synth.get_config("llada_small")
    w = {k: v.cuda() for k, v in synth.make_weights(cfg, "cpu").items()}
    s = schedule.build_schedule(cfg, w, cfg.T, budget=0.5)
    model = B.Denoiser(cfg, w)
    model.set_schedule(cfg.T, s["lifetimes"], s["groups"])
    mask, shape = synth.mask_id(cfg), (cfg.batch, cfg.n_tokens)
    ids = torch.full(shape, mask, dtype=torch.int32, device="cuda")
    cand, score = torch.full(shape, -5, dtype=torch.int32, device="cuda"), torch.full(shape, 9.0, device="cuda")
    logits = torch.empty(*shape, cfg.vocab, dtype=torch.float16, device="cuda")
    left = torch.empty(cfg.batch, dtype=torch.int32, device="cuda")
    share = torch.full((cfg.batch,), cfg.n_tokens // cfg.T, dtype=torch.int32, device="cuda")
    gen = torch.Generator().manual_seed(0)
    scale = kw.get("scale", 1.0)
    for step in range(1, cfg.T + 1):
        u = torch.rand(*shape, 2, generator=gen)
        before, cand0, score0 = ids.clone(), cand.cpu().numpy(), score.cpu().numpy()
        model.step_tokens(ids, ids, logits, synth.timestep(cfg, step), step, cand, score, share, mask, by=by, n_left=left, uniforms=u.cuda(), **kw)
        masked = (before == mask).cpu().numpy()
        z = logits.double().cpu().numpy()
        lp = ot.log_softmax(z.reshape(-1, cfg.vocab), scale).reshape(z.shape)
        got, got_score = cand.cpu().numpy(), score.cpu().numpy()
        for b, n in zip(*np.nonzero(masked)):
            want, _, near = oe.sample(z[b, n], u[b, n].double().numpy(), **kw)
            assert got[b, n] == want or near <= NEAR
        want = np.take_along_axis(lp, got[..., None].clip(0), 2)[..., 0] if by == "confidence" else ot.entropy(lp)
        tol = 186 * U * (1 + 4 * np.abs(want).max() + 4 * np.abs(lp.max(2)).max())  # (test_gpu_token_trajectory.py)
        assert np.abs(got_score - want)[masked].max() <= tol
        assert np.array_equal(got[~masked], cand0[~masked]) and np.array_equal(got_score[~masked], score0[~masked])
        want_ids, want_left = ot.reveal(before.cpu().numpy(), got, got_score, share.cpu().numpy(), mask, by == "entropy")
        assert np.array_equal(ids.cpu().numpy(), want_ids) and np.array_equal(left.cpu().numpy(), want_left)
    model.check_device()
    model.close()


class _Ends:
    """An embedding, an RMS norm and a head of V tokens, trained on a teacher's lists; the products are the caller's own."""

    def __init__(self, B, V, d, rows, k):
        gen = torch.Generator().manual_seed(5)
        self.B, self.scale = B, math.sqrt(d)
        self.table = (0.2 * torch.randn(V, d, generator=gen)).cuda()
        self.g = (1 + 0.1 * torch.randn(d, generator=gen)).bfloat16().cuda()
        self.head = (torch.randn(V, d, generator=gen) / math.sqrt(d)).cuda()
        self.ids = torch.randint(0, V, (rows,), generator=gen, dtype=torch.int32).cuda()
        self.ids[::3] = V - 1
        self.ids[5] = -1
        self.teacher = torch.randint(0, V, (rows, k), generator=gen, dtype=torch.int32).cuda()
        self.logq = torch.log_softmax(torch.randn(rows, k, generator=gen), 1).cuda()
        self.h, self.n = torch.empty(rows, d, device="cuda"), torch.empty(rows, d, device="cuda", dtype=torch.float16)
        self.z = torch.empty(rows, V, device="cuda")
        self.loss, self.dz = torch.empty(rows, device="cuda"), torch.empty(rows, V, device="cuda")
        self.dn, self.dh = torch.empty(rows, d, device="cuda"), torch.empty(rows, d, device="cuda")
        self.dg, self.dtable = torch.empty(d, device="cuda"), torch.empty(V, d, device="cuda")
        self.dhead = torch.empty(V, d, device="cuda")
        self.ws = torch.empty(max(B.sgd_kernel_embedding_grad_workspace(rows, V, d), B.sgd_kernel_norm_grad_workspace(rows, d)),
                              dtype=torch.uint8, device="cuda")

    def step(self):
        B, (rows, d) = self.B, self.h.shape
        B.sgd_kernel_embedding(self.table, self.ids, self.h, scale=self.scale)
        B.sgd_kernel_norm(self.h, self.n, rows, d, 0, g=self.g)
        torch.matmul(self.n.float(), self.head.t(), out=self.z)
        B.sgd_kernel_distill(self.z, self.teacher, self.logq, self.loss, grad=self.dz)
        torch.matmul(self.dz, self.head, out=self.dn)
        torch.matmul(self.dz.t(), self.n.float(), out=self.dhead)
        B.sgd_kernel_norm_grad(self.dn, self.h, 0, dh=self.dh, g=self.g, dg=self.dg, workspace=self.ws)
        B.sgd_kernel_embedding_grad(self.dh, self.ids, self.dtable, scale=self.scale, workspace=self.ws)


@pytest.mark.parametrize("V,d,rows", [(300, 64, 90), (1000, 256, 192)])
def test_training_step_of_both_ends(B, V, d, rows):
    torch.backends.cuda.matmul.allow_tf32 = False
    e = _Ends(B, V, d, rows, 6)
    e.step()
    table, g, head = e.table.double().requires_grad_(), e.g.double().requires_grad_(), e.head.double()
    here = (e.ids >= 0)[:, None]
    h = torch.where(here, table[e.ids.long().clamp(min=0)], 0.0) * float(np.float32(e.scale))
    n = h / torch.sqrt(h.pow(2).mean(1, keepdim=True) + 1e-6) * g
    z = n @ head.t()
    # (the list's first occurrence of a token counts; what is left of 1 is the tail's, here nothing)
    lp, same = torch.log_softmax(z, 1), torch.tril(e.teacher[:, :, None] == e.teacher[:, None, :], -1).any(2)
    q = torch.where(same, 0.0, e.logq.double().exp())
    inside = torch.zeros_like(z, dtype=torch.bool).scatter_(1, e.teacher.long(), True)
    qt = (1 - q.sum(1)).clamp(min=0)
    lpt = torch.logsumexp(torch.where(inside, -math.inf, lp), 1)
    loss = (torch.xlogy(q, q) - q * torch.gather(lp, 1, e.teacher.long())).sum(1) + torch.xlogy(qt, qt) - qt * lpt
    loss.sum().backward()
    # The normed rows are fp16 (2^-11 of them): logits of sqrt(d) such terms of 1 / sqrt(d) are off by some 2^-11, and dz as much relative to p
    # and q.  What comes back sums V terms of the head, and of a token's rows, so that errors of 2^-11 a term stay below ten times
    # that of the gradients' norms.
    assert (e.loss.double() - loss.detach()).abs().max() <= 10 * 2.0 ** -11
    for got, want in ((e.dtable, table.grad), (e.dg, g.grad)):
        assert (got.double() - want).norm() <= 10 * 2.0 ** -11 * want.norm()
    assert (e.dtable[~torch.isin(torch.arange(V, device="cuda"), e.ids)] == 0).all()


def test_training_step_in_a_graph(B):
    """The step captured once and replayed over changed parameters gives what the calls give one after another."""
    e, f = _Ends(B, 300, 64, 90, 6), _Ends(B, 300, 64, 90, 6)
    e.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        e.step()
    for _ in range(3):
        graph.replay()
        f.step()
        for name in ("loss", "dh", "dg", "dtable", "dhead"):
            assert torch.equal(getattr(e, name), getattr(f, name)), name
        for x in (e, f):
            x.table -= 0.05 * x.dtable
            x.g -= (0.05 * x.dg).bfloat16()
            x.head -= 0.05 * x.dhead
    # the trained logits are drawn from
    u = torch.rand(90, 2, device="cuda")
    a, b = torch.empty(90, dtype=torch.int32, device="cuda"), torch.empty(90, dtype=torch.int32, device="cuda")
    B.sgd_kernel_sample(e.z, u, a, top_p=0.9)
    B.sgd_kernel_sample(f.z, u, b, top_p=0.9)
    assert torch.equal(a, b) and (a >= 0).all() and (a < 300).all()
