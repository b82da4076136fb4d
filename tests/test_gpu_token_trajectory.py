"""The operators on a token model's logits in a run together, as they are used: a masked-token trajectory whose positions
are revealed by the scheduled model's own logits, and the distillation of that model from the full one's
likeliest tokens.  Each step of the run is checked against oracle/tokens.py on the logits that the step wrote."""
import numpy as np
import pytest
import torch

from oracle import tokens as ot
from paper_2609_29505_gb300 import synth

pytestmark = pytest.mark.gpu

SUM = 186 * 2.0 ** -24  # of a row's sum (test_gpu_tokens.py)


@pytest.fixture(scope="module")
def models():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2609_29505_gb300 import binding, build, schedule
    build.build()
    cfg = synth.get_config("llada_small")
    w = {k: v.cuda() for k, v in synth.make_weights(cfg, "cpu").items()}
    made = {}
    for budget in (1.0, 0.5):
        s = schedule.build_schedule(cfg, w, cfg.T, budget=budget)
        m = binding.Denoiser(cfg, w)
        m.set_schedule(cfg.T, s["lifetimes"], s["groups"])
        made[budget] = m
    yield binding, cfg, made
    for m in made.values():
        m.close()


def _buffers(cfg):
    shape = (cfg.batch, cfg.n_tokens)
    return dict(ids=torch.full(shape, synth.mask_id(cfg), dtype=torch.int32, device="cuda"),
                cand=torch.full(shape, -5, dtype=torch.int32, device="cuda"), score=torch.full(shape, 9.0, device="cuda"),
                logits=torch.empty(*shape, cfg.vocab, dtype=torch.float16, device="cuda"),
                left=torch.empty(cfg.batch, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("by", ["confidence", "entropy"])
@pytest.mark.parametrize("blocks", [False, True])
def test_trajectory_reveals_what_the_logits_say(models, by, blocks):
    binding, cfg, made = models
    model, mask, T, N = made[0.5], synth.mask_id(cfg), cfg.T, cfg.n_tokens
    x = _buffers(cfg)
    model.reset()
    for s in range(1, T + 1):
        # whole samples, or two halves one after the other
        half, first = N // 2, s <= T // 2
        window = None
        steps = T
        if blocks:
            window = torch.tensor([[0, half] if first else [half, N]] * cfg.batch, dtype=torch.int32, device="cuda")
            steps = T // 2
        share = torch.full((cfg.batch,), (half if blocks else N) // steps, dtype=torch.int32, device="cuda")
        before, cand0, score0 = x["ids"].clone(), x["cand"].clone(), x["score"].clone()
        model.step_tokens(x["ids"], x["ids"], x["logits"], synth.timestep(cfg, s), s, x["cand"], x["score"], share, mask,
                          by=by, window=window, n_left=x["left"])
        torch.cuda.synchronize()
        masked = (before == mask).cpu().numpy()
        z = x["logits"].double().cpu().numpy().reshape(-1, cfg.vocab)
        lp = ot.log_softmax(z)
        best = ot.top(z, 1)[:, 0].reshape(masked.shape)
        cand, score = x["cand"].cpu().numpy(), x["score"].cpu().numpy()
        assert np.array_equal(cand[masked], best[masked]) and np.array_equal(cand[~masked], cand0.cpu().numpy()[~masked])
        assert np.array_equal(score[~masked], score0.cpu().numpy()[~masked])
        want = (lp.max(1) if by == "confidence" else ot.entropy(lp)).reshape(masked.shape)
        assert np.abs(score - want)[masked].max() <= SUM * (1 + 4 * np.abs(want).max() + 4 * np.abs(lp.max(1)).max())
        ids, left = ot.reveal(before.cpu().numpy(), cand, score, share.cpu().numpy(), mask, by == "entropy",
                              None if window is None else window.cpu().numpy())
        assert np.array_equal(x["ids"].cpu().numpy(), ids) and np.array_equal(x["left"].cpu().numpy(), left)
    assert (x["left"] == N - T * (N // T)).all()
    model.check_device()


def test_distillation_from_the_full_model(models):
    binding, cfg, made = models
    rows, k, V = cfg.batch * cfg.n_tokens, 16, cfg.vocab
    ids = synth.token_ids_at(cfg, synth.make_inputs(cfg, "cpu"), cfg.T).cuda()  # (the last step: earlier ones freeze nothing yet)
    logits = {}
    for budget, model in made.items():
        model.reset()
        out = torch.empty(cfg.batch, cfg.n_tokens, V, dtype=torch.float16, device="cuda")
        for s in range(1, cfg.T + 1):
            x = synth.token_ids_at(cfg, synth.make_inputs(cfg, "cpu"), s).cuda()
            model.step(x, out, synth.timestep(cfg, s), s)
        logits[budget] = out.view(rows, V)
    top, logq = torch.empty(rows, k, dtype=torch.int32, device="cuda"), torch.empty(rows, k, device="cuda")
    binding.sgd_kernel_logprobs(logits[1.0], top_ids=top, top_logprobs=logq)
    # only what is still masked counts
    w = (ids.view(-1) == synth.mask_id(cfg)).float()
    w /= w.sum()
    loss, grad = torch.empty(rows, device="cuda"), torch.empty(rows, V, device="cuda")
    binding.sgd_kernel_distill(logits[0.5], top, logq, loss, grad=grad, row_weight=w)
    total = loss.sum().item()
    z, tops, lqs, ws = logits[0.5].double().cpu().numpy(), top.cpu().numpy(), logq.double().cpu().numpy(), w.double().cpu().numpy()
    got_l, got_g = loss.double().cpu().numpy(), grad.double().cpu().numpy()
    for r in range(rows):
        L, g = ot.distill_row(z[r], tops[r], lqs[r], 1.0, True, ws[r])
        assert abs(got_l[r] - L) <= ws[r] * 4 * SUM * (1 + L / max(ws[r], 1e-30))
        assert np.abs(got_g[r] - g).max() <= ws[r] * 4 * SUM
    assert total > 0 and np.isfinite(total)
    # the full model against its own lists: nothing
    binding.sgd_kernel_distill(logits[1.0], top, logq, loss, grad=grad, row_weight=w)
    assert loss.abs().sum().item() < 4 * SUM and grad.abs().max().item() < 4 * SUM * w.max().item()
    for model in made.values():
        model.check_device()
