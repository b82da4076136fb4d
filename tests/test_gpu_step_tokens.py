"""Denoiser.step_tokens of a token model with cross-attention blocks: it takes the conditioning that step takes, and
gives what the step and the two operators give one after another."""
import pytest
import torch

from paper_2609_29505_gb300 import synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("by", ["confidence", "entropy"])
def test_a_model_with_cross_attention(by):
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2609_29505_gb300 import binding, build, schedule
    build.build()
    cfg = synth.get_config("sdxl_small").with_(name="tokens_xattn", stem="embed", head="logits", vocab=1000, d_in=0, d_out=1000,
                                               out_channels=1000, T=3)
    w = {k: v.cuda() for k, v in synth.make_weights(cfg, "cpu").items()}
    ctx = synth.make_inputs(cfg, "cpu").ctx.cuda()
    s = schedule.build_schedule(cfg, w, cfg.T, budget=1.0)
    model = binding.Denoiser(cfg, w)
    model.set_schedule(cfg.T, s["lifetimes"], s["groups"])
    mask, shape = synth.mask_id(cfg), (cfg.batch, cfg.n_tokens)
    share = torch.full((cfg.batch,), 60, dtype=torch.int32, device="cuda")

    def buffers():
        return (torch.full(shape, mask, dtype=torch.int32, device="cuda"), torch.full(shape, -5, dtype=torch.int32, device="cuda"),
                torch.full(shape, 9.0, device="cuda"), torch.empty(*shape, cfg.vocab, dtype=torch.float16, device="cuda"))
    runs = []
    for together in (True, False):
        ids, cand, score, logits = buffers()
        model.reset()
        for step in range(1, cfg.T + 1):
            t = synth.timestep(cfg, step)
            if together:
                model.step_tokens(ids, ids, logits, t, step, cand, score, share, mask, by=by, ctx=ctx)
                continue
            model.step(ids, logits, t, step, ctx=ctx)
            out = dict(top_logprobs=score.view(-1, 1)) if by == "confidence" else dict(entropy=score.view(-1))
            binding.sgd_kernel_logprobs(logits.view(-1, cfg.vocab), top_ids=cand.view(-1, 1), row_ids=ids.view(-1), row_id=mask, **out)
            binding.sgd_sampler_reveal(ids, cand, score, share, ids, mask, lowest=by == "entropy")
        runs.append((ids, cand, score, logits))
    for a, b in zip(*runs):
        assert torch.equal(a, b)
    assert int((runs[0][0] != mask).sum()) >= 2 * 3 * 50  # (a best token may be the mask)
    model.check_device()
    model.close()


def test_a_candidate_that_is_the_mask():
    """It is taken, leaves its position masked, and counts as chosen."""
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2609_29505_gb300 import binding, build
    build.build()
    ids = torch.full((1, 6), 7, dtype=torch.int32, device="cuda")
    cand = torch.tensor([[7, 1, 2, 7, 3, 4]], dtype=torch.int32, device="cuda")
    score = torch.tensor([[5.0, 4.0, 3.0, 2.0, 1.0, 0.0]], device="cuda")
    out, left = torch.empty_like(ids), torch.empty(1, dtype=torch.int32, device="cuda")
    binding.sgd_sampler_reveal(ids, cand, score, torch.tensor([4], dtype=torch.int32, device="cuda"), out, 7, n_left=left)
    assert out.tolist() == [[7, 1, 2, 7, 7, 7]] and left.tolist() == [2]
