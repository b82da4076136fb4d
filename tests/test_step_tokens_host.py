"""What Denoiser.step_tokens refuses, before the model's step is launched (no GPU needed), and its limits as the library has
them."""
import os
import re

import pytest
import torch

from paper_2609_29505_gb300 import binding, synth


@pytest.fixture
def model():
    """A denoiser without a context, whose steps are counted."""
    m = binding.Denoiser.__new__(binding.Denoiser)
    m.cfg, m.steps = synth.get_config("llada_small"), 0

    def step(*a, **k):
        m.steps += 1
    m.step = step
    return m


def _args(cfg, **kw):
    shape = (cfg.batch, cfg.n_tokens)
    a = dict(ids=torch.zeros(shape, dtype=torch.int32), logits=torch.zeros(*shape, cfg.vocab, dtype=torch.float16), t=0.5, step=1,
             cand=torch.zeros(shape, dtype=torch.int32), score=torch.zeros(shape), n_reveal=torch.zeros(cfg.batch, dtype=torch.int32),
             mask_id=999)
    a["ids_out"] = a["ids"]
    a.update(kw)
    return a


B, N, V = 2, 192, 1000


@pytest.mark.parametrize("kw,error,match", [
    (dict(by="chance"), ValueError, "by must"),
    (dict(logits=torch.zeros(B, N, V)), TypeError, "logits"),
    (dict(logits=torch.zeros(B, N, V - 1, dtype=torch.float16)), ValueError, "logits"),
    (dict(logits=torch.zeros(B * N, V, dtype=torch.float16)), ValueError, "logits"),
    (dict(logits=torch.zeros(B, N, 2 * V, dtype=torch.float16)[:, :, :V]), ValueError, "contiguous"),
    (dict(ids=torch.zeros(B, N, dtype=torch.int64)), TypeError, "ids"),
    (dict(ids=torch.zeros(B, N - 1, dtype=torch.int32)), ValueError, "ids"),
    (dict(ids_out=torch.zeros(N, B, dtype=torch.int32).t()), ValueError, "contiguous"),
    (dict(ids_out=None), TypeError, "ids_out"),
    (dict(cand=torch.zeros(B, N, dtype=torch.int64)), TypeError, "cand"),
    (dict(cand=torch.zeros(B, N, 2, dtype=torch.int32)[:, :, 0]), ValueError, "cand"),
    (dict(score=torch.zeros(B, N, dtype=torch.float16)), TypeError, "score"),
    (dict(n_reveal=torch.zeros(B, dtype=torch.int64)), TypeError, "n_reveal"),
    (dict(n_reveal=torch.zeros(B + 1, dtype=torch.int32)), ValueError, "n_reveal"),
    (dict(window=torch.zeros(B, dtype=torch.int32)), ValueError, "window"),
    (dict(n_left=torch.zeros(1, dtype=torch.int32)), ValueError, "n_left"),
    (dict(class_ids=torch.zeros(B, dtype=torch.int64)), TypeError, "class_ids"),
    (dict(ctx=torch.zeros(B, 4, 8)), TypeError, "ctx"),
    (dict(ctx=torch.zeros(B, 4, 8, dtype=torch.bfloat16)), ValueError, "ctx"),
    (dict(scale=0.0), ValueError, "scale"),
    (dict(scale=1e-60), ValueError, "scale"),
    (dict(scale=1e60), ValueError, "scale"),
    (dict(scale=float("nan")), ValueError, "scale"),
    (dict(mask_id=2 ** 31), ValueError, "mask_id"),
    (dict(), ValueError, "CUDA"),
])
def test_step_tokens_refuses_before_the_step(model, kw, error, match):
    with pytest.raises(error, match=match):
        model.step_tokens(**_args(model.cfg, **kw))
    assert model.steps == 0


@pytest.mark.parametrize("change", [dict(head="linear"), dict(stem="patch"), dict(d_out=(3 << 19) + 1), dict(n_tokens=49153)])
def test_step_tokens_refuses_models(model, change):
    args = _args(model.cfg)
    model.cfg = model.cfg.with_(**change)
    with pytest.raises(ValueError):
        model.step_tokens(**args)
    assert model.steps == 0


def test_limits_follow_the_library():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = open(os.path.join(root, "paper_2609_29505_gb300", "csrc", "kernels.h")).read()
    assert re.search(r"kMaxRowBytes = 3ll << 20;", src) and binding.MAX_ROW_BYTES == 3 << 20
    assert int(re.search(r"kRevealMaxTokens = (\d+);", src).group(1)) == binding.REVEAL_MAX_TOKENS
