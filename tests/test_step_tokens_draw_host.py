"""What Denoiser.step_tokens refuses of drawn candidates, before the model's step is launched (no GPU needed)."""
import pytest
import torch

from paper_2609_29505_gb300 import binding, synth


@pytest.mark.parametrize("kw,error,match", [
    (dict(top_k=5), ValueError, "uniforms"),
    (dict(top_p=0.9), ValueError, "uniforms"),
    (dict(min_p=0.1), ValueError, "uniforms"),
    (dict(uniforms=torch.zeros(2, 192)), ValueError, "uniforms"),
    (dict(uniforms=torch.zeros(2, 192, 2).double()), TypeError, "uniforms"),
    (dict(uniforms=torch.zeros(2, 2, 192).transpose(1, 2)), ValueError, "contiguous"),
    (dict(uniforms=torch.zeros(2, 192, 2), top_k=-1), ValueError, "top_k"),
    (dict(uniforms=torch.zeros(2, 192, 2), top_k=2 ** 31), ValueError, "top_k"),
    (dict(uniforms=torch.zeros(2, 192, 2), top_p=0.0), ValueError, "top_p"),
    (dict(uniforms=torch.zeros(2, 192, 2), top_p=1.5), ValueError, "top_p"),
    (dict(uniforms=torch.zeros(2, 192, 2), top_p=float("nan")), ValueError, "top_p"),
    (dict(uniforms=torch.zeros(2, 192, 2), min_p=-0.1), ValueError, "min_p"),
    (dict(uniforms=torch.zeros(2, 192, 2), min_p=1.1), ValueError, "min_p"),
    (dict(uniforms=torch.zeros(2, 192, 2)), ValueError, "CUDA"),  # (all of it is on the CPU here)
])
def test_step_tokens_refuses(kw, error, match):
    m = binding.Denoiser.__new__(binding.Denoiser)
    m.cfg, m.steps = synth.get_config("llada_small"), 0

    def step(*a, **k):
        m.steps += 1
    m.step = step
    shape = (m.cfg.batch, m.cfg.n_tokens)
    assert shape == (2, 192)
    ids = torch.zeros(shape, dtype=torch.int32)
    with pytest.raises(error, match=match):
        m.step_tokens(ids, ids, torch.zeros(*shape, m.cfg.vocab, dtype=torch.float16), 0.5, 1, torch.zeros_like(ids), torch.zeros(shape),
                      torch.zeros(2, dtype=torch.int32), 999, **kw)
    assert m.steps == 0
