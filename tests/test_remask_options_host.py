"""The command's remasking trajectory (kernel_bench trajectory --remask): which options draw its candidates (no GPU needed)."""
import json
import types

import pytest
import torch

from paper_2609_29505_gb300 import binding, build, kernel_bench, synth


@pytest.mark.parametrize("options,want", [
    ([], None),
    (["--temperature", "1"], dict(scale=1.0, top_k=0, top_p=1.0, min_p=0.0)),
    (["--temperature", "1.0"], dict(scale=1.0, top_k=0, top_p=1.0, min_p=0.0)),
    (["--temperature", "0.5"], dict(scale=2.0, top_k=0, top_p=1.0, min_p=0.0)),
    (["--top-p", "0.9"], dict(scale=1.0, top_k=0, top_p=0.9, min_p=0.0)),
    (["--temperature", "1", "--top-k", "5"], dict(scale=1.0, top_k=5, top_p=1.0, min_p=0.0)),
    (["--min-p", "0.1"], dict(scale=1.0, top_k=0, top_p=1.0, min_p=0.1)),
])
def test_which_options_draw(monkeypatch, capsys, options, want):
    """No option takes the best token; any temperature, 1 among them, or a filter draws, by numbers of each step's own."""
    def here(f):
        return lambda *a, device=None, **kw: f(*a, **kw)
    cfg, calls = synth.get_config("llada_small"), []
    on_cpu = types.SimpleNamespace(**{n: here(getattr(torch, n)) for n in ("full", "empty", "rand", "empty_like")}, int32=torch.int32)
    model = types.SimpleNamespace(step_tokens=lambda *a, **kw: calls.append(kw))

    def case(a):
        run, _ = kernel_bench._remask(a, cfg, model, None)
        run()
        return {}
    monkeypatch.setattr(kernel_bench, "torch", on_cpu)
    monkeypatch.setattr(kernel_bench, "case_trajectory", case)
    monkeypatch.setattr(build, "build", lambda: None)
    monkeypatch.setattr(binding, "lib", lambda: None)
    monkeypatch.setattr(binding, "sgd_kernel_status", lambda: 0)
    monkeypatch.setattr("sys.argv", ["kernel_bench", "trajectory", "--T", "3", "--remask", "confidence", *options])
    kernel_bench.main()
    assert json.loads(capsys.readouterr().out)["status"] == 0
    assert len(calls) == 3
    if want is None:
        assert all("uniforms" not in c and "scale" not in c for c in calls)
        return
    for c in calls:
        assert {k: c[k] for k in want} == want
        assert c["uniforms"].shape == (cfg.batch, cfg.n_tokens, 2)
    assert not torch.equal(calls[0]["uniforms"], calls[1]["uniforms"])
