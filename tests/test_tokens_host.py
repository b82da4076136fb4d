"""Refusals of the operators on a token model's logits, before the device is touched (no GPU needed)."""
import math

import numpy as np
import pytest
import torch

from paper_2609_29505_gb300 import binding


@pytest.fixture(scope="module")
def lib():
    from paper_2609_29505_gb300 import build
    build.build()
    return binding.lib()


P = 4096  # an address that nothing reads


def _logprobs(lib, **kw):
    a = dict(logits=P, dtype=0, ld=64, rows=2, vocab=64, scale=1.0, row_ids=None, row_id=0, tokens=P, n_tokens=1,
             token_logprobs=P, entropy=P, top_k=2, top_ids=P, top_logprobs=P, stream=None)
    a.update(kw)
    return lib.sgd_kernel_logprobs(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(logits=None), binding.SGD_ERR_ARG),
    (dict(dtype=3), binding.SGD_ERR_ARG),
    (dict(dtype=-1), binding.SGD_ERR_ARG),
    (dict(rows=-1), binding.SGD_ERR_ARG),
    (dict(vocab=0), binding.SGD_ERR_ARG),
    (dict(ld=63), binding.SGD_ERR_ARG),
    (dict(ld=0), binding.SGD_ERR_ARG),
    (dict(ld=-64), binding.SGD_ERR_ARG),
    (dict(scale=0.0), binding.SGD_ERR_ARG),
    (dict(scale=-1.0), binding.SGD_ERR_ARG),
    (dict(scale=math.inf), binding.SGD_ERR_ARG),
    (dict(scale=math.nan), binding.SGD_ERR_ARG),
    (dict(logits=P + 1), binding.SGD_ERR_ARG),
    (dict(logits=P + 2, dtype=2), binding.SGD_ERR_ARG),
    (dict(entropy=P + 2), binding.SGD_ERR_ARG),
    (dict(row_ids=P + 1), binding.SGD_ERR_ARG),
    (dict(n_tokens=-1), binding.SGD_ERR_ARG),
    (dict(n_tokens=0), binding.SGD_ERR_ARG),
    (dict(tokens=None), binding.SGD_ERR_ARG),
    (dict(token_logprobs=None), binding.SGD_ERR_ARG),
    (dict(top_k=65, vocab=100, ld=100), binding.SGD_ERR_ARG),
    (dict(top_k=-1), binding.SGD_ERR_ARG),
    (dict(top_k=3, vocab=2), binding.SGD_ERR_ARG),
    (dict(top_k=0), binding.SGD_ERR_ARG),
    (dict(top_ids=None, top_logprobs=None), binding.SGD_ERR_ARG),
    (dict(tokens=None, token_logprobs=None, n_tokens=0, entropy=None, top_k=0, top_ids=None, top_logprobs=None),
     binding.SGD_ERR_ARG),
    (dict(vocab=(3 << 19) + 1, ld=1 << 22), binding.SGD_ERR_SHAPE),
    (dict(dtype=2, vocab=(3 << 18) + 1, ld=1 << 22), binding.SGD_ERR_SHAPE),
    (dict(rows=(1 << 27)), binding.SGD_ERR_SHAPE),
    (dict(rows=0), binding.SGD_OK),
])
def test_logprobs_refuses(lib, kw, code):
    assert _logprobs(lib, **kw) == code
    assert code == binding.SGD_OK or b"logprobs" in lib.sgd_last_error()


def _distill(lib, **kw):
    a = dict(logits=P, dtype=0, ld=64, rows=2, vocab=64, scale=1.0, ids=P, logq=P, top_k=2, weight=None, tail=1,
             loss=P, grad=2 * P, grad_dtype=0, ld_grad=64, stream=None)
    a.update(kw)
    return lib.sgd_kernel_distill(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(logits=None), binding.SGD_ERR_ARG),
    (dict(dtype=9), binding.SGD_ERR_ARG),
    (dict(scale=0.0), binding.SGD_ERR_ARG),
    (dict(ids=None), binding.SGD_ERR_ARG),
    (dict(logq=None), binding.SGD_ERR_ARG),
    (dict(loss=None), binding.SGD_ERR_ARG),
    (dict(loss=P + 2), binding.SGD_ERR_ARG),
    (dict(weight=P + 1), binding.SGD_ERR_ARG),
    (dict(top_k=0), binding.SGD_ERR_ARG),
    (dict(top_k=65), binding.SGD_ERR_ARG),
    (dict(tail=2), binding.SGD_ERR_ARG),
    (dict(grad_dtype=3), binding.SGD_ERR_ARG),
    (dict(ld_grad=63), binding.SGD_ERR_ARG),
    (dict(grad=2 * P + 2, grad_dtype=2), binding.SGD_ERR_ARG),
    # overlapping without being the logits: another place, another type, other rows
    (dict(grad=P + 2), binding.SGD_ERR_ARG),
    (dict(grad=P + 2 * 127), binding.SGD_ERR_ARG),
    (dict(grad=P - 2), binding.SGD_ERR_ARG),
    (dict(grad=P, grad_dtype=1), binding.SGD_ERR_ARG),
    (dict(grad=P, ld_grad=72), binding.SGD_ERR_ARG),
    (dict(vocab=(3 << 19) + 1, ld=1 << 22, grad=None), binding.SGD_ERR_SHAPE),
    (dict(rows=0), binding.SGD_OK),
    (dict(rows=0, grad=P), binding.SGD_OK),
    (dict(rows=0, grad=None, grad_dtype=7, ld_grad=0), binding.SGD_OK),
])
def test_distill_refuses(lib, kw, code):
    assert _distill(lib, **kw) == code
    assert code == binding.SGD_OK or b"distill" in lib.sgd_last_error()


def _reveal(lib, **kw):
    a = dict(ids=P, cand=P, cand_stride=1, score=P, score_stride=1, lowest=0, n_reveal=P, window=None, ids_out=P,
             n_left=None, batch=2, n_tokens=64, mask_id=0, stream=None)
    a.update(kw)
    return lib.sgd_sampler_reveal(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(ids=None), binding.SGD_ERR_ARG),
    (dict(cand=None), binding.SGD_ERR_ARG),
    (dict(score=None), binding.SGD_ERR_ARG),
    (dict(n_reveal=None), binding.SGD_ERR_ARG),
    (dict(ids_out=None), binding.SGD_ERR_ARG),
    (dict(batch=-1), binding.SGD_ERR_ARG),
    (dict(n_tokens=-1), binding.SGD_ERR_ARG),
    (dict(cand_stride=0), binding.SGD_ERR_ARG),
    (dict(score_stride=0), binding.SGD_ERR_ARG),
    (dict(score=P + 2), binding.SGD_ERR_ARG),
    (dict(window=P + 1), binding.SGD_ERR_ARG),
    (dict(n_left=P + 1), binding.SGD_ERR_ARG),
    (dict(n_tokens=49153), binding.SGD_ERR_SHAPE),
    (dict(batch=0), binding.SGD_OK),
    (dict(n_tokens=0), binding.SGD_OK),
])
def test_reveal_refuses(lib, kw, code):
    assert _reveal(lib, **kw) == code
    assert code == binding.SGD_OK or b"reveal" in lib.sgd_last_error()


def test_binding_refuses_what_the_pointers_cannot_show():
    z = torch.zeros(2, 8)
    with pytest.raises(ValueError, match="CUDA"):
        binding.sgd_kernel_logprobs(z, entropy=torch.zeros(2))
    with pytest.raises(TypeError, match="float16"):
        binding.sgd_kernel_logprobs(z.double(), entropy=torch.zeros(2))
    with pytest.raises(ValueError, match="CUDA"):
        binding.sgd_kernel_distill(z, torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, 1), torch.zeros(2))
    ids = torch.zeros(2, 8, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        binding.sgd_sampler_reveal(ids, ids, z, ids[:, 0], ids, 0)
    # shapes, types, layouts and devices of the single arguments
    cpu = torch.device("cpu")
    with pytest.raises(TypeError):
        binding._tensor(z, "x", torch.int32, (2, 8), cpu)
    with pytest.raises(ValueError, match="shape"):
        binding._tensor(z, "x", torch.float32, (2, 9), cpu)
    with pytest.raises(ValueError, match="contiguous"):
        binding._tensor(torch.zeros(8, 2).t(), "x", torch.float32, (2, 8), cpu)
    with pytest.raises(ValueError, match="is on"):
        binding._tensor(z, "x", torch.float32, (2, 8), torch.device("cuda:0"))
    assert binding._column(torch.zeros(2, 8, 3)[:, :, 1], "x", torch.float32, (2, 8), cpu)[1] == 3
    assert binding._column(torch.zeros(2, 1, 3)[:, :, 1], "x", torch.float32, (2, 1), cpu)[1] == 3
    for bad in (torch.zeros(2, 9)[:, :8], torch.zeros(2, 1).expand(2, 8), torch.zeros(1, 1).expand(2, 8)):
        with pytest.raises(ValueError, match="evenly"):
            binding._column(bad, "x", torch.float32, (2, 8), cpu)


def test_type_codes_follow_the_header():
    import os
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = open(os.path.join(root, "include", "sgd_kernels.h")).read()
    want = {n: int(v) for n, v in re.findall(r"\b(SGD_(?:F16|BF16|F32|TAIL_RENORM|TAIL_BUCKET)) = (\d)", src)}
    assert want == {"SGD_F16": binding.DTYPES["float16"], "SGD_BF16": binding.DTYPES["bfloat16"],
                    "SGD_F32": binding.DTYPES["float32"], "SGD_TAIL_RENORM": binding.TAIL_RENORM,
                    "SGD_TAIL_BUCKET": binding.TAIL_BUCKET}
