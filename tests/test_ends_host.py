"""Refusals of the operators at a token model's two ends, before the device is touched (no GPU needed)."""
import ctypes as C
import math

import pytest
import torch

from paper_2609_29505_gb300 import binding

P = 1 << 20  # an address that nothing reads
ARG, SHAPE, OK = binding.SGD_ERR_ARG, binding.SGD_ERR_SHAPE, binding.SGD_OK


@pytest.fixture(scope="module")
def lib():
    from paper_2609_29505_gb300 import build
    build.build()
    return binding.lib()


def _sample(lib, **kw):
    a = dict(logits=P, dtype=0, ld=64, rows=2, vocab=64, scale=1.0, top_k=0, top_p=1.0, min_p=0.0, uniforms=P, row_ids=None, row_id=0,
             ids=P, logprobs=None, stream=None)
    a.update(kw)
    return lib.sgd_kernel_sample(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(logits=None), ARG), (dict(uniforms=None), ARG), (dict(ids=None), ARG), (dict(dtype=3), ARG), (dict(rows=-1), ARG),
    (dict(vocab=0), ARG), (dict(ld=63), ARG), (dict(scale=0.0), ARG), (dict(scale=math.inf), ARG), (dict(scale=math.nan), ARG),
    (dict(scale=2.1e38), ARG), (dict(top_k=-1), ARG), (dict(top_p=0.0), ARG), (dict(top_p=-0.5), ARG), (dict(top_p=1.0001), ARG),
    (dict(top_p=math.nan), ARG), (dict(min_p=-0.1), ARG), (dict(min_p=1.1), ARG), (dict(min_p=math.nan), ARG),
    (dict(uniforms=P + 2), ARG), (dict(ids=P + 1), ARG), (dict(logprobs=P + 2), ARG), (dict(row_ids=P + 2), ARG),
    (dict(logits=P + 1), ARG), (dict(vocab=(3 << 19) + 1, ld=1 << 22), SHAPE), (dict(rows=1 << 27), SHAPE),
    (dict(rows=0), OK), (dict(rows=0, logits=None, uniforms=None, ids=None), OK), (dict(rows=0, top_p=0.0), ARG),
])
def test_sample_refuses(lib, kw, code):
    assert _sample(lib, **kw) == code
    assert code == OK or b"sample" in lib.sgd_last_error()


def _embedding(lib, **kw):
    a = dict(table=P, dtype=1, ld=8, vocab=4, d=8, ids=2 * P, rows=2, scale=1.0, out=3 * P, out_dtype=2, ld_out=8, stream=None)
    a.update(kw)
    return lib.sgd_kernel_embedding(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(table=None), ARG), (dict(ids=None), ARG), (dict(out=None), ARG), (dict(dtype=3), ARG), (dict(out_dtype=-1), ARG),
    (dict(ld=7), ARG), (dict(ld_out=7), ARG), (dict(vocab=0), ARG), (dict(d=0), ARG), (dict(rows=-1), ARG), (dict(table=P + 1), ARG),
    (dict(out=3 * P + 2), ARG), (dict(ids=2 * P + 2), ARG), (dict(out=P), ARG), (dict(out=P + 60), ARG), (dict(out=2 * P + 4), ARG),
    (dict(d=(1 << 20) + 1, ld=1 << 21, ld_out=1 << 21), SHAPE), (dict(rows=1 << 27), SHAPE), (dict(ld=1 << 41), SHAPE),
    (dict(rows=0), OK), (dict(rows=0, table=None, ids=None, out=None), OK),
])
def test_embedding_refuses(lib, kw, code):
    assert _embedding(lib, **kw) == code
    assert code == OK or b"embedding" in lib.sgd_last_error()


def _need(lib, rows, vocab, d):
    n = C.c_int64(0)
    assert lib.sgd_kernel_embedding_grad_workspace(rows, vocab, d, C.byref(n)) == OK
    return n.value


def _embedding_grad(lib, **kw):
    a = dict(grad=P, grad_dtype=1, ld_grad=8, ids=2 * P, rows=2, vocab=4, d=8, scale=1.0, accumulate=0, dtable=3 * P, dtable_dtype=2,
             ld=8, workspace=4 * P, workspace_bytes=_need(lib, 2, 4, 8), stream=None)
    a.update(kw)
    return lib.sgd_kernel_embedding_grad(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(grad=None), ARG), (dict(ids=None), ARG), (dict(dtable=None), ARG), (dict(grad_dtype=3), ARG), (dict(dtable_dtype=7), ARG),
    (dict(ld_grad=7), ARG), (dict(ld=7), ARG), (dict(vocab=0), ARG), (dict(d=0), ARG), (dict(rows=-1), ARG), (dict(grad=P + 1), ARG),
    (dict(dtable=3 * P + 2), ARG), (dict(ids=2 * P + 1), ARG), (dict(workspace=None), ARG), (dict(workspace=4 * P + 8), ARG),
    (dict(workspace_bytes=10), ARG), (dict(dtable=P + 16), ARG), (dict(dtable=2 * P), ARG), (dict(dtable=4 * P + 64), ARG), (dict(workspace=P), ARG),
    (dict(workspace=2 * P), ARG),
    (dict(d=(1 << 20) + 1, ld=1 << 21, ld_grad=1 << 21), SHAPE), (dict(rows=1 << 27), SHAPE),
])
def test_embedding_grad_refuses(lib, kw, code):
    assert _embedding_grad(lib, **kw) == code
    assert b"embedding_grad" in lib.sgd_last_error()


def test_embedding_grad_of_no_rows_without_a_table_to_clear(lib):
    assert _embedding_grad(lib, rows=0, grad=None, ids=None, accumulate=1, workspace=None, workspace_bytes=0) == OK


@pytest.mark.parametrize("a", [(-1, 4, 8), (2, 0, 8), (2, 4, 0)])
def test_workspace_of_no_call(lib, a):
    n = C.c_int64(0)
    assert lib.sgd_kernel_embedding_grad_workspace(*a, C.byref(n)) == ARG
    assert lib.sgd_kernel_embedding_grad_workspace(2, 4, 8, None) == ARG


def test_workspace_sizes_are_bounded(lib):
    # order and tokens, and two rows of partial sums per 16 rows or more
    for rows, d in ((1, 1), (17, 300), (8192, 4096), (8193, 4096), (65536, 64), (1 << 20, 64)):
        n = _need(lib, rows, 1000, d)
        assert 8 * rows <= n <= 24 * rows + 8 * (d + 8) * (rows // 16 + 2) + 8192


def _norm_grad(lib, **kw):
    a = dict(h=P, dout=2 * P, dtype=1, rows=2, d=8, kind=0, g=3 * P, b=None, scale=None, ld_mod=0, rows_per_batch=1, eps=1e-6,
             residual=None, dh=4 * P, dg=5 * P, db=None, dshift=None, dscale=None, ld_dmod=0, workspace=6 * P, workspace_bytes=1 << 16,
             stream=None)
    a.update(kw)
    return lib.sgd_kernel_norm_grad(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(h=None), ARG), (dict(dout=None), ARG), (dict(dtype=3), ARG), (dict(d=6), ARG), (dict(d=0), ARG), (dict(d=4100), ARG),
    (dict(rows=-1), ARG), (dict(kind=3), ARG), (dict(g=None), ARG), (dict(db=5 * P), ARG), (dict(dshift=5 * P), ARG),
    (dict(dscale=5 * P), ARG), (dict(dh=None, dg=None), ARG), (dict(dh=None, residual=7 * P), ARG), (dict(h=P + 4), ARG),
    (dict(dh=4 * P + 8), ARG), (dict(dout=2 * P + 4), ARG), (dict(dout=2 * P + 8, dtype=2), ARG), (dict(g=3 * P + 2), ARG),
    (dict(dg=5 * P + 4), ARG), (dict(residual=7 * P + 4), ARG), (dict(workspace=None), ARG), (dict(workspace=6 * P + 8), ARG),
    (dict(workspace_bytes=63), ARG), (dict(scale=7 * P, ld_mod=7), ARG), (dict(scale=7 * P, ld_mod=8, rows_per_batch=0), ARG),
    (dict(scale=7 * P, ld_mod=8, dscale=8 * P, ld_dmod=7), ARG), (dict(scale=7 * P + 2, ld_mod=8), ARG),
    (dict(dh=P), ARG), (dict(dh=P + 16), ARG), (dict(dh=2 * P), ARG), (dict(dh=4 * P, residual=4 * P + 16), ARG),
    (dict(rows=1 << 27), SHAPE),
])
def test_norm_grad_refuses(lib, kw, code):
    assert _norm_grad(lib, **kw) == code
    assert b"norm_grad" in lib.sgd_last_error()


def test_norm_grad_of_no_rows(lib):
    assert _norm_grad(lib, rows=0, h=None, dout=None, dg=None, workspace=None, workspace_bytes=0) == OK
    n = C.c_int64(0)
    for a in ((-1, 8, 0), (2, 6, 0), (2, 8, -1), (2, 4100, 0)):
        assert lib.sgd_kernel_norm_grad_workspace(*a, C.byref(n)) == ARG
    assert lib.sgd_kernel_norm_grad_workspace(0, 8, 0, C.byref(n)) == OK and n.value == 0


def test_binding_refuses_what_the_pointers_cannot_show():
    z, ids, u = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32), torch.zeros(2, 2)
    with pytest.raises(ValueError, match="CUDA"):
        binding.sgd_kernel_sample(z, u, ids)
    with pytest.raises(TypeError, match="float16"):
        binding.sgd_kernel_sample(z.double(), u, ids)
    with pytest.raises(ValueError, match="CUDA"):
        binding.sgd_kernel_embedding(z, ids, z)
    with pytest.raises(ValueError, match="CUDA"):
        binding.sgd_kernel_embedding_grad(z, ids, z)
    with pytest.raises(ValueError, match="CUDA"):
        binding.sgd_kernel_norm_grad(z, z, 0, dh=z)
    cpu = torch.device("cpu")
    assert binding._modulation(torch.zeros(2, 24)[:, 8:16], "x", 2, 8, cpu)[1] == 24
    assert binding._modulation(torch.zeros(1, 24)[:, 8:16], "x", 1, 8, cpu)[1] == 24
    for bad in (torch.zeros(8, 2).t(), torch.zeros(2, 9), torch.zeros(3, 8)):
        with pytest.raises(ValueError):
            binding._modulation(bad, "x", 2, 8, cpu)
    with pytest.raises(TypeError):
        binding._modulation(torch.zeros(2, 8).half(), "x", 2, 8, cpu)


def test_block_is_the_headers():
    import os
    import re
    from oracle import ends
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = open(os.path.join(root, "include", "sgd_kernels.h")).read()
    assert int(re.search(r"#define SGD_SAMPLE_BLOCK (\d+)", src).group(1)) == ends.BLOCK
