"""sgd_kernel_embedding and sgd_kernel_embedding_grad on the GPU, against oracle/ends.py in float64 on the same inputs.

Tolerances (u = 2^-24): a looked-up value is one product rounded to fp32, then to its type (half a step, eps / 2 of the
value, or of its smallest normal number).  A sum of n rows has n - 1 roundings at most in whatever order, and one of the product:
n u of the sum of magnitudes; then the type's half step, and with accumulate one rounding of fp32 more.
"""
import math

import numpy as np
import pytest
import torch

from oracle import ends as oe

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2609_29505_gb300 import binding, build
    build.build()
    binding.lib()
    return binding


def _matrix(rows, d, dtype, seed, pad=0, offset=0, fill=None):
    """A [rows, d] view with `pad` columns between rows and `offset` elements before them, all of which hold 77."""
    buf = torch.full((offset + rows * (d + pad) + 16,), 77.0, dtype=DT[dtype], device="cuda")
    v = buf[offset:offset + rows * (d + pad)].view(rows, d + pad)[:, :d]
    if fill is None:
        v.copy_(torch.from_numpy(np.random.default_rng(seed).standard_normal((rows, d))))
    else:
        v.fill_(fill)
    return v, buf


def _np(t):
    return t.double().cpu().numpy()


def _half_step(want, dtype):
    f = torch.finfo(DT[dtype])
    return np.maximum(np.abs(want), f.tiny) * f.eps / 2


def _outside(buf, v):
    """What lies around a view is as it was."""
    mask = torch.ones_like(buf, dtype=torch.bool)
    mask.as_strided(v.shape, v.stride(), v.storage_offset()).fill_(False)
    return bool((buf[mask] == 77.0).all())


def _ids(rows, vocab, seed, hot=0.0, pad=0.0):
    rng = np.random.default_rng(seed)
    ids = np.minimum((vocab ** rng.random(rows)).astype(np.int64) - 1, vocab - 1)
    ids[rng.random(rows) < hot] = vocab // 2
    out = rng.random(rows) < pad
    ids[out] = rng.choice([-1, -2 ** 31, vocab, 2 ** 31 - 1], out.sum())
    return torch.from_numpy(ids.astype(np.int32)).cuda()


SHAPES = [(1, 1, 1), (3, 5, 7), (5, 9, 8), (17, 40, 12), (33, 100, 64), (64, 1000, 250), (7, 300, 1152), (300, 1000, 256), (40, 2000, 4096)]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("out", list(DT))
@pytest.mark.parametrize("rows,vocab,d", SHAPES)
def test_lookup(B, rows, vocab, d, dtype, out):
    for pad, offset, pad_out, offset_out, scale in ((0, 0, 0, 0, 1.0), (8, 8, 16, 8, 16.0), (3, 1, 5, 3, -0.37), (0, 0, 1, 0, 2.5)):
        table, _ = _matrix(vocab, d, dtype, 1, pad, offset)
        got, buf = _matrix(rows, d, out, 2, pad_out, offset_out, fill=55.0)
        ids = _ids(rows, vocab, 3, hot=0.2, pad=0.2)
        B.sgd_kernel_embedding(table, ids, got, scale=scale)
        want = oe.embedding(_np(table), ids.cpu().numpy(), scale)
        assert (np.abs(_np(got) - want) <= U * np.abs(want) + _half_step(want, out)).all()
        assert _outside(buf, got)


def test_lookup_of_values_out_of_range(B):
    table = torch.tensor([[60000.0, -60000.0, 1e-7, math.nan, math.inf, 0.0, 1.0, -1.0]], device="cuda")
    out = torch.empty(2, 8, dtype=torch.float16, device="cuda")
    B.sgd_kernel_embedding(table, torch.tensor([0, 1], dtype=torch.int32, device="cuda"), out, scale=2.0)
    want = (table * 2).half()
    assert torch.equal(out[0].nan_to_num(7.0), want[0].nan_to_num(7.0)) and (out[1] == 0).all()


def _grad(B, rows, vocab, d, dtype, out, seed=0, hot=0.0, pad_rows=0.0, scale=1.0, accumulate=False, layout=(0, 0, 0, 0), ids=None):
    grad, _ = _matrix(rows, d, dtype, seed, layout[0], layout[1])
    table, buf = _matrix(vocab, d, out, seed + 1, layout[2], layout[3])
    if ids is None:
        ids = _ids(rows, vocab, seed + 2, hot, pad_rows)
    before = _np(table)
    ws = torch.full((B.sgd_kernel_embedding_grad_workspace(rows, vocab, d),), 255, dtype=torch.uint8, device="cuda")  # (NaN)
    B.sgd_kernel_embedding_grad(grad, ids, table, scale=scale, accumulate=accumulate, workspace=ws)
    want, size, n = oe.embedding_grad(_np(grad), ids.cpu().numpy(), vocab, scale)
    got = _np(table)
    assert _outside(buf, table)
    tol = n[:, None] * U * size
    if accumulate:
        assert np.array_equal(got[n == 0], before[n == 0])
        want = np.where(n[:, None] > 0, want + before, before)
        tol = tol + U * np.abs(want)
    else:
        assert (got[n == 0] == 0).all()
    tol = tol + _half_step(want, out)
    err = np.abs(got - want)[n > 0]
    assert (err <= tol[n > 0]).all(), np.max(err / tol[n > 0])
    return grad, ids, table


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("bf16", "f32"), ("f32", "f16"), ("f16", "f16"), ("f32", "bf16")])
@pytest.mark.parametrize("rows,vocab,d", SHAPES)
def test_gradient(B, rows, vocab, d, dtype, out, accumulate):
    for i, layout in enumerate(((0, 0, 0, 0), (8, 8, 16, 8), (3, 1, 5, 3))):
        _grad(B, rows, vocab, d, dtype, out, seed=i, hot=0.3, pad_rows=0.2, scale=(1.0, 16.0, -0.37)[i], accumulate=accumulate, layout=layout)


@pytest.mark.parametrize("hot", [0.0, 0.5, 1.0])
@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 31, 33, 255, 1000, 2049, 4096, 6143, 6144, 6145, 8191, 8192, 8193, 10000, 20481, 70001])
def test_gradient_of_many_rows(B, rows, hot):
    """Either sort; tokens whose rows fill chunks, end at their borders or pass many of them."""
    for vocab in (3, 700) if rows > 5000 else (1, 3, 255, 256, 257, 70000):
        _grad(B, rows, vocab, 24, "bf16", "f32", seed=rows, hot=hot, pad_rows=0.1)


@pytest.mark.parametrize("rows", [160, 9600])
@pytest.mark.parametrize("run", [1, 15, 16, 17, 32, 48, 64, 100, 160])
def test_gradient_of_runs_at_borders(B, rows, run):
    """Runs of one length, so that they end everywhere in a chunk; rows in descending order of the token."""
    ids = torch.arange(rows - 1, -1, -1, device="cuda", dtype=torch.int32) // run
    _grad(B, rows, rows // run + 1, 40, "f32", "f32", seed=run, ids=ids)


@pytest.mark.parametrize("rows", [500, 9000])
def test_gradient_of_no_token(B, rows):
    for value in (-1, 77, 2 ** 31 - 1, -2 ** 31):
        ids = torch.full((rows,), value, dtype=torch.int32, device="cuda")
        for accumulate in (False, True):
            _grad(B, rows, 77, 16, "f16", "f16", ids=ids, accumulate=accumulate)


def test_padded_rows_are_not_read(B):
    grad = torch.ones(40, 64, device="cuda")
    ids = torch.arange(40, dtype=torch.int32, device="cuda") % 4
    ids[10:20] = -1
    grad[10:20] = math.nan
    table = torch.empty(4, 64, device="cuda")
    B.sgd_kernel_embedding_grad(grad, ids, table)
    assert torch.equal(table, torch.bincount(ids[ids >= 0].long(), minlength=4).float()[:, None].expand(4, 64))


def test_gradient_of_no_rows(B):
    table = torch.full((5, 8), 3.0, device="cuda")
    none, ids = torch.empty(0, 8, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    B.sgd_kernel_embedding_grad(none, ids, table, accumulate=True)
    assert (table == 3).all()
    B.sgd_kernel_embedding_grad(none, ids, table)
    assert (table == 0).all()
    B.sgd_kernel_embedding(table, ids, none)


def test_the_order_of_the_sum_is_the_rows(B):
    """1e8 + 1 - 1e8 in fp32 depends on the order; runs shorter than a chunk are added in the rows' order."""
    grad = torch.zeros(9, 4, device="cuda")
    grad[:, :] = torch.tensor([1e8, 1.0, -1e8, 1.0, 1.0, 1e8, -1e8, 1.0, 1.0], device="cuda")[:, None]
    ids = torch.tensor([3, 3, 3, 1, 3, 3, 3, 3, 1], dtype=torch.int32, device="cuda")
    table = torch.empty(5, 4, device="cuda")
    B.sgd_kernel_embedding_grad(grad, ids, table)
    want = np.float32(0)
    for v in (1e8, 1.0, -1e8, 1.0, 1e8, -1e8, 1.0):
        want = np.float32(want + np.float32(v))
    assert (table[3] == float(want)).all() and (table[1] == 2).all()


@pytest.mark.parametrize("rows", [3000, 20000])
def test_same_on_every_run_streams_and_graphs(B, rows):
    grad, ids, want = _grad(B, rows, 900, 512, "bf16", "f32", hot=0.4)
    tables = [torch.empty_like(want) for _ in range(3)]
    streams = [torch.cuda.Stream() for _ in tables]
    torch.cuda.synchronize()
    for t, s in zip(tables, streams):
        B.sgd_kernel_embedding_grad(grad, ids, t, stream=s)  # a workspace of its own each
    torch.cuda.synchronize()
    assert all(torch.equal(t, want) for t in tables)
    ws = torch.empty(B.sgd_kernel_embedding_grad_workspace(rows, 900, 512), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.sgd_kernel_embedding_grad(grad, ids, tables[0], workspace=ws)
        B.sgd_kernel_embedding_grad(grad, ids, tables[1])  # (allocated in the graph's pool)
    for t in tables:
        t.zero_()
    g.replay()
    assert torch.equal(tables[0], want) and torch.equal(tables[1], want)


def test_offsets_of_more_than_32_bits(B):
    """A table of 4.6e9 elements: the last tokens' rows."""
    vocab, d = 1126464, 4096
    if torch.cuda.mem_get_info()[0] < 30e9:
        pytest.skip("needs 30 GB")
    table = torch.zeros(vocab, d, dtype=torch.bfloat16, device="cuda")
    table[-1] = 3.0
    table[-7] = 5.0
    ids = torch.tensor([vocab - 1, vocab - 7, 0], dtype=torch.int32, device="cuda")
    out = torch.empty(3, d, device="cuda")
    B.sgd_kernel_embedding(table, ids, out, scale=2.0)
    assert (out[0] == 6).all() and (out[1] == 10).all() and (out[2] == 0).all()
    grad = torch.ones(5, d, device="cuda")
    ids = torch.tensor([vocab - 1, vocab - 7, 0, vocab - 1, vocab], dtype=torch.int32, device="cuda")
    B.sgd_kernel_embedding_grad(grad, ids, table, accumulate=True)
    assert (table[-1] == 5).all() and (table[-7] == 6).all() and (table[0] == 1).all() and (table[1] == 0).all()
    table.fill_(9.0)
    B.sgd_kernel_embedding_grad(grad, ids, table)
    assert (table[-1] == 2).all() and (table[-7] == 1).all() and (table[0] == 1).all()
    assert table[:, 0].float().sum() == 4 and table[:, -1].float().sum() == 4


def test_binding_refuses(B):
    table, out = torch.zeros(4, 8, device="cuda"), torch.zeros(3, 8, device="cuda")
    ids = torch.zeros(3, dtype=torch.int32, device="cuda")
    for a in ((table, ids.long(), out), (table.double(), ids, out), (table, ids, out.int())):
        with pytest.raises(TypeError):
            B.sgd_kernel_embedding(*a)
    for a in ((table, ids[:2], out), (table, ids, out[:, :4]), (table, ids, out.cpu()), (table.t(), ids, out), (table[0], ids, out)):
        with pytest.raises(ValueError):
            B.sgd_kernel_embedding(*a)
    for a in ((out, ids.long(), table), (out, ids, table.int())):
        with pytest.raises(TypeError):
            B.sgd_kernel_embedding_grad(*a)
    for a in ((out, ids[:2], table), (out, ids, table[:, :4]), (out, ids, table.cpu())):
        with pytest.raises(ValueError):
            B.sgd_kernel_embedding_grad(*a)
    with pytest.raises(B.SgdError, match="workspace"):
        B.sgd_kernel_embedding_grad(out, ids, table, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError, match="workspace"):
        B.sgd_kernel_embedding_grad(out, ids, table, workspace=torch.empty(1 << 16, dtype=torch.uint8))
    with pytest.raises(B.SgdError, match="overlaps"):
        B.sgd_kernel_embedding(table, ids, table[:3])
    with pytest.raises(B.SgdError, match="overlaps"):
        B.sgd_kernel_embedding_grad(table, torch.zeros(4, dtype=torch.int32, device="cuda"), table)
