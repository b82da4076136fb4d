"""The operators at a token model's two ends on the GPU at the limits of their arguments, against oracle/ends.py in float64 with the
tolerances of their own tests."""
import pytest
import torch

from test_gpu_norm_grad import B, _run  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("per", [2 ** 31 - 1, 2 ** 31 - 48, 2 ** 31 - 63, 2 ** 31, 2 ** 32 + 5, 2 ** 40])
@pytest.mark.parametrize("rows,d", [(1, 8), (64, 64), (700, 1152), (40, 4096)])
def test_modulation_of_one_sample_by_any_period(B, rows, d, per):
    _run(B, rows, d, "bf16", "ln", "gb", per=per, residual=True, seed=rows)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("vocab", [2 ** 31 - 1, 2 ** 31 - 1024, 2 ** 31 - 1217])
def test_gradient_of_the_longest_table(B, vocab, dtype):
    """Tokens up to the largest integer: every row of the table is written."""
    ids = torch.tensor([vocab - 1, 0, 5, vocab - 1, -1, 5, 2 ** 30], dtype=torch.int32, device="cuda")
    grad = torch.arange(1.0, 8.0, device="cuda")[:, None].to(dtype)
    table = torch.ones(vocab, 1, dtype=dtype, device="cuda")
    B.sgd_kernel_embedding_grad(grad, ids, table, scale=2.0)
    got = [float(table[i, 0]) for i in (0, 5, 2 ** 30, vocab - 1)]
    assert got == [4.0, 18.0, 14.0, 10.0]
    assert int(torch.count_nonzero(table)) == 4
    B.sgd_kernel_embedding_grad(grad, ids, table, accumulate=True)
    assert [float(table[i, 0]) for i in (0, 5, 2 ** 30, vocab - 1)] == [6.0, 27.0, 21.0, 15.0]
    assert int(torch.count_nonzero(table)) == 4
    out = torch.full((7, 1), 9.0, dtype=dtype, device="cuda")
    B.sgd_kernel_embedding(table, ids, out)
    assert out[:, 0].tolist() == [15.0, 6.0, 27.0, 15.0, 0.0, 27.0, 21.0]


@pytest.mark.parametrize("which", ["none", "handle", "object", "other"])
def test_workspace_of_a_call_belongs_to_its_stream(B, which):
    """Memory that torch's allocator hands out again is ordered behind the call only on the stream that it was allocated on."""
    other = torch.cuda.Stream()
    stream = {"none": None, "handle": 0, "object": torch.cuda.default_stream(), "other": other.cuda_stream}[which]
    want = other.cuda_stream if which == "other" else 0
    torch.cuda.synchronize()
    torch.cuda.empty_cache()  # (else the inputs come to lie in a large segment that an earlier test left, and the workspace beside them)
    # (a workspace of 17 MB: larger than what is left over of a segment of torch's allocator)
    grad, ids = torch.ones(1 << 16, 1024, device="cuda"), torch.zeros(1 << 16, dtype=torch.int32, device="cuda")
    table = torch.empty(4, 1024, device="cuda")
    before = {s["address"] for s in torch.cuda.memory_snapshot()}
    B.sgd_kernel_embedding_grad(grad, ids, table, stream=stream)
    new = [s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] not in before]
    torch.cuda.synchronize()
    assert new and all(s == want for s in new)
    assert (table[0] == 1 << 16).all() and (table[1:] == 0).all()


def test_matrices_between_one_anothers_rows(B):
    """Columns of one buffer: the rows looked up beside the table, the table's gradient beside the rows', a modulation's gradients beside it."""
    gen = torch.Generator().manual_seed(2)
    both = torch.randn(40, 96, generator=gen).cuda()
    table, out, rest = both[:, :32], both[:30, 32:64], both[:, 64:].clone()
    ids = torch.randint(0, 40, (30,), generator=gen, dtype=torch.int32).cuda()
    before = table.clone()
    B.sgd_kernel_embedding(table, ids, out, scale=2.0)
    assert torch.equal(out, 2.0 * before[ids.long()]) and torch.equal(table, before) and torch.equal(both[:, 64:], rest)
    grad, dtable = both[:30, 32:64], both[:, 64:]
    want = torch.zeros(40, 32, device="cuda", dtype=torch.float64).index_add_(0, ids.long(), grad.double())
    B.sgd_kernel_embedding_grad(grad, ids, dtable)
    # (30 rows at most of a token, each sum rounded to 2^-24 of magnitudes of at most 30 times the largest)
    assert (dtable.double() - want).abs().max() <= 30 * 30 * 2.0 ** -24 * float(grad.abs().max()) and torch.equal(table, before)
    x, want = _run(B, 50, 64, "f32", "ln_plain", per=20, seed=4)
    mod = torch.full((3, 200), 7.0, device="cuda")
    mod[:, 4:68] = x.pop("scale")
    dh = torch.empty_like(x["h"])
    B.sgd_kernel_norm_grad(kind=2, rows_per_batch=20, scale=mod[:, 4:68], dh=dh, dshift=mod[:, 68:132], dscale=mod[:, 132:196], **x)
    assert torch.equal(dh, want["dh"]) and torch.equal(mod[:, 68:132], want["dshift"]) and torch.equal(mod[:, 132:196], want["dscale"])
    assert (mod[:, :4] == 7).all() and (mod[:, 196:] == 7).all()
