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
