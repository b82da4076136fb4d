"""The operators at a token model's two ends on the GPU at the limits of their arguments, against oracle/ends.py in float64 with the
tolerances of their own tests."""
import pytest

from test_gpu_norm_grad import B, _run  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("per", [2 ** 31 - 1, 2 ** 31 - 48, 2 ** 31 - 63, 2 ** 31, 2 ** 32 + 5, 2 ** 40])
@pytest.mark.parametrize("rows,d", [(1, 8), (64, 64), (700, 1152), (40, 4096)])
def test_modulation_of_one_sample_by_any_period(B, rows, d, per):
    _run(B, rows, d, "bf16", "ln", "gb", per=per, residual=True, seed=rows)
