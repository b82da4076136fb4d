"""Scales out of range, and calls without a row, a sample or a position: an empty tensor's address may be null (no GPU needed: nothing is launched)."""
import pytest

from paper_2609_29505_gb300 import binding

P = 4096  # an address that nothing reads


@pytest.fixture(scope="module")
def lib():
    from paper_2609_29505_gb300 import build
    build.build()
    return binding.lib()


@pytest.mark.parametrize("n,k", [(0, 0), (3, 0), (0, 5), (3, 5)])
def test_logprobs_of_no_rows(lib, n, k):
    call = lambda rows, k=k, n=n, **o: lib.sgd_kernel_logprobs(  # noqa: E731
        None, 0, 64, rows, 64, 1.0, None, 0, None, n, None, o.get("entropy"), k, None, None, None)
    assert call(0) == binding.SGD_OK and call(0, entropy=P) == binding.SGD_OK
    assert call(1, entropy=P) == binding.SGD_ERR_ARG
    # sizes are looked at all the same
    assert call(0, k=65) == binding.SGD_ERR_ARG and call(0, n=-1) == binding.SGD_ERR_ARG
    assert lib.sgd_kernel_logprobs(None, 0, 63, 0, 64, 1.0, None, 0, None, n, None, None, k, None, None, None) == binding.SGD_ERR_ARG
    assert lib.sgd_kernel_logprobs(None, 9, 64, 0, 64, 1.0, None, 0, None, n, None, None, k, None, None, None) == binding.SGD_ERR_ARG


def test_distillation_of_no_rows(lib):
    call = lambda rows, k=4: lib.sgd_kernel_distill(None, 0, 64, rows, 64, 1.0, None, None, k, None, 1, None, None, 0, 64, None)  # noqa: E731
    assert call(0) == binding.SGD_OK
    assert call(1) == binding.SGD_ERR_ARG and call(0, k=65) == binding.SGD_ERR_ARG


def test_reveal_of_no_sample_or_position(lib):
    call = lambda batch, n, n_reveal=None: lib.sgd_sampler_reveal(  # noqa: E731
        None, None, 1, None, 1, 0, n_reveal, None, None, None, batch, n, 0, None)
    assert call(0, 64) == binding.SGD_OK and call(0, 0) == binding.SGD_OK and call(2, 0, P) == binding.SGD_OK
    assert call(2, 64, P) == binding.SGD_ERR_ARG and call(2, 0) == binding.SGD_ERR_ARG and call(0, -1) == binding.SGD_ERR_ARG


@pytest.mark.parametrize("scale,code", [(2.1e38, binding.SGD_ERR_ARG), (3.4e38, binding.SGD_ERR_ARG), (2e38, binding.SGD_OK), (1e-45, binding.SGD_OK)])
def test_scales_whose_product_with_log2_e_is_out_of_range(lib, scale, code):
    """2.4e38 log2(e) is infinite in fp32: 0 times it would be no number."""
    assert lib.sgd_kernel_logprobs(None, 0, 64, 0, 64, scale, None, 0, None, 0, None, None, 1, None, None, None) == code
    assert lib.sgd_kernel_distill(None, 0, 64, 0, 64, scale, None, None, 4, None, 1, None, None, 0, 64, None) == code
