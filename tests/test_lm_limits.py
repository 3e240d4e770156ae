"""Limits of the entry points of include/hmoe_lm.h (no GPU needed)."""
import pytest

from tests.test_lm_abi import F, lib, refused  # noqa: F401 (lib: the fixture)


@pytest.mark.parametrize("scale", [1.8e38, 2.4e38, 3.4e38])
def test_scales_whose_product_with_log2_e_may_overflow(lib, scale):  # noqa: F811
    refused(lib.hmoe_token_logprob(16, 64, None, 1, 10, 64, F(scale), 16, 3, 16, 16, 16, 16, 16, 16, None, 0, None), -1,
            "scale")
    refused(lib.hmoe_token_logprob_backward(16, 64, None, 1, 10, 64, F(scale), 16, 16, 16, 16, 16, 32, 64, None), -1,
            "scale")
