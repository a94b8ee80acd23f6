"""The low-precision entry points without a GPU: a null context, and tensors that are not on one."""

import pytest
import torch

from paper_2608_09231_gb300 import bag


@pytest.fixture(scope="module")
def lib():
    from paper_2608_09231_gb300 import build
    build.build()
    return bag.load()


@pytest.mark.parametrize("name", ["bag_quant_fp8", "bag_ln_mod_fp8", "bag_gemm_fp8", "bag_cache_write", "bag_cache_read",
                                  "bag_block_pool", "bag_block_select", "bag_attention_blocks"])
def test_null_context(lib, name):
    f = getattr(lib, name)
    assert f(*[None if t is not bag._I and t is not bag._L else 1 for t in f.argtypes]) == 1


def test_host_tensors_are_refused():
    with pytest.raises(ValueError, match="device matrix"):
        bag._mat(torch.zeros(2, 2, dtype=torch.uint8), "codes")
    with pytest.raises(ValueError, match="device vector"):
        bag._vec(torch.zeros(3), "bias", 3)
    assert bag._vec(None, "bias", 3) is None
