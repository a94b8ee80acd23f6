"""The operators' status without a GPU: a null context."""

import pytest

from paper_2608_09231_gb300 import bag


@pytest.mark.parametrize("name", ["bag_operators_status", "bag_check_operator_timeout"])
def test_null_context(name):
    from paper_2608_09231_gb300 import build
    build.build()
    assert getattr(bag.load(), name)(None) == 1
