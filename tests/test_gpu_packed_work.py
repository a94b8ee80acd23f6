"""The workspace that attention of packed sequences asks for, through the binding."""

import pytest

from paper_2608_09231_gb300 import bag

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(lib):
    c = bag.create("tiny", T=2, B=1)
    yield c
    c.close()


def test_unknown_keys_are_any_number(ctx):
    """Sizes told for an unknown longest sequence serve a known one of any length."""
    for nq, seqs, max_q, prefix in ((1, 1, 1, 0), (64, 1, 64, 0), (30, 30, 1, 500)):
        told = ctx.attention_work(nq, 28, 128, 4, seqs, max_q, None, prefix)
        assert told == ctx.attention_work(nq, 28, 128, 4, seqs, max_q, 0, prefix)
        for k in (1, 300, 5000, 131072, 10 ** 7, 1 << 30):
            assert ctx.attention_work(nq, 28, 128, 4, seqs, max_q, k, prefix) <= told
        assert told > 0
