"""The low-precision block where torch's current stream is not the context's."""

import pytest
import torch

from paper_2608_09231_gb300 import bag, lowbit

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ctx(lib):
    c = bag.create("tiny", T=2, B=1)
    yield c
    c.close()


def busy():
    """Some milliseconds of work on the current stream; a zero that comes out of it."""
    x = torch.randn(8192, 8192, device=DEV)
    for _ in range(20):
        x = x @ x * 1e-4
    return 0.0 * x.sum().nan_to_num(0.0, 0.0, 0.0)


@pytest.mark.parametrize("side", ["current", "context"])
def test_steps_follow_the_current_stream(side, ctx):
    """Weights, input and outputs made behind other work on the current stream, and read there: the bits of
    a block on one stream."""
    tokens, d, F = 700, 384, 1024
    g = torch.Generator(device=DEV).manual_seed(1)
    w = lowbit.random_weights(d, F)
    h0, h1 = (torch.randn(tokens, d, generator=g, device=DEV) for _ in range(2))
    mod = [0.5 * torch.randn(d, generator=g, device=DEV) for _ in range(6)]
    want, again = torch.empty_like(h0), torch.empty_like(h0)
    ctx.set_stream(0)
    block = lowbit.LowBitBlock(ctx, w, tokens, keep=3)
    block.full(h0, want, mod)
    block.reuse(h1, again)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    if side == "context":
        ctx.set_stream(s.cuda_stream)
    try:
        with torch.cuda.stream(s if side == "current" else torch.cuda.default_stream()):
            late = {n: t + busy().to(t.dtype) for n, t in w.items()}
            block = lowbit.LowBitBlock(ctx, late, tokens, keep=3)
            h, r = torch.full_like(h0, 7.0), torch.full_like(h0, 7.0)
            for _ in range(2):
                a, b = h0 + busy(), h1 + busy()
                block.full(a, h, mod)
                got = h.clone()
                h.fill_(7.0)
                block.reuse(b, r)
                kept = r.clone()
                r.fill_(7.0)
            torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(kept, again)
    finally:
        ctx.set_stream(0)
