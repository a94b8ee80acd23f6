"""GELU in the 8-bit product's epilogue, alone: operands of zeros, so that y is the bias."""

import numpy as np
import pytest
import torch

from paper_2608_09231_gb300 import bag

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ctx(lib):
    c = bag.create("tiny", T=2, B=1)
    yield c
    c.close()


@pytest.mark.parametrize("M", [1, 40, 3000])  # few rows, and CTA pairs
def test_gelu(M, ctx):
    """y / (1 + 2^x), x = -2 log2(e) sqrt(2/pi) (y + 0.044715 y^3), in fp32.  x comes out of three
    roundings and two rounded constants, 2^-24 of it each where the terms of its sum have one sign
    (they do): |x| 2.5 2^-23, which 2^x turns into 0.7 of that relative to itself.  exp2, the sum, the
    reciprocal and the product are good to 2^-22 each: 2^-20 together.  Below 2^-110 the special
    functions flush to zero."""
    g = np.random.default_rng(M)
    y = np.concatenate([np.linspace(-14, 14, 3001), g.standard_normal(500) * 4, -np.exp2(np.linspace(-40, 6, 200)),
                        np.exp2(np.linspace(-40, 100, 200)), [0.0, -0.0, 3e38, -3e38, 1e-45]]).astype(np.float32)
    N = len(y)
    u8 = lambda *s: torch.zeros(*s, device=DEV, dtype=torch.uint8)  # noqa: E731
    out = torch.full((M, N), 9.0, device=DEV)
    ctx.gemm_fp8(u8(M, 128), u8(M, 4), u8(N, 128), u8(N, 4), out, 128, bias=torch.from_numpy(y).to(DEV), gelu=True)
    yd = y.astype(np.longdouble)
    with np.errstate(over="ignore"):
        x = -2 * np.longdouble(1.4426950408889634074) * np.sqrt(2 / np.longdouble(np.pi)) * (yd + np.longdouble(0.044715) * yd ** 3)
        ref = yd / (1 + np.exp2(x))
    rel = 2.0 ** -20 + 0.7 * 2.5 * 2.0 ** -23 * np.minimum(np.abs(x), 150)
    got = out.cpu().numpy().astype(np.longdouble)
    assert (np.abs(got - ref) <= np.abs(ref) * rel + 2.0 ** -110).all()
