"""Operands of the 8-bit product that are parts of wider buffers."""

import numpy as np
import pytest
import torch

import lowbit_ref as R
from paper_2608_09231_gb300 import bag

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ctx(lib):
    c = bag.create("tiny", T=2, B=1)
    yield c
    c.close()


def buffers(g, rows, cols):
    """Codes and scale bytes of a matrix, any of them finite."""
    codes = g.integers(0, 256, (rows, cols)).astype(np.uint8)
    codes[(codes & 127) == 127] = 0
    return codes, g.integers(121, 134, (rows, cols // 128)).astype(np.uint8)


@pytest.mark.parametrize("M,N", [(1, 300), (17, 640), (300, 256), (2500, 2304)])
@pytest.mark.parametrize("first,blocks", [(4, 4), (12, 4), (8, 7), (4, 1)])
def test_columns_of_a_wider_matrix(M, N, first, blocks, ctx):
    """Columns [128 first, 128 (first + blocks)) of both operands, whose last row ends where its buffer
    does, against a copy of their own: the same bits."""
    g = np.random.default_rng([M, N, first, blocks])
    ops, own = [], []
    for rows in (M, N):
        codes, scales = buffers(g, rows, 16 * 128)
        c, s = (torch.from_numpy(t).to(DEV) for t in (codes, scales))
        ops += [c[:, 128 * first:128 * (first + blocks)], s[:, first:R.up(first + blocks, 4)]]
        dense = torch.full((rows, R.up(blocks, 4)), 255, device=DEV, dtype=torch.uint8)
        dense[:, :blocks] = s[:, first:first + blocks]
        own += [ops[-2].contiguous(), dense]
    out, want = torch.empty(M, N, device=DEV), torch.empty(M, N, device=DEV)
    ctx.gemm_fp8(*ops, out, 128 * blocks)
    ctx.gemm_fp8(*own, want, 128 * blocks)
    assert torch.equal(out, want)
    exact = [R.decode(c.cpu().numpy(), s[:, :blocks].cpu().numpy()) for c, s in (own[:2], own[2:])]
    a, w = (torch.from_numpy(t).to(DEV) for t in exact)
    eps = 4 * 128 * blocks * 2.0 ** -24 * (a.abs() @ w.abs().T)  # of fp32 sums of exact products
    assert bool(((out.double() - a @ w.T).abs() <= eps).all())
