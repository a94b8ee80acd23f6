"""The 8-bit product's sums: every form of its kernels, and sums long enough for passes."""

import numpy as np
import pytest
import torch

import lowbit_ref as R
import test_gpu_lowbit as L
from fp8_shapes import FORMS, LONG
from paper_2608_09231_gb300 import bag

pytestmark = pytest.mark.gpu
DEV = "cuda"
KINDS = ["f32", "bf16", "fp8", "resid"]
LIMIT = {"f32": 32, "bf16": 64, "fp8": 20, "resid": 32}  # K blocks of one sum on the tensor core


@pytest.fixture(scope="module")
def ctx(lib):
    c = bag.create("tiny", T=2, B=1)
    yield c
    c.close()


def ids(forms):
    return [f"{rows}-row tiles, {ctas} CTAs" if rows else "pairs" for rows, ctas in forms]


@pytest.mark.parametrize("M,N,K", FORMS.values(), ids=ids(FORMS))
@pytest.mark.parametrize("kind", KINDS)
def test_every_form(M, N, K, kind, ctx):
    """At test_gemm_fp8's bounds."""
    L.test_gemm_fp8(M, N, K, kind, ctx)


@pytest.mark.parametrize("M,N,K", LONG.values(), ids=ids(LONG))
@pytest.mark.parametrize("kind", KINDS)
def test_every_form_in_passes(M, N, K, kind, ctx):
    """At test_gemm_fp8's bounds."""
    L.test_gemm_fp8(M, N, K, kind, ctx)


@pytest.mark.parametrize("M,N,K", [(1, 5120, 28672), (1, 5120, 53248), (16, 512, 65536), (8, 512, 262144), (17, 500, 69000),
                                   (64, 300, 70016), (250, 500, 68000), (600, 2048, 69000)])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("last", [2, 10 ** 6])
def test_nothing_is_lost_a_pass_away(M, N, K, kind, last, ctx):
    """One large product in the first K block, and products that would fall below the last bits of a sum
    that holds it in the two blocks from the limit of a pass on, or in every one.  Each pass, each part of K and their
    total are exact in fp32, so that fp32 outputs have every bit.  For the narrower outputs the large
    one is the middle of two of their values, which rounds down (to even) where nothing is added and
    up with the small ones."""
    blocks, first = -(-K // 128), LIMIT[kind]
    end = min(K, 128 * (first + last))
    middle = {"f32": 2.0 ** -8, "resid": 2.0 ** -8, "bf16": 2.0 ** -8, "fp8": 2.0 ** -4}[kind]
    code = {float(v): c for c, v in enumerate(R.E4M3) if c < 127}
    a = torch.zeros(M, R.up(K, 16), device=DEV, dtype=torch.uint8)
    w = torch.zeros(N, R.up(K, 16), device=DEV, dtype=torch.uint8)
    a_s, w_s = (torch.full((n, R.up(blocks, 4)), 127, device=DEV, dtype=torch.uint8) for n in (M, N))
    a[:, :K] = code[1.0]
    w[:, 0], w[:, 1] = code[1.0], code[middle]
    w[:, 128 * first:end] = code[1.0]
    w_s[:, first:] = 127 - 30                           # products of 2^-30, 128 or fewer a block
    w[::128, 0], w[::128, 1] = code[448.0], 0           # the code block's scale: 1
    w[::128, 128:] = 0
    small = max(0, end - 128 * first) * 2.0 ** -30        # below 2^-12: a multiple of 2^-30, 18 bits
    value = np.full(N, 1.0 + middle + small)
    value[::128] = 448.0
    if kind == "fp8":
        c, s = L.encoded(M, N)
        ctx.gemm_fp8(a, a_s, w, w_s, c[1:M + 1], K, out_scales=s[1:M + 1])
        want = torch.full((N,), code[1.0 + 2.0 ** -3 if small else 1.0], device=DEV, dtype=torch.uint8)
        want[::128] = code[448.0]
        assert bool((s[1:M + 1, :-(-N // 128)] == 127).all())
        assert torch.equal(c[1:M + 1, :N], want.expand(M, N))
        return
    out = torch.zeros(M, N, device=DEV, dtype=torch.bfloat16 if kind == "bf16" else torch.float32)
    ctx.gemm_fp8(a, a_s, w, w_s, out, K, residual=kind == "resid")
    # the total rounds once where its parts are added: to the nearest fp32
    want = value.astype(np.float32)
    if kind == "bf16":
        want = R.bf16(value.astype(np.float32))
    assert np.array_equal(out.float().cpu().numpy(), np.broadcast_to(want, (M, N)))


@pytest.mark.parametrize("M,N,K", [(1, 512, 32768), (16, 512, 65536), (8, 512, 262144), (64, 300, 70016), (250, 500, 68000)])
def test_longer_sums_stay_in_fp32(M, N, K, ctx):
    """Normal rows at the bound of the sums of 13824 products: 1e-6 in the 2-norm.  (A pass of 4096
    is off by 2.5e-7 at most, towards zero, and so is a sum of passes; adding up to 64 parts in fp32
    adds their roundings, 6e-8 each at random.)"""
    L.test_gemm_fp8_keeps_long_sums_in_fp32(M, N, K, ctx)
