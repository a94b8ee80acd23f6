"""Pooled vectors, block selection and attention over selected blocks on the GPU, against plain
restatements (the pooled codes and the selection bit for bit, the attention in float64)."""

import numpy as np
import pytest
import torch

import lowbit_ref as R
from paper_2608_09231_gb300 import bag

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ctx(lib):
    c = bag.create("tiny", T=2, B=1)
    yield c
    c.close()


def normal(key, *shape):
    g = torch.Generator(device=DEV).manual_seed(key)
    return torch.randn(*shape, generator=g, device=DEV)


def rows(key, n, heads, dtype, pad=0):
    """[n, 128 * heads] inside rows that are `pad` elements longer, NaN around."""
    x = torch.full((n, 128 * heads + pad), float("nan"), device=DEV).to(TYPES[dtype])
    x[:, pad:] = normal(key, n, 128 * heads).to(TYPES[dtype])
    return x[:, pad:]


def f32(t):
    return t.float().cpu().numpy()


def pooled(ctx, x, heads, more=0):
    nb = -(-x.shape[0] // 128) + more
    c = torch.full((heads, nb, 128), 77, device=DEV, dtype=torch.int8)
    s = torch.full((heads, nb), -3.0, device=DEV)
    ctx.block_pool(x, c, s)
    return c, s


@pytest.mark.parametrize("n", [1, 2, 127, 128, 129, 300, 1000])
@pytest.mark.parametrize("heads", [1, 3])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("pad", [0, 1, 8])  # 16-byte rows and not
def test_pool_is_bit_exact(n, heads, dtype, pad, ctx):
    x = rows(n + heads, n, heads, dtype, pad)
    c, s = pooled(ctx, x, heads, more=2)
    codes, scales = R.pool(f32(x), heads)
    nb = codes.shape[1]
    assert np.array_equal(c[:, :nb].cpu().numpy(), codes) and np.array_equal(s[:, :nb].cpu().numpy(), scales)
    assert bool((c[:, nb:] == 77).all() and (s[:, nb:] == -3.0).all())


def test_pool_of_zeros_and_values_that_are_not_finite(ctx):
    x = normal(1, 512, 256).half()
    x[:128, :128] = 0
    x[130, 3], x[300, 200], x[400, 5] = float("inf"), float("nan"), -float("inf")
    c, s = pooled(ctx, x, 2)
    codes, scales = R.pool(f32(x), 2)
    assert np.array_equal(c.cpu().numpy(), codes) and np.array_equal(s.cpu().numpy(), scales)
    assert (scales == 0).sum() == 4 and (codes[scales == 0] == 0).all()


@pytest.mark.parametrize("nq,nk,heads,kv_heads,keep", [
    (1, 1, 1, 1, 1), (1, 700, 4, 4, 3), (129, 1000, 2, 1, 8), (300, 33 * 128, 6, 2, 33), (257, 257 * 128 - 5, 1, 1, 40),
    (64, 600 * 128, 2, 2, 1), (128, 1100 * 128, 1, 1, 1099),
])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_selection_is_the_definitions(nq, nk, heads, kv_heads, keep, dtype, ctx):
    q, k = rows(nq, nq, heads, dtype), rows(nk + 1, nk, kv_heads, dtype)
    c, s = pooled(ctx, k, kv_heads, more=1)
    nqb, nkb = -(-nq // 128), -(-nk // 128)
    blocks = torch.full((heads, nqb, keep), -9, device=DEV, dtype=torch.int32)
    ctx.block_select(q, c, s, blocks, nkb)
    want = R.select(R.pool(f32(q), heads)[0], c[:, :nkb].cpu().numpy(), s[:, :nkb].cpu().numpy(), keep)
    assert np.array_equal(blocks.cpu().numpy(), want)


@pytest.mark.parametrize("nkb,keep", [(1, 1), (7, 3), (300, 17), (300, 299), (8192, 100), (8192, 8192)])
def test_selection_among_equal_scores(nkb, keep, ctx):
    """Scores of a few values only, in mixed order: ties go to the lower index."""
    g = np.random.default_rng(nkb + keep)
    k = g.integers(-2, 3, (1, nkb, 128)).astype(np.int8)
    k[0, :, 1:] = 0
    scales = g.choice(np.float32([0, 0.5, 1.0]), (1, nkb))
    q = torch.zeros(5, 128, device=DEV).half()
    q[:, 0] = 1.0
    blocks = torch.zeros(1, 1, keep, device=DEV, dtype=torch.int32)
    ctx.block_select(q, torch.from_numpy(k).to(DEV), torch.from_numpy(scales).to(DEV), blocks)
    assert np.array_equal(blocks.cpu().numpy(), R.select(R.pool(f32(q), 1)[0], k, scales, keep))


def attend(ctx, nq, nk, heads, kv_heads, dtype, blocks, key, pad=0, scale=1.0):
    """Kernel output and reference; what lies past the last key of V, and around rows, is NaN."""
    q, k = rows(key, nq, heads, dtype, pad) * scale, rows(key + 1, nk, kv_heads, dtype, pad)
    if pad:  # the product above is dense
        qq = torch.full((nq, 128 * heads + pad), float("nan"), device=DEV).to(TYPES[dtype])
        qq[:, pad:] = q
        q = qq[:, pad:]
    vpad = R.up(nk, 8) + 8
    vt = torch.full((kv_heads, 128, vpad), float("nan"), device=DEV).to(TYPES[dtype])
    vt[:, :, :nk] = normal(key + 2, kv_heads, 128, nk).to(TYPES[dtype])
    o = torch.full((nq + 1, 128 * heads + pad), 9.0, device=DEV).bfloat16()
    ctx.attention_blocks(q, k, vt, o[:nq, :128 * heads], torch.from_numpy(blocks).to(DEV), heads, kv_heads)
    got = o[:nq, :128 * heads].double().cpu().numpy().reshape(nq, heads, 128)
    assert bool((o[nq] == 9.0).all() and (o[:, 128 * heads:] == 9.0).all())
    ref = R.attention(f32(q).astype(np.float64).reshape(nq, heads, 128), f32(k).astype(np.float64).reshape(nk, kv_heads, 128),
                      f32(vt[:, :, :nk]).astype(np.float64).transpose(2, 0, 1), blocks)
    return got, ref


def check(got, ref, dtype):
    """As for the dense kernel: fp16 operands to the output's bf16 rounding, 2^-8 of the value and
    2^-10 of the largest; bf16 operands (P is rounded to bf16 too) to 2^-7 of the largest."""
    top = np.abs(ref).max()
    bound = 2.0 ** -8 * np.abs(ref) + 2.0 ** -10 * top if dtype == "f16" else 2.0 ** -7 * top
    assert (np.abs(got - ref) <= bound).all(), float((np.abs(got - ref) / np.maximum(bound, 1e-30)).max())


def lists(g, heads, nqb, nkb, keep):
    return np.stack([np.sort(g.permutation(nkb)[:keep]) for _ in range(heads * nqb)]).reshape(heads, nqb, keep).astype(np.int32)


@pytest.mark.parametrize("nq,nk,heads,kv_heads,keep", [
    (1, 1, 1, 1, 1), (1, 129, 2, 2, 2), (1, 4000, 3, 1, 9), (1, 5000, 2, 2, 40), (127, 128, 1, 1, 1), (128, 640, 2, 2, 4),
    (130, 1000, 4, 2, 8), (500, 2500, 6, 6, 5), (300, 9000, 1, 1, 70), (1200, 1200, 40, 40, 3), (2600, 1300, 16, 4, 11),
])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("pad", [0, 8])
def test_attention_blocks(nq, nk, heads, kv_heads, keep, dtype, pad, ctx):
    """One unit a CTA or two, one to sixteen parts a list, short last blocks, shared key heads."""
    g = np.random.default_rng(nq + nk + keep)
    blocks = lists(g, heads, -(-nq // 128), -(-nk // 128), keep)
    got, ref = attend(ctx, nq, nk, heads, kv_heads, dtype, blocks, nq + nk, pad)
    check(got, ref, dtype)


@pytest.mark.parametrize("how", ["equal", "alike", "disjoint", "twice", "shorter"])
@pytest.mark.parametrize("heads,kv_heads,nq,nk", [(40, 40, 1300, 2500), (44, 11, 1281, 2432)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_attention_of_neighbouring_lists(how, heads, kv_heads, nq, nk, dtype, ctx):
    """Two lists a CTA that hold the same blocks, some of them, or none (with an odd number of units,
    whose last has no neighbour); one that lists a block twice; one that ends early.  With key heads
    that four query heads share, neighbours are of other heads too.  The last key block is short or
    whole, and among the common blocks or not."""
    g = np.random.default_rng(heads + len(how))
    nqb, nkb, keep = -(-nq // 128), -(-nk // 128), 9
    flat = np.zeros((heads * nqb, keep), np.int32)
    for u in range(len(flat)):
        if u % 2 == 0 or how == "twice":
            a = np.sort(g.permutation(nkb)[:keep])
        if how == "equal":
            flat[u] = a
        elif how == "alike":
            b = a.copy()
            if u % 2:
                b[g.integers(0, keep, 3)] = g.permutation(np.setdiff1d(np.arange(nkb), a))[0]
                b = np.unique(b)
                b = np.sort(np.concatenate([b, g.permutation(np.setdiff1d(np.arange(nkb), b))[:keep - len(b)]]))
            flat[u] = b
        elif how == "disjoint":
            flat[u] = a if u % 2 == 0 else np.sort(g.permutation(np.setdiff1d(np.arange(nkb), a))[:keep])
        elif how == "twice":
            flat[u] = a
            if u % 3 == 0:
                flat[u, 4] = flat[u, 2]
        else:
            flat[u] = a
            flat[u, g.integers(0, keep + 1):] = -1
    got, ref = attend(ctx, nq, nk, heads, kv_heads, dtype, flat.reshape(heads, nqb, keep), heads)
    check(got, ref, dtype)


def test_attention_over_half_a_million_keys(ctx):
    """4097 key blocks, the last one short and in every list."""
    heads, nq, nk = 28, 1500, 4097 * 128 - 3
    g = np.random.default_rng(0)
    blocks = np.sort(g.integers(0, 4096, (heads, 12, 3)), axis=2).astype(np.int32)
    blocks[:, :, 2] = 4096
    got, ref = attend(ctx, nq, nk, heads, 1, "f16", blocks, 9)
    check(got, ref, "f16")


@pytest.mark.parametrize("nq,heads,keep", [(130, 2, 4), (700, 60, 4), (1, 3, 20), (257, 5, 1)])
def test_attention_of_short_and_empty_lists(nq, heads, keep, ctx):
    """Lists that end early, at an index past the last block or at once: the last give zeros."""
    nk = 128 * 20 + 17
    g = np.random.default_rng(keep)
    blocks = lists(g, heads, -(-nq // 128), 21, keep)
    flat = blocks.reshape(-1, keep)
    for i in range(len(flat)):
        n = g.integers(0, keep + 1)
        flat[i, n:] = g.choice([-1, 21, 2 ** 31 - 1], keep - n)
        if n + 1 < keep:
            flat[i, n + 1] = 0  # past the end: not read
    flat[-1] = -1
    got, ref = attend(ctx, nq, nk, heads, heads, "f16", blocks, 5)
    check(got, ref, "f16")
    h, i = (len(flat) - 1) // blocks.shape[1], (len(flat) - 1) % blocks.shape[1]
    assert (got[128 * i:, h] == 0).all()


def test_attention_of_large_scores(ctx):
    """Scores of hundreds, so that the running maximum moves from block to block."""
    g = np.random.default_rng(3)
    blocks = lists(g, 2, 3, 12, 7)
    got, ref = attend(ctx, 300, 12 * 128, 2, 2, "f16", blocks, 11, scale=30.0)
    check(got, ref, "f16")


def test_all_blocks_is_dense_attention(ctx):
    """Every block listed: the dense tensor-core kernel's result, to two bf16 roundings."""
    n, heads = 1000, 4
    q, k = rows(1, n, heads, "f16"), rows(2, n, heads, "f16")
    vt = normal(3, heads, 128, n).half()
    o, dense = (torch.empty(n, 128 * heads, device=DEV).bfloat16() for _ in range(2))
    blocks = torch.arange(8, device=DEV, dtype=torch.int32).repeat(heads, 8, 1)
    ctx.attention_blocks(q, k, vt, o, blocks, heads)
    ctx.attention_f16(q, k, vt, dense, n, n, heads, 128, n)
    d = (o.double() - dense.double()).abs()
    assert bool((d <= 2.0 ** -7 * dense.double().abs() + 2.0 ** -9 * dense.double().abs().max()).all())


def test_nan_keys_reach_only_the_queries_that_list_them(ctx):
    n, heads = 640, 2
    q, k = rows(1, n, heads, "f16"), rows(2, n, heads, "f16").clone()
    k[256 + 5, :128] = float("nan")
    vt = normal(3, heads, 128, n).half()
    blocks = np.array([[[0, 1], [2, 3], [3, 4], [1, 2], [0, 4]]] * 2, np.int32)
    o = torch.empty(n, 128 * heads, device=DEV).bfloat16()
    ctx.attention_blocks(q, k, vt, o, torch.from_numpy(blocks).to(DEV), heads)
    nan = torch.isnan(o).view(5, 128, 2, 128)
    want = torch.zeros_like(nan)
    want[1, :, 0], want[3, :, 0] = True, True
    assert torch.equal(nan, want)
