"""Text layers whose steps were refused before, and the workspace that a layer keeps for all of its steps."""

import math

import pytest
import torch

import test_gpu_prompt as T
from paper_2608_09231_gb300 import bag, prompt

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ctx(lib):
    c = bag.create("tiny", T=2, B=1)
    yield c
    c.operators_status()
    c.close()


@pytest.mark.parametrize("prefix", [0, 30])
def test_a_refused_step_leaves_no_trace(prefix, ctx):
    """Refusals for the rows, the type, the layer's size and the texts' places; then the steps give what they give alone."""
    outs = []
    for refused in (False, True):
        cache = prompt.TextCache(2, 64)
        layer = T.layer_of(ctx, cache, 40, prefix)
        layer.k.fill_(math.nan)
        layer.v.fill_(math.nan)
        if refused and prefix:
            with pytest.raises(ValueError, match="prefix comes first"):
                layer.step(T.texts(1, 2), cache.extend([1, 1]))
        if prefix:
            layer.prefix(T.texts(9, prefix))
        got = []
        for key, new in enumerate(([20, 5], [1, 1], [0, 9])):
            n = sum(new)
            if refused:
                for bad, rows in ((T.texts(1, n + 1), new), (T.texts(1, n).double(), new), (T.texts(1, n)[:, :380], new),
                                  (T.texts(1, 41), [41 - n, n])):
                    with pytest.raises((ValueError, bag.BagError)):
                        layer.step(bad, cache.extend(rows))
                other = prompt.TextCache(3, 64)
                with pytest.raises(ValueError, match="a layer for 2"):
                    layer.step(T.texts(1, 3), other.extend([1, 1, 1]))
            h = T.texts(key, n)
            layer.step(h, cache.extend(new))
            got.append(h)
        assert cache.lens == [21, 15]
        outs.append(got)
    assert all(bool(torch.isfinite(a).all()) and torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("prefix", [0, 8])
def test_rows_of_another_width(prefix, ctx):
    """Rows that are wider than the weights, but not than the memory for their codes, are refused before anything runs."""
    weights = prompt.random_weights(380, 6, 2)
    cache = prompt.TextCache(1, 16)
    layer = prompt.TextAttention(ctx, weights, 6, 2, cache, 16, prefix)
    if prefix:
        with pytest.raises(ValueError):
            layer.prefix(T.texts(1, prefix))
        layer.prefix(T.texts(1, prefix)[:, :380].contiguous())
    layer.k.fill_(9.0)
    h = T.texts(2, 4)
    before = h.clone()
    with pytest.raises(ValueError):
        layer.step(h, cache.extend([4]))
    assert torch.equal(h, before) and bool((layer.k == 9).all()) and cache.lens == [0]


@pytest.mark.parametrize("texts,room,rows,prefix,heads,kv_heads", [(8, 16384, 1024, 0, 32, 8), (1, 32768, 512, 0, 28, 4),
                                                                  (1, 16384, 512, 700, 28, 4), (16, 600, 2048, 1024, 6, 2)])
def test_a_layer_keeps_memory_for_every_step(texts, room, rows, prefix, heads, kv_heads, ctx):
    """What the library asks for a step's own sizes, and for the sizes of any that the layer may take, the layer has."""
    cache = prompt.TextCache(texts, room)
    layer = prompt.TextAttention(ctx, prompt.random_weights(256, heads, kv_heads), heads, kv_heads, cache, rows, prefix)
    for n in (1, 2, 3, 8, 31, 32, 64, 128, 129, 256, 500, rows):
        for q in {min(n, room), -(-n // texts)}:
            for k in {q, min(room, q + room // 2), room}:
                for p in {0, prefix}:
                    assert ctx.attention_work(n, heads, 128, kv_heads, texts, q, k, p) <= layer.work.numel()
    assert ctx.attention_work(prefix, heads, 128, kv_heads, 1, None, prefix) <= layer.work.numel()
    assert layer.work.numel() < 200e6
