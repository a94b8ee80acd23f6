"""Rotary positions, cache and attention as a text layer uses them together: prompts, more tokens, single ones,
with and without a shared prefix."""

import contextlib
import math

import pytest
import torch

import prompt_ref as R
from paper_2608_09231_gb300 import bag, prompt

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ctx(lib):
    c = bag.create("tiny", T=2, B=1)
    yield c
    c.operators_status()
    c.close()


def layer_of(ctx, cache, rows, prefix=0, heads=6, kv_heads=2, dh=128, **more):
    return prompt.TextAttention(ctx, prompt.random_weights(384, heads, kv_heads, dh), heads, kv_heads, cache, rows, prefix, dh,
                                **more)


def texts(key, n):
    return torch.randn(n, 384, generator=torch.Generator(device=DEV).manual_seed(key), device=DEV)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("prefix", [0, 150])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_steps_against_their_own_cache(dh, prefix, layout, ctx):
    """The attention of every step against 64 bits on the layer's own rotated queries and cache, and the rotation
    against 64 bits on its projections."""
    cache = prompt.TextCache(4, 300)
    layer = layer_of(ctx, cache, 400, prefix, dh=dh, layout=layout, factor=4.0, original=64)
    layer.k.fill_(math.nan)
    layer.v.fill_(math.nan)
    if prefix:
        layer.prefix(texts(9, prefix))
    for key, new in enumerate(([33, 0, 200, 1], [1, 1, 1, 1], [40, 2, 0, 140], [1, 1, 1, 1], [0, 1, 0, 0])):
        s = cache.extend(new)
        h = texts(key, s["rows"])
        before = h.clone()
        layer.step(h, s)
        n = s["rows"]
        H, Hk = layer.heads, layer.kv_heads
        q, k, v = layer.qkv[:n].split([H * dh, Hk * dh, Hk * dh], 1)
        pos, at = s["pos"] + prefix, s["slots"].long()
        for x, y in ((q, layer.q[:n]), (k, layer.k[at])):
            want, tol = R.rope(x, pos, layer.freqs, dh, layout, layer.scale)
            assert bool(((y.double() - want).abs() <= tol).all())
        assert torch.equal(layer.v[at], v)
        seqs = [(s["q_start"][i].item(), m, i * 300, cache.lens[i]) for i, m in enumerate(new)]
        want, tol, _, _ = R.attention(layer.q[:n], layer.k, layer.v, H, Hk, seqs, pk=layer.pk if prefix else None,
                                      pv=layer.pv if prefix else None)
        assert bool(((layer.o[:n].double().reshape(n, H, dh) - want).abs() <= tol).all())
        assert bool(torch.isfinite(h).all()) and not torch.equal(h, before)


def test_a_prompt_at_once_and_token_by_token(ctx):
    """The same tokens in one step, in uneven steps and one by one fill the cache with the same bits and give
    outputs within twice the attention's bound (and then the 8-bit output product's steps: compared before it)."""
    n = 70
    h = texts(3, n)
    outs, caches = [], []
    for steps in ([n], [1] * n, [5, 64, 1]):
        cache = prompt.TextCache(1, 80)
        layer = layer_of(ctx, cache, n)
        rows = []
        at = 0
        for m in steps:
            layer.step(h[at:at + m].clone(), cache.extend([m]))
            rows.append(layer.o[:m].clone())
            at += m
        outs.append(torch.cat(rows))
        caches.append((layer.k[:n].clone(), layer.v[:n].clone(), layer))
    q = caches[0][2].q[:n]
    _, tol, _, _ = R.attention(q, caches[0][0], caches[0][1], 6, 2, [(0, n, 0, n)])
    for i in (1, 2):
        # the projections' sums may be split otherwise for other numbers of rows: bf16 steps of the cache's values
        for a, b in zip(caches[0][:2], caches[i][:2]):
            assert float((a.double() - b.double()).abs().max()) <= 2.0 ** -7 * float(a.abs().max())
        close = (outs[0].double() - outs[i].double()).abs().reshape(n, 6, 128) <= 2 * tol + 2.0 ** -6 * outs[0].double().abs().max()
        assert bool(close.all())


def test_on_another_stream(ctx):
    cache, again = prompt.TextCache(2, 64), prompt.TextCache(2, 64)
    a, b = layer_of(ctx, cache, 64), layer_of(ctx, again, 64)
    h = texts(5, 50)
    want = h.clone()
    a.step(want, cache.extend([20, 30]))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        x = torch.randn(4096, 4096, device=DEV)
        for _ in range(10):
            x = x @ x * 1e-3
        got = h + 0 * x.sum().nan_to_num(0.0, 0.0, 0.0)
        b.step(got, again.extend([20, 30]))
        got = got.clone()
    s.synchronize()
    assert torch.equal(got, want)


def test_no_work_of_torch_once_the_context_waits(ctx, monkeypatch):
    """Behind a prefix, on another stream: what torch makes for a step is there when the context's stream has waited
    for torch's (which is kept busy from then on)."""
    n = 40
    h, first = texts(6, 30), texts(7, n)
    outs, real = [], prompt.ordered

    @contextlib.contextmanager
    def busy(c):
        with real(c):
            torch.cuda._sleep(50_000_000)  # some 25 ms
            yield

    for late in (False, True):
        cache = prompt.TextCache(2, 64)
        layer = layer_of(ctx, cache, 64, n)
        got = h.clone()
        if late:
            monkeypatch.setattr(prompt, "ordered", busy)
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                layer.prefix(first.clone())
                layer.step(got, cache.extend([10, 20]))
            s.synchronize()
        else:
            layer.prefix(first.clone())
            layer.step(got, cache.extend([10, 20]))
        outs.append((got, layer.q[:30].clone()))
    torch.cuda.synchronize()
    assert torch.equal(outs[0][1], outs[1][1]) and torch.equal(outs[0][0], outs[1][0])


def test_an_empty_prefix(ctx):
    cache = prompt.TextCache(2, 16)
    layer = layer_of(ctx, cache, 16)
    layer.prefix(texts(1, 0))
    h = texts(1, 3)
    layer.step(h, cache.extend([1, 2]))
    assert bool(torch.isfinite(h).all())


def test_refusals(ctx):
    cache = prompt.TextCache(2, 16)
    layer = layer_of(ctx, cache, 16, prefix=8)
    h = texts(1, 16)
    with pytest.raises(ValueError, match="prefix comes first"):
        layer.step(h[:2], prompt.TextCache(2, 16).extend([1, 1]))
    with pytest.raises(ValueError):
        layer.prefix(h[:7])
    layer.prefix(h[:8].clone())
    with pytest.raises(ValueError):
        layer.step(h[:3], cache.extend([1, 1]))
    with pytest.raises(ValueError):
        prompt.TextAttention(ctx, prompt.random_weights(384, 6, 2), 6, 3, cache, 16)


def test_as_a_command(lib, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["prompt", "--texts", "3", "--tokens", "20", "--prefix", "30", "--heads", "4", "--kv-heads", "2"])
    prompt.main()
    out = capsys.readouterr().out
    assert "prefix of 30 tokens" in out and "3 prompts of 20 tokens" in out and "a token of each" in out
