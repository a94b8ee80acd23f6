"""Rotary positions on the GPU against a plain form in 64 bits (tests/prompt_ref.py has the bounds)."""

import math

import numpy as np
import pytest
import torch

import prompt_ref as R
from paper_2608_09231_gb300 import bag

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ctx(lib):
    c = bag.create("tiny", T=2, B=1)
    yield c
    c.close()


def freqs(n, theta=10000.0):
    return np.array([theta ** (-i / n) for i in range(n)])


def rows(key, n, cols, dtype, pad=0):
    """[n, cols] inside rows that are `pad` elements longer, NaN around."""
    g = torch.Generator(device=DEV).manual_seed(key)
    x = torch.full((n, cols + pad), math.nan, device=DEV, dtype=dtype)
    x[:, pad:] = torch.randn(n, cols, generator=g, device=DEV).to(dtype)
    return x[:, pad:]


def close(got, want, tol):
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), float((err - tol).max())


@pytest.mark.parametrize("dh,pairs", [(128, 64), (64, 32), (128, 32), (80, 20), (2, 1), (6, 2), (256, 128), (12, 6), (128, 24)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,pad", [(1, 0), (37, 1), (700, 16)])
def test_rotation(dh, pairs, layout, dtype, n, pad, ctx):
    """Queries, keys and values at positions from 0 to 2^31, wide and odd rows, few and many of them."""
    dt, H, Hk = TYPES[dtype], 3, 2
    q, k, v = (rows(i, n, h * dh, dt, pad) for i, h in enumerate((H, Hk, Hk)))
    pos = torch.randint(0, 1 << 20, (n,), device=DEV, dtype=torch.int32)
    pos[0] = (1 << 31) - 1
    pos[-1] = 0 if n > 1 else 5
    f = freqs(pairs)
    qo, ko, vo = (torch.full((n + 1, h * dh + pad), 9.0, device=DEV, dtype=dt) for h in (H, Hk, Hk))
    ctx.rope(q, qo[:n, pad:], f, dh, pos=pos, k=k, k_out=ko[:n, pad:], v=v, v_out=vo[:n, pad:], layout=layout)
    for x, y in ((q, qo), (k, ko)):
        close(y[:n, pad:], *R.rope(x, pos, f, dh, layout))
        assert bool((y[n] == 9).all() and (y[:, :pad] == 9).all())
    assert torch.equal(vo[:n, pad:], v) and bool((vo[n] == 9).all() and (vo[:, :pad] == 9).all())


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_positions_from_a_start(layout, ctx):
    x = rows(3, 50, 256, torch.float32)
    y = torch.empty_like(x)
    f = freqs(64, 500000.0)
    for start in (0, 12345, -7):
        ctx.rope(x, y, f, 128, pos0=start, layout=layout, scale=1.25)
        pos = torch.arange(start, start + 50, device=DEV)
        close(y, *R.rope(x, pos, f, 128, layout, 1.25))


def test_exact_angles_far_out(ctx):
    """One radian a position at 2^31 - 1: the angle of 64-bit arithmetic of more precision."""
    x = torch.zeros(1, 2, device=DEV)
    x[0, 0] = 1.0
    y = torch.empty_like(x)
    for p, cos, sin in ((2147483647, -0.6888366918779438, -0.7249165551445564), (1000000007, math.cos(1000000007), math.sin(1000000007))):
        ctx.rope(x, y, [1.0], 2, pos0=p)
        got = y.double().cpu().numpy()[0]
        # 2^-34 turns of the fraction of a turn, the angle's rounding to 24 bits, sincospif's two units
        assert abs(got[0] - cos) <= 12 * 2.0 ** -24 and abs(got[1] - sin) <= 12 * 2.0 ** -24


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pool", [64, 300])
def test_into_slots(dtype, pool, ctx):
    """Keys and values go to their slots, those outside the cache nowhere; other rows stay."""
    n, dt = 64, TYPES[dtype]
    q, k, v = (rows(i, n, 4 * 64, dt) for i in range(3))
    slots = torch.randperm(pool, device=DEV)[:n].int()
    slots[5], slots[9] = -1, pool
    qo, ko, vo = torch.empty_like(q), torch.full((pool, 256), 9.0, device=DEV, dtype=dt), torch.full((pool, 256), 9.0, device=DEV, dtype=dt)
    f = freqs(16)
    ctx.rope(q, qo, f, 64, k=k, k_out=ko, v=v, v_out=vo, slots=slots)
    pos = torch.arange(n, device=DEV)
    close(qo, *R.rope(q, pos, f, 64, "half"))
    kept = (slots >= 0) & (slots < pool)
    at = slots[kept].long()
    want, tol = R.rope(k, pos, f, 64, "half")
    close(ko[at], want[kept], tol[kept])
    assert torch.equal(vo[at], v[kept])
    rest = torch.ones(pool, dtype=torch.bool, device=DEV)
    rest[at] = False
    assert bool((ko[rest] == 9).all() and (vo[rest] == 9).all())


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("pairs", [64, 16, 5])
def test_in_place_and_parts(layout, pairs, ctx):
    """In place, in columns of one wider matrix, and each tensor alone: the same bits."""
    n, f = 90, freqs(pairs)
    qkv = rows(1, n, 5 * 128, torch.bfloat16).contiguous()
    q, k, v = qkv[:, :256], qkv[:, 256:384], qkv[:, 512:]
    outs = [torch.empty_like(t.contiguous()) for t in (q, k, v)]
    ctx.rope(q, outs[0], f, 128, k=k, k_out=outs[1], v=v, v_out=outs[2], layout=layout)
    alone = torch.empty_like(outs[1])
    ctx.rope(None, None, f, 128, k=k, k_out=alone, layout=layout)
    assert torch.equal(alone, outs[1])
    ctx.rope(None, None, f, 128, v=v, v_out=alone, layout=layout)
    assert torch.equal(alone, v)
    side, before = qkv[:, 384:512], qkv.clone()
    ctx.rope(None, None, f, 128, k=k, k_out=side, layout=layout)  # beside its own input
    assert torch.equal(side, outs[1]) and torch.equal(qkv[:, :384], before[:, :384])
    ctx.rope(q, q, f, 128, k=k, k_out=k, v=v, v_out=v, layout=layout)
    assert torch.equal(q, outs[0]) and torch.equal(k, outs[1]) and torch.equal(v, before[:, 512:])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_backward(layout, ctx):
    """The gradient of sum(y g) by x is g rotated backwards: against the formula, and against differences of
    the forward pass (linear in x, so exact but for roundings)."""
    n, dh, f = 40, 64, freqs(24)
    x, g = rows(1, n, 2 * dh, torch.float32), rows(2, n, 2 * dh, torch.float32)
    pos = torch.randint(0, 100000, (n,), device=DEV, dtype=torch.int32)
    grad = torch.empty_like(x)
    ctx.rope(g, grad, f, dh, pos=pos, layout=layout, scale=0.75, inverse=True)
    close(grad, *R.rope(g, pos, f, dh, layout, 0.75, inverse=True))
    a, b = torch.empty_like(x), torch.empty_like(x)
    for col in (0, 1, 23, 24, 47, 48, 63, 64, 127):
        up, down = x.clone(), x.clone()
        up[:, col] += 1.0
        down[:, col] -= 1.0
        ctx.rope(up, a, f, dh, pos=pos, layout=layout, scale=0.75)
        ctx.rope(down, b, f, dh, pos=pos, layout=layout, scale=0.75)
        diff = ((a.double() - b.double()) * g.double()).sum(1) / (up[:, col].double() - down[:, col].double())
        # two outputs of each of two evaluations, each off by 15 units of |a| + |b| <= 12, times |g| <= 6
        assert bool(((grad[:, col].double() - diff).abs() <= 4 * 15 * 2.0 ** -24 * 12 * 6).all())


def test_values_that_are_not_finite_stay_in_their_pair(ctx):
    x = rows(4, 8, 128, torch.float32).clone()
    x[3, 10], x[5, 100] = math.nan, math.inf
    y = torch.empty_like(x)
    ctx.rope(x, y, freqs(32), 128)  # pairs (i, i + 32) of the first 64
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[3, 10] = want[3, 42] = want[5, 100] = True
    assert torch.equal(bad, want)


def test_offsets_past_32_bits(ctx):
    """A cache row whose elements lie past 2^32 bytes and 2^31 elements."""
    ld, n = 1 << 16, 40000
    cache = torch.empty(n, ld, device=DEV, dtype=torch.bfloat16)
    k = rows(1, 3, 128, torch.bfloat16).contiguous()
    slots = torch.tensor([n - 1, 0, 33000], device=DEV, dtype=torch.int32)
    ctx.rope(None, None, freqs(64), 128, k=k, k_out=cache[:, :128], slots=slots)
    want, tol = R.rope(k, torch.arange(3, device=DEV), freqs(64), 128, "half")
    close(cache[slots.long(), :128], want, tol)
    big = cache[:, 128:256]
    big.copy_(torch.randn(n, 1, device=DEV).expand(n, 128))
    y = torch.empty(n, 128, device=DEV, dtype=torch.bfloat16)
    ctx.rope(big, y, freqs(64), 128)
    want, tol = R.rope(big[-5:], torch.arange(n - 5, n, device=DEV), freqs(64), 128, "half")
    close(y[-5:], want, tol)


def test_captured_and_replayed(ctx):
    x = rows(1, 33, 256, torch.bfloat16).contiguous()
    pos = torch.arange(33, device=DEV, dtype=torch.int32)
    y, want = torch.empty_like(x), torch.empty_like(x)
    s = torch.cuda.Stream()
    try:
        with torch.cuda.stream(s):
            ctx.set_stream(s.cuda_stream)
            graph = torch.cuda.CUDAGraph()
            f = freqs(64)
            with torch.cuda.graph(graph, stream=s):
                ctx.rope(x, y, f, 128, pos=pos)
            f[:] = 0  # read before the call returned
            for shift in (0, 100):
                pos.copy_(torch.arange(shift, shift + 33, device=DEV))
                x.mul_(1.5)
                graph.replay()
                ctx.rope(x, want, freqs(64), 128, pos=pos)
                s.synchronize()
                assert torch.equal(y, want)
    finally:
        ctx.set_stream(0)


def test_refusals(ctx):
    x, y = torch.zeros(8, 256, device=DEV), torch.empty(8, 256, device=DEV)
    f = freqs(64)
    for call in (
        lambda: ctx.rope(x, y, freqs(65), 128),                                # more pairs than a head has
        lambda: ctx.rope(x, y, [], 128),
        lambda: ctx.rope(x[:, :255], y[:, :255], [1.0], 85),                   # an odd width
        lambda: ctx.rope(x, y, [math.nan], 128),
        lambda: ctx.rope(x, y, [math.inf], 128),
        lambda: ctx.rope(x, y, f, 128, scale=math.inf),
        lambda: ctx.rope(torch.zeros(8, 264, device=DEV), torch.empty(8, 264, device=DEV), freqs(4), 264),
        lambda: ctx.rope(x, x, f, 128, k=x, k_out=y),  # q_out over k
        lambda: ctx.rope(x[:4], x[2:6], f, 128),                               # moved by two rows
        lambda: ctx.rope(x[:, :128], x[:, 64:192], f, 128),                    # and by half a head
        lambda: ctx.rope(x, y, f, 128, k=x, k_out=y),                          # one output for both
        lambda: ctx.rope(x, y, f, 128, pos=y.view(torch.int32)[1, :8]),        # positions in an output
        lambda: ctx.rope(None, None, f, 128, k=x, k_out=x, slots=torch.arange(8, device=DEV, dtype=torch.int32)),
    ):
        with pytest.raises(bag.BagError) as e:
            call()
        assert e.value.status == 1
    for call in (
        lambda: ctx.rope(x, None, f, 128),
        lambda: ctx.rope(x, y.half(), f, 128),
        lambda: ctx.rope(x, y[:4], f, 128),
        lambda: ctx.rope(x, y, f, 100),
        lambda: ctx.rope(x.t(), y.t(), f, 8),
        lambda: ctx.rope(x, y, f, 128, pos=torch.zeros(7, device=DEV, dtype=torch.int32)),
        lambda: ctx.rope(x, y, f, 128, pos=torch.zeros(8, device=DEV, dtype=torch.int64)),
        lambda: ctx.rope(x, y, f, 128, k=x[:4], k_out=y[:4]),
        lambda: ctx.rope(x.double(), y.double(), f, 128),
    ):
        with pytest.raises(ValueError):
            call()
    ctx.rope(x[:0], y[:0], f, 128)
    assert bool((x == 0).all())
