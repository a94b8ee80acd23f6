"""Attention of packed sequences where scores are minus infinity or weights vanish, in every form of the kernels: few and
many rows, keys in parts, behind a prefix."""

import math

import pytest
import torch

import test_gpu_packed as P
from paper_2608_09231_gb300 import bag

pytestmark = pytest.mark.gpu
DEV = "cuda"
HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def ctx(lib):
    c = bag.create("tiny", T=2, B=1)
    yield c
    c.operators_status()
    c.close()


def plain(b, causal=True):
    """o and lse in float64 by the definition (a row that sees no key: zeros; one that sees only scores of minus infinity:
    NaN and minus infinity), and bounds: a weight's rounding to the type, scores of dh products (of the finite
    ones) twice, sums that may cut, exp2 and the division, the output's half step."""
    G, dh, u = b.heads // b.kv_heads, b.dh, HALF_STEP[b.dt]
    n, scale, f16 = b.starts[-1], 1.0 / math.sqrt(b.dh), b.dt == torch.float16
    o = torch.zeros(n, b.heads, dh, dtype=torch.float64, device=DEV)
    lse = torch.full((n, b.heads), -math.inf, dtype=torch.float64, device=DEV)
    tol, ltol = torch.zeros_like(o), torch.zeros_like(lse)
    for q0, lq, k0, lk in b.seqs:
        for h in range(b.heads):
            c = slice(h // G * dh, (h // G + 1) * dh)
            k, v = b.k[k0:k0 + lk, c].double(), b.v[k0:k0 + lk, c].double()
            seen = torch.ones(lq, lk, dtype=torch.bool, device=DEV)
            if causal:
                seen = torch.arange(lk, device=DEV) <= torch.arange(lq, device=DEV).unsqueeze(1) + (lk - lq)
            if b.pk is not None:
                k, v = torch.cat([b.pk[:, c].double(), k]), torch.cat([b.pv[:, c].double(), v])
                seen = torch.cat([torch.ones(lq, b.pk.shape[0], dtype=torch.bool, device=DEV), seen], 1)
            if k.shape[0] == 0:
                continue
            q = b.q[q0:q0 + lq, h * dh:(h + 1) * dh].double()
            z = (q @ k.T * scale).masked_fill(~seen, -math.inf)
            top = z.amax(1, keepdim=True)
            w = torch.where(z == -math.inf, torch.zeros_like(z), torch.exp(z - top))
            l = w.sum(1, keepdim=True)
            got = torch.where(l > 0, w @ v / l, torch.where(seen.any(1, keepdim=True), math.nan, 0.0))
            a = w @ v.abs() / l.clamp(min=1e-300)
            kept = torch.where(k.isinf(), torch.zeros_like(k), k)
            products = scale * (q.abs() @ kept.abs().T).amax(1, keepdim=True)
            more = 2 * (dh + 8) * 2.0 ** -23 * products + k.shape[0] * 2.0 ** -23 + 2.0 ** -21
            t = u * a + a * more
            if f16:  # weights below the normal range: half a step of 2^-24, where the largest weight is 2^7 or more
                t = t + 2.0 ** -32 * (w > 0).double() @ v.abs() / l.clamp(min=1e-300)
            o[q0:q0 + lq, h] = got
            tol[q0:q0 + lq, h] = t + u * (got.abs().nan_to_num() + t) + (2.0 ** -25 if f16 else 0.0)
            lse[q0:q0 + lq, h] = (top + torch.log(l)).squeeze(1)
            ltol[q0:q0 + lq, h] = (more + 2.0 ** -22 * (top.abs() + torch.log(l).abs())).nan_to_num(0, 0, 0).squeeze(1)
    return o, tol, lse, ltol


def check(b, causal=True):
    o, tol, lse, ltol = plain(b, causal)
    n = b.starts[-1]
    got, gotl = b.o[:n].double().reshape(o.shape), b.lse[:n].double()
    assert torch.equal(got.isnan(), o.isnan())
    finite = ~o.isnan()
    assert bool(((got - o).abs() <= tol)[finite].all()), float(((got - o).abs() - tol)[finite].max())
    low = torch.isneginf(lse)
    assert torch.equal(low, torch.isneginf(gotl))
    assert bool(((gotl - lse).abs() <= ltol)[~low].all())
    return o


LENS = {
    "token": [(1, 700)],
    "tokens": [(1, 40), (1, 0), (1, 6000), (1, 129)],
    "pieces": [(2, 9000)],
    "prompt": [(300, 300), (5, 3)],
    "parts": [(40, 6000), (64, 100)],
}


@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("prefix", [None, 300])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("workspace", [True, False])
def test_keys_of_minus_infinity(lens, prefix, dh, dtype, workspace, ctx):
    """Keys with an infinity that all queries turn into a score of minus infinity: all keys of the first sequence, and every
    key but a few of the others; then the prefix's as well."""
    for hidden in (False, True) if prefix else (False,):
        b = P.Batch(LENS[lens], 8, 2, dh, dtype, key=7, prefix=prefix)
        cols = [h * dh for h in range(8)]
        b.q[:, cols] = b.q[:, cols].abs() + 0.25
        keys = [0, dh]  # the first column of each key head
        for i, (_, _, k0, lk) in enumerate(b.seqs):
            at = torch.arange(k0, k0 + lk, device=DEV)
            if i:
                at = at[torch.arange(lk, device=DEV) % 50 != 49]
            for c in keys:
                b.k[at, c] = -math.inf
        if hidden:
            b.pk[:, keys] = -math.inf
        o = check(b.run(ctx, work="all" if workspace else None))
        if prefix is None or hidden:
            assert bool(o.isnan().any())


@pytest.mark.parametrize("lq", [1, 3, 70])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("at", [0, 30000, 59999])
@pytest.mark.parametrize("prefix", [False, True])
def test_many_small_weights(lq, dh, at, prefix, ctx):
    """One key, and 60,000 of 2^-25.5 of its weight with all the values that are not zero: together 1.3e-3 of the result."""
    n, z = 60000, -17.671875
    b = P.Batch([(lq, 1 if prefix else n)], 4, 2, dh, "f16", prefix=n if prefix else None, pad=0, behind=0)
    k, v = (b.pk, b.pv) if prefix else (b.k[b.seqs[0][2]:][:n], b.v[b.seqs[0][2]:][:n])
    b.q.zero_()
    b.q[:, [h * dh for h in range(4)]] = 8.0
    scale = 1.0 / 8.0
    k.zero_()
    k[:, [0, dh]] = z
    k[at] = 0.0
    v.fill_(1.0)
    v[at] = 0.0
    if prefix:  # an own key that weighs nothing
        k0 = b.seqs[0][2]
        b.k[k0:k0 + 1] = 0.0
        b.k[k0:k0 + 1, [0, dh]] = -200.0
        b.v[k0:k0 + 1] = 0.0
    b.run(ctx, scale=scale, causal=False)
    w = math.exp(z)
    want = (n - 1) * w / (1.0 + (n - 1) * w)
    # a weight's rounding (2^-32 of the largest at most), the score's few operations on 17.7 twice, sums that may cut,
    # exp2 and the division; the output's half step
    tol = n * 2.0 ** -32 + want * (8 * 18 * 2.0 ** -23 + n * 2.0 ** -23 + 2.0 ** -21 + 2.0 ** -11) + 2.0 ** -25
    assert float((b.o.double() - want).abs().max()) <= tol
