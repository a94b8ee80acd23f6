"""Plain 64-bit restatements of rotary positions and of attention of packed sequences, with the error that
the operators may have.  Test code only."""

import math

import torch

HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def rope(x, pos, freqs, dh, layout, scale=1.0, inverse=False):
    """x [rows, heads * dh] in float64, and a bound of what an fp32 evaluation rounded to x's type may differ by:
    the angle (2^-24 of half a turn, and sincospif's own error of 2 units) and the products' and scale's
    roundings (5), relative to |a| + |b| of the pair, then the output's half step."""
    rows, n = x.shape[0], len(freqs)
    y = x.double().reshape(rows, -1, dh).clone()
    mag = torch.zeros_like(y)
    angle = pos.double().unsqueeze(1) * torch.tensor(list(freqs), dtype=torch.float64, device=x.device)
    angle = -angle if inverse else angle
    i = torch.arange(n, device=x.device)
    i0, i1 = (i, i + n) if layout == "half" else (2 * i, 2 * i + 1)
    c, s = torch.cos(angle).unsqueeze(1) * scale, torch.sin(angle).unsqueeze(1) * scale
    a, b = y[:, :, i0], y[:, :, i1]
    y[:, :, i0], y[:, :, i1] = a * c - b * s, a * s + b * c
    mag[:, :, i0] = mag[:, :, i1] = (a.abs() + b.abs()) * abs(scale)
    # far positions: the product of two doubles above is itself off by 2^-53 of the angle
    far = float(angle.abs().max()) * 2.0 ** -52 if rows else 0.0
    tol = mag * ((math.pi + 7) * 2.0 ** -24 + far)
    tol = tol + HALF_STEP[x.dtype] * (y.abs() + tol) * (mag > 0)
    if x.dtype == torch.float16:
        tol = tol + 2.0 ** -25 * (mag > 0)  # half a step below the smallest normal
    return y.reshape(rows, -1), tol.reshape(rows, -1)


def attention(q, k, v, heads, kv_heads, seqs, causal=True, scale=None, pk=None, pv=None):
    """o [nq, heads, dh] and lse [nq, heads] in float64 (rows of no sequence: NaN), and bounds of the error.
    seqs: (first query, queries, first key, keys) of each.

    With weights w <= 1 (the largest 1), l their sum, A = sum w |v| / l, and u the half step of the type:
    weights are rounded to the type, by max(u w, 2^-25) with fp16 (below its normal range) or u w; a
    score carries dh roundings of the products' magnitude and a few of its own, twice in w / l; n sums
    in fp32 that may cut instead of rounding; 2^-21 for exp2 and the division; then the output's half
    step."""
    nq, G = q.shape[0], heads // kv_heads
    dh = q.shape[1] // heads
    scale = 1.0 / math.sqrt(dh) if scale is None else scale
    dev, u, f16 = q.device, HALF_STEP[q.dtype], q.dtype == torch.float16
    out = torch.full((nq, heads, dh), math.nan, dtype=torch.float64, device=dev)
    lse = torch.full((nq, heads), math.nan, dtype=torch.float64, device=dev)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    for q0, lq, k0, lk in seqs:
        if lq == 0:
            continue
        for h in range(heads):
            c = slice(h // G * dh, (h // G + 1) * dh)
            kk, vv = k[k0:k0 + lk, c].double(), v[k0:k0 + lk, c].double()
            seen = torch.ones(lq, lk, dtype=torch.bool, device=dev)
            if causal:
                seen = torch.arange(lk, device=dev) <= torch.arange(lq, device=dev).unsqueeze(1) + (lk - lq)
            if pk is not None:
                kk, vv = torch.cat([pk[:, c].double(), kk]), torch.cat([pv[:, c].double(), vv])
                seen = torch.cat([torch.ones(lq, pk.shape[0], dtype=torch.bool, device=dev), seen], 1)
            qq = q[q0:q0 + lq, h * dh:(h + 1) * dh].double()
            z = (qq @ kk.T * scale).masked_fill(~seen, -math.inf)
            n = kk.shape[0]
            if n == 0:
                out[q0:q0 + lq, h], lse[q0:q0 + lq, h] = 0.0, -math.inf
                continue
            top = z.amax(1, keepdim=True)
            w = torch.exp(z - top.clamp(min=-1e300)) * seen
            l = w.sum(1, keepdim=True)
            empty = l == 0
            l = torch.where(empty, torch.ones_like(l), l)
            o = w @ vv / l
            a = w @ vv.abs() / l
            rounded = torch.clamp(u * w, min=2.0 ** -25) * seen if f16 else u * w
            products = scale * (qq.abs() @ kk.abs().T).masked_fill(~seen, 0).amax(1, keepdim=True)
            score = (dh + 8) * 2.0 ** -23 * products
            more = 2 * score + n * 2.0 ** -23 + 2.0 ** -21
            t = rounded @ vv.abs() / l + a * more
            tol[q0:q0 + lq, h] = t + u * (o.abs() + t) + (2.0 ** -25 if f16 else 0.0)
            out[q0:q0 + lq, h] = torch.where(empty, torch.zeros_like(o), o)
            lse[q0:q0 + lq, h] = (top + torch.log(l)).squeeze(1)
            ltol[q0:q0 + lq, h] = (more + 2.0 ** -22 * (top.abs().clamp(max=1e30) + torch.log(l))).squeeze(1)
            lse[q0:q0 + lq, h][empty.squeeze(1)] = -math.inf
    return out, tol, lse, ltol
