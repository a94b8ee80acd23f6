"""Plain restatements (numpy, float64 unless a step is fp32 by definition) of the 8-bit format,
the quantised cache and the block selection, shared by their tests.  Test code only."""

import numpy as np

GROUP, TOP = {8: 128, 4: 32}, {8: 127, 4: 7}


def up(n, m):
    return (n + m - 1) // m * m


# every e4m3 value by its code, from the format: sign, 4 exponent bits (bias 7), 3 fraction bits;
# 0x7f and 0xff are NaN
_E, _F = (np.arange(256) >> 3) & 15, np.arange(256) & 7
E4M3 = np.where(_E == 0, _F * 2.0 ** -9, (8 + _F) * 2.0 ** (_E - 10.0)) * np.where(np.arange(256) >= 128, -1, 1)
E4M3[[0x7F, 0xFF]] = np.nan


def e4m3_code(v):
    """The code nearest to each |v| <= 448, ties to the even code."""
    mag = E4M3[:127]
    a = np.abs(v)
    hi = np.clip(np.searchsorted(mag, a), 1, 126)
    lo = hi - 1
    dl, dh = a - mag[lo], mag[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return (code + np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def quant(x):
    """(codes, scale bytes) of float32 rows."""
    rows, cols = x.shape
    x = x.astype(np.float64)
    nb = -(-cols // 128)
    codes, scales = np.zeros((rows, cols), np.uint8), np.zeros((rows, nb), np.uint8)
    for j in range(nb):
        v = x[:, 128 * j:128 * j + 128]
        amax = np.max(np.abs(v), axis=1)
        for r in range(rows):
            if not np.isfinite(amax[r]):
                scales[r, j], codes[r, 128 * j:128 * j + v.shape[1]] = 255, 0x7F
                continue
            b = 0
            while amax[r] > 448.0 * 2.0 ** (b - 127):
                b += 1
            scales[r, j] = b
            codes[r, 128 * j:128 * j + v.shape[1]] = e4m3_code(v[r] * 2.0 ** (127 - b))
    return codes, scales


def decode(codes, scales):
    """float64 values of an encoded matrix."""
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return E4M3[codes] * np.repeat(s, 128, axis=1)[:, :codes.shape[1]]


def gelu(y):
    return 0.5 * y * (1 + np.tanh(np.sqrt(2 / np.pi) * (y + 0.044715 * y ** 3)))


def bf16(x):
    """float32 rounded to bf16 (ties to even), as float32."""
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)


def cache(x, bits):
    """(integer codes, scales) of float32 rows, finite."""
    rows, cols = x.shape
    n = GROUP[bits]
    ng = -(-cols // n)
    codes, scales = np.zeros((rows, cols), np.int32), np.zeros((rows, ng), np.float32)
    for g in range(ng):
        v = x[:, g * n:g * n + n]
        s = bf16(np.max(np.abs(v), axis=1) * (np.float32(1) / np.float32(TOP[bits])))
        s = np.where(s < np.float32(2.0 ** -126), np.float32(0), s)
        scales[:, g] = s
        for r in range(rows):
            if s[r] > 0:
                q = np.rint(v[r] * (np.float32(1) / s[r]))
                codes[r, g * n:g * n + n] = np.clip(q, -TOP[bits], TOP[bits])
    return codes, scales


def pack(codes, bits):
    """Cache bytes of integer codes."""
    if bits == 8:
        return codes.astype(np.int8).view(np.uint8)
    c = np.pad(codes, ((0, 0), (0, codes.shape[1] % 2))) & 15
    return (c[:, 0::2] | c[:, 1::2] << 4).astype(np.uint8)


def pool(x, heads):
    """(codes [heads, blocks, 128], scales) of float32 rows [n, 128 * heads]."""
    n = x.shape[0]
    nb = -(-n // 128)
    v = np.zeros((nb * 128, heads * 128), np.float32)
    v[:n] = x
    v = v.reshape(nb, 128, heads, 128)
    with np.errstate(invalid="ignore", over="ignore"):
        for h in (64, 32, 16, 8, 4, 2, 1):
            v = v[:, :h] + v[:, h:2 * h]
        count = np.full(nb, 128, np.float32)
        count[-1] = n - 128 * (nb - 1)
        mean = v[:, 0].transpose(1, 0, 2) * (np.float32(1) / count)[None, :, None]
        amax = np.max(np.abs(mean), axis=2)
        scale = np.where(np.isfinite(amax), amax * (np.float32(1) / np.float32(127)), np.float32(0)).astype(np.float32)
        scale = np.where(scale < np.float32(2.0 ** -126), np.float32(0), scale)
        inv = np.where(scale > 0, np.float32(1) / np.where(scale > 0, scale, np.float32(1)), np.float32(0))
        codes = np.where(scale[..., None] > 0, np.clip(np.rint(mean * inv[..., None]), -127, 127), 0)
    return codes.astype(np.int8), scale


def select(qcodes, kcodes, kscales, keep):
    """Block lists [heads, query blocks, keep]."""
    H, nq, _ = qcodes.shape
    group = H // kcodes.shape[0]
    out = np.zeros((H, nq, keep), np.int32)
    for h in range(H):
        dot = qcodes[h].astype(np.int64) @ kcodes[h // group].astype(np.int64).T
        score = dot.astype(np.float32) * kscales[h // group][None]
        for i in range(nq):
            out[h, i] = np.sort(np.argsort(-score[i], kind="stable")[:keep])
    return out


def attention(q, k, v, blocks):
    """float64 attention over listed blocks: q [nq, H, 128], k, v [nk, Hk, 128], blocks [H, nqb, keep]
    (a list ends at its first entry that names no block; no keys: zeros)."""
    nq, H, _ = q.shape
    nk, Hk, _ = k.shape
    out = np.zeros((nq, H, 128))
    for h in range(H):
        for i in range(blocks.shape[1]):
            names = (blocks[h, i] >= 0) & (blocks[h, i] < -(-nk // 128))
            n = len(names) if names.all() else int(np.argmin(names))
            at = [np.arange(128 * j, min(nk, 128 * j + 128)) for j in blocks[h, i, :n]]
            if not at:
                continue
            at = np.concatenate(at)
            s = q[128 * i:128 * i + 128, h] @ k[at, h // (H // Hk)].T / np.sqrt(128.0)
            p = np.exp(s - s.max(axis=1, keepdims=True))
            out[128 * i:128 * i + 128, h] = p @ v[at, h // (H // Hk)] / p.sum(axis=1, keepdims=True)
    return out
