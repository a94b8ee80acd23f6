"""The 8-bit operands, their product and the quantised cache on the GPU, against plain restatements
in 64 bits, at the sizes where they can go wrong."""

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


def rng(*key):
    return np.random.default_rng([abs(int(k)) for k in key])


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def encoded(rows, cols, fill=0x55):
    """Empty buffers of an encoded matrix with a row of guard bytes before and after."""
    c = torch.full((rows + 2, R.up(cols, 16) + 16), fill, device=DEV, dtype=torch.uint8)
    s = torch.full((rows + 2, R.up(-(-cols // 128), 4) + 4), fill, device=DEV, dtype=torch.uint8)
    return c, s


def untouched(c, s, rows, cols, fill=0x55):
    nb = -(-cols // 128)
    for t, n in ((c, cols), (s, nb)):
        assert bool((t[0] == fill).all() and (t[rows + 1:] == fill).all() and (t[:, n:] == fill).all())


def spread(g, rows, cols):
    """Rows of very different size, with blocks of zeros, exact powers of two and 448 times one."""
    x = g.standard_normal((rows, cols)) * np.exp2(g.integers(-40, 40, (rows, 1)))
    x[g.random((rows, cols)) < 0.05] *= 1e-4
    for r in range(rows):
        for j in range(0, cols, 128):
            u = g.random()
            if u < 0.1:
                x[r, j:j + 128] = 0
            elif u < 0.3:
                x[r, j:j + 128] = np.clip(x[r, j:j + 128], -1, 1)
                x[r, j] = 448.0 * 2.0 ** g.integers(-9, 3)
    return x.astype(np.float32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 127), (2, 128), (5, 129), (9, 513), (4, 1025), (7, 2052), (64, 5120)])
@pytest.mark.parametrize("pad", [0, 1, 8])  # 16-byte rows and not
def test_quant_is_bit_exact(rows, cols, dtype, pad, ctx):
    x = spread(rng(rows, cols, pad), rows, cols)
    if dtype == "bf16":
        x = R.bf16(x)
    buf = torch.full((rows, cols + pad), float("nan"), device=DEV)
    buf[:, pad:] = dev(x)
    if dtype == "bf16":
        buf = buf.bfloat16()
    c, s = encoded(rows, cols)
    ctx.quant_fp8(buf[:, pad:], c[1:rows + 1], s[1:rows + 1])
    codes, scales = R.quant(x)
    assert np.array_equal(s[1:rows + 1, :scales.shape[1]].cpu().numpy(), scales)
    got = c[1:rows + 1, :cols].cpu().numpy()
    zero = (got & 127) == 0  # a zero's sign is the element's
    assert np.array_equal(np.where(zero, 0, got), np.where((codes & 127) == 0, 0, codes))
    untouched(c, s, rows, cols)


def test_quant_extremes(ctx):
    """The smallest and largest fp32 blocks, and infinities and NaN, which take their own block
    alone with them."""
    x = np.zeros((6, 384), np.float32)
    x[:, 128:256] = rng(1).standard_normal((6, 128))
    x[0, 5] = np.float32(1e-45)
    x[1, 5] = np.finfo(np.float32).max
    x[2, 5] = np.inf
    x[3, 5] = -np.inf
    x[4, 5] = np.nan
    x[5, 5], x[5, 300] = np.float32(3e-38), -np.float32(2.0 ** -126)
    c, s = encoded(6, 384)
    ctx.quant_fp8(dev(x), c[1:7], s[1:7])
    codes, scales = R.quant(x)
    assert np.array_equal(s[1:7, :3].cpu().numpy(), scales)
    got = R.decode(c[1:7, :384].cpu().numpy(), scales)
    want = R.decode(codes, scales)
    assert np.array_equal(got, want, equal_nan=True)
    assert list(scales[2:5, 0]) == [255] * 3 and scales[2, 1] != 255


@pytest.mark.parametrize("cols", [4, 124, 128, 132, 508, 3072, 3076, 5120, 5124, 6144])
@pytest.mark.parametrize("mod", [True, False])
def test_ln_mod_fp8(cols, mod, ctx):
    """Against float64: half a step of e4m3 (2^-4 of a normal code's value, 2^-10 of the block's
    scale below) on top of fp32 statistics (2e-5 of the row's largest value covers sums over 6144
    columns); the scale is the least that fits, up to that error of the block's maximum."""
    g = rng(cols)
    x = (2.0 * g.standard_normal((5, cols)) + 0.5).astype(np.float32)
    sh, sc = (0.5 * g.standard_normal(cols).astype(np.float32) for _ in range(2))
    c, s = encoded(5, cols)
    ctx.ln_mod_fp8(dev(x), dev(sh) if mod else None, dev(sc) if mod else None, c[1:6], s[1:6])
    xd = x.astype(np.float64)
    ref = (xd - xd.mean(1, keepdims=True)) / np.sqrt(xd.var(1, keepdims=True) + 1e-6)
    if mod:
        ref = ref * (1 + sc.astype(np.float64)) + sh
    nb = -(-cols // 128)
    scales = s[1:6, :nb].cpu().numpy()
    got = R.decode(c[1:6, :cols].cpu().numpy(), scales)
    step = np.repeat(2.0 ** (scales.astype(np.float64) - 127), 128, axis=1)[:, :cols]
    eps = 2e-5 * np.abs(ref).max(1, keepdims=True)
    assert (np.abs(got - ref) <= 2.0 ** -4 * np.abs(ref) + 2.0 ** -10 * step + eps).all()
    for j in range(nb):
        amax = np.abs(ref[:, 128 * j:128 * j + 128]).max(1)
        b = 2.0 ** (scales[:, j].astype(np.float64) - 127)
        assert (amax <= 448 * b + eps[:, 0]).all() and (amax >= 224 * b - eps[:, 0]).all()
    untouched(c, s, 5, cols)


def operand(g, rows, cols, spread_bits=6):
    """A random encoded matrix (every finite code, scales that differ from block to block) with
    guard bytes that would be NaN around it; returns device views and float64 values."""
    nb = -(-cols // 128)
    codes = g.integers(0, 256, (rows, cols)).astype(np.uint8)
    codes[(codes & 127) == 127] = 0
    scales = g.integers(127 - spread_bits, 128 + spread_bits, (rows, nb)).astype(np.uint8)
    c = torch.full((rows + 1, R.up(cols, 16) + 16), 0x7F, device=DEV, dtype=torch.uint8)
    s = torch.full((rows + 1, R.up(nb, 4) + 4), 255, device=DEV, dtype=torch.uint8)
    c[:rows, :cols], s[:rows, :nb] = dev(codes), dev(scales)
    return c[:rows], s[:rows], dev(R.decode(codes, scales))


GEMM_SHAPES = [
    (1, 1, 1), (1, 128, 128), (1, 300, 640), (3, 64, 5000), (16, 130, 129), (17, 257, 512), (33, 128, 1664),
    (65, 512, 127), (128, 1000, 1152), (129, 384, 2048), (200, 96, 8192), (455, 1536, 512), (1373, 640, 768),
    (255, 2000, 272), (257, 4097, 384), (700, 5120, 1040), (2500, 2304, 640),
]


@pytest.mark.parametrize("M,N,K", GEMM_SHAPES)
@pytest.mark.parametrize("kind", ["f32", "bf16", "fp8", "resid"])
def test_gemm_fp8(M, N, K, kind, ctx):
    """Every product is exact in fp32, so the error is that of the fp32 sums: at most 4 K 2^-24 of
    the sum of magnitudes (as for the bf16 product), then the output's own rounding: bf16 2^-8, e4m3
    2^-4 (below its normal range 2^-10 of the block's scale), fp32 2^-22 with GELU's 2^-19."""
    g = rng(M, N, K)
    a, a_s, A = operand(g, M, K)
    w, w_s, W = operand(g, N, K)
    bias = dev(g.standard_normal(N).astype(np.float32))
    y = A @ W.T + bias.double()
    # GELU would leave only its linear part of sums this large: bring them to a few units
    gelu = (M + N + K) % 2 == 0 and kind != "resid"
    if gelu:
        a_s -= int(np.ceil(np.log2(max(1.0, float(y.abs().max()) / 8))))
        A = A * 2.0 ** (float(a_s[0, 0]) - float(g_first(M, N, K)))
        y = A @ W.T + bias.double()
    eps = 4 * K * 2.0 ** -24 * (A.abs() @ W.abs().T + bias.double().abs())
    ref = torch.from_numpy(R.gelu(y.cpu().numpy())).to(DEV) if gelu else y
    eps = eps * 1.2 + 2.0 ** -19 * ref.abs() + 1e-7
    if kind == "fp8":
        c, s = encoded(M, N)
        ctx.gemm_fp8(a, a_s, w, w_s, c[1:M + 1], K, bias=bias, gelu=gelu, out_scales=s[1:M + 1])
        nb = -(-N // 128)
        sc = s[1:M + 1, :nb].cpu().numpy()
        got = dev(R.decode(c[1:M + 1, :N].cpu().numpy(), sc))
        step = dev(np.repeat(2.0 ** (sc.astype(np.float64) - 127), 128, axis=1)[:, :N])
        assert bool(((got - ref).abs() <= 2.0 ** -4 * ref.abs() + 2.0 ** -10 * step + 1.1 * eps).all())
        top = torch.nn.functional.pad(ref.abs(), (0, nb * 128 - N)).view(M, nb, 128).amax(2)
        more = torch.nn.functional.pad(eps, (0, nb * 128 - N)).view(M, nb, 128).amax(2)
        assert bool((top <= 448 * step[:, ::128] + more).all() and (top >= 224 * step[:, ::128] - more).all())
        untouched(c, s, M, N)
        return
    out = torch.full((M + 2, N + 3), 7.0, device=DEV, dtype=torch.bfloat16 if kind == "bf16" else torch.float32)
    o = out[1:M + 1, :N]
    if kind == "resid":
        h, gate = (dev(g.standard_normal((M, N)).astype(np.float32)), dev(g.standard_normal(N).astype(np.float32)))
        o.copy_(h)
        ctx.gemm_fp8(a, a_s, w, w_s, o, K, bias=bias, gate=gate, residual=True)
        ref = h.double() + gate.double() * y
        eps = eps * gate.double().abs() + 2.0 ** -22 * (ref.abs() + h.double().abs())
    else:
        ctx.gemm_fp8(a, a_s, w, w_s, o, K, bias=bias, gelu=gelu)
        eps = eps + 2.0 ** (-8 if kind == "bf16" else -22) * ref.abs()
    assert bool(((o.double() - ref).abs() <= eps).all()), float(((o.double() - ref).abs() / eps).max())
    out[1:M + 1, :N] = 7.0
    assert bool((out == 7.0).all())


def g_first(M, N, K):
    """The first scale byte that operand() gives to test_gemm_fp8's A."""
    g = rng(M, N, K)
    g.integers(0, 256, (M, K))
    return g.integers(121, 134, (M, -(-K // 128))).astype(np.uint8)[0, 0]


@pytest.mark.parametrize("M,N,K", [(2500, 2304, 640), (2433, 2309, 1040), (2305, 2050, 127), (4700, 1156, 2176),
                                   (130, 19500, 384), (19500, 136, 4224), (5000, 2500, 13824)])
@pytest.mark.parametrize("kind,aligned", [("f32", True), ("bf16", True), ("fp8", True), ("resid", True), ("f32", False),
                                          ("bf16", False), ("resid", False)])
def test_gemm_fp8_of_many_tiles(M, N, K, kind, aligned, ctx):
    """Enough 256 x 256 tiles for a CTA pair each and more, ragged in M, N and K, one to seven runs of
    scale words, scale rows of whole 16-byte units and not, output rows that TMA can address and rows
    that it cannot (code rows always are).  Bounds as in test_gemm_fp8."""
    g = rng(M, N, K)
    a, a_s, A = operand(g, M, K)
    w, w_s, W = operand(g, N, K)
    if aligned:  # 16-byte scale rows
        nb = -(-K // 128)
        t = torch.full((M, R.up(nb, 16)), 255, device=DEV, dtype=torch.uint8)
        t[:, :nb], a_s = a_s[:, :nb], t
    bias, gate = (dev(g.standard_normal(N).astype(np.float32)) for _ in range(2))
    y = A @ W.T + bias.double()
    eps = 4 * K * 2.0 ** -24 * (A.abs() @ W.abs().T + bias.double().abs())
    if kind == "fp8":
        c, s = encoded(M, N)
        ctx.gemm_fp8(a, a_s, w, w_s, c[1:M + 1], K, bias=bias, out_scales=s[1:M + 1])
        nb = -(-N // 128)
        codes, sc = c[1:M + 1, :N].contiguous(), s[1:M + 1, :nb].double()
        step = torch.exp2(sc - 127).repeat_interleave(128, 1)[:, :N]
        got = codes.view(torch.float8_e4m3fn).double() * step
        assert bool(((got - y).abs() <= 2.0 ** -4 * y.abs() + 2.0 ** -10 * step + 1.1 * eps).all())
        top = torch.nn.functional.pad(y.abs(), (0, nb * 128 - N)).view(M, nb, 128).amax(2)
        more = torch.nn.functional.pad(eps, (0, nb * 128 - N)).view(M, nb, 128).amax(2)
        assert bool((top <= 448 * step[:, ::128] + more).all() and (top >= 224 * step[:, ::128] - more).all())
        untouched(c, s, M, N)
        return
    width = R.up(N, 8) + 8 if aligned else R.up(N, 8) + 1
    out = torch.full((M + 2, width), 7.0, device=DEV, dtype=torch.bfloat16 if kind == "bf16" else torch.float32)
    o = out[1:M + 1, :N]
    if kind == "resid":
        h = dev(g.standard_normal((M, N)).astype(np.float32))
        o.copy_(h)
        ctx.gemm_fp8(a, a_s, w, w_s, o, K, bias=bias, gate=gate, residual=True)
        ref = h.double() + gate.double() * y
        eps = eps * gate.double().abs() + 2.0 ** -22 * (ref.abs() + h.double().abs())
    else:
        ctx.gemm_fp8(a, a_s, w, w_s, o, K, bias=bias)
        ref, eps = y, eps + 2.0 ** (-8 if kind == "bf16" else -22) * y.abs()
    assert bool(((o.double() - ref).abs() <= eps).all()), float(((o.double() - ref).abs() / eps).max())
    out[1:M + 1, :N] = 7.0
    assert bool((out == 7.0).all())


@pytest.mark.parametrize("M,N,K", [(5, 300, 640), (600, 1024, 512), (3000, 2048, 640)])
def test_gemm_fp8_without_bias_or_gate(M, N, K, ctx):
    g = rng(M, N)
    a, a_s, A = operand(g, M, K)
    w, w_s, W = operand(g, N, K)
    out = torch.zeros(M, N, device=DEV)
    ctx.gemm_fp8(a, a_s, w, w_s, out, K, residual=True)
    again = torch.zeros(M, N, device=DEV)
    ctx.gemm_fp8(a, a_s, w, w_s, again, K)
    eps = 4 * K * 2.0 ** -24 * (A.abs() @ W.abs().T)
    assert bool(((out.double() - A @ W.T).abs() <= eps).all()) and torch.equal(out, again)
    ctx.gemm_fp8(a[:0], a_s[:0], w, w_s, out, K)  # no rows: nothing happens
    assert torch.equal(out, again)


@pytest.mark.parametrize("M,N", [(1, 512), (77, 13824), (300, 640), (2500, 2304)])
@pytest.mark.parametrize("K", [8192, 8320, 13824])
def test_gemm_fp8_keeps_long_sums_in_fp32(M, N, K, ctx):
    """The tensor core drops what an addend has below the accumulator's last bits, so sums of more than
    8192 products are taken in parts (passes, or the CTAs that share K).  On normal rows one part of
    13824 products is off by 1.2e-6 (2-norm), and the error grows with the length: at most 1e-6."""
    g = torch.Generator(device=DEV).manual_seed(M + N + K)
    ops, exact = [], []
    for rows in (M, N):
        c, s = encoded(rows, K)
        ctx.quant_fp8(torch.randn(rows, K, generator=g, device=DEV), c[1:rows + 1], s[1:rows + 1])
        ops += [c[1:rows + 1], s[1:rows + 1]]
        step = torch.exp2(ops[-1][:, :-(-K // 128)].double() - 127).repeat_interleave(128, 1)[:, :K]
        exact.append(ops[-2][:, :K].contiguous().view(torch.float8_e4m3fn).double() * step)
    out = torch.empty(M, N, device=DEV)
    ctx.gemm_fp8(*ops, out, K)
    ref = exact[0] @ exact[1].T
    assert float((out.double() - ref).norm() / ref.norm()) <= 1e-6


@pytest.mark.parametrize("M", [4, 900])
def test_gemm_fp8_nan_scale_reaches_its_row_only(M, ctx):
    g = rng(M)
    K, N = 640, 1280
    a, a_s, _ = operand(g, M, K)
    w, w_s, _ = operand(g, N, K)
    a_s[2, 3], w_s[77, 1] = 255, 255
    out = torch.zeros(M, N, device=DEV)
    ctx.gemm_fp8(a, a_s, w, w_s, out, K)
    nan = torch.isnan(out)
    want = torch.zeros_like(nan)
    want[2], want[:, 77] = True, True
    assert torch.equal(nan, want)


# ---------------------------------------------------------------------------
# quantised cache
# ---------------------------------------------------------------------------
def cache_buffers(cap, cols, bits, fill=0x5A):
    c = torch.full((cap, R.up((cols * bits + 7) // 8, 16) + 16), fill, device=DEV, dtype=torch.uint8)
    s = torch.full((cap, -(-cols // R.GROUP[bits]) + 3), 9.0, device=DEV, dtype=torch.bfloat16)
    return c, s


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("rows,cols", [(1, 1), (2, 3), (5, 31), (3, 32), (4, 33), (7, 127), (2, 129), (9, 515), (33, 1536)])
@pytest.mark.parametrize("slotted", [False, True])
@pytest.mark.parametrize("pad", [0, 1])
def test_cache_write_and_read(rows, cols, bits, slotted, pad, ctx):
    g = rng(rows, cols, bits)
    h = (g.standard_normal((rows, cols + pad)) * 3).astype(np.float32)
    x = (h + g.standard_normal((rows, cols + pad)) * np.exp2(g.integers(-20, 20, (rows, 1)))).astype(np.float32)
    x[:, :cols // 3] = h[:, :cols // 3]  # groups of zeros
    cap = rows + 4
    c, s = cache_buffers(cap, cols, bits)
    slots = g.permutation(cap)[:rows].astype(np.int32) if slotted else np.arange(rows, dtype=np.int32)
    if slotted and rows > 4:
        slots[1], slots[3] = -1, cap  # no slot: skipped, and read as zeros
    kw = dict(slots=dev(slots) if slotted else None)
    hd, xd = dev(h)[:, pad:], dev(x)[:, pad:]
    ctx.cache_write(xd, c, s, bits, base=hd, **kw)
    codes, scales = R.cache((x - h)[:, pad:], bits)
    want_c, want_s = np.full(c.shape, 0x5A, np.uint8), np.full(s.shape, 9.0, np.float32)
    held = [r for r in range(rows) if 0 <= slots[r] < cap]
    packed = R.pack(codes, bits)
    for r in held:
        want_c[slots[r], :packed.shape[1]], want_s[slots[r], :scales.shape[1]] = packed[r], scales[r]
    assert np.array_equal(c.cpu().numpy(), want_c) and np.array_equal(s.float().cpu().numpy(), want_s)
    value = np.zeros((rows, cols))
    for r in held:
        value[r] = codes[r] * np.repeat(scales[r].astype(np.float64), R.GROUP[bits])[:cols]
    out = torch.full((rows + 1, cols + 1), 5.0, device=DEV)
    ctx.cache_read(c, s, out[:rows, :cols], bits, base=hd, **kw)
    got = out[:rows, :cols].double().cpu().numpy()
    ref = h[:, pad:].astype(np.float64) + value
    assert (np.abs(got - ref) <= 2.0 ** -23 * (np.abs(ref) + np.abs(value))).all()
    assert bool((out[rows] == 5.0).all() and (out[:, cols] == 5.0).all())
    ctx.cache_read(c, s, out[:rows, :cols], bits, **kw)
    got = out[:rows, :cols].double().cpu().numpy()
    assert (np.abs(got - value) <= 2.0 ** -24 * np.abs(value)).all()
    ctx.cache_read(c, s, hd, bits, base=hd, **kw)  # in place
    assert (np.abs(hd.double().cpu().numpy() - ref) <= 2.0 ** -23 * (np.abs(ref) + np.abs(value))).all()


@pytest.mark.parametrize("bits", [8, 4])
def test_cache_of_values_that_are_not_finite(bits, ctx):
    """An infinity, a NaN or an overflowing difference makes its group read as NaN, and no other;
    groups too small for a scale are kept as zeros."""
    n = R.GROUP[bits]
    x = np.ones((4, 2 * n), np.float32)
    x[0, 3], x[1, n + 1], x[2, 0] = np.inf, np.nan, 3e38
    x[3, n:] = 1e-40
    h = np.zeros_like(x)
    h[2, 0] = -3e38
    c, s = cache_buffers(4, 2 * n, bits)
    ctx.cache_write(dev(x), c, s, bits, base=dev(h))
    out = torch.empty(4, 2 * n, device=DEV)
    ctx.cache_read(c, s, out, bits)
    nan = np.isnan(out.cpu().numpy()).reshape(4, 2, n)
    assert nan[0, 0].all() and nan[1, 1].all() and nan[2, 0].all() and nan.sum() == 3 * n
    one = R.TOP[bits] * R.bf16(np.float32(1) / np.float32(R.TOP[bits]))
    assert (out.cpu().numpy()[3, n:] == 0).all() and (out.cpu().numpy()[3, :n] == one).all()


@pytest.mark.parametrize("bits", [8, 4])
def test_cache_offsets_past_32_bits(bits, ctx):
    """The last slots of a cache of more than 2^32 bytes of codes and of 2^31 scales' bytes."""
    cols = 4096
    ldc = cols * bits // 8
    cap = (1 << 32) // ldc + 5
    c = torch.empty(cap, ldc, device=DEV, dtype=torch.uint8)
    s = torch.empty(cap, cols // R.GROUP[bits], device=DEV, dtype=torch.bfloat16)
    x = rng(bits).standard_normal((3, cols)).astype(np.float32)
    slots = dev(np.array([cap - 1, 0, cap - 4], np.int32))
    ctx.cache_write(dev(x), c, s, bits, slots=slots)
    codes, scales = R.cache(x, bits)
    packed = R.pack(codes, bits)
    for r, slot in enumerate((cap - 1, 0, cap - 4)):
        assert np.array_equal(c[slot].cpu().numpy(), packed[r])
        assert np.array_equal(s[slot].float().cpu().numpy(), scales[r])
    out = torch.empty(3, cols, device=DEV)
    ctx.cache_read(c, s, out, bits, slots=slots)
    ref = codes * np.repeat(scales.astype(np.float64), R.GROUP[bits], axis=1)
    assert (np.abs(out.double().cpu().numpy() - ref) <= 2.0 ** -24 * np.abs(ref)).all()
