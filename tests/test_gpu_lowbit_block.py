"""The low-precision block: its steps against the same block in float64, the calls captured in a
graph, on another stream, and what they refuse."""

import math

import pytest
import torch

from paper_2608_09231_gb300 import bag, lowbit

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ctx(lib):
    c = bag.create("tiny", T=2, B=1)
    yield c
    c.close()


def plain(w, h, mod, heads):
    """The block in float64 with every key block listed."""
    def ln(x, shift, scale):
        d = x - x.mean(1, keepdim=True)
        return d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-6) * (1 + scale) + shift

    w = {n: t.double() for n, t in w.items()}
    sa, ca, ga, sm, cm, gm = (m.double() for m in mod)
    h = h.double()
    x = ln(h, sa, ca)
    q, k, v = x @ w["wq"].T + w["bq"], x @ w["wk"].T + w["bk"], x @ w["wv"].T
    q, k, v = (t.view(-1, heads, 128).transpose(0, 1) for t in (q, k, v))
    o = torch.softmax(q @ k.transpose(1, 2) / math.sqrt(128), 2) @ v
    h = h + ga * (o.transpose(0, 1).reshape(h.shape) @ w["wo"].T + w["bo"])
    u = ln(h, sm, cm) @ w["wu"].T + w["bu"]
    u = 0.5 * u * (1 + torch.tanh(math.sqrt(2 / math.pi) * (u + 0.044715 * u ** 3)))
    return h + gm * (u @ w["wd"].T + w["bd"])


@pytest.mark.parametrize("tokens,d,F", [(300, 256, 640), (1000, 512, 1536)])
@pytest.mark.parametrize("bits", [8, 4])
def test_block_full_and_reused_steps(tokens, d, F, bits, ctx):
    """An operand rounded to e4m3 carries a relative error of 2.6 % (a step of 1/8 to 1/16 of the value,
    uniformly: 1/16/sqrt(3) to half of that), a product of two 3.7 % of its size; the update passes
    three projections in a row at most (v, o or up, down, whose errors add as squares): 6.4 %, and
    8 % is allowed.  The cache then adds its own step: 0.7 % of the change with 8 bits, 9 % with 4."""
    g = torch.Generator(device=DEV).manual_seed(tokens)
    w = lowbit.random_weights(d, F, 3)
    block = lowbit.LowBitBlock(ctx, w, tokens, keep=10 ** 6, bits=bits)
    h0 = torch.randn(tokens, d, generator=g, device=DEV)
    mod = [0.5 * torch.randn(d, generator=g, device=DEV) for _ in range(6)]
    h = torch.empty_like(h0)
    block.full(h0, h, mod)
    ref = plain(w, h0, mod, d // 128)
    change = ref - h0.double()
    assert float((h.double() - ref).norm() / change.norm()) <= 0.08
    other = torch.randn(tokens, d, generator=g, device=DEV)
    out = torch.empty_like(h0)
    block.reuse(other, out)
    kept = (h - h0).double()
    err = float((out.double() - other.double() - kept).norm() / kept.norm())
    assert err <= (0.011 if bits == 8 else 0.13), err
    outs = [torch.empty_like(h0) for _ in range(3)]
    block.run([h0, other, h0], outs, [mod] * 3, [1, 0, 1])
    assert torch.equal(outs[0], h) and torch.equal(outs[1], out) and torch.equal(outs[2], h)
    with pytest.raises(ValueError):
        block.run([h0], outs, [mod], [0])


def test_graph_and_streams_give_the_same_bits(ctx):
    """The block's calls captured on one stream and replayed, and called on another stream."""
    tokens, d, F = 700, 384, 1024
    g = torch.Generator(device=DEV).manual_seed(1)
    block = lowbit.LowBitBlock(ctx, lowbit.random_weights(d, F), tokens, keep=3)
    h0 = torch.randn(tokens, d, generator=g, device=DEV)
    mod = [0.5 * torch.randn(d, generator=g, device=DEV) for _ in range(6)]
    want, got = torch.empty_like(h0), torch.empty_like(h0)
    block.full(h0, want, mod)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx.set_stream(s.cuda_stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            block.full(h0, got, mod)
        got.zero_()
        graph.replay()
        graph.replay()
        s.synchronize()
        assert torch.equal(got, want)
        # right behind work on the same stream: the input is made there
        big = torch.randn(4096, 4096, device=DEV)
        for _ in range(8):
            big = big @ big * 1e-3
        late = h0 + 0.0 * big.sum().nan_to_num(0.0, 0.0, 0.0)
        got.zero_()
        block.full(late, got, mod)
        s.synchronize()
        assert torch.equal(got, want)
    ctx.set_stream(0)


def _raises(status, call, *args, **kw):
    with pytest.raises(bag.BagError) as e:
        call(*args, **kw)
    assert e.value.status == status and len(str(e.value)) > 12, str(e.value)


def test_refusals_of_the_library(ctx):
    EINVAL, EUNSUPPORTED = 1, 7
    u8 = lambda *s: torch.zeros(*s, device=DEV, dtype=torch.uint8)  # noqa: E731
    x = torch.zeros(4, 256, device=DEV)
    # encoded matrices: strides and alignment
    _raises(EINVAL, ctx.quant_fp8, x, u8(4, 264), u8(4, 4))
    _raises(EINVAL, ctx.quant_fp8, x, u8(4 * 272 + 1)[1:].view(4, 272), u8(4, 4))
    _raises(EINVAL, ctx.quant_fp8, x, u8(4, 256), u8(4, 6))
    _raises(EINVAL, ctx.quant_fp8, x, u8(4, 256), u8(4 * 4 + 1)[1:].view(4, 4))
    # LayerNorm: widths and alignment of its rows
    _raises(EUNSUPPORTED, ctx.ln_mod_fp8, torch.zeros(4, 254, device=DEV), None, None, u8(4, 256), u8(4, 4))
    _raises(EUNSUPPORTED, ctx.ln_mod_fp8, torch.zeros(2, 6148, device=DEV), None, None, u8(2, 6160), u8(2, 52))
    _raises(EUNSUPPORTED, ctx.ln_mod_fp8, torch.zeros(1025, device=DEV)[1:].view(4, 256), None, None, u8(4, 256), u8(4, 4))
    # products
    a, s, out = u8(4, 256), u8(4, 4), torch.zeros(4, 4, device=DEV)
    _raises(EINVAL, ctx.gemm_fp8, a, s, a, s, out, 0)
    _raises(EINVAL, ctx.gemm_fp8, a, s, a, s, out, 256, gelu=True, residual=True)
    _raises(EINVAL, ctx.gemm_fp8, a, s, a, s, out, 256, gate=torch.zeros(4, device=DEV))
    lib = ctx.lib
    p = [t.data_ptr() for t in (a, s, out)]
    call = lambda **k: lib.bag_gemm_fp8(ctx.h, p[0], 256, p[1], 4, p[0], 256, p[1], 4, None, k.get("M", 4), k.get("N", 4),  # noqa: E731
                                        256, k.get("act", 0), k.get("kind", 0), None, k.get("out", p[2]), k.get("ldo", 4), None, 0)
    assert call() == 0
    for bad in (dict(M=-1), dict(N=0), dict(act=2), dict(kind=4), dict(kind=-1), dict(out=None), dict(out=p[2] + 1),
                dict(ldo=3), dict(M=2 ** 32), dict(kind=2)):
        assert call(**bad) == EINVAL, bad
    # caches
    c, sc = u8(4, 256), torch.zeros(4, 8, device=DEV, dtype=torch.bfloat16)
    _raises(EINVAL, ctx.cache_write, x, c, sc, 5)
    _raises(EINVAL, ctx.cache_write, torch.zeros(5, 256, device=DEV), c, sc, 8)   # more rows than slots
    _raises(EINVAL, ctx.cache_read, u8(4, 264), sc, x, 8)
    # block attention
    q = torch.zeros(300, 256, device=DEV).half()
    vt, o = torch.zeros(2, 128, 304, device=DEV).half(), torch.zeros(300, 256, device=DEV).bfloat16()
    lists = torch.zeros(2, 3, 3, device=DEV, dtype=torch.int32)
    pool, ps = torch.zeros(2, 3, 128, device=DEV, dtype=torch.int8), torch.zeros(2, 3, device=DEV)
    _raises(EINVAL, ctx.block_select, q, pool, ps, torch.zeros(2, 3, 4, device=DEV, dtype=torch.int32))  # keep > blocks
    big = torch.zeros(1, 8193, 128, device=DEV, dtype=torch.int8)
    _raises(EUNSUPPORTED, ctx.block_select, q, big, torch.zeros(1, 8193, device=DEV), lists)
    _raises(EUNSUPPORTED, ctx.attention_blocks, torch.zeros(300, 260, device=DEV).half()[:, 4:], q, vt, o, lists, 2)
    _raises(EINVAL, ctx.attention_blocks, torch.zeros(300, 384, device=DEV).half(), q, vt,
            torch.zeros(300, 384, device=DEV).bfloat16(), torch.zeros(3, 3, 3, device=DEV, dtype=torch.int32), 3, 2)
    ctx.attention_blocks(q, q, vt, o, lists, 2)  # the context still works
    torch.cuda.synchronize()


def test_lengths_of_zero(ctx):
    """No rows: nothing happens.  No keys: every query gets zeros, and nothing beside them changes."""
    u8 = lambda *s: torch.zeros(*s, device=DEV, dtype=torch.uint8)  # noqa: E731
    ctx.quant_fp8(torch.zeros(0, 256, device=DEV), u8(0, 256), u8(0, 4))
    ctx.ln_mod_fp8(torch.zeros(0, 256, device=DEV), None, None, u8(0, 256), u8(0, 4))
    out = torch.ones(4, 8, device=DEV)
    ctx.gemm_fp8(u8(0, 256), u8(0, 4), u8(8, 256), u8(8, 4), out, 256)
    sc = torch.zeros(4, 8, device=DEV, dtype=torch.bfloat16)
    ctx.cache_write(torch.zeros(0, 256, device=DEV), u8(4, 256), sc, 8)
    ctx.cache_read(u8(4, 256), sc, torch.zeros(0, 256, device=DEV), 8)
    pool, ps = torch.ones(2, 3, 128, device=DEV, dtype=torch.int8), torch.ones(2, 3, device=DEV)
    q = torch.ones(300, 256, device=DEV).half()
    ctx.block_pool(q[:0], pool, ps)
    ctx.block_select(q[:0], pool, ps, torch.zeros(2, 0, 3, device=DEV, dtype=torch.int32))
    vt, o = torch.zeros(2, 128, 8, device=DEV).half(), torch.full((301, 264), 5.0, device=DEV).bfloat16()
    lists = torch.zeros(2, 3, 3, device=DEV, dtype=torch.int32)
    ctx.attention_blocks(q[:0], q, vt.new_zeros(2, 128, 304), o[:0, :256], lists[:, :0], 2)
    torch.cuda.synchronize()
    assert bool((out == 1).all() and (pool == 1).all() and (ps == 1).all() and (o == 5).all())
    ctx.attention_blocks(q, q[:0], vt, o[:300, :256], lists, 2)
    torch.cuda.synchronize()
    assert bool((o[:300, :256] == 0).all() and (o[300] == 5).all() and (o[:, 256:] == 5).all())


def test_refusals_of_the_binding(ctx):
    """Types, devices and shapes that would reach the library as plausible pointers."""
    u8 = lambda *s: torch.zeros(*s, device=DEV, dtype=torch.uint8)  # noqa: E731
    x, c, s = torch.zeros(4, 256, device=DEV), u8(4, 256), u8(4, 4)
    bad = [
        lambda: ctx.quant_fp8(x.double(), c, s),
        lambda: ctx.quant_fp8(x.cpu(), c, s),
        lambda: ctx.quant_fp8(x.T, c, s),
        lambda: ctx.quant_fp8(x, c[:3], s),
        lambda: ctx.quant_fp8(x, c, s[:, :1]),
        lambda: ctx.quant_fp8(x, x, s),
        lambda: ctx.ln_mod_fp8(x, x[0, :5], None, c, s),
        lambda: ctx.gemm_fp8(c, s, c, s, torch.zeros(4, 3, device=DEV), 256),
        lambda: ctx.gemm_fp8(c, s, c, s, torch.zeros(4, 4, device=DEV).half(), 256),
        lambda: ctx.gemm_fp8(c, s, c, s, torch.zeros(4, 4, device=DEV), 257),
        lambda: ctx.gemm_fp8(c, s, c, s, torch.zeros(4, 4, device=DEV).bfloat16(), 256, residual=True),
        lambda: ctx.gemm_fp8(c, s, c, s, torch.zeros(4, 4, device=DEV), 256, bias=torch.zeros(3, device=DEV)),
        lambda: ctx.cache_write(x, c, s, 8),
        lambda: ctx.cache_write(x, c, torch.zeros(4, 1, device=DEV).bfloat16(), 8),
        lambda: ctx.cache_write(x, c, torch.zeros(4, 2, device=DEV).bfloat16(), 8, base=x[:3]),
        lambda: ctx.cache_read(c, torch.zeros(4, 2, device=DEV).bfloat16(), x, 8, slots=torch.zeros(4, device=DEV)),
        lambda: ctx.block_pool(x, torch.zeros(2, 1, 128, device=DEV, dtype=torch.int8), torch.zeros(2, 1, device=DEV)),
        lambda: ctx.block_pool(x.half(), torch.zeros(1, 1, 128, device=DEV, dtype=torch.int8), torch.zeros(1, 1, device=DEV)),
        lambda: ctx.attention_blocks(x.half(), x.bfloat16(), x, x, torch.zeros(2, 1, 1, device=DEV, dtype=torch.int32), 2),
        lambda: ctx.attention_blocks(x.half(), x.half(), torch.zeros(2, 128, 8, device=DEV).half(), x.bfloat16(),
                                     torch.zeros(2, 2, 1, device=DEV, dtype=torch.int32), 2),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("accepted:", i)


def test_sizes_past_the_grid_are_refused(ctx):
    """Rows whose count of work items passes a grid, or 64 bits, launch nothing."""
    lib, h = ctx.lib, ctx.h
    x, c, s = torch.ones(8, 2048, device=DEV), torch.zeros(8, 2048, device=DEV, dtype=torch.uint8), \
        torch.zeros(8, 64, device=DEV, dtype=torch.bfloat16)
    slots = torch.zeros(8, device=DEV, dtype=torch.int32)
    p, pc, ps, pi = (t.data_ptr() for t in (x, c, s, slots))
    for rows in (2 ** 35, 2 ** 62 + 2, 2 ** 63 - 1):
        assert lib.bag_quant_fp8(h, p, 0, 2048, rows, 2048, pc, 2048, ps, 128) != 0
        assert lib.bag_ln_mod_fp8(h, p, 2048, None, None, rows, 2048, pc, 2048, ps, 128) != 0
        assert lib.bag_cache_write(h, p, 2048, None, 0, pi, rows, 2048, 8, pc, 2048, ps, 64, 8) != 0
        assert lib.bag_cache_read(h, pc, 2048, ps, 64, 8, pi, rows, 2048, 8, None, 0, p, 2048) != 0
    for cols in (2 ** 32, 2 ** 63 - 1):
        assert lib.bag_quant_fp8(h, p, 0, cols, 1, cols, pc, cols & ~15, ps, 2 ** 60) != 0
        assert lib.bag_cache_write(h, p, cols, None, 0, pi, 1, cols, 8, pc, cols & ~15, ps, 2 ** 60, 8) != 0
    torch.cuda.synchronize()
    assert bool((c == 0).all() and (s == 0).all() and (x == 1).all())
