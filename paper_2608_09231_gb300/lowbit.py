"""A transformer block on the low-precision operators, under a compute-or-reuse mask.

`LowBitBlock` is one block of adaLN-modulated self-attention and MLP on a residual stream (the
shape of a Wan-type image-stream block, without its cross-attention and rotary embedding):

  x  = LN-mod(h)                        encoded to 8 bits (ln_mod_fp8)
  q, k = x Wq^T, x Wk^T                 8-bit products, bf16 out; V^T = Wv x^T, the same product
                                        with its operands exchanged, so that V arrives transposed
  o  = attention of q over the `keep` key blocks of each query block's list (block_pool,
       block_select, attention_blocks)
  h += gate_a * (o Wo^T + bo)           o encoded (quant_fp8), update in the product's epilogue
  x  = LN-mod(h), u = GELU(x Wu^T + bu) encoded in the product's epilogue
  h += gate_m * (u Wd^T + bd)

q, k and V are bf16, the 16-bit type that the products store, and so are the softmax's weights: about
the output's own rounding, and a tenth of what 8-bit operands of the next projection lose.

A full step runs it and keeps its change h_out - h_in in a cache of 8 or 4 bits; a reused step
adds the kept change to its own h_in (the residual reuse of Algorithm 2, here of one block).

All arithmetic runs in the CUDA library, on the context's stream; torch supplies the device memory
and copies h_in, on its current stream.  Where the two differ each waits for the other, so that a
step follows what the caller did on the current stream and comes before what the caller does next.
As a command it times both kinds of step:

  python -m paper_2608_09231_gb300.lowbit [--tokens 32760] [--hidden 5120] [--mlp 13824] [--keep 64]
"""

import argparse
import contextlib

import torch

from . import bag, configs

DEV = "cuda"


def _up(n, m):
    return (n + m - 1) // m * m


@contextlib.contextmanager
def ordered(ctx):
    """Calls of ctx after the work on torch's current stream, and before what follows there."""
    here = torch.cuda.current_stream()
    if here.cuda_stream == ctx.stream:
        yield
        return
    there = torch.cuda.ExternalStream(ctx.stream) if ctx.stream else torch.cuda.default_stream()
    there.wait_stream(here)
    try:
        yield
    finally:
        here.wait_stream(there)


def _overlap(a, b):
    """Whether two matrices with dense rows share elements."""
    def end(t):
        return t.data_ptr() + t.element_size() * (1 + sum((n - 1) * s for n, s in zip(t.shape, t.stride())))

    if a.numel() == 0 or b.numel() == 0 or a.data_ptr() >= end(b) or b.data_ptr() >= end(a):
        return False
    ld, width = a.stride(0) * a.element_size(), a.shape[1] * a.element_size()
    apart = (b.data_ptr() - a.data_ptr()) % ld  # columns of one wider matrix, side by side
    return not (a.stride() == b.stride() and width <= apart <= ld - b.shape[1] * b.element_size())


class Encoded:
    """A matrix [rows, cols] as e4m3 codes with a scale for each 128 columns of a row."""

    def __init__(self, rows, cols):
        self.rows, self.cols = rows, cols
        self.codes = torch.zeros(rows, _up(cols, 16), device=DEV, dtype=torch.uint8)
        self.scales = torch.zeros(rows, _up(-(-cols // bag.SCALE_BLOCK), 16), device=DEV, dtype=torch.uint8)

    @classmethod
    def of(cls, ctx, x):
        e = cls(*x.shape)
        with ordered(ctx):
            ctx.quant_fp8(x, e.codes, e.scales)
        return e


class Cache:
    """A quantised cache of `rows` rows of `cols` elements."""

    def __init__(self, rows, cols, bits):
        self.bits = bits
        self.codes = torch.zeros(rows, _up(-(-cols * bits // 8), 16), device=DEV, dtype=torch.uint8)
        self.scales = torch.zeros(rows, -(-cols // bag.CACHE_GROUP[bits]), device=DEV, dtype=torch.bfloat16)

    def nbytes(self):
        return self.codes.numel() + 2 * self.scales.numel()


class LowBitBlock:
    """weights: dict of device tensors wq, wk, wv, wo [d, d], wu [F, d], wd [d, F] (fp32 or bf16) and
    biases bq, bk, bo, bd [d], bu [F] (fp32); ctx: the context whose calls are used."""

    def __init__(self, ctx, weights, tokens, keep, bits=8):
        self.ctx, self.tokens = ctx, tokens
        F, d = weights["wu"].shape
        if d % 128:
            raise ValueError(f"heads are 128 wide: hidden {d} is not a multiple")
        self.d, self.F, self.heads = d, F, d // 128
        self.w = {n: Encoded.of(ctx, weights[n]) for n in ("wq", "wk", "wv", "wo", "wu", "wd")}
        self.b = {n: weights[n] for n in ("bq", "bk", "bo", "bu", "bd")}
        blocks = -(-tokens // bag.ATTN_BLOCK)
        self.x, self.u = Encoded(tokens, d), Encoded(tokens, F)
        bf16 = dict(device=DEV, dtype=torch.bfloat16)
        self.q, self.k, self.o = (torch.empty(tokens, d, **bf16) for _ in range(3))
        self.vt = torch.zeros(self.heads, 128, _up(tokens, 8), **bf16)
        self.pool = torch.zeros(self.heads, blocks, 128, device=DEV, dtype=torch.int8)
        self.pool_s = torch.zeros(self.heads, blocks, device=DEV)
        self.lists = torch.zeros(self.heads, blocks, min(keep, blocks), device=DEV, dtype=torch.int32)
        self.cache = Cache(tokens, d, bits)

    def _project(self, x, w, out, **more):
        self.ctx.gemm_fp8(x.codes, x.scales, w.codes, w.scales, out, w.cols, **more)

    def full(self, h_in, h, mod):
        """The block on h_in into h, its change kept.  mod: (shift_a, scale_a, gate_a, shift_m, scale_m,
        gate_m), fp32 [d] each.  h_in is needed to the end, for the change: h may not be it."""
        if _overlap(h_in, h):
            raise ValueError("h_in and h share memory: the block's change would be lost")
        h.copy_(h_in)
        with ordered(self.ctx):
            self._full(h_in, h, mod)

    def _full(self, h_in, h, mod):
        c, x, w, b = self.ctx, self.x, self.w, self.b
        c.ln_mod_fp8(h, mod[0], mod[1], x.codes, x.scales)
        self._project(x, w["wq"], self.q, bias=b["bq"])
        self._project(x, w["wk"], self.k, bias=b["bk"])
        self._project(w["wv"], x, self.vt.view(self.d, -1))
        c.block_pool(self.k, self.pool, self.pool_s)
        c.block_select(self.q, self.pool, self.pool_s, self.lists)
        c.attention_blocks(self.q, self.k, self.vt, self.o, self.lists, self.heads)
        c.quant_fp8(self.o, x.codes, x.scales)
        self._project(x, w["wo"], h, bias=b["bo"], gate=mod[2], residual=True)
        c.ln_mod_fp8(h, mod[3], mod[4], x.codes, x.scales)
        self._project(x, w["wu"], self.u.codes, bias=b["bu"], gelu=True, out_scales=self.u.scales, N=self.F)
        self._project(self.u, w["wd"], h, bias=b["bd"], gate=mod[5], residual=True)
        c.cache_write(h, self.cache.codes, self.cache.scales, self.cache.bits, base=h_in)

    def reuse(self, h_in, h):
        """h = h_in + the change kept by the last full step."""
        with ordered(self.ctx):
            self.ctx.cache_read(self.cache.codes, self.cache.scales, h, self.cache.bits, base=h_in)

    def run(self, streams, outs, mods, mask):
        """The steps of a sample: step t computes where mask[t] is 1 (mask[0] must be), else reuses.  Waits
        for them and raises if a kernel gave up (not while a graph is captured)."""
        if not mask[0]:
            raise ValueError("the first step has nothing to reuse")
        for t, full in enumerate(mask):
            if full:
                self.full(streams[t], outs[t], mods[t])
            else:
                self.reuse(streams[t], outs[t])
        if not torch.cuda.is_current_stream_capturing():
            with ordered(self.ctx):
                self.ctx.operators_status()


def random_weights(d, F, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: 0.02 * torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    w = {n: r(d, d).bfloat16() for n in ("wq", "wk", "wv", "wo")}
    w.update(wu=r(F, d).bfloat16(), wd=r(d, F).bfloat16(), bu=r(F), **{n: r(d) for n in ("bq", "bk", "bo", "bd")})
    return w


def main():
    wan = configs.get_config("wan")
    p = argparse.ArgumentParser(description="times a full and a reused step of one low-precision block")
    p.add_argument("--tokens", type=int, default=wan["n_img"])
    p.add_argument("--hidden", type=int, default=wan["hidden"])
    p.add_argument("--mlp", type=int, default=wan["mlp"])
    p.add_argument("--keep", type=int, default=64)
    p.add_argument("--bits", type=int, default=8, choices=(8, 4))
    a = p.parse_args()
    ctx = bag.create("tiny")
    ctx.set_stream(torch.cuda.current_stream().cuda_stream)
    block = LowBitBlock(ctx, random_weights(a.hidden, a.mlp), a.tokens, a.keep, a.bits)
    h_in = torch.randn(a.tokens, a.hidden, device=DEV)
    h = torch.empty_like(h_in)
    mod = [0.3 * torch.randn(a.hidden, device=DEV) for _ in range(6)]

    def ms(call, n=10):
        for _ in range(3):
            call()
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record()
        for _ in range(n):
            call()
        e1.record()
        torch.cuda.synchronize()
        return e0.elapsed_time(e1) / n

    full = ms(lambda: block.full(h_in, h, mod))
    reuse = ms(lambda: block.reuse(h_in, h))
    print(f"{a.tokens} tokens, hidden {a.hidden}, MLP {a.mlp}, {block.lists.shape[2]} of {block.lists.shape[1]} key blocks: "
          f"full step {full:.3f} ms, reused {reuse:.3f} ms, cache {block.cache.nbytes() / 1e6:.0f} MB "
          f"({a.bits} bits; fp32 {4e-6 * h.numel():.0f} MB)")
    ctx.close()


if __name__ == "__main__":
    main()
