"""A text's side of a sampler: causal attention over texts that grow, with their keys and values in a cache.

The text tokens that condition a DiT come from a decoder-only encoder, whose attention this is:

  x        = LayerNorm(h)                      encoded to 8 bits (ln_mod_fp8)
  q, k, v  = x W^T                             one 8-bit product, bf16 out
  q, k     rotated by their positions; k and v into the texts' rows of a cache (rope)
  o        = attention of q over each text's own rows (attention_packed), and over a prefix that all of
             them start with (attention_prefix)
  h       += o Wo^T                            o encoded (quant_fp8), update in the product's epilogue

The projections have no biases.

`TextCache` says where texts lie and what a step adds to them: whole prompts, more tokens of each, or
one each.  `TextAttention` is the layer.  `rope_frequencies` makes the table of a rotary embedding, also for
contexts longer than it was trained for.

All arithmetic runs in the CUDA library, on the context's stream; torch supplies the device memory.  Where
torch's current stream is another one, each waits for the other (lowbit.ordered).  As a command it times
a layer on a batch of prompts, then a token of each:

  python -m paper_2608_09231_gb300.prompt [--texts 32] [--tokens 256] [--prefix 1024] [--heads 32]
"""

import argparse
import math

import numpy as np
import torch

from . import bag
from .lowbit import DEV, Encoded, ordered


def rope_frequencies(pairs, theta=10000.0, factor=1.0, scaling="parts", original=8192, slow=1.0, fast=32.0):
    """(radians a position of each pair, factor of the results) of a rotary embedding: theta^(-i / pairs), for
    contexts `factor` times as long as the original one
      linear  all frequencies divided by the factor (positions interpolated)
      base    theta raised so that the lowest frequency is divided by it and the highest stays
      parts   those that turn fewer than `slow` times in the original length are divided by it, those that turn
              more than `fast` times stay, linearly in between; results times 0.1 ln(factor) + 1 (YaRN, Peng
              et al. 2023)"""
    if pairs < 1 or not theta > 1.0 or not factor >= 1.0:
        raise ValueError("a rotary embedding needs pairs, a base above 1 and a factor of at least 1")
    i = np.arange(pairs, dtype=np.float64)
    if factor == 1.0:
        return theta ** (-i / pairs), 1.0
    if scaling == "linear":
        return theta ** (-i / pairs) / factor, 1.0
    if scaling == "base":
        if pairs > 1:
            theta = theta * factor ** (pairs / (pairs - 1.0))
        return theta ** (-i / pairs), 1.0
    if scaling != "parts" or not fast > slow:
        raise ValueError(f"scaling {scaling!r} is none of linear, base and parts, or its bounds are not in order")
    f = theta ** (-i / pairs)
    stay = np.clip((original * f / (2.0 * math.pi) - slow) / (fast - slow), 0.0, 1.0)
    return f * (stay + (1.0 - stay) / factor), 0.1 * math.log(factor) + 1.0


class TextCache:
    """Rows of the texts in a cache: text i has rows [i * room, i * room + its length).  Lengths grow when a step is made
    (extend), so that every step runs through every layer, or is taken back."""

    def __init__(self, texts, room):
        self.texts, self.room, self.lens = texts, room, [0] * texts
        self.made = 0   # steps so far
        self.gone = []  # ranges of those that were taken back

    def extend(self, new):
        """What a step that adds new[i] tokens to text i hands to the operators (rows in the texts' order).  The host makes
        it, and waits until it is on the device."""
        if len(new) != self.texts or any(n < 0 or n + m > self.room for n, m in zip(new, self.lens)):
            raise ValueError(f"{self.texts} texts of at most {self.room} tokens, of {self.lens}, cannot take {new}")
        first = np.concatenate([[0], np.cumsum(new)])
        pos = np.concatenate([np.arange(m, m + n) for n, m in zip(new, self.lens)] or [[]])
        place = np.repeat(np.arange(self.texts) * self.room, new)
        before, self.lens = list(self.lens), [n + m for n, m in zip(new, self.lens)]
        self.made += 1
        ints = np.concatenate([first, np.arange(self.texts) * self.room, self.lens, pos, place + pos])
        dev = torch.from_numpy(ints.astype(np.int32)).to(DEV)  # one copy for all
        n, s = int(first[-1]), self.texts
        q_start, k_start, k_len, pos, slots = dev.split([s + 1, s, s, n, n])
        return dict(q_start=q_start, k_start=k_start, k_len=k_len, pos=pos, slots=slots, rows=n,
                    max_q=max(new, default=0), max_k=max(self.lens, default=0), cache=self, number=self.made,
                    before=before, after=list(self.lens), ran=set())

    def take_back(self, step):
        """Lengths as before `step`, which does not run, nor do those made after it.  A layer does this itself with a
        step that it refuses."""
        if not any(first <= step["number"] < end for first, end in self.gone):
            self.lens = list(step["before"])
            self.gone = [r for r in self.gone if r[0] < step["number"]] + [(step["number"], self.made + 1)]

    def stands(self, step):
        """Whether `step` may run: one that was taken back does so if no other has been made since, and counts again."""
        n = step["number"]
        if not any(first <= n < end for first, end in self.gone):
            return True
        first, end = self.gone[-1]
        if not first <= n < end or end != self.made + 1 or self.lens != step["before"]:
            return False
        self.gone[-1] = (n + 1, end)
        self.lens = list(step["after"])
        return True


class TextAttention:
    """weights: wqkv [(heads + 2 kv_heads) * dh, d] and wo [d, heads * dh] (fp32 or bf16, on the device); cache: the
    TextCache that its steps come from; rows: the most tokens of a step; prefix: those of a shared
    prefix.  dh 64 or 128."""

    def __init__(self, ctx, weights, heads, kv_heads, cache, rows, prefix=0, dh=128, theta=10000.0, layout="half", **scaling):
        self.ctx, self.heads, self.kv_heads, self.dh, self.layout = ctx, heads, kv_heads, dh, layout
        self.texts, self.room = cache.texts, cache.room
        wq, d = weights["wqkv"].shape
        if wq != (heads + 2 * kv_heads) * dh or weights["wo"].shape != (d, heads * dh):
            raise ValueError(f"weights of {tuple(weights['wqkv'].shape)} and {tuple(weights['wo'].shape)} do not fit "
                             f"{heads} and {kv_heads} heads of {dh}")
        self.wqkv, self.wo = (Encoded.of(ctx, weights[n]) for n in ("wqkv", "wo"))
        self.freqs, self.scale = rope_frequencies(dh // 2, theta, **scaling)
        bf16 = dict(device=DEV, dtype=torch.bfloat16)
        self.x, self.e = Encoded(rows, d), Encoded(rows, heads * dh)
        self.qkv, self.q = torch.empty(rows, wq, **bf16), torch.empty(rows, heads * dh, **bf16)
        self.o = torch.empty(rows, heads * dh, **bf16)
        self.k, self.v = (torch.empty(cache.texts * cache.room, kv_heads * dh, **bf16) for _ in range(2))
        self.pk, self.pv = (torch.empty(prefix, kv_heads * dh, **bf16) for _ in range(2))
        self.seen = 0  # tokens of the prefix so far
        # for steps of any number of tokens, and for the prefix
        self.work = torch.empty(max(ctx.attention_work(rows, heads, dh, kv_heads, cache.texts, min(rows, cache.room), cache.room, prefix),
                                    ctx.attention_work(prefix, heads, dh, kv_heads, 1, prefix, prefix)),
                                device=DEV, dtype=torch.uint8)

    def _project(self, h):
        n, c = h.shape[0], self.ctx
        c.ln_mod_fp8(h, None, None, self.x.codes[:n], self.x.scales[:n])
        qkv = self.qkv[:n]
        c.gemm_fp8(self.x.codes[:n], self.x.scales[:n], self.wqkv.codes, self.wqkv.scales, qkv, self.wqkv.cols)
        return qkv.split([self.heads * self.dh, self.kv_heads * self.dh, self.kv_heads * self.dh], 1)

    def _out(self, h):
        n, c = h.shape[0], self.ctx
        c.quant_fp8(self.o[:n], self.e.codes[:n], self.e.scales[:n])
        c.gemm_fp8(self.e.codes[:n], self.e.scales[:n], self.wo.codes, self.wo.scales, h, self.wo.cols, residual=True)

    def prefix(self, h):
        """The tokens h [n, d] (fp32, updated in place) of the prefix that all texts start with, before any of theirs."""
        n = h.shape[0]
        if h.shape != (self.pk.shape[0], self.wqkv.cols) or n > self.q.shape[0]:
            raise ValueError(f"a prefix of {tuple(h.shape)}, and a layer for one of {self.pk.shape[0]} rows of {self.wqkv.cols}, of "
                             f"at most {self.q.shape[0]}")
        if n == 0:
            return
        start = torch.tensor([0, n], device=DEV, dtype=torch.int32)
        with ordered(self.ctx):
            q, k, v = self._project(h)
            self.ctx.rope(q, self.q[:n], self.freqs, self.dh, k=k, k_out=self.pk, v=v, v_out=self.pv, layout=self.layout,
                          scale=self.scale)
            self.ctx.attention_packed(self.q[:n], self.pk, self.pv, self.o[:n], start, self.heads, self.kv_heads,
                                      work=self.work)
            self._out(h)
        self.seen = n

    def step(self, h, step):
        """The tokens h [rows, d] (fp32, updated in place) that TextCache.extend made `step` for.  A step that is refused is
        taken back: the texts are as long as before it, and it may be given again unless another is made first."""
        cache = step["cache"]
        try:
            if (cache.texts, cache.room) != (self.texts, self.room):
                raise ValueError(f"a step of {cache.texts} texts of {cache.room} tokens, and a layer for {self.texts} of "
                                 f"{self.room}")
            if not cache.stands(step):
                raise ValueError("the step was taken back, and others have been made since")
            self._run(h, step)
            step["ran"].add(id(self))
        except Exception:
            if id(self) not in step["ran"]:
                cache.take_back(step)
            raise

    def _run(self, h, step):
        n, c = step["rows"], self.ctx
        if h.shape != (n, self.wqkv.cols) or n > self.q.shape[0]:
            raise ValueError(f"{tuple(h.shape)} for a step of {n} rows of {self.wqkv.cols}, of at most {self.q.shape[0]}")
        if self.seen != self.pk.shape[0]:
            raise ValueError("the prefix comes first")
        if n == 0:
            return
        pos = step["pos"] + self.seen if self.seen else step["pos"]  # torch's work, before the context's waits for it
        with ordered(c):
            q, k, v = self._project(h)
            c.rope(q, self.q[:n], self.freqs, self.dh, pos=pos, k=k, k_out=self.k, v=v, v_out=self.v, slots=step["slots"],
                   layout=self.layout, scale=self.scale)
            args = [self.q[:n], self.k, self.v, self.o[:n], step["q_start"]]
            if self.seen:
                args += [self.pk, self.pv]
            (c.attention_prefix if self.seen else c.attention_packed)(
                *args, self.heads, self.kv_heads, k_start=step["k_start"], k_len=step["k_len"], max_q=step["max_q"],
                max_k=step["max_k"], work=self.work)
            self._out(h)


def random_weights(d, heads, kv_heads, dh=128, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return {n: (0.02 * torch.randn(*s, generator=g, device=DEV)).bfloat16()
            for n, s in (("wqkv", ((heads + 2 * kv_heads) * dh, d)), ("wo", (d, heads * dh)))}


def main():
    p = argparse.ArgumentParser(description="times one attention layer on a batch of prompts, and on a token of each")
    p.add_argument("--texts", type=int, default=32)
    p.add_argument("--tokens", type=int, default=256)
    p.add_argument("--prefix", type=int, default=1024)
    p.add_argument("--heads", type=int, default=32)
    p.add_argument("--kv-heads", type=int, default=8)
    a = p.parse_args()
    d, rows = a.heads * 128, max(a.texts * a.tokens, a.prefix)
    ctx = bag.create("tiny")
    ctx.set_stream(torch.cuda.current_stream().cuda_stream)
    cache = TextCache(a.texts, a.tokens + 64)
    layer = TextAttention(ctx, random_weights(d, a.heads, a.kv_heads), a.heads, a.kv_heads, cache, rows, a.prefix)
    h = torch.randn(rows, d, device=DEV)

    def ms(call, n=20):
        for _ in range(3):
            call()
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record()
        for _ in range(n):
            call()
        e1.record()
        torch.cuda.synchronize()
        return e0.elapsed_time(e1) / n

    if a.prefix:
        print(f"prefix of {a.prefix} tokens {ms(lambda: layer.prefix(h[:a.prefix])):.3f} ms")
    prompts = cache.extend([a.tokens] * a.texts)
    print(f"{a.texts} prompts of {a.tokens} tokens {ms(lambda: layer.step(h[:prompts['rows']], prompts)):.3f} ms")
    token = cache.extend([1] * a.texts)
    print(f"a token of each {ms(lambda: layer.step(h[:a.texts], token)):.3f} ms")
    ctx.operators_status()
    ctx.close()


if __name__ == "__main__":
    main()
