"""Attention of packed sequences on the GPU against a plain form in 64 bits (tests/prompt_ref.py has the
bounds)."""

import math
import random

import pytest
import torch

import prompt_ref as R
from paper_2608_09231_gb300 import bag

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ctx(lib):
    c = bag.create("tiny", T=2, B=1)
    yield c
    c.operators_status()
    c.close()


def i32(x):
    return torch.tensor(x, device=DEV, dtype=torch.int32)


def normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


class Batch:
    """Sequences of (queries, keys) whose keys lie apart in a cache of NaN; rows of q before the first and
    behind the last sequence; all tensors columns of wider ones."""

    def __init__(self, lens, heads, kv_heads, dh, dtype, key=0, prefix=None, pad=8, before=0, behind=3, loud=1.0):
        g = torch.Generator(device=DEV).manual_seed(key)
        dt = TYPES[dtype]
        self.heads, self.kv_heads, self.dh, self.dt = heads, kv_heads, dh, dt
        self.starts = [before]
        for lq, _ in lens:
            self.starts.append(self.starts[-1] + lq)
        nq = self.starts[-1] + behind
        order = torch.randperm(len(lens), generator=g, device=DEV).tolist()
        k0, at = [0] * len(lens), 3
        for i in order:
            k0[i] = at
            at += lens[i][1] + 5

        def wide(n, cols):
            x = torch.full((n, cols + 2 * pad), math.nan, device=DEV, dtype=dt)
            return x[:, pad:pad + cols] if pad else x

        self.q = wide(nq, heads * dh)
        self.q.copy_((loud * normal(g, nq, heads * dh)).to(dt))
        self.k, self.v = wide(at, kv_heads * dh), wide(at, kv_heads * dh)
        self.seqs = [(self.starts[i], lq, k0[i], lk) for i, (lq, lk) in enumerate(lens)]
        for _, _, k, lk in self.seqs:
            self.k[k:k + lk] = normal(g, lk, kv_heads * dh).to(dt)
            self.v[k:k + lk] = (normal(g, lk, kv_heads * dh) + 0.5).to(dt)
        self.pk = self.pv = None
        if prefix is not None:
            self.pk, self.pv = wide(prefix, kv_heads * dh), wide(prefix, kv_heads * dh)
            self.pk.copy_(normal(g, prefix, kv_heads * dh).to(dt))
            self.pv.copy_((normal(g, prefix, kv_heads * dh) + 0.5).to(dt))
        self.wide_o = torch.full((nq, heads * dh + 2 * pad), 9.0, device=DEV, dtype=dt)
        self.o = self.wide_o[:, pad:pad + heads * dh]
        self.lse = torch.full((nq, heads), 9.0, device=DEV)
        self.max_q, self.max_k = max(x for x, _ in lens), max(x for _, x in lens)
        self.dev = dict(k_start=i32(k0), k_len=i32([x for _, x in lens]))

    def work(self, ctx, share=1.0):
        n = ctx.attention_work(self.q.shape[0], self.heads, self.dh, self.kv_heads, len(self.seqs), self.max_q,
                               self.max_k, 0 if self.pk is None else self.pk.shape[0])
        n = int(n * share) // 16 * 16
        return torch.full((n // 4,), math.nan, device=DEV) if n else None

    def run(self, ctx, work="all", hints=True, **more):
        args = dict(self.dev, lse=self.lse, work=self.work(ctx) if isinstance(work, str) else work)
        if hints:
            args.update(max_q=self.max_q, max_k=self.max_k)
        args.update(more)
        tensors = [self.q, self.k, self.v, self.o, i32(self.starts)]
        if self.pk is not None:
            ctx.attention_prefix(*tensors, self.pk, self.pv, self.heads, self.kv_heads, **args)
        else:
            ctx.attention_packed(*tensors, self.heads, self.kv_heads, **args)
        return self

    def check(self, causal=True, scale=None):
        n, dh = self.q.shape[0], self.dh
        o, tol, lse, ltol = R.attention(self.q, self.k, self.v, self.heads, self.kv_heads, self.seqs, causal, scale,
                                        self.pk, self.pv)
        got = self.o.double().reshape(n, self.heads, dh)
        inside = torch.zeros(n, dtype=torch.bool, device=DEV)
        inside[self.starts[0]:self.starts[-1]] = True
        err = (got - o).abs()[inside]
        assert bool((err <= tol[inside]).all()), float((err - tol[inside]).max())
        le = (self.lse.double() - lse)[inside]
        none = torch.isneginf(lse[inside])
        assert torch.equal(none, torch.isneginf(self.lse[inside]))
        assert bool((le.abs() <= ltol[inside])[~none].all())
        rest = torch.full_like(self.wide_o, 9.0)
        pad = (self.wide_o.shape[1] - self.heads * dh) // 2
        rest[inside, pad:pad + self.heads * dh] = self.o[inside]
        assert torch.equal(rest, self.wide_o) and bool((self.lse[~inside] == 9).all())


LENS = {
    "one": [(1, 1)],
    "token": [(1, 1000)],
    "tokens": [(1, 1), (1, 40), (1, 0), (1, 129), (1, 700), (1, 16)],
    "prompt": [(77, 77)],
    "tiles": [(128, 128), (256, 256), (129, 129), (1, 1), (127, 127)],
    "mixed": [(5, 5), (0, 0), (1, 300), (130, 130), (0, 17), (64, 300), (3, 3)],
    "extend": [(40, 700), (2, 513), (17, 128)],
    "short": [(40, 10), (3, 1), (9, 0)],       # the first queries see nothing
    "long": [(300, 1500), (1, 2100)],
    "ends": [(33, n) for n in (33, 47, 48, 49, 63, 64, 65, 112, 127, 144)],
}


@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (7, 1), (12, 4), (16, 2)])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
def test_packed(lens, heads, kv_heads, dh, dtype, causal, ctx):
    b = Batch(LENS[lens], heads, kv_heads, dh, dtype, key=len(lens) + heads)
    b.run(ctx, causal=causal).check(causal)


@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("prefix", [1, 127, 128, 300, 1111])
@pytest.mark.parametrize("heads,kv_heads,dh,dtype", [(7, 1, 128, "bf16"), (12, 4, 64, "f16"), (8, 8, 128, "f16"), (40, 2, 64, "bf16")])
def test_prefix(lens, prefix, heads, kv_heads, dh, dtype, ctx):
    b = Batch(LENS[lens], heads, kv_heads, dh, dtype, key=prefix, prefix=prefix)
    b.run(ctx).check()


def many(n, seed, lq, lk):
    """n sequences of random lengths up to lq new and lk more keys, some of them empty."""
    g = random.Random(seed)
    out = []
    for _ in range(n):
        m = 0 if g.random() < 0.1 else g.randint(1, lq)
        out.append((m, max(0, m + g.randint(-2, lk))))
    return out


@pytest.mark.parametrize("n", [31, 32, 33, 127, 128, 129, 300, 700])
@pytest.mark.parametrize("lq,lk", [(1, 60), (1, 700), (3, 40), (60, 100)])
@pytest.mark.parametrize("prefix", [None, 200])
def test_many_sequences(n, lq, lk, prefix, ctx):
    """More sequences than a warp finds at once, or a CTA adds up at once; queries that start behind others' rows."""
    if n * lq > 12000:
        n = 12000 // lq
    b = Batch(many(n, n + lq, lq, lk), 4, 2, 64, "f16", key=n, prefix=prefix, before=2)
    b.run(ctx).check()


@pytest.mark.parametrize("heads,kv_heads", [(28, 1), (40, 1), (48, 1), (13, 1), (130, 1), (131, 1), (256, 2), (10, 2), (33, 3)])
@pytest.mark.parametrize("lens", ["prompt", "mixed", "tokens", "extend"])
def test_groups_of_heads(heads, kv_heads, lens, ctx):
    """Groups that do not divide a tile's rows, or do not fit them."""
    b = Batch(LENS[lens], heads, kv_heads, 64, "bf16", key=heads)
    b.run(ctx).check()


@pytest.mark.parametrize("lens", ["mixed", "tokens"])
def test_strides_of_their_own(lens, ctx):
    """q, k, v and o as columns of wider tensors of four different widths, and a prefix likewise."""
    b = Batch(LENS[lens], 6, 2, 128, "f16", prefix=140)

    def inside(x, width, at):
        y = torch.full((x.shape[0], width), math.nan, device=DEV, dtype=x.dtype)
        y[:, at:at + x.shape[1]] = x
        return y[:, at:at + x.shape[1]]

    b.q, b.k, b.v = inside(b.q, 1000, 64), inside(b.k, 264, 8), inside(b.v, 600, 320)
    b.pk, b.pv = inside(b.pk, 272, 0), inside(b.pv, 1024, 512)
    b.run(ctx).check()


@pytest.mark.parametrize("dh", [64, 128])
def test_prefix_alone(dh, ctx):
    """No own keys at all, and no rows for them; and no mask."""
    for lens in ([(1, 0)], [(3, 0), (200, 0)]):
        b = Batch(lens, 4, 2, dh, "bf16", prefix=500)
        b.k, b.v = b.k[:0], b.v[:0]
        b.run(ctx).check()
        b = Batch([(70, 30), (5, 5)], 4, 2, dh, "bf16", prefix=77)
        b.run(ctx, causal=False).check(False)


@pytest.mark.parametrize("share", [0.0, 0.2, 0.55, 1.0])
@pytest.mark.parametrize("lens", [[(1, 9000)], [(1, 3000), (1, 10), (1, 2999), (2, 40)], [(40, 5000)], [(300, 4000), (5, 4000)]])
@pytest.mark.parametrize("prefix", [None, 900])
def test_less_workspace(share, lens, prefix, ctx):
    for dtype in ("f16", "bf16"):
        b = Batch(lens, 8, 2, 128, dtype, prefix=prefix)
        work = b.work(ctx, share)
        b.run(ctx, work=work).check()


@pytest.mark.parametrize("lens", [[(1, 9000)], [(1, 3000), (1, 10), (1, 2999), (2, 40)], [(40, 5000), (1, 1)]])
@pytest.mark.parametrize("max_q,max_k", [(1, 1), (1, 500), (100000, 100000), (0, 0), (5, 2999)])
def test_wrong_estimates(lens, max_q, max_k, ctx):
    for prefix in (None, 600):
        b = Batch(lens, 8, 2, 64, "f16", prefix=prefix)
        n = ctx.attention_work(b.q.shape[0], 8, 64, 2, len(lens), max_q, max_k, prefix or 0)
        work = torch.full((max(n, 16) // 4,), math.nan, device=DEV)
        b.run(ctx, work=work, max_q=max_q, max_k=max_k).check()


@pytest.mark.parametrize("before", [0, 4])
def test_keys_of_the_queries_rows(before, ctx):
    """Without starts and lengths a sequence's keys are the rows of its queries."""
    lens = [(5, 5), (130, 130), (1, 1), (64, 64)]
    b = Batch(lens, 12, 4, 128, "bf16", before=before)
    n = b.q.shape[0]
    g = torch.Generator(device=DEV).manual_seed(9)
    b.k, b.v = (normal(g, n, 512).bfloat16() for _ in range(2))
    b.seqs = [(q0, lq, q0, lk) for q0, lq, _, lk in b.seqs]
    b.run(ctx, k_start=None, k_len=None).check()


@pytest.mark.parametrize("heads,kv_heads", [(4, 2), (32, 1)])
@pytest.mark.parametrize("scale", [0.02, 0.3])
def test_scale_and_loud_scores(heads, kv_heads, scale, ctx):
    """Scores far apart: running maxima that move often, weights that vanish."""
    for dtype in ("f16", "bf16"):
        b = Batch([(60, 700), (1, 300), (300, 300)], heads, kv_heads, 128, dtype, loud=6.0)
        b.run(ctx, scale=scale).check(scale=scale)


@pytest.mark.parametrize("lens", [[(1, 600), (1, 70)], [(64, 600), (100, 100)]])
def test_scores_that_grow_and_fall(lens, ctx):
    """Keys in order of their score, both ways: the maximum moves at every step, or never after the first."""
    for sign in (1.0, -1.0):
        b = Batch(lens, 4, 4, 64, "f16")
        for _, _, k0, lk in b.seqs:
            b.k[k0:k0 + lk] = (torch.linspace(-1, 1, lk, device=DEV).unsqueeze(1) * sign).half()
        b.q.copy_(b.q.abs() * 4)
        b.run(ctx).check()


def test_equal_scores(ctx):
    """All scores zero: the mean of the values seen."""
    b = Batch([(50, 50), (1, 333)], 2, 1, 128, "bf16")
    b.q.zero_()
    b.run(ctx).check()


def test_values_that_are_not_finite(ctx):
    """A NaN score or an infinite one makes its own rows NaN and no others'; rows that do not see it stay, also where the
    same call holds it in another sequence or head."""
    b = Batch([(40, 40), (30, 90)], 4, 2, 128, "bf16")
    b.q[7, 128:256] = math.nan      # query 7, head 1
    b.run(ctx)
    bad = ~torch.isfinite(b.o.reshape(-1, 4, 128)[:70]).all(2)
    want = torch.zeros_like(bad)
    want[7, 1] = True
    assert torch.equal(bad, want)
    b = Batch([(40, 40), (30, 90)], 4, 2, 128, "bf16")
    b.k[b.seqs[0][2] + 39, 0:128] = math.nan   # the last key of sequence 0, seen by its last query only
    b.run(ctx)
    bad = ~torch.isfinite(b.o.reshape(-1, 4, 128)[:70]).all(2)
    want = torch.zeros_like(bad)
    want[39, :2] = True
    assert torch.equal(bad, want)


@pytest.mark.parametrize("lens", [[(1, 6000), (1, 6000)], [(40, 6000), (3, 6000)]])
@pytest.mark.parametrize("prefix", [None, 700])
def test_nan_queries_with_keys_in_parts(lens, prefix, ctx):
    """No part of a row's keys may lose that its scores are NaN."""
    b = Batch(lens, 4, 2, 128, "f16", prefix=prefix)
    b.q[0, :128] = math.nan
    b.run(ctx)
    n = b.starts[-1]
    bad = ~torch.isfinite(b.o.reshape(-1, 4, 128)[:n]).all(2)
    want = torch.zeros_like(bad)
    want[0, 0] = True
    assert torch.equal(bad, want) and torch.equal(torch.isnan(b.lse[:n]), want)


def test_a_prefix_equals_its_keys_in_front(ctx):
    """The same attention written in two ways, both within their bound of 64 bits and of each other."""
    b = Batch([(1, 200), (60, 60), (3, 9)], 14, 2, 128, "f16", prefix=260)
    b.run(ctx).check()
    c = Batch([(1, 460), (60, 320), (3, 269)], 14, 2, 128, "f16")
    c.q.copy_(b.q)
    for (_, _, k0, lk), (_, _, j0, _) in zip(b.seqs, c.seqs):
        for x, y, z in ((b.k, b.pk, c.k), (b.v, b.pv, c.v)):
            z[j0:j0 + 260] = y
            z[j0 + 260:j0 + 260 + lk] = x[k0:k0 + lk]
    c.run(ctx).check()


def test_ranges_are_clipped(ctx):
    """Starts and lengths that leave the tensors' rows."""
    b = Batch([(10, 50), (20, 60)], 2, 2, 64, "f16", behind=5)
    n, rows = b.q.shape[0], b.k.shape[0]
    b.k.copy_(torch.randn(rows, 128, device=DEV).half())
    b.v.copy_(torch.randn(rows, 128, device=DEV).half())
    b.run(ctx, k_start=i32([-5, rows - 7]), k_len=i32([rows + 100, 1000000]))
    b.seqs = [(0, 10, 0, rows), (10, 20, rows - 7, 7)]
    b.check()
    b.run(ctx, k_start=i32([rows + 9, 3]), k_len=i32([4, -3]))
    b.seqs = [(0, 10, 0, 0), (10, 20, 0, 0)]
    b.check()
    b.starts = [0, 10, n + 50]
    b.run(ctx, k_start=i32([0, 0]), k_len=i32([40, 41]))
    b.starts = [0, 10, n]
    b.seqs = [(0, 10, 0, 40), (10, n - 10, 0, 41)]
    b.check()


def test_offsets_past_32_bits(ctx):
    """Keys past 2^32 bytes and 2^31 elements of the cache."""
    n, ld = 70000, 1 << 15
    k = torch.empty(n, ld, device=DEV, dtype=torch.bfloat16)
    b = Batch([(1, 700), (70, 300)], 4, 2, 128, "bf16", pad=0)
    at = [n - 700, 66000]
    small = [b.k, b.v]
    b.k, b.v = k[:, :256], k[:, 1024:1280]
    for (_, _, k0, lk), to in zip(b.seqs, at):
        b.k[to:to + lk] = small[0][k0:k0 + lk]
        b.v[to:to + lk] = small[1][k0:k0 + lk]
    b.seqs = [(q0, lq, to, lk) for (q0, lq, _, lk), to in zip(b.seqs, at)]
    b.run(ctx, k_start=i32(at)).check()


@pytest.mark.parametrize("prefix", [None, 333])
def test_repeats_give_the_same_bits(prefix, ctx):
    b = Batch([(1, 5000), (33, 900), (200, 200)], 8, 2, 128, "bf16", prefix=prefix)
    work = b.work(ctx)
    first = b.run(ctx, work=work).o.clone()
    for _ in range(5):
        b.o.fill_(9.0)
        b.run(ctx, work=work)
        assert torch.equal(b.o, first)


@pytest.mark.parametrize("prefix", [None, 200])
def test_captured_with_lengths_that_change(prefix, ctx):
    """A graph is replayed on other lengths, starts and values: all are read when it runs.  Two graphs take turns
    on one workspace."""
    lens = [(1, 700), (1, 40), (1, 1)]
    s = torch.cuda.Stream()
    try:
        with torch.cuda.stream(s):
            ctx.set_stream(s.cuda_stream)
            b = Batch(lens, 8, 2, 128, "bf16", prefix=prefix, behind=0)
            c = Batch([(30, 300), (40, 40)], 8, 2, 128, "bf16", prefix=prefix, behind=0)
            n = max(x.work(ctx).numel() if x.work(ctx) is not None else 4 for x in (b, c))
            work = torch.full((n,), math.nan, device=DEV)
            starts, cstarts = i32(b.starts), i32(c.starts)

            def call(x, at):
                args = dict(x.dev, lse=x.lse, work=work, max_q=x.max_q, max_k=x.max_k)
                if x.pk is not None:
                    ctx.attention_prefix(x.q, x.k, x.v, x.o, at, x.pk, x.pv, 8, 2, **args)
                else:
                    ctx.attention_packed(x.q, x.k, x.v, x.o, at, 8, 2, **args)

            graphs = []
            for x, at in ((b, starts), (c, cstarts)):
                graphs.append(torch.cuda.CUDAGraph())
                with torch.cuda.graph(graphs[-1], stream=s):
                    call(x, at)
            for ks, kl in (([3, 710, 755], [700, 40, 1]), ([3, 3, 10], [5, 699, 0]), ([0, 0, 0], [0, 0, 0])):
                b.k.copy_(torch.randn_like(b.k))
                b.v.copy_(torch.randn_like(b.v))
                b.dev["k_start"].copy_(i32(ks))
                b.dev["k_len"].copy_(i32(kl))
                b.seqs = [(i, 1, x, y) for i, (x, y) in enumerate(zip(ks, kl))]
                for _ in range(2):
                    for g in graphs:
                        g.replay()
                b.check()
                c.check()
            starts.copy_(i32([0, 0, 3, 3]))     # all rows to the second sequence
            b.dev["k_start"].copy_(i32([0, 5, 0]))
            b.dev["k_len"].copy_(i32([3, 100, 3]))
            b.seqs = [(0, 0, 0, 3), (0, 3, 5, 100), (3, 0, 0, 3)]
            graphs[0].replay()
            b.check()
    finally:
        ctx.set_stream(0)


@pytest.mark.parametrize("captured", [False, True])
def test_own_keys_that_outlast_the_prefix(captured, ctx):
    """An estimate of one key leaves 40,000 to a CTA each, which end long after the prefix's kernel has: what follows on
    the stream, the joined sums and then what overwrites the cache, waits for both."""
    s = torch.cuda.Stream()
    try:
        with torch.cuda.stream(s):
            ctx.set_stream(s.cuda_stream)
            b = Batch([(1, 40000), (1, 5), (2, 20000)], 8, 2, 128, "bf16", prefix=130)
            n = ctx.attention_work(b.q.shape[0], 8, 128, 2, 3, 2, 1, 130)
            work = torch.full((n // 4,), math.nan, device=DEV)
            k, v, starts = b.k.clone(), b.v.clone(), i32(b.starts)
            outs = []

            def call():
                b.k.copy_(k)
                b.v.copy_(v)
                ctx.attention_prefix(b.q, b.k, b.v, b.o, starts, b.pk, b.pv, 8, 2, **b.dev, max_q=2, max_k=1, lse=b.lse,
                                     work=work)
                b.k.fill_(7.0)
                b.v.fill_(math.nan)

            if captured:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=s):
                    call()
            for _ in range(4):
                graph.replay() if captured else call()
                outs.append(b.o.clone())
            s.synchronize()
            b.k.copy_(k)
            b.v.copy_(v)
            b.check()
            assert all(torch.equal(outs[0].view(torch.int16), x.view(torch.int16)) for x in outs)
    finally:
        ctx.set_stream(0)


def test_on_another_stream(ctx):
    """Inputs made on a stream right before the call, read right after it."""
    s = torch.cuda.Stream()
    try:
        with torch.cuda.stream(s):
            ctx.set_stream(s.cuda_stream)
            b = Batch([(1, 5000), (100, 300)], 8, 2, 128, "bf16")
            work = b.work(ctx)
            x = torch.randn(4096, 4096, device=DEV)
            for _ in range(10):
                x = x @ x * 1e-3
            b.q.add_(0 * x.sum().nan_to_num(0.0, 0.0, 0.0).to(b.dt))
            b.run(ctx, work=work)
            got = b.o.clone()
            b.o.fill_(9.0)
            b.o.copy_(got)
            b.check()
    finally:
        ctx.set_stream(0)


def test_refusals(ctx):
    b = Batch([(4, 9)], 4, 2, 128, "bf16", pad=0)
    q, k, v, o, st = b.q, b.k, b.v, b.o, i32(b.starts)

    def call(*t, heads=4, kv_heads=2, **more):
        return lambda: ctx.attention_packed(*t, heads, kv_heads, **dict(b.dev, **more))

    wide = torch.zeros(7, 520, device=DEV, dtype=b.dt)
    for f, status in (
        (call(q, k, v, q, st), 1),                                           # o over q
        (call(q, k, v, o, o.view(torch.int32)[0, :2]), 1),                   # and over the starts
        (call(q, k, v, o, st, work=o), 1),
        (call(q, k, v, o, st, scale=-1.0), 1),
        (call(q, k, v, o, st, scale=math.inf), 1),
        (call(q, k, v, o, st, k_len=None), 1),
        (call(q, k[:2], v[:2], o, st, k_start=None, k_len=None), 1),         # fewer keys than queries
        (call(q, k, v, o, st, max_q=-1), 1),
        (call(q, k, v, o, st, work=torch.zeros(65, device=DEV)[1:]), 1),     # not aligned
        (call(wide[:, 1:513], k, v, o, st), 7),
        (call(q[:, :384], k[:, :192], v[:, :192], o[:, :384], st), 7),       # heads of 96
    ):
        with pytest.raises(bag.BagError) as e:
            f()
        assert e.value.status == status, str(e.value)
    for f in (
        call(q, k, v, o, st, heads=3, kv_heads=1),
        call(q, k.half(), v, o, st),
        call(q, k, v[:3], o, st),
        call(q, k, v, o[:2], st),
        call(q, k, v, o, st.long()),
        call(q, k, v, o, st, lse=torch.zeros(7, 3, device=DEV)),
        call(q.float(), k, v, o, st),
    ):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(ValueError):
        ctx.attention_prefix(q, k, v, o, st, k[:, :128], v, 4, 2, **b.dev)
    with pytest.raises(bag.BagError) as e:
        ctx.attention_prefix(q, k, v, o, st, o[:, :256], v[:7], 4, 2, **b.dev)  # o over the prefix
    assert e.value.status == 1
    with pytest.raises(bag.BagError) as e:
        ctx.attention_work(4, 5, 128, 2, 1, 4, 9)
    assert e.value.status == 1
    assert bool((o == 9).all())
    ctx.attention_packed(q[:0], k, v, o[:0], st, 4, 2, **b.dev)
    ctx.attention_packed(q, k, v, o, st[:1], 4, 2, k_start=st[:0], k_len=st[:0])
    assert bool((o == 9).all())


@pytest.mark.parametrize("heads, kv_heads", [(0, 2), (4, 0), (0, 0), (-4, -2)])
def test_heads_that_are_none(heads, kv_heads, ctx):
    b = Batch([(4, 9)], 4, 2, 128, "bf16", pad=0)
    with pytest.raises((ValueError, bag.BagError)):
        ctx.attention_packed(b.q, b.k, b.v, b.o, i32(b.starts), heads, kv_heads, **b.dev)
    assert bool((b.o == 9).all())
