"""Performance cases of the operators of a prompt's side: rotary positions on the way into a key-value
cache, attention over packed sequences of different lengths, and attention of a batch whose
sequences share a prefix.

  rope    `Context.rope`: queries and keys of packed rows are rotated by their positions; keys go, with
          the values, into rows of a cache.  With `inverse` the rotation by the negative angle, which
          is the backward pass of the queries and keys
  packed  `Context.attention_packed`: causal attention of packed sequences, each over its own rows of
          a cache; grouped heads; a sequence's queries are its last tokens, so one query a sequence
          is the step of generation and all of them a whole prompt
  prefix  `Context.attention_prefix`: the same, where all sequences see a prefix first, whose keys
          and values are there once

Rotation.  Pair i of a head's first `rot` columns, (2i, 2i + 1) interleaved or (i, i + rot / 2) in halves,
turns by the angle position * f_i and is multiplied by `scale`; other columns are copied.
f_i = theta^(-2i / rot); for long contexts (`factor` above 1) by parts: frequencies that turn fewer
than once in the `original` length are divided by the factor, those that turn more than 32 times
stay, in between linearly, and scale = 0.1 ln(factor) + 1.

Attention.  Query t of a sequence of lq queries and lk keys sees its keys 0 .. t + lk - lq (and the whole
prefix); weights are the softmax of q . k / sqrt(head width).
"""

import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"
DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # the next token of one text, into the cache that its attention reads: all latency
        dict(name="rope_token", op="rope", rows=1, heads=28, kv_heads=4, dh=128, rot=128, layout="half", dtype="bf16",
             far=32768, factor=1.0, pool=4096, inverse=False),
        # the text of a reduced backbone, neighbouring pairs, fp32
        dict(name="rope_text", op="rope", rows=77, heads=4, kv_heads=4, dh=64, rot=64, layout="interleaved",
             dtype="f32", far=77, factor=1.0, pool=0, inverse=False),
        # a batch of prompts, ragged, half of each head rotated, long-context frequencies
        dict(name="rope_prompts", op="rope", rows=6111, heads=32, kv_heads=8, dh=128, rot=64, layout="half",
             dtype="bf16", far=131072, factor=4.0, pool=16384, inverse=False),
        # gradients of a video's queries and keys (81 frames 480x832)
        dict(name="rope_backward", op="rope", rows=32760, heads=40, kv_heads=40, dh=128, rot=128,
             layout="interleaved", dtype="bf16", far=32760, factor=1.0, pool=0, inverse=True),
        # the two prompts of a guided sample through a small text encoder
        dict(name="packed_pair", op="packed", seqs=2, lq_lo=7, lq_hi=77, past_lo=0, past_hi=0, mix=1,
             heads=12, kv_heads=12, dh=64, dtype="f16"),
        # a batch of prompts of very different lengths
        dict(name="packed_prompts", op="packed", seqs=32, lq_lo=8, lq_hi=512, past_lo=0, past_hi=0, mix=2,
             heads=28, kv_heads=4, dh=128, dtype="bf16"),
        # one long document
        dict(name="packed_long", op="packed", seqs=1, lq_lo=16384, lq_hi=16384, past_lo=0, past_hi=0, mix=3,
             heads=32, kv_heads=8, dh=128, dtype="bf16"),
        # conversations that go on: some new tokens each, behind cached ones
        dict(name="packed_extend", op="packed", seqs=8, lq_lo=16, lq_hi=512, past_lo=1000, past_hi=16384, mix=4,
             heads=32, kv_heads=8, dh=128, dtype="f16"),
        # one token each of a batch of texts
        dict(name="packed_tokens", op="packed", seqs=64, lq_lo=1, lq_hi=1, past_lo=511, past_hi=32767, mix=5,
             heads=32, kv_heads=8, dh=128, dtype="bf16"),
        # the next token of one long text
        dict(name="packed_token", op="packed", seqs=1, lq_lo=1, lq_hi=1, past_lo=131070, past_hi=131070, mix=6, heads=28,
             kv_heads=4, dh=128, dtype="f16"),
        # prompts behind the instructions that all of them start with
        dict(name="prefix_prompts", op="prefix", seqs=24, lq_lo=16, lq_hi=300, past_lo=0, past_hi=0, mix=7, prefix=1003, heads=28,
             kv_heads=4, dh=128, dtype="bf16"),
        # one token each of many texts that continue one document
        dict(name="prefix_tokens", op="prefix", seqs=128, lq_lo=1, lq_hi=1, past_lo=0, past_hi=511, mix=8, prefix=16384, heads=32,
             kv_heads=8, dh=128, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    if lo <= 0:
        return max(0, _log_int(rng, 1, hi + 1) - 1) if hi > 0 else 0
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))) if hi > lo else lo


def _heads(rng):
    kv_heads = rng.choice([1, 2, 4, 5, 8])
    return kv_heads * rng.choice([1, 2, 4, 7, 8]), kv_heads


def draw(rng):
    op = rng.choice(["rope", "packed", "packed", "prefix"])
    heads, kv_heads = _heads(rng)
    dh, dtype = rng.choice([64, 128, 128]), rng.choice(["bf16", "f16"])
    if op == "rope":
        rows = _log_int(rng, 1, 32760)
        return dict(op=op, rows=rows, heads=heads, kv_heads=kv_heads, dh=dh, rot=rng.choice([dh, dh, dh // 2, dh // 4]),
                    layout=rng.choice(["half", "interleaved"]), dtype=rng.choice([dtype, dtype, "f32"]),
                    far=_log_int(rng, rows, 1 << 20), factor=rng.choice([1.0, 4.0, 10.0]),
                    pool=rng.choice([0, rows + _log_int(rng, 1, 4096)]), inverse=rng.random() < 0.25)
    kind = rng.choice(["prompts", "extend", "tokens"])
    seqs = _log_int(rng, 1, 64)
    lq_lo = lq_hi = 1
    if kind != "tokens":
        lq_hi = _log_int(rng, 16, max(16, 8192 // seqs))
        lq_lo = rng.choice([0 if seqs > 4 else 1, 1, lq_hi // 2, lq_hi])
    past_lo = past_hi = 0
    if kind != "prompts":
        past_lo, past_hi = rng.choice([0, 100]), _log_int(rng, 512, 32768 if kind == "tokens" else 8192)
    case = dict(op=op, seqs=seqs, lq_lo=lq_lo, lq_hi=lq_hi, past_lo=past_lo, past_hi=past_hi,
                mix=rng.randrange(1 << 30), heads=heads, kv_heads=kv_heads, dh=dh, dtype=dtype)
    if op == "prefix":
        case["prefix"] = _log_int(rng, 1, 16384 if kind == "tokens" else 4096)
    return case


def _lens(case):
    """Queries and keys of each sequence."""
    rng = random.Random(case["mix"])
    lq = [_log_int(rng, case["lq_lo"], case["lq_hi"]) for _ in range(case["seqs"])]
    return lq, [n + _log_int(rng, case["past_lo"], case["past_hi"]) for n in lq]


# ---------------------------------------------------------------------------
# inputs and state
# ---------------------------------------------------------------------------
def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _frequencies(case):
    """Radians a position of each pair, and the factor of all results."""
    rot, factor, original = case["rot"], case["factor"], 8192
    f = [10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)]
    if factor == 1.0:
        return f, 1.0
    out = []
    for x in f:
        keep = min(1.0, max(0.0, (original * x / (2.0 * math.pi) - 1.0) / 31.0))
        out.append(x * (keep + (1.0 - keep) / factor))
    return out, 0.1 * math.log(factor) + 1.0


def _rope_inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    rows, H, Hk, dh, dt = case["rows"], case["heads"], case["kv_heads"], case["dh"], DTYPE[case["dtype"]]
    # queries, keys and values are columns of one projection's output
    qkv = torch.empty(rows, (H + 2 * Hk) * dh, device=DEV, dtype=dt)
    for r in range(0, rows, 4096):
        part = qkv[r:r + 4096]
        part.copy_(_randn(g, *part.shape))
    s = dict(q=qkv[:, :H * dh], k=qkv[:, H * dh:(H + Hk) * dh], v=qkv[:, (H + Hk) * dh:])
    # packed sequences: positions run on from somewhere in each
    pos = torch.arange(rows, device=DEV, dtype=torch.int32)
    for cut in torch.randint(0, rows, (4,), generator=g, device=DEV).tolist():
        pos[cut:] += -pos[cut] + torch.randint(0, max(1, case["far"] - rows + cut), (1,), generator=g, device=DEV).int()
    s["pos"] = pos.contiguous()
    s["slots"] = None
    if case["pool"] and not case["inverse"]:
        s["slots"] = torch.randperm(case["pool"], generator=g, device=DEV)[:rows].to(torch.int32)
    cap = case["pool"] if s["slots"] is not None else rows
    s["q_out"] = torch.zeros(rows, H * dh, device=DEV, dtype=dt)
    s["k_out"] = torch.zeros(cap, Hk * dh, device=DEV, dtype=dt)
    if not case["inverse"]:
        s["v_out"] = torch.zeros(cap, Hk * dh, device=DEV, dtype=dt)
    freqs, s["scale"] = _frequencies(case)
    s["freqs"] = np.array(freqs)
    return s


def _attention_inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    H, Hk, dh, dt = case["heads"], case["kv_heads"], case["dh"], DTYPE[case["dtype"]]
    lq, lk = _lens(case)
    nq = sum(lq)
    # the sequences lie in the cache in some order, with rows of earlier ones between them
    order = torch.randperm(len(lk), generator=g, device=DEV).tolist()
    gaps = torch.randint(0, 64, (len(lk) + 1,), generator=g, device=DEV).tolist()
    start, at = [0] * len(lk), gaps[-1]
    for i in order:
        start[i] = at
        at += lk[i] + gaps[i]
    s = dict(lq=lq, lk=lk, start=start)
    s["q"] = torch.empty(nq, H * dh, device=DEV, dtype=dt)
    s["k"], s["v"] = (torch.empty(at, Hk * dh, device=DEV, dtype=dt) for _ in range(2))
    # heads differ in how sharp their weights are; some tokens matter to all
    sharp = 0.5 + 1.5 * torch.rand(1, H, 1, generator=g, device=DEV)
    for r in range(0, nq, 8192):
        n = min(8192, nq - r)
        s["q"][r:r + n].view(n, H, dh).copy_(sharp * _randn(g, n, H, dh))

    def keys(x, v):
        for r in range(0, x.shape[0], 32768):
            n = min(32768, x.shape[0] - r)
            loud = 1.0 + (torch.rand(n, 1, generator=g, device=DEV) < 0.01)
            x[r:r + n].copy_(loud * _randn(g, n, Hk * dh))
            v[r:r + n].copy_(_randn(g, n, Hk * dh))

    keys(s["k"], s["v"])
    if case["op"] == "prefix":
        s["pk"], s["pv"] = (torch.empty(case["prefix"], Hk * dh, device=DEV, dtype=dt) for _ in range(2))
        keys(s["pk"], s["pv"])
    return s


def _inputs(case, seed):
    return _rope_inputs(case, seed) if case["op"] == "rope" else _attention_inputs(case, seed)


def prepare(case, seed):
    s = dict(case=case, **_inputs(case, seed))
    if case["op"] != "rope":
        ints = dict(device=DEV, dtype=torch.int32)
        s["q_start"] = torch.tensor([sum(s["lq"][:i]) for i in range(case["seqs"] + 1)], **ints)
        s["k_start"], s["k_len"] = torch.tensor(s["start"], **ints), torch.tensor(s["lk"], **ints)
        s["o"] = torch.zeros(sum(s["lq"]), case["heads"] * case["dh"], device=DEV, dtype=DTYPE[case["dtype"]])
        s["max_q"], s["max_k"] = max(s["lq"]), max(s["lk"])
    if own:  # the calls need a context for their stream and errors, and a workspace; a program has both
        from paper_2608_09231_gb300 import bag
        s["ctx"] = bag.create("tiny", weight_seed=int(seed) & 0x7FFFFFFF)
        if case["op"] != "rope":
            n = s["ctx"].attention_work(s["q"].shape[0], case["heads"], case["dh"], case["kv_heads"], case["seqs"],
                                        s["max_q"], s["max_k"], case.get("prefix", 0))
            s["work"] = torch.empty(n, device=DEV, dtype=torch.uint8)
    return s


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _rotate(x, cos, sin, dh, layout):
    """Heads of x [rows, heads * dh] in fp32; cos, sin [rows, 1, pairs]."""
    n = cos.shape[2]
    h = x.float().view(x.shape[0], -1, dh)
    if layout == "half":
        a, b = h[:, :, :n], h[:, :, n:2 * n]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos, h[:, :, 2 * n:]], 2)
    else:
        a, b = h[:, :, 0:2 * n:2], h[:, :, 1:2 * n:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], 3).flatten(2)
        turned = torch.cat([turned, h[:, :, 2 * n:]], 2)
    return turned.view(x.shape[0], -1).to(x.dtype)


def _plain_rope(s):
    case = s["case"]
    angle = s["pos"].double().unsqueeze(1) * torch.tensor(s["freqs"], device=DEV, dtype=torch.float64)
    angle = -angle if case["inverse"] else angle
    cos, sin = ((f(angle) * s["scale"]).float().unsqueeze(1) for f in (torch.cos, torch.sin))
    at = slice(None) if s["slots"] is None else s["slots"].long()
    s["q_out"].copy_(_rotate(s["q"], cos, sin, case["dh"], case["layout"]))
    s["k_out"][at] = _rotate(s["k"], cos, sin, case["dh"], case["layout"])
    if not case["inverse"]:
        s["v_out"][at] = s["v"]
    return _rope_outputs(s)


def _rope_outputs(s):
    return {n: s[n] for n in ("q_out", "k_out", "v_out") if n in s}


def _split(x, heads, dh):
    """[rows, heads * dh] -> fp32 [heads, rows, dh]."""
    return x.float().view(x.shape[0], heads, dh).transpose(0, 1)


def _plain_attention(s):
    case = s["case"]
    H, Hk, dh = case["heads"], case["kv_heads"], case["dh"]
    G, scale = H // Hk, 1.0 / math.sqrt(dh)
    at = 0
    prefix = "pk" in s
    if prefix:  # all queries meet the prefix together
        q = _split(s["q"], H, dh).reshape(Hk, -1, dh)
        zp = (q @ _split(s["pk"], Hk, dh).transpose(1, 2) * scale).view(H, -1, s["pk"].shape[0])
        pv = _split(s["pv"], Hk, dh)
        top = zp.amax(2, keepdim=True)
        wp = (zp - top).exp_()
        den = wp.sum(2, keepdim=True)
        out = (wp.view(Hk, -1, wp.shape[2]) @ pv).view(H, -1, dh)
        del zp, wp, q
    for lq, lk, k0 in zip(s["lq"], s["lk"], s["start"]):
        if lq == 0:
            continue
        hidden = torch.arange(lk, device=DEV) > torch.arange(lq, device=DEV).unsqueeze(1) + (lk - lq)
        group = 1 if Hk * G * lq * lk > 1 << 30 else Hk  # key heads at a time
        for h in range(0, Hk, group):
            cq, ck = slice(h * G * dh, (h + group) * G * dh), slice(h * dh, (h + group) * dh)
            q = _split(s["q"][at:at + lq, cq], group * G, dh).reshape(group, G * lq, dh)
            k, v = (_split(s[n][k0:k0 + lk, ck], group, dh) for n in ("k", "v"))
            z = (q @ k.transpose(1, 2)).mul_(scale).view(group * G, lq, lk)
            z.masked_fill_(hidden, -math.inf)
            m = z.amax(2, keepdim=True)
            w = z.sub_(m).exp_()
            o, d = (w.view(group, G * lq, lk) @ v).view(group * G, lq, dh), w.sum(2, keepdim=True)
            if prefix:
                mp, dp, op = (t[h * G:(h + group) * G, at:at + lq] for t in (top, den, out))
                both = torch.maximum(m, mp)
                a, b = torch.exp(m - both), torch.exp(mp - both)
                o, d = o * a + op * b, d * a + dp * b
            s["o"][at:at + lq, cq] = (o / d).transpose(0, 1).reshape(lq, -1).to(s["o"].dtype)
        at += lq
    return s["o"]


def run(s):
    case = s["case"]
    if not own:
        return _plain_rope(s) if case["op"] == "rope" else _plain_attention(s)
    ctx = s["ctx"]
    if case["op"] == "rope":
        values = {} if case["inverse"] else dict(v=s["v"], v_out=s["v_out"])
        ctx.rope(s["q"], s["q_out"], s["freqs"], case["dh"], pos=s["pos"], k=s["k"], k_out=s["k_out"],
                 slots=s["slots"], layout=case["layout"], scale=s["scale"], inverse=case["inverse"], **values)
        return _rope_outputs(s)
    sequences = dict(k_start=s["k_start"], k_len=s["k_len"], max_q=s["max_q"], max_k=s["max_k"], work=s["work"])
    if case["op"] == "packed":
        ctx.attention_packed(s["q"], s["k"], s["v"], s["o"], s["q_start"], case["heads"], case["kv_heads"], **sequences)
    else:
        ctx.attention_prefix(s["q"], s["k"], s["v"], s["o"], s["q_start"], s["pk"], s["pv"], case["heads"],
                             case["kv_heads"], **sequences)
    return s["o"]


# ---------------------------------------------------------------------------
# what each pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    H, Hk, dh = case["heads"], case["kv_heads"], case["dh"]
    if case["op"] == "rope":
        rows, es = case["rows"], 4 if case["dtype"] == "f32" else 2
        n = rows * dh * (H + (1 if case["inverse"] else 2) * Hk)
        index = 8 if case["pool"] and not case["inverse"] else 4
        return {"bytes": 2 * es * n + index * rows, "flops": 3 * rows * case["rot"] * (H + Hk)}
    lq, lk = _lens(case)
    prefix = case.get("prefix", 0)
    seen = sum(n * (m - n) + n * (n + 1) // 2 for n, m in zip(lq, lk)) + sum(lq) * prefix
    keys = sum(m for n, m in zip(lq, lk) if n) + prefix
    return {"bytes": 4 * dh * (H * sum(lq) + Hk * keys) + 12 * case["seqs"], "flops": 4 * dh * H * seen}


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------
def _exact_rope(case, s):
    rows, dh, n = case["rows"], case["dh"], len(s["freqs"])
    sign = -1.0 if case["inverse"] else 1.0
    pair = torch.arange(n, device=DEV)
    first, second = (pair, pair + n) if case["layout"] == "half" else (2 * pair, 2 * pair + 1)
    f = torch.tensor(s["freqs"], device=DEV, dtype=torch.float64)

    def turned(x):
        y = x.double().view(rows, -1, dh).clone()
        for r in range(0, rows, 4096):
            t = torch.outer(s["pos"][r:r + 4096].double(), f)
            z = torch.complex(y[r:r + 4096, :, first], y[r:r + 4096, :, second])
            z = z * torch.polar(torch.full_like(t, s["scale"]), sign * t).unsqueeze(1)
            y[r:r + 4096, :, first], y[r:r + 4096, :, second] = z.real, z.imag
        return y.view(rows, -1)

    out = {"q_out": turned(s["q"]), "k_out": s["k_out"].double()}
    at = torch.arange(rows, device=DEV) if s["slots"] is None else s["slots"].long()
    out["k_out"][at] = turned(s["k"])
    if not case["inverse"]:
        out["v_out"] = s["v_out"].double()
        out["v_out"][at] = s["v"].double()
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "rope":
        return _exact_rope(case, s)
    H, Hk, dh = case["heads"], case["kv_heads"], case["dh"]
    out = torch.zeros(sum(s["lq"]), H * dh, device=DEV, dtype=torch.float64)
    row = 0
    for lq, lk, k0 in zip(s["lq"], s["lk"], s["start"]):
        for h in range(Hk):
            c = slice(h * dh, (h + 1) * dh)
            k, v = s["k"][k0:k0 + lk, c], s["v"][k0:k0 + lk, c]
            if "pk" in s:
                k, v = torch.cat([s["pk"][:, c], k]), torch.cat([s["pv"][:, c], v])
            k, v = k.double(), v.double()
            for g in range(h * (H // Hk), (h + 1) * (H // Hk)):
                for r in range(0, lq, 4096):
                    n = min(4096, lq - r)
                    last = k.shape[0] - lq + r + n  # keys that the last of these queries sees
                    z = s["q"][row + r:row + r + n, g * dh:(g + 1) * dh].double() @ k[:last].T / math.sqrt(dh)
                    z += torch.full_like(z, -math.inf).triu(last - n + 1)
                    out[row + r:row + r + n, g * dh:(g + 1) * dh] = torch.softmax(z, 1) @ v[:last]
        row += lq
    return out
