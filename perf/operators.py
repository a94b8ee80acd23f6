"""Performance cases of the operators that make full and reused steps cheaper: rows in 8-bit
floating point with a scale for each block of 128, their matrix product, the quantised
cache, and attention over selected blocks of keys.

  quant  `Context.quant_fp8`: rows of fp32 or bf16 to e4m3 codes and power-of-two scales
  norm   `Context.ln_mod_fp8`: LayerNorm + adaLN modulation straight to codes and scales
  gemm   `Context.gemm_fp8`: product of two such operands; stores fp32 / bf16 (with GELU),
         quantises its output for the next product, or updates a residual stream
  cache  `Context.cache_write`, then `Context.cache_read`: a residual (h_out - h_in) is
         quantised into slots of a cache and read back on top of h_in
  read   `Context.cache_read` alone, as the reused steps of a sample call it
  attn   `Context.block_pool`, `Context.block_select` and `Context.attention_blocks`: every
         block of 128 queries attends to the `keep` blocks of 128 keys whose score is highest;
         with `pooled` the keys stay from pass to pass, and so do their pooled vectors

Formats.  Codes: float8 e4m3, scale byte b of a block of 128 columns = 2^(b - 127), the least
power of two with amax / scale <= 448.  Cache: 8 bits, codes -127..127, one bf16 scale
amax / 127 for 128 columns; 4 bits, codes -7..7, two in a byte (even column low), one bf16
scale amax / 7 for 32 columns.

Scores.  The mean of each block's rows (summed in halves: row r + row r + 64, then r + 32, ...)
is rounded to integers of 8 bits under one scale amax / 127; the score of a query block and a
key block is the integer dot product times the key block's scale.  Integer sums are exact, so
the selection does not depend on the order in which anything is summed; ties go to the lower
index.
"""

import math

import torch

own = False
DEV = "cuda"
BLOCK = 128
GROUP = {8: 128, 4: 32}
TOP = {8: 127, 4: 7}


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # tokens of the smallest backbone before a projection: a call that is all latency
        dict(name="quant_tiny", op="quant", rows=256, cols=256, dtype="f32", pad=0),
        # a Wan-shaped video's attention output (81 frames 480x832), before its out-projection
        dict(name="quant_wan", op="quant", rows=32760, cols=5120, dtype="bf16", pad=0),
        # a ragged reduced stream (18 x 21 image + 77 text tokens)
        dict(name="norm_small", op="norm", rows=455, cols=512),
        # the joint sequence of the FLUX shape before a block's projections
        dict(name="norm_flux_joint", op="norm", rows=4608, cols=3072),
        # one token: a conditioning vector through an MLP-sized projection
        dict(name="gemm_token", op="gemm", M=1, N=13824, K=5120, out="f32", gelu=False),
        # text tokens of a reduced backbone through its MLP up-projection
        dict(name="gemm_text_small", op="gemm", M=77, N=2048, K=512, out="bf16", gelu=True),
        # FLUX-shaped MLP up-projection with GELU, its output quantised for the next product
        dict(name="gemm_up_flux", op="gemm", M=4608, N=12288, K=3072, out="fp8", gelu=True),
        # Wan-shaped MLP down-projection of the whole video into the gated residual stream
        dict(name="gemm_down_wan", op="gemm", M=32760, N=5120, K=13824, out="resid", gelu=False),
        # a reduced sample's residual into scattered slots of a pool, 4 bits
        dict(name="cache_small_4", op="cache", rows=378, cols=512, bits=4, pool=1024),
        # the residual of a Qwen-shaped sample (83 x 83 tokens), 8 bits, written and read once
        dict(name="cache_qwen_8", op="cache", rows=6889, cols=3072, bits=8, pool=0),
        # one query token against a Wan-shaped video's keys, an eighth of its blocks
        dict(name="attn_token", op="attn", nq=1, nk=32760, heads=40, kv_heads=40, keep=32, dtype="f16",
             pooled=True),
        # four heads of a Wan-shaped video's self-attention, a quarter of its blocks
        dict(name="attn_wan", op="attn", nq=32760, nk=32760, heads=4, kv_heads=4, keep=64, dtype="f16",
             pooled=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quant", "norm", "gemm", "gemm", "gemm", "cache", "read", "attn", "attn"])
    if op == "quant":
        return dict(op=op, rows=_log_int(rng, 1, 32760), cols=_log_int(rng, 64, 5120),
                    dtype=rng.choice(["f32", "bf16"]), pad=rng.choice([0, 0, 1, 8]))
    if op == "norm":
        return dict(op=op, rows=_log_int(rng, 1, 32760), cols=4 * _log_int(rng, 64, 1536))
    if op == "gemm":
        out = rng.choice(["f32", "bf16", "fp8", "resid"])
        M, N, K = _log_int(rng, 1, 8192), _log_int(rng, 64, 13824), _log_int(rng, 64, 13824)
        if rng.random() < 0.5:   # widths of whole blocks, as a model has them
            N, K = max(1, N // 128) * 128, max(1, K // 128) * 128
        return dict(op=op, M=M, N=N, K=K, out=out, gelu=out != "resid" and rng.random() < 0.5)
    if op == "attn":
        kv_heads = rng.choice([1, 2, 4, 8, 12, 24])
        heads = kv_heads * rng.choice([1, 1, 1, 2, 4])
        most = 4 * 32760 ** 2 / heads                    # of nq * nk
        nk = _log_int(rng, 1, min(32760, int(math.sqrt(most))))
        nq = rng.choice([nk, nk, 1, _log_int(rng, 1, nk)])
        return dict(op=op, nq=nq, nk=nk, heads=heads, kv_heads=kv_heads,
                    keep=rng.randint(1, max(1, -(-nk // 128) // 3)), dtype=rng.choice(["f16", "bf16"]),
                    pooled=nq == 1 or rng.random() < 0.3)
    rows = _log_int(rng, 1, 32760)
    return dict(op=op, rows=rows, cols=_log_int(rng, 64, 5120), bits=rng.choice([8, 4]),
                pool=rng.choice([0, rows + _log_int(rng, 1, 4096)]))


# ---------------------------------------------------------------------------
# inputs and state
# ---------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _up(n, m):
    return (n + m - 1) // m * m


def _stream(g, rows, cols):
    """Tokens of a residual stream: rows of different size, a few channels much larger."""
    x = _randn(g, rows, cols)
    x *= 0.5 + torch.rand(rows, 1, generator=g, device=DEV)
    return x.mul_(1.0 + 9.0 * (torch.rand(cols, generator=g, device=DEV) < 0.01))


def _slots(g, case):
    if not case["pool"]:
        return None
    return torch.randperm(case["pool"], generator=g, device=DEV)[:case["rows"]].to(torch.int32)


def _encode(x):
    """Codes and scale bytes of rows, in the layout of the library: code rows of a multiple of
    16 bytes, scale rows of a multiple of 4."""
    rows, cols = x.shape
    codes, b = _fp8(x)
    c = torch.zeros(rows, _up(cols, 16), device=DEV, dtype=torch.uint8)
    c[:, :cols] = codes.view(torch.uint8)
    s = torch.zeros(rows, _up(b.shape[1], 4), device=DEV, dtype=torch.uint8)
    s[:, :b.shape[1]] = b
    return c, s


def _context(seed):
    """The framework's calls need a context for their stream and errors; a program has one."""
    if not own:
        return None
    from paper_2608_09231_gb300 import bag
    return bag.create("tiny", weight_seed=int(seed) & 0x7FFFFFFF)


def _inputs(case, seed):
    g, op = _gen(seed), case["op"]
    if op == "quant":
        x = _stream(g, case["rows"], case["cols"] + case["pad"])
        return dict(x=(x if case["dtype"] == "f32" else x.bfloat16())[:, case["pad"]:])
    if op == "norm":
        return dict(x=_stream(g, case["rows"], case["cols"]) + 0.3,
                    shift=0.3 * _randn(g, case["cols"]), scale=0.3 * _randn(g, case["cols"]))
    if op == "gemm":
        M, N, K = case["M"], case["N"], case["K"]
        s = dict(zip(("a", "sa"), _encode(_stream(g, M, K))))
        s.update(zip(("w", "sw"), _encode(0.02 * _randn(g, N, K))))
        s["bias"] = 0.02 * _randn(g, N)
        if case["out"] == "resid":
            s.update(h0=_stream(g, M, N), gate=0.3 * _randn(g, N))
        return s
    if op == "attn":
        dt = torch.float16 if case["dtype"] == "f16" else torch.bfloat16
        nq, nk, H, Hk = case["nq"], case["nk"], case["heads"], case["kv_heads"]
        # neighbouring tokens are alike: a part that each run of 256 shares, and one of its own
        common = _randn(g, nk // 256 + 1, Hk, 128)
        k = _randn(g, nk, Hk, 128) + common.repeat_interleave(256, 0)[:nk]
        common = common.repeat_interleave(H // Hk, 1)[torch.randperm(nk // 256 + 1, generator=g, device=DEV)]
        q = _randn(g, nq, H, 128) + 0.5 * common.repeat_interleave(256, 0)[:nq]
        vt = torch.zeros(Hk, 128, _up(nk, 8), device=DEV, dtype=dt)
        vt[:, :, :nk] = _randn(g, Hk, 128, nk).to(dt)
        return dict(q=q.view(nq, -1).to(dt), k=k.view(nk, -1).to(dt), vt=vt)
    rows, cols, bits = case["rows"], case["cols"], case["bits"]
    s = dict(h_in=_stream(g, rows, cols), slots=_slots(g, case))
    if op == "cache":
        s["h_out"] = s["h_in"] + _stream(g, rows, cols)
        return s
    cap = case["pool"] or rows
    codes, scales = _quantise(_stream(g, cap, cols), bits)
    c = codes.to(torch.int32) & (0xFF if bits == 8 else 0xF)
    if bits == 4:
        c = torch.nn.functional.pad(c, (0, _up(cols, 2) - cols))
        c = c[:, 0::2] | (c[:, 1::2] << 4)
    s["codes"] = torch.zeros(cap, _up(c.shape[1], 16), device=DEV, dtype=torch.uint8)
    s["codes"][:, :c.shape[1]] = c.to(torch.uint8)
    s["scales"] = torch.zeros(cap, _up(scales.shape[1], 8), device=DEV, dtype=torch.bfloat16)
    s["scales"][:, :scales.shape[1]] = scales
    return s


def prepare(case, seed):
    op = case["op"]
    s = dict(case=case, ctx=_context(seed), **_inputs(case, seed))
    if op in ("quant", "norm"):
        rows, cols = case["rows"], case["cols"]
        s["codes"] = torch.zeros(rows, _up(cols, 16), device=DEV, dtype=torch.uint8)
        s["scales"] = torch.zeros(rows, _up(_up(cols, BLOCK) // BLOCK, 4), device=DEV, dtype=torch.uint8)
    elif op == "gemm":
        M, N = case["M"], case["N"]
        if case["out"] == "fp8":
            s["out"] = torch.zeros(M, _up(N, 16), device=DEV, dtype=torch.uint8)
            s["out_s"] = torch.zeros(M, _up(_up(N, BLOCK) // BLOCK, 4), device=DEV, dtype=torch.uint8)
        else:
            s["out"] = torch.empty(M, N, device=DEV,
                                   dtype=torch.bfloat16 if case["out"] == "bf16" else torch.float32)
    elif op == "attn":
        nqb, nkb = -(-case["nq"] // BLOCK), -(-case["nk"] // BLOCK)
        s["blocks"] = torch.zeros(case["heads"], nqb, case["keep"], device=DEV, dtype=torch.int32)
        if case["pooled"]:
            codes, s["pool_s"] = _pool(s["k"], case["kv_heads"])
            s["pool"] = codes.to(torch.int8).contiguous()
            s["pool_s"] = s["pool_s"].contiguous()
        else:
            s["pool"] = torch.zeros(case["kv_heads"], nkb, 128, device=DEV, dtype=torch.int8)
            s["pool_s"] = torch.zeros(case["kv_heads"], nkb, device=DEV)
        s["out"] = torch.empty(case["nq"], case["heads"] * 128, device=DEV, dtype=torch.bfloat16)
    else:
        rows, cols, bits = case["rows"], case["cols"], case["bits"]
        s["out"] = torch.empty(rows, cols, device=DEV)
        if op == "cache":
            cap = case["pool"] or rows
            s["codes"] = torch.zeros(cap, _up(_up(cols * bits, 8) // 8, 16), device=DEV, dtype=torch.uint8)
            s["scales"] = torch.zeros(cap, _up(_up(cols, GROUP[bits]) // GROUP[bits], 8), device=DEV,
                                      dtype=torch.bfloat16)
    return s


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _blocks(x, n):
    """[rows, cols] -> [rows, blocks, n], zeros past the last column."""
    return torch.nn.functional.pad(x, (0, _up(x.shape[1], n) - x.shape[1])).view(x.shape[0], -1, n)


def _pow2(e):
    """2^e for whole e in -126..127, from the bits of a float."""
    return ((e.clamp(-126, 127) + 127) << 23).to(torch.int32).view(torch.float32)


def _fp8(x):
    """e4m3 codes of rows and the scale byte of each block of 128."""
    v = _blocks(x.float(), BLOCK)
    # the least b with amax <= 448 * 2^(b - 127); 448 = 0.875 * 2^9
    m, e = torch.frexp(v.abs().amax(2))                  # amax = m 2^e, 0.5 <= m < 1
    b = torch.where(m > 0.875, e - 8, e - 9) + 127
    b = torch.where(m == 0, torch.zeros_like(b), b).clamp(0, 254)
    q = (v * _pow2(127 - b).unsqueeze(2)).to(torch.float8_e4m3fn)
    return q.view(x.shape[0], -1)[:, :x.shape[1]], b.to(torch.uint8)


def _values(codes, b, cols):
    v = _blocks(codes[:, :cols].contiguous().view(torch.float8_e4m3fn).float(), BLOCK)
    e = b[:, :v.shape[1]].to(torch.int32) - 127
    return (v * _pow2(e).unsqueeze(2)).view(codes.shape[0], -1)[:, :cols]


def _quantise(x, bits):
    """Integer codes of rows and the bf16 scale of each group of columns."""
    v = _blocks(x, GROUP[bits])
    scale = (v.abs().amax(2) * (1.0 / TOP[bits])).bfloat16()
    s = scale.float().unsqueeze(2)
    q = torch.where(s > 0, torch.round(v * (1.0 / s)), torch.zeros_like(v)).clamp_(-TOP[bits], TOP[bits])
    return q.view(x.shape[0], -1)[:, :x.shape[1]].to(torch.int8), scale


def _dequantise(codes, scales, bits, cols):
    if bits == 8:
        q = codes[:, :cols].view(torch.int8).float()
    else:
        c = codes.to(torch.int32)
        q = torch.stack([c & 15, c >> 4], 2).view(codes.shape[0], -1)[:, :cols]
        q = torch.where(q > 7, q - 16, q).float()
    v = _blocks(q, GROUP[bits])
    return (v * scales[:, :v.shape[1]].float().unsqueeze(2)).view(codes.shape[0], -1)[:, :cols]


def _gelu(y):
    return 0.5 * y * (1.0 + torch.tanh(0.7978845608028654 * (y + 0.044715 * y * y * y)))


def _layer_norm(x, shift, scale):
    d = x - x.mean(1, keepdim=True)
    return d * torch.rsqrt((d * d).mean(1, keepdim=True) + 1e-6) * (1.0 + scale) + shift


def _pool(x, heads):
    """Integer codes [heads, blocks, 128] of the blocks' mean rows, and their scales."""
    n, blocks = x.shape[0], -(-x.shape[0] // BLOCK)
    v = torch.nn.functional.pad(x.float(), (0, 0, 0, blocks * BLOCK - n)).view(blocks, BLOCK, heads, 128)
    v = v[:, :64] + v[:, 64:]
    v = v[:, :32] + v[:, 32:]
    v = v[:, :16] + v[:, 16:]
    v = v[:, :8] + v[:, 8:]
    v = v[:, :4] + v[:, 4:]
    v = v[:, :2] + v[:, 2:]
    v = (v[:, 0] + v[:, 1]).transpose(0, 1)
    count = torch.full((blocks, 1), float(BLOCK), device=DEV)
    count[-1] = n - (blocks - 1) * BLOCK
    v = v * (1.0 / count)
    scale = v.abs().amax(2) * (1.0 / 127.0)
    s = scale.unsqueeze(2)
    return torch.where(s > 0, torch.round(v * (1.0 / s)), torch.zeros_like(v)).clamp_(-127.0, 127.0), scale


def _block_attention(s):
    case = s["case"]
    nq, nk, H, Hk, keep = (case[n] for n in ("nq", "nk", "heads", "kv_heads", "keep"))
    pq = _pool(s["q"], H)[0]
    pk, scale = (s["pool"].float(), s["pool_s"]) if case["pooled"] else _pool(s["k"], Hk)
    score = (pq.view(Hk, -1, 128) @ pk.transpose(1, 2)).view(H, -1, pk.shape[1])
    score = score * scale.repeat_interleave(H // Hk, 0).unsqueeze(1)
    blocks = score.sort(dim=2, descending=True, stable=True).indices[:, :, :keep].sort(dim=2).values
    taken = torch.zeros_like(score).scatter_(2, blocks, 1.0)
    q = s["q"].float().view(nq, H, 128).transpose(0, 1).reshape(Hk, -1, 128)
    k = s["k"].float().view(nk, Hk, 128).permute(1, 2, 0)
    p = ((q @ k) * (1.0 / math.sqrt(128.0))).view(H, nq, nk)
    row, col = torch.arange(nq, device=DEV) // BLOCK, torch.arange(nk, device=DEV) // BLOCK
    p.masked_fill_(taken[:, :, col][:, row] == 0, -math.inf)
    p -= p.amax(2, keepdim=True)
    p.exp_()
    p /= p.sum(2, keepdim=True)
    o = p.view(Hk, -1, nk) @ s["vt"][:, :, :nk].float().transpose(1, 2)
    return {"blocks": blocks.to(torch.int32), "o": o.view(H, nq, 128).transpose(0, 1).reshape(nq, -1).bfloat16()}


def _plain(s):
    case, op = s["case"], s["case"]["op"]
    if op in ("quant", "norm"):
        codes, b = _fp8(s["x"] if op == "quant" else _layer_norm(s["x"], s["shift"], s["scale"]))
        return {"codes": codes, "scales": b.view(torch.float8_e8m0fnu)}
    if op == "gemm":
        K = case["K"]
        y = _values(s["a"], s["sa"], K) @ _values(s["w"], s["sw"], K).T + s["bias"]
        if case["out"] == "resid":
            return s["h0"] + s["gate"] * y
        y = _gelu(y) if case["gelu"] else y
        if case["out"] == "fp8":
            codes, b = _fp8(y)
            return {"codes": codes, "scales": b.view(torch.float8_e8m0fnu)}
        return y if case["out"] == "f32" else y.bfloat16()
    if op == "attn":
        return _block_attention(s)
    bits, cols = case["bits"], case["cols"]
    if op == "cache":
        q, scale = _quantise(s["h_out"] - s["h_in"], bits)
        v = _blocks(q.float(), GROUP[bits]) * scale.float().unsqueeze(2)
        return s["h_in"] + v.view(case["rows"], -1)[:, :cols]
    at = s["slots"].long() if s["slots"] is not None else slice(None)
    return s["h_in"] + _dequantise(s["codes"][at], s["scales"][at], bits, cols)


def run(s):
    if not own:
        return _plain(s)
    case, op, ctx = s["case"], s["case"]["op"], s["ctx"]
    if op == "quant":
        ctx.quant_fp8(s["x"], s["codes"], s["scales"])
    elif op == "norm":
        ctx.ln_mod_fp8(s["x"], s["shift"], s["scale"], s["codes"], s["scales"])
    if op in ("quant", "norm"):
        return {"codes": s["codes"][:, :case["cols"]].view(torch.float8_e4m3fn),
                "scales": s["scales"][:, :_up(case["cols"], BLOCK) // BLOCK].view(torch.float8_e8m0fnu)}
    if op == "gemm":
        K, out = case["K"], case["out"]
        args = (s["a"], s["sa"], s["w"], s["sw"], s["out"], K)
        if out == "resid":
            s["out"].copy_(s["h0"])
            ctx.gemm_fp8(*args, bias=s["bias"], gate=s["gate"], residual=True)
            return s["out"]
        if out == "fp8":
            ctx.gemm_fp8(*args, bias=s["bias"], gelu=case["gelu"], out_scales=s["out_s"], N=case["N"])
            return {"codes": s["out"][:, :case["N"]].view(torch.float8_e4m3fn),
                    "scales": s["out_s"][:, :_up(case["N"], BLOCK) // BLOCK].view(torch.float8_e8m0fnu)}
        ctx.gemm_fp8(*args, bias=s["bias"], gelu=case["gelu"])
        return s["out"]
    if op == "attn":
        if not case["pooled"]:
            ctx.block_pool(s["k"], s["pool"], s["pool_s"])
        ctx.block_select(s["q"], s["pool"], s["pool_s"], s["blocks"])
        ctx.attention_blocks(s["q"], s["k"], s["vt"], s["out"], s["blocks"], case["heads"], case["kv_heads"])
        return {"blocks": s["blocks"], "o": s["out"]}
    if op == "cache":
        ctx.cache_write(s["h_out"], s["codes"], s["scales"], case["bits"], base=s["h_in"], slots=s["slots"])
    ctx.cache_read(s["codes"], s["scales"], s["out"], case["bits"], base=s["h_in"], slots=s["slots"])
    return s["out"]


# ---------------------------------------------------------------------------
# what each pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op in ("quant", "norm"):
        n = case["rows"] * case["cols"]
        es = 2 if op == "quant" and case["dtype"] == "bf16" else 4
        more = 8 * case["cols"] if op == "norm" else 0
        return {"bytes": n * (es + 1) + n / 128 + more, "flops": (2 if op == "quant" else 10) * n}
    if op == "gemm":
        M, N, K = case["M"], case["N"], case["K"]
        size = {"f32": 4, "bf16": 2, "fp8": 1 + 1 / 128, "resid": 8}[case["out"]]
        more = 8 * N if case["out"] == "resid" else 4 * N
        return {"bytes": (M + N) * K * (1 + 1 / 128) + M * N * size + more, "flops": 2 * M * N * K}
    if op == "attn":
        nq, nk, H, Hk, keep = (case[n] for n in ("nq", "nk", "heads", "kv_heads", "keep"))
        nqb, nkb = -(-nq // BLOCK), -(-nk // BLOCK)
        keys = min(nk, keep * BLOCK)                     # of one query
        # q is read for the scores, and the keys (or their pooled vectors); q again with the output,
        # and the selected keys and values of each block of queries if these are few, else all once
        pool = 256 * nq * H + (132 * nkb * Hk if case["pooled"] else 256 * nk * Hk)
        return {"bytes": pool + 512 * nq * H + 512 * Hk * min(nk, nqb * (H // Hk) * keys) + 4 * H * nqb * keep,
                "flops": 512 * nq * H * keys + 256 * H * nqb * nkb}
    n, bits = case["rows"] * case["cols"], case["bits"]
    held = bits / 8 + 2 / GROUP[bits]
    index = 4 * case["rows"] if case["pool"] else 0
    if op == "read":
        return {"bytes": n * (held + 8) + index, "flops": 2 * n}
    # the write reads both tensors and writes the cache; the read takes h_in again
    return {"bytes": n * (8 + held) + n * (held + 8) + 2 * index, "flops": 5 * n}


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------
def _exact_e4m3(v):
    """The e4m3 value nearest to each v (ties to an even significand), |v| <= 448, in float64."""
    _, e = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), torch.clamp(e - 4, min=-9))
    return torch.round(v / step) * step


def _exact_fp8(y):
    """Code values and scales of float64 rows."""
    rows, cols = y.shape
    n = -(-cols // 128)
    codes = torch.empty(rows, cols, device=DEV, dtype=torch.float64)
    scales = torch.empty(rows, n, device=DEV, dtype=torch.float64)
    for j in range(n):
        v = y[:, 128 * j:128 * j + 128]
        top = v.abs().amax(1)
        p = torch.ceil(torch.log2(top / 448.0)).clamp(min=-127.0)
        p = torch.where(top <= 448.0 * torch.exp2(p - 1.0), p - 1.0, p).clamp(min=-127.0)  # log2 rounds
        scales[:, j] = torch.exp2(p)
        codes[:, 128 * j:128 * j + 128] = _exact_e4m3(v / scales[:, j:j + 1])
    return {"codes": codes, "scales": scales}


def _exact_operand(codes, b, cols):
    """float64 values of an encoded operand, from the bits of its codes."""
    u = codes[:, :cols].long()
    exp, frac = (u >> 3) & 15, (u & 7).double()
    mag = torch.where(exp == 0, frac * 2.0 ** -9, (8.0 + frac) * torch.exp2(exp.double() - 10.0))
    del exp, frac
    v = torch.where(u >= 128, -mag, mag)
    del u, mag
    for j in range(-(-cols // 128)):
        v[:, 128 * j:128 * j + 128] *= torch.exp2(b[:, j].double() - 127.0).unsqueeze(1)
    return v


def _exact_round(x, bits):
    """What a cache of `bits` bits gives back of float64 rows."""
    out = torch.empty_like(x)
    n, top = GROUP[bits], TOP[bits]
    for c in range(0, x.shape[1], n):
        v = x[:, c:c + n]
        s = (v.abs().amax(1, keepdim=True).float() * (1.0 / top)).bfloat16().double()
        q = torch.where(s > 0, torch.round(v / torch.where(s > 0, s, torch.ones_like(s))), torch.zeros_like(v))
        out[:, c:c + n] = q.clamp(-top, top) * s
    return out


def _exact_pool(x):
    """The pooled codes of one head's rows [n, 128]: the definition fixes the order of its fp32
    sums, the rest is exact."""
    codes, scales = [], []
    for r in range(0, x.shape[0], 128):
        v = x[r:r + 128].float()
        n = v.shape[0]
        v = torch.cat([v, torch.zeros(128 - n, 128, device=DEV)])
        while v.shape[0] > 1:
            half = v.shape[0] // 2
            v = v[:half] + v[half:]
        v = v[0] * torch.reciprocal(torch.tensor(float(n), device=DEV))
        s = v.abs().max() * torch.tensor(1.0 / 127.0, device=DEV)
        codes.append(torch.round(v * torch.reciprocal(s)).clamp(-127, 127) if s > 0 else torch.zeros_like(v))
        scales.append(s)
    return torch.stack(codes).double(), torch.stack(scales)


def _exact_attention(case, s):
    nq, H, group, keep = case["nq"], case["heads"], case["heads"] // case["kv_heads"], case["keep"]
    out = torch.empty(nq, H * 128, device=DEV, dtype=torch.float64)
    for h in range(H):
        c, ck = slice(128 * h, 128 * h + 128), slice(128 * (h // group), 128 * (h // group) + 128)
        k, v = s["k"][:, ck], s["vt"][h // group, :, :case["nk"]].double().T
        (pq, _), (pk, scale) = _exact_pool(s["q"][:, c]), _exact_pool(k)
        score = (pq @ pk.T).float() * scale
        for i, row in enumerate(score):
            best = torch.sort(row, descending=True, stable=True).indices[:keep].tolist()
            at = torch.cat([torch.arange(128 * j, min(128 * j + 128, case["nk"]), device=DEV) for j in best])
            z = s["q"][128 * i:128 * i + 128, c].double() @ k[at].double().T / math.sqrt(128.0)
            out[128 * i:128 * i + 128, c] = torch.softmax(z, 1) @ v[at]
    return {"blocks": None, "o": out}


def exact(case, seed):
    op = case["op"]
    s = _inputs(case, seed)
    if op == "quant":
        return _exact_fp8(s["x"].double())
    if op == "norm":
        x = s["x"].double()
        y = (x - x.mean(1, keepdim=True)) / torch.sqrt(x.var(1, unbiased=False, keepdim=True) + 1e-6)
        return _exact_fp8(y * (1.0 + s["scale"].double()) + s["shift"].double())
    if op == "gemm":
        K = case["K"]
        w = _exact_operand(s["w"], s["sw"], K)
        parts = []
        for r in range(0, case["M"], 4096):
            y = _exact_operand(s["a"][r:r + 4096], s["sa"][r:r + 4096], K) @ w.T
            parts.append(y + s["bias"].double())
        y = torch.cat(parts)
        del w, parts
        if case["out"] == "resid":
            return s["h0"].double() + s["gate"].double() * y
        if case["gelu"]:
            u = math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)
            y = y / (1.0 + torch.exp(-2.0 * u))
        return _exact_fp8(y) if case["out"] == "fp8" else y
    if op == "attn":
        return _exact_attention(case, s)
    bits, cols = case["bits"], case["cols"]
    if op == "cache":
        # the residual is an fp32 tensor by definition
        return s["h_in"].double() + _exact_round((s["h_out"] - s["h_in"]).double(), bits)
    at = s["slots"].long() if s["slots"] is not None else torch.arange(case["rows"], device=DEV)
    codes, scales = s["codes"][at].long(), s["scales"][at].double()
    if bits == 8:
        q = codes[:, :cols]
        q = torch.where(q >= 128, q - 256, q)
    else:
        q = torch.stack([codes % 16, codes // 16], 2).view(case["rows"], -1)[:, :cols]
        q = torch.where(q >= 8, q - 16, q)
    return s["h_in"].double() + q.double() * scales.repeat_interleave(GROUP[bits], 1)[:, :cols]
