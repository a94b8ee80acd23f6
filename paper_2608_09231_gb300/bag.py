"""Python binding of the BAG C ABI (include/bag.h): argument marshalling only.

Every computation happens in libbag.so's CUDA kernels; this module converts configs to
the C structs, passes device pointers (torch tensors' data_ptr) and host buffers, and
turns status codes into exceptions.  It never falls back to anything: if the library is
missing or fails to load, load() raises.
"""

import ctypes
import os

import numpy as np

from . import configs as _configs

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbag.so")

KIND = {"single": 0, "mmdit": 1, "wan": 2}
DTYPE = {"f32": 0, "bf16": 1}
GATE_KIND = {"mlp3": 0, "flux6": 1, "wan6": 2}
SAMPLER = {"euler": 0, "unipc": 1}
OBSERVABLE = {"modulated": 0, "embedded": 1}
POLICY_BAG, POLICY_FULL, POLICY_MASK, POLICY_STATIC_UNIFORM, POLICY_THRESHOLD = 0, 1, 2, 3, 4
LOG_FLOATS = 16
# Output kinds of gemm_fp8
FP8_F32, FP8_BF16, FP8_CODES, FP8_RESID = 0, 1, 2, 3
SCALE_BLOCK = 128                  # columns of one scale of an encoded matrix
CACHE_GROUP = {8: 128, 4: 32}      # columns of one scale of a quantised cache, by bits
ATTN_BLOCK = 128                   # rows of a block of queries or keys
STATUS = {0: "BAG_OK", 1: "BAG_EINVAL", 2: "BAG_ENOMEM", 3: "BAG_ECUDA", 4: "BAG_EORDER",
          5: "BAG_EDEVICE_TIMEOUT", 6: "BAG_ESTATE", 7: "BAG_EUNSUPPORTED"}

EXPORTS = ["bag_create", "bag_destroy", "bag_last_error", "bag_set_stream", "bag_load_gate",
           "bag_set_policy", "bag_set_budget", "bag_reset", "bag_step", "bag_run", "bag_run_host",
           "bag_get_weight", "bag_forward_block", "bag_prepare", "bag_launch_count",
           "bag_gemm_bf16", "bag_attention_bf16", "bag_attention_f16", "bag_ln_mod", "bag_residual_add",
           "bag_profile_run", "bag_profile_launches", "bag_rel_l1", "bag_rel_l1_noalloc",
           "bag_check_wait_timeout", "bag_quant_fp8", "bag_ln_mod_fp8", "bag_gemm_fp8",
           "bag_cache_write", "bag_cache_read", "bag_block_pool", "bag_block_select",
           "bag_attention_blocks"]

PROF_KINDS = ["gemm", "attention", "norm", "signal", "gate", "cache"]


class BagError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status


class Arch(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int), ("hidden", ctypes.c_int), ("heads", ctypes.c_int),
                ("mlp", ctypes.c_int), ("n_double", ctypes.c_int), ("n_single", ctypes.c_int),
                ("n_wan", ctypes.c_int), ("grid", ctypes.c_int * 3), ("n_txt", ctypes.c_int),
                ("patch_ch", ctypes.c_int), ("rope_axes", ctypes.c_int * 3),
                ("dtype", ctypes.c_int), ("weight_seed", ctypes.c_uint64),
                ("gate_seed", ctypes.c_uint64), ("tau", ctypes.c_float),
                ("gate_kind", ctypes.c_int), ("cfg", ctypes.c_int), ("guidance", ctypes.c_float),
                ("qk_norm", ctypes.c_int), ("sampler", ctypes.c_int), ("shift", ctypes.c_float),
                ("observable", ctypes.c_int)]


class Cond(ctypes.Structure):
    _fields_ = [("txt", ctypes.c_void_p), ("pooled", ctypes.c_void_p),
                ("txt_uncond", ctypes.c_void_p), ("pooled_uncond", ctypes.c_void_p)]


class ProfEntry(ctypes.Structure):
    _fields_ = [("launches", ctypes.c_long), ("ms", ctypes.c_double), ("flops", ctypes.c_double),
                ("bytes", ctypes.c_double)]


class ProfLaunch(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int), ("m", ctypes.c_int), ("n", ctypes.c_int),
                ("k", ctypes.c_int), ("ms", ctypes.c_float), ("flops", ctypes.c_double),
                ("bytes", ctypes.c_double), ("variant", ctypes.c_int)]


class Stats(ctypes.Structure):
    _fields_ = [("mask", ctypes.POINTER(ctypes.c_uint8)), ("log", ctypes.POINTER(ctypes.c_float)),
                ("nfe", ctypes.c_int), ("T", ctypes.c_int), ("B", ctypes.c_int)]


_lib = None

_P = ctypes.c_void_p
_I = ctypes.c_int
_L = ctypes.c_long


def load(path=None):
    """Load libbag.so (raises if it is missing; no fallback path exists)."""
    global _lib
    if _lib is not None:
        return _lib
    path = path or LIB_PATH
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with __graft_entry__.build()")
    lib = ctypes.CDLL(path)
    sig = {
        "bag_create": ([ctypes.POINTER(Arch), _I, _I, ctypes.POINTER(_P)], _I),
        "bag_destroy": ([_P], None),
        "bag_last_error": ([_P], ctypes.c_char_p),
        "bag_set_stream": ([_P, _P], _I),
        "bag_load_gate": ([_P, _P, _I, _P, _P], _I),
        "bag_set_policy": ([_P, _I, _P, ctypes.c_float], _I),
        "bag_set_budget": ([_P, _I], _I),
        "bag_check_wait_timeout": ([_P], _I),
        "bag_reset": ([_P], _I),
        "bag_step": ([_P, _P, _I, ctypes.POINTER(Cond), _P, _P], _I),
        "bag_run": ([_P, _P, ctypes.POINTER(Cond), ctypes.POINTER(Stats)], _I),
        "bag_run_host": ([_P, _P, ctypes.POINTER(Cond), ctypes.POINTER(Stats)], _I),
        "bag_get_weight": ([_P, _I, ctypes.c_char_p, _P, ctypes.c_size_t], _I),
        "bag_forward_block": ([_P, _I, _I, _P], _I),
        "bag_prepare": ([_P, ctypes.POINTER(Cond)], _I),
        "bag_launch_count": ([_P, ctypes.POINTER(_L)], _I),
        "bag_gemm_bf16": ([_P, _P, _L, _P, _L, _P, _P, _L, _I, _I, _I, _I, _I], _I),
        "bag_attention_bf16": ([_P, _P, _P, _P, _P, _L, _I, _I, _I, _I, _L, _I], _I),
        "bag_attention_f16": ([_P, _P, _P, _P, _P, _L, _I, _I, _I, _I, _L], _I),
        "bag_ln_mod": ([_P, _P, _P, _P, _P, _I, _I], _I),
        "bag_residual_add": ([_P, _P, _P, _P, _L], _I),
        "bag_quant_fp8": ([_P, _P, _I, _L, _L, _L, _P, _L, _P, _L], _I),
        "bag_ln_mod_fp8": ([_P, _P, _L, _P, _P, _L, _L, _P, _L, _P, _L], _I),
        "bag_gemm_fp8": ([_P, _P, _L, _P, _L, _P, _L, _P, _L, _P, _L, _L, _L, _I, _I, _P, _P, _L,
                          _P, _L], _I),
        "bag_cache_write": ([_P, _P, _L, _P, _L, _P, _L, _L, _I, _P, _L, _P, _L, _L], _I),
        "bag_cache_read": ([_P, _P, _L, _P, _L, _L, _P, _L, _L, _I, _P, _L, _P, _L], _I),
        "bag_block_pool": ([_P, _P, _I, _L, _L, _I, _P, _P, _L], _I),
        "bag_block_select": ([_P, _P, _I, _L, _L, _I, _P, _P, _L, _L, _I, _I, _P], _I),
        "bag_attention_blocks": ([_P, _P, _L, _P, _L, _P, _L, _I, _L, _L, _I, _I, _P, _I, _P, _L], _I),
        "bag_rel_l1": ([_P, _P, _P, _I, _L, _L, _P, _P], _I),
        "bag_rel_l1_noalloc": ([_P, _P, _I, _L, _L, _P, _P], _I),
        "bag_profile_run": ([_P, _P, ctypes.POINTER(Cond), ctypes.POINTER(Stats),
                             ctypes.POINTER(ProfEntry)], _I),
        "bag_profile_launches": ([_P, ctypes.POINTER(ProfLaunch), _L, ctypes.POINTER(_L)], _I),
    }
    for name, (args, res) in sig.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = res
    _lib = lib
    return lib


def arch_from_config(cfg, tau=0.5):
    a = Arch()
    a.kind = KIND[cfg["kind"]]
    a.hidden, a.heads, a.mlp = cfg["hidden"], cfg["heads"], cfg["mlp"]
    a.n_double, a.n_single, a.n_wan = cfg["n_double"], cfg["n_single"], cfg["n_wan"]
    a.grid[:] = list(cfg["grid"])
    a.n_txt, a.patch_ch = cfg["n_txt"], cfg["patch_ch"]
    a.rope_axes[:] = list(cfg["rope_axes"])
    a.dtype = DTYPE[cfg["dtype"]]
    a.weight_seed, a.gate_seed = cfg["weight_seed"], cfg["gate_seed"]
    a.tau = tau
    a.gate_kind = GATE_KIND[cfg.get("gate_kind", "mlp3")]
    g = cfg.get("guidance")
    a.cfg = 0 if g is None else 1
    a.guidance = 0.0 if g is None else float(g)
    a.qk_norm = 1 if cfg.get("qk_norm") else 0
    a.sampler = SAMPLER[cfg.get("sampler", "euler")]
    a.shift = float(cfg.get("shift", 1.0))
    a.observable = OBSERVABLE[cfg.get("observable", "modulated")]
    return a


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _dp(t):
    return None if t is None else t.data_ptr()


def _cond(txt, pooled, txt_u=None, pooled_u=None):
    """Device conditioning (torch tensors; the *_u pair is the unconditional branch of
    a guided context)."""
    return Cond(_dp(txt), _dp(pooled), _dp(txt_u), _dp(pooled_u))


class Context:
    """A bag_ctx: one model instance, one sample at a time (bag_create ... bag_destroy)."""

    def __init__(self, cfg, T=None, B=None, tau=0.5):
        self.lib = load()
        self.cfg = cfg
        self.T = cfg["T"] if T is None else T
        self.B = cfg["budgets"][0] if B is None else B
        self._arch = arch_from_config(cfg, tau)
        h = ctypes.c_void_p()
        st = self.lib.bag_create(ctypes.byref(self._arch), self.T, self.B, ctypes.byref(h))
        if st != 0:
            raise BagError(st, self.lib.bag_last_error(None).decode())
        self.h = h

    def _chk(self, st):
        if st != 0:
            raise BagError(st, self.lib.bag_last_error(self.h).decode())

    def close(self):
        if getattr(self, "h", None):
            self.lib.bag_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # --- API mirror -----------------------------------------------------------------
    def set_stream(self, stream):
        self._chk(self.lib.bag_set_stream(self.h, ctypes.c_void_p(stream)))

    def load_gate(self, theta, mu=None, sd=None):
        th = np.ascontiguousarray(theta, np.float32)
        mu_a = None if mu is None else np.ascontiguousarray(mu, np.float32)
        sd_a = None if sd is None else np.ascontiguousarray(sd, np.float32)
        self._chk(self.lib.bag_load_gate(self.h, th.ctypes.data, th.size,
                                         None if mu_a is None else mu_a.ctypes.data,
                                         None if sd_a is None else sd_a.ctypes.data))

    def set_policy(self, policy, mask=None, delta=0.0):
        m = None if mask is None else np.ascontiguousarray(mask, np.uint8)
        self._chk(self.lib.bag_set_policy(self.h, policy, None if m is None else m.ctypes.data,
                                          float(delta)))

    def set_budget(self, B):
        """Budget of later samples (the step graph is re-captured on the next run)."""
        self._chk(self.lib.bag_set_budget(self.h, int(B)))
        self.B = int(B)

    def reset(self):
        self._chk(self.lib.bag_reset(self.h))

    def check_wait_timeout(self):
        """bag_check_wait_timeout: returns the status (BAG_EDEVICE_TIMEOUT expected)."""
        return self.lib.bag_check_wait_timeout(self.h)

    def prepare(self, txt, pooled, txt_u=None, pooled_u=None):
        c = _cond(txt, pooled, txt_u, pooled_u)
        self._chk(self.lib.bag_prepare(self.h, ctypes.byref(c)))

    def step(self, x, t, txt, pooled, x_out, flag=None, txt_u=None, pooled_u=None):
        c = _cond(txt, pooled, txt_u, pooled_u)
        self._chk(self.lib.bag_step(self.h, _ptr(x), t, ctypes.byref(c), _ptr(x_out), _ptr(flag)))

    def _stats(self):
        mask = np.zeros(self.T, np.uint8)
        log = np.zeros((self.T, LOG_FLOATS), np.float32)
        s = Stats(mask.ctypes.data_as(ctypes.POINTER(ctypes.c_uint8)),
                  log.ctypes.data_as(ctypes.POINTER(ctypes.c_float)), 0, 0, 0)
        return s, mask, log

    def run(self, x, txt, pooled, txt_u=None, pooled_u=None):
        """All T steps in place on device tensor x; returns (mask, log, nfe)."""
        c = _cond(txt, pooled, txt_u, pooled_u)
        s, mask, log = self._stats()
        self._chk(self.lib.bag_run(self.h, _ptr(x), ctypes.byref(c), ctypes.byref(s)))
        return mask, log, s.nfe

    def profile_run(self, x, txt, pooled, txt_u=None, pooled_u=None):
        """Profiled sample (direct launches with events); returns (mask, log, nfe, prof)
        where prof maps a kernel class to dict(launches, ms, flops, bytes)."""
        c = _cond(txt, pooled, txt_u, pooled_u)
        s, mask, log = self._stats()
        out = (ProfEntry * len(PROF_KINDS))()
        self._chk(self.lib.bag_profile_run(self.h, _ptr(x), ctypes.byref(c), ctypes.byref(s), out))
        prof = {k: dict(launches=out[i].launches, ms=out[i].ms, flops=out[i].flops,
                        bytes=out[i].bytes) for i, k in enumerate(PROF_KINDS)}
        return mask, log, s.nfe, prof

    def profile_launches(self):
        """Per-launch records of the last profile_run as a list of dicts."""
        n = ctypes.c_long()
        self._chk(self.lib.bag_profile_launches(self.h, None, 0, ctypes.byref(n)))
        arr = (ProfLaunch * max(1, n.value))()
        self._chk(self.lib.bag_profile_launches(self.h, arr, n.value, ctypes.byref(n)))
        return [dict(kind=PROF_KINDS[r.kind], m=r.m, n=r.n, k=r.k, ms=r.ms, flops=r.flops,
                     bytes=r.bytes, variant=r.variant) for r in arr[:n.value]]

    def run_host(self, x, txt, pooled, txt_u=None, pooled_u=None):
        """All T steps with host numpy buffers (x updated in place); returns (mask, log, nfe)."""
        assert x.dtype == np.float32 and x.flags.c_contiguous
        keep = [None if a is None else np.ascontiguousarray(a, np.float32)
                for a in (txt, pooled, txt_u, pooled_u)]
        c = Cond(*[None if a is None else a.ctypes.data for a in keep])
        s, mask, log = self._stats()
        self._chk(self.lib.bag_run_host(self.h, x.ctypes.data, ctypes.byref(c), ctypes.byref(s)))
        return mask, log, s.nfe

    def get_weight(self, block, name, n):
        out = np.empty(n, np.float32)
        self._chk(self.lib.bag_get_weight(self.h, block, name.encode(), out.ctypes.data, n))
        return out

    def forward_block(self, block, t_mod, h):
        self._chk(self.lib.bag_forward_block(self.h, block, t_mod, _ptr(h)))

    def launch_count(self):
        n = ctypes.c_long()
        self._chk(self.lib.bag_launch_count(self.h, ctypes.byref(n)))
        return n.value

    def gemm_bf16(self, A, W, bias, C, M, N, K, epilogue=0, force_simt=0):
        self._chk(self.lib.bag_gemm_bf16(self.h, _ptr(A), A.stride(0), _ptr(W), W.stride(0),
                                         _ptr(bias), _ptr(C), C.stride(0), M, N, K, epilogue,
                                         force_simt))

    def attention_bf16(self, q, k, v, o, nq, nk, heads, dh, vpad=0, force_simt=0):
        """v: [nk, ld] when vpad == 0, else transposed per head [heads, dh, vpad]."""
        self._chk(self.lib.bag_attention_bf16(self.h, _ptr(q), _ptr(k), _ptr(v), _ptr(o),
                                              q.stride(0), nq, nk, heads, dh, vpad, force_simt))

    def attention_f16(self, q, k, v, o, nq, nk, heads, dh, vpad):
        """fp16 q, k and v (v transposed per head, [heads, dh, vpad]); bf16 output."""
        self._chk(self.lib.bag_attention_f16(self.h, _ptr(q), _ptr(k), _ptr(v), _ptr(o),
                                             q.stride(0), nq, nk, heads, dh, vpad))

    def ln_mod(self, x, shift, scale, y, rows, cols):
        self._chk(self.lib.bag_ln_mod(self.h, _ptr(x), _ptr(shift), _ptr(scale), _ptr(y), rows,
                                      cols))

    def rel_l1(self, a, b, rows, cols, scratch, out, bf16=None):
        dt = (1 if a.dtype.itemsize == 2 else 0) if bf16 is None else int(bf16)
        self._chk(self.lib.bag_rel_l1(self.h, _ptr(a), _ptr(b), dt, rows, cols, _ptr(scratch),
                                      _ptr(out)))

    def residual_add(self, out, h_in, R, n):
        self._chk(self.lib.bag_residual_add(self.h, _ptr(out), _ptr(h_in), _ptr(R), n))

    # --- 8-bit operands, quantised cache, block-sparse attention (see include/bag.h) ----
    def quant_fp8(self, x, codes, scales):
        """Rows of x (fp32 or bf16 [rows, cols]) as e4m3 codes and power-of-two scales."""
        _rows(x, "x", _itemsize(_is(x, "x", "float32", "bfloat16")))
        rows, cols = x.shape
        self._chk(self.lib.bag_quant_fp8(self.h, _ptr(x), int(_itemsize(x) == 2), _ld(x), rows, cols,
                                         *_encoded(codes, scales, "codes", rows, cols)))

    def ln_mod_fp8(self, x, shift, scale, codes, scales):
        """ln_mod of fp32 rows, encoded as by quant_fp8."""
        _rows(_is(x, "x", "float32"), "x", 4)
        rows, cols = x.shape
        self._chk(self.lib.bag_ln_mod_fp8(self.h, _ptr(x), _ld(x), _vector(shift, "shift", cols),
                                          _vector(scale, "scale", cols), rows, cols,
                                          *_encoded(codes, scales, "codes", rows, cols)))

    def gemm_fp8(self, a, a_scales, w, w_scales, out, K, bias=None, gelu=False, gate=None, residual=False,
                 out_scales=None, N=None):
        """Product of encoded a [M, K] and w [N, K]: out fp32 or bf16 [M, N]; encoded, where
        out_scales is given (N then says how many columns, default w's rows); or, with residual,
        fp32 out += gate * (product + bias)."""
        M, N = a.shape[0], w.shape[0] if N is None else N
        if out_scales is not None:
            kind = FP8_CODES
            o, ldo, os, ldos = _encoded(out, out_scales, "out", M, N)
        else:
            _rows(_is(out, "out", "float32", "bfloat16"), "out", _itemsize(out))
            if out.shape[0] < M or out.shape[1] < N:
                raise ValueError(f"out: {tuple(out.shape)} does not hold {M} x {N} elements")
            kind = FP8_BF16 if _itemsize(out) == 2 else (FP8_RESID if residual else FP8_F32)
            o, ldo, os, ldos = _ptr(out), _ld(out), None, 0
        if residual and kind != FP8_RESID:
            raise ValueError("a residual update needs an fp32 out")
        self._chk(self.lib.bag_gemm_fp8(self.h, *_encoded(a, a_scales, "a", M, K), *_encoded(w, w_scales, "w", N, K),
                                        _vector(bias, "bias", N), M, N, K, int(gelu), kind,
                                        _vector(gate, "gate", N), o, ldo, os, ldos))

    def _cache(self, codes, scales, bits, base, slots, rows, cols):
        group = CACHE_GROUP.get(bits, 128)
        _rows(codes, "codes", 1)
        _rows(_is(scales, "scales", "bfloat16"), "scales", 2)
        if codes.shape[1] * 8 < cols * bits or scales.shape[1] * group < cols or codes.shape[0] != scales.shape[0]:
            raise ValueError(f"codes {tuple(codes.shape)} and scales {tuple(scales.shape)} hold no rows of {cols}")
        if base is not None:
            _rows(_is(base, "base", "float32"), "base", 4)
            if tuple(base.shape) != (rows, cols):
                raise ValueError(f"base: {rows} x {cols} elements are needed, got {tuple(base.shape)}")
        if slots is not None:
            _is(slots, "slots", "int32")
            if not slots.is_cuda or slots.dim() != 1 or slots.shape[0] != rows or (rows > 1 and slots.stride(0) != 1):
                raise ValueError(f"slots: {rows} dense int32 on the device are needed, got {tuple(slots.shape)}")
        return _ptr(base), 0 if base is None else _ld(base), _ptr(slots)

    def cache_write(self, x, codes, scales, bits, base=None, slots=None):
        """Keep rows of x - base (or of x) in slots of a quantised cache."""
        _rows(_is(x, "x", "float32"), "x", 4)
        rows, cols = x.shape
        b, ldb, s = self._cache(codes, scales, bits, base, slots, rows, cols)
        self._chk(self.lib.bag_cache_write(self.h, _ptr(x), _ld(x), b, ldb, s, rows, cols, bits, _ptr(codes),
                                           _ld(codes), _ptr(scales), _ld(scales), codes.shape[0]))

    def cache_read(self, codes, scales, out, bits, base=None, slots=None):
        """out = base + the cache's rows (or the rows alone)."""
        _rows(_is(out, "out", "float32"), "out", 4)
        rows, cols = out.shape
        b, ldb, s = self._cache(codes, scales, bits, base, slots, rows, cols)
        self._chk(self.lib.bag_cache_read(self.h, _ptr(codes), _ld(codes), _ptr(scales), _ld(scales), codes.shape[0],
                                          s, rows, cols, bits, b, ldb, _ptr(out), _ld(out)))

    def _pooled(self, codes, scales):
        _is(_rows(codes, "codes", 1, 3), "codes", "int8")
        _is(scales, "scales", "float32")
        heads, blocks = codes.shape[:2]
        if (codes.shape[2] != 128 or tuple(scales.shape) != (heads, blocks) or not scales.is_cuda
                or not codes.is_contiguous() or not scales.is_contiguous()):
            raise ValueError("pooled vectors: dense int8 [heads, blocks, 128] and fp32 [heads, blocks] are needed, got "
                             f"{tuple(codes.shape)} and {tuple(scales.shape)}")
        return heads, blocks

    def block_pool(self, x, codes, scales):
        """Pooled vectors of the blocks of 128 rows of x [rows, 128 * heads]."""
        _rows(_is(x, "x", "float16", "bfloat16"), "x", 2)
        heads, blocks = self._pooled(codes, scales)
        if x.shape[1] != 128 * heads:
            raise ValueError(f"x: {heads} heads of 128 columns are needed, got {tuple(x.shape)}")
        self._chk(self.lib.bag_block_pool(self.h, _ptr(x), _type16(x), _ld(x), x.shape[0], heads, _ptr(codes),
                                          _ptr(scales), blocks))

    def _lists(self, blocks, nq):
        if not blocks.is_cuda or blocks.dim() != 3 or not blocks.is_contiguous() or \
                blocks.shape[1] != (nq + ATTN_BLOCK - 1) // ATTN_BLOCK:
            raise ValueError("blocks: dense int32 [heads, query blocks, keep] is needed, got "
                             f"{tuple(blocks.shape)} for {nq} queries")
        _is(blocks, "blocks", "int32")
        return blocks.shape[0], blocks.shape[2]

    def block_select(self, q, codes, scales, blocks, nkb=None):
        """The key blocks (pooled vectors codes, scales; the first nkb of them) of highest score for
        each head and block of queries of q, into blocks [heads, query blocks, keep]."""
        _rows(_is(q, "q", "float16", "bfloat16"), "q", 2)
        kv_heads, ldb = self._pooled(codes, scales)
        heads, keep = self._lists(blocks, q.shape[0])
        if q.shape[1] != 128 * heads:
            raise ValueError(f"q: {heads} heads of 128 columns are needed, got {tuple(q.shape)}")
        if nkb is not None and nkb > ldb:
            raise ValueError(f"nkb: the pooled vectors are {ldb} blocks, not {nkb}")
        self._chk(self.lib.bag_block_select(self.h, _ptr(q), _type16(q), _ld(q), q.shape[0], heads, _ptr(codes),
                                            _ptr(scales), ldb, ldb if nkb is None else nkb, kv_heads, keep,
                                            _ptr(blocks)))

    def attention_blocks(self, q, k, vt, o, blocks, heads, kv_heads=None):
        """Attention of q [nq, 128 * heads] over the listed blocks of k [nk, 128 * kv_heads]; vt
        [kv_heads, 128, vpad] of the same type; o bf16 [nq, 128 * heads]."""
        kv_heads = heads if kv_heads is None else kv_heads
        _rows(_is(q, "q", "float16", "bfloat16"), "q", 2)
        _rows(_is(k, "k", _name(q)), "k", 2)
        _rows(_is(o, "o", "bfloat16"), "o", 2)
        _rows(_is(vt, "vt", _name(q)), "vt", 2, 3)
        lists, keep = self._lists(blocks, q.shape[0])
        if lists != heads or q.shape[1] != 128 * heads or k.shape[1] != 128 * kv_heads or \
                tuple(o.shape) != tuple(q.shape) or tuple(vt.shape[:2]) != (kv_heads, 128) or not vt.is_contiguous():
            raise ValueError(f"{heads} heads over {kv_heads}: q {tuple(q.shape)}, k {tuple(k.shape)}, vt "
                             f"{tuple(vt.shape)}, o {tuple(o.shape)}, blocks {tuple(blocks.shape)} do not fit")
        self._chk(self.lib.bag_attention_blocks(self.h, _ptr(q), _ld(q), _ptr(k), _ld(k), _ptr(vt), vt.shape[2],
                                                _type16(q), q.shape[0], k.shape[0], heads, kv_heads, _ptr(blocks),
                                                keep, _ptr(o), _ld(o)))


# --- shapes and types of tensors handed to the low-precision operators -------------------
# Checked here, because a wrong stride or element type would reach the kernels as a plausible
# pointer; sizes, alignment and everything else are checked by the library.
def _itemsize(t):
    return t.dtype.itemsize


def _rows(t, name, size, dims=2):
    """A device tensor whose last dimension is dense and whose elements have `size` bytes."""
    if not t.is_cuda or t.dim() != dims or _itemsize(t) != size or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError(f"{name}: a {dims}-dimensional device tensor of {size}-byte elements with dense rows is "
                         f"needed, got {tuple(t.shape)} {t.dtype} strides {t.stride()}")
    return t


def _ld(t):
    """Row stride (of one row: its length)."""
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _name(t):
    return str(t.dtype).replace("torch.", "")


def _is(t, name, *types):
    if _name(t) not in types:
        raise ValueError(f"{name}: {' or '.join(types)} is needed, got {t.dtype}")
    return t


def _type16(t):
    return 2 if _name(t) == "float16" else DTYPE["bf16"]


def _vector(t, name, n):
    if t is None:
        return None
    _is(t, name, "float32")
    if not t.is_cuda or t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{name}: {n} dense floats on the device are needed, got {tuple(t.shape)}")
    return _ptr(t)


def _encoded(codes, scales, name, rows, cols):
    """Pointers and strides of an encoded matrix [rows, cols]."""
    _rows(codes, name, 1)
    _rows(scales, name + " scales", 1)
    blocks = (cols + SCALE_BLOCK - 1) // SCALE_BLOCK
    if codes.shape[0] < rows or codes.shape[1] < cols or scales.shape[0] < rows or scales.shape[1] < blocks:
        raise ValueError(f"{name}: codes {tuple(codes.shape)} and scales {tuple(scales.shape)} do not hold "
                         f"{rows} x {cols} elements")
    return _ptr(codes), _ld(codes), _ptr(scales), _ld(scales)


def rel_l1_noalloc(a, b, rows, cols, out, stream=0, bf16=None):
    """bag_rel_l1_noalloc: the signal reduction with no context and no allocation
    (scratch in a fixed device array of the library; see include/bag.h)."""
    lib = load()
    dt = (1 if a.dtype.itemsize == 2 else 0) if bf16 is None else int(bf16)
    st = lib.bag_rel_l1_noalloc(_ptr(a), _ptr(b), dt, rows, cols, _ptr(out),
                                ctypes.c_void_p(stream))
    if st != 0:
        raise BagError(st, lib.bag_last_error(None).decode())


def create(cfg_or_name, T=None, B=None, tau=0.5, **overrides):
    cfg = (_configs.get_config(cfg_or_name, **overrides) if isinstance(cfg_or_name, str)
           else cfg_or_name)
    return Context(cfg, T=T, B=B, tau=tau)
