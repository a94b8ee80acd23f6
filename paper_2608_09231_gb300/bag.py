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
           "bag_attention_blocks", "bag_operators_status", "bag_check_operator_timeout"]

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
        "bag_operators_status": ([_P], _I),
        "bag_check_operator_timeout": ([_P], _I),
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
        self.stream = 0  # the caller's, as set_stream gave it

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
        self.stream = int(stream or 0)

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
    def operators_status(self):
        """Waits for the context's stream; raises where a wait expired in one of the operators below
        since the last such call (their outputs are invalid then)."""
        self._chk(self.lib.bag_operators_status(self.h))

    def check_operator_timeout(self):
        """bag_check_operator_timeout: a wait that expires, for operators_status to report."""
        self._chk(self.lib.bag_check_operator_timeout(self.h))

    def quant_fp8(self, x, codes, scales):
        """Rows of x (fp32 or bf16 [rows, cols]) as e4m3 codes and power-of-two scales."""
        p, ld, rows, cols, kind = _mat(x, "x", ("float32", "bfloat16"))
        self._chk(self.lib.bag_quant_fp8(self.h, p, int(kind == "bfloat16"), ld, rows, cols,
                                         *_encoded(codes, scales, "codes", rows, cols)))

    def ln_mod_fp8(self, x, shift, scale, codes, scales):
        """ln_mod of fp32 rows, encoded as by quant_fp8."""
        p, ld, rows, cols, _ = _mat(x, "x", ("float32",))
        self._chk(self.lib.bag_ln_mod_fp8(self.h, p, ld, _vec(shift, "shift", cols), _vec(scale, "scale", cols),
                                          rows, cols, *_encoded(codes, scales, "codes", rows, cols)))

    def gemm_fp8(self, a, a_scales, w, w_scales, out, K, bias=None, gelu=False, gate=None, residual=False,
                 out_scales=None, N=None):
        """Product of encoded a [M, K] and w [N, K]: out fp32 or bf16 [M, N]; encoded, where
        out_scales is given; or, with residual, fp32 out += gate * (product + bias).  N: how many
        rows of w (default all)."""
        M, N = a.shape[0], w.shape[0] if N is None else N
        if out_scales is not None:
            kind = FP8_CODES
            o, ldo, os, ldos = _encoded(out, out_scales, "out", M, N)
        else:
            o, ldo, rows, cols, name = _mat(out, "out", ("float32", "bfloat16"))
            os, ldos = None, 0
            kind = FP8_BF16 if name == "bfloat16" else (FP8_RESID if residual else FP8_F32)
            if rows < M or cols < N:
                raise ValueError(f"out: {tuple(out.shape)} does not hold {M} x {N} elements")
        if residual and kind != FP8_RESID:
            raise ValueError("a residual update needs an fp32 out")
        self._chk(self.lib.bag_gemm_fp8(self.h, *_encoded(a, a_scales, "a", M, K), *_encoded(w, w_scales, "w", N, K),
                                        _vec(bias, "bias", N), M, N, K, int(gelu), kind, _vec(gate, "gate", N), o, ldo,
                                        os, ldos))

    @staticmethod
    def _cache(codes, scales, bits, base, slots, rows, cols):
        c, ldc, cap, nc, _ = _mat(codes, "codes")
        s, lds, ns, ng, _ = _mat(scales, "scales", ("bfloat16",))
        if nc * 8 < cols * bits or ng * CACHE_GROUP.get(bits, 128) < cols or cap != ns:
            raise ValueError(f"codes {tuple(codes.shape)} and scales {tuple(scales.shape)} hold no rows of {cols}")
        b, ldb = None, 0
        if base is not None:
            b, ldb, br, bc, _ = _mat(base, "base", ("float32",))
            if br != rows or bc != cols:
                _want(base, "base", f"a matrix of {rows} x {cols}")
        return c, ldc, s, lds, cap, b, ldb, _vec(slots, "slots", rows, "int32")

    def cache_write(self, x, codes, scales, bits, base=None, slots=None):
        """Keep rows of x - base (or of x) in slots of a quantised cache."""
        p, ld, rows, cols, _ = _mat(x, "x", ("float32",))
        c, ldc, s, lds, cap, b, ldb, at = self._cache(codes, scales, bits, base, slots, rows, cols)
        self._chk(self.lib.bag_cache_write(self.h, p, ld, b, ldb, at, rows, cols, bits, c, ldc, s, lds, cap))

    def cache_read(self, codes, scales, out, bits, base=None, slots=None):
        """out = base + the cache's rows (or the rows alone)."""
        p, ld, rows, cols, _ = _mat(out, "out", ("float32",))
        c, ldc, s, lds, cap, b, ldb, at = self._cache(codes, scales, bits, base, slots, rows, cols)
        self._chk(self.lib.bag_cache_read(self.h, c, ldc, s, lds, cap, at, rows, cols, bits, b, ldb, p, ld))

    @staticmethod
    def _pooled(codes, scales):
        if codes.dim() != 3 or codes.shape[2] != 128 or _type(codes)[0] != "int8" or not codes.is_cuda or \
                not codes.is_contiguous():
            _want(codes, "codes", "dense int8 [heads, blocks, 128] on the device")
        heads, blocks = codes.shape[:2]
        if scales.shape != (heads, blocks) or _type(scales)[0] != "float32" or not scales.is_cuda or \
                not scales.is_contiguous():
            _want(scales, "scales", f"dense float32 [{heads}, {blocks}] on the device")
        return codes.data_ptr(), scales.data_ptr(), heads, blocks

    @staticmethod
    def _heads16(x, name, heads, types=("float16", "bfloat16")):
        p, ld, rows, cols, kind = _mat(x, name, types)
        if cols != 128 * heads:
            _want(x, name, f"{heads} heads of 128 columns")
        return p, ld, rows, kind

    def block_pool(self, x, codes, scales):
        """Pooled vectors of the blocks of 128 rows of x [rows, 128 * heads]."""
        c, s, heads, blocks = self._pooled(codes, scales)
        p, ld, rows, kind = self._heads16(x, "x", heads)
        self._chk(self.lib.bag_block_pool(self.h, p, _T16[kind], ld, rows, heads, c, s, blocks))

    @staticmethod
    def _lists(blocks, nq):
        if blocks.dim() != 3 or blocks.shape[1] != (nq + ATTN_BLOCK - 1) // ATTN_BLOCK or not blocks.is_cuda or \
                not blocks.is_contiguous() or _type(blocks)[0] != "int32":
            _want(blocks, "blocks", f"dense int32 [heads, query blocks, keep] for {nq} queries on the device")
        return blocks.data_ptr(), blocks.shape[0], blocks.shape[2]

    def block_select(self, q, codes, scales, blocks, nkb=None):
        """The key blocks (pooled vectors codes, scales; the first nkb of them) of highest score for
        each head and block of queries of q, into blocks [heads, query blocks, keep]."""
        c, s, kv_heads, ldb = self._pooled(codes, scales)
        at, heads, keep = self._lists(blocks, q.shape[0])
        p, ld, nq, kind = self._heads16(q, "q", heads)
        self._chk(self.lib.bag_block_select(self.h, p, _T16[kind], ld, nq, heads, c, s, ldb,
                                            ldb if nkb is None else nkb, kv_heads, keep, at))

    def attention_blocks(self, q, k, vt, o, blocks, heads, kv_heads=None):
        """Attention of q [nq, 128 * heads] over the listed blocks of k [nk, 128 * kv_heads]; vt
        [kv_heads, 128, vpad] of the same type; o bf16 [nq, 128 * heads]."""
        kv_heads = heads if kv_heads is None else kv_heads
        qp, ldq, nq, kind = self._heads16(q, "q", heads)
        kp, ldk, nk, _ = self._heads16(k, "k", kv_heads, (kind,))
        op, ldo, no, _ = self._heads16(o, "o", heads, ("bfloat16",))
        at, lists, keep = self._lists(blocks, nq)
        if vt.dim() != 3 or vt.shape[0] != kv_heads or vt.shape[1] != 128 or _type(vt)[0] != kind or \
                not vt.is_cuda or not vt.is_contiguous():
            _want(vt, "vt", f"dense {kind} [{kv_heads}, 128, vpad] on the device")
        if no != nq or lists != heads:
            raise ValueError(f"o {tuple(o.shape)} or blocks {tuple(blocks.shape)} does not fit {nq} queries of {heads} heads")
        self._chk(self.lib.bag_attention_blocks(self.h, qp, ldq, kp, ldk, vt.data_ptr(), vt.shape[2], _T16[kind], nq, nk,
                                                heads, kv_heads, at, keep, op, ldo))


# --- tensors handed to the low-precision operators ---------------------------------------
# A wrong element type or a row whose elements are not dense would reach the kernels as a
# plausible pointer, so these are checked here; sizes, strides and alignment are checked by the
# library as well.
_TYPES = {}  # dtype -> (name, bytes)


def _type(t):
    d = t.dtype
    r = _TYPES.get(d)
    if r is None:
        r = _TYPES[d] = (str(d).replace("torch.", ""), d.itemsize)
    return r


def _want(t, name, what):
    raise ValueError(f"{name}: {what} is needed, got {tuple(t.shape)} {t.dtype} on {t.device}, strides {t.stride()}")


def _mat(t, name, types=None):
    """(pointer, row stride, rows, columns, type name) of a device matrix with dense rows, of one
    of `types` (None: of one-byte elements)."""
    shape, (kind, size) = t.shape, _type(t)
    if len(shape) != 2 or not t.is_cuda or (size != 1 if types is None else kind not in types):
        _want(t, name, f"a device matrix of {types or 'one-byte elements'}")
    rows, cols = shape
    ld, step = t.stride()
    if step != 1 and cols > 1:
        _want(t, name, "a matrix with dense rows")
    return t.data_ptr(), ld if rows > 1 else max(ld, cols), rows, cols, kind


def _vec(t, name, n, kind="float32"):
    if t is None:
        return None
    if t.shape != (n,) or _type(t)[0] != kind or not t.is_cuda or (n > 1 and t.stride(0) != 1):
        _want(t, name, f"a dense device vector of {n} {kind}")
    return t.data_ptr()


def _encoded(codes, scales, name, rows, cols):
    """Pointers and strides of an encoded matrix [rows, cols]."""
    c, ldc, rc, cc, _ = _mat(codes, name)
    s, lds, rs, cs, _ = _mat(scales, name)
    if rc < rows or cc < cols or rs < rows or cs * SCALE_BLOCK < cols:
        raise ValueError(f"{name}: codes {tuple(codes.shape)} and scales {tuple(scales.shape)} do not hold "
                         f"{rows} x {cols} elements")
    return c, ldc, s, lds


_T16 = {"float16": 2, "bfloat16": 1}  # BAG_F16, BAG_BF16


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
