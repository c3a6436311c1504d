"""DC-Leap denoise step on one GB300: Python binding of libdcleap.so.

Argument marshalling only: every step of the decoding path runs in the CUDA
kernels of ``libdcleap.so`` (built in-tree by ``paper_2607_20467_gb300.build``).
There is no CPU fallback: if the library is missing, ``lib()`` raises.

Two layers:
* ``lib()`` - the raw ctypes functions, under their C names (``dcl_create``, ...);
* ``Context`` - a thin object over one ``dcl_ctx*`` whose methods take torch
  tensors (device buffers) or numpy arrays (host buffers) and raise ``DcleapError``
  on a non-zero status.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdcleap.so")

DCL_TILE_PAIR = 2
DCL_KV_BF16, DCL_KV_FP8, DCL_KV_Q4 = 0, 1, 4
DCL_KV_EXP_MIN = -64
DCL_OK, DCL_ERR_INVALID_ARG, DCL_ERR_STATE, DCL_ERR_OOM, DCL_ERR_CUDA, DCL_ERR_TIMEOUT, \
    DCL_ERR_UNSUPPORTED = range(7)
STATUS_NAMES = ["OK", "INVALID_ARG", "STATE", "OOM", "CUDA", "TIMEOUT", "UNSUPPORTED"]

(DCL_W_EMBED, DCL_W_ATTN_NORM, DCL_W_Q, DCL_W_K, DCL_W_V, DCL_W_O, DCL_W_MLP_NORM, DCL_W_GATE,
 DCL_W_UP, DCL_W_DOWN, DCL_W_FINAL_NORM, DCL_W_LM_HEAD) = range(12)

KERNEL_KINDS = ["embed", "rmsnorm", "gemm_qkv", "attention", "gemm_o", "gemm_gateup",
                "gemm_down", "gemm_lmhead", "combine", "dcv", "v_transpose", "row_plan", "gemm_mlp"]


class ModelConfig(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("ffn_dim", ctypes.c_int32),
                ("vocab", ctypes.c_int32), ("mask_id", ctypes.c_int32),
                ("rope_theta", ctypes.c_float), ("rms_eps", ctypes.c_float)]


class DecodeConfig(ctypes.Structure):
    _fields_ = [("tau_commit", ctypes.c_float), ("tau_draft", ctypes.c_float),
                ("max_window", ctypes.c_int32), ("block_len", ctypes.c_int32),
                ("gen_len", ctypes.c_int32), ("kv_cache", ctypes.c_int32),
                ("min_commit", ctypes.c_int32), ("contiguous_drafts", ctypes.c_int32),
                ("confidence", ctypes.c_int32), ("acceptance", ctypes.c_int32)]


class Stats(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_int64), ("tokens", ctypes.c_int64),
                ("elapsed_ms", ctypes.c_double), ("done", ctypes.c_int32),
                ("jpde_bound", ctypes.c_double)]


class Allocator(ctypes.Structure):
    _fields_ = [("alloc", ctypes.c_void_p), ("free", ctypes.c_void_p), ("user", ctypes.c_void_p)]


class KvCacheDesc(ctypes.Structure):
    _fields_ = [("n_pages", ctypes.c_int32), ("page_len", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("format", ctypes.c_int32), ("k_dev", ctypes.c_void_p),
                ("v_dev", ctypes.c_void_p), ("k_exp_dev", ctypes.c_void_p), ("v_exp_dev", ctypes.c_void_p)]


class KvPagesDesc(ctypes.Structure):
    _fields_ = [("n_pages", ctypes.c_int32), ("page_len", ctypes.c_int32), ("batch", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("table_dev", ctypes.c_void_p), ("held_dev", ctypes.c_void_p),
                ("free_dev", ctypes.c_void_p), ("n_free_dev", ctypes.c_void_p)]


_P = ctypes.c_void_p
_I = ctypes.c_int32
_L = ctypes.c_int64
_F = ctypes.c_float
# name: (restype, argtypes)
SIGNATURES = {
    "dcl_create": (_I, [ctypes.POINTER(ModelConfig), _I, _I, _P, ctypes.POINTER(Allocator),
                        ctypes.POINTER(_P)]),
    "dcl_set_weight": (_I, [_P, _I, _I, _P, _I]),
    "dcl_init_random_weights": (_I, [_P, ctypes.c_uint64, _F, _F, _F]),
    "dcl_set_prompt": (_I, [_P, _I, _P, _I, ctypes.POINTER(DecodeConfig)]),
    "dcl_step": (_I, [_P, _P]),
    "dcl_generate": (_I, [_P, _I, _P, ctypes.POINTER(Stats)]),
    "dcl_restart": (_I, [_P]),
    "dcl_get_state": (_I, [_P, _P, _P]),
    "dcl_set_state": (_I, [_P, _P, _P]),
    "dcl_forward_debug": (_I, [_P, _P, _P, _P, _P, _P, _P]),
    "dcl_debug_hidden": (_I, [_P, _I, _P]),
    "dcl_forward_debug_from": (_I, [_P, _I, _P, _I, _P, _P, _P, _P, _P, _P]),
    "dcl_launch_floor": (_I, [_P, _I, _I, ctypes.POINTER(ctypes.c_float)]),
    "dcl_accept": (_I, [_P, _P, _I, _I, _I, _P, _P, ctypes.POINTER(DecodeConfig), _P]),
    "dcl_accept_noalloc": (_I, [_P, _I, _I, _I, _P, _P, ctypes.POINTER(DecodeConfig), _P, _P]),
    "dcl_fp8_quantise": (_I, [_P, ctypes.c_int64, ctypes.c_int64, _P, _P]),
    "dcl_kv_write": (_I, [_P, _P, _P, _P, _L, _P, _I]),
    "dcl_kv_read": (_I, [_P, _P, _P, _I, _P, _P, _L]),
    "dcl_kv_attention": (_I, [_P, _P, _P, _L, _P, _P, _I, _P, _I, _I, _I, _I, _I, _F, _P, _P]),
    "dcl_kv_plan": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _I]),
    "dcl_qk_norm_rope": (_I, [_P, _P, _L, _P, _L, _P, _I, _I, _I, _I, _I, _F, _P, _P, _F, _P, _L, _P, _L]),
    "dcl_sample": (_I, [_P, _P, _L, _P, _L, _I, _I, _P, _P, _P, _P, _P, _P, _P]),
    "dcl_synchronise": (_I, [_P]),
    "dcl_op_rmsnorm": (_I, [_P, _P, _P, _P, _I, _I, _F]),
    "dcl_op_linear": (_I, [_P, _P, _P, _P, _I, _I, _I, _I, _I]),
    "dcl_op_attention": (_I, [_P, _P, _P, _I, _I, _I, _I, _I, _I]),
    "dcl_op_lmhead_top2": (_I, [_P, _P, _P, _I, _I, _I, _P, _P, _P, _P, _I]),
    "dcl_op_generate": (_I, [_P, _P, ctypes.c_uint64, _I, ctypes.c_int64, ctypes.c_int64, _F, _F]),
    "dcl_selftest_wait_timeout": (_I, [_P, _I]),
    "dcl_set_profiling": (_I, [_P, _I]),
    "dcl_profile_last_step": (_I, [_P, _P, _P, _I, _P]),
    "dcl_last_error": (ctypes.c_char_p, [_P]),
    "dcl_destroy": (None, [_P]),
}

_lib = None


def lib():
    """The loaded libdcleap.so with typed functions (raises if it was not built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with "
                              "`python -m paper_2607_20467_gb300.build` (no CPU fallback exists)")
        handle = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


def __getattr__(name):  # module-level access to the raw C functions: dcl_step, ...
    if name in SIGNATURES:
        return getattr(lib(), name)
    raise AttributeError(name)


class DcleapError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"{STATUS_NAMES[status] if 0 <= status < 7 else status}: {message}")
        self.status = status


def _ptr(t):
    """Device pointer of a torch tensor / host pointer of a numpy array / None."""
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        if not t.flags["C_CONTIGUOUS"]:
            raise ValueError("host array must be C-contiguous")
        return t.ctypes.data
    if hasattr(t, "data_ptr"):
        if not t.is_contiguous():
            raise ValueError("tensor must be contiguous")
        return t.data_ptr()
    if isinstance(t, int):
        return t
    raise TypeError(f"cannot pass {type(t)} as a pointer")


def _dev(t, name, itemsize, count=0):
    """Device pointer for a ``*_dev`` argument: a contiguous CUDA tensor of ``itemsize``-byte
    elements holding at least ``count`` of them (None passes as NULL, an int as a raw device
    address).  A host array, a CPU tensor, another element size or a short buffer is
    refused here, before a kernel could read or write past it."""
    if t is None or isinstance(t, int):
        return t
    if not getattr(t, "is_cuda", False):
        raise ValueError(f"{name}: a device buffer (a CUDA tensor) is required")
    if t.element_size() != itemsize:
        raise TypeError(f"{name}: elements of {itemsize} bytes expected, got {t.dtype}")
    if t.numel() < count:
        raise ValueError(f"{name}: at least {count} elements needed, {t.numel()} given")
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return t.data_ptr()


# What a buffer of each kind holds: bytes of an element, and the torch types it may have (bit patterns of the
# kind's size among them).  A type of another meaning is refused: its bits would be read as this one's.
_KINDS = {"bf16": (2, ("torch.bfloat16", "torch.int16", "torch.uint16")), "f32": (4, ("torch.float32",)),
          "i32": (4, ("torch.int32", "torch.uint32")), "e4m3": (1, ("torch.float8_e4m3fn", "torch.uint8", "torch.int8")),
          "i8": (1, ("torch.int8", "torch.uint8")), "u8": (1, ("torch.uint8", "torch.int8"))}
_fits = {kind: set() for kind in _KINDS}  # types that have been looked at and taken


def _check_type(t, name, kind):
    size, types = _KINDS[kind]
    if t.element_size() != size:
        raise TypeError(f"{name}: elements of {size} bytes expected, got {t.dtype}")
    if str(t.dtype).startswith("torch.") and str(t.dtype) not in types:
        raise TypeError(f"{name}: {types[0]} expected, got {t.dtype}")
    _fits[kind].add(t.dtype)


def _dev_of(t, name, kind, count=0):
    """_dev of a kind: the type's meaning is checked, not its size alone."""
    if t is None or isinstance(t, int):
        return t
    if not getattr(t, "is_cuda", False):
        raise ValueError(f"{name}: a device buffer (a CUDA tensor) is required")
    if t.dtype not in _fits[kind]:
        _check_type(t, name, kind)
    if t.numel() < count:
        raise ValueError(f"{name}: at least {count} elements needed, {t.numel()} given")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    return t.data_ptr()


def _dev_rows(t, name, kind, rows, cols):
    """Device pointer and row stride (elements) of `rows` rows of `cols` elements each: a CUDA tensor
    whose first dimension may be strided and whose rows are contiguous (a column block of a
    wider matrix is)."""
    if not getattr(t, "is_cuda", False):
        raise ValueError(f"{name}: a device buffer (a CUDA tensor) is required")
    if t.dtype not in _fits[kind]:
        _check_type(t, name, kind)
    shape, stride = t.shape, t.stride()  # (looked at once each: a call's host time is a few microseconds)
    n, inner = shape[0], 1
    for i in range(len(shape) - 1, 0, -1):
        size = shape[i]
        if stride[i] != inner and size != 1:
            raise ValueError(f"{name}: the elements of a row must be contiguous")
        inner *= size
    if n < rows or inner != cols:
        raise ValueError(f"{name}: {rows} rows of {cols} elements expected, got {tuple(shape)}")
    if n <= 1:
        return t.data_ptr(), cols
    if stride[0] < cols:
        raise ValueError(f"{name}: rows overlap")
    return t.data_ptr(), stride[0]


_bf16_types = _fits["bf16"]
_i32_types = _fits["i32"]


def _dev_heads(t, name, n, heads, hd):
    """_dev_rows of n rows [heads][hd] in bf16: the usual layout at once (a call's host time is several such looks)."""
    if t.dtype in _bf16_types and t.is_cuda and t.shape == (n, heads, hd):
        s0, s1, s2 = t.stride()
        if s2 == 1 and s1 == hd and (s0 >= heads * hd or n == 1):
            return t.data_ptr(), s0 if n > 1 else heads * hd
    return _dev_rows(t, name, "bf16", n, heads * hd)


def _dev_i32(t, name, count):
    """_dev_of an int32 vector of `count` elements: the usual one at once."""
    if t is not None and not isinstance(t, int) and t.dtype in _i32_types and t.is_cuda and t.numel() >= count and t.is_contiguous():
        return t.data_ptr()
    return _dev_of(t, name, "i32", count)


class KvCache:
    """A paged key / value cache of one layer in the caller's tensors (dcl_kv_cache): k, v
    [pages][kv heads][page_len][head_dim], bf16, or 1-byte E4M3 codes with k_exp, v_exp int8
    [pages][kv heads][page_len], or 4-bit codes uint8 [pages][kv heads][page_len][head_dim / 2] with
    scale bytes k_exp, v_exp uint8 [pages][kv heads][page_len][head_dim / 32], a shape that tells them from
    exponents: as many bytes in another are refused.  ``KvCache.empty`` allocates one."""

    def __init__(self, k, v, k_exp=None, v_exp=None):
        if len(k.shape) != 4:
            raise ValueError("k: [pages][kv heads][page_len][head_dim] expected")
        pages, heads, page_len, hd = k.shape
        small = k.element_size() == 1
        if small and (k_exp is None or v_exp is None):
            raise ValueError("an FP8 cache needs k_exp and v_exp, a 4-bit one its scales in their place")
        if not small and (k_exp is not None or v_exp is not None):
            raise ValueError("a bf16 cache has no exponents")
        side_shape = tuple(getattr(k_exp, "shape", ()))  # (a raw address has none)
        q4 = small and len(side_shape) == 4 and 16 * side_shape[3] == hd  # (hd / 2 bytes of codes, hd / 32 scales)
        n, kind = pages * heads * page_len, "u8" if q4 else "e4m3" if small else "bf16"
        if tuple(v.shape) != tuple(k.shape):
            raise ValueError("k and v differ in shape")
        codes, side = n * hd, n
        if q4:
            hd *= 2
            side = n * (hd // 32)
            for t, name in ((k_exp, "k_exp"), (v_exp, "v_exp")):
                shape = tuple(getattr(t, "shape", ()))
                if shape != (pages, heads, page_len, hd // 32):
                    raise ValueError(f"{name}: [pages][kv heads][page_len][head_dim / 32] scales expected, got {shape}")
        elif small and hd in (32, 64) and "float8" not in str(k.dtype):  # (4-bit codes of 64 or 128 components have as many bytes)
            for t, name in ((k_exp, "k_exp"), (v_exp, "v_exp")):
                if getattr(t, "is_cuda", False) and t.numel() == n * (hd // 16):
                    raise ValueError(f"{name}: {n * (hd // 16)} bytes are scales of a 4-bit cache, which are [pages][kv heads][page_len]"
                                     f"[head_dim / 32], or more than the {n} exponents of an FP8 one; got {tuple(t.shape)}")
        self.k, self.v, self.k_exp, self.v_exp = k, v, k_exp, v_exp
        self.n_pages, self.n_kv_heads, self.page_len, self.head_dim = pages, heads, page_len, hd
        self.format = DCL_KV_Q4 if q4 else DCL_KV_FP8 if small else DCL_KV_BF16
        self.desc = KvCacheDesc(pages, page_len, heads, hd, self.format, _dev_of(k, "k", kind, codes),
                                _dev_of(v, "v", kind, codes), _dev_of(k_exp, "k_exp", "u8" if q4 else "i8", side),
                                _dev_of(v_exp, "v_exp", "u8" if q4 else "i8", side))
        self.ptr = ctypes.addressof(self.desc)
        self.row = heads * hd  # elements of a position's keys

    @classmethod
    def empty(cls, n_pages, page_len, n_kv_heads, head_dim, fp8=True, device="cuda", q4=False):
        """A cache in new, uninitialised memory (FP8 unless fp8 is False; 4 bits with q4)."""
        import torch
        shape = (n_pages, n_kv_heads, page_len)
        new = lambda s, t: torch.empty(s, dtype=t, device=device)
        if q4:
            return cls(*(new(shape + (head_dim // d,), torch.uint8) for d in (2, 2, 32, 32)))
        shape += (head_dim,)
        if not fp8:
            return cls(new(shape, torch.bfloat16), new(shape, torch.bfloat16))
        return cls(new(shape, torch.uint8), new(shape, torch.uint8), new(shape[:3], torch.int8),
                   new(shape[:3], torch.int8))


class KvPages:
    """Pages of many sequences in the caller's int32 tensors (dcl_kv_pages): table [batch][max_pages],
    held [batch], free [pages] (a stack, its top the last of n_free), n_free [1].  ``KvPages.new``
    allocates them with every page free."""

    def __init__(self, table, held, free, n_free, page_len):
        if len(table.shape) != 2 or len(free.shape) != 1:
            raise ValueError("table: [batch][max_pages], free: [pages] expected")
        batch, width = table.shape
        self.table, self.held, self.free, self.n_free, self.page_len = table, held, free, n_free, page_len
        self.batch, self.max_pages, self.n_pages = batch, width, free.shape[0]
        self.desc = KvPagesDesc(self.n_pages, page_len, batch, width, _dev_of(table, "table", "i32", batch * width),
                                _dev_of(held, "held", "i32", batch), _dev_of(free, "free", "i32", self.n_pages),
                                _dev_of(n_free, "n_free", "i32", 1))
        self.ptr = ctypes.addressof(self.desc)

    @classmethod
    def new(cls, n_pages, page_len, batch, max_pages, device="cuda"):
        import torch
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=device)
        return cls(i32(batch, max_pages) - 1, i32(batch), torch.arange(n_pages, dtype=torch.int32, device=device),
                   i32(1) + n_pages, page_len)


def weight_elements(shape, kind) -> int:
    """Elements of weight tensor `kind` (DCL_W_*) of a model of this shape: matrices in the
    nn.Linear layout [out_features][in_features], gains [d_model]."""
    d, hd, H, G, F, V = shape.d_model, shape.head_dim, shape.n_heads, shape.n_kv_heads, shape.ffn_dim, shape.vocab
    return {DCL_W_EMBED: V * d, DCL_W_ATTN_NORM: d, DCL_W_Q: H * hd * d, DCL_W_K: G * hd * d,
            DCL_W_V: G * hd * d, DCL_W_O: d * H * hd, DCL_W_MLP_NORM: d, DCL_W_GATE: F * d,
            DCL_W_UP: F * d, DCL_W_DOWN: d * F, DCL_W_FINAL_NORM: d, DCL_W_LM_HEAD: V * d}[kind]


def fp8_quantise(w_bits: np.ndarray):
    """dcl_fp8_quantise on a host bf16 weight (uint16 bit patterns [rows][cols]): returns
    (codes uint8 [rows][cols], exps int32 [rows]), row n storing w[n] ~ value(codes[n]) *
    2^exps[n] (E4M3, one power-of-two scale per row).  Host only: no GPU is used."""
    w_bits = np.ascontiguousarray(w_bits)
    if w_bits.dtype != np.uint16 or w_bits.ndim != 2:
        raise TypeError("w_bits: a 2-D array of bf16 bit patterns (uint16)")
    rows, cols = w_bits.shape
    codes = np.empty((rows, cols), np.uint8)
    exps = np.empty(rows, np.int32)
    st = lib().dcl_fp8_quantise(_ptr(w_bits), rows, cols, _ptr(codes), _ptr(exps))
    if st != DCL_OK:
        raise DcleapError(st, lib().dcl_last_error(None).decode())
    return codes, exps


def model_config(shape) -> ModelConfig:
    return ModelConfig(shape.n_layers, shape.d_model, shape.n_heads, shape.n_kv_heads,
                       shape.head_dim, shape.ffn_dim, shape.vocab, shape.mask_id,
                       shape.rope_theta, shape.rms_eps)


def decode_config(tau_commit=0.70, tau_draft=0.98, max_window=0, block_len=32, gen_len=0,
                  kv_cache=0, min_commit=1, contiguous_drafts=0, confidence=0,
                  acceptance=0) -> DecodeConfig:
    """confidence: 0 = top-1 probability, 1 = exp(-entropy); acceptance: 0 = DCV (contiguous),
    1 = Eq. threshold_pd in the semi-autoregressive block."""
    return DecodeConfig(tau_commit, tau_draft, max_window, block_len, gen_len, kv_cache,
                        min_commit, int(bool(contiguous_drafts)), confidence, acceptance)


class Context:
    """One dcl_ctx: a model (or ops-only when shape is None) on the current device."""

    def __init__(self, shape=None, max_batch=1, max_seq=1, stream=None):
        L = lib()
        self._L = L
        self.shape = shape
        self.stream = stream  # None: the context owns a blocking stream
        out = ctypes.c_void_p()
        cfg = model_config(shape) if shape is not None else None
        st = L.dcl_create(ctypes.byref(cfg) if cfg is not None else None, max_batch, max_seq,
                          self.stream, None, ctypes.byref(out))
        if st != DCL_OK:
            raise DcleapError(st, L.dcl_last_error(None).decode())
        self.ptr = out.value
        self.batch = 0
        self.n_prompt = 0
        self.gen_len = 0

    # ------------------------------------------------------------------ plumbing
    def _check(self, st):
        if st != DCL_OK:
            raise DcleapError(st, self._L.dcl_last_error(self.ptr).decode())

    def close(self):
        if getattr(self, "ptr", None):
            self._L.dcl_destroy(self.ptr)
            self.ptr = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    # ------------------------------------------------------------------ the ABI
    def set_weight(self, kind, layer, src):
        """src: numpy bf16 bits (uint16) on the host, or a torch bf16 tensor on the device."""
        is_dev = 0 if isinstance(src, np.ndarray) else int(src.is_cuda)
        if isinstance(src, np.ndarray) and src.dtype != np.uint16:
            raise TypeError("host weights are bf16 bit patterns (uint16)")
        if not isinstance(src, np.ndarray) and src.element_size() != 2:
            raise TypeError(f"weights are bf16 (2-byte elements), got {src.dtype}")
        if self.shape is not None and 0 <= kind <= DCL_W_LM_HEAD:
            need = weight_elements(self.shape, kind)
            have = src.size if isinstance(src, np.ndarray) else src.numel()
            if have < need:
                raise ValueError(f"weight {kind}: {need} elements needed, {have} given")
        self._check(self._L.dcl_set_weight(self.ptr, kind, layer, _ptr(src), is_dev))

    def init_random_weights(self, seed, std=0.02, lm_head_scale=1.0, norm_gain_std=0.0):
        self._check(self._L.dcl_init_random_weights(self.ptr, seed, std, lm_head_scale, norm_gain_std))

    def set_prompt(self, prompt, cfg: DecodeConfig):
        prompt = np.ascontiguousarray(np.atleast_2d(prompt), dtype=np.int32)
        self._check(self._L.dcl_set_prompt(self.ptr, prompt.shape[0], _ptr(prompt), prompt.shape[1],
                                           ctypes.byref(cfg)))
        self.batch, self.n_prompt, self.gen_len = prompt.shape[0], prompt.shape[1], cfg.gen_len
        self.dcfg = cfg

    def step(self, return_k=False):
        if return_k:
            k = np.zeros(self.batch, np.int32)
            self._check(self._L.dcl_step(self.ptr, _ptr(k)))
            return k
        self._check(self._L.dcl_step(self.ptr, None))
        return None

    def generate(self, max_steps=1 << 20, out=True, check=True):
        """Returns (x[N:N+M] per row as int32 [batch][M] or None, Stats, status).
        ``out`` may be a preallocated (e.g. pinned) int32 [batch][M] host array."""
        if isinstance(out, np.ndarray):
            buf = out
        else:
            buf = np.zeros((self.batch, self.gen_len), np.int32) if out else None
        st = Stats()
        status = self._L.dcl_generate(self.ptr, max_steps, _ptr(buf), ctypes.byref(st))
        if check and status not in (DCL_OK,):
            self._check(status)
        return buf, st, status

    def restart(self):
        self._check(self._L.dcl_restart(self.ptr))

    def get_state(self):
        x = np.zeros((self.batch, self.n_prompt + self.gen_len), np.int32)
        p = np.zeros(self.batch, np.int32)
        self._check(self._L.dcl_get_state(self.ptr, _ptr(x), _ptr(p)))
        return x, p

    def set_state(self, x, p):
        x = np.ascontiguousarray(x, dtype=np.int32)
        p = np.ascontiguousarray(p, dtype=np.int32)
        self._check(self._L.dcl_set_state(self.ptr, _ptr(x), _ptr(p)))

    def _outs(self, logits, top1, p1, p2, conf, entropy):
        """Device pointers of the per-position outputs of a forward ([batch][M], logits
        [batch][M][vocab])."""
        n = self.batch * self.gen_len
        vocab = self.shape.vocab if self.shape is not None else 0
        return (_dev(logits, "logits", 2, n * vocab), _dev(top1, "top1", 4, n), _dev(p1, "p1", 4, n),
                _dev(p2, "p2", 4, n), _dev(conf, "conf", 4, n), _dev(entropy, "entropy", 4, n))

    def _stream_elems(self):
        """Elements of a residual stream buffer: float [batch*(N+M)][d_model]."""
        d = self.shape.d_model if self.shape is not None else 0
        return self.batch * (self.n_prompt + self.gen_len) * d

    def forward_debug(self, logits=None, top1=None, p1=None, p2=None, conf=None, entropy=None):
        self._check(self._L.dcl_forward_debug(self.ptr, *self._outs(logits, top1, p1, p2, conf, entropy)))

    def debug_hidden(self, layer, h):
        self._check(self._L.dcl_debug_hidden(self.ptr, layer, _dev(h, "h", 4, self._stream_elems())))

    def forward_debug_from(self, layer, h, commit=False, logits=None, top1=None, p1=None, p2=None, conf=None,
                           entropy=None):
        self._check(self._L.dcl_forward_debug_from(self.ptr, layer, _dev(h, "h", 4, self._stream_elems()),
                                                   int(bool(commit)),
                                                   *self._outs(logits, top1, p1, p2, conf, entropy)))

    def accept(self, logits, committed, x, cfg: DecodeConfig, k):
        B, P, V = logits.shape
        self._check(self._L.dcl_accept(self.ptr, _dev(logits, "logits", 2, B * P * V),
                                       B, P, V, _dev(committed, "committed", 4, B), _dev(x, "x", 4, B * P),
                                       ctypes.byref(cfg), _dev(k, "k", 4, B)))

    def synchronise(self):
        """Wait for the context stream; raises what its kernels recorded."""
        self._check(self._L.dcl_synchronise(self.ptr))

    def kv_write(self, cache, k, v, slots):
        """Store rows k, v [n][kv heads][head_dim] (bf16, rows may be strided) at slots (int32 [n],
        negative: skipped)."""
        n, heads, hd = k.shape[0], cache.n_kv_heads, cache.head_dim
        kp, ks = _dev_heads(k, "k", n, heads, hd)
        vp, vs = _dev_heads(v, "v", n, heads, hd)
        if ks != vs and n > 1:
            raise ValueError("k and v differ in row stride")
        st = self._L.dcl_kv_write(self.ptr, cache.ptr, kp, vp, ks, _dev_i32(slots, "slots", n), n)
        if st:
            self._check(st)

    def kv_read(self, cache, slots, k, v):
        """Read the positions at slots (int32 [n], negative: zeros) into k, v [n][kv heads][head_dim]."""
        n, heads, hd = slots.shape[0], cache.n_kv_heads, cache.head_dim
        kp, ks = _dev_heads(k, "k", n, heads, hd)
        vp, vs = _dev_heads(v, "v", n, heads, hd)
        if ks != vs and n > 1:
            raise ValueError("k and v differ in row stride")
        st = self._L.dcl_kv_read(self.ptr, cache.ptr, _dev_i32(slots, "slots", n), n, kp, vp, ks)
        if st:
            self._check(st)

    def kv_attention(self, cache, q, q_start, page_table, seq_len, out, max_new, causal=False, scale=0.0, lse=None):
        """Attention of the rows q [n_q][heads][head_dim] (bf16, rows may be strided; rows
        [q_start[b], q_start[b + 1]) are sequence b's) over the first seq_len[b] positions of the
        pages page_table[b]; out [n_q][heads][head_dim] bf16, lse [n_q][heads] float."""
        n_q, heads, hd = q.shape
        batch, max_pages = page_table.shape
        if hd != cache.head_dim:
            raise ValueError(f"q: head_dim {cache.head_dim} expected, got {hd}")
        qp, qs = _dev_heads(q, "q", n_q, heads, hd)
        st = self._L.dcl_kv_attention(
            self.ptr, cache.ptr, qp, qs, _dev_i32(q_start, "q_start", batch + 1), _dev_i32(page_table, "page_table", 0),
            max_pages, _dev_i32(seq_len, "seq_len", batch), batch, n_q, max_new, heads, 1 if causal else 0, scale,
            _dev_of(out, "out", "bf16", n_q * heads * hd), _dev_of(lse, "lse", "f32", n_q * heads))
        if st:
            self._check(st)

    def kv_plan(self, pages, start, new, q_start, seq_len, slots, pos):
        """Lay out a step: sequence b keeps start[b] cached positions and gets new[b] rows (int32 [batch]).
        Moves pages between the sequences and the stack; writes q_start [batch + 1], seq_len [batch], and
        slots, pos [rows] (-1 past the last sequence's).  A sequence that is given no rows has seq_len start.  seq_len
        may be start itself: the next step goes on from it."""
        B, rows = pages.batch, slots.shape[0]
        st = self._L.dcl_kv_plan(self.ptr, pages.ptr, _dev_i32(start, "start", B), _dev_i32(new, "new", B),
                                 _dev_i32(q_start, "q_start", B + 1), _dev_i32(seq_len, "seq_len", B),
                                 _dev_i32(slots, "slots", rows), _dev_i32(pos, "pos", rows), rows)
        if st:
            self._check(st)

    def qk_norm_rope(self, q, k, pos, q_out, k_out, theta, q_gain=None, k_gain=None, eps=1e-6, rot_dim=None):
        """Norm (where there is a gain, bf16 [head_dim]) and rotate by pos (int32 [n], negative: the row is left
        out) every head of q [n][heads][head_dim] and k [n][kv heads][head_dim] (bf16, rows may be strided)
        into q_out, k_out (as q, k, or these themselves)."""
        n, H, hd = q.shape
        G = k.shape[1]
        qp, qs = _dev_heads(q, "q", n, H, hd)
        kp, ks = _dev_heads(k, "k", n, G, hd)
        qo, qos = (qp, qs) if q_out is q else _dev_heads(q_out, "q_out", n, H, hd)
        ko, kos = (kp, ks) if k_out is k else _dev_heads(k_out, "k_out", n, G, hd)
        st = self._L.dcl_qk_norm_rope(self.ptr, qp, qs, kp, ks, _dev_i32(pos, "pos", n), n, H, G, hd,
                                      hd if rot_dim is None else rot_dim, theta, _dev_of(q_gain, "q_gain", "bf16", hd),
                                      _dev_of(k_gain, "k_gain", "bf16", hd), eps, qo, qos, ko, kos)
        if st:
            self._check(st)

    def sample(self, logits, token, noise=None, temperature=None, top_k=None, top_p=None, min_p=None, prob=None,
               conf=None):
        """Draw token [rows] from logits [rows][V] (bf16, rows may be strided) and Gumbel numbers noise
        [rows][V]; temperature, top_k, top_p, min_p, prob, conf [rows] each (see dcl_sample)."""
        rows, V = logits.shape
        zp, zs = _dev_rows(logits, "logits", "bf16", rows, V)
        np_, ns = _dev_rows(noise, "noise", "f32", rows, V) if noise is not None else (None, V)
        self._check(self._L.dcl_sample(
            self.ptr, zp, zs, np_, ns, rows, V, _dev_of(temperature, "temperature", "f32", rows),
            _dev_of(top_k, "top_k", "i32", rows), _dev_of(top_p, "top_p", "f32", rows),
            _dev_of(min_p, "min_p", "f32", rows), _dev_of(token, "token", "i32", rows),
            _dev_of(prob, "prob", "f32", rows), _dev_of(conf, "conf", "f32", rows)))

    def op_rmsnorm(self, x, gain, y, eps):
        rows, d = x.shape
        self._check(self._L.dcl_op_rmsnorm(self.ptr, _dev(x, "x", 4, rows * d), _dev(gain, "gain", 2, d),
                                           _dev(y, "y", 2, rows * d), rows, d, eps))

    def op_linear(self, a, w, out, mode=0, tile=0):
        M, K = a.shape
        N = w.shape[0]
        self._check(self._L.dcl_op_linear(self.ptr, _dev(a, "a", 2, M * K), _dev(w, "w", 2, N * K),
                                          _dev(out, "out", 4 if mode == 1 else 2, M * N), M, N, K, mode, tile))

    def op_attention(self, qkv, out, batch, T, H, G, hd, q_rows=0):
        rows = batch * T
        self._check(self._L.dcl_op_attention(self.ptr, _dev(qkv, "qkv", 2, rows * (H + 2 * G) * hd),
                                             _dev(out, "out", 2, rows * H * hd), batch, T, H, G, hd, q_rows))

    def op_lmhead_top2(self, x, w, top1, p1, p2, tile=0, entropy=None):
        R, d = x.shape
        V = w.shape[0]
        self._check(self._L.dcl_op_lmhead_top2(self.ptr, _dev(x, "x", 2, R * d), _dev(w, "w", 2, V * d), R, V, d,
                                               _dev(top1, "top1", 4, R), _dev(p1, "p1", 4, R),
                                               _dev(p2, "p2", 4, R), _dev(entropy, "entropy", 4, R), tile))

    def op_generate(self, dst, seed, tid, start, count, std, mean=0.0):
        self._check(self._L.dcl_op_generate(self.ptr, _dev(dst, "dst", 2, count), seed, tid, start, count, std,
                                            mean))

    def selftest_wait_timeout(self, which):
        """Status of the bounded-wait self-test (DCL_ERR_TIMEOUT is the expected one)."""
        return self._L.dcl_selftest_wait_timeout(self.ptr, which)

    def launch_floor(self, n_kernels, reps=200):
        """Mean ms of a CUDA graph of n_kernels empty dependent launches."""
        ms = ctypes.c_float()
        self._check(self._L.dcl_launch_floor(self.ptr, n_kernels, reps, ctypes.byref(ms)))
        return ms.value

    def set_profiling(self, enable):
        self._check(self._L.dcl_set_profiling(self.ptr, int(bool(enable))))

    def profile_last_step(self, cap=4096):
        ms = np.zeros(cap, np.float32)
        kind = np.zeros(cap, np.int32)
        n = ctypes.c_int32(0)
        self._check(self._L.dcl_profile_last_step(self.ptr, _ptr(ms), _ptr(kind), cap, ctypes.byref(n)))
        return ms[:n.value].copy(), kind[:n.value].copy()

    # ------------------------------------------------------------------ helpers
    def load_weights(self, weights: dict):
        """Upload a dict of float32 (bf16-exact) arrays: embed, final_norm, lm_head and
        per-layer attn_norm, wq, wk, wv, wo, mlp_norm, w_gate, w_up, w_down."""
        import torch

        def up(kind, layer, a):
            bits = torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(torch.bfloat16)
            self.set_weight(kind, layer, bits.view(torch.int16).numpy().view(np.uint16))
        up(DCL_W_EMBED, 0, weights["embed"])
        up(DCL_W_FINAL_NORM, 0, weights["final_norm"])
        up(DCL_W_LM_HEAD, 0, weights["lm_head"])
        names = [(DCL_W_ATTN_NORM, "attn_norm"), (DCL_W_Q, "wq"), (DCL_W_K, "wk"), (DCL_W_V, "wv"),
                 (DCL_W_O, "wo"), (DCL_W_MLP_NORM, "mlp_norm"), (DCL_W_GATE, "w_gate"),
                 (DCL_W_UP, "w_up"), (DCL_W_DOWN, "w_down")]
        for li, lw in enumerate(weights["layers"]):
            for kind, key in names:
                up(kind, li, lw[key])


def exported_symbols():
    """Names declared in include/dcleap.h (for the ABI test)."""
    return [n for n in SIGNATURES]
