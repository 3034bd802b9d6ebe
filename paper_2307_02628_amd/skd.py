"""Thin ctypes binding of libskd.so (include/skd.h): argument marshalling only.

Every step of the decode path runs inside the HIP library; there is no Python
or CPU fallback.  If the library has not been built, loading fails loudly.
PyTorch is used by callers only to own device memory and streams; this module
itself needs numpy and ctypes.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, List, Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libskd.so")

OK, ERR_NULL, ERR_SHAPE, ERR_RANGE, ERR_ORDER, ERR_SCHEDULE, ERR_NOMEM, ERR_HIP = 0, -1, -2, -3, -4, -5, -6, -7
BF16, FP32, BF16_KV8 = 0, 1, 2
HOST, DEVICE = 0, 1
W_FP32, W_BF16 = 0, 1
KV_BF16, KV_FP8 = 0, 1

EXPORTS = ["skd_schedule", "skd_active_layers", "skd_create", "skd_create_with_schedule", "skd_state_active_layers", "skd_prefill", "skd_decode_step",
           "skd_logits_argmax", "skd_logits_argmax_noalloc", "skd_logits_sample", "skd_rewind", "skd_profile_enable", "skd_profile_read", "skd_kv_len", "skd_kv_pages_reserved", "skd_kv_pages_dense", "skd_synchronize",
           "skd_debug_read_hidden", "skd_debug_kv_load", "skd_debug_kv_read", "skd_destroy", "skd_strerror",
           "skd_last_hip_error", "skd_kv_page_bytes", "skd_kv_append", "skd_kv_read", "skd_kv_attend", "skd_kv_attend_workspace",
           "skd_logits_sample_rows", "skd_sample", "skd_sample_workspace", "skd_decode_chunk"]


class Config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "L", "d_model", "n_heads", "ffn", "vocab", "max_pos",
        "batch", "prompt_size", "sequence_length", "n_min", "n_max", "warmup",
        "page_tokens", "dtype", "io_on_device")]


class Sampling(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("temperature", "top_k", "top_p", "min_p")]


_PP = C.POINTER(C.c_void_p)


class Weights(C.Structure):
    _fields_ = ([("location", C.c_int32), ("elem", C.c_int32)] +
                [(n, C.c_void_p) for n in ("tok_emb", "pos_emb", "lnf_g", "lnf_b", "lm_head")] +
                [(n, _PP) for n in ("ln1_g", "ln1_b", "wqkv", "bqkv", "wo", "bo",
                                    "ln2_g", "ln2_b", "w1", "b1", "w2", "b2")])


PROF_CLASSES = ("embed_ln", "gemm_qkv", "attention", "gemm_out", "reduce_ln", "gemm_ffn1", "gemm_ffn2", "lm_head",
                "argmax", "other")
PER_LAYER = ("ln1_g", "ln1_b", "wqkv", "bqkv", "wo", "bo", "ln2_g", "ln2_b", "w1", "b1", "w2", "b2")

_lib: Optional[C.CDLL] = None


def lib() -> C.CDLL:
    """Load libskd.so (built by paper_2307_02628_amd._build / __graft_entry__.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it first (python -m paper_2307_02628_amd._build); "
                               "there is no fallback path")
        l = C.CDLL(LIB_PATH)
        l.skd_schedule.argtypes = [C.c_int32] * 6
        l.skd_active_layers.argtypes = [C.c_int32, C.c_void_p, C.c_void_p]
        l.skd_create.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        l.skd_create_with_schedule.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        l.skd_state_active_layers.argtypes = [C.c_void_p, C.c_int32, C.c_void_p]
        l.skd_prefill.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
        l.skd_decode_step.argtypes = [C.c_void_p, C.c_int32, C.c_void_p]
        l.skd_logits_argmax.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
        l.skd_logits_argmax_noalloc.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
        l.skd_logits_sample.argtypes = [C.c_void_p, C.c_void_p, C.c_float, C.c_float, C.c_void_p, C.c_void_p]
        l.skd_rewind.argtypes = [C.c_void_p, C.c_int32]
        l.skd_profile_enable.argtypes = [C.c_void_p, C.c_int32]
        l.skd_profile_read.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
        l.skd_kv_len.argtypes = [C.c_void_p, C.c_int32]
        l.skd_kv_pages_reserved.argtypes = [C.c_void_p]
        l.skd_kv_pages_reserved.restype = C.c_int64
        l.skd_kv_pages_dense.argtypes = [C.c_void_p]
        l.skd_kv_pages_dense.restype = C.c_int64
        l.skd_synchronize.argtypes = [C.c_void_p]
        l.skd_debug_read_hidden.argtypes = [C.c_void_p, C.c_void_p]
        l.skd_debug_kv_load.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
        l.skd_debug_kv_read.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
        l.skd_destroy.argtypes = [C.c_void_p]
        l.skd_destroy.restype = None
        l.skd_strerror.argtypes = [C.c_int]
        l.skd_strerror.restype = C.c_char_p
        l.skd_last_hip_error.argtypes = []
        P, I32, I64 = C.c_void_p, C.c_int32, C.c_int64
        l.skd_kv_page_bytes.argtypes, l.skd_kv_page_bytes.restype = [P], I64
        l.skd_kv_append.argtypes = [P, P, P, I64, P, I64, P]
        l.skd_kv_read.argtypes = [P, P, I32, P, I64, P, I64, P]
        l.skd_kv_attend.argtypes = [P, P, I32, C.c_float, P, I64, P, I64, P, I64, P, I64, P, I64, P]
        l.skd_kv_attend_workspace.argtypes, l.skd_kv_attend_workspace.restype = [P, P, I32], I64
        l.skd_logits_sample_rows.argtypes = [P] * 5
        l.skd_decode_chunk.argtypes = [P, I32, I32, P]
        l.skd_sample.argtypes = [P, I64, I32, I32, P, P, P, P, I64, P]
        l.skd_sample_workspace.argtypes, l.skd_sample_workspace.restype = [I32, I32], I64
        _lib = l
    return _lib


class SkdError(RuntimeError):
    def __init__(self, code: int, where: str):
        msg = lib().skd_strerror(code).decode()
        extra = f" (hipError {lib().skd_last_hip_error()})" if code == ERR_HIP else ""
        super().__init__(f"{where}: {msg}{extra} [{code}]")
        self.code = code


_DTYPES: dict = {}


def _dtype_of(t) -> str:
    name = _DTYPES.get(t.dtype)
    if name is None:
        name = _DTYPES[t.dtype] = str(t.dtype)
    return name


def _check(rc: int, where: str) -> int:
    if rc < 0:
        raise SkdError(rc, where)
    return rc


def skd_schedule(t: int, prompt_size: int, sequence_length: int, n_min: int, n_max: int, L: int) -> int:
    """n(t), or a negative error code (no exception: mirrors the C call)."""
    return lib().skd_schedule(t, prompt_size, sequence_length, n_min, n_max, L)


def skd_active_layers(t: int, cfg: Config) -> List[int]:
    out = (C.c_int32 * max(cfg.L, 1))()
    n = _check(lib().skd_active_layers(t, C.byref(cfg), out), "skd_active_layers")
    return [int(out[i]) for i in range(n)]


def make_config(shape, batch: int, prompt_size: int, sequence_length: int, n_min: int, n_max: int, warmup: int = 0,
                dtype: int = BF16, page_tokens: int = 0, io_on_device: int = 0) -> Config:
    """`shape` needs attributes L, d, H, f, V, max_pos."""
    return Config(shape.L, shape.d, shape.H, shape.f, shape.V, shape.max_pos, batch, prompt_size, sequence_length,
                  n_min, n_max, warmup, page_tokens, dtype, io_on_device)


def _ptr_of(a) -> int:
    if a is None:
        return 0
    if isinstance(a, np.ndarray):
        return a.ctypes.data
    if hasattr(a, "data_ptr"):      # torch tensor (device or host)
        return a.data_ptr()
    return int(a)


class Decoder:
    """One decoding state (skd_create .. skd_destroy)."""

    def __init__(self, cfg: Config, weights: Dict[str, object], location: int = HOST, elem: int = W_FP32,
                 stream: int = 0, n_table=None):
        """weights: dict with tok_emb, pos_emb, lnf_g, lnf_b, optional lm_head, and per-layer lists named as in
        skd_weights.  Entries are numpy arrays (host), torch tensors, or raw addresses; fp32, or uint16/bfloat16
        bit patterns with elem=W_BF16."""
        self._lib = lib()
        self.cfg = cfg
        self._keep = []
        w = Weights()
        w.location, w.elem = location, elem

        def prep(a):
            if isinstance(a, np.ndarray):
                a = np.ascontiguousarray(a, dtype=np.float32 if elem == W_FP32 else np.uint16)
            self._keep.append(a)
            return _ptr_of(a)

        for n in ("tok_emb", "pos_emb", "lnf_g", "lnf_b"):
            setattr(w, n, prep(weights[n]))
        w.lm_head = prep(weights["lm_head"]) if weights.get("lm_head") is not None else None
        for n in PER_LAYER:
            lst = weights[n]
            if len(lst) != cfg.L:
                raise ValueError(f"{n}: expected {cfg.L} layers, got {len(lst)}")
            tab = (C.c_void_p * cfg.L)(*[prep(a) for a in lst])
            self._keep.append(tab)
            setattr(w, n, C.cast(tab, _PP))
        h = C.c_void_p()
        if n_table is None:
            _check(self._lib.skd_create(C.byref(cfg), C.byref(w), C.c_void_p(stream), C.byref(h)), "skd_create")
        else:
            tab = np.ascontiguousarray(n_table, dtype=np.int32)
            if tab.shape != (cfg.sequence_length,):
                raise ValueError("n_table needs one entry per position")
            _check(self._lib.skd_create_with_schedule(C.byref(cfg), C.byref(w), C.c_void_p(stream), tab.ctypes.data,
                                                      C.byref(h)), "skd_create_with_schedule")
        self._h = h
        self._keep = []   # the library has copied everything

    # -- lifecycle
    def close(self):
        if getattr(self, "_h", None):
            self._lib.skd_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    # -- the four calls of the path
    def prefill_rc(self, tokens, attn_mask=None) -> int:
        if isinstance(tokens, np.ndarray):
            tokens = np.ascontiguousarray(tokens, dtype=np.int32)
        if isinstance(attn_mask, np.ndarray):
            attn_mask = np.ascontiguousarray(attn_mask, dtype=np.uint8)
        return self._lib.skd_prefill(self._h, _ptr_of(tokens), _ptr_of(attn_mask))

    def prefill(self, tokens, attn_mask=None):
        _check(self.prefill_rc(tokens, attn_mask), "skd_prefill")

    def decode_step_rc(self, t: int, tokens_in=None) -> int:
        if isinstance(tokens_in, np.ndarray):
            tokens_in = np.ascontiguousarray(tokens_in, dtype=np.int32)
        return self._lib.skd_decode_step(self._h, t, _ptr_of(tokens_in))

    def decode_step(self, t: int, tokens_in=None):
        _check(self.decode_step_rc(t, tokens_in), "skd_decode_step")

    def decode_chunk_rc(self, t: int, tokens) -> int:
        """tokens: [B][cols] host array, or [cols][B] int32 device tensor with io_on_device."""
        if isinstance(tokens, np.ndarray):
            tokens = np.ascontiguousarray(tokens, dtype=np.int32)
            if tokens.ndim != 2:
                raise ValueError("expected tokens of two dimensions")
        else:
            _expect(tokens, "int32", 2)
        if bool(self.cfg.io_on_device) != bool(getattr(tokens, "is_cuda", False)):
            raise ValueError("expected tokens in " + ("device" if self.cfg.io_on_device else "host") + " memory")
        B, cols = tokens.shape if not self.cfg.io_on_device else tuple(tokens.shape)[::-1]
        if B != self.cfg.batch:
            raise ValueError(f"tokens of {self.cfg.batch} rows expected")
        return self._lib.skd_decode_chunk(self._h, t, cols, _ptr_of(tokens))

    def decode_chunk(self, t: int, tokens):
        _check(self.decode_chunk_rc(t, tokens), "skd_decode_chunk")

    def logits_argmax(self, want_logits: bool = True):
        """Host-I/O form: returns (tokens[B] int32, logits[B,V] float32 or None)."""
        assert not self.cfg.io_on_device
        tok = np.zeros(self.cfg.batch, dtype=np.int32)
        lg = np.zeros((self.cfg.batch, self.cfg.vocab), dtype=np.float32) if want_logits else None
        _check(self._lib.skd_logits_argmax(self._h, tok.ctypes.data, _ptr_of(lg)), "skd_logits_argmax")
        return tok, lg

    def logits_sample_rc(self, u, temperature: float, top_p: float, want_logits: bool = True):
        """Host-I/O form of skd_logits_sample: returns (rc, tokens[B], logits[B,V] or None)."""
        assert not self.cfg.io_on_device
        uu = np.ascontiguousarray(u, dtype=np.float32)
        tok = np.zeros(self.cfg.batch, dtype=np.int32)
        lg = np.zeros((self.cfg.batch, self.cfg.vocab), dtype=np.float32) if want_logits else None
        rc = self._lib.skd_logits_sample(self._h, uu.ctypes.data, temperature, top_p, tok.ctypes.data, _ptr_of(lg))
        return rc, tok, lg

    def logits_sample(self, u, temperature: float, top_p: float, want_logits: bool = True):
        rc, tok, lg = self.logits_sample_rc(u, temperature, top_p, want_logits)
        _check(rc, "skd_logits_sample")
        return tok, lg

    def logits_sample_device(self, u, temperature: float, top_p: float, tokens_out=None, logits_out=None):
        """Device-I/O form: u, tokens_out, logits_out are device pointers / torch tensors; asynchronous."""
        _check(self._lib.skd_logits_sample(self._h, _ptr_of(u), temperature, top_p, _ptr_of(tokens_out),
                                           _ptr_of(logits_out)), "skd_logits_sample")

    def logits_sample_rows_rc(self, u, temperature=None, top_k=None, top_p=None, min_p=None, want_logits: bool = True):
        """Host-I/O form of skd_logits_sample_rows, parameters [B] or None: returns (rc, tokens[B], logits[B,V] or None)."""
        assert not self.cfg.io_on_device
        arrays = [None if a is None else np.ascontiguousarray(a, dtype=t) for a, t in
                  ((temperature, np.float32), (top_k, np.int32), (top_p, np.float32), (min_p, np.float32))]
        uu = np.ascontiguousarray(u, dtype=np.float32)
        for a in arrays + [uu]:
            if a is not None and a.shape != (self.cfg.batch,):
                raise ValueError("parameters have one entry per row")
        tok = np.zeros(self.cfg.batch, dtype=np.int32)
        lg = np.zeros((self.cfg.batch, self.cfg.vocab), dtype=np.float32) if want_logits else None
        rc = self._lib.skd_logits_sample_rows(self._h, uu.ctypes.data, C.byref(Sampling(*[_ptr_of(a) for a in arrays])), tok.ctypes.data,
                                              _ptr_of(lg))
        return rc, tok, lg

    def logits_sample_rows(self, u, temperature=None, top_k=None, top_p=None, min_p=None, want_logits: bool = True):
        rc, tok, lg = self.logits_sample_rows_rc(u, temperature, top_k, top_p, min_p, want_logits)
        _check(rc, "skd_logits_sample_rows")
        return tok, lg

    def logits_sample_rows_device(self, u, temperature=None, top_k=None, top_p=None, min_p=None, tokens_out=None, logits_out=None):
        """Device-I/O form: device pointers / torch tensors (top_k and tokens_out int32, the others float32); asynchronous."""
        assert self.cfg.io_on_device
        B = self.cfg.batch
        for t, dtype, shape in ((u, "float32", (B,)), (temperature, "float32", (B,)), (top_k, "int32", (B,)), (top_p, "float32", (B,)),
                                (min_p, "float32", (B,)), (tokens_out, "int32", (B,)), (logits_out, "float32", (B, self.cfg.vocab))):
            if hasattr(t, "data_ptr"):
                _expect(t, dtype, len(shape))
                if tuple(t.shape) != shape or not t.is_cuda:
                    raise ValueError(f"expected device memory of shape {shape}")
            elif isinstance(t, np.ndarray):
                raise ValueError("expected device memory")
        p = Sampling(*[_ptr_of(a) for a in (temperature, top_k, top_p, min_p)])
        _check(self._lib.skd_logits_sample_rows(self._h, _ptr_of(u), C.byref(p), _ptr_of(tokens_out), _ptr_of(logits_out)),
               "skd_logits_sample_rows")

    def logits_argmax_device(self, tokens_out=None, logits_out=None):
        """Device-I/O form: pointers / torch tensors on the device; asynchronous."""
        _check(self._lib.skd_logits_argmax(self._h, _ptr_of(tokens_out), _ptr_of(logits_out)), "skd_logits_argmax")

    def logits_argmax_noalloc_rc(self, tokens_out=None, logits_out=None) -> int:
        """skd_logits_argmax_noalloc (device I/O only): the return code, no exception."""
        return self._lib.skd_logits_argmax_noalloc(self._h, _ptr_of(tokens_out), _ptr_of(logits_out))

    def rewind(self, t: int):
        _check(self._lib.skd_rewind(self._h, t), "skd_rewind")

    def profile_enable(self, mode):
        """0 / False: off; 1 / True: each kernel's own begin and end time stamps; 2: event brackets on the stream."""
        _check(self._lib.skd_profile_enable(self._h, int(mode)), "skd_profile_enable")

    def profile_read(self) -> Dict[str, Dict[str, float]]:
        ms = (C.c_double * len(PROF_CLASSES))()
        n = (C.c_int64 * len(PROF_CLASSES))()
        _check(self._lib.skd_profile_read(self._h, ms, n), "skd_profile_read")
        return {name: {"ms": float(ms[i]), "launches": int(n[i])} for i, name in enumerate(PROF_CLASSES)}

    def active_layers(self, t: int) -> List[int]:
        out = (C.c_int32 * max(self.cfg.L, 1))()
        n = _check(self._lib.skd_state_active_layers(self._h, t, out), "skd_state_active_layers")
        return [int(out[i]) for i in range(n)]

    # -- bookkeeping and hooks
    def kv_len(self, layer: int) -> int:
        return _check(self._lib.skd_kv_len(self._h, layer), "skd_kv_len")

    def kv_pages(self):
        return int(self._lib.skd_kv_pages_reserved(self._h)), int(self._lib.skd_kv_pages_dense(self._h))

    def synchronize(self):
        _check(self._lib.skd_synchronize(self._h), "skd_synchronize")

    def read_hidden(self) -> np.ndarray:
        x = np.zeros((self.cfg.batch, self.cfg.d_model), dtype=np.float32)
        _check(self._lib.skd_debug_read_hidden(self._h, x.ctypes.data), "skd_debug_read_hidden")
        return x

    def kv_load(self, cols: int, K: Sequence[Optional[np.ndarray]], V: Sequence[Optional[np.ndarray]], start=None):
        keep = []

        def tab(lst):
            ptrs = []
            for a in lst:
                if a is None:
                    ptrs.append(None)
                else:
                    a = np.ascontiguousarray(a, dtype=np.float32)
                    assert a.shape == (self.cfg.batch, cols, self.cfg.d_model)
                    keep.append(a)
                    ptrs.append(a.ctypes.data)
            return (C.c_void_p * self.cfg.L)(*ptrs)

        kt, vt = tab(K), tab(V)
        st = None if start is None else np.ascontiguousarray(start, dtype=np.int32)
        _check(self._lib.skd_debug_kv_load(self._h, cols, kt, vt, _ptr_of(st)), "skd_debug_kv_load")

    def kv_read(self, layer: int, b: int):
        n = self.kv_len(layer)
        k = np.zeros((n, self.cfg.d_model), dtype=np.float32)
        v = np.zeros((n, self.cfg.d_model), dtype=np.float32)
        _check(self._lib.skd_debug_kv_read(self._h, layer, b, k.ctypes.data, v.ctypes.data), "skd_debug_kv_read")
        return k, v


class Kv(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("elem", "kv_heads", "head_dim", "page_tokens", "pages", "rows", "max_pages")] +
                [("pool", C.c_void_p), ("block_table", C.c_void_p)])


class Chunk(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("tokens", "max_new", "max_past")] + [("first", C.c_void_p), ("past", C.c_void_p)]


class KvChunk:
    """The tokens of a call on a KvCache (skd_kv_chunk): first [rows + 1] and past [rows] are int32 device tensors."""

    def __init__(self, first, past, tokens: int, max_new: int, max_past: int):
        _expect(first, "int32", 1)
        _expect(past, "int32", 1)
        if len(first) != len(past) + 1:
            raise ValueError("first needs one entry more than past")
        self._keep = (first, past)
        self.rows, self.tokens = len(past), tokens
        self.c = Chunk(tokens, max_new, max_past, _ptr_of(first), _ptr_of(past))
        self.ref = C.byref(self.c)


class KvCache:
    """Keys and values in pages of the caller's memory (skd_kv): pool [pages][..] and block_table [rows][max_pages] (int32) are
    contiguous device tensors, kept alive by this object; calls run on `stream` (0: the default stream)."""

    def __init__(self, pool, block_table, kv_heads: int, head_dim: int, page_tokens: int, elem: int = KV_BF16):
        self._lib = lib()
        _expect(block_table, "int32", 2)
        if not pool.is_contiguous() or pool.dim() < 1:
            raise ValueError("pool must be contiguous, pages first")
        self._keep = (pool, block_table)
        self.rows, self.heads, self.dh = block_table.shape[0], kv_heads, head_dim
        self.c = Kv(elem, kv_heads, head_dim, page_tokens, pool.shape[0], block_table.shape[0], block_table.shape[1],
                    _ptr_of(pool), _ptr_of(block_table))
        self.ref = C.byref(self.c)
        self.page_bytes = _check(self._lib.skd_kv_page_bytes(self.ref), "skd_kv_page_bytes")
        if pool.numel() * pool.element_size() != self.page_bytes * pool.shape[0]:
            raise ValueError(f"a page of the pool needs {self.page_bytes} bytes")

    def _rows_of(self, chunk: KvChunk, heads: int, t, *types):
        """Pointer and stride of [tokens][heads][head_dim] or [tokens][heads * head_dim]."""
        if chunk.rows != self.rows:
            raise ValueError("chunk and block table differ in rows")
        shape, stride = tuple(t.shape), t.stride()
        if shape not in ((chunk.tokens, heads, self.dh), (chunk.tokens, heads * self.dh)) or stride[-1] != 1 or (len(shape) == 3 and heads > 1 and stride[1] != self.dh):
            raise ValueError(f"expected [{chunk.tokens}][{heads}][{self.dh}] with dense tokens")
        if _dtype_of(t) not in types:
            raise ValueError(f"expected {' or '.join(types)}")
        return t.data_ptr(), heads * self.dh if shape[0] < 2 else stride[0]  # (one token: whatever its stride says)

    def append(self, chunk: KvChunk, k, v, stream: int = 0):
        _check(self._lib.skd_kv_append(self.ref, chunk.ref, *self._rows_of(chunk, self.heads, k, "torch.bfloat16"),
                                       *self._rows_of(chunk, self.heads, v, "torch.bfloat16"), stream), "skd_kv_append")

    def read(self, chunk: KvChunk, k_out, v_out, stream: int = 0):
        """k_out, v_out: both float32 or both bfloat16."""
        elem = W_FP32 if _dtype_of(k_out) == "torch.float32" else W_BF16
        types = ("torch.float32",) if elem == W_FP32 else ("torch.bfloat16",)
        _check(self._lib.skd_kv_read(self.ref, chunk.ref, elem, *self._rows_of(chunk, self.heads, k_out, *types),
                                     *self._rows_of(chunk, self.heads, v_out, *types), stream), "skd_kv_read")

    def attend_workspace(self, chunk: KvChunk, heads: int) -> int:
        return _check(self._lib.skd_kv_attend_workspace(self.ref, chunk.ref, heads), "skd_kv_attend_workspace")

    def attend(self, chunk: KvChunk, q, out, scale: float, k=None, v=None, workspace=None, stream: int = 0):
        """q, out [tokens][heads][head_dim]; workspace: a device tensor of attend_workspace bytes (None where that is 0)."""
        heads = q.shape[1] if q.dim() == 3 else q.shape[1] // self.dh
        kk = (0, 0) if k is None else self._rows_of(chunk, self.heads, k, "torch.bfloat16")
        vv = (0, 0) if v is None else self._rows_of(chunk, self.heads, v, "torch.bfloat16")
        ws = (0, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
        _check(self._lib.skd_kv_attend(self.ref, chunk.ref, heads, scale, *self._rows_of(chunk, heads, q, "torch.bfloat16"), *kk, *vv,
                                       *self._rows_of(chunk, heads, out, "torch.bfloat16"), *ws, stream), "skd_kv_attend")


def _expect(t, dtype: str, dims: int):
    if _dtype_of(t) != "torch." + dtype or t.dim() != dims or not t.is_contiguous():
        raise ValueError(f"expected a contiguous {dtype} tensor of {dims} dimensions")


def sample_workspace(rows: int, vocab: int) -> int:
    return _check(lib().skd_sample_workspace(rows, vocab), "skd_sample_workspace")


def sample(logits, u, tokens_out, temperature=None, top_k=None, top_p=None, min_p=None, workspace=None, stream: int = 0):
    """skd_sample on device tensors: logits [rows][vocab] float32 with dense rows, u and the parameters [rows] (None: off)."""
    if _dtype_of(logits) != "torch.float32" or logits.dim() != 2 or logits.stride(1) != 1:
        raise ValueError("expected float32 logits with dense rows")
    rows, vocab = logits.shape
    for t, dtype in ((u, "float32"), (tokens_out, "int32"), (temperature, "float32"), (top_k, "int32"), (top_p, "float32"), (min_p, "float32")):
        if t is not None:
            _expect(t, dtype, 1)
            if len(t) != rows:
                raise ValueError("one entry per row")
    p = Sampling(*[_ptr_of(a) for a in (temperature, top_k, top_p, min_p)])
    ws = (0, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    _check(lib().skd_sample(logits.data_ptr(), max(logits.stride(0), vocab) if rows < 2 else logits.stride(0), rows, vocab, C.byref(p), u.data_ptr(), tokens_out.data_ptr(), *ws,
                            stream), "skd_sample")
