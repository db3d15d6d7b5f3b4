"""Thin Python binding of the Block-GTQ C ABI (include/blockgtq.h).

Argument marshalling only: every step of the path runs in libblockgtq.so.
PyTorch provides device memory (tensors) and the stream.  The binding raises
if the library is missing or a call returns an error; there is no fallback.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
from dataclasses import dataclass

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libblockgtq.so")

BGTQ_FP32, BGTQ_BF16 = 0, 1
HEAD_DIM = 128
N_BLOCKS = 64
MAX_GROUPS = 8

EXPORTED = [
    "blockgtq_last_error", "blockgtq_energy_scores", "blockgtq_allocate", "blockgtq_codebook",
    "blockgtq_layout_bytes", "blockgtq_cache_bytes", "blockgtq_workspace_bytes",
    "blockgtq_layout_init", "blockgtq_quantize_append", "blockgtq_decode_attn",
    "blockgtq_decode_attn_fp16", "blockgtq_prefill_workspace_bytes", "blockgtq_prefill_attn",
    "blockgtq_window_bytes", "blockgtq_window_append", "blockgtq_protected_workspace_bytes",
    "blockgtq_decode_attn_protected", "blockgtq_rope_step_workspace_bytes", "blockgtq_rope_decode_step",
    "blockgtq_read_probe", "blockgtq_decode_attn_noalloc", "blockgtq_dequantize_rows",
    "blockgtq_cross_workspace_bytes", "blockgtq_cross_attn", "blockgtq_shared_workspace_bytes",
    "blockgtq_decode_attn_shared", "blockgtq_norm_rope", "blockgtq_paged_append", "blockgtq_paged_workspace_bytes",
    "blockgtq_paged_attn",
]


class BlockGTQError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"blockgtq error {code}: {msg}")
        self.code = code


class _Config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "n_layers", "batch", "n_kv_heads", "group", "head_dim", "capacity",
        "k_budget", "v_bits", "in_dtype")]


class _Cache(ctypes.Structure):
    _fields_ = [("k_codes", ctypes.c_void_p), ("k_norms", ctypes.c_void_p),
                ("v_codes", ctypes.c_void_p), ("v_norms", ctypes.c_void_p)]


class _Rope(ctypes.Structure):
    _fields_ = [("n_axes", ctypes.c_int32), ("axis", ctypes.c_uint8 * N_BLOCKS), ("theta", ctypes.c_double * N_BLOCKS)]


class _Chunk(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("cu_new", "ctx_len", "pages")] + [
        (n, ctypes.c_int32) for n in ("n_seqs", "n_tokens", "max_pages", "max_new", "max_ctx")]


class _Scores(ctypes.Structure):
    _fields_ = [("cap", ctypes.c_float), ("slopes", ctypes.c_void_p), ("prefix_len", ctypes.c_void_p)]


_lib_handle = None


def lib():
    """Load libblockgtq.so (built by paper_2606_24033_amd.build.build())."""
    global _lib_handle
    if _lib_handle is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing; run __graft_entry__.build() first")
        L = ctypes.CDLL(LIB_PATH)
        L.blockgtq_last_error.restype = ctypes.c_char_p
        P, I32, I64, SZ, F32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
        PSZ = ctypes.POINTER(ctypes.c_size_t)
        sig = {
            "blockgtq_energy_scores": [P, P, I32, I32, I32, P],
            "blockgtq_allocate": [P, I32, I32, I32, I32, I32, P],
            "blockgtq_codebook": [I32, P, P],
            "blockgtq_layout_bytes": [P, PSZ],
            "blockgtq_cache_bytes": [P, PSZ, PSZ, PSZ, PSZ],
            "blockgtq_workspace_bytes": [P, I32, I32, I32, PSZ],
            "blockgtq_layout_init": [P, P, P, P, P, P],
            "blockgtq_quantize_append": [P, P, I32, P, P, I32, P, P, P],
            "blockgtq_decode_attn": [P, P, I32, P, P, I32, P, P, P, SZ, I32, P],
            "blockgtq_decode_attn_fp16": [P, I32, P, P, I32, P, P, P, P, SZ, I32, P],
            "blockgtq_prefill_workspace_bytes": [P, I32, PSZ],
            "blockgtq_prefill_attn": [P, P, I32, P, I32, P, I32, P, P, P, SZ, P],
            "blockgtq_window_bytes": [P, I32, I32, PSZ],
            "blockgtq_window_append": [P, I32, P, P, I32, P, I32, I32, P, P],
            "blockgtq_protected_workspace_bytes": [P, I32, I32, I32, PSZ],
            "blockgtq_decode_attn_protected": [P, P, I32, P, P, I32, P, P, I32, I32, P, P, SZ, I32, P],
            "blockgtq_rope_step_workspace_bytes": [P, I32, I32, PSZ],
            "blockgtq_rope_decode_step": [P, P, ctypes.c_double, P, P, P, P, I32, P, P, P, SZ, I32, P],
            "blockgtq_read_probe": [P, SZ, P, P],
            "blockgtq_decode_attn_noalloc": [P, P, I32, P, P, I32, P, P, I32, P],
            "blockgtq_dequantize_rows": [P, P, I32, P, I32, P, P, P, P, I32, P],
            "blockgtq_cross_workspace_bytes": [P, I32, I32, I32, I32, PSZ],
            "blockgtq_cross_attn": [P, P, I32, P, I32, P, I32, P, P, I32, P, SZ, I32, P],
            "blockgtq_shared_workspace_bytes": [P, P, I32, I32, I32, I32, PSZ],
            "blockgtq_norm_rope": [P, P, I32, P, I64, P, I64, P, P, P, F32, P, I64, P, I64, I32, P],
            "blockgtq_paged_append": [P, P, I32, P, I64, P, I64, P, P, P],
            "blockgtq_paged_workspace_bytes": [P, I32, I32, I32, I32, I32, PSZ],
            "blockgtq_paged_attn": [P, P, I32, P, P, P, P, P, I32, P, SZ, I32, P],
            "blockgtq_decode_attn_shared": [P, P, I32, P, P, P, P, I32, P, I32, P, P, I32, P, SZ, I32, P],
        }
        for name, args in sig.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = ctypes.c_int
        _lib_handle = L
    return _lib_handle


def _check(rc):
    if rc != 0:
        raise BlockGTQError(rc, lib().blockgtq_last_error().decode())


def _ptr(a):
    if a is None:
        return None
    if isinstance(a, np.ndarray):
        return a.ctypes.data_as(ctypes.c_void_p)
    return ctypes.c_void_p(a.data_ptr())


@dataclass
class Config:
    n_layers: int
    batch: int
    n_kv_heads: int
    group: int
    capacity: int
    k_budget: int
    v_bits: int
    in_dtype: int = BGTQ_BF16
    head_dim: int = HEAD_DIM

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        self.__dict__.pop("_made", None)  # (behind the field: a call of another thread in between makes what it pops)

    def _make(self):
        """What the calls need of the fields, made again after one is set: the C struct, and the cache tensors' shapes."""
        while True:
            layers, batch, kv, group, dim, C, budget, v_bits, dtype = was = self._fields()
            lead = (layers, batch, kv)
            made = (_Config(layers, batch, kv, group, dim, C, budget, v_bits, dtype),
                    (lead + (C, self.k_words), lead + (C * MAX_GROUPS,), lead + (C // 32, HEAD_DIM, v_bits), lead + (C,)))
            self.__dict__["_made"] = made
            if self._fields() == was:  # (else another thread has set one meanwhile, and popped what was there before)
                return made

    def _fields(self):
        return (self.n_layers, self.batch, self.n_kv_heads, self.group, self.head_dim, self.capacity, self.k_budget, self.v_bits,
                self.in_dtype)

    def __getstate__(self):
        return {k: v for k, v in self.__dict__.items() if k != "_made"}

    def c(self):
        return (self.__dict__.get("_made") or self._make())[0]

    @property
    def n_q_heads(self):
        return self.n_kv_heads * self.group

    @property
    def k_words(self):
        return (2 * self.k_budget + 31) // 32


def _stream(stream):
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


# ----------------------------------------------------------------- host calls

def blockgtq_energy_scores(q_cal: np.ndarray, k_cal: np.ndarray) -> np.ndarray:
    q = np.ascontiguousarray(q_cal, dtype=np.float32)
    k = np.ascontiguousarray(k_cal, dtype=np.float32)
    n, g, d = q.shape
    out = np.zeros(d // 2, dtype=np.float64)
    _check(lib().blockgtq_energy_scores(_ptr(q), _ptr(k), n, g, d, _ptr(out)))
    return out


def blockgtq_allocate(scores: np.ndarray, budget: int, b_min: int = 1, b_max: int = 8) -> np.ndarray:
    s = np.ascontiguousarray(np.atleast_2d(scores), dtype=np.float64)
    out = np.zeros(s.shape, dtype=np.uint8)
    _check(lib().blockgtq_allocate(_ptr(s), s.shape[0], s.shape[1], budget, b_min, b_max, _ptr(out)))
    return out


def blockgtq_codebook(b: int):
    c16 = np.zeros(1 << b, dtype=np.uint16)
    thr = np.zeros((1 << b) - 1, dtype=np.float32)
    _check(lib().blockgtq_codebook(b, _ptr(c16), _ptr(thr)))
    return c16.view(np.float16), thr


def cache_bytes(cfg: Config):
    vals = [ctypes.c_size_t() for _ in range(4)]
    _check(lib().blockgtq_cache_bytes(ctypes.byref(cfg.c()), *[ctypes.byref(v) for v in vals]))
    return [v.value for v in vals]


def workspace_bytes(cfg: Config, n_layers_in_call: int, n_splits: int, max_ctx: int) -> int:
    v = ctypes.c_size_t()
    _check(lib().blockgtq_workspace_bytes(ctypes.byref(cfg.c()), n_layers_in_call, n_splits, max_ctx,
                                          ctypes.byref(v)))
    return v.value


# ---------------------------------------------------------------- device state

class Layout:
    """Device layout blob (rotations, codebooks, per-head grouping tables)."""

    def __init__(self, cfg: Config, k_bits: np.ndarray, rot_k_flat: np.ndarray, rot_v: np.ndarray,
                 device="cuda", stream=None):
        import torch
        n = ctypes.c_size_t()
        _check(lib().blockgtq_layout_bytes(ctypes.byref(cfg.c()), ctypes.byref(n)))
        self.blob = torch.empty(n.value, dtype=torch.uint8, device=device)
        bits = np.ascontiguousarray(k_bits, dtype=np.uint8).reshape(cfg.n_layers * cfg.n_kv_heads, N_BLOCKS)
        rk = np.ascontiguousarray(rot_k_flat, dtype=np.float32)
        rv = np.ascontiguousarray(rot_v, dtype=np.float32)
        _check(lib().blockgtq_layout_init(ctypes.byref(cfg.c()), _ptr(bits), _ptr(rk), _ptr(rv),
                                          _ptr(self.blob), _stream(stream)))
        self.k_bits = bits
        self.k_budget = cfg.k_budget


class Cache:
    """The packed cache (zero-filled torch tensors in the documented layout)."""

    def __init__(self, cfg: Config, device="cuda"):
        import torch
        L, B, H, C = cfg.n_layers, cfg.batch, cfg.n_kv_heads, cfg.capacity
        self.k_codes = torch.zeros((L, B, H, C, cfg.k_words), dtype=torch.int32, device=device)
        self.k_norms = torch.zeros((L, B, H, C * MAX_GROUPS), dtype=torch.float16, device=device)
        self.v_codes = torch.zeros((L, B, H, C // 32, HEAD_DIM, cfg.v_bits), dtype=torch.int32, device=device)
        self.v_norms = torch.zeros((L, B, H, C), dtype=torch.float16, device=device)

    def c(self):
        return _Cache(self.k_codes.data_ptr(), self.k_norms.data_ptr(), self.v_codes.data_ptr(),
                      self.v_norms.data_ptr())

    def nbytes_used(self, cfg: Config, n_groups_per_row: np.ndarray, tokens: int) -> int:
        """Bytes of codes and norms for `tokens` rows of every (layer, seq, head)."""
        per_row = cfg.k_words * 4 + HEAD_DIM * cfg.v_bits // 8 + 2
        rows = cfg.batch * tokens
        return int(rows * (per_row * cfg.n_layers * cfg.n_kv_heads + 2 * int(np.sum(n_groups_per_row))))


def _check_dev(t, dtype=None):
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("device tensors must be contiguous CUDA tensors")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"expected {dtype}, got {t.dtype}")


def _in_dtype(cfg):
    import torch
    return torch.bfloat16 if cfg.in_dtype == BGTQ_BF16 else torch.float32


def blockgtq_quantize_append(cfg: Config, layout: Layout, layer: int, k, v, write_pos, cache: Cache,
                             stream=None, host_write_pos=None):
    """Append n_new rows per sequence.  k, v: [batch, n_new, H_kv, 128] (or with a
    leading layer dim for layer == -1).  write_pos: int32 device tensor [batch].
    host_write_pos (optional list) lets the binding check the capacity bound."""
    import torch
    for t in (k, v):
        _check_dev(t, _in_dtype(cfg))
    _check_dev(write_pos, torch.int32)
    n_new = k.shape[-3]
    if host_write_pos is not None and max(host_write_pos) + n_new > cfg.capacity:
        raise BlockGTQError(-3, "append beyond capacity")
    _check(lib().blockgtq_quantize_append(ctypes.byref(cfg.c()), _ptr(layout.blob), layer, _ptr(k), _ptr(v),
                                          n_new, _ptr(write_pos), ctypes.byref(cache.c()), _stream(stream)))


def blockgtq_decode_attn(cfg: Config, layout: Layout, layer: int, q, ctx_len, max_ctx: int, cache: Cache,
                         out=None, workspace=None, n_splits: int = 0, stream=None):
    import torch
    _check_dev(q, _in_dtype(cfg))
    _check_dev(ctx_len, torch.int32)
    n_lc = cfg.n_layers if layer < 0 else 1
    if out is None:
        out = torch.empty(q.shape, dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = torch.zeros(workspace_bytes(cfg, n_lc, n_splits, max_ctx), dtype=torch.uint8, device=q.device)
    _check(lib().blockgtq_decode_attn(ctypes.byref(cfg.c()), _ptr(layout.blob), layer, _ptr(q), _ptr(ctx_len),
                                      max_ctx, ctypes.byref(cache.c()), _ptr(out), _ptr(workspace),
                                      workspace.numel(), n_splits, _stream(stream)))
    return out


def blockgtq_decode_attn_noalloc(cfg: Config, layout: Layout, layer: int, q, ctx_len, max_ctx: int, cache: Cache,
                                 out, n_splits: int = 0, stream=None):
    """blockgtq_decode_attn with its workspace in the library's static device
    array (no allocation in the call; `out` is the caller's)."""
    import torch
    _check_dev(q, _in_dtype(cfg))
    _check_dev(ctx_len, torch.int32)
    _check_dev(out, torch.float32)
    _check(lib().blockgtq_decode_attn_noalloc(ctypes.byref(cfg.c()), _ptr(layout.blob), layer, _ptr(q),
                                              _ptr(ctx_len), max_ctx, ctypes.byref(cache.c()), _ptr(out), n_splits,
                                              _stream(stream)))
    return out


def blockgtq_decode_attn_fp16(cfg: Config, layer: int, q, ctx_len, max_ctx: int, k16, v16, out=None,
                              workspace=None, n_splits: int = 0, stream=None):
    import torch
    _check_dev(q, _in_dtype(cfg))
    _check_dev(ctx_len, torch.int32)
    _check_dev(k16, torch.float16)
    _check_dev(v16, torch.float16)
    n_lc = cfg.n_layers if layer < 0 else 1
    if out is None:
        out = torch.empty(q.shape, dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = torch.zeros(workspace_bytes(cfg, n_lc, n_splits, max_ctx), dtype=torch.uint8, device=q.device)
    _check(lib().blockgtq_decode_attn_fp16(ctypes.byref(cfg.c()), layer, _ptr(q), _ptr(ctx_len), max_ctx,
                                           _ptr(k16), _ptr(v16), _ptr(out), _ptr(workspace), workspace.numel(),
                                           n_splits, _stream(stream)))
    return out


def prefill_workspace_bytes(cfg: Config, n_q: int) -> int:
    v = ctypes.c_size_t()
    _check(lib().blockgtq_prefill_workspace_bytes(ctypes.byref(cfg.c()), n_q, ctypes.byref(v)))
    return v.value


def blockgtq_prefill_attn(cfg: Config, layout: Layout, layer: int, q, q_pos0, max_pos: int, cache: Cache,
                          out=None, workspace=None, stream=None):
    """Causal prefill attention of one layer.  q: [batch, n_q, Hq, 128] in the
    config's input dtype; q_pos0: int32 device tensor [batch] (position of
    query 0 of each sequence); max_pos: host bound of q_pos0 + n_q - 1."""
    import torch
    _check_dev(q, _in_dtype(cfg))
    _check_dev(q_pos0, torch.int32)
    n_q = q.shape[1]
    if out is None:
        out = torch.empty(q.shape, dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = torch.empty(max(prefill_workspace_bytes(cfg, n_q), 1), dtype=torch.uint8, device=q.device)
    _check(lib().blockgtq_prefill_attn(ctypes.byref(cfg.c()), _ptr(layout.blob), layer, _ptr(q), n_q, _ptr(q_pos0),
                                       max_pos, ctypes.byref(cache.c()), _ptr(out), _ptr(workspace),
                                       workspace.numel(), _stream(stream)))
    return out


# ---------------------------------------------------------------- protected fp16 window

def window_bytes(cfg: Config, n_sink: int, n_recent: int) -> int:
    v = ctypes.c_size_t()
    _check(lib().blockgtq_window_bytes(ctypes.byref(cfg.c()), n_sink, n_recent, ctypes.byref(v)))
    return v.value


def protected_workspace_bytes(cfg: Config, n_layers_in_call: int, n_splits: int, max_ctx: int) -> int:
    v = ctypes.c_size_t()
    _check(lib().blockgtq_protected_workspace_bytes(ctypes.byref(cfg.c()), n_layers_in_call, n_splits, max_ctx,
                                                    ctypes.byref(v)))
    return v.value


def blockgtq_window_append(cfg: Config, layer: int, k, v, write_pos, n_sink: int, n_recent: int, window,
                           stream=None):
    """fp16 copies of appended rows into the window (same k, v, write_pos as
    blockgtq_quantize_append).  window: fp16 device tensor of window_bytes."""
    import torch
    for t in (k, v):
        _check_dev(t, _in_dtype(cfg))
    _check_dev(write_pos, torch.int32)
    _check_dev(window, torch.float16)
    if window.numel() * 2 < window_bytes(cfg, n_sink, n_recent):
        raise BlockGTQError(-1, "window tensor too small")
    _check(lib().blockgtq_window_append(ctypes.byref(cfg.c()), layer, _ptr(k), _ptr(v), k.shape[-3], _ptr(write_pos),
                                        n_sink, n_recent, _ptr(window), _stream(stream)))


def blockgtq_decode_attn_protected(cfg: Config, layout: Layout, layer: int, q, ctx_len, max_ctx: int, cache: Cache,
                                   window, n_sink: int, n_recent: int, out=None, workspace=None, n_splits: int = 0,
                                   stream=None):
    import torch
    _check_dev(q, _in_dtype(cfg))
    _check_dev(ctx_len, torch.int32)
    _check_dev(window, torch.float16)
    if window.numel() * 2 < window_bytes(cfg, n_sink, n_recent):
        raise BlockGTQError(-1, "window tensor too small")
    n_lc = cfg.n_layers if layer < 0 else 1
    if out is None:
        out = torch.empty(q.shape, dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = torch.zeros(protected_workspace_bytes(cfg, n_lc, n_splits, max_ctx), dtype=torch.uint8,
                                device=q.device)
    _check(lib().blockgtq_decode_attn_protected(ctypes.byref(cfg.c()), _ptr(layout.blob), layer, _ptr(q),
                                                _ptr(ctx_len), max_ctx, ctypes.byref(cache.c()), _ptr(window),
                                                n_sink, n_recent, _ptr(out), _ptr(workspace), workspace.numel(),
                                                n_splits, _stream(stream)))
    return out


# ---------------------------------------------------------------- decode step from pre-RoPE inputs

def rope_step_workspace_bytes(cfg: Config, max_ctx: int, n_splits: int = 0) -> int:
    v = ctypes.c_size_t()
    _check(lib().blockgtq_rope_step_workspace_bytes(ctypes.byref(cfg.c()), max_ctx, n_splits, ctypes.byref(v)))
    return v.value


def blockgtq_rope_decode_step(cfg: Config, layout: Layout, rope_base: float, q_pre, k_pre, v, pos, max_ctx: int,
                              cache: Cache, out=None, workspace=None, n_splits: int = 0, stream=None):
    """One all-layer decode step from pre-RoPE q [L, B, Hq, 128] and k, v
    [L, B, 1, H_kv, 128] (in_dtype) at device positions pos (int32 [B])."""
    import torch
    for t in (q_pre, k_pre, v):
        _check_dev(t, _in_dtype(cfg))
    _check_dev(pos, torch.int32)
    if out is None:
        out = torch.empty(q_pre.shape, dtype=torch.float32, device=q_pre.device)
    if workspace is None:
        workspace = torch.zeros(rope_step_workspace_bytes(cfg, max_ctx, n_splits), dtype=torch.uint8,
                                device=q_pre.device)
    _check(lib().blockgtq_rope_decode_step(ctypes.byref(cfg.c()), _ptr(layout.blob), float(rope_base), _ptr(q_pre),
                                           _ptr(k_pre), _ptr(v), _ptr(pos), max_ctx, ctypes.byref(cache.c()),
                                           _ptr(out), _ptr(workspace), workspace.numel(), n_splits,
                                           _stream(stream)))
    return out


# ---------------------------------------------------------------- packed rows read by other callers

def _check_shape(what, t, shape, dtype):
    if t.shape != shape or t.dtype != dtype:
        raise ValueError(f"{what}: expected {tuple(shape)} of {dtype}, got {tuple(t.shape)} of {t.dtype}")


def _cache_tensors(cfg: Config, cache: Cache, what="cache"):
    import torch
    shapes = (cfg.__dict__.get("_made") or cfg._make())[1]
    t = (cache.k_codes, cache.k_norms, cache.v_codes, cache.v_norms)
    i32, f16 = torch.int32, torch.float16
    if not (t[0].shape == shapes[0] and t[1].shape == shapes[1] and t[2].shape == shapes[2] and t[3].shape == shapes[3] and
            t[0].dtype == t[2].dtype == i32 and t[1].dtype == t[3].dtype == f16):
        for name, x, shape, dtype in zip(("k_codes", "k_norms", "v_codes", "v_norms"), t, shapes, (i32, f16, i32, f16)):
            _check_shape(f"{what}.{name}", x, shape, dtype)
    return t


def _check_layout(cfg: Config, layout: Layout):
    rows = cfg.n_layers * cfg.n_kv_heads
    if layout.k_bits.shape[0] != rows or layout.k_budget != cfg.k_budget:
        raise ValueError(f"layout of {layout.k_bits.shape[0]} (layer, head) rows with a key budget of {layout.k_budget}, "
                         f"the configuration has {rows} with {cfg.k_budget}")


def _on(stream):
    """Where a call allocates: on the stream it runs on, so that what is filled
    there is filled before, and what is freed there is reused after it."""
    import torch
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _call(fn, stream, args, *tensors, rows=()):
    """fn(*args, stream) on the one GPU that holds all the tensors (None is
    skipped), whichever is current: on `stream`, or that GPU's current one.
    `rows`: tensors whose strides the call takes."""
    import torch
    tensors = [t for t in tensors if t is not None]
    for t in tensors:
        if not t.is_contiguous():
            raise ValueError("device tensors must be contiguous CUDA tensors")
    tensors += [t for t in rows if t is not None]
    d = tensors[0].get_device()
    if stream is not None and stream.device_index != d:
        raise ValueError(f"a stream of device {stream.device_index} for tensors on device {d}")
    for t in tensors:
        on = t.get_device()
        if on < 0:
            raise ValueError("device tensors must be contiguous CUDA tensors")
        if on != d:
            raise ValueError("tensors on different devices: " + ", ".join(sorted({str(x.device) for x in tensors})))
    if torch._C._cuda_getDevice() == d:
        _check(fn(*args, torch._C._cuda_getCurrentRawStream(d) if stream is None else stream.cuda_stream))
        return
    with torch.cuda.device(d):
        _check(fn(*args, torch._C._cuda_getCurrentRawStream(d) if stream is None else stream.cuda_stream))


def _at(t):
    return None if t is None else t.data_ptr()


def _out_type(dtype):
    import torch
    if dtype not in (torch.float32, torch.bfloat16):
        raise ValueError(f"output dtype {dtype}: torch.float32 or torch.bfloat16")
    return BGTQ_BF16 if dtype == torch.bfloat16 else BGTQ_FP32


def _lead(cfg, layer):
    """Leading dimensions of a call's tensors: a layer dimension for all layers."""
    return (cfg.n_layers, cfg.batch) if layer < 0 else (cfg.batch,)


def blockgtq_dequantize_rows(cfg: Config, layout: Layout, layer: int, cache: Cache, read_pos, n_rows: int, ctx_len=None,
                             k_out=None, v_out=None, out_dtype=None, stream=None):
    """Rows read_pos[b] .. + n_rows - 1 of each sequence as plain keys and values
    [batch, n_rows, H_kv, 128] (with a leading layer dim for layer == -1).
    Rows outside the cache or at or past ctx_len[b] are left as they were in
    k_out / v_out.  With only one of k_out and v_out given, only that one is
    read; with neither, both are allocated (zeros; out_dtype, fp32 by default).
    Returns (k_out, v_out)."""
    import torch
    _check_layout(cfg, layout)
    _check_shape("read_pos", read_pos, (cfg.batch,), torch.int32)
    if ctx_len is not None:
        _check_shape("ctx_len", ctx_len, (cfg.batch,), torch.int32)
    shape = _lead(cfg, layer) + (max(n_rows, 0), cfg.n_kv_heads, HEAD_DIM)
    if k_out is None and v_out is None:
        with _on(stream):
            k_out, v_out = (torch.zeros(shape, dtype=out_dtype or torch.float32, device=read_pos.device) for _ in range(2))
    dtype = (v_out if k_out is None else k_out).dtype
    if out_dtype is not None and dtype != out_dtype:
        raise ValueError(f"out_dtype {out_dtype}, but the outputs are {dtype}")
    for name, t in (("k_out", k_out), ("v_out", v_out)):
        if t is not None:
            _check_shape(name, t, shape, dtype)
    _call(lib().blockgtq_dequantize_rows, stream,
          (ctypes.byref(cfg.c()), layout.blob.data_ptr(), layer, ctypes.byref(cache.c()), n_rows, read_pos.data_ptr(),
           _at(ctx_len), _at(k_out), _at(v_out), _out_type(dtype)),
          read_pos, layout.blob, ctx_len, k_out, v_out, *_cache_tensors(cfg, cache))
    return k_out, v_out


def cross_workspace_bytes(cfg: Config, n_layers_in_call: int, n_q: int, n_splits: int, max_ctx: int) -> int:
    v = ctypes.c_size_t()
    _check(lib().blockgtq_cross_workspace_bytes(ctypes.byref(cfg.c()), n_layers_in_call, n_q, n_splits, max_ctx,
                                                ctypes.byref(v)))
    return v.value


def shared_workspace_bytes(cfg: Config, prefix_cfg: Config, n_layers_in_call: int, n_splits: int, max_prefix: int,
                           max_ctx: int) -> int:
    v = ctypes.c_size_t()
    _check(lib().blockgtq_shared_workspace_bytes(ctypes.byref(cfg.c()), ctypes.byref(prefix_cfg.c()), n_layers_in_call,
                                                 n_splits, max_prefix, max_ctx, ctypes.byref(v)))
    return v.value


def _out_of(q, out, out_dtype, stream):
    import torch
    if out is None:
        with _on(stream):
            out = torch.empty(q.shape, dtype=out_dtype or torch.float32, device=q.device)
    elif out_dtype is not None and out.dtype != out_dtype:
        raise ValueError(f"out_dtype {out_dtype}, but out is {out.dtype}")
    _check_shape("out", out, q.shape, out.dtype)
    return out, _out_type(out.dtype)


def blockgtq_cross_attn(cfg: Config, layout: Layout, layer: int, q, ctx_len, max_ctx: int, cache: Cache, out=None,
                        workspace=None, n_splits: int = 0, out_dtype=None, stream=None):
    """q [batch, n_q, Hq, 128] (with a leading layer dim for layer == -1), every
    query row attending rows [0, ctx_len[b]) of its sequence's packed cache.
    Returns out, of q's shape in out's or out_dtype (fp32 by default)."""
    import torch
    _check_layout(cfg, layout)
    n_lc = cfg.n_layers if layer < 0 else 1
    lead = _lead(cfg, layer)
    if q.dim() != len(lead) + 3:
        raise ValueError(f"q: expected {lead + ('n_q', cfg.n_q_heads, HEAD_DIM)}, got {tuple(q.shape)}")
    n_q = q.shape[len(lead)]
    _check_shape("q", q, lead + (n_q, cfg.n_q_heads, HEAD_DIM), _in_dtype(cfg))
    _check_shape("ctx_len", ctx_len, (cfg.batch,), torch.int32)
    out, kind = _out_of(q, out, out_dtype, stream)
    if workspace is None:
        with _on(stream):
            workspace = torch.empty(max(cross_workspace_bytes(cfg, n_lc, n_q, n_splits, max_ctx), 1), dtype=torch.uint8,
                                    device=q.device)
    _call(lib().blockgtq_cross_attn, stream,
          (ctypes.byref(cfg.c()), layout.blob.data_ptr(), layer, q.data_ptr(), n_q, ctx_len.data_ptr(), max_ctx,
           ctypes.byref(cache.c()), out.data_ptr(), kind, workspace.data_ptr(),
           workspace.numel() * workspace.element_size(), n_splits),
          q, layout.blob, ctx_len, out, workspace, *_cache_tensors(cfg, cache))
    return out


def blockgtq_decode_attn_shared(cfg: Config, layout: Layout, layer: int, q, prefix_cfg: Config, prefix: Cache, prefix_len,
                                max_prefix: int, ctx_len, max_ctx: int, cache: Cache, out=None, workspace=None,
                                n_splits: int = 0, out_dtype=None, stream=None):
    """One decode step of a batch behind one packed prefix: q [batch, Hq, 128]
    (with a leading layer dim for layer == -1) against rows [0, prefix_len[0])
    of `prefix` and rows [0, ctx_len[b]) of the sequence's own cache, one
    softmax.  prefix_cfg: cfg with batch 1 and the prefix cache's capacity.
    Returns out, of q's shape in out's or out_dtype (fp32 by default)."""
    import torch
    _check_layout(cfg, layout)
    n_lc = cfg.n_layers if layer < 0 else 1
    _check_shape("q", q, _lead(cfg, layer) + (cfg.n_q_heads, HEAD_DIM), _in_dtype(cfg))
    _check_shape("ctx_len", ctx_len, (cfg.batch,), torch.int32)
    _check_shape("prefix_len", prefix_len, (1,), torch.int32)
    out, kind = _out_of(q, out, out_dtype, stream)
    if workspace is None:
        with _on(stream):
            workspace = torch.empty(shared_workspace_bytes(cfg, prefix_cfg, n_lc, n_splits, max_prefix, max_ctx),
                                    dtype=torch.uint8, device=q.device)
    _call(lib().blockgtq_decode_attn_shared, stream,
          (ctypes.byref(cfg.c()), layout.blob.data_ptr(), layer, q.data_ptr(), ctypes.byref(prefix_cfg.c()),
           ctypes.byref(prefix.c()), prefix_len.data_ptr(), max_prefix, ctx_len.data_ptr(), max_ctx,
           ctypes.byref(cache.c()), out.data_ptr(), kind, workspace.data_ptr(),
           workspace.numel() * workspace.element_size(), n_splits),
          q, layout.blob, prefix_len, ctx_len, out, workspace, *_cache_tensors(cfg, cache),
          *_cache_tensors(prefix_cfg, prefix, "prefix"))
    return out


# ---------------------------------------------------------------- a serving step over pages

class Rope:
    """Rotation of a head's 64 blocks: radians per position of each, and the
    position (of a token's `n_axes`) that each turns with (the only one by default)."""

    def __init__(self, theta, axis=None, n_axes: int | None = None):
        axis = [0] * N_BLOCKS if axis is None else [int(a) for a in axis]
        theta = [float(t) for t in theta]
        if len(theta) != N_BLOCKS or len(axis) != N_BLOCKS or not all(0 <= a < 256 for a in axis):
            raise ValueError(f"a Rope needs {N_BLOCKS} thetas and as many axes")
        self.n_axes = max(axis) + 1 if n_axes is None else n_axes
        self._c = _Rope(self.n_axes, (ctypes.c_uint8 * N_BLOCKS)(*axis), (ctypes.c_double * N_BLOCKS)(*theta))

    def c(self):
        return self._c


def _token_rows(what, t, n, heads, dtype):
    """The token stride of [n, heads, 128] rows (a view of wider rows, too)."""
    if t.shape != (n, heads, HEAD_DIM) or t.dtype != dtype:
        _check_shape(what, t, (n, heads, HEAD_DIM), dtype)
    by = t.stride()
    if by[2] != 1 or (by[1] != HEAD_DIM and heads > 1):
        raise ValueError(f"{what}: the heads of a token must lie one after the other")
    return by[0] if n > 1 else heads * HEAD_DIM


def blockgtq_norm_rope(cfg: Config, rope: Rope, q, k, pos, q_weight=None, k_weight=None, eps: float = 1e-6, q_out=None,
                       k_out=None, out_dtype=None, stream=None):
    """q [n_tokens, Hq, 128] and k [n_tokens, H_kv, 128] (either may be None; the
    token stride is free), each head normed where its weight (fp32 [128]) is given
    and rotated at pos (int32 [n_tokens, n_axes]).  Returns (q_out, k_out), in the
    outputs' or out_dtype (the inputs' by default); an output may be its input."""
    import torch
    if q is None and k is None:
        raise ValueError("neither q nor k")
    if (q is None and q_out is not None) or (k is None and k_out is not None):
        raise ValueError("an output without its input")
    n = (k if q is None else q).shape[0]
    _check_shape("pos", pos, (n, rope.n_axes), torch.int32)
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w is not None:
            _check_shape(name, w, (HEAD_DIM,), torch.float32)
    given = k_out if q_out is None else q_out
    in_dtype = _in_dtype(cfg)
    dtype = given.dtype if given is not None else out_dtype or in_dtype
    if out_dtype is not None and out_dtype != dtype:
        raise ValueError(f"out_dtype {out_dtype}, but the outputs are {dtype}")
    if (q is not None and q_out is None) or (k is not None and k_out is None):
        with _on(stream):
            if q is not None and q_out is None:
                q_out = torch.empty(q.shape, dtype=dtype, device=q.device)
            if k is not None and k_out is None:
                k_out = torch.empty(k.shape, dtype=dtype, device=k.device)
    hk, qs, ks, qos, kos = cfg.n_kv_heads, 0, 0, 0, 0
    if q is not None:
        qs, qos = _token_rows("q", q, n, hk * cfg.group, in_dtype), _token_rows("q_out", q_out, n, hk * cfg.group, dtype)
    if k is not None:
        ks, kos = _token_rows("k", k, n, hk, in_dtype), _token_rows("k_out", k_out, n, hk, dtype)
    _call(lib().blockgtq_norm_rope, stream,
          (ctypes.byref(cfg.c()), ctypes.byref(rope.c()), n, _at(q), qs, _at(k), ks, pos.data_ptr(), _at(q_weight), _at(k_weight),
           eps, _at(q_out), qos, _at(k_out), kos, _out_type(dtype)),
          pos, q_weight, k_weight, rows=(q, k, q_out, k_out))
    return q_out, k_out


class Chunk:
    """What one serving step adds to a ragged batch over pages: int32 device
    tensors cu_new [n_seqs + 1] (each sequence's new tokens among the call's
    rows), ctx_len [n_seqs] (its rows with the new ones) and pages [n_seqs,
    max_pages], and the host's bounds of a sequence's new tokens and rows."""

    def __init__(self, cu_new, ctx_len, pages, max_new: int, max_ctx: int):
        import torch
        n = ctx_len.shape[0]
        _check_shape("ctx_len", ctx_len, (n,), torch.int32)
        _check_shape("cu_new", cu_new, (n + 1,), torch.int32)
        if pages.dim() != 2:
            raise ValueError(f"pages: expected [{n}, max_pages], got {tuple(pages.shape)}")
        _check_shape("pages", pages, (n, pages.shape[1]), torch.int32)
        self.cu_new, self.ctx_len, self.pages, self.max_new, self.max_ctx = cu_new, ctx_len, pages, max_new, max_ctx
        self.n_seqs = n

    def c(self, n_tokens: int):
        return _Chunk(self.cu_new.data_ptr(), self.ctx_len.data_ptr(), self.pages.data_ptr(), self.n_seqs, n_tokens,
                      self.pages.shape[1], self.max_new, self.max_ctx)

    def tensors(self):
        return self.cu_new, self.ctx_len, self.pages


def blockgtq_paged_append(cfg: Config, layout: Layout, layer: int, k, v, chunk: Chunk, cache: Cache, stream=None):
    """Quantizes and packs the chunk's rows k, v [n_tokens, H_kv, 128] (token
    strides free) of one layer into the sequences' pages.  cache: the pool,
    cfg.batch pages of cfg.capacity rows."""
    _check_layout(cfg, layout)
    n = k.shape[0]
    strides = [_token_rows(name, t, n, cfg.n_kv_heads, _in_dtype(cfg)) for name, t in (("k", k), ("v", v))]
    _call(lib().blockgtq_paged_append, stream,
          (ctypes.byref(cfg.c()), layout.blob.data_ptr(), layer, k.data_ptr(), strides[0], v.data_ptr(), strides[1],
           ctypes.byref(chunk.c(n)), ctypes.byref(cache.c())),
          layout.blob, *chunk.tensors(), *_cache_tensors(cfg, cache), rows=(k, v))


def paged_workspace_bytes(cfg: Config, chunk: Chunk, n_tokens: int, n_splits: int = 0) -> int:
    v = ctypes.c_size_t()
    _check(lib().blockgtq_paged_workspace_bytes(ctypes.byref(cfg.c()), chunk.n_seqs, n_tokens, chunk.max_new, chunk.max_ctx,
                                                n_splits, ctypes.byref(v)))
    return v.value


def blockgtq_paged_attn(cfg: Config, layout: Layout, layer: int, q, chunk: Chunk, cache: Cache, cap: float = 0.0,
                        slopes=None, prefix=None, out=None, workspace=None, n_splits: int = 0, out_dtype=None, stream=None):
    """q [n_tokens, Hq, 128], the chunk's tokens, each attending the rows of its
    sequence up to its own position and the first prefix[s] ones (int32 [n_seqs]);
    cap: logits capped by cap tanh(x / cap); slopes (fp32 [Hq]): a bias of
    -slopes[h] |position - row|.  Returns out, of q's shape in out's or out_dtype
    (fp32 by default)."""
    import torch
    _check_layout(cfg, layout)
    n = q.shape[0]
    _check_shape("q", q, (n, cfg.n_q_heads, HEAD_DIM), _in_dtype(cfg))
    if slopes is not None:
        _check_shape("slopes", slopes, (cfg.n_q_heads,), torch.float32)
    if prefix is not None:
        _check_shape("prefix", prefix, (chunk.n_seqs,), torch.int32)
    out, kind = _out_of(q, out, out_dtype, stream)
    if workspace is None:
        with _on(stream):
            workspace = torch.empty(max(paged_workspace_bytes(cfg, chunk, n, n_splits), 1), dtype=torch.uint8, device=q.device)
    scores = _Scores(cap, _at(slopes), _at(prefix))
    _call(lib().blockgtq_paged_attn, stream,
          (ctypes.byref(cfg.c()), layout.blob.data_ptr(), layer, q.data_ptr(), ctypes.byref(chunk.c(n)), ctypes.byref(scores),
           ctypes.byref(cache.c()), out.data_ptr(), kind, workspace.data_ptr(),
           workspace.numel() * workspace.element_size(), n_splits),
          q, layout.blob, out, workspace, slopes, prefix, *chunk.tensors(), *_cache_tensors(cfg, cache))
    return out


def blockgtq_read_probe(src, sink, stream=None):
    """Stream-read every byte of the device tensor `src` (measurement helper)."""
    _check_dev(src)
    _check(lib().blockgtq_read_probe(_ptr(src), src.numel() * src.element_size(), _ptr(sink), _stream(stream)))

