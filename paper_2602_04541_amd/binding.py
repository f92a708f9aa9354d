"""Thin ctypes binding of liblychee.so: argument marshalling only.

Function names and argument order follow include/lychee.h.  Tensors are torch tensors used
purely as device-memory handles (`data_ptr()`); the stream is torch's current HIP stream
unless one is given.  If the shared library is missing the import of this module fails
loudly: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblychee.so")

OK, EINVAL, EUNSUPPORTED, EWORKSPACE, EHIP, EARENA = 0, -1, -2, -3, -4, -5
KERNEL_STREAM, KERNEL_GATHER, KERNEL_THRESHOLD, KERNEL_SELECT, KERNEL_COMBINE = 0, 1, 2, 3, 4
N_KERNEL_CLASSES = 5
OPT_DEFAULTS = 0
OPT_SELECT_LEAD = 10
OPT_WAIT_POLLS = 11
STATIC_SCRATCH_BYTES = 32 << 20
Q4_TILE_TOKENS, Q4_TILE_BYTES, Q4_MAX_GROUP = 16, 2176, 16
OPT_WG_PER_CU, OPT_STEP_MODE, OPT_GATHER_BLOCK, OPT_N_WG, OPT_TAIL_PERMILLE, OPT_SELECT_MARGIN = 1, 2, 6, 7, 8, 9
STEP_PHASED, STEP_LAYERWISE = 1, 0
RULE_THRESHOLD, RULE_TOP_P = 1, 2

EXPORTS = [
    "lychee_create", "lychee_destroy", "lychee_check_shape", "lychee_workspace_bytes",
    "lychee_step_workspace_bytes",
    "lychee_decode_attn", "lychee_decode_attn_static", "lychee_decode_attn_deferred", "lychee_select_flush",
    "lychee_dense_decode_attn", "lychee_decode_step",
    "lychee_dense_decode_step", "lychee_decode_step_append", "lychee_append_kv", "lychee_select_stats",
    "lychee_wait_timeouts",
    "lychee_validate_idx", "lychee_set_option", "lychee_timing_enable",
    "lychee_timing_read", "lychee_probe_read", "lychee_probe_copy", "lychee_strerror",
    "lychee_check_paged", "lychee_paged_workspace_bytes", "lychee_release_pages", "lychee_plan_pages",
    "lychee_q4_append", "lychee_q4_read", "lychee_q4_decode_attn", "lychee_select_scores",
]


class Shape(ctypes.Structure):
    """Mirror of `lychee_shape`."""
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("max_len", ctypes.c_int32), ("k", ctypes.c_int32),
                ("kv_stride_batch", ctypes.c_int64), ("kv_stride_head", ctypes.c_int64),
                ("kv_stride_tok", ctypes.c_int64), ("keep_ppm", ctypes.c_int32),
                ("block_size", ctypes.c_int32), ("prob_rule", ctypes.c_int32),
                ("prob_param", ctypes.c_float)]


class Paged(ctypes.Structure):
    """Mirror of `lychee_paged`."""
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("table_stride", ctypes.c_int32), ("page_tiles", ctypes.c_int32),
                ("k", ctypes.c_int32)]


class LycheeError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s failed: %s (%d)" % (where, strerror(code), code))


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError("liblychee.so is not built (run `python -m paper_2602_04541_amd.build` "
                          "or __graft_entry__.build()); there is no fallback path")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    shp = ctypes.POINTER(Shape)
    lib.lychee_create.argtypes = [ctypes.POINTER(vp), ctypes.c_int]
    lib.lychee_destroy.argtypes = [vp]
    lib.lychee_check_shape.argtypes = [shp, vp, ctypes.c_int]
    lib.lychee_workspace_bytes.argtypes = [shp]
    lib.lychee_workspace_bytes.restype = sz
    lib.lychee_step_workspace_bytes.argtypes = [shp, i32]
    lib.lychee_step_workspace_bytes.restype = sz
    lib.lychee_decode_attn.argtypes = [vp, shp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.lychee_decode_attn_deferred.argtypes = lib.lychee_decode_attn.argtypes
    lib.lychee_decode_attn_static.argtypes = [vp, shp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.lychee_select_flush.argtypes = [vp, vp]
    lib.lychee_dense_decode_attn.argtypes = [vp, shp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.lychee_decode_step.argtypes = [vp, shp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.lychee_dense_decode_step.argtypes = [vp, shp, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.lychee_decode_step_append.argtypes = [vp, shp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.lychee_append_kv.argtypes = [vp, shp, vp, vp, vp, vp, vp, vp]
    lib.lychee_select_stats.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(i64), vp]
    lib.lychee_wait_timeouts.argtypes = [vp, ctypes.POINTER(i64), vp]
    lib.lychee_validate_idx.argtypes = [vp, shp, vp, vp, ctypes.POINTER(i64), vp]
    lib.lychee_set_option.argtypes = [vp, i32, i32]
    lib.lychee_timing_enable.argtypes = [vp, ctypes.c_int]
    lib.lychee_timing_read.argtypes = [vp, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(i32)]
    lib.lychee_probe_read.argtypes = [vp, vp, sz, vp, vp]
    lib.lychee_probe_copy.argtypes = [vp, vp, vp, sz, vp]
    pgd = ctypes.POINTER(Paged)
    lib.lychee_check_paged.argtypes = [pgd, vp, ctypes.c_int]
    lib.lychee_paged_workspace_bytes.argtypes = [pgd]
    lib.lychee_paged_workspace_bytes.restype = sz
    lib.lychee_release_pages.argtypes = [vp, pgd, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.lychee_plan_pages.argtypes = [vp, pgd, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp]
    lib.lychee_q4_append.argtypes = [vp, pgd, vp, vp, i64, i64, vp, i32, vp, vp]
    lib.lychee_q4_read.argtypes = [vp, pgd, vp, vp, vp, vp, vp, vp, i64, i64, i64, i32, vp]
    lib.lychee_q4_decode_attn.argtypes = [vp, pgd, vp, vp, vp, vp, vp, vp, vp, vp, i64, vp, sz, vp]
    lib.lychee_select_scores.argtypes = [vp, pgd, vp, i64, vp, vp, vp, vp, vp]
    lib.lychee_strerror.argtypes = [ctypes.c_int]
    lib.lychee_strerror.restype = ctypes.c_char_p
    for name in EXPORTS:
        if name not in ("lychee_workspace_bytes", "lychee_step_workspace_bytes", "lychee_paged_workspace_bytes",
                        "lychee_strerror"):
            getattr(lib, name).restype = ctypes.c_int
    return lib


_lib = _load()


def strerror(code: int) -> str:
    return _lib.lychee_strerror(code).decode()


def _check(code: int, where: str) -> None:
    if code != OK:
        raise LycheeError(code, where)


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, torch.Tensor):
        return t.data_ptr()
    return int(t)


def _stream(stream) -> Optional[int]:
    if stream is None:
        stream = torch.cuda.current_stream()
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream or None
    return int(stream) or None


def make_shape(batch: int, n_q_heads: int, n_kv_heads: int, max_len: int, k: int,
               kv: Optional[torch.Tensor] = None, head_dim: int = 128,
               strides: Optional[Sequence[int]] = None, keep_ppm: int = 0,
               block_size: int = 0, prob_rule: int = 0, prob_param: float = 0.0) -> Shape:
    """A `lychee_shape`; KV strides (elements) come from a [B,H_kv,L_cap,128] tensor or `strides`."""
    if strides is None:
        if kv is not None:
            strides = (kv.stride(0), kv.stride(1), kv.stride(2))
        else:
            strides = (n_kv_heads * max_len * head_dim, max_len * head_dim, head_dim)
    return Shape(batch, n_q_heads, n_kv_heads, head_dim, max_len, k, *[int(s) for s in strides],
                 int(keep_ppm), int(block_size), int(prob_rule), float(prob_param))


def check_shape(shape: Shape, head_type_mask: Optional[np.ndarray] = None,
                has_idx_in: bool = True) -> int:
    """lychee_check_shape: returns the status code (pure host)."""
    m = None
    if head_type_mask is not None:
        m = np.ascontiguousarray(head_type_mask, dtype=np.uint8)
    return _lib.lychee_check_shape(ctypes.byref(shape), None if m is None else m.ctypes.data,
                                   int(has_idx_in))


def workspace_bytes(shape: Shape) -> int:
    return int(_lib.lychee_workspace_bytes(ctypes.byref(shape)))


def step_workspace_bytes(shape: Shape, n_layers: int) -> int:
    return int(_lib.lychee_step_workspace_bytes(ctypes.byref(shape), n_layers))


def make_paged(batch: int, n_q_heads: int, n_kv_heads: int, n_pages: int, page_size: int, max_pages: int, k: int = 1,
               table_stride: int = 0, page_tiles: int = 0, head_dim: int = 128) -> Paged:
    """A `lychee_paged`; table rows and pages lie one behind the other unless strides are given."""
    return Paged(batch, n_q_heads, n_kv_heads, head_dim, n_pages, page_size, max_pages, table_stride or max_pages,
                 page_tiles or n_kv_heads * (page_size // Q4_TILE_TOKENS), k)


def check_paged(paged: Paged, head_type_mask: Optional[np.ndarray] = None, has_idx_in: bool = True) -> int:
    """lychee_check_paged: returns the status code (pure host)."""
    m = None if head_type_mask is None else np.ascontiguousarray(head_type_mask, dtype=np.uint8)
    return _lib.lychee_check_paged(ctypes.byref(paged), None if m is None else m.ctypes.data, int(has_idx_in))


def paged_workspace_bytes(paged: Paged) -> int:
    return int(_lib.lychee_paged_workspace_bytes(ctypes.byref(paged)))


def _mask_ptr(head_type_mask, n_q_heads: int):
    """The host array of head types and its address (None: every head is a retrieval head)."""
    if head_type_mask is None:
        return None, None
    m = np.ascontiguousarray(head_type_mask, dtype=np.uint8)
    assert m.shape == (n_q_heads,)
    return m, m.ctypes.data


def _at(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _raw_stream(device: int) -> Optional[int]:
    """torch's current stream of a device as a hipStream_t."""
    return _current_raw_stream(device) or None


# (torch.cuda.current_stream builds a Stream object, 2.9 us of a call; the getter behind it takes 0.07)
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                              lambda device: torch.cuda.current_stream(device).cuda_stream)


def _is_rows(scores) -> bool:
    """Whether row (b, g) of [B, H_kv, n] lies (b * H_kv + g) strides behind the first."""
    return scores.stride(2) == 1 and (scores.shape[0] == 1 or scores.stride(0) == scores.shape[1] * scores.stride(1))


class Context:
    """Owner of a `lychee_ctx*`."""

    def __init__(self, device: int = 0):
        h = ctypes.c_void_p()
        _check(_lib.lychee_create(ctypes.byref(h), device), "lychee_create")
        self._h = h
        self.device = device

    def close(self) -> None:
        if self._h:
            _lib.lychee_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- the path -----------------------------------------------------------------------
    def decode_attn(self, shape: Shape, q, k_cache, v_cache, head_type_mask: np.ndarray, idx_in,
                    out, idx_out, lengths, workspace, stream=None) -> None:
        mask = np.ascontiguousarray(head_type_mask, dtype=np.uint8)
        _check(_lib.lychee_decode_attn(self._h, ctypes.byref(shape), _ptr(q), _ptr(k_cache),
                                       _ptr(v_cache), mask.ctypes.data, _ptr(idx_in), _ptr(out),
                                       _ptr(idx_out), _ptr(lengths), _ptr(workspace),
                                       workspace.numel() * workspace.element_size(),
                                       _stream(stream)), "lychee_decode_attn")

    def decode_attn_static(self, shape: Shape, q, k_cache, v_cache, head_type_mask: np.ndarray, idx_in,
                           out, idx_out, lengths, stream=None) -> None:
        """lychee_decode_attn on the library's own static scratch: no workspace, no allocation."""
        mask = np.ascontiguousarray(head_type_mask, dtype=np.uint8)
        _check(_lib.lychee_decode_attn_static(self._h, ctypes.byref(shape), _ptr(q), _ptr(k_cache),
                                              _ptr(v_cache), mask.ctypes.data, _ptr(idx_in), _ptr(out),
                                              _ptr(idx_out), _ptr(lengths), _stream(stream)),
               "lychee_decode_attn_static")

    def decode_attn_deferred(self, shape: Shape, q, k_cache, v_cache, head_type_mask: np.ndarray,
                             idx_in, out, idx_out, lengths, workspace, stream=None) -> None:
        """The layer call that leaves its selection for the next such call (or select_flush);
        `workspace` holds two layers (alloc_workspace(..., n_layers=2))."""
        mask = np.ascontiguousarray(head_type_mask, dtype=np.uint8)
        _check(_lib.lychee_decode_attn_deferred(self._h, ctypes.byref(shape), _ptr(q), _ptr(k_cache),
                                                _ptr(v_cache), mask.ctypes.data, _ptr(idx_in), _ptr(out),
                                                _ptr(idx_out), _ptr(lengths), _ptr(workspace),
                                                workspace.numel() * workspace.element_size(),
                                                _stream(stream)), "lychee_decode_attn_deferred")

    def select_flush(self, stream=None) -> None:
        _check(_lib.lychee_select_flush(self._h, _stream(stream)), "lychee_select_flush")

    def dense_decode_attn(self, shape: Shape, q, k_cache, v_cache, out, lengths, workspace,
                          stream=None) -> None:
        _check(_lib.lychee_dense_decode_attn(self._h, ctypes.byref(shape), _ptr(q), _ptr(k_cache),
                                             _ptr(v_cache), _ptr(out), _ptr(lengths),
                                             _ptr(workspace),
                                             workspace.numel() * workspace.element_size(),
                                             _stream(stream)), "lychee_dense_decode_attn")

    def decode_step(self, shape: Shape, q: Sequence, k_cache: Sequence, v_cache: Sequence,
                    head_type_masks: np.ndarray, idx_in, out: Sequence, idx_out, lengths,
                    workspace, stream=None) -> None:
        n = len(q)
        arr = ctypes.c_void_p * n
        masks = np.ascontiguousarray(head_type_masks, dtype=np.uint8)
        assert masks.shape == (n, shape.n_q_heads)
        _check(_lib.lychee_decode_step(self._h, ctypes.byref(shape), n,
                                       arr(*[_ptr(t) for t in q]), arr(*[_ptr(t) for t in k_cache]),
                                       arr(*[_ptr(t) for t in v_cache]), masks.ctypes.data,
                                       _ptr(idx_in), arr(*[_ptr(t) for t in out]), _ptr(idx_out),
                                       _ptr(lengths), _ptr(workspace),
                                       workspace.numel() * workspace.element_size(),
                                       _stream(stream)), "lychee_decode_step")

    def decode_step_append(self, shape: Shape, q: Sequence, k_new: Sequence, v_new: Sequence,
                           k_cache: Sequence, v_cache: Sequence, head_type_masks: np.ndarray, idx_in,
                           out: Sequence, idx_out, lengths, workspace, stream=None) -> None:
        n = len(q)
        arr = ctypes.c_void_p * n
        masks = np.ascontiguousarray(head_type_masks, dtype=np.uint8)
        assert masks.shape == (n, shape.n_q_heads)
        _check(_lib.lychee_decode_step_append(
            self._h, ctypes.byref(shape), n, arr(*[_ptr(t) for t in q]), arr(*[_ptr(t) for t in k_new]),
            arr(*[_ptr(t) for t in v_new]), arr(*[_ptr(t) for t in k_cache]),
            arr(*[_ptr(t) for t in v_cache]), masks.ctypes.data, _ptr(idx_in),
            arr(*[_ptr(t) for t in out]), _ptr(idx_out), _ptr(lengths), _ptr(workspace),
            workspace.numel() * workspace.element_size(), _stream(stream)), "lychee_decode_step_append")

    def append_kv(self, shape: Shape, k_new, v_new, k_cache, v_cache, lengths, stream=None) -> None:
        _check(_lib.lychee_append_kv(self._h, ctypes.byref(shape), _ptr(k_new), _ptr(v_new), _ptr(k_cache),
                                     _ptr(v_cache), _ptr(lengths), _stream(stream)), "lychee_append_kv")

    def dense_decode_step(self, shape: Shape, q: Sequence, k_cache: Sequence, v_cache: Sequence,
                          out: Sequence, lengths, workspace, stream=None) -> None:
        n = len(q)
        arr = ctypes.c_void_p * n
        _check(_lib.lychee_dense_decode_step(self._h, ctypes.byref(shape), n,
                                             arr(*[_ptr(t) for t in q]), arr(*[_ptr(t) for t in k_cache]),
                                             arr(*[_ptr(t) for t in v_cache]), arr(*[_ptr(t) for t in out]),
                                             _ptr(lengths), _ptr(workspace),
                                             workspace.numel() * workspace.element_size(),
                                             _stream(stream)), "lychee_dense_decode_step")

    # -- the paged 4-bit cache ----------------------------------------------------------
    # (calls of a few microseconds: what marshals their arguments is kept short)
    def _on(self, stream):
        """The stream of a call: the given one, or the current one of the context's device (not of the current device)."""
        if stream is None:
            return _raw_stream(self.device)
        return _stream(stream)

    def release_pages(self, paged: Paged, done, lengths, block_table, free_pages, free_count, lengths_out=None,
                      free_count_out=None, stream=None) -> None:
        """lychee_release_pages; lengths and count are updated in place unless outputs are given."""
        _check(_lib.lychee_release_pages(self._h, ctypes.byref(paged), _at(done), _at(lengths), _at(block_table),
                                         _at(free_pages), _at(free_count),
                                         _at(lengths if lengths_out is None else lengths_out),
                                         _at(free_count if free_count_out is None else free_count_out),
                                         self._on(stream)), "lychee_release_pages")

    def plan_pages(self, paged: Paged, lengths, new_tokens, block_table, free_pages, free_count, lengths_out,
                   free_count_out, slots, token_start, status, stream=None) -> None:
        """lychee_plan_pages; lengths_out / free_count_out None: in place."""
        _check(_lib.lychee_plan_pages(self._h, ctypes.byref(paged), _at(lengths), _at(new_tokens), _at(block_table),
                                      _at(free_pages), _at(free_count),
                                      _at(lengths if lengths_out is None else lengths_out),
                                      _at(free_count if free_count_out is None else free_count_out), _at(slots),
                                      slots.numel(), _at(token_start), _at(status), self._on(stream)),
               "lychee_plan_pages")

    def q4_append(self, paged: Paged, k_new, v_new, slots, cache, stream=None) -> None:
        """lychee_q4_append; k_new and v_new are [n_tokens, H_kv, 128] with the same strides, a token for every slot."""
        assert k_new.stride() == v_new.stride() and k_new.stride(2) == 1
        assert len(k_new) >= slots.numel() <= len(v_new)
        _check(_lib.lychee_q4_append(self._h, ctypes.byref(paged), _at(k_new), _at(v_new), k_new.stride(0),
                                     k_new.stride(1), _at(slots), slots.numel(), _at(cache), self._on(stream)),
               "lychee_q4_append")

    def q4_read(self, paged: Paged, cache, block_table, first, last, k_out, v_out, stream=None) -> None:
        """lychee_q4_read; k_out and v_out are [B, H_kv, rows, 128] with the same strides."""
        assert k_out.stride() == v_out.stride() and k_out.stride(3) == 1
        _check(_lib.lychee_q4_read(self._h, ctypes.byref(paged), _at(cache), _at(block_table), _at(first), _at(last),
                                   _at(k_out), _at(v_out), k_out.stride(0), k_out.stride(1), k_out.stride(2),
                                   k_out.shape[2], self._on(stream)), "lychee_q4_read")

    def q4_decode_attn(self, paged: Paged, q, cache, block_table, lengths, head_type_mask, idx_in, out, scores, workspace,
                       stream=None) -> None:
        """lychee_q4_decode_attn; scores None or [B, H_kv, row] with contiguous (b, g) rows."""
        mask, at = _mask_ptr(head_type_mask, paged.n_q_heads)
        assert scores is None or _is_rows(scores)
        _check(_lib.lychee_q4_decode_attn(self._h, ctypes.byref(paged), _at(q), _at(cache), _at(block_table),
                                          _at(lengths), at, _at(idx_in), _at(out), _at(scores),
                                          0 if scores is None else scores.stride(1), _at(workspace),
                                          workspace.numel() * workspace.element_size(), self._on(stream)),
               "lychee_q4_decode_attn")

    def select_scores(self, paged: Paged, scores, lengths, head_type_mask, idx_in, idx_out, stream=None) -> None:
        """lychee_select_scores; scores [B, H_kv, row] with contiguous (b, g) rows."""
        mask, at = _mask_ptr(head_type_mask, paged.n_q_heads)
        assert _is_rows(scores)
        _check(_lib.lychee_select_scores(self._h, ctypes.byref(paged), _at(scores), scores.stride(1), _at(lengths), at,
                                         _at(idx_in), _at(idx_out), self._on(stream)),
               "lychee_select_scores")

    # -- helpers ------------------------------------------------------------------------
    def select_stats(self, stream=None):
        """(too_few, too_many): score rows the select ranked whole since the context was created."""
        a, b = ctypes.c_int64(-1), ctypes.c_int64(-1)
        _check(_lib.lychee_select_stats(self._h, ctypes.byref(a), ctypes.byref(b), _stream(stream)),
               "lychee_select_stats")
        return int(a.value), int(b.value)

    def wait_timeouts(self, stream=None) -> int:
        """Bounded waits inside layer launches that gave up since the context was created."""
        n = ctypes.c_int64(-1)
        _check(_lib.lychee_wait_timeouts(self._h, ctypes.byref(n), _stream(stream)), "lychee_wait_timeouts")
        return int(n.value)

    def validate_idx(self, shape: Shape, idx, lengths, stream=None) -> int:
        n_bad = ctypes.c_int64(-1)
        _check(_lib.lychee_validate_idx(self._h, ctypes.byref(shape), _ptr(idx), _ptr(lengths),
                                        ctypes.byref(n_bad), _stream(stream)), "lychee_validate_idx")
        return int(n_bad.value)

    def set_option(self, option: int, value: int) -> None:
        _check(_lib.lychee_set_option(self._h, option, value), "lychee_set_option")

    def timing_enable(self, on: bool) -> None:
        _check(_lib.lychee_timing_enable(self._h, int(on)), "lychee_timing_enable")

    def timing_read(self):
        ms = (ctypes.c_float * N_KERNEL_CLASSES)()
        n = (ctypes.c_int32 * N_KERNEL_CLASSES)()
        _check(_lib.lychee_timing_read(self._h, ms, n), "lychee_timing_read")
        return list(ms), list(n)

    def probe_read(self, src, nbytes: int, sink, stream=None) -> None:
        _check(_lib.lychee_probe_read(self._h, _ptr(src), nbytes, _ptr(sink), _stream(stream)),
               "lychee_probe_read")

    def probe_copy(self, dst, src, nbytes: int, stream=None) -> None:
        _check(_lib.lychee_probe_copy(self._h, _ptr(dst), _ptr(src), nbytes, _stream(stream)),
               "lychee_probe_copy")


def alloc_workspace(shape: Shape, device="cuda", n_layers: int = 1) -> torch.Tensor:
    """A device buffer of lychee_step_workspace_bytes(shape, n_layers) bytes (torch only
    allocates it); n_layers = 1 is what the single-layer calls need."""
    n = step_workspace_bytes(shape, n_layers)
    if n == 0:
        raise LycheeError(_lib.lychee_check_shape(ctypes.byref(shape), None, 1), "lychee_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def alloc_paged_workspace(paged: Paged, device="cuda") -> torch.Tensor:
    """A device buffer of lychee_paged_workspace_bytes(paged) bytes."""
    n = paged_workspace_bytes(paged)
    if n == 0:
        raise LycheeError(check_paged(paged), "lychee_paged_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def alloc_q4_cache(paged: Paged, device="cuda") -> torch.Tensor:
    """The pages of one layer's cache, [n_pages, page_tiles * Q4_TILE_BYTES] bytes."""
    if check_paged(paged) != OK:
        raise LycheeError(check_paged(paged), "lychee_check_paged")
    return torch.empty((paged.n_pages, paged.page_tiles * Q4_TILE_BYTES), dtype=torch.uint8, device=device)
