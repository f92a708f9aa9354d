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
    "lychee_check_prompt", "lychee_prompt_workspace_bytes", "lychee_prompt_attn", "lychee_prompt_attn_backward",
    "lychee_q4_prompt_workspace_bytes", "lychee_q4_prompt_attn",
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


_MAX_STRIDE = 1 << 24  # of tokens and query heads, as lychee.h has it


class Prompt(ctypes.Structure):
    """Mirror of `lychee_prompt`."""
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("n_tokens", ctypes.c_int32), ("max_len", ctypes.c_int32),
                ("q_stride_tok", ctypes.c_int64), ("q_stride_head", ctypes.c_int64), ("kv_stride_batch", ctypes.c_int64),
                ("kv_stride_head", ctypes.c_int64), ("kv_stride_tok", ctypes.c_int64)]


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
    pmt = ctypes.POINTER(Prompt)
    lib.lychee_check_prompt.argtypes = [pmt]
    lib.lychee_prompt_workspace_bytes.argtypes = [pmt]
    lib.lychee_prompt_workspace_bytes.restype = sz
    lib.lychee_prompt_attn.argtypes = [vp, pmt, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.lychee_prompt_attn_backward.argtypes = [vp, pmt, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.lychee_q4_prompt_workspace_bytes.argtypes = [pgd, i32]
    lib.lychee_q4_prompt_workspace_bytes.restype = sz
    lib.lychee_q4_prompt_attn.argtypes = [vp, pgd, vp, i64, i64, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.lychee_strerror.argtypes = [ctypes.c_int]
    lib.lychee_strerror.restype = ctypes.c_char_p
    for name in EXPORTS:
        if name not in ("lychee_workspace_bytes", "lychee_step_workspace_bytes", "lychee_paged_workspace_bytes",
                        "lychee_prompt_workspace_bytes", "lychee_q4_prompt_workspace_bytes", "lychee_strerror"):
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
    try:
        m, at = _mask_ptr(head_type_mask, paged.n_q_heads, "lychee_check_paged")
    except LycheeError as e:
        return _lib.lychee_check_paged(ctypes.byref(paged), None, int(has_idx_in)) or e.code
    return _lib.lychee_check_paged(ctypes.byref(paged), at, int(has_idx_in))


def paged_workspace_bytes(paged: Paged) -> int:
    return int(_lib.lychee_paged_workspace_bytes(ctypes.byref(paged)))


def _stride(t: torch.Tensor, dim: int, least: int, packed: int) -> int:
    """A tensor's stride; that of a dimension of one entry is any number, also one that the library does not take: `packed` then."""
    stride = t.stride(dim)
    return stride if t.shape[dim] > 1 or (stride % 8 == 0 and least <= stride <= _MAX_STRIDE) else packed


def make_prompt(batch: int, q: torch.Tensor, kv: torch.Tensor) -> Prompt:
    """A `lychee_prompt` for q [n_tokens, H_q, 128] and keys (and values) like kv: [n_tokens, H_kv, 128], packed like q, or a cache
    [B, H_kv, L_cap, 128]; sizes and strides are theirs."""
    (T, heads, d), n_kv = q.shape, kv.shape[1]
    if kv.dim() == 4:
        max_len, of_rows = kv.shape[2], _stride(kv, 2, d, d)
        strides = (_stride(kv, 0, 0, n_kv * max_len * d), _stride(kv, 1, 0, max_len * d), of_rows)
    else:
        max_len, strides = 0, (0, _stride(kv, 1, 0, d), _stride(kv, 0, d, n_kv * d))
    return Prompt(batch, heads, n_kv, d, T, max_len, _stride(q, 0, d, heads * d), _stride(q, 1, 0, d), *strides)


def check_prompt(prompt: Prompt) -> int:
    """lychee_check_prompt: returns the status code (pure host)."""
    return _lib.lychee_check_prompt(ctypes.byref(prompt))


def prompt_workspace_bytes(prompt: Prompt) -> int:
    return int(_lib.lychee_prompt_workspace_bytes(ctypes.byref(prompt)))


def q4_prompt_workspace_bytes(paged: Paged, n_tokens: int) -> int:
    return int(_lib.lychee_q4_prompt_workspace_bytes(ctypes.byref(paged), n_tokens))


# The calls of the paged 4-bit cache look at what they are given: the library sees addresses alone, and would misread a view
# or another type, and write past a buffer that is too short.  That costs about 0.15 us a tensor (release and plan
# together 12.3 us, 10.3 without, 14 with a function's call for every tensor), so what a call is mostly given is looked at
# first, and what is not that gets a second look, and its message, from the functions below.
_I32, _BF16, _F32 = torch.int32, torch.bfloat16, torch.float32


def _refuse(call: str, name: str, t, want: str):
    have = "%s %s strides %s on %s" % (t.dtype, list(t.shape), list(t.stride()), t.device) if isinstance(t, torch.Tensor) else type(t).__name__
    raise LycheeError(EINVAL, "%s: %s is %s, not %s; it" % (call, name, have, want))


def _mask_ptr(head_type_mask, n_q_heads: int, call: str):
    """The host array of head types and its address (None: every head is a retrieval head)."""
    if head_type_mask is None:
        return None, None
    given = np.asarray(head_type_mask)
    m = np.ascontiguousarray(given, dtype=np.uint8)
    if m.shape != (n_q_heads,) or (m is not given and not np.array_equal(m, given)):
        raise LycheeError(EINVAL, "%s: head_type_mask is %s %s, not %d zeros and ones; it" % (call, given.dtype, list(given.shape), n_q_heads))
    return m, m.ctypes.data


def _arrays(call: str, device: int, *wanted):
    """The addresses of (name, tensor, type, n): n entries or more that lie one behind the other.  None stays None, which the
    library refuses where it has to."""
    at = []
    for name, t, dtype, n in wanted:
        if t is None:
            at.append(None)
            continue
        try:
            if not (t.dtype is dtype and t.numel() >= n and t.is_contiguous() and t.get_device() == device):
                _refuse(call, name, t, "a contiguous %s of %d entries on device %d" % (dtype, n, device))
        except AttributeError:
            _refuse(call, name, t, "a tensor")
        at.append(t.data_ptr())
    return at


def _on_device(t, device: int, itemsize: int) -> bool:
    return isinstance(t, torch.Tensor) and t.element_size() == itemsize and t.get_device() == device


def _strided(t, *row: int) -> bool:
    """Whether the last dimensions are at least so large, and the last of them contiguous."""
    return t.dim() >= len(row) and t.stride(-1) == 1 and all(a >= b for a, b in zip(t.shape[t.dim() - len(row):], row))


def _table_at(call: str, t, paged: Paged, device: int) -> Optional[int]:
    """The address of a block table: [B, >= max_pages] with rows table_stride apart, or as many entries in a row."""
    if t is None:
        return None
    B, stride = paged.batch, paged.table_stride
    if not (isinstance(t, torch.Tensor) and t.dtype is _I32 and t.shape == (B, stride) and t.is_contiguous() and t.get_device() == device):
        n = paged.max_pages
        ok = _on_device(t, device, 4) and t.dtype is _I32
        if ok and t.dim() == 2:
            ok = _strided(t, B, n) and (t.stride(0) == stride or B == 1)
        elif ok:
            ok = t.is_contiguous() and t.numel() >= (B - 1) * stride + n
        if not ok:
            _refuse(call, "block_table", t, "a torch.int32 [%d, %d] with rows %d apart on device %d" % (B, n, stride, device))
    return t.data_ptr()


def _cache_at(call: str, t, paged: Paged, device: int) -> Optional[int]:
    """The address of a layer's pages: bytes in a row, or [n_pages, bytes of a page] with pages page_tiles tiles apart."""
    if t is None:
        return None
    pages, apart = paged.n_pages, paged.page_tiles * Q4_TILE_BYTES
    if not (_on_device(t, device, 1) and t.is_contiguous() and t.numel() >= pages * apart):
        page = paged.n_kv_heads * (paged.page_size // Q4_TILE_TOKENS) * Q4_TILE_BYTES
        ok = _on_device(t, device, 1)
        if ok and t.is_contiguous():  # (the last of several interleaved layers ends before its last page does)
            ok = t.numel() >= (pages - 1) * apart + page
        elif ok:
            ok = t.dim() == 2 and _strided(t, pages, page) and t.stride(0) == apart
        if not ok:
            _refuse(call, "cache", t, "%d pages of %d bytes, %d apart, on device %d" % (pages, page, apart, device))
    return t.data_ptr()


def _scores_at(call: str, t, paged: Paged, device: int):
    """The address of score rows [B, H_kv, row] and their distance: row (b, g) lies (b * H_kv + g) strides behind the first, and
    the last of them too has room for max_pages * page_size."""
    if t is None:
        return None, 0
    B, H, n = paged.batch, paged.n_kv_heads, paged.max_pages * paged.page_size
    ok = _on_device(t, device, 4) and t.dtype is _F32 and t.dim() == 3
    if not (ok and t.is_contiguous() and t.shape[0] >= B and t.shape[1] == H and t.shape[2] >= n):
        ok = ok and _strided(t, B, H, 0) and (B == 1 or (t.shape[1] == H and t.stride(0) == H * t.stride(1)))
        if ok and t.shape[2] < n:  # (a view of the first positions)
            ok = t.untyped_storage().nbytes() // 4 - t.storage_offset() >= (B * H - 1) * t.stride(1) + n
        if not ok:
            _refuse(call, "scores", t, "a torch.float32 [%d, %d, %d], evenly spaced rows, on device %d" % (B, H, n, device))
    return t.data_ptr(), t.stride(1)


def _rows_at(call: str, names, k, v, shape, device: int):
    """The addresses of two bf16 tensors of a shape at least, with the same strides and contiguous rows, and the strides."""
    if k is None or v is None:
        return None, None, (0,) * len(shape)
    ok = False
    if _on_device(k, device, 2) and _on_device(v, device, 2):
        strides = k.stride()
        ok = k.dtype is _BF16 and v.dtype is _BF16 and k.shape == shape and v.shape == shape and strides[-1] == 1 and v.stride() == strides
    if not ok:
        for name, t in zip(names, (k, v)):
            if not (_on_device(t, device, 2) and t.dtype is _BF16 and t.dim() == len(shape) and _strided(t, *shape)
                    and t.stride() == k.stride()):
                _refuse(call, name, t, "a torch.bfloat16 %s, strided like %s, on device %d" % (list(shape), names[0], device))
        strides = k.stride()
    return k.data_ptr(), v.data_ptr(), strides


def _strided_at(call: str, name: str, t, shape, strides, device: int) -> Optional[int]:
    """The address of a bf16 tensor of this shape with these strides (those of dimensions of one entry do not count)."""
    if t is None:
        return None
    if not (_on_device(t, device, 2) and t.dtype is _BF16 and t.shape == shape
            and (t.stride() == strides or all(n <= 1 or a == b for n, a, b in zip(shape, t.stride(), strides)) or 0 in shape)):
        _refuse(call, name, t, "a torch.bfloat16 %s with strides %s on device %d" % (list(shape), list(strides), device))
    return t.data_ptr()


def _dtype_of(t):
    return t.dtype if isinstance(t, torch.Tensor) else torch.uint8


# (torch.cuda.current_stream builds a Stream object, 2.9 us of a call; the getter behind it takes 0.07)
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                              lambda device: torch.cuda.current_stream(device).cuda_stream)


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
        return _current_raw_stream(self.device) if stream is None else _stream(stream)

    def release_pages(self, paged: Paged, done, lengths, block_table, free_pages, free_count, lengths_out=None,
                      free_count_out=None, stream=None) -> None:
        """lychee_release_pages; lengths and count are updated in place unless outputs are given.  done: bytes or bool."""
        B, pages, device = paged.batch, paged.n_pages, self.device
        lengths_out = lengths if lengths_out is None else lengths_out
        free_count_out = free_count if free_count_out is None else free_count_out
        try:
            fine = (done.element_size() == 1 and lengths.dtype is block_table.dtype is free_pages.dtype is free_count.dtype
                    is lengths_out.dtype is free_count_out.dtype is _I32
                    and done.get_device() == lengths.get_device() == block_table.get_device() == free_pages.get_device()
                    == free_count.get_device() == lengths_out.get_device() == free_count_out.get_device() == device
                    and done.is_contiguous() and lengths.is_contiguous() and block_table.is_contiguous()
                    and free_pages.is_contiguous() and lengths_out.is_contiguous()
                    and block_table.shape == (B, paged.table_stride) and lengths.numel() >= B <= lengths_out.numel()
                    and free_pages.numel() >= pages and free_count.numel() >= 1 <= free_count_out.numel() and done.numel() >= B)
        except AttributeError:  # (None, say)
            fine = False
        if fine:
            at = (done.data_ptr(), lengths.data_ptr(), block_table.data_ptr(), free_pages.data_ptr(), free_count.data_ptr(),
                  lengths_out.data_ptr(), free_count_out.data_ptr())
        else:
            call, byte = "lychee_release_pages", isinstance(done, torch.Tensor) and done.element_size() == 1
            at = _arrays(call, device, ("done", done, done.dtype if byte else torch.uint8, B), ("lengths", lengths, _I32, B),
                         ("free_pages", free_pages, _I32, pages), ("free_count", free_count, _I32, 1),
                         ("lengths_out", lengths_out, _I32, B), ("free_count_out", free_count_out, _I32, 1))
            at.insert(2, _table_at(call, block_table, paged, device))
        _check(_lib.lychee_release_pages(self._h, paged, *at, self._on(stream)), "lychee_release_pages")

    def plan_pages(self, paged: Paged, lengths, new_tokens, block_table, free_pages, free_count, lengths_out,
                   free_count_out, slots, token_start, status, stream=None) -> None:
        """lychee_plan_pages; lengths_out / free_count_out None: in place."""
        B, pages, device = paged.batch, paged.n_pages, self.device
        lengths_out = lengths if lengths_out is None else lengths_out
        free_count_out = free_count if free_count_out is None else free_count_out
        try:
            fine = (lengths.dtype is new_tokens.dtype is block_table.dtype is free_pages.dtype is free_count.dtype is lengths_out.dtype
                    is free_count_out.dtype is slots.dtype is token_start.dtype is status.dtype is _I32
                    and lengths.get_device() == new_tokens.get_device() == block_table.get_device() == free_pages.get_device()
                    == free_count.get_device() == lengths_out.get_device() == free_count_out.get_device() == slots.get_device()
                    == token_start.get_device() == status.get_device() == device
                    and lengths.is_contiguous() and new_tokens.is_contiguous() and block_table.is_contiguous()
                    and free_pages.is_contiguous() and lengths_out.is_contiguous() and slots.is_contiguous()
                    and token_start.is_contiguous()
                    and block_table.shape == (B, paged.table_stride) and lengths.numel() >= B <= new_tokens.numel()
                    and lengths_out.numel() >= B < token_start.numel() and free_pages.numel() >= pages
                    and free_count.numel() >= 1 <= free_count_out.numel() and status.numel() >= 1)
        except AttributeError:
            fine = False
        if fine:
            at = (lengths.data_ptr(), new_tokens.data_ptr(), block_table.data_ptr(), free_pages.data_ptr(), free_count.data_ptr(),
                  lengths_out.data_ptr(), free_count_out.data_ptr(), slots.data_ptr(), slots.numel(), token_start.data_ptr(),
                  status.data_ptr())
        else:
            call = "lychee_plan_pages"
            at = _arrays(call, device, ("lengths", lengths, _I32, B), ("new_tokens", new_tokens, _I32, B),
                         ("free_pages", free_pages, _I32, pages), ("free_count", free_count, _I32, 1),
                         ("lengths_out", lengths_out, _I32, B), ("free_count_out", free_count_out, _I32, 1),
                         ("slots", slots, _I32, 0), ("token_start", token_start, _I32, B + 1), ("status", status, _I32, 1))
            at.insert(2, _table_at(call, block_table, paged, device))
            at.insert(8, 0 if slots is None else slots.numel())
        _check(_lib.lychee_plan_pages(self._h, paged, *at, self._on(stream)), "lychee_plan_pages")

    def q4_append(self, paged: Paged, k_new, v_new, slots, cache, stream=None) -> None:
        """lychee_q4_append; k_new and v_new are [n_tokens, H_kv, 128] with the same strides, a token for every slot."""
        call, device = "lychee_q4_append", self.device
        (slot,) = _arrays(call, device, ("slots", slots, _I32, 0))
        n = 0 if slots is None else slots.numel()
        k, v, strides = _rows_at(call, ("k_new", "v_new"), k_new, v_new, (n, paged.n_kv_heads, paged.head_dim), device)
        _check(_lib.lychee_q4_append(self._h, paged, k, v, strides[0], strides[1], slot, n, _cache_at(call, cache, paged, device),
                                     self._on(stream)), call)

    def q4_read(self, paged: Paged, cache, block_table, first, last, k_out, v_out, stream=None) -> None:
        """lychee_q4_read; k_out and v_out are [B, H_kv, rows, 128] with the same strides."""
        call, device, B = "lychee_q4_read", self.device, paged.batch
        begin, end = _arrays(call, device, ("first", first, _I32, B), ("last", last, _I32, B))
        n = k_out.shape[2] if isinstance(k_out, torch.Tensor) and k_out.dim() == 4 else 0
        k, v, strides = _rows_at(call, ("k_out", "v_out"), k_out, v_out, (B, paged.n_kv_heads, n, paged.head_dim), device)
        _check(_lib.lychee_q4_read(self._h, paged, _cache_at(call, cache, paged, device), _table_at(call, block_table, paged, device),
                                   begin, end, k, v, strides[0], strides[1], strides[2], n, self._on(stream)), call)

    def q4_decode_attn(self, paged: Paged, q, cache, block_table, lengths, head_type_mask, idx_in, out, scores, workspace,
                       stream=None) -> None:
        """lychee_q4_decode_attn; q, out [B, H_q, 128]; scores None or [B, H_kv, row] with evenly spaced (b, g) rows."""
        call, device, B, heads = "lychee_q4_decode_attn", self.device, paged.batch, paged.n_q_heads
        mask, types = _mask_ptr(head_type_mask, heads, call)
        n = B * heads * paged.head_dim
        kind = workspace.dtype if isinstance(workspace, torch.Tensor) else torch.uint8
        at_q, length, idx, at_out, ws = _arrays(
            call, device, ("q", q, _BF16, n), ("lengths", lengths, _I32, B),
            ("idx_in", idx_in, _I32, B * paged.n_kv_heads * paged.k), ("out", out, _BF16, n), ("workspace", workspace, kind, 0))
        score, stride = _scores_at(call, scores, paged, device)
        _check(_lib.lychee_q4_decode_attn(self._h, paged, at_q, _cache_at(call, cache, paged, device),
                                          _table_at(call, block_table, paged, device), length, types, idx, at_out, score, stride, ws,
                                          0 if ws is None else workspace.nbytes, self._on(stream)), call)

    def select_scores(self, paged: Paged, scores, lengths, head_type_mask, idx_in, idx_out, stream=None) -> None:
        """lychee_select_scores; scores [B, H_kv, row] with evenly spaced (b, g) rows."""
        call, B = "lychee_select_scores", paged.batch
        mask, types = _mask_ptr(head_type_mask, paged.n_q_heads, call)
        n = B * paged.n_kv_heads * paged.k
        length, idx, new = _arrays(call, self.device, ("lengths", lengths, _I32, B), ("idx_in", idx_in, _I32, n),
                                   ("idx_out", idx_out, _I32, n))
        score, stride = _scores_at(call, scores, paged, self.device)
        _check(_lib.lychee_select_scores(self._h, paged, score, stride, length, types, idx, new, self._on(stream)), call)

    # -- whole prompts ------------------------------------------------------------------
    def _rows_like(self, call: str, prompt: Prompt, *named):
        """The addresses of (name, tensor) like q: [n_tokens, H_q, 128], strided as in the prompt."""
        n, heads, d = prompt.n_tokens, prompt.n_q_heads, prompt.head_dim
        return [_strided_at(call, name, t, (n, heads, d), (prompt.q_stride_tok, prompt.q_stride_head, 1), self.device) for name, t in named]

    def _keys_like(self, call: str, prompt: Prompt, cached: bool, *named):
        """The same of (name, tensor) like k: packed rows [n_tokens, H_kv, 128] or a cache [B, H_kv, max_len, 128]."""
        tok, head, d = prompt.kv_stride_tok, prompt.kv_stride_head, prompt.head_dim
        shape, strides = (prompt.n_tokens, prompt.n_kv_heads, d), (tok, head, 1)
        if cached:
            shape, strides = (prompt.batch, prompt.n_kv_heads, prompt.max_len, d), (prompt.kv_stride_batch, head, tok, 1)
        return [_strided_at(call, name, t, shape, strides, self.device) for name, t in named]

    def prompt_attn(self, prompt: Prompt, q, k, v, token_start, lengths, out, lse, workspace, stream=None) -> None:
        """lychee_prompt_attn; q [n_tokens, H_q, 128]; k and v [n_tokens, H_kv, 128], or with lengths [B, H_kv, max_len, 128]; out
        [n_tokens, H_q, 128]; lse None or [H_q, n_tokens]."""
        device, B, T, heads, kv, d = self.device, prompt.batch, prompt.n_tokens, prompt.n_q_heads, prompt.n_kv_heads, prompt.head_dim
        n, tok, head, cached = T * heads, prompt.kv_stride_tok, prompt.kv_stride_head, lengths is not None
        shape = (B, kv, prompt.max_len, d) if cached else (T, kv, d)
        strides = (prompt.kv_stride_batch, head, tok, 1) if cached else (tok, head, 1)
        try:
            fine = (q.dtype is k.dtype is v.dtype is out.dtype is _BF16 and token_start.dtype is _I32
                    and q.get_device() == k.get_device() == v.get_device() == out.get_device() == token_start.get_device()
                    == workspace.get_device() == device
                    and q.shape == (T, heads, d) and q.stride() == (prompt.q_stride_tok, prompt.q_stride_head, 1)
                    and k.shape == shape == v.shape and k.stride() == strides == v.stride()
                    and out.is_contiguous() and token_start.is_contiguous() and workspace.is_contiguous()
                    and out.numel() >= n * d and token_start.numel() > B
                    and (not cached or (lengths.dtype is _I32 and lengths.get_device() == device and lengths.is_contiguous()
                                        and lengths.numel() >= B))
                    and (lse is None or (lse.dtype is _F32 and lse.get_device() == device and lse.is_contiguous() and lse.numel() >= n)))
        except AttributeError:  # (None, say)
            fine = False
        if fine:
            at = (q.data_ptr(), k.data_ptr(), v.data_ptr(), token_start.data_ptr(), lengths.data_ptr() if cached else None, out.data_ptr(),
                  None if lse is None else lse.data_ptr(), workspace.data_ptr(), workspace.nbytes)
        else:
            call = "lychee_prompt_attn"
            at = self._rows_like(call, prompt, ("q", q)) + self._keys_like(call, prompt, cached, ("k", k), ("v", v)) + _arrays(
                call, device, ("token_start", token_start, _I32, B + 1), ("lengths", lengths, _I32, B), ("out", out, _BF16, n * d),
                ("lse", lse, _F32, n), ("workspace", workspace, _dtype_of(workspace), 0)) + [0 if workspace is None else workspace.nbytes]
        _check(_lib.lychee_prompt_attn(self._h, prompt, *at, self._on(stream)), "lychee_prompt_attn")

    def prompt_attn_backward(self, prompt: Prompt, d_out, q, k, v, out, lse, token_start, dq, dk, dv, workspace, stream=None) -> None:
        """lychee_prompt_attn_backward; dq strided like q, dk and dv like k and v."""
        device, B, T, heads, kv, d = self.device, prompt.batch, prompt.n_tokens, prompt.n_q_heads, prompt.n_kv_heads, prompt.head_dim
        n = T * heads
        rows, keys = (T, heads, d), (T, kv, d)
        of_rows, of_keys = (prompt.q_stride_tok, prompt.q_stride_head, 1), (prompt.kv_stride_tok, prompt.kv_stride_head, 1)
        try:
            fine = (d_out.dtype is q.dtype is k.dtype is v.dtype is out.dtype is dq.dtype is dk.dtype is dv.dtype is _BF16
                    and lse.dtype is _F32 and token_start.dtype is _I32
                    and d_out.get_device() == q.get_device() == k.get_device() == v.get_device() == out.get_device() == lse.get_device()
                    == token_start.get_device() == dq.get_device() == dk.get_device() == dv.get_device() == workspace.get_device() == device
                    and q.shape == rows == dq.shape and q.stride() == of_rows == dq.stride()
                    and k.shape == keys == v.shape and k.stride() == of_keys == v.stride()
                    and dk.shape == keys == dv.shape and dk.stride() == of_keys == dv.stride()
                    and d_out.is_contiguous() and out.is_contiguous() and lse.is_contiguous() and token_start.is_contiguous()
                    and workspace.is_contiguous() and d_out.numel() >= n * d <= out.numel() and lse.numel() >= n
                    and token_start.numel() > B)
        except AttributeError:
            fine = False
        if fine:
            at = (d_out.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(), token_start.data_ptr(),
                  dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), workspace.data_ptr(), workspace.nbytes)
        else:
            call = "lychee_prompt_attn_backward"
            at_q, at_dq = self._rows_like(call, prompt, ("q", q), ("dq", dq))
            at_k, at_v, at_dk, at_dv = self._keys_like(call, prompt, False, ("k", k), ("v", v), ("dk", dk), ("dv", dv))
            at_g, at_out, at_lse, start, ws = _arrays(
                call, device, ("d_out", d_out, _BF16, n * d), ("out", out, _BF16, n * d), ("lse", lse, _F32, n),
                ("token_start", token_start, _I32, B + 1), ("workspace", workspace, _dtype_of(workspace), 0))
            at = (at_g, at_q, at_k, at_v, at_out, at_lse, start, at_dq, at_dk, at_dv, ws, 0 if ws is None else workspace.nbytes)
        _check(_lib.lychee_prompt_attn_backward(self._h, prompt, *at, self._on(stream)), "lychee_prompt_attn_backward")

    def q4_prompt_attn(self, paged: Paged, q, cache, block_table, lengths, token_start, out, workspace, stream=None) -> None:
        """lychee_q4_prompt_attn; q [n_tokens, H_q, 128], strided; out [n_tokens, H_q, 128]."""
        device, B, heads, d, pages, width = self.device, paged.batch, paged.n_q_heads, paged.head_dim, paged.n_pages, paged.table_stride
        try:
            n, strides = q.shape[0], q.stride()
            if n == 1 or heads == 1:
                strides = (_stride(q, 0, d, heads * d), _stride(q, 1, 0, d)) + strides[2:]
            fine = (q.dtype is out.dtype is _BF16 and lengths.dtype is token_start.dtype is block_table.dtype is _I32
                    and cache.element_size() == 1
                    and q.get_device() == cache.get_device() == block_table.get_device() == lengths.get_device() == token_start.get_device()
                    == out.get_device() == workspace.get_device() == device
                    and q.shape == (n, heads, d) and n > 0 and strides[2] == 1
                    and cache.is_contiguous() and block_table.is_contiguous() and lengths.is_contiguous() and token_start.is_contiguous()
                    and out.is_contiguous() and workspace.is_contiguous() and block_table.shape == (B, width)
                    and cache.numel() >= pages * paged.page_tiles * Q4_TILE_BYTES and lengths.numel() >= B < token_start.numel()
                    and out.numel() >= n * heads * d)
        except (AttributeError, IndexError):
            fine = False
        if fine:
            at = (q.data_ptr(), strides[0], strides[1], n, cache.data_ptr(), block_table.data_ptr(), lengths.data_ptr(),
                  token_start.data_ptr(), out.data_ptr(), workspace.data_ptr(), workspace.nbytes)
        else:
            call = "lychee_q4_prompt_attn"
            n = q.shape[0] if isinstance(q, torch.Tensor) and q.dim() == 3 else 0
            strides = (_stride(q, 0, d, heads * d), _stride(q, 1, 0, d), 1) if n else (d, 0, 1)
            at_q = _strided_at(call, "q", q, (n, heads, d), strides, device)
            length, start, at_out, ws = _arrays(
                call, device, ("lengths", lengths, _I32, B), ("token_start", token_start, _I32, B + 1), ("out", out, _BF16, n * heads * d),
                ("workspace", workspace, _dtype_of(workspace), 0))
            at = (at_q, strides[0], strides[1], n, _cache_at(call, cache, paged, device), _table_at(call, block_table, paged, device), length,
                  start, at_out, ws, 0 if ws is None else workspace.nbytes)
        _check(_lib.lychee_q4_prompt_attn(self._h, paged, *at, self._on(stream)), "lychee_q4_prompt_attn")

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


def alloc_prompt_workspace(prompt: Prompt, device="cuda") -> torch.Tensor:
    """A device buffer of lychee_prompt_workspace_bytes(prompt) bytes."""
    n = prompt_workspace_bytes(prompt)
    if n == 0:
        raise LycheeError(check_prompt(prompt), "lychee_prompt_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def alloc_q4_prompt_workspace(paged: Paged, n_tokens: int, device="cuda") -> torch.Tensor:
    """A device buffer of lychee_q4_prompt_workspace_bytes(paged, n_tokens) bytes."""
    n = q4_prompt_workspace_bytes(paged, n_tokens)
    if n == 0:
        raise LycheeError(check_paged(paged) or EUNSUPPORTED, "lychee_q4_prompt_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def alloc_q4_cache(paged: Paged, device="cuda") -> torch.Tensor:
    """The pages of one layer's cache, [n_pages, page_tiles * Q4_TILE_BYTES] bytes."""
    if check_paged(paged) != OK:
        raise LycheeError(check_paged(paged), "lychee_check_paged")
    return torch.empty((paged.n_pages, paged.page_tiles * Q4_TILE_BYTES), dtype=torch.uint8, device=device)
