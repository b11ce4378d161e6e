"""Thin ctypes binding of ``libsablock.so``: argument marshalling only.

Function names mirror the C ABI (``include/sablock.h``).  Tensors are torch
tensors on the GPU (device memory and the current stream are the only things
torch provides); every step of the path runs in the library's HIP kernels.
There is no CPU fallback: if the library is missing, loading raises.
"""

from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass
from functools import lru_cache
from typing import NamedTuple, Optional, Sequence, Tuple

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsablock.so")
_lib = _torch = None

SABLOCK_OK = 0
STATUS_NAMES = {0: "OK", 1: "INVALID_ARG", 2: "UNSUPPORTED", 3: "WORKSPACE_TOO_SMALL", 4: "DEVICE"}
SABLOCK_F32, SABLOCK_BF16 = 0, 1

EXPORTS = ("sablock_version", "sablock_last_error", "sablock_workspace_bytes", "sablock_score",
           "sablock_refine", "sablock_search_blocks", "sablock_select", "sablock_compact",
           "sablock_segment_count", "sablock_segment_offsets", "sablock_decode_workspace_bytes",
           "sablock_decode_attention", "sablock_score_all_heads_workspace_bytes", "sablock_score_all_heads",
           "sablock_compact_shared", "sablock_search_select", "sablock_window_attention_workspace_bytes",
           "sablock_window_attention", "sablock_score_static", "sablock_stream_probe", "sablock_validate_segments",
           "sablock_segment_slices", "sablock_segment_slice_count", "sablock_segment_slice_offsets",
           "sablock_compact_paged", "sablock_append_paged", "sablock_decode_paged_workspace_bytes", "sablock_decode_paged",
           "sablock_select_pages_workspace_bytes", "sablock_select_pages")


class SablockError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"sablock status {status} ({STATUS_NAMES.get(status, '?')}): {msg}")
        self.status = status


class CTuning(ctypes.Structure):
    """Launch parameters (``sablock_tuning``); all zero = the library's own plan."""

    _fields_ = [("compute_units", ctypes.c_int32), ("score_chunk", ctypes.c_int32), ("window_chunk", ctypes.c_int32),
                ("topb_slices", ctypes.c_int32), ("stats_per_key", ctypes.c_int32), ("reserved", ctypes.c_int32 * 3)]


class CShape(ctypes.Structure):
    _fields_ = [("n_seq", ctypes.c_int32), ("n_layers", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("seq_len", ctypes.c_int32),
                ("window", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("q_stride", ctypes.c_int64 * 4), ("k_stride", ctypes.c_int64 * 4), ("v_stride", ctypes.c_int64 * 4),
                ("tuning", CTuning)]


class CHparams(ctypes.Structure):
    _fields_ = [("eps", ctypes.c_float), ("alpha", ctypes.c_float), ("eta", ctypes.c_float), ("tau", ctypes.c_float)]


class CPages(ctypes.Structure):
    """A paged cache (``sablock_pages``)."""

    _fields_ = [("n_seq", ctypes.c_int32), ("n_layers", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("page_size", ctypes.c_int32), ("n_pages", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("compute_units", ctypes.c_int32), ("reserved", ctypes.c_int32 * 2),
                ("k_stride", ctypes.c_int64 * 4), ("v_stride", ctypes.c_int64 * 4)]


class CNewTokens(ctypes.Structure):
    """The new tokens of an append (``sablock_new_tokens``)."""

    _fields_ = [("n_new", ctypes.c_int32), ("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("q_stride", ctypes.c_int64 * 4), ("k_stride", ctypes.c_int64 * 4), ("v_stride", ctypes.c_int64 * 4)]


def load():
    """Load the HIP library (built in-tree by ``paper_2510_22556_amd.build``); raises if absent."""
    global _lib, _torch
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} not found: build it with `python -m paper_2510_22556_amd.build` "
                "(there is no fallback path)")
        # torch first: it ships its own copy of the HIP runtime, and a process must hold one runtime only (device
        # pointers and streams of torch are meaningless to a second copy loaded through this library)
        import torch

        _torch = torch
        lib = ctypes.CDLL(LIB_PATH)
        vp, i32, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float
        sp = ctypes.POINTER(CShape)
        lib.sablock_version.restype = ctypes.c_char_p
        lib.sablock_last_error.restype = ctypes.c_char_p
        lib.sablock_workspace_bytes.argtypes = [sp, i32, i32, ctypes.POINTER(ctypes.c_size_t)]
        lib.sablock_score.argtypes = [sp, vp, vp, vp, f32, vp, vp, vp, ctypes.c_size_t, vp]
        lib.sablock_score_static.argtypes = [sp, vp, vp, vp, f32, vp, vp, vp]
        lib.sablock_stream_probe.argtypes = [sp, vp, i32, vp, vp, vp, vp]
        lib.sablock_refine.argtypes = [sp, vp, vp, vp, ctypes.POINTER(i32), i32, ctypes.POINTER(CHparams),
                                       vp, vp, vp, ctypes.c_size_t, vp]
        lib.sablock_search_blocks.argtypes = [sp, vp, vp, ctypes.POINTER(i32), i32, ctypes.POINTER(i32), i32,
                                              i32, f32, vp, vp, vp, vp, ctypes.c_size_t, vp]
        lib.sablock_select.argtypes = [sp, vp, vp, ctypes.POINTER(i32), i32, vp, vp, vp, i32, vp, vp, vp,
                                       ctypes.c_size_t, vp]
        lib.sablock_compact.argtypes = [sp, vp, vp, vp, vp, i32, i32, vp, vp, vp]
        lib.sablock_search_select.argtypes = [sp, vp, vp, ctypes.POINTER(i32), i32, ctypes.POINTER(i32), i32, i32, f32,
                                              vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        lib.sablock_segment_count.argtypes = [vp, ctypes.c_int64, i32, i32, ctypes.POINTER(i32), i32, vp, vp]
        lib.sablock_segment_offsets.argtypes = [vp, ctypes.c_int64, i32, i32, ctypes.POINTER(i32), i32,
                                                ctypes.POINTER(i32), vp, vp]
        lib.sablock_segment_slices.argtypes = [i32, i32]
        lib.sablock_segment_slice_count.argtypes = lib.sablock_segment_count.argtypes
        lib.sablock_segment_slice_offsets.argtypes = lib.sablock_segment_offsets.argtypes
        lib.sablock_validate_segments.argtypes = [vp, ctypes.POINTER(i32), i32, i32, vp, vp]
        lib.sablock_decode_workspace_bytes.argtypes = [sp, ctypes.POINTER(ctypes.c_size_t)]
        lib.sablock_decode_attention.argtypes = [sp, vp, vp, vp, vp, i32, vp, vp, ctypes.c_size_t, vp]
        lib.sablock_score_all_heads_workspace_bytes.argtypes = [sp, ctypes.POINTER(ctypes.c_size_t)]
        lib.sablock_score_all_heads.argtypes = [sp, vp, vp, vp, f32, vp, vp, vp, ctypes.c_size_t, vp]
        lib.sablock_compact_shared.argtypes = [sp, vp, vp, vp, vp, i32, i32, vp, vp, vp]
        lib.sablock_window_attention_workspace_bytes.argtypes = [sp, ctypes.POINTER(ctypes.c_size_t)]
        lib.sablock_window_attention.argtypes = [sp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        pp = ctypes.POINTER(CPages)
        lib.sablock_compact_paged.argtypes = [sp, vp, vp, vp, i32, i32, pp, vp, vp, vp, vp, vp, vp]
        lib.sablock_append_paged.argtypes = [pp, ctypes.POINTER(CNewTokens)] + [vp] * 13
        lib.sablock_decode_paged_workspace_bytes.argtypes = [pp, ctypes.POINTER(ctypes.c_size_t)]
        lib.sablock_decode_paged.argtypes = [pp, vp, vp, vp, vp, vp, vp, i32, vp, vp, ctypes.c_size_t, vp]
        lib.sablock_select_pages_workspace_bytes.argtypes = [pp, ctypes.POINTER(ctypes.c_size_t)]
        lib.sablock_select_pages.argtypes = [pp, vp, vp, vp, vp, i32, i32, i32, vp, vp, ctypes.c_size_t, vp]
        for n in EXPORTS[2:]:
            getattr(lib, n).restype = ctypes.c_int
        _lib = lib
    return _lib


def _check(status: int):
    if status != SABLOCK_OK:
        raise SablockError(status, load().sablock_last_error().decode())


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream, device: Optional[int] = None) -> Optional[int]:
    """Handle of the stream, or of the current one of the device (None = the current device)."""
    if stream is None:
        # the handle alone: torch.cuda.current_stream() builds an object around it, 2.8 us
        return _torch._C._cuda_getCurrentRawStream(_torch.cuda.current_device() if device is None else device) or None
    return stream.cuda_stream or None


def _pointers(*tensors):
    """The current device, and device pointers (None stays) of tensors that are all on it: another one's, or the host's, the kernels could not
    follow."""
    device, pointers = None, [None]
    for t in tensors:
        if t is None:
            pointers.append(None)
            continue
        at = t.get_device()
        if at != device:
            if at < 0 or device is not None:
                raise ValueError(f"tensors on {[str(t.device) for t in tensors if t is not None]}: the calls take device memory, of one device")
            device = at
        pointers.append(t.data_ptr())
    current = _torch._C._cuda_getDevice()      # torch.cuda.current_device() asks first whether the device is initialised; with a tensor there it is
    if device != current:
        raise ValueError(f"tensors on cuda:{device} while cuda:{current} is the current device")
    pointers[0] = device
    return pointers


def _dense(dtype, n: int, *tensors):
    """Dense tensors of at least n elements: what the calls index without strides."""
    _all_dense(*[(dtype, n, t) for t in tensors])


def _all_dense(*wanted):
    for dtype, n, t in wanted:
        if t is not None and (t.dtype is not dtype or t.numel() < n or not t.is_contiguous()):
            raise ValueError(f"need a dense {dtype} tensor of at least {n} elements, got {t.dtype} {tuple(t.shape)} with strides {t.stride()}")


class _Extent(NamedTuple):
    """Where a call looks in a tensor ``[.., .., .., .., D]`` that it indexes by a descriptor."""

    what: str
    sizes: Tuple[int, ...]
    steps: Tuple[int, ...]
    dense: int                                 # elements, if the steps are those of a dense tensor


def _extent(what: str, sizes, steps) -> _Extent:
    dense = 1
    for n, step in zip(reversed(sizes), reversed(steps)):
        dense = dense * n if n == 1 or step == dense else 0
    return _Extent(what, tuple(sizes), tuple(steps), dense)


def _strided(dtype, *wanted):
    """Tensors that hold an extent: of the type and as dense as it (how a dense one is cut into axes is not looked at), or as long on every axis and with
    the same steps on those of more than one entry.  Of another number of axes: memory that reaches as far."""
    for t, (what, sizes, steps, dense) in wanted:
        if t.dtype is dtype and (t.numel() >= dense and t.is_contiguous() if dense else t.shape == sizes and t.stride() == steps):
            continue
        if t.dim() == 5:
            ok = all(m >= n for m, n in zip(t.shape, sizes)) and all(n <= 1 or a == b for n, a, b in zip(sizes, t.stride(), steps))
        else:
            last = sum((n - 1) * max(a, 0) for n, a in zip(sizes, steps))
            ok = last < t.untyped_storage().nbytes() // t.element_size() - t.storage_offset()
        if t.dtype is not dtype or not ok:
            raise ValueError(f"{what}: the descriptor says {dtype} {sizes} with strides {steps}, got {t.dtype} {tuple(t.shape)} with strides {t.stride()}")


def make_shape(q, k, v=None, **tuning) -> CShape:
    """Shape descriptor from ``q [n_seq, n_layers, Hq, W, D]`` and ``k, v [n_seq, n_layers, Hkv, L, D]``;
    keyword arguments set fields of ``shape.tuning`` (e.g. ``score_chunk=2048``)."""
    import torch

    assert q.dim() == 5 and k.dim() == 5 and q.stride(-1) == 1 and k.stride(-1) == 1
    assert q.dtype == k.dtype and q.dtype in (torch.float32, torch.bfloat16)
    s = CShape()
    s.n_seq, s.n_layers, s.n_q_heads, s.window, s.head_dim = q.shape
    s.n_kv_heads, s.seq_len = k.shape[2], k.shape[3]
    s.dtype = SABLOCK_F32 if q.dtype == torch.float32 else SABLOCK_BF16
    vv = k if v is None else v
    for a in range(4):
        s.q_stride[a] = q.stride(a)
        s.k_stride[a] = k.stride(a)
        s.v_stride[a] = vv.stride(a)
    for name, val in tuning.items():
        setattr(s.tuning, name, int(val))
    return s


@dataclass
class Segments:
    """Segment offsets: ``seg_off`` device int32 CSR, ``seg_ptr`` host ints, ``max_segments`` row stride."""

    seg_off: "object"
    seg_ptr: Sequence[int]
    max_segments: int

    def c_ptr(self):
        return (ctypes.c_int32 * len(self.seg_ptr))(*[int(x) for x in self.seg_ptr])


def make_segments(seg_off_host, seg_ptr_host, device) -> Segments:
    import numpy as np
    import torch

    ptr = [int(x) for x in seg_ptr_host]
    mx = max(ptr[i + 1] - ptr[i] - 1 for i in range(len(ptr) - 1))
    return Segments(torch.as_tensor(np.asarray(seg_off_host, dtype=np.int32)).to(device), ptr, mx)


def sablock_workspace_bytes(shape: CShape, max_segments: int, budget: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().sablock_workspace_bytes(ctypes.byref(shape), max_segments, budget, ctypes.byref(out)))
    return int(out.value)


def n_problems(shape: CShape) -> int:
    return shape.n_seq * shape.n_layers * shape.n_kv_heads


def sablock_score(shape: CShape, q, k, s_out, ent_out, ws, eps: float = 1e-6, row_lse=None, stream=None):
    _check(load().sablock_score(ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(row_lse), eps, _ptr(s_out),
                                _ptr(ent_out), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def sablock_stream_probe(shape: CShape, k, sink, read_lds: bool = False, s_out=None, ent_out=None, stream=None):
    """Measurement aid: K through the scoring kernels' load ring, no arithmetic; with ``s_out`` / ``ent_out`` also
    the column pass's stores."""
    _check(load().sablock_stream_probe(ctypes.byref(shape), _ptr(k), 1 if read_lds else 0, _ptr(s_out), _ptr(ent_out),
                                       _ptr(sink), _stream(stream)))


STATIC_SCRATCH_BYTES = 8 << 20
SLICE_TOKENS, MAX_SLICES = 16384, 128          # of the segmentation by slices (sablock_segment_slices)


def sablock_score_static(shape: CShape, q, k, s_out, ent_out, eps: float = 1e-6, row_lse=None, stream=None):
    """``sablock_score`` without a workspace argument: the row statistics live in the library's own static array."""
    _check(load().sablock_score_static(ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(row_lse), eps, _ptr(s_out),
                                       _ptr(ent_out), _stream(stream)))


def sablock_refine(shape: CShape, s, ent, seg: Segments, s_tilde_out, ws, alpha=0.9, eta=1.0,
                   omega_out=None, stream=None):
    hp = CHparams(0.0, alpha, eta, 0.0)
    _check(load().sablock_refine(ctypes.byref(shape), _ptr(s), _ptr(ent), _ptr(seg.seg_off), seg.c_ptr(),
                                 seg.max_segments, ctypes.byref(hp), _ptr(s_tilde_out), _ptr(omega_out),
                                 _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def sablock_search_blocks(shape: CShape, s_tilde, seg: Segments, cand: Sequence[int], budget: int, tau: float,
                          seg_budget_out, block_size_out, ws, stream=None, topb_out=None):
    c = (ctypes.c_int32 * len(cand))(*[int(x) for x in cand])
    _check(load().sablock_search_blocks(ctypes.byref(shape), _ptr(s_tilde), _ptr(seg.seg_off), seg.c_ptr(),
                                        seg.max_segments, c, len(cand), budget, tau, _ptr(seg_budget_out),
                                        _ptr(block_size_out), _ptr(topb_out), _ptr(ws),
                                        ws.numel() * ws.element_size(), _stream(stream)))


def sablock_select(shape: CShape, s_tilde, seg: Segments, seg_budget, block_size, budget: int,
                   idx_out, n_sel_out, ws, stream=None, topb=None):
    _check(load().sablock_select(ctypes.byref(shape), _ptr(s_tilde), _ptr(seg.seg_off), seg.c_ptr(),
                                 seg.max_segments, _ptr(seg_budget), _ptr(block_size), _ptr(topb), budget,
                                 _ptr(idx_out), _ptr(n_sel_out), _ptr(ws), ws.numel() * ws.element_size(),
                                 _stream(stream)))


def sablock_search_select(shape: CShape, s_tilde, seg: Segments, cand: Sequence[int], budget: int, tau: float,
                          seg_budget_out, block_size_out, idx_out, n_sel_out, ws, stream=None, topb_out=None):
    c = (ctypes.c_int32 * len(cand))(*[int(x) for x in cand])
    _check(load().sablock_search_select(ctypes.byref(shape), _ptr(s_tilde), _ptr(seg.seg_off), seg.c_ptr(),
                                        seg.max_segments, c, len(cand), budget, tau, _ptr(seg_budget_out),
                                        _ptr(block_size_out), _ptr(topb_out), _ptr(idx_out), _ptr(n_sel_out),
                                        _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def sablock_compact(shape: CShape, k, v, idx, n_sel, budget: int, append_window: bool, k_out, v_out,
                    stream=None):
    _check(load().sablock_compact(ctypes.byref(shape), _ptr(k), _ptr(v), _ptr(idx), _ptr(n_sel), budget,
                                  1 if append_window else 0, _ptr(k_out), _ptr(v_out), _stream(stream)))


def sablock_segment_count(token_ids, delims: Sequence[int], seg_count_out, stream=None):
    """``token_ids [n_seq, T]`` int32 (row stride in elements taken from the tensor) -> ``seg_count_out [n_seq]``."""
    d = (ctypes.c_int32 * max(len(delims), 1))(*[int(x) for x in delims])
    _check(load().sablock_segment_count(_ptr(token_ids), token_ids.stride(0), token_ids.shape[0], token_ids.shape[1],
                                        d, len(delims), _ptr(seg_count_out), _stream(stream)))


def sablock_segment_offsets(token_ids, delims: Sequence[int], seg_ptr: Sequence[int], seg_off_out, stream=None):
    d = (ctypes.c_int32 * max(len(delims), 1))(*[int(x) for x in delims])
    sp = (ctypes.c_int32 * len(seg_ptr))(*[int(x) for x in seg_ptr])
    _check(load().sablock_segment_offsets(_ptr(token_ids), token_ids.stride(0), token_ids.shape[0],
                                          token_ids.shape[1], d, len(delims), sp, _ptr(seg_off_out), _stream(stream)))


def sablock_validate_segments(seg_off, seg_ptr: Sequence[int], n_tokens: int, n_bad_out, stream=None):
    sp = (ctypes.c_int32 * len(seg_ptr))(*[int(x) for x in seg_ptr])
    _check(load().sablock_validate_segments(_ptr(seg_off), sp, len(seg_ptr) - 1, int(n_tokens), _ptr(n_bad_out),
                                            _stream(stream)))


def segment(token_ids, delims: Sequence[int]) -> "Segments":
    """Both segmentation calls and the host step between them (one wait for n_seq counts)."""
    import torch

    assert token_ids.dim() == 2 and token_ids.dtype == torch.int32 and token_ids.stride(1) == 1
    lib, stream = load(), torch.cuda.current_stream(token_ids.device)
    n, T = token_ids.shape
    tokens = (token_ids.data_ptr(), token_ids.stride(0), n, T)
    d = (ctypes.c_int32 * max(len(delims), 1))(*[int(x) for x in delims])
    st = stream.cuda_stream or None
    # the kernel writes the counts straight to host memory: no copy between it and the wait
    # up to one slice per sequence, or too many for one call: by whole sequences (one sequence of 5 000 tokens 25.7 us, 26.3 as
    # a slice; of 60 000 39.1 and 27.2)
    per = -(-T // SLICE_TOKENS)
    per = per if per > 1 and n * per <= MAX_SLICES else 0
    counts = torch.empty((n * (per or 1),), dtype=torch.int32, device="cpu", pin_memory=True)
    _check((lib.sablock_segment_slice_count if per else lib.sablock_segment_count)(*tokens, d, len(delims), counts.data_ptr(), st))
    stream.synchronize()
    at, place = 0, [0]                                         # of slices or of whole sequences
    for i, k in enumerate(counts.tolist(), 1):
        at += k + (0 if i % per else 2) if per else k + 1      # a sequence's offsets are its boundaries and both ends
        place.append(at)
    ptr = place[::per or 1]
    seg_off = torch.empty((at,), dtype=torch.int32, device=token_ids.device)
    _check((lib.sablock_segment_slice_offsets if per else lib.sablock_segment_offsets)(
        *tokens, d, len(delims), (ctypes.c_int32 * len(place))(*place), seg_off.data_ptr(), st))
    return Segments(seg_off, ptr, max(b - a for a, b in zip(ptr, ptr[1:])) - 1)


def layer_shape(shape: CShape) -> CShape:
    """The shape to pass to refine / search_blocks / select when scores are per (sequence, layer)."""
    s = CShape.from_buffer_copy(shape)
    s.n_q_heads = s.n_kv_heads = 1
    return s


def sablock_score_all_heads_workspace_bytes(shape: CShape) -> int:
    out = ctypes.c_size_t(0)
    _check(load().sablock_score_all_heads_workspace_bytes(ctypes.byref(shape), ctypes.byref(out)))
    return int(out.value)


def sablock_score_all_heads(shape: CShape, q, k, s_out, ent_out, ws, eps: float = 1e-6, row_lse=None, stream=None):
    _check(load().sablock_score_all_heads(ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(row_lse), eps, _ptr(s_out),
                                          _ptr(ent_out), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def sablock_compact_shared(shape: CShape, k, v, idx, n_sel, budget: int, append_window: bool, k_out, v_out,
                           stream=None):
    _check(load().sablock_compact_shared(ctypes.byref(shape), _ptr(k), _ptr(v), _ptr(idx), _ptr(n_sel), budget,
                                         1 if append_window else 0, _ptr(k_out), _ptr(v_out), _stream(stream)))


def sablock_window_attention_workspace_bytes(shape: CShape) -> int:
    out = ctypes.c_size_t(0)
    _check(load().sablock_window_attention_workspace_bytes(ctypes.byref(shape), ctypes.byref(out)))
    return int(out.value)


def sablock_window_attention(shape: CShape, q, k, v, out, row_lse_out, ws, stream=None):
    _check(load().sablock_window_attention(ctypes.byref(shape), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(row_lse_out),
                                           _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def make_cache_shape(q, k_cache, v_cache=None) -> CShape:
    """Shape of a decode call: ``q [n_seq, n_layers, Hq, D]`` and a cache ``[n_seq, n_layers, Hkv, rows, D]``
    (any strides on the four outer axes; a compacted cache ``[P, rows, D]`` is viewed that way by the caller)."""
    import torch

    assert q.dim() == 4 and k_cache.dim() == 5 and q.is_contiguous() and k_cache.stride(-1) == 1
    assert q.dtype == k_cache.dtype and q.dtype in (torch.float32, torch.bfloat16)
    s = CShape()
    s.n_seq, s.n_layers, s.n_q_heads, s.head_dim = q.shape
    s.n_kv_heads, s.seq_len = k_cache.shape[2], k_cache.shape[3]
    s.window = 1
    s.dtype = SABLOCK_F32 if q.dtype == torch.float32 else SABLOCK_BF16
    vv = k_cache if v_cache is None else v_cache
    for a in range(4):
        s.q_stride[a] = 0
        s.k_stride[a] = k_cache.stride(a)
        s.v_stride[a] = vv.stride(a)
    return s


def sablock_decode_workspace_bytes(shape: CShape) -> int:
    out = ctypes.c_size_t(0)
    _check(load().sablock_decode_workspace_bytes(ctypes.byref(shape), ctypes.byref(out)))
    return int(out.value)


def sablock_decode_attention(shape: CShape, q, k_cache, v_cache, out, ws, n_sel=None, budget: int = 0, stream=None):
    _check(load().sablock_decode_attention(ctypes.byref(shape), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(n_sel),
                                           budget, _ptr(out), _ptr(ws), ws.numel() * ws.element_size(),
                                           _stream(stream)))


def make_pages(k_pool, v_pool, page_table, n_q_heads: int, compute_units: int = 0) -> CPages:
    """Descriptor of a paged cache from its pools ``[n_layers, n_pages, Hkv, page_size, D]`` (any strides on the four outer axes) and
    ``page_table [n_seq, max_pages]`` int32."""
    import torch

    assert k_pool.dim() == 5 and v_pool.shape == k_pool.shape and k_pool.stride(-1) == 1 and v_pool.stride(-1) == 1
    assert k_pool.dtype == v_pool.dtype and k_pool.dtype in (torch.float32, torch.bfloat16)
    assert page_table.dim() == 2 and page_table.dtype == torch.int32 and page_table.is_contiguous()
    c = CPages()
    c.n_layers, c.n_pages, c.n_kv_heads, c.page_size, c.head_dim = k_pool.shape
    c.n_seq, c.max_pages = page_table.shape
    c.n_q_heads, c.compute_units = int(n_q_heads), int(compute_units)
    c.dtype = SABLOCK_F32 if k_pool.dtype == torch.float32 else SABLOCK_BF16
    for a in range(4):
        c.k_stride[a], c.v_stride[a] = k_pool.stride(a), v_pool.stride(a)
    return c


def make_new_tokens(k, v, q=None, rotary_dim: Optional[int] = None, interleaved: bool = False) -> CNewTokens:
    """Descriptor of the new tokens of an append: ``k, v [n_seq, n_layers, Hkv, n_new, D]``, ``q [n_seq, n_layers, Hq, n_new, D]``, any
    strides on the four outer axes; ``rotary_dim`` None = the whole head.  Without ``q`` it describes appends without queries."""
    assert k.dim() == 5 and v.shape == k.shape and k.stride(-1) == 1 and v.stride(-1) == 1 and k.dtype == v.dtype
    assert q is None or (q.dim() == 5 and q.dtype == k.dtype and q.stride(-1) == 1 and (q.shape[:2] + q.shape[3:]) == (k.shape[:2] + k.shape[3:]))
    t = CNewTokens()
    t.n_new, t.rotary_dim, t.interleaved = k.shape[3], k.shape[4] if rotary_dim is None else int(rotary_dim), 1 if interleaved else 0
    for a in range(4):
        t.k_stride[a], t.v_stride[a] = k.stride(a), v.stride(a)
        t.q_stride[a] = 0 if q is None else q.stride(a)
    return t


class _Layout(NamedTuple):
    """What the kernels make of a cache's descriptor."""

    dtype: object
    n_seq: int
    max_pages: int
    k_pool: _Extent
    v_pool: _Extent
    problems: int
    queries: int                               # elements of one query per head
    bounds: int                                # elements


def _dtype_of(code: int):
    return _torch.float32 if code == SABLOCK_F32 else _torch.bfloat16


# By the descriptors' contents: their fields read one by one would cost a call as much as the launch
@lru_cache(256)
def _cache_layout(pages: bytes) -> _Layout:
    n_seq, n_layers, n_q_heads, n_kv_heads, head_dim, dtype, page_size, n_pages, max_pages, _, _, _, *steps = struct.unpack_from("12i8q", pages)
    sizes = (n_layers, n_pages, n_kv_heads, page_size, head_dim)
    return _Layout(_dtype_of(dtype), n_seq, max_pages, _extent("K pool", sizes, (*steps[:4], 1)), _extent("V pool", sizes, (*steps[4:], 1)),
                   n_seq * n_layers * n_kv_heads, n_seq * n_layers * n_q_heads * head_dim, 2 * n_layers * n_pages * n_kv_heads * head_dim)


@lru_cache(256)
def _tokens_layout(pages: bytes, tokens: bytes):
    """The cache's layout, new tokens per sequence, extents of q, k and v, elements of the angles' frequencies."""
    n_seq, n_layers, n_q_heads, n_kv_heads, head_dim = struct.unpack_from("5i", pages)
    n_new, rotary_dim, _, _, *steps = struct.unpack_from("4i12q", tokens)
    sizes = (n_seq, n_layers, n_kv_heads, n_new, head_dim)
    return (_cache_layout(pages), n_new, _extent("q", (n_seq, n_layers, n_q_heads, n_new, head_dim), (*steps[:4], 1)),
            _extent("k", sizes, (*steps[4:8], 1)), _extent("v", sizes, (*steps[8:], 1)), rotary_dim // 2)


def _table(c: _Layout, page_table):
    if page_table.dtype is not _torch.int32 or page_table.numel() != c.n_seq * c.max_pages or not page_table.is_contiguous():
        _dense(_torch.int32, c.n_seq * c.max_pages, page_table)
        if page_table.dim() == 2 and c.n_seq > 1 and page_table.shape[1] != c.max_pages:
            raise ValueError(f"a page table of {page_table.shape[1]} entries per sequence, the descriptor says {c.max_pages}")


def sablock_compact_paged(shape: CShape, k, v, idx, budget: int, append_window: bool, pages: CPages, page_table, k_pool, v_pool, bounds=None,
                          lengths_out=None, stream=None):
    lib = load()
    device, k_at, v_at, idx_at, table, kp, vp, b, lengths = _pointers(k, v, idx, page_table, k_pool, v_pool, bounds, lengths_out)
    c = _cache_layout(bytes(pages))
    _table(c, page_table)
    _strided(c.dtype, (k_pool, c.k_pool), (v_pool, c.v_pool))
    _all_dense((_torch.int32, c.problems * budget, idx), (_torch.int32, c.n_seq, lengths_out), (c.dtype, c.bounds, bounds))
    _check(lib.sablock_compact_paged(ctypes.byref(shape), k_at, v_at, idx_at, budget, 1 if append_window else 0, ctypes.byref(pages), table, kp, vp,
                                     b, lengths, _stream(stream, device)))


def sablock_append_paged(pages: CPages, tokens: CNewTokens, k, v, positions, inv_freq, page_table, lengths, k_pool, v_pool, q=None, q_out=None,
                         counts=None, bounds=None, stream=None):
    """``lengths`` are the rows of every sequence WITH the new tokens; q, k and v have the sizes and strides of those that ``tokens`` was made of."""
    lib = load()
    device, k_at, v_at, pos, freq, table, rows, kp, vp, q_at, out, count, b = _pointers(k, v, positions, inv_freq, page_table, lengths, k_pool, v_pool,
                                                                                        q, q_out, counts, bounds)
    c, n_new, q_extent, k_extent, v_extent, n_freq = _tokens_layout(bytes(pages), bytes(tokens))
    i32 = _torch.int32
    _table(c, page_table)
    if q is not None:
        _strided(c.dtype, (q, q_extent), (k, k_extent), (v, v_extent), (k_pool, c.k_pool), (v_pool, c.v_pool))
    else:
        _strided(c.dtype, (k, k_extent), (v, v_extent), (k_pool, c.k_pool), (v_pool, c.v_pool))
    _all_dense((i32, c.n_seq, lengths), (i32, c.n_seq, positions), (i32, c.n_seq, counts), (_torch.float32, n_freq, inv_freq),
               (c.dtype, c.queries * n_new, q_out), (c.dtype, c.bounds, bounds))
    _check(lib.sablock_append_paged(ctypes.byref(pages), ctypes.byref(tokens), q_at, k_at, v_at, count, pos, freq, table, rows, out, kp, vp, b,
                                    _stream(stream, device)))


def sablock_decode_paged_workspace_bytes(pages: CPages) -> int:
    out = ctypes.c_size_t(0)
    _check(load().sablock_decode_paged_workspace_bytes(ctypes.byref(pages), ctypes.byref(out)))
    return int(out.value)


def sablock_decode_paged(pages: CPages, q, k_pool, v_pool, page_table, lengths, out, ws, page_list=None, stream=None):
    """``page_list [P, n]`` int32, dense: the pages to read (``sablock_select_pages``); None = all."""
    lib = load()
    device, q_at, kp, vp, table, rows, o, ws_at, listed = _pointers(q, k_pool, v_pool, page_table, lengths, out, ws, page_list)
    n = 0 if page_list is None else page_list.shape[-1]
    c = _cache_layout(bytes(pages))
    _table(c, page_table)
    _strided(c.dtype, (k_pool, c.k_pool), (v_pool, c.v_pool))
    _all_dense((_torch.int32, c.n_seq, lengths), (_torch.int32, c.problems * n, page_list), (c.dtype, c.queries, q), (_torch.float32, c.queries, out))
    _check(lib.sablock_decode_paged(ctypes.byref(pages), q_at, kp, vp, table, rows, listed, n, o, ws_at, ws.numel() * ws.element_size(),
                                    _stream(stream, device)))


def sablock_select_pages_workspace_bytes(pages: CPages) -> int:
    out = ctypes.c_size_t(0)
    _check(load().sablock_select_pages_workspace_bytes(ctypes.byref(pages), ctypes.byref(out)))
    return int(out.value)


def sablock_select_pages(pages: CPages, q, bounds, page_table, lengths, n_pick: int, list_out, ws, n_first: int = 1, n_last: int = 1, stream=None):
    lib = load()
    device, q_at, b, table, rows, listed, ws_at = _pointers(q, bounds, page_table, lengths, list_out, ws)
    c = _cache_layout(bytes(pages))
    _table(c, page_table)
    _all_dense((_torch.int32, c.n_seq, lengths), (_torch.int32, c.problems * n_pick, list_out), (c.dtype, c.queries, q), (c.dtype, c.bounds, bounds))
    _check(lib.sablock_select_pages(ctypes.byref(pages), q_at, b, table, rows, n_pick, n_first, n_last, listed, ws_at,
                                    ws.numel() * ws.element_size(), _stream(stream, device)))


class PagedCache:
    """Pools, page table and lengths of a paged cache, page bounds where asked for, and the workspaces of the calls that read it.

    Which pages a sequence has is the caller's to say: ``page_table`` starts as -1 (no page).  The workspaces serve one call at a time:
    calls that may overlap, on two streams or in two captured graphs, bring their own."""

    def __init__(self, n_seq: int, n_layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, page_size: int, n_pages: int, max_pages: int,
                 dtype, device, bounds: bool = True):
        import torch

        self.k_pool, self.v_pool = (torch.zeros((n_layers, n_pages, n_kv_heads, page_size, head_dim), dtype=dtype, device=device) for _ in range(2))
        self.bounds = torch.zeros((n_layers, n_pages, n_kv_heads, 2, head_dim), dtype=dtype, device=device) if bounds else None
        self.page_table = torch.full((n_seq, max_pages), -1, dtype=torch.int32, device=device)
        self.lengths = torch.zeros((n_seq,), dtype=torch.int32, device=device)
        self.pages = make_pages(self.k_pool, self.v_pool, self.page_table, n_q_heads)
        self.ws = torch.empty((sablock_decode_paged_workspace_bytes(self.pages),), dtype=torch.uint8, device=device)
        self.select_ws = torch.empty((sablock_select_pages_workspace_bytes(self.pages),), dtype=torch.uint8, device=device) if bounds else None


class Buffers:
    """Device buffers for one call geometry: outputs of every step plus the workspace.

    Allocation happens here, once; the five ``sablock_*`` calls then only enqueue kernels.  ``dense=False``: without ``k_out`` and
    ``v_out``, for a cache in pages.
    """

    def __init__(self, shape: CShape, seg: Segments, budget: int, device, append_window: bool = True,
                 dtype=None, dense: bool = True):
        import torch

        P, L, W, D = n_problems(shape), shape.seq_len, shape.window, shape.head_dim
        T = L - W
        ms = max(seg.max_segments, 1)
        dt = dtype or (torch.float32 if shape.dtype == SABLOCK_F32 else torch.bfloat16)
        self.budget, self.append_window = budget, append_window
        self.s = torch.empty((P, L), dtype=torch.float32, device=device)
        self.ent = torch.empty((P, L), dtype=torch.float32, device=device)
        self.s_tilde = torch.empty((P, T), dtype=torch.float32, device=device)
        self.omega = torch.empty((P, ms), dtype=torch.float32, device=device)
        self.seg_budget = torch.empty((P, ms), dtype=torch.int32, device=device)
        self.block_size = torch.empty((P, ms), dtype=torch.int32, device=device)
        self.idx = torch.empty((P, max(budget, 1)), dtype=torch.int32, device=device)
        self.n_sel = torch.empty((P,), dtype=torch.int32, device=device)
        self.topb = torch.empty((P, 2), dtype=torch.int32, device=device)
        rows = budget + (W if append_window else 0)
        self.k_out, self.v_out = (torch.empty((P, max(rows, 1), D), dtype=dt, device=device) if dense else None for _ in range(2))
        self.ws = torch.empty((sablock_workspace_bytes(shape, seg.max_segments, budget),), dtype=torch.uint8,
                              device=device)


def compress(shape: CShape, q, k, v, seg: Segments, cand: Sequence[int], budget: int, buf: Buffers,
             eps=1e-6, alpha=0.9, eta=1.0, tau=0.85, row_lse=None, stream=None, fused=True, cache: Optional[PagedCache] = None) -> Buffers:
    """The whole hot path: score, refine, search_blocks + select (one call for both, or the two separate calls with
    ``fused=False``: same results), compact: into ``buf.k_out`` / ``buf.v_out``, or into the pages of ``cache`` where one is given (its
    ``lengths`` are written, and its bounds)."""
    if cache is None and buf.k_out is None:
        raise ValueError("buffers without k_out and v_out are for a cache in pages")
    # the calls above with their arguments marshalled once: small calls are bound by what the host does between launches
    lib, st, sp = load(), _stream(stream), ctypes.byref(shape)
    s, ent, s_tilde, topb, idx, n_sel = (_ptr(t) for t in (buf.s, buf.ent, buf.s_tilde, buf.topb, buf.idx, buf.n_sel))
    kp, bk, g = _ptr(k), _ptr(buf.seg_budget), _ptr(buf.block_size)
    ws = (_ptr(buf.ws), buf.ws.numel() * buf.ws.element_size(), st)
    segs = (_ptr(seg.seg_off), seg.c_ptr(), seg.max_segments)
    cl = ((ctypes.c_int32 * len(cand))(*[int(x) for x in cand]), len(cand))
    _check(lib.sablock_score(sp, _ptr(q), kp, _ptr(row_lse), eps, s, ent, *ws))
    _check(lib.sablock_refine(sp, s, ent, *segs, ctypes.byref(CHparams(0.0, alpha, eta, 0.0)), s_tilde, _ptr(buf.omega), *ws))
    if fused:
        _check(lib.sablock_search_select(sp, s_tilde, *segs, *cl, budget, tau, bk, g, topb, idx, n_sel, *ws))
    else:
        _check(lib.sablock_search_blocks(sp, s_tilde, *segs, *cl, budget, tau, bk, g, topb, *ws))
        _check(lib.sablock_select(sp, s_tilde, *segs, bk, g, topb, budget, idx, n_sel, *ws))
    if cache is not None:
        sablock_compact_paged(shape, k, v, buf.idx, budget, buf.append_window, cache.pages, cache.page_table, cache.k_pool, cache.v_pool,
                              cache.bounds, cache.lengths, stream)
        return buf
    _check(lib.sablock_compact(sp, kp, _ptr(v), idx, n_sel, budget, 1 if buf.append_window else 0, _ptr(buf.k_out),
                               _ptr(buf.v_out), st))
    return buf
