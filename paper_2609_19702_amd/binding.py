"""ctypes binding of ``libdsa.so`` (declared in ``include/dsa.h``).

Argument marshalling only: every step of the decode path runs in the HIP
kernels of the library.  PyTorch supplies device memory (tensors) and the
stream (``torch.cuda.current_stream()``); this module passes their raw
pointers through the C ABI and turns non-zero status codes into
``DSAError``.  There is no fallback: if the library is missing the import
of the entry points fails.
"""

from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional

import torch  # loads the HIP runtime that libdsa.so binds to (same soname)

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libdsa.so")

MODE_DENSE = 0
MODE_DIAGONAL = 1
MODE_WINDOW = 2
KV_BF16 = 0
KV_FP8_E4M3 = 1

FLAG_INACTIVE = 1
FLAG_POS_CLAMPED = 2
FLAG_STATE_BEHIND = 4
FLAG_BAD_OFFSET = 8
FLAG_COUNT = 16
TREE_FLAG_BAD_PARENT = 1
MAX_TREE_NODES = 256
PAGE_FLAG_NO_PAGES = 1
PAGE_FLAG_TOO_LONG = 2
MAX_PAGED_BATCH = 4096
MAX_BEAMS = 16

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP = 0, -1, -2, -3, -4


class DSAError(RuntimeError):
    def __init__(self, status: int, where: str):
        super().__init__(f"{where}: {status_str(status)} (status {status})")
        self.status = status


class Params(C.Structure):
    _fields_ = [("prompt_len", C.c_int32), ("grid_h", C.c_int32), ("grid_w", C.c_int32),
                ("window", C.c_int32), ("n_att", C.c_int32), ("mode", C.c_int32),
                ("sinks", C.c_int32)]

    def __repr__(self):
        return (f"Params(prompt_len={self.prompt_len}, grid={self.grid_h}x{self.grid_w}, "
                f"window={self.window}, n_att={self.n_att}, mode={self.mode}, sinks={self.sinks})")


class Shape(C.Structure):
    _fields_ = [("batch", C.c_int32), ("num_q_heads", C.c_int32),
                ("num_kv_heads", C.c_int32), ("head_dim", C.c_int32)]


class KVLayout(C.Structure):
    _fields_ = [("d_row_base", C.c_void_p), ("stride_batch", C.c_int64),
                ("stride_head", C.c_int64), ("stride_row", C.c_int64),
                ("ring_rows", C.c_int64), ("d_k_scale", C.c_void_p), ("d_v_scale", C.c_void_p),
                ("dtype", C.c_int32)]
    # values of the tensors that ``kv_layout`` was given (no bound is known of raw pointers)
    scales = bases = 1 << 62


class PlanLayout(C.Structure):
    _fields_ = [("count_offset", C.c_size_t), ("flags_offset", C.c_size_t),
                ("indices_offset", C.c_size_t), ("cap", C.c_int32), ("bytes", C.c_size_t)]


class StateLayout(C.Structure):
    _fields_ = [("count_offset", C.c_size_t), ("flags_offset", C.c_size_t),
                ("offsets_offset", C.c_size_t), ("cap", C.c_int32), ("bytes", C.c_size_t),
                ("kept_count_offset", C.c_size_t), ("kept_offset", C.c_size_t),
                ("kept_cap", C.c_int32), ("kept_stride", C.c_int32)]


class LaunchInfo(C.Structure):
    _fields_ = [("rows_per_split", C.c_int32), ("max_splits", C.c_int32),
                ("workgroups", C.c_int32), ("kernel_variant", C.c_int32),
                ("waves_per_group", C.c_int32), ("workspace_bytes", C.c_size_t),
                ("kept_read", C.c_int32)]


class TreeRequest(C.Structure):  # dsa_tree
    _fields_ = [("nodes", C.c_int32), ("d_base", C.c_void_p), ("d_count", C.c_void_p),
                ("d_plan", C.c_void_p)]


class NodeRows(C.Structure):
    _fields_ = [("stride_batch", C.c_int64), ("stride_node", C.c_int64),
                ("stride_head", C.c_int64), ("stride_layer", C.c_int64)]


class TreePlanLayout(C.Structure):
    _fields_ = [("flags_offset", C.c_size_t), ("max_depth_offset", C.c_size_t),
                ("depth_offset", C.c_size_t), ("parent_offset", C.c_size_t),
                ("ancestors_offset", C.c_size_t), ("words", C.c_int32), ("bytes", C.c_size_t)]


class TreeLaunchInfo(C.Structure):
    _fields_ = [("rows_per_tile", C.c_int32), ("row_tiles", C.c_int32), ("splits", C.c_int32),
                ("workgroups", C.c_int32), ("workspace_bytes", C.c_size_t)]


class PagesStruct(C.Structure):  # dsa_pages
    _fields_ = [("page_rows", C.c_int32), ("max_pages", C.c_int32), ("num_pages", C.c_int32),
                ("d_table", C.c_void_p), ("d_refs", C.c_void_p), ("d_cursor", C.c_void_p),
                ("d_prompt", C.c_void_p)]


class PageLayout(C.Structure):
    _fields_ = [("num_pages", C.c_int32), ("page_rows", C.c_int32), ("stride_page", C.c_int64),
                ("stride_head", C.c_int64), ("stride_row", C.c_int64), ("d_k_scale", C.c_void_p),
                ("d_v_scale", C.c_void_p), ("dtype", C.c_int32)]

    def __setattr__(self, name, value):
        super().__setattr__(name, value)
        if name != "_fits":  # what was looked at before is looked at again
            super().__setattr__("_fits", None)


class PagedLaunchInfo(C.Structure):
    _fields_ = [("rows_per_split", C.c_int32), ("max_splits", C.c_int32),
                ("waves_per_group", C.c_int32), ("workgroups", C.c_int32),
                ("workspace_bytes", C.c_size_t)]


# name -> (restype, argtypes); mirrors include/dsa.h
_P, _S = C.POINTER(Params), C.POINTER(Shape)
_T, _R = C.POINTER(TreeRequest), C.POINTER(NodeRows)
_G, _L = C.POINTER(PagesStruct), C.POINTER(PageLayout)
_VP = C.c_void_p
SIGNATURES = {
    "dsa_abi_version": (C.c_int32, []),
    "dsa_status_str": (C.c_char_p, [C.c_int32]),
    "dsa_params_from_sparsity": (C.c_int32, [C.c_int32] * 7 + [_P]),
    "dsa_validate": (C.c_int32, [_P, _S]),
    "dsa_get_state_layout": (C.c_int32, [_P, _S, C.POINTER(StateLayout)]),
    "dsa_get_plan_layout": (C.c_int32, [_P, _S, C.POINTER(PlanLayout)]),
    "dsa_get_launch_info": (C.c_int32, [_P, _S, C.POINTER(LaunchInfo)]),
    "dsa_state_bytes": (C.c_size_t, [_P, _S]),
    "dsa_plan_bytes": (C.c_size_t, [_P, _S]),
    "dsa_workspace_bytes": (C.c_size_t, [_P, _S]),
    "dsa_window_logits_count": (C.c_size_t, [_P, _S]),
    "dsa_state_reset": (C.c_int32, [_P, _S, _VP, _VP, _VP]),
    "dsa_plan": (C.c_int32, [_P, _S, _VP, _VP, _VP, C.c_size_t, _VP]),
    "dsa_decode_attention": (C.c_int32, [_P, _S, _VP, _VP, _VP, C.POINTER(KVLayout), _VP, _VP,
                                         C.c_float, _VP, _VP, _VP, C.c_size_t, _VP]),
    "dsa_decode_attention_timed": (C.c_int32, [_P, _S, _VP, _VP, _VP, C.POINTER(KVLayout), _VP,
                                               _VP, C.c_float, _VP, _VP, _VP, C.c_size_t, _VP,
                                               _VP, _VP]),
    "dsa_decode_step": (C.c_int32, [_P, _S, _VP, _VP, _VP, C.POINTER(KVLayout), _VP, _VP, _VP,
                                    C.c_size_t, C.c_float, _VP, _VP, _VP, C.c_size_t, _VP]),
    "dsa_decode_step_timed": (C.c_int32, [_P, _S, _VP, _VP, _VP, C.POINTER(KVLayout), _VP, _VP,
                                          _VP, C.c_size_t, C.c_float, _VP, _VP, _VP, C.c_size_t,
                                          _VP, _VP, _VP]),
    "dsa_decode_step_noalloc": (C.c_int32, [_P, _S, _VP, _VP, _VP, C.POINTER(KVLayout), _VP, _VP,
                                            _VP, C.c_size_t, C.c_float, _VP, _VP, _VP]),
    "dsa_select": (C.c_int32, [_P, _S, _VP, _VP, _VP, _VP, _VP]),
    "dsa_get_tree_plan_layout": (C.c_int32, [C.c_int32, C.c_int32, C.POINTER(TreePlanLayout)]),
    "dsa_tree_plan_bytes": (C.c_size_t, [C.c_int32, C.c_int32]),
    "dsa_get_tree_launch_info": (C.c_int32, [_P, _S, C.c_int32, C.POINTER(TreeLaunchInfo)]),
    "dsa_tree_workspace_bytes": (C.c_size_t, [_P, _S, C.c_int32]),
    "dsa_tree_plan": (C.c_int32, [C.c_int32, C.c_int32, _VP, _VP, _VP, C.c_size_t, _VP]),
    "dsa_tree_attention": (C.c_int32, [_P, _S, _T, _VP, _R, _VP, _VP, _R, _VP, _VP,
                                       C.POINTER(KVLayout), C.c_float, _VP, C.c_int32, _VP,
                                       C.c_size_t, _VP]),
    "dsa_tree_verify": (C.c_int32, [C.c_int32, C.c_int32, _T] + [_VP] * 8),
    "dsa_kv_append": (C.c_int32, [_P, _S, _T, _VP, _VP, _R, _VP, _VP, C.c_int32, _VP, _VP,
                                  C.POINTER(KVLayout), C.c_int64, _VP]),
    "dsa_get_paged_launch_info": (C.c_int32, [_P, _S, C.POINTER(PagedLaunchInfo)]),
    "dsa_paged_workspace_bytes": (C.c_size_t, [_P, _S]),
    "dsa_page_update": (C.c_int32, [_P, C.c_int32, _G, _VP, _VP, C.c_int32] + [_VP] * 5),
    "dsa_page_reorder": (C.c_int32, [C.c_int32, _G, _VP, _VP]),
    "dsa_paged_append": (C.c_int32, [_S, C.c_int32, _VP, _VP, _VP, _R, C.c_int32, _VP, _VP, _L,
                                     C.c_int64, _VP, _VP]),
    "dsa_paged_attention": (C.c_int32, [_P, _S, _G, _VP, _VP, _VP, _L, _VP, _VP, C.c_float, _VP,
                                        C.c_int32, _VP, _VP, C.c_size_t, _VP]),
    "dsa_beam_workspace_bytes": (C.c_size_t, [C.c_int32] * 3),
    "dsa_beam_select": (C.c_int32, [C.c_int32] * 3 + [_VP, C.c_int64, C.c_int32] + [_VP] * 5
                        + [C.c_size_t, _VP]),
}

NOALLOC_SCRATCH_BYTES = 16 << 20  # DSA_NOALLOC_SCRATCH_BYTES

_lib = None


def lib() -> C.CDLL:
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2609_19702_amd.build` (there is no fallback)")
        L = C.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


def status_str(status: int) -> str:
    return lib().dsa_status_str(int(status)).decode()


def _check(status: int, where: str):
    if status != OK:
        raise DSAError(status, where)


def _ptr(x) -> Optional[int]:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        # the handle of torch.cuda.current_stream() without the Stream object
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _nbytes(x) -> int:
    return x.nbytes


def _need(x, name, dtype=None, min_bytes=0, contiguous=True):
    """Argument checks before a device call (tensors only; raw integer
    pointers pass through unchecked): on the GPU, of the expected element
    type, dense where the library assumes it, and at least ``min_bytes``
    long.  A mismatch raises ``ValueError`` instead of letting the kernels
    read or write outside the tensor."""
    if x is None or isinstance(x, int):
        return
    if (x.is_cuda and (dtype is None or x.dtype is dtype) and x.nbytes >= min_bytes
            and x.is_contiguous()):
        return  # the common case; what follows allows more, or names what is wrong
    if not x.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if dtype is not None and x.dtype not in (dtype if isinstance(dtype, tuple) else (dtype,)):
        raise ValueError(f"{name} must be {dtype}, got {x.dtype}")
    if contiguous and not x.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if _nbytes(x) < min_bytes:
        raise ValueError(f"{name} holds {_nbytes(x)} bytes, needs {min_bytes}")


_KV_DTYPES = (torch.bfloat16, torch.uint8, torch.float8_e4m3fn)


# Sizes by the values of (params, shape): a call asks the library for them once
# and not on every call (at most _SIZES_MOST entries are kept).
_SIZES = {}
_SIZES_MOST = 256


def _sizes(p, s):
    """(status, window logits bytes, plan bytes, state bytes or 0 where there is
    no state); all sizes 0 where the status is not OK."""
    key = bytes(p) + bytes(s)
    z = _SIZES.get(key)
    if z is None:
        L = StateLayout()
        st = lib().dsa_get_state_layout(C.byref(p), C.byref(s), C.byref(L))
        z = (st, window_logits_count(p, s) * 4, plan_bytes(p, s), L.bytes if L.cap else 0)
        if len(_SIZES) >= _SIZES_MOST:
            _SIZES.clear()
        _SIZES[key] = z
    return z


def _need_extents(layout, requests, heads, layers=1):
    """The layout's scales and row bases are those of all pairs that the call reads."""
    if layout.scales < layers * requests * heads:
        raise ValueError(f"the layout holds {layout.scales} scales, the call reads {layers} layers "
                         f"x {requests} requests x {heads} KV heads of them")
    if layout.bases < requests:
        raise ValueError(f"the layout holds {layout.bases} row bases of {requests} requests")


def _need_state(z, state):
    _check(z[0], "dsa_get_state_layout")
    _need(state, "state", None, z[3])


def _check_decode_args(p, s, q, k, v, layout, decode_pos, out, window_logits):
    """Returns the call's ``_sizes``."""
    z = _sizes(p, s)
    B_, Hq, Hkv, d = s.batch, s.num_q_heads, s.num_kv_heads, s.head_dim
    _need(q, "q", torch.bfloat16, B_ * Hq * d * 2)
    _need(out, "out", torch.float32, B_ * Hq * d * 4)
    _need(decode_pos, "decode_pos", torch.int32, B_ * 4)
    _need(window_logits, "window_logits", torch.float32, z[1])
    _need(k, "k", _KV_DTYPES, contiguous=False)
    _need(v, "v", _KV_DTYPES, contiguous=False)
    _need_extents(layout, B_, Hkv)
    if isinstance(k, torch.Tensor) and isinstance(v, torch.Tensor):
        shape = k.shape
        if k.dtype != v.dtype or shape != v.shape or k.stride() != v.stride():
            raise ValueError("k and v must share element type, shape and strides")
        if len(shape) == 4 and layout.d_row_base is None:
            rows_needed = p.prompt_len + (layout.ring_rows if layout.ring_rows else 1)
            nb, nh, rows, nd = shape
            if nb < B_ or nh < Hkv or nd != d or rows < rows_needed:
                raise ValueError(f"cache of shape {tuple(shape)} does not hold {B_} requests x "
                                 f"{Hkv} KV heads x {rows_needed}+ rows of {d} elements")
    return z


# ---- host-only helpers ------------------------------------------------------

def abi_version() -> int:
    return lib().dsa_abi_version()


def make_params(prompt_len, grid_h, grid_w, window, n_att, mode=MODE_DIAGONAL, sinks=0) -> Params:
    return Params(prompt_len, grid_h, grid_w, window, n_att, mode, sinks)


def params_from_sparsity(prompt_len, grid_h, grid_w, window, sparsity_permille,
                         mode=MODE_DIAGONAL, sinks=0) -> Params:
    p = Params()
    _check(lib().dsa_params_from_sparsity(prompt_len, grid_h, grid_w, window,
                                          sparsity_permille, mode, sinks, C.byref(p)),
           "dsa_params_from_sparsity")
    return p


def make_shape(batch, num_q_heads, num_kv_heads, head_dim) -> Shape:
    return Shape(batch, num_q_heads, num_kv_heads, head_dim)


def validate(p: Params, s: Shape) -> int:
    return lib().dsa_validate(C.byref(p), C.byref(s))


def state_layout(p: Params, s: Shape) -> StateLayout:
    out = StateLayout()
    _check(lib().dsa_get_state_layout(C.byref(p), C.byref(s), C.byref(out)), "dsa_get_state_layout")
    return out


def plan_layout(p: Params, s: Shape) -> PlanLayout:
    out = PlanLayout()
    _check(lib().dsa_get_plan_layout(C.byref(p), C.byref(s), C.byref(out)), "dsa_get_plan_layout")
    return out


def launch_info(p: Params, s: Shape) -> LaunchInfo:
    out = LaunchInfo()
    _check(lib().dsa_get_launch_info(C.byref(p), C.byref(s), C.byref(out)), "dsa_get_launch_info")
    return out


def state_bytes(p, s) -> int:
    return lib().dsa_state_bytes(C.byref(p), C.byref(s))


def plan_bytes(p, s) -> int:
    return lib().dsa_plan_bytes(C.byref(p), C.byref(s))


def workspace_bytes(p, s) -> int:
    return lib().dsa_workspace_bytes(C.byref(p), C.byref(s))


def window_logits_count(p, s) -> int:
    return lib().dsa_window_logits_count(C.byref(p), C.byref(s))


# ---- device calls -------------------------------------------------------------

def state_reset(p, s, state, req_mask=None, stream=None):
    _check(lib().dsa_state_reset(C.byref(p), C.byref(s), _ptr(state), _ptr(req_mask),
                                 _stream(stream)), "dsa_state_reset")


def plan(p, s, decode_pos, state, plan_buf, stream=None):
    _need(decode_pos, "decode_pos", torch.int32, s.batch * 4)
    _need_state(_sizes(p, s), state)
    _check(lib().dsa_plan(C.byref(p), C.byref(s), _ptr(decode_pos), _ptr(state), _ptr(plan_buf),
                          _nbytes(plan_buf), _stream(stream)), "dsa_plan")


def kv_layout(k: torch.Tensor, row_base: Optional[torch.Tensor] = None,
              ring_rows: int = 0, k_scale: Optional[torch.Tensor] = None,
              v_scale: Optional[torch.Tensor] = None) -> KVLayout:
    """Layout of a ``[B, Hkv, rows, d]`` cache (any strides with unit stride
    along d); ``row_base`` optionally gives per-request base offsets;
    ``ring_rows = R > 0`` stores decode position ``j`` at row ``L_p + j``
    for the ``S`` sinks and at ``L_p + S + (j - S) % (R - S)`` after them.
    A bf16 cache is ``torch.bfloat16``; an fp8 (OCP E4M3) cache is
    ``torch.float8_e4m3fn`` or its bytes as ``torch.uint8``, with optional
    fp32 ``k_scale``/``v_scale`` of ``B * Hkv`` values; a layout for
    ``kv_append`` of several layers takes those of all of them, ``[layers,
    B * Hkv]``, and each layer's attention a layout with its own.  The layout
    keeps the tensors it points to."""
    sb, sh, sr, sd = k.stride()
    if sd != 1:
        raise ValueError("head_dim must be contiguous")
    _need(row_base, "row_base", torch.int64)
    _need(k_scale, "k_scale", torch.float32)
    _need(v_scale, "v_scale", torch.float32)
    if k.dtype == torch.bfloat16:
        dtype = KV_BF16
    elif k.dtype in (torch.uint8, torch.float8_e4m3fn):
        dtype = KV_FP8_E4M3
    else:
        raise ValueError(f"unsupported KV dtype {k.dtype}")
    out = KVLayout(_ptr(row_base), sb, sh, sr, int(ring_rows), _ptr(k_scale), _ptr(v_scale),
                   dtype)
    out._held = (row_base, k_scale, v_scale)
    held = [x.numel() for x in (k_scale, v_scale) if isinstance(x, torch.Tensor)]
    if held:
        out.scales = min(held)
    if isinstance(row_base, torch.Tensor):
        out.bases = row_base.numel()
    return out


def decode_attention(p, s, q, k, v, layout: KVLayout, decode_pos, plan_buf, sm_scale, out,
                     window_logits=None, workspace=None, stream=None, events=None):
    """``events``: optional (start, stop) pair from ``timing_events()``; they
    then receive the start of the split-K kernel and the end of the call's
    last kernel."""
    z = _check_decode_args(p, s, q, k, v, layout, decode_pos, out, window_logits)
    if p.mode != MODE_DENSE:
        _need(plan_buf, "plan", None, z[2])
    ws_bytes = 0 if workspace is None else _nbytes(workspace)
    args = (C.byref(p), C.byref(s), _ptr(q), _ptr(k), _ptr(v), C.byref(layout), _ptr(decode_pos),
            _ptr(plan_buf), float(sm_scale), _ptr(out), _ptr(window_logits), _ptr(workspace),
            ws_bytes)
    if events is None:
        _check(lib().dsa_decode_attention(*args, _stream(stream)), "dsa_decode_attention")
    else:
        _check(lib().dsa_decode_attention_timed(*args, events[0].cuda_event, events[1].cuda_event,
                                                _stream(stream)), "dsa_decode_attention_timed")


def decode_step(p, s, q, k, v, layout: KVLayout, decode_pos, state, plan_buf, sm_scale, out,
                window_logits, workspace=None, stream=None, events=None):
    """One fused decode step: plan + attention + selection in one pass."""
    _need_state(_check_decode_args(p, s, q, k, v, layout, decode_pos, out, window_logits), state)
    ws_bytes = 0 if workspace is None else _nbytes(workspace)
    pb = 0 if plan_buf is None else _nbytes(plan_buf)
    args = (C.byref(p), C.byref(s), _ptr(q), _ptr(k), _ptr(v), C.byref(layout), _ptr(decode_pos),
            _ptr(state), _ptr(plan_buf), pb, float(sm_scale), _ptr(out), _ptr(window_logits),
            _ptr(workspace), ws_bytes)
    if events is None:
        _check(lib().dsa_decode_step(*args, _stream(stream)), "dsa_decode_step")
    else:
        _check(lib().dsa_decode_step_timed(*args, events[0].cuda_event, events[1].cuda_event,
                                           _stream(stream)), "dsa_decode_step_timed")


def decode_step_noalloc(p, s, q, k, v, layout: KVLayout, decode_pos, state, plan_buf, sm_scale,
                        out, window_logits, stream=None):
    """``decode_step`` without a workspace: the split partials live in the
    library's own per-GPU buffer (for callers that cannot allocate)."""
    _need_state(_check_decode_args(p, s, q, k, v, layout, decode_pos, out, window_logits), state)
    pb = 0 if plan_buf is None else _nbytes(plan_buf)
    _check(lib().dsa_decode_step_noalloc(C.byref(p), C.byref(s), _ptr(q), _ptr(k), _ptr(v),
                                         C.byref(layout), _ptr(decode_pos), _ptr(state),
                                         _ptr(plan_buf), pb, float(sm_scale), _ptr(out),
                                         _ptr(window_logits), _stream(stream)),
           "dsa_decode_step_noalloc")


def timing_events():
    """A (start, stop) pair of timing events that exist on the device (torch
    creates its events lazily, at the first record)."""
    pair = (torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True))
    for e in pair:
        e.record()
    return pair


def select(p, s, decode_pos, plan_buf, window_logits, state, stream=None):
    z = _sizes(p, s)
    _check(z[0], "dsa_get_state_layout")
    if z[3]:
        _need(decode_pos, "decode_pos", torch.int32, s.batch * 4)
        _need(plan_buf, "plan", None, z[2])
        _need(window_logits, "window_logits", torch.float32, z[1])
        _need(state, "state", None, z[3])
    _check(lib().dsa_select(C.byref(p), C.byref(s), _ptr(decode_pos), _ptr(plan_buf),
                            _ptr(window_logits), _ptr(state), _stream(stream)), "dsa_select")


# ---- several tokens of a request at once ----------------------------------------

_OUT_TYPES = {torch.float32: 0, torch.bfloat16: 1}  # DSA_OUT_FP32, DSA_OUT_BF16


class Tree:
    """New tokens of every request (``dsa_tree``): ``nodes`` per request at
    most, ``base`` the decode position of each request's first (int32 [B]),
    ``count`` how many of them each has (int32 [B]; all; 0 for an unused slot,
    which ``tree_verify`` knows by nothing else), ``plan`` a buffer filled by
    ``tree_plan`` (a chain).  Keeps the tensors it points to; they
    can be written, not exchanged."""

    def __init__(self, nodes, base=None, count=None, plan=None):
        _need(base, "base", torch.int32)
        _need(count, "count", torch.int32)
        _need(plan, "plan")
        if plan is not None and nodes > MAX_TREE_NODES:
            raise ValueError(f"a tree has at most {MAX_TREE_NODES} nodes, got {nodes}")
        self._held = (int(nodes), base, count, plan)
        self.c = TreeRequest(int(nodes), _ptr(base), _ptr(count), _ptr(plan))
        self.ref = C.byref(self.c)
        self._seen = None  # the batch and device these tensors were last checked for

    nodes = property(lambda self: self._held[0])
    base = property(lambda self: self._held[1])
    count = property(lambda self: self._held[2])
    plan = property(lambda self: self._held[3])

    def check(self, batch, device, where, base=True):
        if base and self.base is None:
            raise ValueError(f"{where} needs the tree's base positions")
        if (batch, device) != self._seen:
            _need(self.base, "base", torch.int32, batch * 4)
            _need(self.count, "count", torch.int32, batch * 4)
            if self.plan is not None:
                _need(self.plan, "plan", None, tree_plan_bytes(batch, self.nodes))
            for x in (self.base, self.count, self.plan):
                if isinstance(x, torch.Tensor) and x.get_device() != device:
                    raise _elsewhere(x, "the tree", device)
            self._seen = (batch, device)


def make_tree(nodes, base=None, count=None, plan=None) -> Tree:
    return Tree(nodes, base, count, plan)


def tree_plan_layout(batch: int, nodes: int) -> TreePlanLayout:
    out = TreePlanLayout()
    _check(lib().dsa_get_tree_plan_layout(batch, nodes, C.byref(out)), "dsa_get_tree_plan_layout")
    return out


def tree_plan_bytes(batch: int, nodes: int) -> int:
    return lib().dsa_tree_plan_bytes(batch, nodes)


def tree_launch_info(p: Params, s: Shape, nodes: int) -> TreeLaunchInfo:
    out = TreeLaunchInfo()
    _check(lib().dsa_get_tree_launch_info(C.byref(p), C.byref(s), nodes, C.byref(out)),
           "dsa_get_tree_launch_info")
    return out


def tree_workspace_bytes(p: Params, s: Shape, nodes: int) -> int:
    return lib().dsa_tree_workspace_bytes(C.byref(p), C.byref(s), nodes)


# The checks below follow one pattern: a few comparisons that a right call
# passes, and the words for what is wrong only after one of them failed.

def _elsewhere(x, name, device):
    return ValueError(f"{name} is on {x.device}, the current device is cuda:{device}")


def _need_dense(x, name, dtype, shape, device):
    """A dense tensor on the current device, whose stream the call takes."""
    if (x.dtype is dtype and x.shape == shape and x.get_device() == device
            and x.is_contiguous()):
        return
    _need(x, name, dtype)
    if x.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(x.shape)}")
    raise _elsewhere(x, name, device)


def _need_bytes(x, name, device):
    if x is None or (x.get_device() == device and x.is_contiguous()):
        return
    _need(x, name)
    raise _elsewhere(x, name, device)


def _node_rows(x, name, shape, device):
    """Strides of a bf16 tensor of rows ``[(layers,) B, nodes, heads, d]``, the
    rows themselves dense."""
    st = x.stride()
    if not (x.dtype is torch.bfloat16 and x.shape == shape and x.get_device() == device
            and st[-1] == 1):
        _need(x, name, torch.bfloat16, contiguous=False)
        if x.shape != shape:
            raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(x.shape)}")
        if x.get_device() != device:
            raise _elsewhere(x, name, device)
        raise ValueError(f"{name}: head_dim must be contiguous")
    return st


def _new_rows(k_new, v_new, shape, device):
    st = _node_rows(k_new, "k_new", shape, device)
    if _node_rows(v_new, "v_new", shape, device) != st:
        raise ValueError("k_new and v_new must share strides")
    return NodeRows(st[-4], st[-3], st[-2], st[0] if len(st) == 5 else 0)


def _check_caches(p, s, k, v, layout, rows_needed, layers, device):
    _need(k, "k", _KV_DTYPES, contiguous=False)
    _need(v, "v", _KV_DTYPES, contiguous=False)
    shape, st = k.shape, k.stride()
    if k.dtype is not v.dtype or shape != v.shape or st != v.stride():
        raise ValueError("k and v must share element type, shape and strides")
    for x, name in ((k, "k"), (v, "v")):
        if x.get_device() != device:
            raise _elsewhere(x, name, device)
    if (layout.dtype == KV_BF16) != (k.dtype is torch.bfloat16):
        raise ValueError(f"the layout is not of a {k.dtype} cache")
    if layers is not None and (len(shape) != 5 or shape[0] != layers):
        raise ValueError(f"the caches must be of {layers} layers, got shape {tuple(shape)}")
    _need_extents(layout, s.batch, s.num_kv_heads, layers or 1)
    if len(shape) >= 4 and layout.d_row_base is None:
        nb, nh, rows, nd = shape[-4:]
        if (nb < s.batch or nh < s.num_kv_heads or nd != s.head_dim or rows < rows_needed
                or layout.stride_batch != st[-4] or layout.stride_head != st[-3]
                or layout.stride_row != st[-2]):
            raise ValueError(f"cache of shape {tuple(shape)} does not hold {s.batch} requests x "
                             f"{s.num_kv_heads} KV heads x {rows_needed}+ rows of {s.head_dim} "
                             "elements as the layout says")


def tree_plan(parent, count, plan_buf, stream=None):
    """Depths and ancestors of trees: ``parent`` int32 [B, nodes], -1 for none."""
    device = torch.cuda.current_device() if parent.is_cuda else None
    shape = parent.shape
    if len(shape) != 2:
        raise ValueError(f"parent must be [B, nodes], got {tuple(shape)}")
    if plan_buf is None:
        raise ValueError("tree_plan needs a buffer for the plan")
    _need_dense(parent, "parent", torch.int32, shape, device)
    if count is not None:
        _need_dense(count, "count", torch.int32, shape[:1], device)
    _need_bytes(plan_buf, "plan", device)
    _check(lib().dsa_tree_plan(shape[0], shape[1], parent.data_ptr(), _ptr(count),
                               plan_buf.data_ptr(), plan_buf.nbytes, _stream(stream)),
           "dsa_tree_plan")


def tree_attention(p, s, tree: Tree, q, k_new, v_new, k, v, layout: KVLayout, sm_scale, out,
                   workspace=None, stream=None):
    """Attention of every node over the caches and its ancestors.  ``q``
    bf16 [B, nodes, Hq, d], ``k_new`` and ``v_new`` bf16 [B, nodes, Hkv, d]
    (any strides with dense rows, as slices of a fused projection), ``out``
    [B, nodes, Hq, d] in fp32 or bf16."""
    device = torch.cuda.current_device() if q.is_cuda else None
    B_, Hq, Hkv, d, n = s.batch, s.num_q_heads, s.num_kv_heads, s.head_dim, tree.nodes
    shape = (B_, n, Hq, d)
    st = _node_rows(q, "q", shape, device)
    tree.check(B_, device, "tree_attention")
    new_rows = _new_rows(k_new, v_new, (B_, n, Hkv, d), device)
    out_type = _OUT_TYPES.get(out.dtype)
    if out_type is None:
        raise ValueError(f"out must be fp32 or bf16, got {out.dtype}")
    _need_dense(out, "out", out.dtype, shape, device)
    _check_caches(p, s, k, v, layout, p.prompt_len + layout.ring_rows, None, device)
    _need_bytes(workspace, "workspace", device)
    _check(lib().dsa_tree_attention(
        C.byref(p), C.byref(s), tree.ref, q.data_ptr(), C.byref(NodeRows(st[0], st[1], st[2], 0)),
        k_new.data_ptr(), v_new.data_ptr(), C.byref(new_rows), k.data_ptr(), v.data_ptr(),
        C.byref(layout), sm_scale, out.data_ptr(), out_type, _ptr(workspace),
        0 if workspace is None else workspace.nbytes, _stream(stream)), "dsa_tree_attention")


def tree_verify(tree: Tree, tokens, target, draft, uniform, path, accepted, next_token,
                stream=None):
    """Which drafted tokens stand, and the token after them.  ``tokens`` int32
    [B, nodes], ``target`` fp32 [B, nodes, V], ``draft`` the same or None
    (certain drafts), ``uniform`` fp32 [B, nodes + 1]; out: ``path`` int32
    [B, nodes], ``accepted`` and ``next_token`` int32 [B]."""
    device = torch.cuda.current_device() if target.is_cuda else None
    shape = target.shape
    if len(shape) != 3:
        raise ValueError(f"target must be [B, nodes, V], got {tuple(shape)}")
    batch, n, vocab = shape
    if n != tree.nodes:
        raise ValueError(f"target has {n} nodes, the tree {tree.nodes}")
    _need_dense(target, "target", torch.float32, shape, device)
    tree.check(batch, device, "tree_verify", base=False)
    if draft is not None:
        _need_dense(draft, "draft", torch.float32, shape, device)
    _need_dense(tokens, "tokens", torch.int32, (batch, n), device)
    _need_dense(uniform, "uniform", torch.float32, (batch, n + 1), device)
    _need_dense(path, "path", torch.int32, (batch, n), device)
    _need_dense(accepted, "accepted", torch.int32, (batch,), device)
    _need_dense(next_token, "next_token", torch.int32, (batch,), device)
    _check(lib().dsa_tree_verify(batch, vocab, tree.ref, tokens.data_ptr(), target.data_ptr(),
                                 _ptr(draft), uniform.data_ptr(), path.data_ptr(),
                                 accepted.data_ptr(), next_token.data_ptr(), _stream(stream)),
           "dsa_tree_verify")


def kv_append(p, s, tree: Tree, k_new, v_new, k, v, layout: KVLayout, path=None, accepted=None,
              stream=None):
    """K/V rows of new tokens into the caches, from the tree's base positions on:
    ``accepted[b]`` rows (all), the e-th node ``path[b, e]`` (node e).  One
    layer (``k_new`` [B, nodes, Hkv, d], ``k`` [B, Hkv, rows, d]) or all of
    them (both with layers in front, ``layout`` of one layer's cache but with
    the scales of all, [layers, B * Hkv])."""
    device = torch.cuda.current_device() if k_new.is_cuda else None
    B_, Hkv, d, n = s.batch, s.num_kv_heads, s.head_dim, tree.nodes
    layers = k_new.shape[0] if k_new.dim() == 5 else None
    shape = (B_, n, Hkv, d) if layers is None else (layers, B_, n, Hkv, d)
    rows = _new_rows(k_new, v_new, shape, device)
    tree.check(B_, device, "kv_append")
    _check_caches(p, s, k, v, layout,
                  p.prompt_len + (layout.ring_rows or p.grid_h * p.grid_w), layers, device)
    if path is not None:
        _need_dense(path, "path", torch.int32, (B_, n), device)
    if accepted is not None:
        _need_dense(accepted, "accepted", torch.int32, (B_,), device)
    _check(lib().dsa_kv_append(
        C.byref(p), C.byref(s), tree.ref, k_new.data_ptr(), v_new.data_ptr(), C.byref(rows),
        _ptr(path), _ptr(accepted), layers or 1, k.data_ptr(), v.data_ptr(), C.byref(layout),
        k.stride(0) if layers else 0, _stream(stream)), "dsa_kv_append")


def tree_plan_views(batch: int, nodes: int, plan_buf: torch.Tensor):
    """(flags [B], max_depth [B], depth [B, nodes], parent [B, nodes], ancestors
    [B, nodes, words]) int32 views of a tree plan."""
    L = tree_plan_layout(batch, nodes)
    i32 = lambda off, n: plan_buf[off:off + 4 * n].view(torch.int32)
    bn = batch * nodes
    return (i32(L.flags_offset, batch), i32(L.max_depth_offset, batch),
            i32(L.depth_offset, bn).view(batch, nodes),
            i32(L.parent_offset, bn).view(batch, nodes),
            i32(L.ancestors_offset, bn * L.words).view(batch, nodes, L.words))


# ---- a KV cache in pages -----------------------------------------------------------

class Pages:
    """Page tables of all requests (``dsa_pages``): ``table`` int32 [B, M], the
    page of each ``page_rows`` rows or -1; ``refs`` int32 [num_pages], how many
    entries name each page, and ``cursor`` int32 [1], both for ``page_update``
    (``page_reorder`` needs ``refs``); ``prompt`` int32 [B], prompt rows of each
    request (all ``prompt_len``).  Keeps the tensors it points to; they can be
    written, not exchanged."""

    def __init__(self, page_rows, table, refs=None, cursor=None, prompt=None):
        for x, name in ((table, "table"), (refs, "refs"), (cursor, "cursor"), (prompt, "prompt")):
            _need(x, name, torch.int32)
        if table.dim() != 2:
            raise ValueError(f"table must be [B, pages], got {tuple(table.shape)}")
        if refs is not None and refs.dim() != 1:
            raise ValueError(f"refs must be [num_pages], got {tuple(refs.shape)}")
        _need(cursor, "cursor", torch.int32, 4)
        _need(prompt, "prompt", torch.int32, 4 * table.shape[0])
        for x, name in ((refs, "refs"), (cursor, "cursor"), (prompt, "prompt")):
            if x is not None and x.device != table.device:
                raise ValueError(f"{name} is on {x.device}, the table on {table.device}")
        self._held = (table, refs, cursor, prompt)
        self.c = PagesStruct(int(page_rows), table.shape[1], 0 if refs is None else refs.numel(),
                             _ptr(table), _ptr(refs), _ptr(cursor), _ptr(prompt))
        self.ref = C.byref(self.c)
        self.batch, self.device = table.shape[0], table.get_device()

    table = property(lambda self: self._held[0])
    refs = property(lambda self: self._held[1])
    cursor = property(lambda self: self._held[2])
    prompt = property(lambda self: self._held[3])
    page_rows = property(lambda self: self.c.page_rows)


def make_pages(page_rows, table, refs=None, cursor=None, prompt=None) -> Pages:
    return Pages(page_rows, table, refs, cursor, prompt)


def page_layout(k: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
                v_scale: Optional[torch.Tensor] = None) -> PageLayout:
    """Layout of a layer's cache ``[num_pages, Hkv, page_rows, d]`` (any strides
    with unit stride along d), in bf16 or fp8 (as for ``kv_layout``) with
    optional fp32 scales of its KV heads, ``[Hkv]``; for ``paged_append`` of
    several layers those of all of them, ``[layers, Hkv]``.  The layout keeps the
    tensors it points to."""
    if k.dim() != 4:
        raise ValueError(f"a cache is [num_pages, Hkv, page_rows, d], got {tuple(k.shape)}")
    sp, sh, sr, sd = k.stride()
    if sd != 1:
        raise ValueError("head_dim must be contiguous")
    _need(k_scale, "k_scale", torch.float32)
    _need(v_scale, "v_scale", torch.float32)
    if k.dtype not in _KV_DTYPES:
        raise ValueError(f"unsupported KV dtype {k.dtype}")
    out = PageLayout(k.shape[0], k.shape[2], sp, sh, sr, _ptr(k_scale), _ptr(v_scale),
                     KV_BF16 if k.dtype == torch.bfloat16 else KV_FP8_E4M3)
    out._held = (k_scale, v_scale)
    out.scales = min([x.numel() for x in out._held if x is not None], default=1 << 62)
    return out


def paged_launch_info(p: Params, s: Shape) -> PagedLaunchInfo:
    out = PagedLaunchInfo()
    _check(lib().dsa_get_paged_launch_info(C.byref(p), C.byref(s), C.byref(out)),
           "dsa_get_paged_launch_info")
    return out


def paged_workspace_bytes(p: Params, s: Shape) -> int:
    return lib().dsa_paged_workspace_bytes(C.byref(p), C.byref(s))


def _device_of(x):
    """The current device, where x is on a GPU (its context is there)."""
    return torch._C._cuda_getDevice() if x.is_cuda else None


def _stream_on(stream, device):
    return (torch._C._cuda_getCurrentRawStream(device) if stream is None
            else stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _need_pages(pages, device, batch, where, refs=False, cursor=False):
    if pages.device != device:
        raise _elsewhere(pages.table, "the table", device)
    if batch != pages.batch:
        raise ValueError(f"the table has {pages.batch} requests, the call {batch}")
    if refs and pages.refs is None or cursor and pages.cursor is None:
        raise ValueError(f"{where} needs the pages' refs" + " and cursor" * cursor)


def page_update(p, pages: Pages, length, new, slots, pos, copies, flags, stream=None):
    """Pages for a step's new rows: ``length`` int32 [B] (below 0: an unused slot),
    ``new`` int32 [B] or None (1 each); out: ``slots`` int32 [B, N], ``pos`` [B],
    ``copies`` [B, 3], ``flags`` [B], all int32."""
    device = _device_of(length)
    batch = length.shape[0]
    _need_dense(length, "length", torch.int32, (batch,), device)
    _need_pages(pages, device, batch, "page_update", refs=True, cursor=True)
    if new is not None:
        _need_dense(new, "new", torch.int32, (batch,), device)
    if slots.dim() != 2:
        raise ValueError(f"slots must be [B, N], got {tuple(slots.shape)}")
    _need_dense(slots, "slots", torch.int32, (batch, slots.shape[1]), device)
    _need_dense(pos, "pos", torch.int32, (batch,), device)
    _need_dense(copies, "copies", torch.int32, (batch, 3), device)
    _need_dense(flags, "flags", torch.int32, (batch,), device)
    _check(lib().dsa_page_update(
        C.byref(p), batch, pages.ref, length.data_ptr(), _ptr(new), slots.shape[1],
        slots.data_ptr(), pos.data_ptr(), copies.data_ptr(), flags.data_ptr(), _stream_on(stream, device)),
        "dsa_page_update")


def page_reorder(pages: Pages, parent, stream=None):
    """Every request goes on from the pages of request ``parent[b]`` (int32 [B])."""
    device = _device_of(parent)
    _need_dense(parent, "parent", torch.int32, (pages.batch,), device)
    _need_pages(pages, device, pages.batch, "page_reorder", refs=True)
    _check(lib().dsa_page_reorder(pages.batch, pages.ref, parent.data_ptr(), _stream_on(stream, device)),
           "dsa_page_reorder")


def _check_paged(s, k, v, layout, layers, device):
    """The caches against their layout, their scales and the shape."""
    shape, st, dtype = k.shape, k.stride(), k.dtype
    # layout._fits: the caches' values that were last let through
    if (dtype is v.dtype and shape == v.shape and st == v.stride() and k.get_device() == device
            and v.get_device() == device
            and layout._fits == (dtype, shape, st, layers, s.num_kv_heads, s.head_dim, device)):
        return  # what follows has been looked at for these values
    if dtype not in _KV_DTYPES or dtype is not v.dtype or shape != v.shape or st != v.stride():
        raise ValueError("k and v must share element type (bf16 or fp8), shape and strides")
    for x, name in ((k, "k"), (v, "v")):
        if x.get_device() != device:
            _need(x, name, contiguous=False)
            raise _elsewhere(x, name, device)
    if (layout.dtype == KV_BF16) != (dtype is torch.bfloat16):
        raise ValueError(f"the layout is not of a {dtype} cache")
    if len(shape) != (4 if layers is None else 5) or (layers is not None and shape[0] != layers):
        raise ValueError(f"caches of shape {tuple(shape)} are not of "
                         + ("one layer" if layers is None else f"{layers} layers"))
    n, heads, rows, d = shape[-4:]
    if (n < layout.num_pages or heads < s.num_kv_heads or rows != layout.page_rows
            or d != s.head_dim or st[-4:] != (layout.stride_page, layout.stride_head,
                                              layout.stride_row, 1)):
        raise ValueError(f"cache of shape {tuple(shape)} does not hold {layout.num_pages} pages of "
                         f"{layout.page_rows} rows x {s.num_kv_heads} KV heads of {s.head_dim} "
                         "elements as the layout says")
    if layout.scales < (layers or 1) * s.num_kv_heads:
        raise ValueError(f"the layout holds {layout.scales} scales, the call reads {layers or 1} "
                         f"layers x {s.num_kv_heads} KV heads of them")
    for x in layout._held:
        if x is not None and x.get_device() != device:
            raise _elsewhere(x, "a scale", device)
    layout._fits = (dtype, shape, st, layers, s.num_kv_heads, s.head_dim, device)


def paged_append(s, slots, k_new, v_new, k, v, layout: PageLayout, copies=None, stream=None):
    """K/V rows into their slots (int32 [B, N], -1: nowhere), after the rows of shared
    pages that ``copies`` (int32 [B, 3]) names.  One layer (``k_new`` [B, N, Hkv,
    d], ``k`` [num_pages, Hkv, page_rows, d]) or all of them (both with layers in
    front, ``layout`` of one layer's cache but with the scales of all)."""
    device = _device_of(k_new)
    B_, Hkv, d = s.batch, s.num_kv_heads, s.head_dim
    layers = k_new.shape[0] if k_new.dim() == 5 else None
    if slots.dim() != 2:
        raise ValueError(f"slots must be [B, N], got {tuple(slots.shape)}")
    n = slots.shape[1]
    _need_dense(slots, "slots", torch.int32, (B_, n), device)
    shape = (B_, n, Hkv, d) if layers is None else (layers, B_, n, Hkv, d)
    rows = _new_rows(k_new, v_new, shape, device)
    _check_paged(s, k, v, layout, layers, device)
    if copies is not None:
        _need_dense(copies, "copies", torch.int32, (B_, 3), device)
    _check(lib().dsa_paged_append(
        C.byref(s), n, slots.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), C.byref(rows),
        layers or 1, k.data_ptr(), v.data_ptr(), C.byref(layout), k.stride(0) if layers else 0,
        _ptr(copies), _stream_on(stream, device)), "dsa_paged_append")


def paged_attention(p, s, pages: Pages, q, k, v, layout: PageLayout, decode_pos, sm_scale, out,
                    plan_buf=None, window_logits=None, workspace=None, stream=None):
    """Attention of one token per request (``q`` bf16 [B, Hq, d]) over its pages;
    ``out`` [B, Hq, d] in fp32 or bf16.  Diagonal mode takes the step's plan, and
    the window logits fp32 [B, Hq, cap] where the selection is to read them."""
    device = _device_of(q)
    B_, shape = s.batch, (s.batch, s.num_q_heads, s.head_dim)
    _need_dense(q, "q", torch.bfloat16, shape, device)
    _need_pages(pages, device, B_, "paged_attention")
    out_type = _OUT_TYPES.get(out.dtype)
    if out_type is None:
        raise ValueError(f"out must be fp32 or bf16, got {out.dtype}")
    _need_dense(out, "out", out.dtype, shape, device)
    _need_dense(decode_pos, "decode_pos", torch.int32, (B_,), device)
    _check_paged(s, k, v, layout, None, device)
    if p.mode == MODE_DIAGONAL:
        z = _sizes(p, s)
        _need(plan_buf, "plan", None, z[2])
        _need_bytes(plan_buf, "plan", device)
        if window_logits is not None:
            _need(window_logits, "window_logits", torch.float32, z[1])
            _need_bytes(window_logits, "window_logits", device)
    _need_bytes(workspace, "workspace", device)
    _check(lib().dsa_paged_attention(
        C.byref(p), C.byref(s), pages.ref, q.data_ptr(), k.data_ptr(), v.data_ptr(),
        C.byref(layout), decode_pos.data_ptr(), _ptr(plan_buf), sm_scale, out.data_ptr(), out_type,
        _ptr(window_logits), _ptr(workspace), 0 if workspace is None else workspace.nbytes,
        _stream_on(stream, device)), "dsa_paged_attention")


def beam_workspace_bytes(batch: int, beams: int, vocab: int) -> int:
    return lib().dsa_beam_workspace_bytes(batch, beams, vocab)


def beam_select(logits, score, next_score, parent, token, workspace, stream=None):
    """The best ``beams`` candidates of every request: ``logits`` [B, beams, V] in
    fp32 or bf16 (rows dense and evenly apart), ``score`` fp32 [B, beams]; out:
    ``next_score`` fp32 (may be ``score``), ``parent`` and ``token`` int32, all
    [B, beams]; parents as ``page_reorder`` takes them, flattened."""
    device = _device_of(logits)
    if logits.dim() != 3:
        raise ValueError(f"logits must be [B, beams, V], got {tuple(logits.shape)}")
    batch, beams, vocab = logits.shape
    kind = _OUT_TYPES.get(logits.dtype)
    if kind is None:
        raise ValueError(f"logits must be fp32 or bf16, got {logits.dtype}")
    if logits.get_device() != device:
        _need(logits, "logits", contiguous=False)
        raise _elsewhere(logits, "logits", device)
    sb, sw, sv = logits.stride()
    row = sw if beams > 1 else sb if batch > 1 else vocab
    if (vocab > 1 and sv != 1) or (batch > 1 and sb != beams * row) or row < vocab:
        raise ValueError("logits must have dense rows, evenly apart")
    shape = (batch, beams)
    _need_dense(score, "score", torch.float32, shape, device)
    _need_dense(next_score, "next_score", torch.float32, shape, device)
    _need_dense(parent, "parent", torch.int32, shape, device)
    _need_dense(token, "token", torch.int32, shape, device)
    _need_bytes(workspace, "workspace", device)
    _check(lib().dsa_beam_select(
        batch, beams, vocab, logits.data_ptr(), row, kind, score.data_ptr(), next_score.data_ptr(),
        parent.data_ptr(), token.data_ptr(), _ptr(workspace),
        0 if workspace is None else workspace.nbytes, _stream_on(stream, device)), "dsa_beam_select")


# ---- buffers (torch allocations) and views --------------------------------------

@dataclass
class Buffers:
    """Device buffers of one layer: selection state, plan, window logits,
    split workspace and output."""
    state: torch.Tensor
    plan: torch.Tensor
    logits: torch.Tensor
    workspace: Optional[torch.Tensor]
    out: torch.Tensor


def alloc_buffers(p: Params, s: Shape, device="cuda") -> Buffers:
    nb = lambda n: torch.zeros(max(int(n), 1), dtype=torch.uint8, device=device)
    ws = workspace_bytes(p, s)
    return Buffers(
        state=nb(state_bytes(p, s)),
        plan=nb(plan_bytes(p, s)),
        logits=torch.zeros(max(window_logits_count(p, s), 1), dtype=torch.float32, device=device),
        workspace=nb(ws) if ws else None,
        out=torch.zeros((s.batch, s.num_q_heads, s.head_dim), dtype=torch.float32, device=device),
    )


def plan_views(p: Params, s: Shape, plan_buf: torch.Tensor):
    """(count [B*Hkv], flags [B*Hkv], indices [B*Hkv, cap]) int32 views."""
    L = plan_layout(p, s)
    pairs = s.batch * s.num_kv_heads
    i32 = lambda off, n: plan_buf[off:off + 4 * n].view(torch.int32)
    idx = i32(L.indices_offset, pairs * L.cap).view(pairs, L.cap)
    return i32(L.count_offset, pairs), i32(L.flags_offset, pairs), idx


def state_views(p: Params, s: Shape, state_buf: torch.Tensor):
    """(count [B*Hkv] int32, flags [B*Hkv] int32, offsets [B*Hkv, cap] as
    int16 bit patterns of the stored uint16 values)."""
    L = state_layout(p, s)
    pairs = s.batch * s.num_kv_heads
    cnt = state_buf[L.count_offset:L.count_offset + 4 * pairs].view(torch.int32)
    flg = state_buf[L.flags_offset:L.flags_offset + 4 * pairs].view(torch.int32)
    off = state_buf[L.offsets_offset:L.offsets_offset + 2 * pairs * L.cap].view(torch.int16)
    return cnt, flg, off.view(pairs, L.cap)


def kept_views(p: Params, s: Shape, state_buf: torch.Tensor):
    """(tags [B*Hkv, 2] int32: k + 1 for the list of slot s after k skip
    entries, 0 for none; lists [B*Hkv, 2, kept_stride] as int16 bit patterns
    of the stored uint16 kept offsets, largest first)."""
    L = state_layout(p, s)
    pairs = s.batch * s.num_kv_heads
    tags = state_buf[L.kept_count_offset:L.kept_count_offset + 8 * pairs].view(torch.int32)
    n = 2 * pairs * L.kept_stride
    lists = state_buf[L.kept_offset:L.kept_offset + 2 * n].view(torch.int16)
    return tags.view(pairs, 2), lists.view(pairs, 2, L.kept_stride)
