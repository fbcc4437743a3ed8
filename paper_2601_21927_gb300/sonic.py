"""Python binding of libsonic (include/sonic.h): argument marshalling only.

Every step of the path runs in the CUDA library; this module loads
``_lib/libsonic.so`` with ctypes, mirrors the argument structs, and offers the
entry points under their C names taking torch tensors on the GPU:

* :func:`sonic_compact_kv`   -- retention (Sec. 3.2 body removal, App. C),
* :func:`sonic_attn_prefill` -- attention under the Sec. 3.2 mask,
* :func:`sonic_attn_decode`  -- one GQA decode step over the retained cache,
* :func:`sonic_routed_linear` -- the role-routed projections,

and, for caches in four bits a value or kept within a budget of rows,

* :func:`sonic_kv4_compact`, :func:`sonic_kv4_store`, :func:`sonic_kv4_load` --
  rows packed (by the retention rule, or by index) and unpacked,
* :func:`sonic_attn_decode_kv4` -- one GQA decode step over a four-bit cache,
* :func:`sonic_key_mass` -- the attention weight each cached row received,
* :func:`sonic_evict_kv` -- the rows with the least of it dropped.

The wrappers only fill the C structs, allocate the caller-owned workspace as a
torch tensor, pass the current CUDA stream and raise :class:`SonicError` on a
non-OK status.  Those of the second group also refuse tensors of another shape,
type, memory order or device than the call takes.  Importing this module fails loudly if the library is missing;
there is no fallback path.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import Optional

import torch

from . import _build

ROLE_SYS, ROLE_BODY, ROLE_NEXUS, ROLE_CURR = 0, 1, 2, 3
NEXUS_FULL, NEXUS_CAUSAL_SEGMENTS = 0, 1
KEYS_AS_GIVEN, KEYS_RETAINED_FIRST = 0, 1

STATUS = {0: "SONIC_OK", 1: "SONIC_ERR_INVALID_ARGUMENT", 2: "SONIC_ERR_UNSUPPORTED",
          3: "SONIC_ERR_WORKSPACE", 4: "SONIC_ERR_CAPACITY", 5: "SONIC_ERR_DEVICE_TIMEOUT",
          6: "SONIC_ERR_CUDA", 7: "SONIC_ERR_LAYOUT"}

_P = ctypes.c_void_p
_i32, _i64, _f32, _sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t


class SonicError(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__(f"{where}: {STATUS.get(code, code)}")
        self.code = code


class sonic_compact_args(ctypes.Structure):
    _fields_ = [("batch", _i32), ("n_layers", _i32), ("k_start", _P), ("k_len", _P),
                ("reserve", _P), ("row_bytes", _i64), ("in_layer_bytes", _i64),
                ("out_layer_bytes", _i64), ("out_capacity_rows", _i32), ("ret_len", _P),
                ("src_idx", _P), ("out_role", _P), ("out_seg", _P), ("status", _P),
                ("workspace", _P), ("workspace_bytes", _sz), ("total_rows", _i32)]


class sonic_prefill_args(ctypes.Structure):
    _fields_ = [("batch", _i32), ("n_layers", _i32), ("n_heads_q", _i32), ("n_heads_kv", _i32),
                ("head_dim", _i32), ("k_start", _P), ("k_len", _P), ("q_start", _P),
                ("q_len", _P), ("max_q_len", _i32), ("max_k_len", _i32), ("total_q_rows", _i32),
                ("total_k_rows", _i32), ("q_layer_stride", _i64), ("kv_layer_stride", _i64),
                ("o_layer_stride", _i64), ("softmax_scale", _f32), ("nexus_vis", _i32),
                ("lse", _P), ("status", _P), ("workspace", _P), ("workspace_bytes", _sz),
                ("key_order", _i32), ("nexus_mass", _P)]


class sonic_decode_args(ctypes.Structure):
    _fields_ = [("batch", _i32), ("n_layers", _i32), ("n_heads_q", _i32), ("n_heads_kv", _i32),
                ("head_dim", _i32), ("kv_start", _P), ("max_len", _i32), ("total_kv_rows", _i32),
                ("q_layer_stride", _i64), ("kv_layer_stride", _i64), ("o_layer_stride", _i64),
                ("softmax_scale", _f32), ("chunk_len", _i32), ("lse", _P), ("status", _P),
                ("workspace", _P), ("workspace_bytes", _sz), ("role", _P), ("nexus_mass", _P)]


class sonic_out_part(ctypes.Structure):
    _fields_ = [("base", _P), ("row_stride", _i64), ("cols", _i32), ("scatter", _i32),
                ("rows", _i64)]


class sonic_routed_linear_args(ctypes.Structure):
    _fields_ = [("n_rows", _i32), ("d_in", _i32), ("d_out", _i32), ("x_row_stride", _i64),
                ("dst_row", _P), ("n_parts", _i32), ("parts", sonic_out_part * 4),
                ("status", _P), ("workspace", _P), ("workspace_bytes", _sz)]


class sonic_kv4_cache(ctypes.Structure):
    _fields_ = [("k_codes", _P), ("k_scales", _P), ("v_codes", _P), ("v_scales", _P), ("rows", _i32),
                ("codes_layer_bytes", _i64), ("scales_layer_bytes", _i64)]


class sonic_kv4_rows_args(ctypes.Structure):
    _fields_ = [("n_layers", _i32), ("n_heads_kv", _i32), ("head_dim", _i32), ("n_rows", _i32),
                ("src_row", _P), ("dst_row", _P), ("live", _P), ("total_rows", _i32), ("kv_layer_stride", _i64),
                ("status", _P)]


class sonic_kv4_compact_args(ctypes.Structure):
    _fields_ = [("batch", _i32), ("n_layers", _i32), ("n_heads_kv", _i32), ("head_dim", _i32),
                ("k_start", _P), ("k_len", _P), ("reserve", _P), ("total_rows", _i32),
                ("kv_layer_stride", _i64), ("ret_len", _P), ("src_idx", _P), ("out_role", _P),
                ("out_seg", _P), ("status", _P), ("workspace", _P), ("workspace_bytes", _sz)]


class sonic_decode_kv4_args(ctypes.Structure):
    _fields_ = [("batch", _i32), ("n_layers", _i32), ("n_heads_q", _i32), ("n_heads_kv", _i32),
                ("head_dim", _i32), ("kv_start", _P), ("max_len", _i32), ("q_layer_stride", _i64),
                ("o_layer_stride", _i64), ("softmax_scale", _f32), ("lse", _P), ("status", _P),
                ("workspace", _P), ("workspace_bytes", _sz)]


class sonic_key_mass_args(ctypes.Structure):
    _fields_ = [("batch", _i32), ("n_layers", _i32), ("n_heads_q", _i32), ("n_heads_kv", _i32),
                ("head_dim", _i32), ("kv_start", _P), ("max_len", _i32), ("total_kv_rows", _i32),
                ("kv_layer_stride", _i64), ("q_start", _P), ("q_len", _P), ("max_q_len", _i32),
                ("total_q_rows", _i32), ("q_layer_stride", _i64), ("softmax_scale", _f32),
                ("mass_layers", _i32), ("mass_heads", _i32), ("prev", _P), ("keep", _f32),
                ("status", _P)]


class sonic_evict_part(ctypes.Structure):
    _fields_ = [("src", _P), ("dst", _P), ("bytes", _i32), ("src_layer", _i64), ("src_head", _i64),
                ("src_row", _i64), ("dst_layer", _i64), ("dst_head", _i64), ("dst_row", _i64)]


class sonic_evict_args(ctypes.Structure):
    _fields_ = [("batch", _i32), ("n_layers", _i32), ("n_heads_kv", _i32), ("mass_layers", _i32),
                ("mass_heads", _i32), ("kv_start", _P), ("max_len", _i32), ("total_kv_rows", _i32),
                ("budget", _P), ("reserve", _P), ("role", _P), ("keep_roles", ctypes.c_uint32),
                ("recent", _i32), ("out_rows", _i32), ("out_len", _P), ("src_idx", _P),
                ("out_mass", _P), ("out_role", _P), ("n_parts", _i32),
                ("parts", sonic_evict_part * 4), ("status", _P), ("workspace", _P),
                ("workspace_bytes", _sz)]


# Exported C symbols, with their ctypes signatures.
SIGNATURES = {
    "sonic_compact_kv": (_i32, [_P, _P, _P, _P, _P, _P, _P,
                                ctypes.POINTER(sonic_compact_args), _P]),
    "sonic_compact_workspace_size": (_sz, [ctypes.POINTER(sonic_compact_args)]),
    "sonic_attn_prefill": (_i32, [_P, _P, _P, _P, _P, _P,
                                  ctypes.POINTER(sonic_prefill_args), _P]),
    "sonic_prefill_workspace_size": (_sz, [ctypes.POINTER(sonic_prefill_args)]),
    "sonic_attn_prefill_static": (_i32, [_P, _P, _P, _P, _P, _P,
                                         ctypes.POINTER(sonic_prefill_args), _P]),
    "sonic_attn_decode": (_i32, [_P, _P, _P, _P, _P,
                                 ctypes.POINTER(sonic_decode_args), _P]),
    "sonic_decode_workspace_size": (_sz, [ctypes.POINTER(sonic_decode_args)]),
    "sonic_kv4_store": (_i32, [_P, _P, ctypes.POINTER(sonic_kv4_cache),
                               ctypes.POINTER(sonic_kv4_rows_args), _P]),
    "sonic_kv4_load": (_i32, [ctypes.POINTER(sonic_kv4_cache), _P, _P,
                              ctypes.POINTER(sonic_kv4_rows_args), _P]),
    "sonic_kv4_compact": (_i32, [_P, _P, _P, _P, ctypes.POINTER(sonic_kv4_cache), _P,
                                 ctypes.POINTER(sonic_kv4_compact_args), _P]),
    "sonic_kv4_compact_workspace_size": (_sz, [ctypes.POINTER(sonic_kv4_cache),
                                               ctypes.POINTER(sonic_kv4_compact_args)]),
    "sonic_attn_decode_kv4": (_i32, [_P, ctypes.POINTER(sonic_kv4_cache), _P, _P,
                                     ctypes.POINTER(sonic_decode_kv4_args), _P]),
    "sonic_decode_kv4_workspace_size": (_sz, [ctypes.POINTER(sonic_decode_kv4_args)]),
    "sonic_key_mass": (_i32, [_P, _P, ctypes.POINTER(sonic_kv4_cache), _P, _P, _P,
                              ctypes.POINTER(sonic_key_mass_args), _P]),
    "sonic_evict_kv": (_i32, [_P, _P, _P, ctypes.POINTER(sonic_evict_args), _P]),
    "sonic_evict_workspace_size": (_sz, [ctypes.POINTER(sonic_evict_args)]),
    "sonic_routed_linear": (_i32, [_P, _P, _P, _P, ctypes.POINTER(sonic_routed_linear_args),
                                   _P]),
    "sonic_routed_linear_workspace_size": (_sz, [ctypes.POINTER(sonic_routed_linear_args)]),
    "sonic_read_status": (_i32, [_P, _P]),
    "sonic_status_string": (ctypes.c_char_p, [_i32]),
    "sonic_abi_version": (_i32, []),
}

_lib = None


def library_path() -> str:
    return _build.LIB


def load(build_if_missing: bool = True) -> ctypes.CDLL:
    """Load libsonic.so (building it first if asked and it is missing)."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.LIB
    if not os.path.exists(path):
        if not build_if_missing:
            raise ImportError(f"libsonic.so not built ({path}); run __graft_entry__.build()")
        _build.build()
    _lib = open_library(path)
    return _lib


def open_library(path: str) -> ctypes.CDLL:
    """A libsonic build at `path` with the C signatures applied (entry points
    the build lacks are skipped)."""
    lib = ctypes.CDLL(path)
    for name, (res, args) in SIGNATURES.items():
        if not hasattr(lib, name):
            continue
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    return t.data_ptr()


# The current stream's handle: the raw lookup builds no Stream object (1.3 us less a call).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream=None):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def _check(code: int, where: str):
    if code != 0:
        raise SonicError(code, where)


def _workspace(nbytes: int, device, ws: Optional[torch.Tensor]):
    if nbytes == 0:
        return None
    if ws is not None and ws.numel() * ws.element_size() >= nbytes:
        return ws
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def read_status(status: torch.Tensor, stream=None) -> int:
    return int(load().sonic_read_status(_ptr(status), _stream(stream)))


# ---------------------------------------------------------------------------
# Entry points
# ---------------------------------------------------------------------------

def sonic_compact_kv(K: torch.Tensor, V: torch.Tensor, seg_id: Optional[torch.Tensor],
                     role: torch.Tensor, out_K: torch.Tensor, out_V: torch.Tensor,
                     offsets: torch.Tensor, *, k_start: torch.Tensor, k_len: torch.Tensor,
                     reserve: Optional[torch.Tensor] = None, ret_len=None, src_idx=None,
                     out_role=None, out_seg=None, status=None, workspace=None, stream=None):
    """Retention rule over all layers.  K, V: [n_layers, T, ...] (any dtype, rows
    of row_bytes contiguous); out_K, out_V: [n_layers, capacity, ...]."""
    lib = load()
    nl, T = K.shape[:2]
    es = K.element_size()
    row_bytes = math.prod(K.shape[2:]) * es if T > 0 else K.numel() // max(nl, 1) * es
    total_rows = min(T, role.numel())
    if seg_id is not None:
        total_rows = min(total_rows, seg_id.numel())
    # the fields in the struct's order, in one call (setting them one by one took 2 us longer)
    a = sonic_compact_args(
        k_start.numel(), nl, _ptr(k_start), _ptr(k_len), _ptr(reserve), row_bytes,
        K.stride(0) * es, out_K.stride(0) * out_K.element_size(), out_K.shape[1], _ptr(ret_len),
        _ptr(src_idx), _ptr(out_role), _ptr(out_seg), _ptr(status), None, 0, total_rows)
    need = lib.sonic_compact_workspace_size(ctypes.byref(a))
    ws = _workspace(need, K.device, workspace)
    a.workspace, a.workspace_bytes = _ptr(ws), need
    _check(lib.sonic_compact_kv(_ptr(K), _ptr(V), _ptr(seg_id), _ptr(role), _ptr(out_K),
                                _ptr(out_V), _ptr(offsets), ctypes.byref(a), _stream(stream)),
           "sonic_compact_kv")
    return ws


def sonic_attn_prefill(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, seg_id: torch.Tensor,
                       role: torch.Tensor, O: torch.Tensor, *, k_start, k_len, q_start, q_len,
                       max_q_len: int, max_k_len: int, softmax_scale: float = 0.0,
                       nexus_vis: int = NEXUS_FULL, lse=None, status=None, workspace=None,
                       key_order: int = KEYS_AS_GIVEN, nexus_mass=None, stream=None):
    """Masked prefill.  Q, O: [n_layers, Tq, Hq, D] bf16; K, V: [n_layers, Tk, Hkv, D] bf16;
    lse, nexus_mass: [n_layers, Tq, Hq] float32 or None."""
    lib = load()
    nl, tq, hq, d = Q.shape
    _, tk, hkv, _ = K.shape
    a = sonic_prefill_args(
        k_start.numel(), nl, hq, hkv, d, _ptr(k_start), _ptr(k_len), _ptr(q_start), _ptr(q_len),
        max_q_len, max_k_len, tq, tk, Q.stride(0), K.stride(0), O.stride(0), softmax_scale,
        nexus_vis, _ptr(lse), _ptr(status), None, 0, key_order, _ptr(nexus_mass))
    need = lib.sonic_prefill_workspace_size(ctypes.byref(a))
    ws = _workspace(need, Q.device, workspace)
    a.workspace, a.workspace_bytes = _ptr(ws), need
    _check(lib.sonic_attn_prefill(_ptr(Q), _ptr(K), _ptr(V), _ptr(seg_id), _ptr(role), _ptr(O),
                                  ctypes.byref(a), _stream(stream)), "sonic_attn_prefill")
    return ws


def sonic_attn_decode(q: torch.Tensor, K_ret: torch.Tensor, V_ret: torch.Tensor,
                      lens: torch.Tensor, O: torch.Tensor, *, kv_start, max_len: int,
                      softmax_scale: float = 0.0, chunk_len: int = 0, lse=None, status=None,
                      workspace=None, role=None, nexus_mass=None, stream=None):
    """One decode step.  q, O: [n_layers, B, Hq, D]; K_ret, V_ret: [n_layers, T, Hkv, D];
    lse, nexus_mass: [n_layers, B, Hq] float32 or None; role: [T] uint8 (with nexus_mass)."""
    lib = load()
    nl, B, hq, d = q.shape
    _, T, hkv, _ = K_ret.shape
    a = sonic_decode_args(
        B, nl, hq, hkv, d, _ptr(kv_start), max_len, T, q.stride(0), K_ret.stride(0), O.stride(0),
        softmax_scale, chunk_len, _ptr(lse), _ptr(status), None, 0, _ptr(role), _ptr(nexus_mass))
    need = lib.sonic_decode_workspace_size(ctypes.byref(a))
    ws = _workspace(need, q.device, workspace)
    a.workspace, a.workspace_bytes = _ptr(ws), need
    _check(lib.sonic_attn_decode(_ptr(q), _ptr(K_ret), _ptr(V_ret), _ptr(lens), _ptr(O),
                                 ctypes.byref(a), _stream(stream)), "sonic_attn_decode")
    return ws


def sonic_routed_linear(X: torch.Tensor, W: torch.Tensor, W_nexus: torch.Tensor,
                        role: torch.Tensor, parts, *, dst_row=None, status=None, workspace=None,
                        stream=None):
    """Role-routed linear map.  X: [T, >= d_in] bf16 (row-contiguous); W, W_nexus:
    [d_out, d_in] bf16; role: [T] uint8.  parts: list of (out, scatter) with out a
    2-D bf16 tensor whose columns (out.shape[1]) take the next columns of Y and
    whose rows are indexed by t (scatter False) or dst_row[t] (scatter True)."""
    lib = load()
    T = X.shape[0]
    d_out, d_in = W.shape
    a = sonic_routed_linear_args(T, d_in, d_out, X.stride(0) if T > 0 else d_in, _ptr(dst_row),
                                 len(parts))
    for k, (out, scatter) in enumerate(parts):
        shape = out.shape
        a.parts[k] = sonic_out_part(_ptr(out), out.stride(0), shape[1], 1 if scatter else 0,
                                    shape[0])
    a.status = _ptr(status)
    need = lib.sonic_routed_linear_workspace_size(ctypes.byref(a))
    ws = _workspace(need, X.device, workspace)
    a.workspace, a.workspace_bytes = _ptr(ws), need
    _check(lib.sonic_routed_linear(_ptr(X), _ptr(W), _ptr(W_nexus), _ptr(role), ctypes.byref(a),
                                   _stream(stream)), "sonic_routed_linear")
    return ws


def sonic_attn_prefill_static(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor,
                              seg_id: torch.Tensor, role: torch.Tensor, O: torch.Tensor, *,
                              k_start, k_len, q_start, q_len, max_q_len: int, max_k_len: int,
                              softmax_scale: float = 0.0, nexus_vis: int = NEXUS_FULL, lse=None,
                              status=None, nexus_mass=None, stream=None):
    """sonic_attn_prefill for callers that cannot allocate device memory: the
    library keeps the tile summaries and masks in a fixed ~9 MiB device array, so
    no workspace is passed (and this wrapper allocates nothing either).
    Calls overlapping on the GPU share that array and must be serialised."""
    lib = load()
    nl, tq, hq, d = Q.shape
    _, tk, hkv, _ = K.shape
    a = sonic_prefill_args(
        k_start.numel(), nl, hq, hkv, d, _ptr(k_start), _ptr(k_len), _ptr(q_start), _ptr(q_len),
        max_q_len, max_k_len, tq, tk, Q.stride(0), K.stride(0), O.stride(0), softmax_scale,
        nexus_vis, _ptr(lse), _ptr(status), None, 0, KEYS_AS_GIVEN, _ptr(nexus_mass))
    _check(lib.sonic_attn_prefill_static(_ptr(Q), _ptr(K), _ptr(V), _ptr(seg_id), _ptr(role),
                                         _ptr(O), ctypes.byref(a), _stream(stream)),
           "sonic_attn_prefill_static")


# ---------------------------------------------------------------------------
# Four-bit caches, attention weight and eviction
# ---------------------------------------------------------------------------

_U8, _I32, _F32, _BF16 = torch.uint8, torch.int32, torch.float32, torch.bfloat16


# The current device's number (torch.cuda.current_device less its lazy initialisation: a
# call's tensors have seen to that).
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _refuse(where: str, what: str):
    raise SonicError(1, f"{where} ({what})")


def _want(where: str, name: str, t, dtype, shape, dev: int, layered: bool = False):
    """Refuses a tensor that is not on device `dev`, of `dtype` and of `shape`, or not contiguous
    (`layered`: within each entry of its first dimension).  None passes."""
    if t is None or (t.dtype is dtype and t.shape == shape and t.get_device() == dev and t.is_contiguous()):
        return
    if t.dtype is not dtype or t.get_device() != dev:
        _refuse(where, f"{name}: {dtype} on the current device")
    if t.shape != shape:
        _refuse(where, f"{name}: shape {tuple(t.shape)}, not {tuple(shape)}")
    if not t.is_contiguous() and not (layered and t.shape[0] > 0 and t[0].is_contiguous()):
        _refuse(where, f"{name}: memory order")


def _dims(where: str, name: str, t, n: int):
    """The extents of a tensor that has to have n of them."""
    s = t.shape
    if len(s) != n:
        _refuse(where, f"{name}: {n} dimensions")
    return s


def _status_word(where: str, status, dev: int):
    if status is not None and (status.dtype is not _I32 or status.get_device() != dev
                               or status.numel() < 1):
        _refuse(where, "status")


def _cache(where: str, K4, V4, dev: int):
    """(C struct, layers, heads, rows, head_dim) of four-bit rows: K4 = (codes [layers, heads, rows,
    D / 2], scales [layers, heads, rows, D / 16]), both uint8; V4 the same or None."""
    codes, scales = K4
    shape = _dims(where, "codes", codes, 4)
    nl, hkv, rows, half = shape
    small = (nl, hkv, rows, half // 8)
    _want(where, "K4 codes", codes, _U8, shape, dev, True)
    _want(where, "K4 scales", scales, _U8, small, dev, True)
    # (a single layer has no stride)
    ls, lss = (codes.stride(0), scales.stride(0)) if nl > 1 else (0, 0)
    if V4 is None:
        return (sonic_kv4_cache(codes.data_ptr(), scales.data_ptr(), None, None, rows, ls, lss), nl, hkv,
                rows, 2 * half)
    vc, vs = V4
    _want(where, "V4 codes", vc, _U8, shape, dev, True)
    _want(where, "V4 scales", vs, _U8, small, dev, True)
    if nl > 1 and (vc.stride(0) != ls or vs.stride(0) != lss):
        _refuse(where, "K4 and V4: one layer stride")
    return (sonic_kv4_cache(codes.data_ptr(), scales.data_ptr(), vc.data_ptr(), vs.data_ptr(), rows, ls, lss),
            nl, hkv, rows, 2 * half)


def _kv_rows(where: str, K, V, nl: int, hkv: int, d: int, dev: int):
    shape = (nl, _dims(where, "K", K, 4)[1], hkv, d)
    _want(where, "K", K, _BF16, shape, dev, True)
    _want(where, "V", V, _BF16, shape, dev, True)
    if nl > 1 and K.stride(0) != V.stride(0):
        _refuse(where, "K and V: one layer stride")


def _call(where: str, a, call, size, dev: int, ws, stream):
    """call() with the caller's workspace in the struct `a`, or with a new one of size() bytes where there
    is none or it is too small.  Returns the workspace."""
    code = 3
    if ws is not None:
        if ws.get_device() != dev or not ws.is_contiguous():
            _refuse(where, "workspace: contiguous, on the current device")
        a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel() * ws.element_size()
        code = call()
    if code == 3:  # SONIC_ERR_WORKSPACE
        need = size()
        if stream is None:
            ws = _workspace(need, dev, None)
        else:
            with torch.cuda.stream(stream):  # it belongs to the stream that uses it
                ws = _workspace(need, dev, None)
        a.workspace, a.workspace_bytes = _ptr(ws), need
        code = call()
    _check(code, where)
    return ws


def _rows_args(where, K, V, K4, V4, src_row, dst_row, live, n_rows, status, dev):
    c, nl, hkv, rows, d = _cache(where, K4, V4, dev)
    _kv_rows(where, K, V, nl, hkv, d, dev)
    most = None  # the shorter list
    for t in (src_row, dst_row, live):
        if t is not None:
            n = _dims(where, "row list", t, 1)
            _want(where, "row list", t, _I32, n, dev)
            most = n[0] if most is None else min(most, n[0])
    if n_rows is None:
        n_rows = most if most is not None else min(rows, K.shape[1])
    elif most is not None and n_rows > most:
        _refuse(where, "n_rows: longer than the row list")
    _status_word(where, status, dev)
    return c, sonic_kv4_rows_args(nl, hkv, d, n_rows, _ptr(src_row), _ptr(dst_row), _ptr(live), K.shape[1],
                                  K.stride(0) if nl > 1 else 0, _ptr(status))


def sonic_kv4_store(K: torch.Tensor, V: torch.Tensor, K4, V4, *, src_row=None, dst_row=None, live=None,
                    n_rows: Optional[int] = None, status=None, stream=None):
    """Packs rows src_row[j] of K, V ([n_layers, T, Hkv, D] bf16) into rows dst_row[j] of a four-bit
    cache.  K4, V4: (codes [n_layers, Hkv, rows, D / 2], scales [n_layers, Hkv, rows, D / 16]) uint8.
    A list left out counts 0, 1, ..; entries j with live[j] < 0 are skipped; n_rows defaults to the
    shortest list, or the smaller side."""
    where, dev = "sonic_kv4_store", _device()
    c, a = _rows_args(where, K, V, K4, V4, src_row, dst_row, live, n_rows, status, dev)
    _check(load().sonic_kv4_store(_ptr(K), _ptr(V), ctypes.byref(c), ctypes.byref(a), _stream(stream)),
           where)


def sonic_kv4_load(K4, V4, K: torch.Tensor, V: torch.Tensor, *, src_row=None, dst_row=None, live=None,
                   n_rows: Optional[int] = None, status=None, stream=None):
    """The way back: rows src_row[j] of the cache as bf16 rows dst_row[j] of K, V (exact).  With the
    src_idx of sonic_kv4_compact or sonic_evict_kv (one choice) as `live`, a whole cache is read
    without its free rows."""
    where, dev = "sonic_kv4_load", _device()
    c, a = _rows_args(where, K, V, K4, V4, src_row, dst_row, live, n_rows, status, dev)
    _check(load().sonic_kv4_load(ctypes.byref(c), _ptr(K), _ptr(V), ctypes.byref(a), _stream(stream)),
           where)


def sonic_kv4_compact(K: torch.Tensor, V: torch.Tensor, seg_id: Optional[torch.Tensor],
                      role: torch.Tensor, K4, V4, offsets: torch.Tensor, *, k_start: torch.Tensor,
                      k_len: torch.Tensor, reserve=None, ret_len=None, src_idx=None, out_role=None,
                      out_seg=None, status=None, workspace=None, stream=None):
    """sonic_compact_kv into a four-bit cache.  K, V: [n_layers, T, Hkv, D] bf16; K4, V4 as in
    sonic_kv4_store.  No output may lie over an input (ret_len is not k_len).  Returns the workspace."""
    where, dev = "sonic_kv4_compact", _device()
    lib = load()
    c, nl, hkv, rows, d = _cache(where, K4, V4, dev)
    _kv_rows(where, K, V, nl, hkv, d, dev)
    one = _dims(where, "k_start", k_start, 1)
    B, total = one[0], K.shape[1]
    for name, t, dtype in (("role", role, _U8), ("seg_id", seg_id, _I32)):
        if t is not None:
            _want(where, name, t, dtype, _dims(where, name, t, 1), dev)
            total = min(total, t.shape[0])
    for name, t in (("k_start", k_start), ("k_len", k_len), ("reserve", reserve), ("ret_len", ret_len)):
        _want(where, name, t, _I32, one, dev)
    for name, t, dtype in (("src_idx", src_idx, _I32), ("out_seg", out_seg, _I32), ("out_role", out_role, _U8)):
        _want(where, name, t, dtype, (rows,), dev)
    _want(where, "offsets", offsets, _I32, (B + 1,), dev)
    _status_word(where, status, dev)
    a = sonic_kv4_compact_args(B, nl, hkv, d, _ptr(k_start), _ptr(k_len), _ptr(reserve), total,
                               K.stride(0) if nl > 1 else 0, _ptr(ret_len), _ptr(src_idx), _ptr(out_role),
                               _ptr(out_seg), _ptr(status))
    rc, ra = ctypes.byref(c), ctypes.byref(a)
    return _call(where, a, lambda: lib.sonic_kv4_compact(_ptr(K), _ptr(V), _ptr(seg_id), _ptr(role), rc,
                                                         _ptr(offsets), ra, _stream(stream)),
                 lambda: lib.sonic_kv4_compact_workspace_size(rc, ra), dev, workspace, stream)


def sonic_attn_decode_kv4(q: torch.Tensor, K4, V4, lens: torch.Tensor, O: torch.Tensor, *, kv_start,
                          max_len: int, softmax_scale: float = 0.0, lse=None, status=None,
                          workspace=None, stream=None):
    """One decode step over a four-bit cache.  q, O: [n_layers, B, Hq, D] bf16; lse: [n_layers, B,
    Hq] float32 or None.  Returns the workspace."""
    where, dev = "sonic_attn_decode_kv4", _device()
    lib = load()
    c, nl, hkv, rows, d = _cache(where, K4, V4, dev)
    _, B, hq, _ = _dims(where, "q", q, 4)
    shape, one = (nl, B, hq, d), (B,)
    _want(where, "q", q, _BF16, shape, dev, True)
    _want(where, "O", O, _BF16, shape, dev, True)
    _want(where, "lens", lens, _I32, one, dev)
    _want(where, "kv_start", kv_start, _I32, one, dev)
    _want(where, "lse", lse, _F32, shape[:3], dev)
    _status_word(where, status, dev)
    a = sonic_decode_kv4_args(B, nl, hq, hkv, d, _ptr(kv_start), max_len, q.stride(0) if nl > 1 else 0,
                              O.stride(0) if nl > 1 else 0, softmax_scale, _ptr(lse), _ptr(status))
    rc, ra = ctypes.byref(c), ctypes.byref(a)
    return _call(where, a, lambda: lib.sonic_attn_decode_kv4(_ptr(q), rc, _ptr(lens), _ptr(O), ra,
                                                             _stream(stream)),
                 lambda: lib.sonic_decode_kv4_workspace_size(ra), dev, workspace, stream)


def sonic_key_mass(q: torch.Tensor, K, lse: torch.Tensor, lens: torch.Tensor, mass: torch.Tensor, *,
                   kv_start, max_len: int, q_start=None, q_len=None, max_q_len: int = 1, prev=None,
                   keep: float = 1.0, softmax_scale: float = 0.0, status=None, stream=None):
    """mass = keep * prev + the attention weight each cached row received.  q: [n_layers, Tq, Hq, D]
    bf16 and lse: [n_layers, Tq, Hq] float32 of the queries (one per sequence, or q_len[b] from
    q_start[b] on); K: [n_layers, T, Hkv, D] bf16, or a four-bit cache's (codes, scales); mass, prev:
    [n_layers or 1, Hkv or 1, T] float32 (an extent of 1 adds up the layers or heads)."""
    where, dev = "sonic_key_mass", _device()
    four = not isinstance(K, torch.Tensor)
    if four:
        c, nl, hkv, rows, d = _cache(where, K, None, dev)
    else:
        nl, rows, hkv, d = _dims(where, "K", K, 4)
        _want(where, "K", K, _BF16, K.shape, dev, True)
    _, tq, hq, _ = _dims(where, "q", q, 4)
    _want(where, "q", q, _BF16, (nl, tq, hq, d), dev, True)
    _want(where, "lse", lse, _F32, (nl, tq, hq), dev)
    ml, mh, _ = _dims(where, "mass", mass, 3)
    _want(where, "mass", mass, _F32, (ml, mh, rows), dev)
    _want(where, "prev", prev, _F32, (ml, mh, rows), dev)
    one = _dims(where, "lens", lens, 1)
    B = one[0]
    _want(where, "lens", lens, _I32, one, dev)
    _want(where, "kv_start", kv_start, _I32, one, dev)
    _want(where, "q_start", q_start, _I32, one, dev)
    _want(where, "q_len", q_len, _I32, one, dev)
    _status_word(where, status, dev)
    a = sonic_key_mass_args(B, nl, hq, hkv, d, _ptr(kv_start), max_len, rows,
                            0 if four else K.stride(0), _ptr(q_start), _ptr(q_len), max_q_len, tq,
                            q.stride(0) if nl > 1 else 0, softmax_scale, ml, mh, _ptr(prev), keep,
                            _ptr(status))
    _check(load().sonic_key_mass(_ptr(q), None if four else _ptr(K), ctypes.byref(c) if four else None,
                                 _ptr(lse), _ptr(lens), _ptr(mass), ctypes.byref(a), _stream(stream)),
           where)


def sonic_evict_kv(mass: torch.Tensor, parts, lens: torch.Tensor, offsets: torch.Tensor, *, kv_start,
                   max_len: int, budget: torch.Tensor, reserve=None, role=None, keep_roles: int = 0,
                   recent: int = 0, out_len=None, src_idx=None, out_mass=None, out_role=None,
                   status=None, workspace=None, stream=None):
    """Keeps the rows of each sequence with the largest mass ([n_layers or 1, Hkv or 1, T] float32:
    an extent of 1 makes one choice for all layers or heads) within budget[b].  parts: up to four
    (src, dst) pairs of cache arrays, bf16 [n_layers, rows, Hkv, D] or four-bit codes or scales
    (uint8, [n_layers, Hkv, rows, ..]).  src_idx, out_mass, out_role: [.., .., out rows] like mass.
    No output may lie over an input (out_len is not lens).  Returns the workspace."""
    where, dev = "sonic_evict_kv", _device()
    lib = load()
    ml, mh, rows = _dims(where, "mass", mass, 3)
    _want(where, "mass", mass, _F32, mass.shape, dev)
    one = _dims(where, "lens", lens, 1)
    B = one[0]
    if len(parts) > 4:
        _refuse(where, "at most four parts")
    table, seen = [], None  # the parts' C structs; their (layers, heads, output rows)
    for src, dst in parts:
        shape, to = _dims(where, "part", src, 4), _dims(where, "part", dst, 4)
        # in four bits a head's rows lie one after another, in bf16 a row's heads
        if src.dtype is _U8:
            nl, hkv, t, n = shape
            out_rows, dtype, es = to[2], _U8, 1
            want = (nl, hkv, out_rows, n)
            row, head, dhead = n, n * t, n * out_rows
        else:
            nl, t, hkv, n = shape
            out_rows, dtype, es = to[1], _BF16, 2
            want = (nl, out_rows, hkv, n)
            n *= 2
            row, head, dhead = n * hkv, n, n
        _want(where, "part", src, dtype, shape, dev, True)
        _want(where, "part", dst, dtype, want, dev, True)
        if t != rows or (seen is not None and seen != (nl, hkv, out_rows)):
            _refuse(where, "parts: layers, heads or rows differ")
        seen = (nl, hkv, out_rows)
        table.append((src.data_ptr(), dst.data_ptr(), n, src.stride(0) * es, head, row, dst.stride(0) * es,
                      dhead, row))
    if seen is None:
        first = next((t for t in (src_idx, out_mass, out_role) if t is not None), None)
        if first is None:
            _refuse(where, "nothing to write")
        seen = (ml, mh, _dims(where, "output", first, 3)[2])
    nl, hkv, out_rows = seen
    outs = (ml, mh, out_rows)
    _want(where, "src_idx", src_idx, _I32, outs, dev)
    _want(where, "out_mass", out_mass, _F32, outs, dev)
    _want(where, "out_role", out_role, _U8, outs, dev)
    _want(where, "role", role, _U8, (rows,), dev)
    for name, t in (("lens", lens), ("kv_start", kv_start), ("budget", budget), ("reserve", reserve),
                    ("out_len", out_len)):
        _want(where, name, t, _I32, one, dev)
    _want(where, "offsets", offsets, _I32, (B + 1,), dev)
    _status_word(where, status, dev)
    a = sonic_evict_args(B, nl, hkv, ml, mh, _ptr(kv_start), max_len, rows, _ptr(budget), _ptr(reserve),
                         _ptr(role), keep_roles, recent, out_rows, _ptr(out_len), _ptr(src_idx),
                         _ptr(out_mass), _ptr(out_role), len(table), tuple(table), _ptr(status))
    ra = ctypes.byref(a)
    return _call(where, a, lambda: lib.sonic_evict_kv(_ptr(mass), _ptr(lens), _ptr(offsets), ra, _stream(stream)),
                 lambda: lib.sonic_evict_workspace_size(ra), dev, workspace, stream)
