"""Binding over libcoreinfer.so -- argument marshalling only: ctypes, and for the per-token call csrc/binding.c where it is built.

Function names mirror the C ABI (include/coreinfer.h).  Tensors are torch
tensors on the GPU; torch supplies device memory and the current stream,
every step of the path runs in the library's own HIP kernels.  There is no
fallback: if the library is missing, importing this module raises.
"""

from __future__ import annotations

import ctypes
import itertools
import math
import os
from typing import Optional

import torch  # imported first so that the HIP runtime torch ships is the one the library binds to

from .build import BINDING_PATH, LIB_PATH

CI_OK = 0
CI_ERR_INVALID_ARG = -1
CI_ERR_BAD_DTYPE = -2
CI_ERR_BAD_LAYOUT = -3
CI_ERR_WORKSPACE = -4
CI_ERR_HIP = -5
CI_ERR_UNSUPPORTED = -6

CI_F32, CI_F16, CI_BF16 = 0, 1, 2
CI_ACT_RELU, CI_ACT_SWIGLU = 0, 1
CI_ACT_NONE = 2  # w4_matvec only
CI_DOWN_OUT_MAJOR, CI_DOWN_NEURON_MAJOR = 0, 1

DTYPE_CODE = {torch.float32: CI_F32, torch.float16: CI_F16, torch.bfloat16: CI_BF16}
ACT_CODE = {"relu": CI_ACT_RELU, "swiglu": CI_ACT_SWIGLU}
LAYOUT_CODE = {"out_major": CI_DOWN_OUT_MAJOR, "neuron_major": CI_DOWN_NEURON_MAJOR}

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is not built; run `python -m paper_2410_18311_amd.build` "
        "(there is no CPU or PyTorch fallback for the CoreInfer kernels)")

_lib = ctypes.CDLL(LIB_PATH)

_vp, _i64, _int, _dbl, _sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_double, ctypes.c_size_t


class ci_ffn_weights(ctypes.Structure):
    _fields_ = [("w_up", _vp), ("w_gate", _vp), ("b_up", _vp), ("w_down", _vp), ("b_down", _vp),
                ("core_idx", _vp), ("K", _i64), ("d", _i64), ("N", _i64), ("ld_down", _i64),
                ("down_layout", ctypes.c_int32)]


class ci_kv4(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp), ("weight", _vp), ("pos", _vp),
                ("B", _i64), ("H", _i64), ("cap", _i64), ("D", ctypes.c_int32), ("group", ctypes.c_int32)]


class ci_rope(ctypes.Structure):
    _fields_ = [("turns", _vp), ("scale", ctypes.c_float), ("rot", ctypes.c_int32), ("style", ctypes.c_int32)]


class ci_kvp(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("table", _vp), ("pages", _i64), ("most", _i64), ("B", _i64), ("H", ctypes.c_int32),
                ("page", ctypes.c_int32), ("D", ctypes.c_int32), ("dtype", ctypes.c_int32)]


_SIGNATURES = {
    "coreinfer_strerror": (ctypes.c_char_p, [_int]),
    "coreinfer_version": (_int, []),
    "coreinfer_keep_count": (_int, [_dbl, _i64, ctypes.POINTER(_i64)]),
    "coreinfer_select_workspace_size": (_int, [_i64, _i64, ctypes.POINTER(_sz)]),
    "coreinfer_select": (_int, [_vp, _i64, _i64, _i64, _dbl, _dbl, _vp, _vp, _vp, _sz, _vp]),
    "coreinfer_select_batch_workspace_size": (_int, [_i64, _i64, _i64, ctypes.POINTER(_sz)]),
    "coreinfer_select_batch": (_int, [_vp, _i64, _i64, _i64, _i64, _dbl, _dbl, _vp, _vp, _vp, _sz, _vp]),
    "coreinfer_select_hidden": (_int, [_vp, _int, _int, _i64, _i64, _i64, _dbl, _dbl, _vp, _vp, _vp, _sz, _vp]),
    "coreinfer_count_tokens": (_int, [_vp, _i64, _i64, _i64, _dbl, _vp, _int, _vp, _sz, _vp]),
    "coreinfer_count_select": (_int, [_vp, _i64, _i64, _dbl, _vp, _vp, _sz, _vp]),
    "coreinfer_group_select": (_int, [_vp, _i64, _i64, _i64, _dbl, _vp, _vp, _vp, _sz, _vp]),
    "coreinfer_core_similarity": (_int, [_vp, _i64, _vp, _i64, _vp, _vp]),
    "coreinfer_assign_group": (_int, [_vp, _i64, _vp, _i64, _i64, _vp, _vp, _vp]),
    "coreinfer_assign_centroid_workspace_size": (_int, [_i64, ctypes.POINTER(_sz)]),
    "coreinfer_assign_centroid": (_int, [_vp, _i64, _i64, _i64, _vp, _i64, _vp, _vp, _vp, _sz, _vp]),
    "coreinfer_compact_down_ld": (_int, [_i64, _int, ctypes.POINTER(_i64)]),
    "coreinfer_compact_preferred_layout": (_int, [_i64, _i64, _int, _int, ctypes.POINTER(_int)]),
    "coreinfer_compact": (_int, [_vp, _vp, _vp, _vp, _int, _int, _int, _i64, _i64, _vp, _i64,
                                 _vp, _vp, _vp, _vp, _int, _vp, _vp]),
    "coreinfer_compact_update_workspace_size": (_int, [_i64, _i64, ctypes.POINTER(_sz)]),
    "coreinfer_compact_update": (_int, [_vp, _vp, _vp, _vp, _int, _int, _int, _i64, _i64, _vp, _i64, _vp,
                                        _vp, _vp, _vp, _vp, _int, _vp, _vp, _sz, _vp]),
    "coreinfer_ffn_decode_workspace_size": (_int, [_i64, _i64, _i64, ctypes.POINTER(_sz)]),
    "coreinfer_ffn_decode": (_int, [_vp, _i64, ctypes.POINTER(ci_ffn_weights), _int, _int, _vp,
                                    _vp, _sz, _vp]),
    "coreinfer_ffn_decode_status": (_int, [_vp, _vp, _vp]),
    "coreinfer_ffn_decode_static": (_int, [_vp, _i64, ctypes.POINTER(ci_ffn_weights), _int, _int, _vp, _vp, _vp]),
    "coreinfer_union_workspace_size": (_int, [_i64, ctypes.POINTER(_sz)]),
    "coreinfer_union_build": (_int, [_vp, _i64, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _sz, _vp]),
    "coreinfer_ffn_decode_union_workspace_size": (_int, [_i64, _i64, _i64, _int, _int, ctypes.POINTER(_sz)]),
    "coreinfer_ffn_decode_union": (_int, [_vp, _i64, ctypes.POINTER(ci_ffn_weights), _vp, _vp, _vp, _i64,
                                          _int, _int, _vp, _vp, _sz, _vp]),
    "coreinfer_ffn_dense_hidden_workspace_size": (_int, [_i64, _i64, _i64, _int, ctypes.POINTER(_sz)]),
    "coreinfer_ffn_dense_hidden": (_int, [_vp, _i64, _vp, _vp, _vp, _vp, _vp, _int, _int, _int, _i64, _i64, _vp, _vp,
                                          _vp, _sz, _vp]),
    "coreinfer_ffn_dense_workspace_size": (_int, [_i64, _i64, _i64, _int, ctypes.POINTER(_sz)]),
    "coreinfer_ffn_dense": (_int, [_vp, _i64, _vp, _vp, _vp, _vp, _vp, _int, _int, _int, _i64, _i64,
                                   _vp, _vp, _vp, _sz, _vp]),
    "coreinfer_w4_size": (_int, [_i64, _i64, _int, ctypes.POINTER(_sz)]),
    "coreinfer_w4_quantize": (_int, [_vp, _i64, _i64, _i64, _int, _int, _vp, _vp]),
    "coreinfer_w4_read": (_int, [_vp, _i64, _i64, _int, _vp, _i64, _int, _vp]),
    "coreinfer_w4_matvec_workspace_size": (_int, [_i64, _i64, _int, ctypes.POINTER(_sz)]),
    "coreinfer_w4_matvec": (_int, [_vp, _i64, _i64, _int, _vp, _vp, _vp, _int, _int, _i64, _i64, _int, _vp, _i64, _int, _vp,
                                   _sz, _vp]),
    "coreinfer_kv4_sizes": (_int, [_i64, _i64, _i64, _int, _int, ctypes.POINTER(_sz), ctypes.POINTER(_sz)]),
    "coreinfer_kv4_append": (_int, [ctypes.POINTER(ci_kv4), _vp, _vp, _i64, ctypes.POINTER(_i64), _int, _vp, _vp, _vp, _vp]),
    "coreinfer_kv4_read": (_int, [ctypes.POINTER(ci_kv4), _vp, _i64, _i64, _vp, _vp, _int, _vp]),
    "coreinfer_kv4_attend_workspace_size": (_int, [_i64, _i64, _int, _i64, _i64, _i64, _int, ctypes.POINTER(_sz)]),
    "coreinfer_kv4_attend": (_int, [ctypes.POINTER(ci_kv4), _vp, _i64, _i64, ctypes.POINTER(_i64), _int, ctypes.c_float, _vp, _i64,
                                    _vp, _vp, _vp, _vp, _sz, _vp]),
    "coreinfer_kv4_evict_workspace_size": (_int, [_i64, _i64, _i64, _i64, ctypes.POINTER(_sz)]),
    "coreinfer_kv4_evict": (_int, [ctypes.POINTER(ci_kv4), _vp, _vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _sz, _vp]),
    "coreinfer_rope_turns": (_int, [_i64, _dbl, _int, _dbl, _dbl, _dbl, _dbl, _vp]),
    "coreinfer_rope": (_int, [_vp, ctypes.POINTER(_i64), _i64, _i64, _i64, _int, _vp, ctypes.c_float, ctypes.POINTER(ci_rope), _vp, _int,
                              _vp, ctypes.POINTER(_i64), _vp]),
    "coreinfer_kvp_append": (_int, [ctypes.POINTER(ci_kvp), _vp, _vp, ctypes.POINTER(_i64), _i64, _vp, _vp, _vp,
                                    ctypes.POINTER(ci_rope), _vp, ctypes.c_float, _vp, _i64, ctypes.POINTER(_i64), _vp, _vp, _vp]),
    "coreinfer_kvp_attend_workspace_size": (_int, [ctypes.POINTER(ci_kvp), _i64, _i64, _i64, _i64, _i64, _i64, ctypes.POINTER(_sz)]),
    "coreinfer_kvp_attend": (_int, [ctypes.POINTER(ci_kvp), _vp, _i64, ctypes.POINTER(_i64), _i64, _vp, _vp, _i64, _i64, _i64, _i64,
                                    ctypes.c_float, _vp, _vp, _vp, _sz, _vp]),
}
for _name, (_res, _args) in _SIGNATURES.items():
    _f = getattr(_lib, _name)
    _f.restype, _f.argtypes = _res, _args

EXPORTS = tuple(_SIGNATURES)

# the per-token calls, with addresses as integers: the C module if it was built for this interpreter, or the same through ctypes
if os.path.exists(BINDING_PATH):
    from . import _binding  # linked against the library that is now loaded
    _decode_call = _binding.ffn_decode
    _w4_matvec_call, _kv4_append_call, _kv4_read_call = _binding.w4_matvec, _binding.kv4_append, _binding.kv4_read
    _kv4_attend_call, _kv4_evict_call = _binding.kv4_attend, _binding.kv4_evict
    _rope_call, _kvp_append_call, _kvp_attend_call = _binding.rope, _binding.kvp_append, _binding.kvp_attend
else:
    _binding = None
    _prototype = lambda name, *args: ctypes.CFUNCTYPE(_int, *args)((name, _lib))  # noqa: E731
    _w4_matvec_call = _prototype("coreinfer_w4_matvec", *_SIGNATURES["coreinfer_w4_matvec"][1])
    _kv4_read_call = _prototype("coreinfer_kv4_read", _vp, *_SIGNATURES["coreinfer_kv4_read"][1][1:])
    _kv4_evict_call = _prototype("coreinfer_kv4_evict", _vp, *_SIGNATURES["coreinfer_kv4_evict"][1][1:])
    _kv4_append_c = _prototype("coreinfer_kv4_append", _vp, *_SIGNATURES["coreinfer_kv4_append"][1][1:])
    _kv4_attend_c = _prototype("coreinfer_kv4_attend", _vp, *_SIGNATURES["coreinfer_kv4_attend"][1][1:])

    def _kv4_append_call(cache, k, v, S, s0, s1, s2, *rest):
        return _kv4_append_c(cache, k, v, S, (_i64 * 3)(s0, s1, s2), *rest)

    def _kv4_attend_call(cache, q, S, Hq, s0, s1, s2, *rest):
        return _kv4_attend_c(cache, q, S, Hq, (_i64 * 3)(s0, s1, s2), *rest)

    _rope_c, _kvp_append_c, _kvp_attend_c = (
        _prototype(name, *(_vp if issubclass(t, ctypes._Pointer) and t is not ctypes.POINTER(_i64) else t for t in _SIGNATURES[name][1]))
        for name in ("coreinfer_rope", "coreinfer_kvp_append", "coreinfer_kvp_attend"))

    def _rope_call(x, s0, s1, T, H, D, dtype, norm, eps, angles, pos, backward, y, y0, y1, stream):
        return _rope_c(x, (_i64 * 2)(s0, s1), T, H, D, dtype, norm, eps, angles, pos, backward, y, (_i64 * 2)(y0, y1), stream)

    def _kvp_append_call(cache, k, v, s0, s1, T, first, lens, pos, angles, k_norm, eps, q, Hq, q0, q1, *rest):
        return _kvp_append_c(cache, k, v, (_i64 * 2)(s0, s1), T, first, lens, pos, angles, k_norm, eps, q, Hq, (_i64 * 2)(q0, q1), *rest)

    def _kvp_attend_call(cache, q, Hq, s0, s1, *rest):
        return _kvp_attend_c(cache, q, Hq, (_i64 * 2)(s0, s1), *rest)
    _decode_call = ctypes.CFUNCTYPE(_int, _vp, _i64, _vp, _int, _int, _vp, _vp, _sz, _vp)(("coreinfer_ffn_decode", _lib))

raw = _lib  # the bare C entry points, for tests of the error paths

# development hook (csrc/coreinfer_dev.h): launch-shape parameters for sweeps, not part of the interface
_lib.coreinfer_dev_set_param.restype = _int
_lib.coreinfer_dev_set_param.argtypes = [ctypes.c_char_p, _int]
_lib.coreinfer_dev_get_param.restype = _int
_lib.coreinfer_dev_get_param.argtypes = [ctypes.c_char_p, ctypes.POINTER(_int)]
_lib.coreinfer_dev_param_name.restype = ctypes.c_char_p
_lib.coreinfer_dev_param_name.argtypes = [_int]
_lib.coreinfer_dev_fused_plan.restype = _int
_lib.coreinfer_dev_fused_plan.argtypes = [_i64, _i64, _int, _int, ctypes.POINTER(_int)]
_lib.coreinfer_dev_decode_slices.restype = _int
_lib.coreinfer_dev_decode_slices.argtypes = [_i64, _i64, _i64, _int, _int, ctypes.POINTER(_int)]
_lib.coreinfer_dev_decode_small.restype = _int
_lib.coreinfer_dev_decode_small.argtypes = [_i64, _i64, _i64, _int, _int, _vp, ctypes.POINTER(_int)]
_lib.coreinfer_dev_decode_small_gave_up.restype = _int
_lib.coreinfer_dev_decode_small_gave_up.argtypes = [ctypes.POINTER(ctypes.c_uint32)]
_lib.coreinfer_dev_dense_plan.restype = _int
_lib.coreinfer_dev_dense_plan.argtypes = [_i64, _i64, _i64, _int, _int, _int, _i64, ctypes.POINTER(_i64)]
_lib.coreinfer_dev_select_layout.restype = _int
_lib.coreinfer_dev_select_layout.argtypes = [_i64, _i64, _i64, ctypes.POINTER(_i64)]
_lib.coreinfer_dev_stream_probe.restype = _int
_lib.coreinfer_dev_stream_probe.argtypes = [_vp, _i64, _i64, _int, _int, _int, _int, _int, _vp, _vp]
_lib.coreinfer_dev_tile_probe.restype = _int
_lib.coreinfer_dev_tile_probe.argtypes = [_vp, _i64, _i64, _int, _int, _int, _int, _int, _vp, _vp]


class CoreInferError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {strerror(status)} ({status})")


def _check(status: int, where: str):
    if status != CI_OK:
        raise CoreInferError(status, where)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


# the current stream's handle without the Stream object that torch.cuda.current_stream builds around it: 0.15
# instead of 3.4 us of a call, which for small layers is a fifth of what a decode call costs the host
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda device: torch.cuda.current_stream(device).cuda_stream)


def _stream(t: torch.Tensor):
    device = t.get_device()     # -1: host memory
    return _raw_stream(device) if device >= 0 else None


def _workspace(nbytes: int, like: torch.Tensor) -> torch.Tensor:
    return torch.empty(nbytes, dtype=torch.uint8, device=like.device)


def strerror(status: int) -> str:
    return _lib.coreinfer_strerror(status).decode()


def version() -> int:
    return _lib.coreinfer_version()


def dev_set_param(name: str, value: int) -> None:
    _check(_lib.coreinfer_dev_set_param(name.encode(), int(value)), "coreinfer_dev_set_param")


def dev_get_param(name: str) -> int:
    out = _int(0)
    _check(_lib.coreinfer_dev_get_param(name.encode(), ctypes.byref(out)), "coreinfer_dev_get_param")
    return out.value


def dev_params() -> dict:
    """All development settings and their present values."""
    names = iter(lambda i=itertools.count(): _lib.coreinfer_dev_param_name(next(i)), None)
    return {n.decode(): dev_get_param(n.decode()) for n in names}


def dev_fused_plan(K: int, d: int, dtype: torch.dtype, act: str) -> dict:
    """Launch shape of the single-launch decode under the current development settings."""
    out = (_int * 5)()
    _check(_lib.coreinfer_dev_fused_plan(K, d, DTYPE_CODE[dtype], ACT_CODE[act], out), "coreinfer_dev_fused_plan")
    return dict(zip(("chunks", "chunk_neurons", "compute_waves", "loads_per_row", "workgroups"), list(out)))


def dev_decode_slices(B: int, K: int, d: int, dtype: torch.dtype, gathered: bool) -> int:
    """Neuron slices per sentence of the two-launch decode under the current development settings."""
    out = _int(0)
    _check(_lib.coreinfer_dev_decode_slices(B, K, d, DTYPE_CODE[dtype], int(bool(gathered)), ctypes.byref(out)),
           "coreinfer_dev_decode_slices")
    return out.value


def dev_decode_small(B: int, K: int, d: int, dtype: torch.dtype, act: str, stream=None) -> str:
    """Which way ffn_decode takes on a stream (a handle; the null stream by default) for neuron-major compact weights."""
    out = _int(0)
    _check(_lib.coreinfer_dev_decode_small(B, K, d, DTYPE_CODE[dtype], ACT_CODE[act], stream, ctypes.byref(out)),
           "coreinfer_dev_decode_small")
    return ("two launches", "all", "shared")[out.value]


def dev_decode_small_gave_up() -> int:
    """Workgroups that computed shared hidden values after all, on the current device so far."""
    out = ctypes.c_uint32(0)
    _check(_lib.coreinfer_dev_decode_small_gave_up(ctypes.byref(out)), "coreinfer_dev_decode_small_gave_up")
    return out.value


def dev_dense_plan(M: int, d: int, N: int, dtype: torch.dtype, act: str, down_layout: str, room: int = 1 << 62) -> dict:
    """How coreinfer_ffn_dense would tile both projections of more than four tokens with `room` bytes for split sums."""
    out = (_i64 * 9)()
    _check(_lib.coreinfer_dev_dense_plan(M, d, N, DTYPE_CODE[dtype], ACT_CODE[act], LAYOUT_CODE[down_layout], room, out),
           "coreinfer_dev_dense_plan")
    return dict(zip(("up", "up_tiles", "down", "full", "tail", "splits", "bytes", "up_once", "down_once"), out))


def dev_select_layout(B: int, M: int, N: int) -> dict:
    """Byte offsets of the pieces of coreinfer_select_batch's workspace (part: -1 if there are no byte counts)."""
    out = (_i64 * 4)()
    _check(_lib.coreinfer_dev_select_layout(B, M, N, out), "coreinfer_dev_select_layout")
    return dict(zip(("thresholds", "histograms", "counts", "part"), list(out)))


def dev_stream_probe(buf: torch.Tensor, window_bytes: int, per_workgroup: bool, workgroups: int, threads: int,
                     depth: int, iters: int, out: torch.Tensor) -> None:
    """Measurement aid: streams 16-byte loads over windows of `buf` (see csrc/coreinfer_dev.h)."""
    _check(_lib.coreinfer_dev_stream_probe(_ptr(buf), buf.numel() * buf.element_size(), int(window_bytes),
                                           int(bool(per_workgroup)), int(workgroups), int(threads), int(depth),
                                           int(iters), _ptr(out), _stream(buf)), "coreinfer_dev_stream_probe")


def dev_tile_probe(buf: torch.Tensor, pitch_bytes: int, shared: bool, workgroups: int, depth: int, ksteps: int,
                   iters: int, out: torch.Tensor) -> None:
    """Measurement aid: the load stream of a GEMM operand tile (see csrc/coreinfer_dev.h)."""
    _check(_lib.coreinfer_dev_tile_probe(_ptr(buf), buf.numel() * buf.element_size(), int(pitch_bytes),
                                         int(bool(shared)), int(workgroups), int(depth), int(ksteps), int(iters),
                                         _ptr(out), _stream(buf)), "coreinfer_dev_tile_probe")


def keep_count(frac: float, n: int) -> int:
    k = _i64(0)
    _check(_lib.coreinfer_keep_count(float(frac), int(n), ctypes.byref(k)), "coreinfer_keep_count")
    return k.value


def select_workspace_size(M: int, N: int) -> int:
    b = _sz(0)
    _check(_lib.coreinfer_select_workspace_size(M, N, ctypes.byref(b)), "coreinfer_select_workspace_size")
    return b.value


def select(act: torch.Tensor, alpha: float, beta: float, core_idx: Optional[torch.Tensor] = None,
           counts: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """coreinfer_select on A [M, N] fp32 (device).  Returns (core_idx, counts)."""
    assert act.dim() == 2 and act.dtype == torch.float32 and act.stride(1) == 1
    M, N = act.shape
    K = keep_count(beta, N)
    if core_idx is None:
        core_idx = torch.empty(K, dtype=torch.int32, device=act.device)
    if counts is None:
        counts = torch.empty(N, dtype=torch.int32, device=act.device)
    if ws is None:
        ws = _workspace(select_workspace_size(M, N), act)
    _check(_lib.coreinfer_select(_ptr(act), M, N, act.stride(0), float(alpha), float(beta),
                                 _ptr(core_idx), _ptr(counts), _ptr(ws), ws.numel(), _stream(act)),
           "coreinfer_select")
    return core_idx, counts


def select_batch_workspace_size(B: int, M: int, N: int) -> int:
    b = _sz(0)
    _check(_lib.coreinfer_select_batch_workspace_size(B, M, N, ctypes.byref(b)), "coreinfer_select_batch_workspace_size")
    return b.value


def select_batch(act: torch.Tensor, B: int, alpha: float, beta: float, core_idx: Optional[torch.Tensor] = None,
                 counts: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """coreinfer_select_batch on act [B * M, N] (fp32): returns (core_idx [B, K], counts [B, N])."""
    BM, N = act.shape
    M = BM // B
    assert M * B == BM
    K = keep_count(beta, N)
    if core_idx is None:
        core_idx = torch.empty((B, K), dtype=torch.int32, device=act.device)
    if counts is None:
        counts = torch.empty((B, N), dtype=torch.int32, device=act.device)
    if ws is None:
        ws = _workspace(select_batch_workspace_size(B, M, N), act)
    _check(_lib.coreinfer_select_batch(_ptr(act), B, M, N, act.stride(0), float(alpha), float(beta), _ptr(core_idx),
                                       _ptr(counts), _ptr(ws), ws.numel(), _stream(act)), "coreinfer_select_batch")
    return core_idx, counts


def select_hidden(hidden: torch.Tensor, act: str, alpha: float, beta: float,
                  core_idx: Optional[torch.Tensor] = None, counts: Optional[torch.Tensor] = None,
                  ws: Optional[torch.Tensor] = None):
    """coreinfer_select_hidden on H [M, N] of the layer's element type.  Returns (core_idx, counts)."""
    assert hidden.dim() == 2 and hidden.stride(1) == 1
    M, N = hidden.shape
    K = keep_count(beta, N)
    if core_idx is None:
        core_idx = torch.empty(K, dtype=torch.int32, device=hidden.device)
    if counts is None:
        counts = torch.empty(N, dtype=torch.int32, device=hidden.device)
    if ws is None:
        ws = _workspace(select_workspace_size(M, N), hidden)
    _check(_lib.coreinfer_select_hidden(_ptr(hidden), DTYPE_CODE[hidden.dtype], ACT_CODE[act], M, N,
                                        hidden.stride(0), float(alpha), float(beta), _ptr(core_idx),
                                        _ptr(counts), _ptr(ws), ws.numel(), _stream(hidden)),
           "coreinfer_select_hidden")
    return core_idx, counts


def count_tokens(act: torch.Tensor, alpha: float, counts: Optional[torch.Tensor] = None,
                 accumulate: bool = False, ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """coreinfer_count_tokens: Eq. 3 over the rows of act, optionally added to existing counts."""
    assert act.dim() == 2 and act.dtype == torch.float32 and act.stride(1) == 1
    M, N = act.shape
    if counts is None:
        assert not accumulate
        counts = torch.empty(N, dtype=torch.int32, device=act.device)
    if ws is None:
        ws = _workspace(select_workspace_size(M, N), act)
    _check(_lib.coreinfer_count_tokens(_ptr(act), M, N, act.stride(0), float(alpha), _ptr(counts),
                                       1 if accumulate else 0, _ptr(ws), ws.numel(), _stream(act)),
           "coreinfer_count_tokens")
    return counts


def count_select(counts: torch.Tensor, max_count: int, beta: float,
                 core_idx: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """coreinfer_count_select: Def. 2 on given counts."""
    N = counts.numel()
    if core_idx is None:
        core_idx = torch.empty(keep_count(beta, N), dtype=torch.int32, device=counts.device)
    if ws is None:
        ws = _workspace(256, counts)
    _check(_lib.coreinfer_count_select(_ptr(counts), N, int(max_count), float(beta), _ptr(core_idx),
                                       _ptr(ws), ws.numel(), _stream(counts)), "coreinfer_count_select")
    return core_idx


def group_select(core_sets: torch.Tensor, N: int, gamma: float, core_idx: Optional[torch.Tensor] = None,
                 counts: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """coreinfer_group_select on core_sets [G, K] int32.  Returns (core_idx, counts)."""
    assert core_sets.dim() == 2 and core_sets.dtype == torch.int32 and core_sets.is_contiguous()
    G, K = core_sets.shape
    if core_idx is None:
        core_idx = torch.empty(keep_count(gamma, N), dtype=torch.int32, device=core_sets.device)
    if counts is None:
        counts = torch.empty(N, dtype=torch.int32, device=core_sets.device)
    if ws is None:
        ws = _workspace(select_workspace_size(G, N), core_sets)
    _check(_lib.coreinfer_group_select(_ptr(core_sets), G, K, N, float(gamma), _ptr(core_idx), _ptr(counts),
                                       _ptr(ws), ws.numel(), _stream(core_sets)), "coreinfer_group_select")
    return core_idx, counts


def core_similarity(set_a: torch.Tensor, set_b: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """coreinfer_core_similarity.  Returns the device tensor [identical, involved]."""
    if out is None:
        out = torch.empty(2, dtype=torch.int32, device=set_a.device)
    _check(_lib.coreinfer_core_similarity(_ptr(set_a), set_a.numel(), _ptr(set_b), set_b.numel(), _ptr(out),
                                          _stream(set_a)), "coreinfer_core_similarity")
    return out


def assign_group(prompt_set: torch.Tensor, group_sets: torch.Tensor):
    """coreinfer_assign_group.  Returns (best [1] int32, inter_union [G, 2] int32) on the device."""
    G, Kg = group_sets.shape
    best = torch.empty(1, dtype=torch.int32, device=group_sets.device)
    iu = torch.empty((G, 2), dtype=torch.int32, device=group_sets.device)
    _check(_lib.coreinfer_assign_group(_ptr(prompt_set), prompt_set.numel(), _ptr(group_sets), G, Kg,
                                       _ptr(best), _ptr(iu), _stream(group_sets)), "coreinfer_assign_group")
    return best, iu


def assign_centroid(act: torch.Tensor, centroids: torch.Tensor, ws: Optional[torch.Tensor] = None):
    """coreinfer_assign_centroid on A [M, N] fp32 and centroids [G, N] fp32 (device).
    Returns (best [1] int32, dist [G] fp32, feature [N] fp32 = a view of the workspace)."""
    M, N = act.shape
    G = centroids.shape[0]
    if ws is None:
        b = _sz(0)
        _check(_lib.coreinfer_assign_centroid_workspace_size(N, ctypes.byref(b)),
               "coreinfer_assign_centroid_workspace_size")
        ws = torch.empty(b.value, dtype=torch.uint8, device=act.device)
    best = torch.empty(1, dtype=torch.int32, device=act.device)
    dist = torch.empty(G, dtype=torch.float32, device=act.device)
    _check(_lib.coreinfer_assign_centroid(_ptr(act), M, N, act.stride(0), _ptr(centroids), G, _ptr(best),
                                          _ptr(dist), _ptr(ws), ws.numel(), _stream(act)),
           "coreinfer_assign_centroid")
    return best, dist, ws[:N * 4].view(torch.float32)


def compact_down_ld(K: int, dtype: torch.dtype) -> int:
    ld = _i64(0)
    _check(_lib.coreinfer_compact_down_ld(int(K), DTYPE_CODE[dtype], ctypes.byref(ld)), "coreinfer_compact_down_ld")
    return ld.value


def compact_preferred_layout(K: int, d: int, dtype: torch.dtype, act: str) -> str:
    out = _int(0)
    _check(_lib.coreinfer_compact_preferred_layout(int(K), int(d), DTYPE_CODE[dtype], ACT_CODE[act], ctypes.byref(out)),
           "coreinfer_compact_preferred_layout")
    return "out_major" if out.value == CI_DOWN_OUT_MAJOR else "neuron_major"


def compact_buffers(K: int, d: int, dtype: torch.dtype, device, gate: bool, bias: bool,
                    down_c_layout: str = "neuron_major") -> dict:
    """Uninitialised compact buffers for coreinfer_compact; `down_c_layout` is recorded in the dict."""
    ld = compact_down_ld(K, dtype)
    down_shape = (K, d) if down_c_layout == "neuron_major" else (d, ld)
    # with an output-major down matrix the bias buffer is padded to whole 16-byte vectors as well
    nb = K if down_c_layout == "neuron_major" else ld
    return {"w_up_c": torch.empty((K, d), dtype=dtype, device=device),
            "w_gate_c": torch.empty((K, d), dtype=dtype, device=device) if gate else None,
            "b_up_c": torch.zeros((nb,), dtype=dtype, device=device) if bias else None,
            "w_down_c": torch.empty(down_shape, dtype=dtype, device=device),
            "down_c_layout": down_c_layout}


def compact(w_up, w_gate, b_up, w_down, down_layout: str, act: str, core_idx: torch.Tensor,
            out: Optional[dict] = None, status: Optional[torch.Tensor] = None,
            down_c_layout: Optional[str] = None) -> dict:
    """coreinfer_compact.  Returns the dict of compact buffers (allocated when `out` is not
    given): w_up_c, w_gate_c, b_up_c [K, ...] and w_down_c, [K, d] ("neuron_major", the
    default) or [d, ld] ("out_major"); the dict also records "down_c_layout"."""
    N, d = w_up.shape
    K = core_idx.numel()
    if out is None:
        out = compact_buffers(K, d, w_up.dtype, w_up.device, w_gate is not None, b_up is not None,
                              down_c_layout or "neuron_major")
    layout_c = out.get("down_c_layout", "neuron_major")
    assert down_c_layout is None or down_c_layout == layout_c
    _check(_lib.coreinfer_compact(_ptr(w_up), _ptr(w_gate), _ptr(b_up), _ptr(w_down),
                                  LAYOUT_CODE[down_layout], DTYPE_CODE[w_up.dtype], ACT_CODE[act],
                                  d, N, _ptr(core_idx), K, _ptr(out["w_up_c"]), _ptr(out["w_gate_c"]),
                                  _ptr(out["b_up_c"]), _ptr(out["w_down_c"]), LAYOUT_CODE[layout_c],
                                  _ptr(status), _stream(w_up)),
           "coreinfer_compact")
    return out


def compact_update(w_up, w_gate, b_up, w_down, down_layout: str, act: str, new_idx: torch.Tensor,
                   slot_idx: torch.Tensor, bufs: dict, changed: Optional[torch.Tensor] = None) -> torch.Tensor:
    """coreinfer_compact_update: `bufs` (from compact) and `slot_idx` are changed in place.
    Returns the device int32 [1] holding the number of rows rewritten."""
    N, d = w_up.shape
    K = new_idx.numel()
    if changed is None:
        changed = torch.zeros(1, dtype=torch.int32, device=w_up.device)
    b = _sz(0)
    _check(_lib.coreinfer_compact_update_workspace_size(N, K, ctypes.byref(b)),
           "coreinfer_compact_update_workspace_size")
    ws = _workspace(b.value, w_up)
    _check(_lib.coreinfer_compact_update(_ptr(w_up), _ptr(w_gate), _ptr(b_up), _ptr(w_down),
                                         LAYOUT_CODE[down_layout], DTYPE_CODE[w_up.dtype], ACT_CODE[act],
                                         d, N, _ptr(new_idx), K, _ptr(slot_idx), _ptr(bufs["w_up_c"]),
                                         _ptr(bufs["w_gate_c"]), _ptr(bufs["b_up_c"]), _ptr(bufs["w_down_c"]),
                                         LAYOUT_CODE[bufs.get("down_c_layout", "neuron_major")],
                                         _ptr(changed), _ptr(ws), ws.numel(), _stream(w_up)),
           "coreinfer_compact_update")
    return changed


def ffn_decode_workspace_size(B: int, K: int, d: int) -> int:
    b = _sz(0)
    _check(_lib.coreinfer_ffn_decode_workspace_size(B, K, d, ctypes.byref(b)),
           "coreinfer_ffn_decode_workspace_size")
    return b.value


def make_weights(w_up, w_gate, b_up, w_down, b_down, core_idx=None, K: Optional[int] = None,
                 down_layout: str = "neuron_major") -> ci_ffn_weights:
    """Fills the ci_ffn_weights descriptor.  Compacted: pass the [K, d] buffers and, for an
    output-major compact down matrix [d, ld], down_layout="out_major".  Gathered: pass the
    resident neuron-major [N, d] weights and core_idx [B, K]."""
    rows, d = w_up.shape
    if core_idx is None:
        K = rows if K is None else K
    else:
        K = core_idx.shape[-1]
    ld = w_down.shape[1] if (w_down is not None and down_layout == "out_major") else 0
    return ci_ffn_weights(_ptr(w_up), _ptr(w_gate), _ptr(b_up), _ptr(w_down), _ptr(b_down),
                          _ptr(core_idx), K, d, rows, ld, LAYOUT_CODE[down_layout])


def make_compact_weights(bufs: dict, b_down) -> ci_ffn_weights:
    """Descriptor over the buffers coreinfer_compact wrote (either layout of w_down_c)."""
    return make_weights(bufs["w_up_c"], bufs["w_gate_c"], bufs["b_up_c"], bufs["w_down_c"], b_down,
                        down_layout=bufs.get("down_c_layout", "neuron_major"))


def decode_workspace(B: int, K: int, d: int, device) -> torch.Tensor:
    """A zeroed workspace for coreinfer_ffn_decode (the single-launch path needs it zeroed once)."""
    return torch.zeros(ffn_decode_workspace_size(B, K, d), dtype=torch.uint8, device=device)


def ffn_decode_status(ws: torch.Tensor) -> int:
    """coreinfer_ffn_decode_status, synchronised: 0, or 1 if a single-launch decode gave up waiting."""
    out = torch.zeros(1, dtype=torch.int32, device=ws.device)
    _check(_lib.coreinfer_ffn_decode_status(_ptr(ws), _ptr(out), _stream(ws)), "coreinfer_ffn_decode_status")
    return int(out.item())


def ffn_decode(x: torch.Tensor, weights: ci_ffn_weights, act: str, y: Optional[torch.Tensor] = None,
               ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """coreinfer_ffn_decode on x [B, d] (or [d])."""
    x2 = x if x.dim() == 2 else x.unsqueeze(0)
    B, d = x2.shape
    if y is None:
        y = torch.empty_like(x2)
    if ws is None:
        ws = decode_workspace(B, weights.K, d, x.device)
    if not isinstance(weights, ci_ffn_weights):
        raise TypeError("weights: a descriptor of make_weights")
    status = _decode_call(x2.data_ptr(), B, ctypes.addressof(weights), DTYPE_CODE[x.dtype], ACT_CODE[act], y.data_ptr(),
                          ws.data_ptr(), ws.numel(), _stream(x))
    if status != CI_OK:
        raise CoreInferError(status, "coreinfer_ffn_decode")
    return y if x2 is x else y.squeeze(0)


def ffn_decode_static(x: torch.Tensor, weights: ci_ffn_weights, act: str, y: Optional[torch.Tensor] = None,
                      status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """coreinfer_ffn_decode_static on x [B, d] (or [d]): the library's own scratch, no allocation in the call
    (pass y to keep this wrapper from allocating the output)."""
    x2 = x if x.dim() == 2 else x.unsqueeze(0)
    B, d = x2.shape
    if y is None:
        y = torch.empty_like(x2)
    _check(_lib.coreinfer_ffn_decode_static(_ptr(x2), B, ctypes.byref(weights), DTYPE_CODE[x.dtype],
                                            ACT_CODE[act], _ptr(y), _ptr(status), _stream(x)),
           "coreinfer_ffn_decode_static")
    return y if x.dim() == 2 else y.squeeze(0)


def union_build(core_idx: torch.Tensor, N: int, max_rows: Optional[int] = None):
    """coreinfer_union_build on core_idx [B, K] int32.  Returns (union_idx [max_rows] int32,
    union_mask [max_rows] int32 holding the uint32 bits, union_count [1] int32), all on the device."""
    B, K = core_idx.shape
    if max_rows is None:
        max_rows = max(1, min(N, B * K))
    dev = core_idx.device
    union_idx = torch.empty(max_rows, dtype=torch.int32, device=dev)
    union_mask = torch.empty(max_rows, dtype=torch.int32, device=dev)
    union_count = torch.empty(1, dtype=torch.int32, device=dev)
    b = _sz(0)
    _check(_lib.coreinfer_union_workspace_size(N, ctypes.byref(b)), "coreinfer_union_workspace_size")
    ws = _workspace(b.value, core_idx)
    _check(_lib.coreinfer_union_build(_ptr(core_idx), B, K, N, max_rows, _ptr(union_idx), _ptr(union_mask),
                                      _ptr(union_count), _ptr(ws), ws.numel(), _stream(core_idx)),
           "coreinfer_union_build")
    return union_idx, union_mask, union_count


def ffn_decode_union_workspace_size(B: int, max_rows: int, d: int, dtype: torch.dtype, act: str) -> int:
    b = _sz(0)
    _check(_lib.coreinfer_ffn_decode_union_workspace_size(B, max_rows, d, DTYPE_CODE[dtype], ACT_CODE[act],
                                                          ctypes.byref(b)),
           "coreinfer_ffn_decode_union_workspace_size")
    return b.value


def ffn_decode_union(x: torch.Tensor, weights: ci_ffn_weights, union_idx: torch.Tensor,
                     union_mask: torch.Tensor, union_count: torch.Tensor, act: str,
                     y: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """coreinfer_ffn_decode_union on x [B, d]; weights = the resident neuron-major matrices."""
    B, d = x.shape
    max_rows = union_idx.numel()
    if y is None:
        y = torch.empty_like(x)
    if ws is None:
        ws = _workspace(ffn_decode_union_workspace_size(B, max_rows, d, x.dtype, act), x)
    _check(_lib.coreinfer_ffn_decode_union(_ptr(x), B, ctypes.byref(weights), _ptr(union_idx), _ptr(union_mask),
                                           _ptr(union_count), max_rows, DTYPE_CODE[x.dtype], ACT_CODE[act],
                                           _ptr(y), _ptr(ws), ws.numel(), _stream(x)),
           "coreinfer_ffn_decode_union")
    return y


def ffn_dense_workspace_size(M: int, d: int, N: int, dtype: torch.dtype) -> int:
    b = _sz(0)
    _check(_lib.coreinfer_ffn_dense_workspace_size(M, d, N, DTYPE_CODE[dtype], ctypes.byref(b)),
           "coreinfer_ffn_dense_workspace_size")
    return b.value


def ffn_dense(X: torch.Tensor, w_up, w_gate, b_up, w_down, b_down, down_layout: str, act: str,
              want_y: bool = True, want_a: bool = False, Y=None, A=None, ws=None):
    """coreinfer_ffn_dense on X [M, d].  Returns (Y or None, A or None)."""
    M, d = X.shape
    N = w_up.shape[0]
    if want_y and Y is None:
        Y = torch.empty((M, d), dtype=X.dtype, device=X.device)
    if want_a and A is None:
        A = torch.empty((M, N), dtype=torch.float32, device=X.device)
    if ws is None:
        ws = _workspace(ffn_dense_workspace_size(M, d, N, X.dtype), X)
    _check(_lib.coreinfer_ffn_dense(_ptr(X), M, _ptr(w_up), _ptr(w_gate), _ptr(b_up), _ptr(w_down),
                                    _ptr(b_down), LAYOUT_CODE[down_layout], DTYPE_CODE[X.dtype],
                                    ACT_CODE[act], d, N, _ptr(Y), _ptr(A), _ptr(ws), ws.numel(),
                                    _stream(X)),
           "coreinfer_ffn_dense")
    return Y, A


def ffn_dense_hidden(X: torch.Tensor, w_up, w_gate, b_up, w_down, b_down, down_layout: str, act: str,
                     want_y: bool = True, Y=None, H=None, ws=None):
    """coreinfer_ffn_dense_hidden on X [M, d].  Returns (Y or None, H [M, N] of X's dtype)."""
    M, d = X.shape
    N = w_up.shape[0]
    if want_y and Y is None:
        Y = torch.empty((M, d), dtype=X.dtype, device=X.device)
    if H is None:
        H = torch.empty((M, N), dtype=X.dtype, device=X.device)
    if ws is None:
        b = _sz(0)
        _check(_lib.coreinfer_ffn_dense_hidden_workspace_size(M, d, N, DTYPE_CODE[X.dtype], ctypes.byref(b)),
               "coreinfer_ffn_dense_hidden_workspace_size")
        ws = _workspace(b.value, X)
    _check(_lib.coreinfer_ffn_dense_hidden(_ptr(X), M, _ptr(w_up), _ptr(w_gate), _ptr(b_up), _ptr(w_down),
                                           _ptr(b_down), LAYOUT_CODE[down_layout], DTYPE_CODE[X.dtype],
                                           ACT_CODE[act], d, N, _ptr(Y), _ptr(H), _ptr(ws), ws.numel(),
                                           _stream(X)),
           "coreinfer_ffn_dense_hidden")
    return Y, H


class W4:
    """Weights [R, C] in 4 bits, in groups along C (w4_quantize)."""

    def __init__(self, packed: torch.Tensor, R: int, C: int, group: int):
        self.packed, self.R, self.C, self.group, self.ptr = packed, R, C, group, packed.data_ptr()


def w4_size(R: int, C: int, group: int) -> int:
    b = _sz(0)
    _check(_lib.coreinfer_w4_size(R, C, group, ctypes.byref(b)), "coreinfer_w4_size")
    return b.value


def w4_quantize(w: torch.Tensor, group: int = 64, packed: Optional[torch.Tensor] = None) -> W4:
    """coreinfer_w4_quantize on w [R, C] (rows may be strided).  Pass `packed` (w4_size bytes) to reuse a buffer."""
    assert w.dim() == 2 and w.stride(1) == 1
    R, C = w.shape
    if packed is None:
        packed = _workspace(w4_size(R, C, group), w)
    assert packed.numel() * packed.element_size() >= w4_size(R, C, group)
    _check(_lib.coreinfer_w4_quantize(_ptr(w), R, C, w.stride(0), DTYPE_CODE[w.dtype], group, _ptr(packed), _stream(w)),
           "coreinfer_w4_quantize")
    return W4(packed, R, C, group)


def w4_read(w: W4, dtype: torch.dtype, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """coreinfer_w4_read: the values that the packed weights stand for, [R, C]."""
    if out is None:
        out = torch.empty((w.R, w.C), dtype=dtype, device=w.packed.device)
    assert out.shape == (w.R, w.C) and out.dtype == dtype and out.stride(1) == 1
    _check(_lib.coreinfer_w4_read(_ptr(w.packed), w.R, w.C, w.group, _ptr(out), out.stride(0), DTYPE_CODE[dtype],
                                  _stream(out)), "coreinfer_w4_read")
    return out


def w4_matvec_workspace_size(M: int, C: int, dtype: torch.dtype) -> int:
    b = _sz(0)
    _check(_lib.coreinfer_w4_matvec_workspace_size(M, C, DTYPE_CODE[dtype], ctypes.byref(b)),
           "coreinfer_w4_matvec_workspace_size")
    return b.value


_W4_ACT = {"none": CI_ACT_NONE, **ACT_CODE}


def w4_matvec(x: torch.Tensor, w: W4, gate: Optional[W4] = None, bias: Optional[torch.Tensor] = None, act: str = "none",
              y: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
              out_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """coreinfer_w4_matvec on x [M, C] (or [C]): act(x W^T + bias), "swiglu" with `gate`: SiLU(x G^T) * (x W^T)."""
    R, C = w.R, w.C
    M, (ldx, last) = (x.shape[0], x.stride()) if x.dim() == 2 else (1, (C, x.stride(0)))
    assert x.shape[-1] == C and last == 1
    assert gate is None or (gate.R, gate.C, gate.group) == (R, C, w.group)
    assert bias is None or (bias.numel() == R and bias.is_contiguous())
    if y is None:
        y = torch.empty((M, R) if x.dim() == 2 else (R,), dtype=out_dtype or x.dtype, device=x.device)
    ldy, last = y.stride() if y.dim() == 2 else (R, y.stride(0))
    assert y.shape[-1] == R and y.numel() == M * R and last == 1
    x_type, y_type = DTYPE_CODE[x.dtype], DTYPE_CODE[y.dtype]
    if ws is None and (M > 4 or M * C > 8192):   # fewer need none
        need = w4_matvec_workspace_size(M, C, x.dtype)
        ws = _workspace(need, x) if need else None
    status = _w4_matvec_call(x.data_ptr(), M, ldx if M > 1 else C, x_type, w.ptr, None if gate is None else gate.ptr,
                             None if bias is None else bias.data_ptr(), 0 if bias is None else DTYPE_CODE[bias.dtype],
                             _W4_ACT[act], R, C, w.group, y.data_ptr(), ldy if M > 1 else R, y_type,
                             None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel(), _stream(x))
    if status != CI_OK:
        raise CoreInferError(status, "coreinfer_w4_matvec")
    return y


class Kv4Cache:
    """A layer's keys and values in 4 bits (kv4_cache), with the accumulated weight and the position of every slot."""

    def __init__(self, k, v, k_scale, v_scale, weight, pos, shape):
        self.k, self.v, self.k_scale, self.v_scale, self.weight, self.pos = k, v, k_scale, v_scale, weight, pos
        self.B, self.H, self.cap, self.D, self.group = shape
        self.desc = ci_kv4(_ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale), _ptr(weight), _ptr(pos), *shape)
        self.ptr = ctypes.addressof(self.desc)


def kv4_cache(B: int, H: int, cap: int, D: int, group: int = 64, weights: bool = True, device="cuda") -> Kv4Cache:
    """Buffers for `cap` slots (a multiple of 32) of B sentences and H heads of D channels; weights: with the
    accumulated weights and positions that kv4_evict goes by."""
    codes, scale = _sz(0), _sz(0)
    _check(_lib.coreinfer_kv4_sizes(B, H, cap, D, group, ctypes.byref(codes), ctypes.byref(scale)), "coreinfer_kv4_sizes")
    buf = lambda n: torch.empty(n, dtype=torch.uint8, device=device)  # noqa: E731
    weight = torch.zeros((B, H, cap), dtype=torch.float32, device=device) if weights else None
    pos = torch.full((B, H, cap), -1, dtype=torch.int32, device=device) if weights else None
    return Kv4Cache(buf(codes.value), buf(codes.value), buf(scale.value), buf(scale.value), weight, pos, (B, H, cap, D, group))


def _check_lens(cache: Kv4Cache, *lens: Optional[torch.Tensor]):
    for t in lens:
        assert t is None or (t.dtype == torch.int32 and t.numel() == cache.B and t.is_contiguous())


def kv4_append(cache: Kv4Cache, k: torch.Tensor, v: torch.Tensor, lens: torch.Tensor, start: Optional[torch.Tensor] = None,
               next_pos: Optional[torch.Tensor] = None) -> None:
    """coreinfer_kv4_append: k, v [B, S, H, D] (any strides, the same for both, channels contiguous) become the last S of
    the lens[b] slots of each sentence."""
    B, S, H, D = shape = k.shape
    stride = k.stride()
    assert v.shape == shape and v.dtype == k.dtype and v.stride() == stride and stride[3] == 1
    assert (B, H, D) == (cache.B, cache.H, cache.D)
    _check_lens(cache, lens, start, next_pos)
    status = _kv4_append_call(cache.ptr, k.data_ptr(), v.data_ptr(), S, stride[0], stride[1], stride[2], DTYPE_CODE[k.dtype],
                              _ptr(start), lens.data_ptr(), _ptr(next_pos), _stream(k))
    if status != CI_OK:
        raise CoreInferError(status, "coreinfer_kv4_append")


def kv4_read(cache: Kv4Cache, lens: torch.Tensor, first: int, count: int, dtype: torch.dtype,
             k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None):
    """coreinfer_kv4_read: the values of slots first .. first + count - 1, (k, v) [B, H, count, D]; zeros from lens on."""
    shape = (cache.B, cache.H, count, cache.D)
    for t in (k, v):
        assert t is None or (t.shape == shape and t.dtype == dtype and t.is_contiguous())
    k = torch.empty(shape, dtype=dtype, device=lens.device) if k is None else k
    v = torch.empty(shape, dtype=dtype, device=lens.device) if v is None else v
    _check_lens(cache, lens)
    status = _kv4_read_call(cache.ptr, lens.data_ptr(), first, count, k.data_ptr(), v.data_ptr(), DTYPE_CODE[dtype], _stream(k))
    if status != CI_OK:
        raise CoreInferError(status, "coreinfer_kv4_read")
    return k, v


def kv4_attend_workspace_size(cache: Kv4Cache, S: int, Hq: int, max_len: int, weights: bool) -> int:
    b = _sz(0)
    _check(_lib.coreinfer_kv4_attend_workspace_size(cache.B, cache.H, cache.D, S, Hq, max_len, int(bool(weights)),
                                                    ctypes.byref(b)), "coreinfer_kv4_attend_workspace_size")
    return b.value


def kv4_attend(q: torch.Tensor, cache: Kv4Cache, lens: torch.Tensor, scale: Optional[float] = None,
               max_len: Optional[int] = None, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
               weight_out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """coreinfer_kv4_attend: q [B, S, Hq, D], the last S tokens of each sentence, over the cache.  scale: 1 / sqrt(D) by
    default; max_len: the most any of lens is (the cache's capacity by default; the launches are sized by it)."""
    B, S, Hq, D = shape = q.shape
    stride, dtype = q.stride(), q.dtype
    assert (B, D) == (cache.B, cache.D) and stride[3] == 1
    _check_lens(cache, lens)
    max_len = cache.cap if max_len is None else max_len
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=q.device)
    assert out.shape == shape and out.dtype == dtype and out.is_contiguous()
    assert lse is None or (lse.shape == (B, S, Hq) and lse.dtype == torch.float32 and lse.is_contiguous())
    assert weight_out is None or (weight_out.shape == (B, cache.H, cache.cap) and weight_out.dtype == torch.float32 and
                                  weight_out.is_contiguous())
    if ws is None:
        ws = _workspace(kv4_attend_workspace_size(cache, S, Hq, max_len, weight_out is not None), q)
    status = _kv4_attend_call(cache.ptr, q.data_ptr(), S, Hq, stride[0], stride[1], stride[2], DTYPE_CODE[dtype],
                              D ** -0.5 if scale is None else float(scale), lens.data_ptr(), max_len, out.data_ptr(), _ptr(lse),
                              _ptr(weight_out), ws.data_ptr(), ws.numel(), _stream(q))
    if status != CI_OK:
        raise CoreInferError(status, "coreinfer_kv4_attend")
    return out


def kv4_evict_workspace_size(cache: Kv4Cache, max_len: int, budget: int) -> int:
    b = _sz(0)
    _check(_lib.coreinfer_kv4_evict_workspace_size(cache.B, cache.H, max_len, budget, ctypes.byref(b)),
           "coreinfer_kv4_evict_workspace_size")
    return b.value


def kv4_evict(cache: Kv4Cache, lens: torch.Tensor, next_pos: torch.Tensor, budget: int, recent: int,
              max_len: Optional[int] = None, weight_out: Optional[torch.Tensor] = None,
              pos_out: Optional[torch.Tensor] = None, lens_out: Optional[torch.Tensor] = None,
              ws: Optional[torch.Tensor] = None) -> None:
    """coreinfer_kv4_evict: cuts heads of more than `budget` slots to those of the last `recent` positions and of the largest
    accumulated weights.  weight_out, pos_out and lens_out are the cache's own and `lens` by default."""
    _check_lens(cache, lens, next_pos, lens_out)
    max_len = cache.cap if max_len is None else max_len
    weight_out = cache.weight if weight_out is None else weight_out
    pos_out = cache.pos if pos_out is None else pos_out
    lens_out = lens if lens_out is None else lens_out
    for t, dtype in ((weight_out, torch.float32), (pos_out, torch.int32)):
        assert t is None or (t.shape == (cache.B, cache.H, cache.cap) and t.dtype == dtype and t.is_contiguous())
    if ws is None:
        ws = _workspace(kv4_evict_workspace_size(cache, max_len, budget), lens)
    status = _kv4_evict_call(cache.ptr, lens.data_ptr(), next_pos.data_ptr(), max_len, budget, recent, _ptr(weight_out),
                             _ptr(pos_out), lens_out.data_ptr(), ws.data_ptr(), ws.numel(), _stream(lens))
    if status != CI_OK:
        raise CoreInferError(status, "coreinfer_kv4_evict")


CI_ROPE_HALF, CI_ROPE_INTERLEAVED = 0, 1
ROPE_STYLE = {"half": CI_ROPE_HALF, "interleaved": CI_ROPE_INTERLEAVED}
ROPE_SCALING = {"none": 0, "linear": 1, "base": 2, "parts": 3}


class RopeAngles:
    """Frequencies of rotary positions on the device (rope_angles): turns [rot / 2] int64."""

    def __init__(self, turns: torch.Tensor, scale: float, rot: int, style: str):
        assert rot >= 0 and rot % 2 == 0 and turns.shape == (rot // 2,) and turns.dtype is torch.int64 and turns.is_contiguous()
        self._turns, self.scale, self.rot, self.style = turns, scale, rot, style
        self.desc = ci_rope(_ptr(turns), scale, rot, ROPE_STYLE[style])
        self.ptr = ctypes.addressof(self.desc)
        self.device = turns.get_device()

    turns = property(lambda self: self._turns)   # calls go by its address: written to, not replaced


def rope_turns(rot: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, original: float = 0.0,
               fast: float = 32.0, slow: float = 1.0) -> torch.Tensor:
    """coreinfer_rope_turns: what each pair turns by a position, in 2^-64ths of a turn, [rot / 2] int64 (the bits of
    uint64) on the host."""
    turns = torch.empty(max(int(rot), 0) // 2, dtype=torch.int64)
    _check(_lib.coreinfer_rope_turns(int(rot), float(base), ROPE_SCALING[scaling], float(factor), float(original), float(fast), float(slow),
                                     _ptr(turns)), "coreinfer_rope_turns")
    return turns


def rope_angles(rot: int, base: float = 10000.0, style: str = "half", scaling: str = "none", factor: float = 1.0,
                original: float = 0.0, fast: float = 32.0, slow: float = 1.0, scale: Optional[float] = None,
                device="cuda") -> RopeAngles:
    """Angles of the first `rot` channels of each head: pairs of channels rot / 2 apart ("half") or of neighbours
    ("interleaved"); scaling "none", "linear", "base" or "parts" for a context `factor` times as long as `original`.  scale:
    of the turned channels; by default 1, and 0.1 ln(factor) + 1 for "parts" where the context is longer, factor > 1."""
    turns = rope_turns(rot, base, scaling, factor, original, fast, slow).to(device)
    if scale is None:
        scale = 0.1 * math.log(factor) + 1.0 if scaling == "parts" and factor > 1.0 else 1.0
    return RopeAngles(turns, float(scale), int(rot), style)


_HOST = "tensors in host memory, which a kernel would read at the host's addresses"


def _check_norm(norm: torch.Tensor, D: int, dtype: torch.dtype, device: int):
    assert norm.shape == (D,) and norm.dtype is dtype and norm.is_contiguous() and norm.get_device() == device


def _check_pos(pos: torch.Tensor, T: int, device: int):
    assert pos.dtype is torch.int32 and pos.shape == (T,) and pos.is_contiguous() and pos.get_device() == device


def rope(x: torch.Tensor, pos: Optional[torch.Tensor], angles: Optional[RopeAngles], norm: Optional[torch.Tensor] = None,
         eps: float = 1e-6, backward: bool = False, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """coreinfer_rope: x [T, H, D] (any strides, channels contiguous), normed by head with `norm` [D] and turned by the
    positions pos [T] int32.  backward: the gradient of the rotation.  out: any strides; may be x."""
    T, H, D = shape = x.shape
    dtype, s = x.dtype, x.stride()
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=x.device)
    o = out.stride()
    device = x.get_device()
    assert s[2] == 1 and o[2] == 1 and out.shape == shape and out.dtype is dtype and out.get_device() == device
    assert angles is None or angles.device == device
    if pos is not None:
        _check_pos(pos, T, device)
    if norm is not None:
        _check_norm(norm, D, dtype, device)
    assert device >= 0, _HOST
    status = _rope_call(x.data_ptr(), s[0], s[1], T, H, D, DTYPE_CODE[dtype], None if norm is None else norm.data_ptr(), eps,
                        None if angles is None else angles.ptr, None if pos is None else pos.data_ptr(), 1 if backward else 0,
                        out.data_ptr(), o[0], o[1], _stream(x))
    if status != CI_OK:
        raise CoreInferError(status, "coreinfer_rope")
    return out


class KvpCache:
    """A layer's keys and values in pages (kvp_cache): k, v [pages, H, page, D], table [B, most]."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor):
        assert k.dim() == 4 and v.shape == k.shape and v.dtype == k.dtype and k.is_contiguous() and v.is_contiguous()
        assert table.dim() == 2 and table.dtype == torch.int32 and table.is_contiguous()
        assert k.get_device() == v.get_device() == table.get_device()
        self._k, self._v, self._table, self.dtype = k, v, table, k.dtype
        self.pages, self.H, self.page, self.D = k.shape
        self.B, self.most = table.shape
        self.device = k.get_device()
        self._shape, self._first, self._lens = (self.H, self.D), (self.B + 1,), (self.B,)   # what calls are compared with
        self.desc = ci_kvp(_ptr(k), _ptr(v), _ptr(table), self.pages, self.most, self.B, self.H, self.page, self.D, DTYPE_CODE[k.dtype])
        self.ptr = ctypes.addressof(self.desc)

    # calls go by their addresses: written to, not replaced
    k, v, table = property(lambda self: self._k), property(lambda self: self._v), property(lambda self: self._table)


def kvp_cache(pages: int, H: int, page: int, D: int, dtype: torch.dtype, table: torch.Tensor) -> KvpCache:
    """Buffers for `pages` pages of `page` slots (16, 32, 64, 128 or 256) of H heads of D channels, on the table's device.  table
    [B, most] int32: the page of each sentence's slots page * i .. + page - 1 (-1: none yet); it is the caller's, who gives
    pages out by writing to it."""
    k, v = (torch.empty((pages, H, page, D), dtype=dtype, device=table.device) for _ in range(2))
    return KvpCache(k, v, table)


def _check_packed(cache: KvpCache, rows: torch.Tensor, first: torch.Tensor, lens: torch.Tensor):
    assert rows.get_device() == first.get_device() == lens.get_device() == cache.device
    assert first.dtype is torch.int32 and first.shape == cache._first and first.is_contiguous()
    assert lens.dtype is torch.int32 and lens.shape == cache._lens and lens.is_contiguous()


def kvp_append(cache: KvpCache, k: torch.Tensor, v: torch.Tensor, first: torch.Tensor, lens: torch.Tensor,
               angles: Optional[RopeAngles] = None, pos: Optional[torch.Tensor] = None, k_norm: Optional[torch.Tensor] = None,
               eps: float = 1e-6, q: Optional[torch.Tensor] = None, q_norm: Optional[torch.Tensor] = None,
               q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """coreinfer_kvp_append: the packed tokens' k, v [T, H, D] (the same strides, channels contiguous) to their slots, keys normed
    and turned on the way; q [T, Hq, D] goes the same way to q_out, which is returned."""
    shape, dtype, s = k.shape, k.dtype, k.stride()
    T, D = shape[0], cache.D
    assert v.shape == shape and v.dtype is dtype and s[2] == 1
    # strides of lengths of one say nothing
    assert v.stride() == s or all(n == 1 or x == y for n, x, y in zip(shape, v.stride(), s))
    assert shape[1:] == cache._shape and dtype is cache.dtype
    _check_packed(cache, k, first, lens)
    device = cache.device
    assert v.get_device() == device and (angles is None or angles.device == device)
    if pos is not None:
        _check_pos(pos, T, device)
    if k_norm is not None:
        _check_norm(k_norm, D, dtype, device)
    if q is not None:
        _, Hq, _ = q_shape = q.shape
        q0, q1, last = q.stride()
        assert q_shape == (T, Hq, D) and q.dtype is dtype and last == 1 and q.get_device() == device
        if q_norm is not None:
            _check_norm(q_norm, D, dtype, device)
        if q_out is None:
            q_out = torch.empty(q_shape, dtype=dtype, device=q.device)
        assert q_out.shape == q_shape and q_out.dtype is dtype and q_out.is_contiguous() and q_out.get_device() == device
        q_ptr, q_out_ptr = q.data_ptr(), q_out.data_ptr()
    else:
        assert q_out is None and q_norm is None
        Hq = q0 = q1 = 0
        q_ptr = q_out_ptr = None
    assert device >= 0, _HOST
    status = _kvp_append_call(cache.ptr, k.data_ptr(), v.data_ptr(), s[0], s[1], T, first.data_ptr(), lens.data_ptr(),
                              None if pos is None else pos.data_ptr(), None if angles is None else angles.ptr,
                              None if k_norm is None else k_norm.data_ptr(), eps, q_ptr, Hq, q0, q1,
                              None if q_norm is None else q_norm.data_ptr(), q_out_ptr, _stream(k))
    if status != CI_OK:
        raise CoreInferError(status, "coreinfer_kvp_append")
    return q_out


def kvp_attend_workspace_size(cache: KvpCache, T: int, Hq: int, max_rows: int, max_len: int, window: int = 0, sinks: int = 0) -> int:
    b = _sz(0)
    _check(_lib.coreinfer_kvp_attend_workspace_size(ctypes.byref(cache.desc), T, Hq, max_rows, max_len, window, sinks, ctypes.byref(b)),
           "coreinfer_kvp_attend_workspace_size")
    return b.value


def kvp_attend(q: torch.Tensor, cache: KvpCache, first: torch.Tensor, lens: torch.Tensor, max_rows: Optional[int] = None,
               max_len: Optional[int] = None, window: int = 0, sinks: int = 0, scale: Optional[float] = None,
               out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """coreinfer_kvp_attend: the packed rows q [T, Hq, D] over their sentences' pages, all that came before them or, with a
    window, the last `window` slots and the first `sinks`.  max_rows, max_len: the most rows and slots of a sentence (all
    rows and the table's slots by default; the launches are chosen and sized by them).  scale: 1 / sqrt(D) by default."""
    T, Hq, D = shape = q.shape
    dtype, s = q.dtype, q.stride()
    assert D == cache.D and dtype is cache.dtype and s[2] == 1
    _check_packed(cache, q, first, lens)
    if max_rows is None:
        max_rows = max(T, 1)
    if max_len is None:
        max_len = cache.most * cache.page
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=q.device)
    device = cache.device
    assert out.shape == shape and out.dtype is dtype and out.is_contiguous() and out.get_device() == device
    assert lse is None or (lse.shape == (T, Hq) and lse.dtype is torch.float32 and lse.is_contiguous() and lse.get_device() == device)
    assert ws is None or (ws.get_device() == device and ws.is_contiguous())
    assert device >= 0, _HOST
    if ws is None:
        need = kvp_attend_workspace_size(cache, T, Hq, max_rows, max_len, window, sinks)
        ws = _workspace(need, q) if need else None
    status = _kvp_attend_call(cache.ptr, q.data_ptr(), Hq, s[0], s[1], T, first.data_ptr(), lens.data_ptr(), max_rows, max_len, window,
                              sinks, D ** -0.5 if scale is None else scale, out.data_ptr(), None if lse is None else lse.data_ptr(),
                              None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel(), _stream(q))
    if status != CI_OK:
        raise CoreInferError(status, "coreinfer_kvp_attend")
    return out
