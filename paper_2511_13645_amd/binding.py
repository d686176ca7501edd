"""Thin binding of the C-ABI HIP library (include/fsa.h), same names as the C entry
points.  Argument marshalling only: every step of the path runs inside the library's
kernels.  PyTorch is used for device memory and the current stream, nothing else.

The functions below are the binding, through ctypes.  The most frequent of them first offer the call to
their counterpart in ``_fsa_host`` (csrc_host/fsa_host.cpp), which does the same without the interpreter for
plain arguments and returns None for anything else.  Without that module they take every call.

The library must have been built (``python -m paper_2511_13645_amd.build`` or
``__graft_entry__.build()``); there is no CPU fallback -- a missing library raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import importlib.machinery
import importlib.util
import os
import warnings
from typing import Optional, Sequence, Tuple

import torch

from . import build

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfsa_hip.so")
HOST_PATH = build.host_lib()
CLASS_HOST_PATH = build.class_host_lib()
BLOCK_HOST_PATH = build.block_host_lib()

FSA_F32, FSA_BF16, FSA_F16 = 0, 1, 2
FSA_I32, FSA_I64 = 0, 1
FSA_OK = 0
FSA_KMAX = 64
FSA_SCRATCH_FLOATS = 8 * 1024 * 1024

EXPORTS = ("fsa_sample_mean_fwd", "fsa_mean_replay_fwd", "fsa_mean_bwd", "fsa_mean_bwd_lp", "fsa_status_string",
           "fsa_sample_mean_layerwise_fwd", "fsa_sample_mean3_fwd", "fsa_mean3_replay_fwd", "fsa_mean3_bwd",
           "fsa_mean3_bwd_noalloc", "fsa_mean_bwd_ws", "fsa_mean_bwd_workspace_bytes",
           "fsa_bwd_workspace_bytes", "fsa_mean_bwd_lp_ws", "fsa_mean3_bwd_ws", "fsa_wmean_bwd_ws",
           "fsa_mean_bwd_dense", "fsa_mean_bwd_dense_workspace_bytes", "fsa_mean_bwd_dense_pays",
           "fsa_sample_wmean_fwd", "fsa_wmean_replay_fwd", "fsa_wmean_bwd",
           "fsa_class_fwd_workspace_bytes", "fsa_class_bwd_workspace_bytes",
           "fsa_xent_fwd", "fsa_xent_bwd", "fsa_distill_fwd", "fsa_distill_bwd",
           "fsa_norm_fwd", "fsa_norm_bwd", "fsa_norm_bwd_workspace_bytes",
           "fsa_gated_fwd", "fsa_gated_bwd", "fsa_gated_fwd_workspace_bytes", "fsa_gated_bwd_workspace_bytes",
           "fsa_gated_keep_pays", "fsa_gated_kept_bytes", "fsa_orthogonalize", "fsa_orthogonalize_workspace_bytes")

_lib: Optional[ctypes.CDLL] = None
_class_host = None                              # the module _fsa_class_host, likewise
_block_host = None                              # and _fsa_block_host
_host = None                                    # the module _fsa_host, once the library is loaded; None without it
_HOST_ENTRIES = ("fsa_sample_mean_fwd", "fsa_sample_wmean_fwd", "fsa_mean_replay_fwd", "fsa_mean_bwd", "fsa_mean_bwd_ws",
                 "fsa_mean_bwd_lp_ws", "fsa_wmean_bwd_ws", "fsa_mean_bwd_dense", "fsa_mean_bwd_dense_workspace_bytes",
                 "fsa_mean_bwd_dense_pays")              # entry points that _fsa_host calls
_CLASS_HOST_ENTRIES = ("fsa_class_fwd_workspace_bytes", "fsa_class_bwd_workspace_bytes", "fsa_xent_fwd", "fsa_xent_bwd",
                       "fsa_distill_fwd", "fsa_distill_bwd")             # the same of _fsa_class_host
_BLOCK_HOST_ENTRIES = ("fsa_norm_fwd", "fsa_norm_bwd", "fsa_norm_bwd_workspace_bytes", "fsa_gated_fwd", "fsa_gated_bwd",
                       "fsa_gated_fwd_workspace_bytes", "fsa_gated_bwd_workspace_bytes", "fsa_gated_keep_pays", "fsa_gated_kept_bytes")      # and of _fsa_block_host
_PLAIN, _WORKSPACE, _LOW_PRECISION, _WEIGHTED = range(4)                # backward entry points, as _fsa_host.bwd counts them


class FsaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s: %s (status %d)" % (where, status_string(status), status))


def lib() -> ctypes.CDLL:
    """Load the HIP library; fail loudly when it has not been built."""
    global _lib, _host, _class_host, _block_host
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("HIP library missing: %s (build it with __graft_entry__.build())" % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64, u64, ci = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_int
        L.fsa_sample_mean_fwd.argtypes = [vp, ci, vp, i64, vp, ci, i64, vp, i64, vp, ci, u64,
                                          vp, vp, vp, vp, vp]
        L.fsa_sample_mean_fwd.restype = ci
        L.fsa_mean_replay_fwd.argtypes = [vp, ci, i64, i64, vp, vp, i64, i32, i32, vp, vp, vp]
        L.fsa_mean_replay_fwd.restype = ci
        L.fsa_mean_bwd.argtypes = [vp, vp, vp, vp, i64, i32, i32, i64, vp, i64, vp]
        L.fsa_mean_bwd.restype = ci
        L.fsa_mean_bwd_ws.argtypes = [vp, vp, vp, vp, i64, i32, i32, i64, vp, i64, vp, i64, vp]
        L.fsa_mean_bwd_ws.restype = ci
        L.fsa_mean_bwd_workspace_bytes.argtypes = [i64, i32, i32, i64]
        L.fsa_mean_bwd_workspace_bytes.restype = i64
        L.fsa_mean_bwd_lp.argtypes = [vp, vp, ci, vp, vp, i64, i32, i32, i64, vp, ci, i64, vp]
        L.fsa_mean_bwd_lp.restype = ci
        L.fsa_sample_wmean_fwd.argtypes = [vp, ci, vp, vp, i64, vp, ci, i64, vp, i64, vp, ci, u64,
                                           vp, vp, vp, vp, vp, vp, vp]
        L.fsa_sample_wmean_fwd.restype = ci
        L.fsa_wmean_replay_fwd.argtypes = [vp, ci, i64, i64, vp, vp, vp, vp, i64, i32, i32, vp, vp, vp]
        L.fsa_wmean_replay_fwd.restype = ci
        L.fsa_wmean_bwd.argtypes = [vp, vp, vp, vp, vp, vp, i64, i32, i32, i64, vp, i64, vp]
        L.fsa_wmean_bwd.restype = ci
        L.fsa_sample_mean_layerwise_fwd.argtypes = [vp, ci, vp, i64, vp, ci, i64, vp, i64, vp, u64,
                                                    vp, vp, vp, vp, vp, vp]
        L.fsa_sample_mean_layerwise_fwd.restype = ci
        L.fsa_sample_mean3_fwd.argtypes = [vp, ci, vp, i64, vp, ci, i64, vp, i64, vp, u64,
                                           vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.fsa_sample_mean3_fwd.restype = ci
        L.fsa_mean3_replay_fwd.argtypes = [vp, ci, i64, i64, vp, vp, vp, i64, i32, i32, i32, vp, vp, vp, vp, vp, vp]
        L.fsa_mean3_replay_fwd.restype = ci
        L.fsa_mean3_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i32, i32, i32, i64, vp, i64, vp, vp]
        L.fsa_mean3_bwd.restype = ci
        L.fsa_mean3_bwd_noalloc.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i32, i32, i32, i64, vp, i64, vp]
        L.fsa_mean3_bwd_noalloc.restype = ci
        L.fsa_bwd_workspace_bytes.argtypes = [i64, i32, i32, i64, ci]
        L.fsa_bwd_workspace_bytes.restype = i64
        L.fsa_mean_bwd_lp_ws.argtypes = [vp, vp, ci, vp, vp, i64, i32, i32, i64, vp, ci, i64, vp, i64, vp]
        L.fsa_mean_bwd_lp_ws.restype = ci
        L.fsa_wmean_bwd_ws.argtypes = [vp, vp, vp, vp, vp, vp, i64, i32, i32, i64, vp, i64, vp, i64, vp]
        L.fsa_wmean_bwd_ws.restype = ci
        L.fsa_mean3_bwd_ws.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i32, i32, i32, i64, vp, i64, vp, vp, i64, vp]
        L.fsa_mean3_bwd_ws.restype = ci
        L.fsa_mean_bwd_dense_workspace_bytes.argtypes = [i64, i32, i32, i64, i64]
        L.fsa_mean_bwd_dense_workspace_bytes.restype = i64
        L.fsa_mean_bwd_dense_pays.argtypes = [i64, i32, i32, i64, ci, i64]
        L.fsa_mean_bwd_dense_pays.restype = ci
        L.fsa_mean_bwd_dense.argtypes = [vp, vp, ci, vp, vp, i64, i32, i32, i64, vp, i64, vp, i64, vp]
        L.fsa_mean_bwd_dense.restype = ci
        f32 = ctypes.c_float
        L.fsa_class_fwd_workspace_bytes.argtypes = [i64, i64, i64, ci, i32, ci]
        L.fsa_class_fwd_workspace_bytes.restype = i64
        L.fsa_class_bwd_workspace_bytes.argtypes = [i64, i64, i64, ci, i32, ci, ci]
        L.fsa_class_bwd_workspace_bytes.restype = i64
        L.fsa_xent_fwd.argtypes = [vp, i64, vp, i64, ci, i64, i64, i64, f32, vp, vp, vp, vp, vp, i64, vp]
        L.fsa_xent_fwd.restype = ci
        L.fsa_xent_bwd.argtypes = [vp, vp, i64, vp, i64, ci, i64, i64, i64, f32, vp, vp, vp, vp, vp, vp, i64, vp]
        L.fsa_xent_bwd.restype = ci
        L.fsa_distill_fwd.argtypes = [vp, i64, vp, i64, ci, i64, i64, i64, f32, f32, vp, vp, ci, i32, vp, vp, vp, vp, i64, vp]
        L.fsa_distill_fwd.restype = ci
        L.fsa_distill_bwd.argtypes = [vp, vp, i64, vp, i64, ci, i64, i64, i64, f32, f32, vp, vp, ci, i32, vp, vp, vp, vp, vp, i64, vp]
        L.fsa_distill_bwd.restype = ci
        L.fsa_norm_fwd.argtypes = [vp, i64, vp, i64, vp, ci, ci, i64, i64, f32, vp, vp, vp]
        L.fsa_norm_fwd.restype = ci
        L.fsa_norm_bwd_workspace_bytes.argtypes = [i64, i64, ci]
        L.fsa_norm_bwd_workspace_bytes.restype = i64
        L.fsa_norm_bwd.argtypes = [vp, vp, vp, i64, vp, ci, ci, i64, i64, f32, vp, vp, vp, i64, vp]
        L.fsa_norm_bwd.restype = ci
        for name in ("fsa_gated_fwd_workspace_bytes", "fsa_gated_bwd_workspace_bytes", "fsa_gated_keep_pays", "fsa_gated_kept_bytes"):
            getattr(L, name).argtypes = [i64, i64, i64, i64, ci]
            getattr(L, name).restype = ci if name == "fsa_gated_keep_pays" else i64
        L.fsa_gated_fwd.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, ci, ci, i64, i64, i64, i64, vp, vp, vp, i64, vp]
        L.fsa_gated_fwd.restype = ci
        L.fsa_gated_bwd.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, ci, ci, i64, i64, i64, i64, vp, vp, vp, vp, vp, vp, i64, vp]
        L.fsa_gated_bwd.restype = ci
        L.fsa_orthogonalize_workspace_bytes.argtypes = [i64, i64, i64, ci]
        L.fsa_orthogonalize_workspace_bytes.restype = i64
        L.fsa_orthogonalize.argtypes = [vp, i64, i64, ci, i64, i64, i64, vp, i32, f32, f32, vp, vp, i64, vp]
        L.fsa_orthogonalize.restype = ci
        L.fsa_status_string.argtypes = [ci]
        L.fsa_status_string.restype = ctypes.c_char_p
        _lib, _host, _class_host = L, _load_host(L), _load_class_host(L)
        _block_host = _load_block_host(L)
    return _lib


def _load_host(L: ctypes.CDLL):
    """The module _fsa_host at HOST_PATH, or None and a warning: it saves host time and nothing else."""
    return _load_module(L, "_fsa_host", HOST_PATH, _HOST_ENTRIES)


def _load_class_host(L: ctypes.CDLL):
    """The same for the class losses."""
    return _load_module(L, "_fsa_class_host", CLASS_HOST_PATH, _CLASS_HOST_ENTRIES)


def _load_block_host(L: ctypes.CDLL):
    """The same for the norm and the gated block."""
    return _load_module(L, "_fsa_block_host", BLOCK_HOST_PATH, _BLOCK_HOST_ENTRIES)


def _load_module(L: ctypes.CDLL, name: str, path: str, entries: Sequence[str]):
    try:
        spec = importlib.util.spec_from_loader(name, importlib.machinery.ExtensionFileLoader(name, path))
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        module.bind(_raw_stream, {e: ctypes.cast(getattr(L, e), ctypes.c_void_p).value for e in entries})
        return module
    except (ImportError, TypeError) as e:
        warnings.warn("calls go through Python only, which takes a few microseconds more: no %s (%s; build it with "
                      "__graft_entry__.build())" % (path, e), RuntimeWarning, stacklevel=4)
        return None


def status_string(status: int) -> str:
    return lib().fsa_status_string(int(status)).decode()


# The per-call checks and lookups below sit on the latency path of small calls (a call of a few seeds is
# bound by its host side), so the common case costs one comparison or one dictionary lookup.
_raw_stream = torch._C._cuda_getCurrentRawStream               # the current stream's handle, without a Stream object
_FLOAT_TYPE = {torch.float32: FSA_F32, torch.bfloat16: FSA_BF16, torch.float16: FSA_F16}


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _x_dtype(x: torch.Tensor) -> int:
    code = _FLOAT_TYPE.get(x.dtype)
    if code is None:
        raise TypeError("expected float32, bfloat16 or float16, got %s" % x.dtype)
    return code


def _indptr_type(indptr: torch.Tensor) -> int:
    if indptr.dtype == torch.int32:
        return FSA_I32
    if indptr.dtype == torch.int64:
        return FSA_I64
    raise TypeError("indptr must be int32 or int64, got %s" % indptr.dtype)


def _need(t: torch.Tensor, name: str, dtype=None) -> None:
    if t.is_cuda and t.is_contiguous() and (dtype is None or t.dtype == dtype):
        return
    if not t.is_cuda:
        raise ValueError("%s must live on the GPU" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))


def _shape(t: Optional[torch.Tensor], name: str, shape) -> None:
    if t is not None and t.shape != shape:
        raise ValueError("%s must be %s, got %s" % (name, tuple(shape), tuple(t.shape)))


def _same_device(ref: torch.Tensor, *named) -> None:
    dev = ref.device
    for t, name in named:
        if t is not None and t.device != dev:
            raise ValueError("%s lives on %s, expected %s" % (name, t.device, dev))


def _stream(stream: Optional[torch.cuda.Stream], like: torch.Tensor) -> int:
    """The stream to launch on: the caller's, else the current stream of the device that holds `like`."""
    return _raw_stream(like.get_device()) if stream is None else stream.cuda_stream


@functools.lru_cache(maxsize=256)
def _host_ints(values: Tuple[int, ...]) -> ctypes.Array:
    """A host array of these int32 values; the library reads it during the call and never writes it."""
    return (ctypes.c_int32 * max(1, len(values)))(*values)


def _taken(r, name: str) -> bool:
    """Whether _fsa_host took a call (it returned something); raises if the library refused it (a status)."""
    if r is None:
        return False
    if type(r) is int and r != FSA_OK:
        raise FsaError(r, name)
    return True


def check_workspace(workspace: torch.Tensor, like: torch.Tensor) -> None:
    """Raises unless `workspace` can serve a call on `like`'s device."""
    _need(workspace, "workspace")
    _same_device(like, (workspace, "workspace"))


def _room(workspace: Optional[torch.Tensor], like: torch.Tensor) -> Tuple[Optional[int], int]:
    """(address, bytes) of the workspace a caller hands to a backward call; (None, 0) without one."""
    if workspace is None:
        return None, 0
    check_workspace(workspace, like)
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def fsa_sample_mean_fwd(indptr: torch.Tensor, indices: torch.Tensor, x: torch.Tensor,
                        seeds: torch.Tensor, fanouts: Sequence[int], seed: int, *,
                        out: Optional[torch.Tensor] = None, out_h1: Optional[torch.Tensor] = None,
                        out_ids1: Optional[torch.Tensor] = None, out_ids2: Optional[torch.Tensor] = None,
                        emit_h1: bool = True, emit_ids: bool = True,
                        stream: Optional[torch.cuda.Stream] = None
                        ) -> Tuple[torch.Tensor, Optional[torch.Tensor], Optional[torch.Tensor], Optional[torch.Tensor]]:
    """Fused sample + mean forward.  Output tensors are allocated here (torch) unless given.
    Returns (out, out_h1, ids1, ids2); entries not asked for are None."""
    if _host is not None and stream is None and out is None and out_h1 is None and out_ids1 is None and out_ids2 is None:
        r = _host.sample_fwd(indptr, indices, None, x, seeds, fanouts, seed, emit_h1, emit_ids)
        if _taken(r, "fsa_sample_mean_fwd"):
            return r
    _need(indptr, "indptr"); _need(indices, "indices", torch.int32); _need(x, "x")
    _need(seeds, "seeds", torch.int32)
    fan = [int(k) for k in fanouts]
    hops = len(fan)
    B, (N, D) = seeds.shape[0], x.shape
    if indptr.shape[0] != N + 1:
        raise ValueError("indptr must have num_nodes+1 entries")
    k1 = fan[0] if hops >= 1 else 0
    k2 = fan[1] if hops >= 2 else 0
    if out is not None or out_h1 is not None or out_ids1 is not None or out_ids2 is not None:
        for t, n, dt, shp in ((out, "out", x.dtype, (B, D)), (out_h1, "out_h1", x.dtype, (B, k1, D)),
                              (out_ids1, "out_ids1", torch.int32, (B, k1)), (out_ids2, "out_ids2", torch.int32, (B, k1, k2))):
            if t is not None:
                _need(t, n, dt)
                _shape(t, n, shp)
                _same_device(x, (t, n))
    _same_device(x, (indptr, "indptr"), (indices, "indices"), (seeds, "seeds"))
    if out is None:
        out = x.new_empty((B, D))
    if hops == 2 and emit_h1 and out_h1 is None:
        out_h1 = x.new_empty((B, k1, D))
    if emit_ids and out_ids1 is None:
        out_ids1 = seeds.new_empty((B, k1))
    if emit_ids and hops == 2 and out_ids2 is None:
        out_ids2 = seeds.new_empty((B, k1, k2))
    fan_host = _host_ints(tuple(fan))
    rc = lib().fsa_sample_mean_fwd(_ptr(indptr), _indptr_type(indptr), _ptr(indices), N,
                                   _ptr(x), _x_dtype(x), D, _ptr(seeds), B,
                                   fan_host, hops, seed & (2**64 - 1),
                                   _ptr(out), _ptr(out_h1), _ptr(out_ids1), _ptr(out_ids2), _stream(stream, x))
    if rc != FSA_OK:
        raise FsaError(rc, "fsa_sample_mean_fwd")
    return out, out_h1, out_ids1, out_ids2


def fsa_mean_replay_fwd(x: torch.Tensor, ids1: torch.Tensor, ids2: Optional[torch.Tensor] = None, *,
                        out: Optional[torch.Tensor] = None, out_h1: Optional[torch.Tensor] = None,
                        emit_h1: bool = True, stream: Optional[torch.cuda.Stream] = None
                        ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Mean over saved IDs (no sampling).  Returns (out, out_h1)."""
    if _host is not None and stream is None and out is None and out_h1 is None:
        r = _host.replay_fwd(x, ids1, ids2, emit_h1)
        if _taken(r, "fsa_mean_replay_fwd"):
            return r
    _need(x, "x"); _need(ids1, "ids1", torch.int32)
    B, k1 = ids1.shape
    N, D = x.shape
    k2 = 0
    if ids2 is not None:
        _need(ids2, "ids2", torch.int32)
        if ids2.shape[0] != B or ids2.shape[1] != k1:
            raise ValueError("ids2 must be [B,k1,k2]")
        k2 = ids2.shape[2]
    for t, n, shp in ((out, "out", (B, D)), (out_h1, "out_h1", (B, k1, D))):
        if t is not None:
            _need(t, n, x.dtype)
            _shape(t, n, shp)
    _same_device(x, (ids1, "ids1"), (ids2, "ids2"), (out, "out"), (out_h1, "out_h1"))
    if out is None:
        out = x.new_empty((B, D))
    if ids2 is not None and emit_h1 and out_h1 is None:
        out_h1 = x.new_empty((B, k1, D))
    rc = lib().fsa_mean_replay_fwd(_ptr(x), _x_dtype(x), D, N, _ptr(ids1), _ptr(ids2), B, k1, k2,
                                   _ptr(out), _ptr(out_h1), _stream(stream, x))
    if rc != FSA_OK:
        raise FsaError(rc, "fsa_mean_replay_fwd")
    return out, out_h1


def fsa_mean_bwd(grad_out: torch.Tensor, ids1: torch.Tensor, ids2: Optional[torch.Tensor] = None,
                 grad_h1: Optional[torch.Tensor] = None, *, grad_x: torch.Tensor,
                 stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Scatter-add the mean's gradient into grad_x [N,D] fp32 (accumulated with atomics, not zeroed)."""
    if _host is not None and stream is None:
        if _taken(_host.bwd(_PLAIN, grad_out, ids1, None, ids2, None, grad_h1, grad_x, None), "fsa_mean_bwd"):
            return grad_x
    _need(grad_out, "grad_out", torch.float32); _need(ids1, "ids1", torch.int32)
    _need(grad_x, "grad_x", torch.float32)
    B, k1 = ids1.shape
    D = grad_out.shape[1]
    N = grad_x.shape[0]
    if grad_x.shape[1] != D or grad_out.shape[0] != B:
        raise ValueError("shape mismatch between grad_out, ids1 and grad_x")
    k2 = 0
    if ids2 is not None:
        _need(ids2, "ids2", torch.int32)
        if ids2.dim() != 3 or tuple(ids2.shape[:2]) != (B, k1):
            raise ValueError("ids2 must be [B,k1,k2]")
        k2 = ids2.shape[2]
    if grad_h1 is not None:
        _need(grad_h1, "grad_h1", torch.float32)
        _shape(grad_h1, "grad_h1", (B, k1, D))
    _same_device(grad_x, (grad_out, "grad_out"), (grad_h1, "grad_h1"), (ids1, "ids1"), (ids2, "ids2"))
    rc = lib().fsa_mean_bwd(_ptr(grad_out), _ptr(grad_h1), _ptr(ids1), _ptr(ids2), B, k1, k2, D,
                            _ptr(grad_x), N, _stream(stream, grad_x))
    if rc != FSA_OK:
        raise FsaError(rc, "fsa_mean_bwd")
    return grad_x


def fsa_mean_bwd_workspace_bytes(B: int, k1: int, k2: int, D: int) -> int:
    """Workspace bytes fsa_mean_bwd_ws can use for this shape (0: it always takes the atomic route)."""
    return int(lib().fsa_mean_bwd_workspace_bytes(B, k1, k2, D))


def fsa_bwd_workspace_bytes(B: int, k1: int, k2: int, D: int, dtype: torch.dtype = torch.float32) -> int:
    """Workspace bytes with which fsa_mean_bwd_lp, fsa_wmean_bwd and fsa_mean3_bwd into a [N,D] table of
    `dtype` update every destination row once (0: atomics whatever the workspace).  Three hops: (B*k1, k2, k3, D)."""
    return int(lib().fsa_bwd_workspace_bytes(B, k1, k2, D, _FLOAT_TYPE[dtype]))


def fsa_mean_bwd_ws(grad_out: torch.Tensor, ids1: torch.Tensor, ids2: Optional[torch.Tensor] = None,
                    grad_h1: Optional[torch.Tensor] = None, *, grad_x: torch.Tensor,
                    workspace: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """fsa_mean_bwd with an optional caller workspace (any contiguous GPU tensor; torch allocations are
    256-byte aligned, sized by fsa_mean_bwd_workspace_bytes).  Given one, wide-row 2-hop calls update every
    destination row once, without atomics: no other work may write grad_x or the workspace while they run."""
    if _host is not None and stream is None:
        if _taken(_host.bwd(_WORKSPACE, grad_out, ids1, None, ids2, None, grad_h1, grad_x, workspace), "fsa_mean_bwd_ws"):
            return grad_x
    _need(grad_out, "grad_out", torch.float32); _need(ids1, "ids1", torch.int32)
    _need(grad_x, "grad_x", torch.float32)
    B, k1 = ids1.shape
    D = grad_out.shape[1]
    N = grad_x.shape[0]
    if grad_x.shape[1] != D or grad_out.shape[0] != B:
        raise ValueError("shape mismatch between grad_out, ids1 and grad_x")
    k2 = 0
    if ids2 is not None:
        _need(ids2, "ids2", torch.int32)
        if ids2.dim() != 3 or tuple(ids2.shape[:2]) != (B, k1):
            raise ValueError("ids2 must be [B,k1,k2]")
        k2 = ids2.shape[2]
    if grad_h1 is not None:
        _need(grad_h1, "grad_h1", torch.float32)
        _shape(grad_h1, "grad_h1", (B, k1, D))
    _same_device(grad_x, (grad_out, "grad_out"), (grad_h1, "grad_h1"), (ids1, "ids1"), (ids2, "ids2"))
    ws, ws_bytes = _room(workspace, grad_x)
    rc = lib().fsa_mean_bwd_ws(_ptr(grad_out), _ptr(grad_h1), _ptr(ids1), _ptr(ids2), B, k1, k2, D,
                               _ptr(grad_x), N, ws, ws_bytes, _stream(stream, grad_x))
    if rc != FSA_OK:
        raise FsaError(rc, "fsa_mean_bwd_ws")
    return grad_x


def fsa_mean_bwd_dense_workspace_bytes(B: int, k1: int, k2: int, D: int, num_nodes: int) -> int:
    """Workspace bytes of fsa_mean_bwd_dense (k2 = 0: one hop); 0 where it is not available."""
    return int(lib().fsa_mean_bwd_dense_workspace_bytes(B, k1, k2, D, num_nodes))


def fsa_mean_bwd_dense_pays(B: int, k1: int, k2: int, D: int, dtype: torch.dtype, num_nodes: int) -> bool:
    """Whether fsa_mean_bwd_dense is expected to be faster than clearing a gradient and adding to it."""
    return bool(lib().fsa_mean_bwd_dense_pays(B, k1, k2, D, _FLOAT_TYPE[dtype], num_nodes))


def fsa_mean_bwd_dense(grad_out: torch.Tensor, ids1: torch.Tensor, ids2: Optional[torch.Tensor] = None,
                       grad_h1: Optional[torch.Tensor] = None, *, grad_x: torch.Tensor, workspace: torch.Tensor,
                       stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The backward as a gradient of its own: writes every row of grad_x [N,D] once, whatever it held (nothing to
    clear).  One type for grad_out, grad_h1 and grad_x.  `workspace`, sized by fsa_mean_bwd_dense_workspace_bytes:
    no other work may write grad_x or the workspace while the call runs."""
    _need(grad_out, "grad_out"); _need(ids1, "ids1", torch.int32); _need(grad_x, "grad_x", grad_out.dtype)
    B, k1 = ids1.shape
    N, D = grad_x.shape
    _shape(grad_out, "grad_out", (B, D))
    k2 = 0
    if ids2 is not None:
        _need(ids2, "ids2", torch.int32)
        if ids2.dim() != 3 or tuple(ids2.shape[:2]) != (B, k1):
            raise ValueError("ids2 must be [B,k1,k2]")
        k2 = ids2.shape[2]
    if grad_h1 is not None:
        _need(grad_h1, "grad_h1", grad_out.dtype)
        _shape(grad_h1, "grad_h1", (B, k1, D))
    _same_device(grad_x, (grad_out, "grad_out"), (grad_h1, "grad_h1"), (ids1, "ids1"), (ids2, "ids2"))
    ws, ws_bytes = _room(workspace, grad_x)
    rc = lib().fsa_mean_bwd_dense(_ptr(grad_out), _ptr(grad_h1), _x_dtype(grad_out), _ptr(ids1), _ptr(ids2), B, k1, k2, D,
                                  _ptr(grad_x), N, ws, ws_bytes, _stream(stream, grad_x))
    if rc != FSA_OK:
        raise FsaError(rc, "fsa_mean_bwd_dense")
    return grad_x


def grad_dense(grad_out: torch.Tensor, ids1: torch.Tensor, ids2: Optional[torch.Tensor], grad_h1: Optional[torch.Tensor],
               num_nodes: int) -> Optional[torch.Tensor]:
    """fsa_mean_bwd_dense into a gradient [num_nodes,D] allocated here, with a workspace that lasts for the call; None
    where clearing a gradient and adding to it is expected to be faster, or where the workspace finds no memory."""
    if _host is not None:
        grad_x = _host.grad_dense(grad_out, ids1, ids2, grad_h1, num_nodes)
        if grad_x is False:
            return None
        if _taken(grad_x, "fsa_mean_bwd_dense"):
            return grad_x
    B, k1 = ids1.shape
    D, k2 = grad_out.shape[1], 0 if ids2 is None else ids2.shape[2]
    if not fsa_mean_bwd_dense_pays(B, k1, k2, D, grad_out.dtype, num_nodes):
        return None
    grad_x = grad_out.new_empty((num_nodes, D))
    try:
        ws = grad_out.new_empty(fsa_mean_bwd_dense_workspace_bytes(B, k1, k2, D, num_nodes), dtype=torch.uint8)
    except torch.cuda.OutOfMemoryError:                        # no room beside the gradient: the other way needs none
        return None
    return fsa_mean_bwd_dense(grad_out, ids1, ids2, grad_h1, grad_x=grad_x, workspace=ws)


def fsa_mean_bwd_lp(grad_out: torch.Tensor, ids1: torch.Tensor, ids2: Optional[torch.Tensor] = None,
                    grad_h1: Optional[torch.Tensor] = None, *, grad_x: torch.Tensor,
                    stream: Optional[torch.cuda.Stream] = None,
                    workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Reduced-precision backward: grad_out / grad_h1 in fp32, bf16 or fp16; grad_x [N,D] either an
    fp32 master gradient or a 16-bit table added to with packed atomics (accumulated, not zeroed).
    `workspace`, sized by fsa_bwd_workspace_bytes: large 2-hop calls update every destination row once,
    without atomics; no other work may write grad_x or the workspace while the call runs."""
    if _host is not None and stream is None:
        if _taken(_host.bwd(_LOW_PRECISION, grad_out, ids1, None, ids2, None, grad_h1, grad_x, workspace), "fsa_mean_bwd_lp"):
            return grad_x
    _need(grad_out, "grad_out"); _need(ids1, "ids1", torch.int32); _need(grad_x, "grad_x")
    B, k1 = ids1.shape
    D = grad_out.shape[1]
    N = grad_x.shape[0]
    if grad_x.shape[1] != D or grad_out.shape[0] != B:
        raise ValueError("shape mismatch between grad_out, ids1 and grad_x")
    k2 = 0
    if ids2 is not None:
        _need(ids2, "ids2", torch.int32)
        if ids2.dim() != 3 or tuple(ids2.shape[:2]) != (B, k1):
            raise ValueError("ids2 must be [B,k1,k2]")
        k2 = ids2.shape[2]
    if grad_h1 is not None:
        _need(grad_h1, "grad_h1", grad_out.dtype)
        _shape(grad_h1, "grad_h1", (B, k1, D))
    _same_device(grad_x, (grad_out, "grad_out"), (grad_h1, "grad_h1"), (ids1, "ids1"), (ids2, "ids2"))
    g_type, x_type = _x_dtype(grad_out), _x_dtype(grad_x)
    ws, ws_bytes = _room(workspace, grad_x)
    rc = lib().fsa_mean_bwd_lp_ws(_ptr(grad_out), _ptr(grad_h1), g_type, _ptr(ids1), _ptr(ids2),
                                  B, k1, k2, D, _ptr(grad_x), x_type, N, ws, ws_bytes, _stream(stream, grad_x))
    if rc != FSA_OK:
        raise FsaError(rc, "fsa_mean_bwd_lp")
    return grad_x


def fsa_sample_mean_layerwise_fwd(indptr: torch.Tensor, indices: torch.Tensor, x: torch.Tensor, seeds: torch.Tensor,
                                  fanouts: Sequence[int], seed: int, *, emit_h1: bool = True, emit_ids: bool = True,
                                  stream: Optional[torch.cuda.Stream] = None):
    """Two-hop forward that also returns the plain hop-1 mean: (out, out_h1 | None, out_m1, ids1 | None, ids2 | None)."""
    _need(indptr, "indptr"); _need(indices, "indices", torch.int32); _need(x, "x"); _need(seeds, "seeds", torch.int32)
    fan = [int(k) for k in fanouts]
    if len(fan) != 2:
        raise ValueError("two fanouts expected")
    k1, k2 = fan
    B, (N, D) = seeds.shape[0], x.shape
    if indptr.shape[0] != N + 1:
        raise ValueError("indptr must have num_nodes+1 entries")
    _same_device(x, (indptr, "indptr"), (indices, "indices"), (seeds, "seeds"))
    out = x.new_empty((B, D))
    out_m1 = x.new_empty((B, D))
    out_h1 = x.new_empty((B, k1, D)) if emit_h1 else None
    ids1 = seeds.new_empty((B, k1)) if emit_ids else None
    ids2 = seeds.new_empty((B, k1, k2)) if emit_ids else None
    fan_host = _host_ints(tuple(fan))
    rc = lib().fsa_sample_mean_layerwise_fwd(_ptr(indptr), _indptr_type(indptr), _ptr(indices), N, _ptr(x), _x_dtype(x), D,
                                             _ptr(seeds), B, fan_host, int(seed) & (2**64 - 1),
                                             _ptr(out), _ptr(out_h1), _ptr(out_m1), _ptr(ids1), _ptr(ids2), _stream(stream, x))
    if rc != FSA_OK:
        raise FsaError(rc, "fsa_sample_mean_layerwise_fwd")
    return out, out_h1, out_m1, ids1, ids2


def fsa_sample_mean3_fwd(indptr: torch.Tensor, indices: torch.Tensor, x: torch.Tensor, seeds: torch.Tensor,
                         fanouts: Sequence[int], seed: int, *, emit_h2: bool = False, emit_ids: bool = True,
                         stream: Optional[torch.cuda.Stream] = None) -> dict:
    """Three-hop forward.  Returns a dict: out, out_h1, out_h2 | None, out_m1, ids1, ids2 | None, ids3 | None, cnt2."""
    _need(indptr, "indptr"); _need(indices, "indices", torch.int32); _need(x, "x"); _need(seeds, "seeds", torch.int32)
    fan = [int(k) for k in fanouts]
    if len(fan) != 3:
        raise ValueError("three fanouts expected")
    k1, k2, k3 = fan
    B, (N, D) = seeds.shape[0], x.shape
    if indptr.shape[0] != N + 1:
        raise ValueError("indptr must have num_nodes+1 entries")
    _same_device(x, (indptr, "indptr"), (indices, "indices"), (seeds, "seeds"))
    r = {"out": x.new_empty((B, D)),
         "out_h1": x.new_empty((B, k1, D)),
         "out_h2": x.new_empty((B, k1, k2, D)) if emit_h2 else None,
         "out_m1": x.new_empty((B, D)),
         "ids1": seeds.new_empty((B, k1)),
         "ids2": seeds.new_empty((B, k1, k2)) if emit_ids else None,
         "ids3": seeds.new_empty((B, k1, k2, k3)) if emit_ids else None,
         "cnt2": seeds.new_empty((B, k1))}
    fan_host = _host_ints(tuple(fan))
    rc = lib().fsa_sample_mean3_fwd(_ptr(indptr), _indptr_type(indptr), _ptr(indices), N, _ptr(x), _x_dtype(x), D,
                                    _ptr(seeds), B, fan_host, int(seed) & (2**64 - 1),
                                    _ptr(r["out"]), _ptr(r["out_h1"]), _ptr(r["out_h2"]), _ptr(r["out_m1"]),
                                    _ptr(r["ids1"]), _ptr(r["ids2"]), _ptr(r["ids3"]), _ptr(r["cnt2"]), _stream(stream, x))
    if rc != FSA_OK:
        raise FsaError(rc, "fsa_sample_mean3_fwd")
    return r


def fsa_mean3_replay_fwd(x: torch.Tensor, ids1: torch.Tensor, ids2: torch.Tensor, ids3: torch.Tensor, *,
                         emit_h2: bool = False, emit_m1: bool = True,
                         stream: Optional[torch.cuda.Stream] = None) -> dict:
    _need(x, "x"); _need(ids1, "ids1", torch.int32); _need(ids2, "ids2", torch.int32); _need(ids3, "ids3", torch.int32)
    B, k1, k2, k3 = ids3.shape
    if tuple(ids1.shape) != (B, k1) or tuple(ids2.shape) != (B, k1, k2):
        raise ValueError("ids1 / ids2 / ids3 shapes do not nest")
    N, D = x.shape
    _same_device(x, (ids1, "ids1"), (ids2, "ids2"), (ids3, "ids3"))
    r = {"out": x.new_empty((B, D)),
         "out_h1": x.new_empty((B, k1, D)),
         "out_h2": x.new_empty((B, k1, k2, D)) if emit_h2 else None,
         "out_m1": x.new_empty((B, D)) if emit_m1 else None,
         "cnt2": ids1.new_empty((B, k1))}
    rc = lib().fsa_mean3_replay_fwd(_ptr(x), _x_dtype(x), D, N, _ptr(ids1), _ptr(ids2), _ptr(ids3), B, k1, k2, k3,
                                    _ptr(r["out"]), _ptr(r["out_h1"]), _ptr(r["out_h2"]), _ptr(r["out_m1"]),
                                    _ptr(r["cnt2"]), _stream(stream, x))
    if rc != FSA_OK:
        raise FsaError(rc, "fsa_mean3_replay_fwd")
    return r


def fsa_mean3_bwd(grad_out: torch.Tensor, ids1: torch.Tensor, ids2: torch.Tensor, ids3: torch.Tensor, *,
                  grad_h1: Optional[torch.Tensor] = None, grad_h2: Optional[torch.Tensor] = None,
                  grad_m1: Optional[torch.Tensor] = None, grad_x: torch.Tensor,
                  work: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None,
                  noalloc: bool = False, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Scatter-add the three-hop mean's gradient into grad_x [N,D] fp32 (accumulated, not zeroed).
    noalloc=True calls fsa_mean3_bwd_noalloc: no workspace, the library's fixed scratch array.
    `workspace`, sized by fsa_bwd_workspace_bytes(B*k1, k2, k3, D): large calls update every destination
    row once, without atomics; no other work may write grad_x or the workspace while the call runs."""
    _need(grad_out, "grad_out", torch.float32); _need(grad_x, "grad_x", torch.float32)
    _need(ids1, "ids1", torch.int32); _need(ids2, "ids2", torch.int32); _need(ids3, "ids3", torch.int32)
    B, k1, k2, k3 = ids3.shape
    D = grad_out.shape[1]
    _shape(ids1, "ids1", (B, k1)); _shape(ids2, "ids2", (B, k1, k2))
    _shape(grad_out, "grad_out", (B, D))
    if grad_x.dim() != 2 or grad_x.shape[1] != D:
        raise ValueError("grad_x must be [N,%d]" % D)
    _same_device(grad_x, (grad_out, "grad_out"), (grad_h1, "grad_h1"), (grad_h2, "grad_h2"), (grad_m1, "grad_m1"),
                 (ids1, "ids1"), (ids2, "ids2"), (ids3, "ids3"), (work, "work"))
    for g, name, shape in ((grad_h1, "grad_h1", (B, k1, D)), (grad_h2, "grad_h2", (B, k1, k2, D)), (grad_m1, "grad_m1", (B, D))):
        if g is not None:
            _need(g, name, torch.float32)
            if tuple(g.shape) != shape:
                raise ValueError("%s must be %s" % (name, shape))
    if noalloc:
        rc = lib().fsa_mean3_bwd_noalloc(_ptr(grad_out), _ptr(grad_h1), _ptr(grad_h2), _ptr(grad_m1), _ptr(ids1), _ptr(ids2),
                                         _ptr(ids3), B, k1, k2, k3, D, _ptr(grad_x), grad_x.shape[0], _stream(stream, grad_x))
        if rc != FSA_OK:
            raise FsaError(rc, "fsa_mean3_bwd_noalloc")
        return grad_x
    if work is None:
        work = torch.empty((B, k1, D), dtype=torch.float32, device=grad_x.device)
    elif work.numel() < B * k1 * D or work.dtype != torch.float32 or not work.is_cuda or not work.is_contiguous():
        raise ValueError("work must be a contiguous GPU tensor that holds B*k1*D floats")
    ws, ws_bytes = _room(workspace, grad_x)
    rc = lib().fsa_mean3_bwd_ws(_ptr(grad_out), _ptr(grad_h1), _ptr(grad_h2), _ptr(grad_m1), _ptr(ids1), _ptr(ids2), _ptr(ids3),
                                B, k1, k2, k3, D, _ptr(grad_x), grad_x.shape[0], _ptr(work), ws, ws_bytes,
                                _stream(stream, grad_x))
    if rc != FSA_OK:
        raise FsaError(rc, "fsa_mean3_bwd")
    return grad_x


def fsa_sample_wmean_fwd(indptr: torch.Tensor, indices: torch.Tensor, edge_weight: torch.Tensor, x: torch.Tensor,
                         seeds: torch.Tensor, fanouts: Sequence[int], seed: int, *,
                         emit_h1: bool = True, emit_ids: bool = True,
                         stream: Optional[torch.cuda.Stream] = None):
    """Weighted fused sample + mean.  Returns (out, out_h1, ids1, ids2, w1, w2); IDs and weights
    are emitted together (emit_ids), entries not asked for are None."""
    if _host is not None and stream is None and edge_weight is not None:
        r = _host.sample_fwd(indptr, indices, edge_weight, x, seeds, fanouts, seed, emit_h1, emit_ids)
        if _taken(r, "fsa_sample_wmean_fwd"):
            return r
    _need(indptr, "indptr"); _need(indices, "indices", torch.int32); _need(x, "x")
    _need(seeds, "seeds", torch.int32); _need(edge_weight, "edge_weight", torch.float32)
    if edge_weight.shape[0] != indices.shape[0]:
        raise ValueError("edge_weight must have one entry per CSR entry")
    fan = [int(k) for k in fanouts]
    hops = len(fan)
    B, (N, D) = seeds.shape[0], x.shape
    dev = x.device
    if indptr.shape[0] != N + 1:
        raise ValueError("indptr must have num_nodes+1 entries")
    _same_device(x, (indptr, "indptr"), (indices, "indices"), (edge_weight, "edge_weight"), (seeds, "seeds"))
    k1 = fan[0] if hops >= 1 else 0
    k2 = fan[1] if hops >= 2 else 0
    out = x.new_empty((B, D))
    out_h1 = x.new_empty((B, k1, D)) if (hops == 2 and emit_h1) else None
    ids1 = seeds.new_empty((B, k1)) if emit_ids else None
    w1 = torch.empty((B, k1), dtype=torch.float32, device=dev) if emit_ids else None
    ids2 = seeds.new_empty((B, k1, k2)) if (emit_ids and hops == 2) else None
    w2 = torch.empty((B, k1, k2), dtype=torch.float32, device=dev) if (emit_ids and hops == 2) else None
    fan_host = _host_ints(tuple(fan))
    rc = lib().fsa_sample_wmean_fwd(_ptr(indptr), _indptr_type(indptr), _ptr(indices), _ptr(edge_weight), N,
                                    _ptr(x), _x_dtype(x), D, _ptr(seeds), B,
                                    fan_host, hops, seed & (2**64 - 1),
                                    _ptr(out), _ptr(out_h1), _ptr(ids1), _ptr(ids2), _ptr(w1), _ptr(w2),
                                    _stream(stream, x))
    if rc != FSA_OK:
        raise FsaError(rc, "fsa_sample_wmean_fwd")
    return out, out_h1, ids1, ids2, w1, w2


def fsa_wmean_replay_fwd(x: torch.Tensor, ids1: torch.Tensor, w1: torch.Tensor,
                         ids2: Optional[torch.Tensor] = None, w2: Optional[torch.Tensor] = None, *,
                         emit_h1: bool = True, stream: Optional[torch.cuda.Stream] = None):
    """Weighted mean over saved IDs and weights.  Returns (out, out_h1)."""
    _need(x, "x"); _need(ids1, "ids1", torch.int32); _need(w1, "w1", torch.float32)
    B, k1 = ids1.shape
    N, D = x.shape
    _shape(w1, "w1", (B, k1))
    k2 = 0
    if ids2 is not None:
        if w2 is None:
            raise ValueError("ids2 needs w2")
        _need(ids2, "ids2", torch.int32); _need(w2, "w2", torch.float32)
        if ids2.dim() != 3 or tuple(ids2.shape[:2]) != (B, k1):
            raise ValueError("ids2 must be [B,k1,k2]")
        k2 = ids2.shape[2]
        _shape(w2, "w2", (B, k1, k2))
    _same_device(x, (ids1, "ids1"), (w1, "w1"), (ids2, "ids2"), (w2, "w2"))
    out = x.new_empty((B, D))
    out_h1 = x.new_empty((B, k1, D)) if (ids2 is not None and emit_h1) else None
    rc = lib().fsa_wmean_replay_fwd(_ptr(x), _x_dtype(x), D, N, _ptr(ids1), _ptr(ids2), _ptr(w1), _ptr(w2),
                                    B, k1, k2, _ptr(out), _ptr(out_h1), _stream(stream, x))
    if rc != FSA_OK:
        raise FsaError(rc, "fsa_wmean_replay_fwd")
    return out, out_h1


def fsa_wmean_bwd(grad_out: torch.Tensor, ids1: torch.Tensor, w1: torch.Tensor,
                  ids2: Optional[torch.Tensor] = None, w2: Optional[torch.Tensor] = None,
                  grad_h1: Optional[torch.Tensor] = None, *, grad_x: torch.Tensor,
                  stream: Optional[torch.cuda.Stream] = None,
                  workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Weighted backward: scatter-add into grad_x [N,D] fp32 (accumulated, not zeroed).
    `workspace`, sized by fsa_bwd_workspace_bytes: large 2-hop calls update every destination row once,
    without atomics; no other work may write grad_x or the workspace while the call runs."""
    if _host is not None and stream is None and w1 is not None:
        if _taken(_host.bwd(_WEIGHTED, grad_out, ids1, w1, ids2, w2, grad_h1, grad_x, workspace), "fsa_wmean_bwd"):
            return grad_x
    _need(grad_out, "grad_out", torch.float32); _need(ids1, "ids1", torch.int32); _need(w1, "w1", torch.float32)
    _need(grad_x, "grad_x", torch.float32)
    B, k1 = ids1.shape
    D = grad_out.shape[1]
    _shape(grad_out, "grad_out", (B, D)); _shape(w1, "w1", (B, k1))
    if grad_x.dim() != 2 or grad_x.shape[1] != D:
        raise ValueError("grad_x must be [N,%d]" % D)
    k2 = 0
    if ids2 is not None:
        if w2 is None:
            raise ValueError("ids2 needs w2")
        _need(ids2, "ids2", torch.int32); _need(w2, "w2", torch.float32)
        if ids2.dim() != 3 or tuple(ids2.shape[:2]) != (B, k1):
            raise ValueError("ids2 must be [B,k1,k2]")
        k2 = ids2.shape[2]
        _shape(w2, "w2", (B, k1, k2))
    if grad_h1 is not None:
        _need(grad_h1, "grad_h1", torch.float32)
        _shape(grad_h1, "grad_h1", (B, k1, D))
    _same_device(grad_x, (grad_out, "grad_out"), (grad_h1, "grad_h1"), (ids1, "ids1"), (ids2, "ids2"), (w1, "w1"), (w2, "w2"))
    ws, ws_bytes = _room(workspace, grad_x)
    rc = lib().fsa_wmean_bwd_ws(_ptr(grad_out), _ptr(grad_h1), _ptr(ids1), _ptr(ids2), _ptr(w1), _ptr(w2),
                                B, k1, k2, D, _ptr(grad_x), grad_x.shape[0], ws, ws_bytes, _stream(stream, grad_x))
    if rc != FSA_OK:
        raise FsaError(rc, "fsa_wmean_bwd")
    return grad_x


# ----------------------------------------------------------------------------------------
# losses over many classes
# ----------------------------------------------------------------------------------------
FSA_CLASS_DMAX = 1024


def _rows(t: torch.Tensor, name: str) -> int:
    """Elements from one row of a matrix to the next; its rows are contiguous."""
    if not t.is_cuda:
        raise ValueError("%s must live on the GPU" % name)
    if t.dim() != 2 or t.shape[1] < 1:
        raise ValueError("%s must be a matrix, got %s" % (name, tuple(t.shape)))
    if t.stride(1) != 1 and t.shape[1] > 1:
        raise ValueError("%s must have contiguous rows" % name)
    if t.shape[0] > 1:
        if t.stride(0) < t.shape[1]:
            raise ValueError("the rows of %s must not overlap" % name)
        return t.stride(0)
    return t.shape[1]


def _class_operands(h: torch.Tensor, w: torch.Tensor, ids: torch.Tensor, logits: Optional[torch.Tensor]):
    """Checked leading arguments of the class losses: (pointers, strides and type, (T, V, D), K)."""
    hs, ws = _rows(h, "h"), _rows(w, "w")
    if h.dtype != w.dtype:
        raise TypeError("h and w must have one type, got %s and %s" % (h.dtype, w.dtype))
    (T, D), V = h.shape, w.shape[0]
    if w.shape[1] != D:
        raise ValueError("h and w must have rows of one length, got %d and %d" % (D, w.shape[1]))
    if logits is None:
        _need(ids, "targets", torch.int32)
        _shape(ids, "targets", (T,))
        K = 1
    else:
        _need(ids, "teacher_ids", torch.int32)
        _need(logits, "teacher_logits")
        _x_dtype(logits)
        if ids.dim() != 2 or ids.shape[0] != T or ids.shape[1] < 1:
            raise ValueError("teacher_ids must be [%d,K], got %s" % (T, tuple(ids.shape)))
        _shape(logits, "teacher_logits", ids.shape)
        K = ids.shape[1]
    _same_device(h, (w, "w"), (ids, "targets" if logits is None else "teacher_ids"), (logits, "teacher_logits"))
    return (_ptr(h), hs, _ptr(w), ws, _x_dtype(h), T, V, D), T, V, D, K


def _allocating(stream: Optional[torch.cuda.Stream]):
    """Allocations within are the call's stream's own: memory that another stream still works on is never handed out, and
    what is dropped goes back to where only later work of that stream gets it."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _class_workspace(workspace: Optional[torch.Tensor], need: int, like: torch.Tensor):
    """The caller's workspace, or one of torch's for the call."""
    if workspace is not None:
        check_workspace(workspace, like)
        return workspace
    return torch.empty(need, dtype=torch.uint8, device=like.device)


def _class_fwd(name: str, h, w, ids, logits, scale: float, temperature: float, emit_row_grad: bool, workspace, stream):
    if _class_host is not None and stream is None and workspace is None:
        r = _class_host.class_fwd(h, w, ids, logits, temperature, scale, emit_row_grad)
        if _taken(r, name):
            return r
    lead, T, V, D, K = _class_operands(h, w, ids, logits)
    L = lib()
    with _allocating(stream):
        loss = torch.empty((T,), dtype=torch.float32, device=h.device)
        lse = torch.empty_like(loss)
        row_grad = torch.empty((T, D), dtype=torch.float32, device=h.device) if emit_row_grad else None
        ws = _class_workspace(workspace, L.fsa_class_fwd_workspace_bytes(T, V, D, lead[4], K, int(emit_row_grad)), h)
    tail = (_ptr(loss), _ptr(lse), _ptr(row_grad), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream, h))
    if logits is None:
        rc = L.fsa_xent_fwd(*lead, scale, _ptr(ids), *tail)
    else:
        rc = L.fsa_distill_fwd(*lead, scale, temperature, _ptr(ids), _ptr(logits), _x_dtype(logits), K, *tail)
    if rc != FSA_OK:
        raise FsaError(rc, name)
    return loss, lse, row_grad


def _class_bwd(name: str, grad_loss, h, w, ids, logits, lse, row_grad, scale: float, temperature: float, want_h: bool, want_w: bool,
               workspace, stream):
    lead, T, V, D, K = _class_operands(h, w, ids, logits)
    for t, n in ((grad_loss, "grad_loss"), (lse, "lse")):
        _need(t, n, torch.float32)
        _shape(t, n, (T,))
    if row_grad is not None:
        _need(row_grad, "row_grad", torch.float32)
        _shape(row_grad, "row_grad", (T, D))
    _same_device(h, (grad_loss, "grad_loss"), (lse, "lse"), (row_grad, "row_grad"))
    L = lib()
    need = L.fsa_class_bwd_workspace_bytes(T, V, D, lead[4], K, int(want_h and row_grad is None), int(want_w))
    with _allocating(stream):
        grad_h = torch.empty((T, D), dtype=h.dtype, device=h.device) if want_h else None
        grad_w = torch.empty((V, D), dtype=w.dtype, device=w.device) if want_w else None
        ws = _class_workspace(workspace, need, h)
    tail = (_ptr(lse), _ptr(row_grad), _ptr(grad_h), _ptr(grad_w), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream, h))
    if logits is None:
        rc = L.fsa_xent_bwd(_ptr(grad_loss), *lead, scale, _ptr(ids), *tail)
    else:
        rc = L.fsa_distill_bwd(_ptr(grad_loss), *lead, scale, temperature, _ptr(ids), _ptr(logits), _x_dtype(logits), K, *tail)
    if rc != FSA_OK:
        raise FsaError(rc, name)
    return grad_h, grad_w


def class_loss(h, w, ids, logits, temperature: float, scale: float) -> Optional[torch.Tensor]:
    """The differentiable loss through the native host path, or None: then autograd.py's own function takes the call."""
    lib()
    if _class_host is not None:
        r = _class_host.class_loss(h, w, ids, logits, temperature, scale)
        if _taken(r, "fsa_xent_fwd" if logits is None else "fsa_distill_fwd"):
            return r
    return None


def fsa_xent_fwd(h: torch.Tensor, w: torch.Tensor, targets: torch.Tensor, scale: float = 1.0, *, emit_row_grad: bool = False,
                 workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None
                 ) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """Softmax cross entropy of rows h [T,D] against the classes w [V,D], the scores never kept; targets [T] int32, a
    negative one is none.  Returns (loss [T], lse [T], row_grad [T,D] | None), fp32.  `workspace`: see
    fsa_class_fwd_workspace_bytes; torch's memory without one.  With `stream`, results and workspace are that stream's, as of
    calls within ``torch.cuda.stream(stream)``: inputs have to be ready there, and whoever uses results elsewhere orders that."""
    return _class_fwd("fsa_xent_fwd", h, w, targets, None, float(scale), 1.0, bool(emit_row_grad), workspace, stream)


def fsa_xent_bwd(grad_loss: torch.Tensor, h: torch.Tensor, w: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor,
                 row_grad: Optional[torch.Tensor] = None, scale: float = 1.0, *, want_h: bool = True, want_w: bool = True,
                 workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None
                 ) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """Gradients (grad_h | None, grad_w | None) of fsa_xent_fwd from grad_loss [T] and what it returned."""
    return _class_bwd("fsa_xent_bwd", grad_loss, h, w, targets, None, lse, row_grad, float(scale), 1.0, bool(want_h), bool(want_w),
                      workspace, stream)


def fsa_distill_fwd(h: torch.Tensor, w: torch.Tensor, teacher_ids: torch.Tensor, teacher_logits: torch.Tensor,
                    temperature: float = 1.0, scale: float = 1.0, *, emit_row_grad: bool = False,
                    workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None
                    ) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """Divergence of the softmax of rows h [T,D] over the classes w [V,D] from a teacher's best classes: teacher_ids
    [T,K] int32 (negative: an empty slot) and their logits [T,K], renormalised over those.  Returns as fsa_xent_fwd."""
    return _class_fwd("fsa_distill_fwd", h, w, teacher_ids, teacher_logits, float(scale), float(temperature), bool(emit_row_grad),
                      workspace, stream)


def fsa_distill_bwd(grad_loss: torch.Tensor, h: torch.Tensor, w: torch.Tensor, teacher_ids: torch.Tensor,
                    teacher_logits: torch.Tensor, lse: torch.Tensor, row_grad: Optional[torch.Tensor] = None,
                    temperature: float = 1.0, scale: float = 1.0, *, want_h: bool = True, want_w: bool = True,
                    workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None
                    ) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """Gradients (grad_h | None, grad_w | None) of fsa_distill_fwd; the teacher gets none."""
    return _class_bwd("fsa_distill_bwd", grad_loss, h, w, teacher_ids, teacher_logits, lse, row_grad, float(scale), float(temperature),
                      bool(want_h), bool(want_w), workspace, stream)


def fsa_class_fwd_workspace_bytes(T: int, V: int, D: int, dtype: torch.dtype, K: int = 1, with_row_grad: bool = False) -> int:
    """Workspace bytes of fsa_xent_fwd (K = 1) and fsa_distill_fwd; 0 for sizes that they refuse."""
    return lib().fsa_class_fwd_workspace_bytes(T, V, D, _FLOAT_TYPE[dtype], K, int(with_row_grad))


def fsa_class_bwd_workspace_bytes(T: int, V: int, D: int, dtype: torch.dtype, K: int = 1, with_row_grad: bool = False,
                                  with_grad_w: bool = True) -> int:
    """Workspace bytes of fsa_xent_bwd and fsa_distill_bwd; `with_row_grad`: grad_h is wanted and no row_grad given."""
    return lib().fsa_class_bwd_workspace_bytes(T, V, D, _FLOAT_TYPE[dtype], K, int(with_row_grad), int(with_grad_w))


# ----------------------------------------------------------------------------------------
# the block between a mean and its loss, and the update of its matrices
# ----------------------------------------------------------------------------------------
FSA_NORM_DMAX = 16384
FSA_GATED_MOST = 1 << 16
FSA_GATED_FINE = 0x100
_ACTIVATIONS = {"silu": 0, "gelu": 1, "relu": 2}
ORTHOGONAL_COEFFICIENTS = (3.4445, -4.7750, 2.0315)     # singular values of 0.01 ... 1 go to 0.7 ... 1.2 in five steps


@contextlib.contextmanager
def _on(t: torch.Tensor, stream: Optional[torch.cuda.Stream]):
    """What a call allocates and launches belongs to `t`'s device and, where given, to the call's stream."""
    with contextlib.ExitStack() as stack:
        if torch.cuda.current_device() != t.get_device():
            stack.enter_context(torch.cuda.device(t.device))
        stack.enter_context(_allocating(stream))
        yield


def _goes_to_a_leaf(node) -> bool:
    """Whether a gradient goes to a leaf, straight or through nodes of one input alone, as casts and views are."""
    for _ in range(8):
        if node is None or node.name() == "torch::autograd::AccumulateGrad":
            return node is not None
        behind = [n for n, _ in node.next_functions if n is not None]
        node = behind[0] if len(behind) == 1 else None
    return False


def refuse_capture(what: str) -> None:
    """Raises in a backward that is captured into a graph while a leaf that its gradient goes to has an eager graph alive, one made on
    another stream (the block's own parameter, or what a cast or a view of it is made of): autograd would have that stream wait for the captured
    one, which ends the process.  Without the native host path, which
    knows the streams of autograd's nodes, in any captured backward whose gradients go to leaves."""
    if _block_host is not None:
        _block_host.refuse_capture(what)
        return
    node = torch._C._current_autograd_node()
    leaves = node is not None and any(_goes_to_a_leaf(n) for n, _ in node.next_functions)
    if leaves and torch.cuda.is_current_stream_capturing():
        raise RuntimeError("the backward of %s cannot be captured without the native host path (an eager graph of the same parameters "
                           "that is alive would end the process)" % what)


def _vector(t: torch.Tensor, name: str, n: int) -> None:
    _need(t, name)
    _x_dtype(t)
    _shape(t, name, (n,))


def _same_type(ref: torch.Tensor, ref_name: str, *named) -> None:
    for t, name in named:
        if t is not None and t.dtype != ref.dtype:
            raise TypeError("%s and %s must have one type, got %s and %s" % (ref_name, name, ref.dtype, t.dtype))


def fsa_norm_fwd(x: torch.Tensor, weight: torch.Tensor, residual: Optional[torch.Tensor] = None, eps: float = 1e-6, *,
                 stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Root-mean-square norm of rows s = x + residual [T,D] (rounded to their type), times weight [D] (of any of the three types).
    Returns (y, s | None), s where there is a residual.  `stream`: see fsa_xent_fwd."""
    if _block_host is not None and stream is None:
        r = _block_host.norm_fwd(x, weight, residual, eps)
        if _taken(r, "fsa_norm_fwd"):
            return r
    xs = _rows(x, "x")
    code = _x_dtype(x)
    T, D = x.shape
    _vector(weight, "weight", D)
    rs = 0
    if residual is not None:
        rs = _rows(residual, "residual")
        _same_type(x, "x", (residual, "residual"))
        _shape(residual, "residual", x.shape)
    _same_device(x, (weight, "weight"), (residual, "residual"))
    with _on(x, stream):
        y = torch.empty((T, D), dtype=x.dtype, device=x.device)
        s = torch.empty_like(y) if residual is not None else None
        rc = lib().fsa_norm_fwd(_ptr(x), xs, _ptr(residual), rs, _ptr(weight), code, _x_dtype(weight), T, D, float(eps),
                                _ptr(y), _ptr(s), _stream(stream, x))
    if rc != FSA_OK:
        raise FsaError(rc, "fsa_norm_fwd")
    return y, s


def norm(x, weight, residual, eps: float):
    """The differentiable (y, s | None) through the native host path, or None: then autograd.py's own function takes the call."""
    lib()
    if _block_host is not None:
        r = _block_host.norm(x, weight, residual, eps)
        if _taken(r, "fsa_norm_fwd"):
            return r
    return None


def fsa_norm_bwd(grad_y: Optional[torch.Tensor], grad_s: Optional[torch.Tensor], s: torch.Tensor, weight: torch.Tensor,
                 eps: float = 1e-6, *, want_x: bool = True, want_weight: bool = True, workspace: Optional[torch.Tensor] = None,
                 stream: Optional[torch.cuda.Stream] = None) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """Gradients (grad_x | None, grad_weight | None) of fsa_norm_fwd; grad_x is the residual's as well.  s [T,D]: the sum that
    the forward returned, or x where there was no residual.  grad_y, grad_s [T,D]: None for none.  `workspace`: see
    fsa_norm_bwd_workspace_bytes; torch's memory without one."""
    stride = _rows(s, "s")
    code = _x_dtype(s)
    T, D = s.shape
    _vector(weight, "weight", D)
    for g, name in ((grad_y, "grad_y"), (grad_s, "grad_s")):
        if g is not None:
            _need(g, name, s.dtype)
            _shape(g, name, s.shape)
    _same_device(s, (weight, "weight"), (grad_y, "grad_y"), (grad_s, "grad_s"))
    L = lib()
    with _on(s, stream):
        grad_x = torch.empty((T, D), dtype=s.dtype, device=s.device) if want_x else None
        grad_weight = torch.empty((D,), dtype=weight.dtype, device=s.device) if want_weight else None
        ws = _class_workspace(workspace, L.fsa_norm_bwd_workspace_bytes(T, D, code) if want_weight else 0, s)
        rc = L.fsa_norm_bwd(_ptr(grad_y), _ptr(grad_s), _ptr(s), stride, _ptr(weight), code, _x_dtype(weight), T, D, float(eps),
                            _ptr(grad_x), _ptr(grad_weight), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream, s))
    if rc != FSA_OK:
        raise FsaError(rc, "fsa_norm_bwd")
    return grad_x, grad_weight


def fsa_norm_bwd_workspace_bytes(T: int, D: int, dtype: torch.dtype) -> int:
    """Workspace bytes of fsa_norm_bwd; 0 for sizes that it refuses."""
    return lib().fsa_norm_bwd_workspace_bytes(T, D, _FLOAT_TYPE[dtype])


def _gated_operands(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, activation: str, fine: bool):
    """Checked arguments of the gated block: (pointers, strides, type, activation and sizes), (T, D, H, O)."""
    act = _ACTIVATIONS.get(activation)
    if act is None:
        raise ValueError("activation must be one of %s, got %r" % (", ".join(sorted(_ACTIVATIONS)), activation))
    named = ((x, "x"), (w_gate, "w_gate"), (w_up, "w_up"), (w_down, "w_down"))
    strides = [_rows(t, name) for t, name in named]
    code = _x_dtype(x) | (FSA_GATED_FINE if fine else 0)
    _same_type(x, "x", *named[1:])
    _same_device(x, *named[1:])
    (T, D), H, O = x.shape, w_gate.shape[0], w_down.shape[0]
    if H < 1 or O < 1:
        raise ValueError("w_gate and w_down must have rows")
    _shape(w_gate, "w_gate", (H, D))
    _shape(w_up, "w_up", (H, D))
    _shape(w_down, "w_down", (O, H))
    lead = [a for (t, _), stride in zip(named, strides) for a in (_ptr(t), stride)]
    return (*lead, code, act, T, D, H, O), (T, D, H, O)


def fsa_gated_fwd(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, *, activation: str = "silu",
                  emit_kept: bool = False, fine: bool = False, workspace: Optional[torch.Tensor] = None,
                  stream: Optional[torch.cuda.Stream] = None):
    """Gated feed-forward block (act(x w_gate^T) * (x w_up^T)) w_down^T: x [T,D], w_gate and w_up [H,D], w_down [O,H], all of one
    type; activation "silu", "gelu" (by the error function) or "relu".  Returns y [T,O], with `emit_kept` (y, kept): bytes
    that spare a backward of the same operands making the hidden products again (fsa_gated_keep_pays).  `fine`: 16-bit calls of any
    size hold what lies between the products in two numbers of the type, as calls of up to 16 rows or 4e9 operations do:
    results are off by their own rounding alone, and large calls take up to twice as long; given to a forward, it is to be given
    to its backward and to the functions of sizes.  `workspace`: see fsa_gated_fwd_workspace_bytes; torch's
    memory without one.  `stream`: see fsa_xent_fwd."""
    if _block_host is not None and stream is None and workspace is None and not emit_kept:
        r = _block_host.gated_fwd(x, w_gate, w_up, w_down, _ACTIVATIONS.get(activation), bool(fine))
        if _taken(r, "fsa_gated_fwd"):
            return r
    lead, (T, D, H, O) = _gated_operands(x, w_gate, w_up, w_down, activation, fine)
    L = lib()
    with _on(x, stream):
        y = torch.empty((T, O), dtype=x.dtype, device=x.device)
        kept = torch.empty((L.fsa_gated_kept_bytes(T, D, H, O, lead[8]),), dtype=torch.uint8, device=x.device) if emit_kept else None
        ws = _class_workspace(workspace, L.fsa_gated_fwd_workspace_bytes(T, D, H, O, lead[8]), x)
        rc = L.fsa_gated_fwd(*lead, _ptr(y), _ptr(kept), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream, x))
    if rc != FSA_OK:
        raise FsaError(rc, "fsa_gated_fwd")
    return (y, kept) if emit_kept else y


def gated(x, w_gate, w_up, w_down, activation: str, fine: bool, keep: Optional[bool]):
    """The differentiable block through the native host path, or None: then autograd.py's own function takes the call."""
    lib()
    if _block_host is not None:
        r = _block_host.gated(x, w_gate, w_up, w_down, _ACTIVATIONS.get(activation), bool(fine), keep if keep is None else bool(keep))
        if _taken(r, "fsa_gated_fwd"):
            return r
    return None


def fsa_gated_bwd(grad_y: torch.Tensor, x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor,
                  kept: Optional[torch.Tensor] = None, *, activation: str = "silu", want: Sequence[bool] = (True, True, True, True),
                  fine: bool = False, workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """Gradients of fsa_gated_fwd by x, w_gate, w_up and w_down from grad_y [T,O]; None where not wanted.  `kept`: what the
    forward emitted, or None.  `fine`: see there."""
    lead, (T, D, H, O) = _gated_operands(x, w_gate, w_up, w_down, activation, fine)
    gs = _rows(grad_y, "grad_y")
    _same_type(x, "x", (grad_y, "grad_y"))
    _shape(grad_y, "grad_y", (T, O))
    L = lib()
    if kept is not None:
        _need(kept, "kept", torch.uint8)
        _shape(kept, "kept", (L.fsa_gated_kept_bytes(T, D, H, O, lead[8]),))
    _same_device(x, (grad_y, "grad_y"), (kept, "kept"))
    with _on(x, stream):
        grads = tuple(torch.empty(t.shape, dtype=x.dtype, device=x.device) if w else None
                      for t, w in zip((x, w_gate, w_up, w_down), want))
        ws = _class_workspace(workspace, L.fsa_gated_bwd_workspace_bytes(T, D, H, O, lead[8]), x)
        rc = L.fsa_gated_bwd(_ptr(grad_y), gs, *lead, _ptr(kept), *(_ptr(g) for g in grads), _ptr(ws), ws.numel() * ws.element_size(),
                             _stream(stream, x))
    if rc != FSA_OK:
        raise FsaError(rc, "fsa_gated_bwd")
    return grads


def fsa_gated_keep_pays(T: int, D: int, H: int, O: int, dtype: torch.dtype) -> bool:
    """Whether a forward whose backward follows had better emit what that can be given."""
    return bool(lib().fsa_gated_keep_pays(T, D, H, O, _FLOAT_TYPE[dtype]))


def fsa_gated_fwd_workspace_bytes(T: int, D: int, H: int, O: int, dtype: torch.dtype, fine: bool = False) -> int:
    """Workspace bytes of fsa_gated_fwd; 0 for sizes that it refuses."""
    return lib().fsa_gated_fwd_workspace_bytes(T, D, H, O, _FLOAT_TYPE[dtype] | (FSA_GATED_FINE if fine else 0))


def fsa_gated_bwd_workspace_bytes(T: int, D: int, H: int, O: int, dtype: torch.dtype, fine: bool = False) -> int:
    """Workspace bytes of fsa_gated_bwd; 0 for sizes that it refuses."""
    return lib().fsa_gated_bwd_workspace_bytes(T, D, H, O, _FLOAT_TYPE[dtype] | (FSA_GATED_FINE if fine else 0))


def fsa_orthogonalize(g: torch.Tensor, coefficients: Sequence = ORTHOGONAL_COEFFICIENTS, steps: int = 5, *, eps: float = 1e-7,
                      scale: float = 1.0, workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None
                      ) -> torch.Tensor:
    """`scale` times the orthogonalised matrix g [M,N], or matrices [B,M,N], by Newton-Schulz steps: X = g / (|g| + eps), then
    X = a X + (b A + c A A) X with A = X X^T.  `coefficients`: (a, b, c) of every step, or one triple for each of `steps` steps; those
    beyond 16 have to keep singular values of 0 to 1 below 8.
    `workspace`: see fsa_orthogonalize_workspace_bytes; torch's memory without one.  `stream`: see fsa_xent_fwd."""
    if not g.is_cuda:
        raise ValueError("g must live on the GPU")
    if g.dim() not in (2, 3) or g.shape[-1] < 1 or g.shape[-2] < 1:
        raise ValueError("g must be a matrix or a batch of matrices, got %s" % (tuple(g.shape),))
    code = _x_dtype(g)
    if len(coefficients) and not isinstance(coefficients[0], (tuple, list)):
        coefficients = [tuple(coefficients)] * int(steps)
    if any(len(c) != 3 for c in coefficients):
        raise ValueError("coefficients must be triples")
    B, (M, N) = (g.shape[0] if g.dim() == 3 else 1), g.shape[-2:]
    if (g.stride(-1) != 1 and N > 1) or (M > 1 and g.stride(-2) < N):
        raise ValueError("g must have contiguous rows that do not overlap")
    stride = g.stride(-2) if M > 1 else N
    host = (ctypes.c_float * max(1, 3 * len(coefficients)))(*(float(x) for c in coefficients for x in c))
    L = lib()
    with _on(g, stream):
        out = torch.empty(g.shape, dtype=g.dtype, device=g.device)
        ws = _class_workspace(workspace, L.fsa_orthogonalize_workspace_bytes(B, M, N, code), g)
        rc = L.fsa_orthogonalize(_ptr(g), g.stride(0) if g.dim() == 3 else 0, stride, code, B, M, N, host, len(coefficients),
                                 float(eps), float(scale), _ptr(out), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream, g))
    if rc != FSA_OK:
        far = any(abs(x) > 16 for x in host)
        raise FsaError(rc, "fsa_orthogonalize" + (" (coefficients beyond 16 have to keep singular values of 0 to 1 below 8)" if far else ""))
    return out


def fsa_orthogonalize_workspace_bytes(B: int, M: int, N: int, dtype: torch.dtype) -> int:
    """Workspace bytes of fsa_orthogonalize; 0 for sizes that it refuses."""
    return lib().fsa_orthogonalize_workspace_bytes(B, M, N, _FLOAT_TYPE[dtype])
