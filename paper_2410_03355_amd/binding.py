"""Thin binding of liblantern.so: argument marshalling only.

PyTorch supplies device memory and the current HIP stream; every step of the
verification path runs in the library's kernels.  There is no CPU fallback: if
the library is missing, load() raises.

The calls of a decoding step first go to their namesakes in _marshal.so, which
take plain device tensors and nothing of the caller's (stream, outputs) without
the interpreter in between; whatever those decline takes the way through ctypes
below, which words the errors.  Without a _marshal.so for this PyTorch every call
takes that way: the same kernels and results, later launches.
"""
from __future__ import annotations

import contextlib
import ctypes
import importlib.machinery
import importlib.util
import os
import warnings
from typing import NamedTuple, Optional

import torch

from .build import LIB_PATH, MARSHAL_PATH, marshal_built_for

F32, BF16, E4M3 = 0, 1, 2
METRIC_L2, METRIC_COSINE = 0, 1
MAX_VOCAB = 1 << 19

OK = 0
E_NULL, E_SHAPE, E_DTYPE, E_DELTA, E_TOKEN, E_WORKSPACE, E_DEVICE = -1, -2, -3, -4, -5, -6, -7

EXPORTS = (
    "lantern_build_knn_workspace_bytes", "lantern_build_knn", "lantern_build_knn_metric",
    "lantern_verify", "lantern_verify_ex", "lantern_verify_divergence", "lantern_verify_greedy",
    "lantern_accept_chains", "lantern_verify_rows", "lantern_verify_greedy_rows", "lantern_accept_trees",
    "lantern_build_random", "lantern_decide_rows", "lantern_resample_selected", "lantern_verify_trees",
    "lantern_verify_trees_greedy", "lantern_verify_trees_sequential_workspace_bytes",
    "lantern_verify_trees_sequential", "lantern_probe_stream_read", "lantern_prepare", "lantern_build_knn_static",
    "lantern_rotate_axes", "lantern_append_cache", "lantern_attend_trees_workspace_bytes", "lantern_attend_trees",
    "lantern_prepare_cache", "lantern_status_string",
    "lantern_version",
)

MAX_AXES = 4
MAX_TREE = 255


class _Rotation(ctypes.Structure):
    _fields_ = [("positions", ctypes.c_void_p), ("freqs", ctypes.c_void_p), ("axes", ctypes.c_int),
                ("pairs", ctypes.c_int * MAX_AXES), ("interleaved", ctypes.c_int)]


class _Cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("dtype", ctypes.c_int), ("pages", ctypes.c_int), ("heads", ctypes.c_int), ("page_tokens", ctypes.c_int),
                ("D", ctypes.c_int)]


_lib = None
_marshal = None


class LanternError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


def load() -> ctypes.CDLL:
    """Loads the built library.  Raises if it has not been built."""
    global _lib, _marshal
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} not found: build it with `python -m paper_2410_03355_amd.build` "
            "(there is no fallback implementation)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, f32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    lib.lantern_build_knn_workspace_bytes.argtypes = [i32, i32, i32, i32]
    lib.lantern_build_knn_workspace_bytes.restype = sz
    lib.lantern_build_knn.argtypes = [vp, i32, i32, i32, i32, vp, vp, sz, vp]
    lib.lantern_build_knn.restype = i32
    lib.lantern_build_knn_metric.argtypes = [vp, i32, i32, i32, i32, i32, vp, vp, sz, vp]
    lib.lantern_build_knn_metric.restype = i32
    lib.lantern_verify.argtypes = [vp, vp, i32, i32, i32, i64, vp, vp, i32, f32, vp, vp, vp, vp]
    lib.lantern_verify.restype = i32
    lib.lantern_verify_ex.argtypes = [vp, vp, i32, i32, i32, i64, vp, vp, i32, f32, vp, vp, vp,
                                      vp, vp, vp, vp, vp, vp]
    lib.lantern_verify_ex.restype = i32
    lib.lantern_verify_divergence.argtypes = [vp, vp, i32, i32, i32, i64, vp, vp, i32, i32, f32, vp, vp, vp,
                                              vp, vp, vp, vp, vp, vp]
    lib.lantern_verify_divergence.restype = i32
    lib.lantern_verify_greedy.argtypes = [vp, i32, i32, i32, i64, vp, vp, i32, f32, vp, vp, vp, vp]
    lib.lantern_verify_greedy.restype = i32
    lib.lantern_accept_chains.argtypes = [vp, vp, i32, i32, vp, vp, vp]
    lib.lantern_accept_chains.restype = i32
    lib.lantern_verify_rows.argtypes = [vp, vp, i32, i32, i32, i64, vp, i32, vp, vp, i32, i32, f32, vp, vp, vp, vp]
    lib.lantern_verify_rows.restype = i32
    lib.lantern_verify_greedy_rows.argtypes = [vp, i32, i32, i32, i64, vp, i32, vp, vp, i32, f32, vp, vp, vp]
    lib.lantern_verify_greedy_rows.restype = i32
    lib.lantern_accept_trees.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, vp]
    lib.lantern_accept_trees.restype = i32
    lib.lantern_decide_rows.argtypes = [vp, vp, i32, i32, i32, i64, vp, i32, vp, vp, i32, i32, f32, vp, vp, vp, vp]
    lib.lantern_decide_rows.restype = i32
    lib.lantern_resample_selected.argtypes = [vp, vp, i32, i32, i32, i64, vp, i32, vp, vp, i32, i32, f32, vp, vp,
                                              i32, vp, vp]
    lib.lantern_resample_selected.restype = i32
    lib.lantern_verify_trees.argtypes = [vp, vp, i32, i32, i32, i64, vp, vp, i32, i32, vp, vp, i32, i32, f32, vp,
                                         vp, vp, vp, vp, vp]
    lib.lantern_verify_trees.restype = i32
    lib.lantern_verify_trees_greedy.argtypes = [vp, i32, i32, i32, i64, vp, vp, i32, i32, vp, vp, i32, f32, vp, vp, vp,
                                                vp, vp, vp]
    lib.lantern_verify_trees_greedy.restype = i32
    lib.lantern_verify_trees_sequential_workspace_bytes.argtypes = [i32, i32, i32]
    lib.lantern_verify_trees_sequential_workspace_bytes.restype = sz
    lib.lantern_verify_trees_sequential.argtypes = [vp, vp, i32, i32, i32, i64, vp, vp, i32, i32, vp, vp, i32, i32, f32,
                                                    vp, vp, vp, vp, vp, sz, vp]
    lib.lantern_verify_trees_sequential.restype = i32
    lib.lantern_probe_stream_read.argtypes = [vp, vp, sz, vp, vp]
    lib.lantern_probe_stream_read.restype = i32
    lib.lantern_build_random.argtypes = [i32, i32, ctypes.c_uint64, vp, vp]
    lib.lantern_build_random.restype = i32
    lib.lantern_build_knn_static.argtypes = [vp, i32, i32, i32, i32, i32, vp, vp, vp]
    lib.lantern_build_knn_static.restype = i32
    lib.lantern_prepare.argtypes = [i32, i32, i32]
    lib.lantern_prepare.restype = i32
    strides = ctypes.POINTER(i64)
    lib.lantern_rotate_axes.argtypes = [vp, strides, i32, vp, strides, i32, i32, i32, i32, ctypes.POINTER(_Rotation), i32,
                                        vp, strides, vp, strides, vp]
    lib.lantern_rotate_axes.restype = i32
    lib.lantern_append_cache.argtypes = [ctypes.POINTER(_Cache), vp, i32, vp, i32, i32, vp, strides, vp, strides, i32,
                                         ctypes.POINTER(_Rotation), vp, vp, vp, vp]
    lib.lantern_append_cache.restype = i32
    lib.lantern_attend_trees_workspace_bytes.argtypes = [i32, i32, i32, i32, ctypes.POINTER(_Cache), i32]
    lib.lantern_attend_trees_workspace_bytes.restype = sz
    lib.lantern_attend_trees.argtypes = [vp, strides, vp, strides, vp, strides, i32, i32, i32, i32, vp, ctypes.POINTER(_Cache),
                                         vp, i32, vp, f32, vp, vp, sz, vp]
    lib.lantern_attend_trees.restype = i32
    lib.lantern_prepare_cache.argtypes = [i32, ctypes.POINTER(_Cache)]
    lib.lantern_prepare_cache.restype = i32
    lib.lantern_status_string.argtypes = [i32]
    lib.lantern_status_string.restype = ctypes.c_char_p
    lib.lantern_version.argtypes = []
    lib.lantern_version.restype = i32
    _marshal = _load_marshal(lib)
    _lib = lib
    return lib


class _Declines:
    """In the place of _marshal.so: every call goes through ctypes."""

    def __getattr__(self, name):
        return lambda *args: None


def _load_marshal(lib):
    try:
        loader = importlib.machinery.ExtensionFileLoader("_marshal", MARSHAL_PATH)
        marshal = importlib.util.module_from_spec(importlib.util.spec_from_loader("_marshal", loader))
        if marshal.BUILT_FOR != marshal_built_for():     # PyTorch's C++ interface differs between its versions
            raise ImportError(f"built for {marshal.BUILT_FOR}, this is {marshal_built_for()}")
    except ImportError as e:
        warnings.warn(f"{MARSHAL_PATH} is not used ({e}): step calls take some microseconds longer on the host until it is "
                      "built with `python -m paper_2410_03355_amd.build`", RuntimeWarning, stacklevel=3)
        return _Declines()
    marshal.bind({name: ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in EXPORTS})
    return marshal


def _checked_status(got, where: str):
    """What a function of _marshal.so returned: the results, or a status that is not zero."""
    if got.__class__ is int:
        raise LanternError(got, where)
    return got


def status_string(status: int) -> str:
    return load().lantern_status_string(int(status)).decode()


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t.dtype}: float32 or bfloat16 expected")


def prepare(logits_dtype, V: int, k: int) -> None:
    """lantern_prepare: raises the LDS limits of every verification kernel for this logit dtype
    (torch.float32 / torch.bfloat16), vocabulary size and table width on the current device, so that
    later calls make no runtime call besides their launches (needed before stream capture)."""
    code = {torch.float32: F32, torch.bfloat16: BF16}[logits_dtype]
    rc = load().lantern_prepare(code, int(V), int(k))
    if rc != OK:
        raise LanternError(rc, "lantern_prepare")


def _stream_ptr(stream) -> int:
    s = torch.cuda.current_stream() if stream is None else stream
    return int(s.cuda_stream)


def _outputs(stream, device, *sizes, dtype=torch.int32, workspace: int = 0):
    """Tensors for the results of work on `stream` (None: the current one), and behind them one of `workspace` bytes if that is not 0.  Their memory
    is that stream's own: what the current stream has freed may still be read or written by work queued there, which another stream does not
    wait for.  And results, once dropped, are given away when the current stream, which may read them, has come to that place."""
    if not (sizes or workspace):
        return []
    current = None if stream is None else torch.cuda.current_stream(device)
    with contextlib.nullcontext() if current == stream else torch.cuda.stream(stream):
        made = [torch.empty(size, dtype=dtype, device=device) for size in sizes]
        room = [torch.empty(workspace, dtype=torch.uint8, device=device)] if workspace else []
    if current != stream:
        for t in made:
            t.record_stream(current)
    return made + room


def _need_cuda(*tensors):
    for t in tensors:
        if t is not None and not t.is_cuda:
            raise ValueError("all tensors must live in device memory")


def knn_workspace_bytes(cb_dtype: int, V: int, d: int, k: int) -> int:
    return int(load().lantern_build_knn_workspace_bytes(cb_dtype, V, d, k))


def build_knn(codebook: torch.Tensor, k: int, metric: str = "l2", stream=None, return_stats: bool = False,
              workspace: torch.Tensor = None, out: torch.Tensor = None):
    """lantern_build_knn on a [V, d] device tensor; returns int32 [V, k] on the device.
    With return_stats also a device int32 scalar tensor: rows ranked by the exact all-pairs pass.
    workspace (uint8, at least knn_workspace_bytes, 256-byte aligned) and out ([V, k] int32) may be
    brought by the caller, who then builds several tables without allocating in between."""
    lib = load()
    _need_cuda(codebook)
    if codebook.dim() != 2 or not codebook.is_contiguous():
        raise ValueError("codebook must be a contiguous [V, d] tensor")
    V, d = codebook.shape
    code = _dtype_code(codebook)
    nbytes = knn_workspace_bytes(code, V, d, k)
    if nbytes == 0:
        raise LanternError(E_SHAPE, "lantern_build_knn_workspace_bytes")
    if workspace is None:
        (ws,) = _outputs(stream, codebook.device, nbytes, dtype=torch.uint8) if return_stats else _outputs(stream, codebook.device, workspace=nbytes)
    else:
        _need_cuda(workspace)
        if workspace.dtype != torch.uint8 or not workspace.is_contiguous() or workspace.numel() < nbytes:
            raise ValueError("workspace must be a contiguous uint8 tensor of at least knn_workspace_bytes")
        ws = workspace
    if out is None:
        (out,) = _outputs(stream, codebook.device, (V, k))
    else:
        _need_cuda(out)
        if out.dtype != torch.int32 or tuple(out.shape) != (V, k) or not out.is_contiguous():
            raise ValueError("out must be a contiguous int32 [V, k] tensor")
    rc = lib.lantern_build_knn_metric(codebook.data_ptr(), code, V, d, k,
                                      {"l2": METRIC_L2, "cosine": METRIC_COSINE}[metric],
                                      out.data_ptr(), ws.data_ptr(), ws.numel(), _stream_ptr(stream))
    if rc != OK:
        raise LanternError(rc, "lantern_build_knn")
    if return_stats:
        return out, ws[:4].view(torch.int32)[0]
    return out


STATIC_MAX_V = 32768


def build_knn_static(codebook: torch.Tensor, k: int, out: torch.Tensor, metric: str = "l2", exact_rows=None,
                     stream=None) -> None:
    """lantern_build_knn_static: the table into the caller's `out` ([V, k] int32, device) using the
    library's static scratch; this wrapper allocates nothing either.  exact_rows: device int32
    tensor of one element, or None."""
    lib = load()
    _need_cuda(codebook, out, exact_rows)
    if codebook.dim() != 2 or not codebook.is_contiguous():
        raise ValueError("codebook must be a contiguous [V, d] tensor")
    V, d = codebook.shape
    if out.dtype != torch.int32 or tuple(out.shape) != (V, k) or not out.is_contiguous():
        raise ValueError("out must be a contiguous int32 [V, k] tensor")
    rc = lib.lantern_build_knn_static(codebook.data_ptr(), _dtype_code(codebook), V, d, k,
                                      {"l2": METRIC_L2, "cosine": METRIC_COSINE}[metric], out.data_ptr(),
                                      None if exact_rows is None else exact_rows.data_ptr(), _stream_ptr(stream))
    if rc != OK:
        raise LanternError(rc, "lantern_build_knn_static")


def _check_verify_args(target_logits, draft_logits, draft_tokens, knn, uniforms):
    _need_cuda(target_logits, draft_logits, draft_tokens, knn, uniforms)
    if target_logits.dim() != 2 or target_logits.shape != draft_logits.shape:
        raise ValueError("logits must be two [N, V] tensors of equal shape")
    if target_logits.dtype != draft_logits.dtype:
        raise TypeError("target and draft logits must share a dtype")
    if target_logits.stride(1) != 1 or draft_logits.stride(1) != 1 or \
            target_logits.stride(0) != draft_logits.stride(0):
        raise ValueError("logit rows must be dense and both tensors must share the row stride")
    N, V = target_logits.shape
    if draft_tokens.dtype != torch.int32 or knn.dtype != torch.int32 or uniforms.dtype != torch.float32:
        raise TypeError("draft_tokens and knn must be int32, uniforms float32")
    if draft_tokens.numel() != N or uniforms.numel() != 2 * N or knn.dim() != 2 or knn.shape[0] != V:
        raise ValueError("shape mismatch between logits, tokens, uniforms and the table")
    if not (draft_tokens.is_contiguous() and knn.is_contiguous() and uniforms.is_contiguous()):
        raise ValueError("draft_tokens, knn and uniforms must be contiguous")
    return N, V, int(knn.shape[1])


def _raise_if_unusable(acc, stream, where: str):
    """Checked mode: waits for the call's stream and raises E_TOKEN if any verification came back unusable."""
    (torch.cuda.current_stream(acc.device) if stream is None else stream).synchronize()
    bad = torch.nonzero(acc < 0).flatten()
    if bad.numel():
        err = LanternError(E_TOKEN, where)
        err.rows = bad.cpu().tolist()
        raise err


def verify(target_logits, draft_logits, draft_tokens, knn, delta: float, uniforms,
           out_accept=None, out_resample=None, stream=None, checked: bool = False):
    """lantern_verify; returns (accept int32[N], resample int32[N]) device tensors.
    checked: synchronise and raise LanternError(E_TOKEN) (with .rows) if a verification was unusable; by
    default the call is asynchronous and such rows carry -1 in both outputs."""
    lib = load()
    if out_accept is None and out_resample is None and stream is None:
        got = _marshal.verify(target_logits, draft_logits, draft_tokens, knn, delta, uniforms)
        if got is not None:
            _checked_status(got, "lantern_verify")
            if checked:
                _raise_if_unusable(got[0], stream, "lantern_verify")
            return got
    N, V, k = _check_verify_args(target_logits, draft_logits, draft_tokens, knn, uniforms)
    dev = target_logits.device
    made = _outputs(stream, dev, *[N for t in (out_accept, out_resample) if t is None])
    acc = made[0] if out_accept is None else out_accept
    res = made[-1] if out_resample is None else out_resample
    rc = lib.lantern_verify(target_logits.data_ptr(), draft_logits.data_ptr(),
                            _dtype_code(target_logits), N, V, target_logits.stride(0) if N > 1 else V,
                            draft_tokens.data_ptr(), knn.data_ptr(), k, float(delta),
                            uniforms.data_ptr(), acc.data_ptr(), res.data_ptr(), _stream_ptr(stream))
    if rc != OK:
        raise LanternError(rc, "lantern_verify")
    if checked:
        _raise_if_unusable(acc, stream, "lantern_verify")
    return acc, res


DIV_TVD, DIV_JSD = 0, 1


def verify_ex(target_logits, draft_logits, draft_tokens, knn, delta: float, uniforms, stream=None,
              divergence: str = "tvd"):
    """lantern_verify_ex (divergence "tvd") or lantern_verify_divergence ("jsd"); returns a dict of
    device tensors with all diagnostics."""
    lib = load()
    N, V, k = _check_verify_args(target_logits, draft_logits, draft_tokens, knn, uniforms)
    dev = target_logits.device
    acc, res, size, path = _outputs(stream, dev, N, N, N, N)
    prob, mass, g_tok = _outputs(stream, dev, N, N, N, dtype=torch.float32)
    out = {"accept": acc, "resample": res, "accept_prob": prob, "mass": mass, "g_tok": g_tok, "a_size": size, "path": path}
    common_in = (target_logits.data_ptr(), draft_logits.data_ptr(), _dtype_code(target_logits), N, V,
                 target_logits.stride(0) if N > 1 else V, draft_tokens.data_ptr(), knn.data_ptr(), k)
    common_out = (uniforms.data_ptr(), out["accept"].data_ptr(), out["resample"].data_ptr(),
                  out["accept_prob"].data_ptr(), out["mass"].data_ptr(), out["g_tok"].data_ptr(),
                  out["a_size"].data_ptr(), out["path"].data_ptr(), _stream_ptr(stream))
    if divergence == "tvd":
        rc = lib.lantern_verify_ex(*common_in, float(delta), *common_out)
    else:
        rc = lib.lantern_verify_divergence(*common_in, {"jsd": DIV_JSD}[divergence], float(delta), *common_out)
    if rc != OK:
        raise LanternError(rc, "lantern_verify_ex")
    return out


def verify_greedy(target_logits, draft_tokens, knn, delta: float, stream=None, want_path: bool = False):
    """lantern_verify_greedy; returns (accept int32[N], token int32[N]) device tensors
    (and the per-row path tensor when want_path)."""
    lib = load()
    if stream is None and not want_path:
        got = _marshal.verify_greedy(target_logits, draft_tokens, knn, delta)
        if got is not None:
            return _checked_status(got, "lantern_verify_greedy")
    _need_cuda(target_logits, draft_tokens, knn)
    if target_logits.dim() != 2 or target_logits.stride(1) != 1:
        raise ValueError("logits must be a [N, V] tensor with dense rows")
    N, V = target_logits.shape
    if draft_tokens.dtype != torch.int32 or knn.dtype != torch.int32:
        raise TypeError("draft_tokens and knn must be int32")
    if draft_tokens.numel() != N or knn.dim() != 2 or knn.shape[0] != V:
        raise ValueError("shape mismatch between logits, tokens and the table")
    if not (draft_tokens.is_contiguous() and knn.is_contiguous()):
        raise ValueError("draft_tokens and knn must be contiguous")
    dev = target_logits.device
    acc, tok, *path = _outputs(stream, dev, *[N] * (3 if want_path else 2))
    path = path[0] if want_path else None
    rc = lib.lantern_verify_greedy(target_logits.data_ptr(), _dtype_code(target_logits), N, V,
                                   target_logits.stride(0) if N > 1 else V, draft_tokens.data_ptr(),
                                   knn.data_ptr(), int(knn.shape[1]), float(delta), acc.data_ptr(),
                                   tok.data_ptr(), path.data_ptr() if want_path else None,
                                   _stream_ptr(stream))
    if rc != OK:
        raise LanternError(rc, "lantern_verify_greedy")
    return (acc, tok, path) if want_path else (acc, tok)


def accept_chains(accept, resample, L: int, stream=None):
    """lantern_accept_chains; accept / resample are int32 device tensors of B*L rows.
    Returns (kept int32[B], next_token int32[B])."""
    lib = load()
    if stream is None:
        got = _marshal.accept_chains(accept, resample, L)
        if got is not None:
            return _checked_status(got, "lantern_accept_chains")
    _need_cuda(accept, resample)
    if accept.dtype != torch.int32 or resample.dtype != torch.int32:
        raise TypeError("accept and resample must be int32")
    if accept.numel() != resample.numel() or L < 1 or accept.numel() % L:
        raise ValueError("accept and resample must hold B*L rows")
    if not (accept.is_contiguous() and resample.is_contiguous()):
        raise ValueError("accept and resample must be contiguous")
    B = accept.numel() // L
    kept, nxt = _outputs(stream, accept.device, B, B)
    rc = lib.lantern_accept_chains(accept.data_ptr(), resample.data_ptr(), B, int(L), kept.data_ptr(),
                                   nxt.data_ptr(), _stream_ptr(stream))
    if rc != OK:
        raise LanternError(rc, "lantern_accept_chains")
    return kept, nxt


def _check_row_index(row_index, N):
    if row_index.dtype != torch.int32 or not row_index.is_contiguous() or row_index.numel() != N:
        raise ValueError("row_index must be a contiguous int32 tensor with one entry per verification")


def verify_rows(target_logits, draft_logits, row_index, draft_tokens, knn, delta: float, uniforms,
                divergence: str = "tvd", stream=None):
    """lantern_verify_rows: verification i reads logit row row_index[i].
    Returns (accept int32[N], resample int32[N]) device tensors."""
    lib = load()
    if stream is None:
        got = _marshal.verify_rows(target_logits, draft_logits, row_index, draft_tokens, knn, delta, uniforms, divergence)
        if got is not None:
            return _checked_status(got, "lantern_verify_rows")
    _need_cuda(target_logits, draft_logits, row_index, draft_tokens, knn, uniforms)
    if target_logits.dim() != 2 or target_logits.shape != draft_logits.shape or \
            target_logits.dtype != draft_logits.dtype:
        raise ValueError("logits must be two [R, V] tensors of equal shape and dtype")
    if target_logits.stride(1) != 1 or draft_logits.stride(1) != 1 or \
            target_logits.stride(0) != draft_logits.stride(0):
        raise ValueError("logit rows must be dense and both tensors must share the row stride")
    R, V = target_logits.shape
    N = draft_tokens.numel()
    _check_row_index(row_index, N)
    if draft_tokens.dtype != torch.int32 or knn.dtype != torch.int32 or uniforms.dtype != torch.float32:
        raise TypeError("draft_tokens and knn must be int32, uniforms float32")
    if uniforms.numel() != 2 * N or knn.dim() != 2 or knn.shape[0] != V:
        raise ValueError("shape mismatch between tokens, uniforms and the table")
    if not (draft_tokens.is_contiguous() and knn.is_contiguous() and uniforms.is_contiguous()):
        raise ValueError("draft_tokens, knn and uniforms must be contiguous")
    dev = target_logits.device
    acc, res = _outputs(stream, dev, N, N)
    rc = lib.lantern_verify_rows(target_logits.data_ptr(), draft_logits.data_ptr(), _dtype_code(target_logits),
                                 R, V, target_logits.stride(0) if R > 1 else V, row_index.data_ptr(), N,
                                 draft_tokens.data_ptr(), knn.data_ptr(), int(knn.shape[1]),
                                 {"tvd": DIV_TVD, "jsd": DIV_JSD}[divergence], float(delta),
                                 uniforms.data_ptr(), acc.data_ptr(), res.data_ptr(), _stream_ptr(stream))
    if rc != OK:
        raise LanternError(rc, "lantern_verify_rows")
    return acc, res


def verify_greedy_rows(target_logits, row_index, draft_tokens, knn, delta: float, stream=None):
    """lantern_verify_greedy_rows; returns (accept int32[N], token int32[N]) device tensors."""
    lib = load()
    if stream is None:
        got = _marshal.verify_greedy_rows(target_logits, row_index, draft_tokens, knn, delta)
        if got is not None:
            return _checked_status(got, "lantern_verify_greedy_rows")
    _need_cuda(target_logits, row_index, draft_tokens, knn)
    if target_logits.dim() != 2 or target_logits.stride(1) != 1:
        raise ValueError("logits must be a [R, V] tensor with dense rows")
    R, V = target_logits.shape
    N = draft_tokens.numel()
    _check_row_index(row_index, N)
    if draft_tokens.dtype != torch.int32 or knn.dtype != torch.int32:
        raise TypeError("draft_tokens and knn must be int32")
    if knn.dim() != 2 or knn.shape[0] != V or not (draft_tokens.is_contiguous() and knn.is_contiguous()):
        raise ValueError("the table must be a contiguous [V, k] tensor, the tokens contiguous")
    dev = target_logits.device
    acc, tok = _outputs(stream, dev, N, N)
    rc = lib.lantern_verify_greedy_rows(target_logits.data_ptr(), _dtype_code(target_logits), R, V,
                                        target_logits.stride(0) if R > 1 else V, row_index.data_ptr(), N,
                                        draft_tokens.data_ptr(), knn.data_ptr(), int(knn.shape[1]), float(delta),
                                        acc.data_ptr(), tok.data_ptr(), _stream_ptr(stream))
    if rc != OK:
        raise LanternError(rc, "lantern_verify_greedy_rows")
    return acc, tok


def accept_trees(accept, resample, parent, M: int, stream=None):
    """lantern_accept_trees; accept / resample / parent are int32 device tensors of B*M rows.
    Returns (len int32[B], path int32[B, M], next_token int32[B])."""
    lib = load()
    if stream is None:
        got = _marshal.accept_trees(accept, resample, parent, M)
        if got is not None:
            return _checked_status(got, "lantern_accept_trees")
    given = [t for t in (accept, resample, parent) if t is not None]
    _need_cuda(*given)
    for t in given:
        if t.dtype != torch.int32 or not t.is_contiguous():
            raise TypeError("accept, resample and parent must be contiguous int32 tensors")
    if any(t.numel() != accept.numel() for t in given) or M < 1 or accept.numel() % M:
        raise ValueError("accept, resample and parent must hold B*M rows")
    B = accept.numel() // M
    dev = accept.device
    n, path, nxt = _outputs(stream, dev, B, (B, M), B)
    rc = lib.lantern_accept_trees(accept.data_ptr(), None if resample is None else resample.data_ptr(),
                                  parent.data_ptr(), B, int(M),
                                  n.data_ptr(), path.data_ptr(), nxt.data_ptr(), _stream_ptr(stream))
    if rc != OK:
        raise LanternError(rc, "lantern_accept_trees")
    return n, path, nxt


RANDOM_MAX_K = 4096


def build_random(V: int, k: int, seed: int, device="cuda", stream=None):
    """lantern_build_random; returns the [V, k] int32 table on the device."""
    lib = load()
    (out,) = _outputs(stream, device, (V, k))
    rc = lib.lantern_build_random(int(V), int(k), int(seed) & 0xFFFFFFFFFFFFFFFF, out.data_ptr(),
                                  _stream_ptr(stream))
    if rc != OK:
        raise LanternError(rc, "lantern_build_random")
    return out


def _rows_args(target_logits, draft_logits, row_index, draft_tokens, knn, uniforms):
    _need_cuda(target_logits, draft_logits, draft_tokens, knn, uniforms)
    if target_logits.dim() != 2 or target_logits.shape != draft_logits.shape or \
            target_logits.dtype != draft_logits.dtype:
        raise ValueError("logits must be two [R, V] tensors of equal shape and dtype")
    if target_logits.stride(1) != 1 or draft_logits.stride(1) != 1 or \
            target_logits.stride(0) != draft_logits.stride(0):
        raise ValueError("logit rows must be dense and both tensors must share the row stride")
    R, V = target_logits.shape
    N = draft_tokens.numel()
    if row_index is not None:
        _need_cuda(row_index)
        _check_row_index(row_index, N)
    elif R != N:
        raise ValueError("without row_index there must be one logit row per verification")
    if draft_tokens.dtype != torch.int32 or knn.dtype != torch.int32 or uniforms.dtype != torch.float32:
        raise TypeError("draft_tokens and knn must be int32, uniforms float32")
    if uniforms.numel() != 2 * N or knn.dim() != 2 or knn.shape[0] != V:
        raise ValueError("shape mismatch between tokens, uniforms and the table")
    if not (draft_tokens.is_contiguous() and knn.is_contiguous() and uniforms.is_contiguous()):
        raise ValueError("draft_tokens, knn and uniforms must be contiguous")
    return R, V, N, target_logits.stride(0) if R > 1 else V


def decide_rows(target_logits, draft_logits, row_index, draft_tokens, knn, delta: float, uniforms,
                divergence: str = "tvd", stream=None, want_path: bool = False):
    """lantern_decide_rows; returns accept int32[N] (device), and the per-row path tensor when want_path."""
    lib = load()
    if stream is None and not want_path:
        got = _marshal.decide_rows(target_logits, draft_logits, row_index, draft_tokens, knn, delta, uniforms, divergence)
        if got is not None:
            return _checked_status(got, "lantern_decide_rows")
    R, V, N, stride = _rows_args(target_logits, draft_logits, row_index, draft_tokens, knn, uniforms)
    acc, *path = _outputs(stream, target_logits.device, *[N] * (2 if want_path else 1))
    path = path[0] if want_path else None
    rc = lib.lantern_decide_rows(target_logits.data_ptr(), draft_logits.data_ptr(), _dtype_code(target_logits),
                                 R, V, stride, None if row_index is None else row_index.data_ptr(), N,
                                 draft_tokens.data_ptr(), knn.data_ptr(), int(knn.shape[1]),
                                 {"tvd": DIV_TVD, "jsd": DIV_JSD}[divergence], float(delta),
                                 uniforms.data_ptr(), acc.data_ptr(),
                                 path.data_ptr() if want_path else None, _stream_ptr(stream))
    if rc != OK:
        raise LanternError(rc, "lantern_decide_rows")
    return (acc, path) if want_path else acc


def resample_selected(target_logits, draft_logits, row_index, draft_tokens, knn, delta: float, uniforms,
                      select, divergence: str = "tvd", stream=None):
    """lantern_resample_selected; returns token int32[len(select)] (device)."""
    lib = load()
    R, V, N, stride = _rows_args(target_logits, draft_logits, row_index, draft_tokens, knn, uniforms)
    _need_cuda(select)
    if select.dtype != torch.int32 or not select.is_contiguous():
        raise TypeError("select must be a contiguous int32 tensor")
    (out,) = _outputs(stream, target_logits.device, select.numel())
    rc = lib.lantern_resample_selected(target_logits.data_ptr(), draft_logits.data_ptr(),
                                       _dtype_code(target_logits), R, V, stride,
                                       None if row_index is None else row_index.data_ptr(), N,
                                       draft_tokens.data_ptr(), knn.data_ptr(), int(knn.shape[1]),
                                       {"tvd": DIV_TVD, "jsd": DIV_JSD}[divergence], float(delta),
                                       uniforms.data_ptr(), select.data_ptr(), select.numel(), out.data_ptr(),
                                       _stream_ptr(stream))
    if rc != OK:
        raise LanternError(rc, "lantern_resample_selected")
    return out


def verify_trees(target_logits, draft_logits, row_index, parent, M: int, draft_tokens, knn, delta: float,
                 uniforms, divergence: str = "tvd", stream=None):
    """lantern_verify_trees; returns (accept int32[B*M], len int32[B], path int32[B, M], next int32[B])."""
    lib = load()
    if stream is None:
        got = _marshal.verify_trees(target_logits, draft_logits, row_index, parent, M, draft_tokens, knn, delta, uniforms, divergence)
        if got is not None:
            return _checked_status(got, "lantern_verify_trees")
    R, V, N, stride = _rows_args(target_logits, draft_logits, row_index, draft_tokens, knn, uniforms)
    _need_cuda(parent)
    if parent.dtype != torch.int32 or not parent.is_contiguous() or parent.numel() != N or M < 1 or N % M:
        raise ValueError("parent must be a contiguous int32 tensor of B*M entries")
    B = N // M
    dev = target_logits.device
    acc, n, path, nxt = _outputs(stream, dev, N, B, (B, M), B)
    rc = lib.lantern_verify_trees(target_logits.data_ptr(), draft_logits.data_ptr(), _dtype_code(target_logits),
                                  R, V, stride, None if row_index is None else row_index.data_ptr(),
                                  parent.data_ptr(), B, int(M),
                                  draft_tokens.data_ptr(), knn.data_ptr(), int(knn.shape[1]),
                                  {"tvd": DIV_TVD, "jsd": DIV_JSD}[divergence], float(delta), uniforms.data_ptr(),
                                  acc.data_ptr(), n.data_ptr(), path.data_ptr(), nxt.data_ptr(), _stream_ptr(stream))
    if rc != OK:
        raise LanternError(rc, "lantern_verify_trees")
    return acc, n, path, nxt


def verify_trees_sequential(target_logits, draft_logits, row_index, parent, M: int, draft_tokens, knn, delta: float,
                            uniforms, divergence: str = "tvd", workspace=None, stream=None):
    """lantern_verify_trees_sequential; returns (len int32[B], path int32[B, M], next int32[B]).
    workspace: a uint8 device tensor of at least trees_sequential_workspace_bytes(B, M, V) bytes, or None
    to allocate one."""
    lib = load()
    if stream is None:
        got = _marshal.verify_trees_sequential(target_logits, draft_logits, row_index, parent, M, draft_tokens, knn, delta, uniforms, divergence,
                                               workspace)
        if got is not None:
            return _checked_status(got, "lantern_verify_trees_sequential")
    R, V, N, stride = _rows_args(target_logits, draft_logits, row_index, draft_tokens, knn, uniforms)
    _need_cuda(parent)
    if parent.dtype != torch.int32 or not parent.is_contiguous() or parent.numel() != N or M < 1 or N % M:
        raise ValueError("parent must be a contiguous int32 tensor of B*M entries")
    B = N // M
    dev = target_logits.device
    need = int(lib.lantern_verify_trees_sequential_workspace_bytes(B, int(M), V))
    _need_cuda(workspace)
    n, path, nxt, *room = _outputs(stream, dev, B, (B, M), B, workspace=max(need, 256) if workspace is None else 0)
    workspace = room[0] if room else workspace
    rc = lib.lantern_verify_trees_sequential(target_logits.data_ptr(), draft_logits.data_ptr(),
                                             _dtype_code(target_logits), R, V, stride,
                                             None if row_index is None else row_index.data_ptr(),
                                             parent.data_ptr(), B, int(M), draft_tokens.data_ptr(), knn.data_ptr(),
                                             int(knn.shape[1]), {"tvd": DIV_TVD, "jsd": DIV_JSD}[divergence],
                                             float(delta), uniforms.data_ptr(), n.data_ptr(), path.data_ptr(),
                                             nxt.data_ptr(), workspace.data_ptr(),
                                             workspace.numel() * workspace.element_size(), _stream_ptr(stream))
    if rc != OK:
        raise LanternError(rc, "lantern_verify_trees_sequential")
    return n, path, nxt


def trees_sequential_workspace_bytes(B: int, M: int, V: int) -> int:
    return int(load().lantern_verify_trees_sequential_workspace_bytes(int(B), int(M), int(V)))


def verify_trees_greedy(target_logits, row_index, parent, M: int, draft_tokens, knn, delta: float, stream=None):
    """lantern_verify_trees_greedy; returns (accept int32[B*M], token int32[B*M], len int32[B],
    path int32[B, M], next int32[B])."""
    lib = load()
    if stream is None:
        got = _marshal.verify_trees_greedy(target_logits, row_index, parent, M, draft_tokens, knn, delta)
        if got is not None:
            return _checked_status(got, "lantern_verify_trees_greedy")
    given = [t for t in (target_logits, row_index, parent, draft_tokens, knn) if t is not None]
    _need_cuda(*given)
    if target_logits.dim() != 2 or target_logits.stride(1) != 1:
        raise ValueError("logits must be a [R, V] tensor with dense rows")
    R, V = target_logits.shape
    N = draft_tokens.numel()
    if row_index is not None:
        _check_row_index(row_index, N)
    elif R != N:
        raise ValueError("without row_index there must be one logit row per candidate")
    for t in (parent, draft_tokens, knn):
        if t.dtype != torch.int32 or not t.is_contiguous():
            raise TypeError("parent, draft_tokens and knn must be contiguous int32 tensors")
    if parent.numel() != N or M < 1 or N % M or knn.dim() != 2 or knn.shape[0] != V:
        raise ValueError("shape mismatch between parent, tokens and the table")
    B = N // M
    dev = target_logits.device
    acc, tok, n, path, nxt = _outputs(stream, dev, N, N, B, (B, M), B)
    rc = lib.lantern_verify_trees_greedy(target_logits.data_ptr(), _dtype_code(target_logits), R, V,
                                         target_logits.stride(0) if R > 1 else V,
                                         None if row_index is None else row_index.data_ptr(), parent.data_ptr(), B,
                                         int(M), draft_tokens.data_ptr(), knn.data_ptr(), int(knn.shape[1]),
                                         float(delta), acc.data_ptr(), tok.data_ptr(), n.data_ptr(), path.data_ptr(),
                                         nxt.data_ptr(), _stream_ptr(stream))
    if rc != OK:
        raise LanternError(rc, "lantern_verify_trees_greedy")
    return acc, tok, n, path, nxt


class Cache(NamedTuple):
    """Paged cache of one layer's keys and values (lantern_cache): k [pages, heads, page_tokens, D] and
    v [pages, heads, D, page_tokens], bfloat16, or float8_e4m3fn with k_scale and v_scale [pages, heads] float32.
    The calls take any tuple of these four."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: Optional[torch.Tensor] = None
    v_scale: Optional[torch.Tensor] = None


def make_cache(pages: int, heads: int, page_tokens: int, D: int, dtype=torch.float8_e4m3fn, device="cuda") -> Cache:
    """An empty cache (zeros, scales of one)."""
    if dtype not in (torch.bfloat16, torch.float8_e4m3fn):
        raise TypeError("a cache is bfloat16 or float8_e4m3fn")
    if page_tokens not in (16, 32, 64, 128) or D not in (32, 64, 96, 128) or pages < 1 or heads < 1:
        raise ValueError("page_tokens must be 16, 32, 64 or 128, D 32, 64, 96 or 128, pages and heads positive")
    k = torch.zeros((pages, heads, page_tokens, D), dtype=dtype, device=device)
    v = torch.zeros((pages, heads, D, page_tokens), dtype=dtype, device=device)
    if dtype == torch.bfloat16:
        return Cache(k, v)
    return Cache(k, v, torch.ones((pages, heads), device=device), torch.ones((pages, heads), device=device))


def _need_here(stream, *tensors):
    """Device tensors, all on the current device: the kernels are launched there."""
    _need_cuda(*tensors)
    here = torch.cuda.current_device()
    if any(t is not None and t.device.index != here for t in tensors) or (stream is not None and stream.device.index != here):
        raise ValueError("all tensors and the stream must belong to the current device")


def _fits(*sizes):
    """Sizes that the library takes as 32-bit integers: ctypes would cut them off."""
    if any(ctypes.c_int(n).value != n for n in sizes):
        raise ValueError("sizes must fit 32 bits")


def _strides(*values):
    return (ctypes.c_int64 * len(values))(*values)


def _cache_args(cache):
    """(lantern_cache, its tensors) of a cache's tensors."""
    k, v, k_scale, v_scale = cache
    if k.dim() != 4 or v.dim() != 4 or not (k.is_contiguous() and v.is_contiguous()):
        raise ValueError("the cache must be two contiguous tensors, [pages, heads, page_tokens, D] and [pages, heads, D, page_tokens]")
    pages, heads, page_tokens, D = k.shape
    _fits(*k.shape)
    if tuple(v.shape) != (pages, heads, D, page_tokens) or k.dtype != v.dtype:
        raise ValueError("the cache's keys and values must have the same sizes and dtype")
    scales = ()
    if k.dtype == torch.float8_e4m3fn:
        scales = (k_scale, v_scale)
        for s in scales:
            if s is None or s.dtype != torch.float32 or tuple(s.shape) != (pages, heads) or not s.is_contiguous():
                raise ValueError("an 8-bit cache needs k_scale and v_scale, contiguous float32 [pages, heads]")
    elif k.dtype != torch.bfloat16:
        raise TypeError("a cache is bfloat16 or float8_e4m3fn")
    c = _Cache(k.data_ptr(), v.data_ptr(), scales[0].data_ptr() if scales else None, scales[1].data_ptr() if scales else None,
               E4M3 if scales else BF16, pages, heads, page_tokens, D)
    return c, (k, v, *scales)


def _table_args(table, lengths, B):
    if table.dtype != torch.int32 or lengths.dtype != torch.int32:
        raise TypeError("table and lengths must be int32")
    if table.dim() != 2 or table.shape[0] != B or table.shape[1] < 1 or lengths.numel() != B or \
            not (table.is_contiguous() and lengths.is_contiguous()):
        raise ValueError("table must be contiguous [B, pages of a sequence], lengths contiguous [B]")
    _fits(*table.shape)


def _rotation_args(positions, freqs, sections, interleaved, rows: int):
    sections = tuple(int(n) for n in sections)
    _fits(*sections)
    if positions.dtype != torch.int32 or freqs.dtype != torch.float32:
        raise TypeError("positions must be int32, freqs float32")
    if not 1 <= len(sections) <= MAX_AXES or positions.numel() != rows * len(sections) or freqs.numel() != sum(sections) or \
            not (positions.is_contiguous() and freqs.is_contiguous()):
        raise ValueError("positions must be contiguous with one entry per row and axis, freqs with one per pair of the sections")
    return _Rotation(positions.data_ptr(), freqs.data_ptr(), len(sections), (ctypes.c_int * MAX_AXES)(*sections), int(bool(interleaved)))


def _wants_gradients(*tensors) -> bool:
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


def _no_tangents(*tensors):
    if any(t is not None and torch.autograd.forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise ValueError("forward-mode derivatives are not formed here: a tangent would be lost")


def _nothing_recorded(*tensors):
    """Where there is no derivative of either mode: none of these may ask for one."""
    _no_tangents(*tensors)
    if _wants_gradients(*tensors):
        raise ValueError("there is no backward pass here: call it under torch.no_grad()")


def _written(*tensors):
    """Tensors of the caller's that a call has written: autograd, which may have saved them, sees a new version."""
    torch.autograd.graph.increment_version([t for t in tensors if not t.is_inference()])


class _Turned(torch.autograd.Function):
    """rotate_axes where gradients are wanted: turning is orthogonal, so theirs is to turn back."""

    @staticmethod
    def forward(ctx, q, k, positions, freqs, sections, interleaved, inverse):
        ctx.save_for_backward(positions, freqs)
        ctx.how = sections, interleaved, inverse
        return rotate_axes(q, k, positions, freqs, sections, interleaved, inverse)

    @staticmethod
    def backward(ctx, *grads):
        sections, interleaved, inverse = ctx.how
        grads = [g if g is None or g.shape[2] == 1 or g.stride(2) == 1 else g.contiguous() for g in grads]
        return (*rotate_axes(*grads, *ctx.saved_tensors, sections, interleaved, not inverse), None, None, None, None, None)


def rotate_axes(q, k, positions, freqs, sections, interleaved: bool = False, inverse: bool = False, out=None, stream=None):
    """lantern_rotate_axes: q [N, heads, D] and k [N, heads, D] (or None) turned by positions [N, axes]; sections: pairs of
    each axis, freqs [their sum].  Returns (q, k) turned, new tensors or those of `out` (a pair, which may be q and k
    themselves).  inverse turns back, which is the gradient: it takes the outputs' gradients to the inputs'.  Where autograd
    records q or k that is done in their backward pass (with out or stream such a call is refused; freqs have no gradient, and there are no
    forward-mode derivatives: tangents are refused)."""
    lib = load()
    if out is None and stream is None:
        got = _marshal.rotate_axes(q, k, positions, freqs, sections, interleaved, inverse)
        if got is not None:
            return _checked_status(got, "lantern_rotate_axes")
    ts = [t for t in (q, k) if t is not None]
    for t in ts:
        if t.dim() != 3 or t.shape[0] != q.shape[0] or t.shape[2] != q.shape[2] or t.dtype != q.dtype or (t.shape[2] > 1 and t.stride(2) != 1):
            raise ValueError("q and k must be [N, heads, D] of the same N, D and dtype, with dense heads")
        _fits(*t.shape)
    recorded = (*ts, freqs, *(() if out is None else out))
    _no_tangents(*recorded)
    if _wants_gradients(*recorded):
        if out is not None or stream is not None or freqs.requires_grad:
            raise ValueError("gradients are recorded without out and stream, and freqs have none")
        return _Turned.apply(q, k, positions, freqs, sections, interleaved, inverse)
    _need_here(stream, *ts, positions, freqs)
    N, _, D = q.shape
    code = _dtype_code(q)
    rot = _rotation_args(positions, freqs, sections, interleaved, N)
    if out is None:
        outs = _outputs(stream, q.device, *[t.shape for t in ts], dtype=q.dtype)
    else:
        outs = [t for t in out if t is not None]
        if len(outs) != len(ts) or any(o.shape != t.shape or o.dtype != t.dtype or (D > 1 and o.stride(2) != 1) for o, t in zip(outs, ts)):
            raise ValueError("out must hold tensors like q and k, with dense heads")
        _need_here(stream, *outs)
    has_k = k is not None
    rc = lib.lantern_rotate_axes(q.data_ptr(), _strides(*q.stride()[:2]), q.shape[1], k.data_ptr() if has_k else None,
                                 _strides(*k.stride()[:2]) if has_k else None, k.shape[1] if has_k else 0, code, N, D,
                                 ctypes.byref(rot), int(bool(inverse)), outs[0].data_ptr(), _strides(*outs[0].stride()[:2]),
                                 outs[1].data_ptr() if has_k else None, _strides(*outs[1].stride()[:2]) if has_k else None,
                                 _stream_ptr(stream))
    if rc != OK:
        raise LanternError(rc, "lantern_rotate_axes")
    if out is not None:
        _written(*outs)
    return outs[0], outs[1] if has_k else None


def _rows_of_cache(cache: _Cache, k, v):
    if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.shape[2] != cache.heads or k.shape[3] != cache.D or \
            k.stride(3) != 1 or v.stride(3) != 1:
        raise ValueError("k and v must be [B, rows, heads, D] of the cache's heads and D, of one dtype, with dense heads")
    _fits(*k.shape)


def append_cache(cache, table, lengths, k, v, positions=None, freqs=None, sections=None, interleaved: bool = False,
                 path=None, count=None, stream=None):
    """lantern_append_cache: rows of k and v [B, T, heads, D] into the pages of table [B, width] from lengths [B] on, the keys
    turned by positions [B, T, axes] if given.  Which rows: path [B, T-1] and count [B] as verify_trees returns them (row 0,
    then the accepted candidates), or the first count [B], or all.  Returns the new lengths int32[B] (-2: left as it was)."""
    lib = load()
    if stream is None:
        got = _marshal.append_cache(cache, table, lengths, k, v, positions, freqs, sections, interleaved, path, count)
        if got is not None:
            return _checked_status(got, "lantern_append_cache")
    _nothing_recorded(k, v, freqs, *cache)
    c, parts = _cache_args(cache)
    _rows_of_cache(c, k, v)
    B, T = k.shape[:2]
    _table_args(table, lengths, B)
    rot = None
    if positions is not None:
        if freqs is None or sections is None:
            raise ValueError("positions come with freqs and sections")
        rot = _rotation_args(positions, freqs, sections, interleaved, B * T)
    for t, n in ((path, B * (T - 1)), (count, B)):
        if t is not None and (t.dtype != torch.int32 or t.numel() != n or not t.is_contiguous()):
            raise ValueError("path must be a contiguous int32 [B, T-1], count a contiguous int32 [B]")
    if path is not None and (count is None or T < 2):
        raise ValueError("path comes with count, and with rows for its candidates")
    _need_here(stream, *parts, table, lengths, k, v, positions, freqs, path, count)
    (out,) = _outputs(stream, k.device, B)
    rc = lib.lantern_append_cache(ctypes.byref(c), table.data_ptr(), table.shape[1], lengths.data_ptr(), B, T, k.data_ptr(),
                                  _strides(*k.stride()[:3]), v.data_ptr(), _strides(*v.stride()[:3]), _dtype_code(k),
                                  None if rot is None else ctypes.byref(rot), None if path is None else path.data_ptr(),
                                  None if count is None else count.data_ptr(), out.data_ptr(), _stream_ptr(stream))
    if rc != OK:
        raise LanternError(rc, "lantern_append_cache")
    _written(*parts)
    return out


def attend_trees_workspace_bytes(dtype, B: int, M: int, q_heads: int, cache, width: int) -> int:
    """Bytes of workspace attend_trees needs for trees of M candidates and a table of `width` pages (0: none)."""
    code = {torch.float32: F32, torch.bfloat16: BF16}[dtype]
    sizes = int(B), int(M), int(q_heads), int(width)
    _fits(*sizes)
    return int(load().lantern_attend_trees_workspace_bytes(code, *sizes[:3], ctypes.byref(_cache_args(cache)[0]), sizes[3]))


def attend_trees(q, k, v, parent, cache, table, lengths, scale=None, workspace=None, stream=None):
    """lantern_attend_trees: q [B, 1 + M, heads, D] and the rows' own k, v [B, 1 + M, key heads, D] over the cache and the
    tree of parent int32[B*M] (None: every row follows the one before it).  scale: D ** -0.5 unless given.  workspace: a
    uint8 tensor of at least attend_trees_workspace_bytes, or None to allocate one.  Returns out [B, 1 + M, heads, D]."""
    lib = load()
    if stream is None:
        got = _marshal.attend_trees(q, k, v, parent, cache, table, lengths, scale, workspace)
        if got is not None:
            return _checked_status(got, "lantern_attend_trees")
    _nothing_recorded(q, k, v, *cache)
    c, parts = _cache_args(cache)
    _rows_of_cache(c, k, v)
    B, T = k.shape[:2]
    if q.dim() != 4 or q.shape[:2] != k.shape[:2] or q.shape[3] != c.D or q.dtype != k.dtype or q.stride(3) != 1:
        raise ValueError("q must be [B, rows, heads, D] like k and v, with dense heads")
    _fits(*q.shape)
    _table_args(table, lengths, B)
    if parent is not None and (parent.dtype != torch.int32 or parent.numel() != B * (T - 1) or not parent.is_contiguous()):
        raise ValueError("parent must be a contiguous int32 tensor of B*M entries")
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    _need_here(stream, *parts, table, lengths, q, k, v, parent, workspace)
    code, Hq, width = _dtype_code(q), q.shape[2], table.shape[1]
    need = int(lib.lantern_attend_trees_workspace_bytes(code, B, T - 1, Hq, ctypes.byref(c), width))
    out, *room = _outputs(stream, q.device, (B, T, Hq, c.D), dtype=q.dtype, workspace=need if workspace is None else 0)
    workspace = room[0] if room else workspace
    rc = lib.lantern_attend_trees(q.data_ptr(), _strides(*q.stride()[:3]), k.data_ptr(), _strides(*k.stride()[:3]), v.data_ptr(),
                                  _strides(*v.stride()[:3]), code, B, T - 1, Hq, None if parent is None else parent.data_ptr(),
                                  ctypes.byref(c), table.data_ptr(), width, lengths.data_ptr(),
                                  c.D ** -0.5 if scale is None else float(scale), out.data_ptr(),
                                  None if workspace is None else workspace.data_ptr(),
                                  0 if workspace is None else workspace.numel() * workspace.element_size(), _stream_ptr(stream))
    if rc != OK:
        raise LanternError(rc, "lantern_attend_trees")
    return out


def prepare_cache(dtype, cache) -> None:
    """lantern_prepare_cache: kernels and LDS limits of the three calls above for this dtype and cache, before a capture."""
    rc = load().lantern_prepare_cache({torch.float32: F32, torch.bfloat16: BF16}[dtype], ctypes.byref(_cache_args(cache)[0]))
    if rc != OK:
        raise LanternError(rc, "lantern_prepare_cache")
