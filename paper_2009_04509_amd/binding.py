"""ctypes binding of libpointid (include/pointid.h), argument marshalling only.

Each function carries the name of the C entry point it calls.  Tensors are
torch tensors on the handle's device; the binding checks dtype, shape and
contiguity, passes raw device pointers and the current HIP stream, and raises
``PointIdError`` on a non-OK status.  Every step of the computation runs in the
library's HIP kernels; if the library is not built this module fails to import.
"""

from __future__ import annotations

import ctypes
import os
from typing import NamedTuple

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
# POINTID_LIB selects another build of the same library (the sanitized host
# builds, libpointid_asan.so / libpointid_tsan.so, for checking runs)
LIB_PATH = os.environ.get("POINTID_LIB") or os.path.join(_PKG, "libpointid.so")

POINTID_OK = 0
POINTID_EINVAL = -1
POINTID_ENOMEM = -2
POINTID_EHIP = -3
POINTID_ENODEV = -4
POINTID_EUNSUPPORTED = -5
POINTID_EIO = -6
POINTID_FP32 = 0
POINTID_BF16 = 1
POINTID_FP16 = 2
POINTID_FP8 = 3
MAX_PLANES = 64
ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3, "sigmoid": 4}

_STATUS = {0: "OK", -1: "EINVAL", -2: "ENOMEM", -3: "EHIP", -4: "ENODEV", -5: "EUNSUPPORTED",
           -6: "EIO"}
_WEIGHT_FIELDS = ("conv_w", "conv_b", "fc1_w", "fc1_b", "fc2_w", "fc2_b",
                  "cls_w", "cls_b", "mic_w", "mic_b")
_WEIGHT_SIZES = {"conv_w": 48 * 25, "conv_b": 48, "fc1_w": 92928 * 128, "fc1_b": 128,
                 "fc2_w": 128 * 32, "fc2_b": 32, "cls_w": 32 * 3, "cls_b": 3,
                 "mic_w": 32, "mic_b": 1}


class PointIdError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_STATUS.get(status, status)}: {message}")
        self.status = status


class _Weights(ctypes.Structure):
    _fields_ = [(name, ctypes.POINTER(ctypes.c_float)) for name in _WEIGHT_FIELDS]


class _Plane(ctypes.Structure):
    _fields_ = [("image", ctypes.c_void_p), ("n_wires", ctypes.c_int32),
                ("n_ticks", ctypes.c_int32)]


class _Request(ctypes.Structure):
    _fields_ = [("hits", ctypes.c_void_p), ("n_hits", ctypes.c_int64),
                ("plane", ctypes.c_int32), ("scores", ctypes.c_void_p)]


class _Matrix(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("ld", ctypes.c_int64)]


class _Packed(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("exponents", ctypes.c_void_p)]


class _Drop(ctypes.Structure):
    _fields_ = [("p", ctypes.c_double), ("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64),
                ("step", ctypes.c_void_p)]


class _NormOf(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("eps", ctypes.c_float), ("weight", ctypes.c_void_p),
                ("bias", ctypes.c_void_p)]


class _Block(ctypes.Structure):
    """pointid_block, its members' members one after another (they stand so)"""
    _fields_ = _Matrix._fields_ + _NormOf._fields_ + [("gate", ctypes.c_void_p), ("scale", ctypes.c_float)] + \
        _Drop._fields_


class _NormGrads(ctypes.Structure):
    """pointid_norm_grads, likewise"""
    _fields_ = [("dx", ctypes.c_void_p), ("ld_dx", ctypes.c_int64), ("dout", ctypes.c_void_p),
                ("ld_dout", ctypes.c_int64)] + [(name, ctypes.c_void_p) for name in (
                    "dweight", "dbias", "dblock_weight", "dblock_bias", "dgate")]


class _Kept(ctypes.Structure):
    _fields_ = [("full", _Matrix), ("packed", _Packed)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is not built; run `python -m paper_2009_04509_amd.build` "
            "(or __graft_entry__.build()) first")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, u64, cint = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_int
    mat, kept = ctypes.POINTER(_Matrix), ctypes.POINTER(_Kept)
    sig = {
        "pointid_create": (cint, [ctypes.POINTER(_Weights), cint, cint, ctypes.POINTER(vp)]),
        "pointid_destroy": (cint, [vp]),
        "pointid_trim": (cint, [vp, ctypes.c_uint64, ctypes.POINTER(ctypes.c_uint64)]),
        "pointid_precision": (cint, [vp]),
        "pointid_classify": (cint, [vp, vp, i32, i32, vp, i64, vp, vp]),
        "pointid_classify_planes": (cint, [vp, ctypes.POINTER(_Plane), i32, vp, i64, vp, vp]),
        "pointid_classify_patches": (cint, [vp, vp, i64, vp, vp]),
        "pointid_classify_planes_noalloc": (cint, [vp, ctypes.POINTER(_Plane), i32, vp, i64, vp,
                                                   vp]),
        "pointid_classify_planes_ds": (cint, [vp, ctypes.POINTER(_Plane), i32, i32, vp, i64, vp,
                                              vp]),
        "pointid_downsample": (cint, [vp, i32, i32, i32, vp, vp]),
        "pointid_classify_requests": (cint, [vp, ctypes.POINTER(_Plane), i32,
                                             ctypes.POINTER(_Request), i32, vp]),
        "pointid_batcher_create": (cint, [vp, ctypes.POINTER(_Plane), i32, i32, i32,
                                          ctypes.POINTER(vp)]),
        "pointid_batcher_destroy": (cint, [vp]),
        "pointid_batcher_submit": (cint, [vp, ctypes.POINTER(_Request), vp,
                                            ctypes.POINTER(ctypes.c_uint64)]),
        "pointid_batcher_wait": (cint, [vp, ctypes.c_uint64]),
        "pointid_gather": (cint, [vp, i32, i32, vp, i64, vp, cint, vp]),
        "pointid_gather_planes": (cint, [ctypes.POINTER(_Plane), i32, vp, i64, vp, cint, vp]),
        "pointid_find_hits": (cint, [vp, ctypes.POINTER(_Plane), i32, ctypes.c_float, vp, i64,
                                     vp, vp]),
        "pointid_server_start": (cint, [vp, ctypes.POINTER(_Plane), i32, ctypes.c_char_p, i32, i32,
                                        ctypes.POINTER(vp)]),
        "pointid_server_stop": (cint, [vp]),
        "pointid_client_connect": (cint, [ctypes.c_char_p, ctypes.POINTER(vp)]),
        "pointid_client_classify": (cint, [vp, i32, vp, i64, vp, ctypes.POINTER(i64)]),
        "pointid_client_classify_patches": (cint, [vp, vp, i64, vp, ctypes.POINTER(i64)]),
        "pointid_client_close": (cint, [vp]),
        "pointid_layers_create": (cint, [cint, ctypes.POINTER(vp)]),
        "pointid_layers_destroy": (cint, [vp]),
        "pointid_layers_trim": (cint, [vp, ctypes.c_uint64, ctypes.POINTER(ctypes.c_uint64)]),
        "pointid_dense": (cint, [vp, cint, cint, i64, i64, i64, mat, mat, vp, mat, mat, kept, vp]),
        "pointid_dense_backward": (cint, [vp, cint, cint, i64, i64, i64, mat, kept, mat, kept, mat, mat,
                                          vp, vp]),
        "pointid_gated": (cint, [vp, cint, cint, i64, i64, i64, mat, mat, mat, vp, vp, mat, kept, kept,
                                 vp]),
        "pointid_gated_backward": (cint, [vp, cint, cint, i64, i64, i64, mat, kept, mat, mat, kept, kept,
                                          mat, mat, mat, vp, vp, vp]),
        "pointid_checkpoint_save": (cint, [cint, i64, i64, mat, ctypes.POINTER(_Packed), vp]),
        "pointid_checkpoint_load": (cint, [cint, i64, i64, ctypes.POINTER(_Packed), mat, vp]),
        "pointid_dropout": (cint, [vp, cint, i64, i64, mat, ctypes.POINTER(_Drop), mat, mat, vp]),
        "pointid_norm": (cint, [vp, cint, i64, i64, mat, ctypes.POINTER(_NormOf), ctypes.POINTER(_Block), mat, mat,
                                vp, vp]),
        "pointid_norm_backward": (cint, [vp, cint, i64, i64, mat, mat, vp, ctypes.POINTER(_NormOf),
                                         ctypes.POINTER(_Block), mat, ctypes.POINTER(_NormGrads), vp, u64, vp]),
        "pointid_norm_backward_scratch": (u64, [vp, i64, i64]),
        "pointid_logprobs": (cint, [vp, cint, i64, i64, mat, ctypes.c_float, vp, vp, vp, vp, i32, vp, vp, vp, u64,
                                    vp]),
        "pointid_logprobs_scratch": (u64, [vp, i64, i64, i32]),
        "pointid_logprobs_backward": (cint, [vp, cint, i64, i64, mat, ctypes.c_float, vp, vp, vp, vp, vp, vp, mat,
                                             vp]),
        "pointid_timing_enable": (cint, [cint]),
        "pointid_timing_reset": (cint, []),
        "pointid_timing_query": (cint, [ctypes.c_char_p, ctypes.POINTER(ctypes.c_double),
                                        ctypes.POINTER(ctypes.c_int64)]),
        "pointid_last_error": (ctypes.c_char_p, []),
        "pointid_version": (ctypes.c_char_p, []),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


lib = _load()
EXPORTED = ("pointid_create", "pointid_destroy", "pointid_precision", "pointid_trim",
            "pointid_classify",
            "pointid_classify_planes", "pointid_classify_planes_noalloc", "pointid_classify_requests",
            "pointid_classify_patches",
            "pointid_batcher_create", "pointid_batcher_destroy", "pointid_batcher_submit",
            "pointid_batcher_wait",
            "pointid_gather",
            "pointid_gather_planes", "pointid_find_hits", "pointid_classify_planes_ds",
            "pointid_downsample", "pointid_server_start", "pointid_server_stop",
            "pointid_client_connect", "pointid_client_classify", "pointid_client_classify_patches",
            "pointid_client_close", "pointid_layers_create", "pointid_layers_destroy", "pointid_layers_trim",
            "pointid_dense", "pointid_dense_backward", "pointid_gated", "pointid_gated_backward",
            "pointid_checkpoint_save", "pointid_checkpoint_load",
            "pointid_dropout", "pointid_norm", "pointid_norm_backward", "pointid_norm_backward_scratch",
            "pointid_logprobs", "pointid_logprobs_scratch", "pointid_logprobs_backward", "pointid_timing_enable", "pointid_timing_reset",
            "pointid_timing_query", "pointid_last_error", "pointid_version")


def _check(status: int):
    if status != POINTID_OK:
        raise PointIdError(status, lib.pointid_last_error().decode())
    return status


def pointid_last_error() -> str:
    return lib.pointid_last_error().decode()


def pointid_version() -> str:
    return lib.pointid_version().decode()


def pointid_timing_enable(on: bool = True):
    _check(lib.pointid_timing_enable(1 if on else 0))


def pointid_timing_reset():
    _check(lib.pointid_timing_reset())


def pointid_timing_query(kernel: str):
    """(total_ms, launches) of `kernel` since the last reset."""
    ms = ctypes.c_double()
    n = ctypes.c_int64()
    _check(lib.pointid_timing_query(kernel.encode(), ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value


def _precision(p) -> int:
    if isinstance(p, str):
        return {"fp32": POINTID_FP32, "bf16": POINTID_BF16, "fp16": POINTID_FP16,
                "fp8": POINTID_FP8}[p]
    return int(p)


def _stream_ptr(stream, device=None):
    if stream is None:
        stream = torch.cuda.current_stream(device)
    if isinstance(stream, int):
        return ctypes.c_void_p(stream)
    return ctypes.c_void_p(stream.cuda_stream)


# the current stream's handle without the Stream object around it (2 us a call), where torch has it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _check_on(device: int, call, *args):
    """A call that has no handle to make its device current."""
    if torch.cuda.current_device() == device:
        return _check(call(*args))
    with torch.cuda.device(device):
        return _check(call(*args))


def _make(stream, device: int, outputs):
    """outputs(), the tensors that a call returns, in its stream's memory: the current stream may
    still be using what its own memory had before.  (Not called without a stream of their own:
    0.3 us of a small call's 9.)"""
    raw = stream if isinstance(stream, int) else stream.cuda_stream
    if _raw_stream is not None and raw == _raw_stream(device):
        return outputs()
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(raw, device=device) if raw else torch.cuda.default_stream(device)
    with torch.cuda.stream(stream):
        return outputs()


def _empty(shape, dtype, device, stream):
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    return _make(stream, device.index, lambda: torch.empty(shape, dtype=dtype, device=device))


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else ctypes.c_void_p(0)


def _need(t, dtype, name, device=None, tail_shape=None):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if device is not None and t.device.index != device:
        raise ValueError(f"{name} is on cuda:{t.device.index}, handle is on cuda:{device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if tail_shape is not None and tuple(t.shape[1:]) != tuple(tail_shape):
        raise ValueError(f"{name} must have shape [n, {', '.join(map(str, tail_shape))}]")


class Handle:
    """A created classifier; frees itself on garbage collection."""

    def __init__(self, raw: ctypes.c_void_p, device: int, precision: int):
        self._raw = raw
        self.device = device
        self.precision = precision

    @property
    def raw(self):
        if not self._raw:
            raise ValueError("handle was destroyed")
        return self._raw

    def close(self):
        if self._raw:
            _check(lib.pointid_destroy(self._raw))
            self._raw = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def pointid_create(weights: dict, precision="fp32", device: int = 0) -> Handle:
    """Upload ``weights`` (dict of float32 arrays, layouts of include/pointid.h)."""
    arrays = {}
    for name in _WEIGHT_FIELDS:
        a = np.ascontiguousarray(np.asarray(weights[name], dtype=np.float32))
        if a.size != _WEIGHT_SIZES[name]:
            raise ValueError(f"{name} has {a.size} values, expected {_WEIGHT_SIZES[name]}")
        arrays[name] = a
    w = _Weights(**{n: arrays[n].ctypes.data_as(ctypes.POINTER(ctypes.c_float))
                    for n in _WEIGHT_FIELDS})
    raw = ctypes.c_void_p()
    prec = _precision(precision)
    _check(lib.pointid_create(ctypes.byref(w), prec, int(device), ctypes.byref(raw)))
    return Handle(raw, int(device), prec)


def pointid_destroy(h: Handle):
    h.close()


def pointid_trim(h: Handle, keep_bytes: int = 0) -> int:
    """Free the handle's idle cached scratch buffers down to keep_bytes;
    returns the bytes still cached."""
    cached = ctypes.c_uint64()
    _check(lib.pointid_trim(h.raw, ctypes.c_uint64(int(keep_bytes)), ctypes.byref(cached)))
    return int(cached.value)


def pointid_classify(h: Handle, image: torch.Tensor, hits: torch.Tensor,
                     scores: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Scores [n][4] for int32 hits [n][2] = (wire, tick) on fp32 image [W][T]."""
    _need(image, torch.float32, "image", h.device)
    if image.dim() != 2:
        raise ValueError("image must be [n_wires][n_ticks]")
    _need(hits, torch.int32, "hits", h.device, (2,))
    n = hits.shape[0]
    if scores is None:
        scores = _empty((n, 4), torch.float32, image.device, stream)
    _need(scores, torch.float32, "scores", h.device, (4,))
    _check(lib.pointid_classify(h.raw, _ptr(image), image.shape[0], image.shape[1], _ptr(hits),
                                n, _ptr(scores), _stream_ptr(stream, image.device)))
    return scores


def _plane_array(images):
    if len(images) < 1 or len(images) > MAX_PLANES:
        raise ValueError("between 1 and 64 planes")
    arr = (_Plane * len(images))()
    for i, im in enumerate(images):
        _need(im, torch.float32, f"images[{i}]")
        if im.dim() != 2:
            raise ValueError("each image must be [n_wires][n_ticks]")
        arr[i] = _Plane(im.data_ptr(), im.shape[0], im.shape[1])
    return arr


def pointid_classify_planes(h: Handle, images, hits: torch.Tensor,
                            scores: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Scores for int32 hits [n][3] = (plane, wire, tick) over a list of plane images."""
    arr = _plane_array(images)
    _need(hits, torch.int32, "hits", h.device, (3,))
    n = hits.shape[0]
    if scores is None:
        scores = _empty((n, 4), torch.float32, hits.device, stream)
    _need(scores, torch.float32, "scores", h.device, (4,))
    _check(lib.pointid_classify_planes(h.raw, arr, len(images), _ptr(hits), n, _ptr(scores),
                                       _stream_ptr(stream, hits.device)))
    return scores


def pointid_classify_planes_noalloc(h: Handle, images, hits: torch.Tensor,
                                    scores: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """pointid_classify_planes with its scratch in the library's fixed device
    array (at most 8192 hits; calls on one GPU must not overlap)."""
    _need(hits, torch.int32, "hits", h.device, (3,))
    n = hits.shape[0]
    if scores is None:
        scores = _empty((n, 4), torch.float32, hits.device, stream)
    _need(scores, torch.float32, "scores", h.device, (4,))
    arr = _plane_array(images)
    _check(lib.pointid_classify_planes_noalloc(h.raw, arr, len(images), _ptr(hits), n, _ptr(scores),
                                               _stream_ptr(stream, hits.device)))
    return scores


def pointid_classify_planes_ds(h: Handle, images, hits: torch.Tensor, ticks_per_column: int,
                               scores: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Scores with patches of ``ticks_per_column`` ticks per column; hits are
    (plane, wire, tick) in unbinned ticks over the unbinned plane images."""
    arr = _plane_array(images)
    _need(hits, torch.int32, "hits", h.device, (3,))
    n = hits.shape[0]
    if scores is None:
        scores = _empty((n, 4), torch.float32, hits.device, stream)
    _need(scores, torch.float32, "scores", h.device, (4,))
    _check(lib.pointid_classify_planes_ds(h.raw, arr, len(images), int(ticks_per_column),
                                          _ptr(hits), n, _ptr(scores),
                                          _stream_ptr(stream, hits.device)))
    return scores


def pointid_downsample(image: torch.Tensor, ticks_per_column: int,
                       out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """fp32 image [W][T] binned into [W][ceil(T / D)] columns of D ticks."""
    _need(image, torch.float32, "image")
    if image.dim() != 2:
        raise ValueError("image must be [n_wires][n_ticks]")
    D = int(ticks_per_column)
    W, T = image.shape
    J = -(-T // D) if D >= 1 else 0
    if out is None:
        out = _empty((W, max(J, 1)), torch.float32, image.device, stream)
    _need(out, torch.float32, "out")
    if tuple(out.shape) != (W, J):
        raise ValueError(f"out must be [{W}, {J}]")
    _check_on(image.get_device(), lib.pointid_downsample, _ptr(image), W, T, D, _ptr(out),
              _stream_ptr(stream, image.device))
    return out


def pointid_classify_requests(h: Handle, images, requests, stream=None):
    """Classify several requests in one batched call.

    ``requests`` is a list of ``(plane, hits, scores)``: ``plane`` an index into
    ``images`` with int32 hits [n][2] = (wire, tick), or -1 with hits [n][3] =
    (plane, wire, tick); ``scores`` a float32 [n][4] output, or None to allocate
    one.  Returns the list of score tensors."""
    arr = _plane_array(images)
    reqs = (_Request * max(len(requests), 1))()
    outs = []
    dev = None
    for i, (plane, hits, scores) in enumerate(requests):
        plane = int(plane)
        _need(hits, torch.int32, f"requests[{i}].hits", h.device, (2,) if plane >= 0 else (3,))
        n = hits.shape[0]
        if scores is None:
            scores = _empty((n, 4), torch.float32, hits.device, stream)
        _need(scores, torch.float32, f"requests[{i}].scores", h.device, (4,))
        reqs[i] = _Request(hits.data_ptr(), n, plane, scores.data_ptr())
        outs.append(scores)
        dev = hits.device
    _check(lib.pointid_classify_requests(h.raw, arr, len(images), reqs, len(requests),
                                         _stream_ptr(stream, dev)))
    return outs


class Batcher:
    """Dynamic batcher over a handle and resident plane images (see
    pointid_batcher_create).  submit() returns a ticket; wait(ticket) blocks
    until that request's scores are written.  The hits and scores tensors of a
    request are kept alive here until its wait returns."""

    def __init__(self, h: Handle, images, max_requests: int = 64, max_delay_us: int = 200):
        self._arr = _plane_array(images)
        self._images = list(images)
        self._h = h
        raw = ctypes.c_void_p()
        _check(lib.pointid_batcher_create(h.raw, self._arr, len(images), int(max_requests),
                                          int(max_delay_us), ctypes.byref(raw)))
        self.raw = raw
        self._live = {}

    def submit(self, plane: int, hits: torch.Tensor, scores: torch.Tensor | None = None,
               stream=None) -> int:
        """Queue a request; the batch that classifies it starts after the work
        enqueued on `stream` (the current stream by default) before this call,
        so `hits` may still be in production there and `scores` may be a fresh
        allocation of that stream."""
        plane = int(plane)
        _need(hits, torch.int32, "hits", self._h.device, (2,) if plane >= 0 else (3,))
        n = hits.shape[0]
        if scores is None:
            scores = _empty((n, 4), torch.float32, hits.device, stream)
        _need(scores, torch.float32, "scores", self._h.device, (4,))
        req = _Request(hits.data_ptr(), n, plane, scores.data_ptr())
        ticket = ctypes.c_uint64()
        _check(lib.pointid_batcher_submit(self.raw, ctypes.byref(req),
                                          _stream_ptr(stream, hits.device), ctypes.byref(ticket)))
        self._live[ticket.value] = (hits, scores)
        return ticket.value

    def wait(self, ticket: int) -> torch.Tensor:
        """Blocks until the request is classified; returns its scores tensor."""
        try:
            _check(lib.pointid_batcher_wait(self.raw, ctypes.c_uint64(ticket)))
        finally:
            pair = self._live.pop(ticket, None)
        return pair[1] if pair else None

    def close(self):
        if self.raw:
            _check(lib.pointid_batcher_destroy(self.raw))
            self.raw = None
            self._live.clear()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def pointid_classify_patches(h: Handle, patches: torch.Tensor,
                             scores: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Scores for fp32 patches [n][48][48]."""
    _need(patches, torch.float32, "patches", h.device, (48, 48))
    n = patches.shape[0]
    if scores is None:
        scores = _empty((n, 4), torch.float32, patches.device, stream)
    _need(scores, torch.float32, "scores", h.device, (4,))
    _check(lib.pointid_classify_patches(h.raw, _ptr(patches), n, _ptr(scores),
                                        _stream_ptr(stream, patches.device)))
    return scores


def pointid_gather(image: torch.Tensor, hits: torch.Tensor, out_dtype="fp32",
                   out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Patches [n][48][48]: float32, or bf16 / fp16 bit patterns as int16."""
    _need(image, torch.float32, "image")
    _need(hits, torch.int32, "hits", None, (2,))
    code = _precision(out_dtype)
    n = hits.shape[0]
    tdt = torch.float32 if code == POINTID_FP32 else torch.int16
    if out is None:
        out = _empty((n, 48, 48), tdt, image.device, stream)
    _check_on(image.get_device(), lib.pointid_gather, _ptr(image), image.shape[0], image.shape[1], _ptr(hits), n,
              _ptr(out), code, _stream_ptr(stream, image.device))
    return out


def pointid_gather_planes(images, hits: torch.Tensor, out_dtype="fp32",
                          out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    arr = _plane_array(images)
    _need(hits, torch.int32, "hits", None, (3,))
    code = _precision(out_dtype)
    n = hits.shape[0]
    tdt = torch.float32 if code == POINTID_FP32 else torch.int16
    if out is None:
        out = _empty((n, 48, 48), tdt, hits.device, stream)
    _check_on(hits.get_device(), lib.pointid_gather_planes, arr, len(images), _ptr(hits), n, _ptr(out), code,
              _stream_ptr(stream, hits.device))
    return out


def pointid_find_hits(h: Handle, images, threshold: float, capacity: int | None = None,
                      hits_out: torch.Tensor | None = None, n_found: torch.Tensor | None = None,
                      stream=None):
    """Hits (plane, wire, tick) of fp32 plane images, found on the device.

    Returns ``(hits_out, n_found)``: int32 [capacity][3], of which the first
    min(n_found, capacity) rows are written, and a device int64 [1] holding the
    number of hits found (read it after the stream has passed the call).
    ``capacity`` defaults to ``hits_out``'s length, else to 65,536.
    """
    arr = _plane_array(images)
    dev = images[0].device
    if hits_out is None:
        cap = 65536 if capacity is None else int(capacity)
        hits_out = _empty((cap, 3), torch.int32, dev, stream)
    _need(hits_out, torch.int32, "hits_out", h.device, (3,))
    cap = hits_out.shape[0] if capacity is None else int(capacity)
    if cap > hits_out.shape[0]:
        raise ValueError("capacity exceeds hits_out")
    if n_found is None:
        n_found = _empty((1,), torch.int64, dev, stream)
    _need(n_found, torch.int64, "n_found", h.device)
    _check(lib.pointid_find_hits(h.raw, arr, len(images), float(threshold),
                                 _ptr(hits_out) if cap > 0 else ctypes.c_void_p(0), cap,
                                 _ptr(n_found), _stream_ptr(stream, dev)))
    return hits_out, n_found


class Server:
    """pointid_server_start / pointid_server_stop: a local request server over
    resident device planes (the handle and the planes must outlive it)."""

    def __init__(self, h: Handle, images, socket_path: str, max_requests: int = 0,
                 max_delay_us: int = 200):
        self._images = list(images)
        arr = _plane_array(self._images) if self._images else None
        raw = ctypes.c_void_p()
        _check(lib.pointid_server_start(h.raw, arr, len(self._images), socket_path.encode(),
                                        int(max_requests), int(max_delay_us), ctypes.byref(raw)))
        self._raw = raw
        self._h = h
        self.path = socket_path

    def close(self):
        if self._raw:
            _check(lib.pointid_server_stop(self._raw))
            self._raw = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Client:
    """pointid_client_*: host arrays in, host scores out (numpy; no GPU)."""

    def __init__(self, socket_path: str):
        raw = ctypes.c_void_p()
        _check(lib.pointid_client_connect(socket_path.encode(), ctypes.byref(raw)))
        self._raw = raw
        self.server_ns = 0

    def classify(self, hits: np.ndarray, plane: int = -1) -> np.ndarray:
        """Scores [n][4] of int32 hits [n][2] on `plane`, or [n][3] when plane < 0."""
        hits = np.ascontiguousarray(hits, dtype=np.int32)
        width = 2 if plane >= 0 else 3
        if hits.ndim != 2 or hits.shape[1] != width:
            raise ValueError(f"hits must be [n][{width}]")
        out = np.empty((hits.shape[0], 4), np.float32)
        ns = ctypes.c_int64()
        _check(lib.pointid_client_classify(self._raw, int(plane), hits.ctypes.data_as(ctypes.c_void_p),
                                           hits.shape[0], out.ctypes.data_as(ctypes.c_void_p),
                                           ctypes.byref(ns)))
        self.server_ns = ns.value
        return out

    def classify_patches(self, patches: np.ndarray) -> np.ndarray:
        patches = np.ascontiguousarray(patches, dtype=np.float32)
        if patches.ndim != 3 or patches.shape[1:] != (48, 48):
            raise ValueError("patches must be [n][48][48]")
        out = np.empty((patches.shape[0], 4), np.float32)
        ns = ctypes.c_int64()
        _check(lib.pointid_client_classify_patches(self._raw,
                                                   patches.ctypes.data_as(ctypes.c_void_p),
                                                   patches.shape[0],
                                                   out.ctypes.data_as(ctypes.c_void_p),
                                                   ctypes.byref(ns)))
        self.server_ns = ns.value
        return out

    def close(self):
        if self._raw:
            _check(lib.pointid_client_close(self._raw))
            self._raw = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- layers

NORMS = {"rms": 1, "layer": 2}
_LAYER_TYPES = {torch.float32: POINTID_FP32, torch.bfloat16: POINTID_BF16, torch.float16: POINTID_FP16}


class Layers:
    """pointid_layers: a device and its cache of scratch buffers; frees itself on
    garbage collection."""

    def __init__(self, raw: ctypes.c_void_p, device: int):
        self._raw = raw
        self.device = device

    @property
    def raw(self):
        if not self._raw:
            raise ValueError("layers handle was destroyed")
        return self._raw

    def close(self):
        if self._raw:
            _check(lib.pointid_layers_destroy(self._raw))
            self._raw = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Checkpoint:
    """An 8-bit checkpoint of a matrix [m][n]: e4m3 codes (uint8 [m][n]) and the biased
    exponents of the blocks of 32 columns (uint8 [m][ceil(n / 32)])."""

    __slots__ = ("codes", "exponents")

    def __init__(self, codes: torch.Tensor, exponents: torch.Tensor):
        _need(codes, torch.uint8, "codes")
        _need(exponents, torch.uint8, "exponents", codes.device.index)
        if codes.dim() != 2 or tuple(exponents.shape) != (codes.shape[0], -(-codes.shape[1] // 32)):
            raise ValueError("codes must be [m, n] and exponents [m, ceil(n / 32)]")
        self.codes = codes
        self.exponents = exponents

    @classmethod
    def empty(cls, m: int, n: int, device="cuda") -> "Checkpoint":
        c = cls.__new__(cls)
        c.codes = torch.empty((m, n), dtype=torch.uint8, device=device)
        c.exponents = torch.empty((m, -(-n // 32)), dtype=torch.uint8, device=device)
        return c

    @property
    def shape(self):
        return self.codes.shape

    @property
    def device(self):
        return self.codes.device


def pointid_layers_create(device: int = 0) -> Layers:
    raw = ctypes.c_void_p()
    _check(lib.pointid_layers_create(int(device), ctypes.byref(raw)))
    return Layers(raw, int(device))


def pointid_layers_destroy(layers: Layers):
    layers.close()


def pointid_layers_trim(layers: Layers, keep_bytes: int = 0) -> int:
    """Free the idle scratch buffers down to keep_bytes; returns the bytes still cached."""
    cached = ctypes.c_uint64()
    _check(lib.pointid_layers_trim(layers.raw, ctypes.c_uint64(int(keep_bytes)), ctypes.byref(cached)))
    return int(cached.value)


def _layer_stream(stream, device: int):
    if stream is None and _raw_stream is not None:
        return _raw_stream(device)
    return _stream_ptr(stream, torch.device("cuda", device))


def _matrix(t, name, dtype, shape, device):
    """The descriptor of a matrix (rows of unit stride, any pitch), or None."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.get_device() != device:
        raise ValueError(f"{name} is on cuda:{t.get_device()}, the call's device is cuda:{device}")
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    rows, cols = shape
    pitch, unit = t.stride()
    if cols > 1 and unit != 1:
        raise ValueError(f"the rows of {name} must have unit stride")
    if rows > 1 and pitch < cols:
        raise ValueError(f"the rows of {name} overlap")
    return _Matrix(t.data_ptr(), pitch if rows > 1 else cols)


def _output(t, like, name, dtype, shape, device, stream=None):
    """An output that is given, or made like a tensor of the call, and its descriptor."""
    if t is not None:
        return t, _matrix(t, name, dtype, shape, device)
    t = like.new_empty(shape, dtype=dtype) if stream is None else _empty(shape, dtype, like.device, stream)
    return t, _Matrix(t.data_ptr(), shape[1])


def _kept(t, name, dtype, shape, device):
    if t is None:
        return None
    if isinstance(t, Checkpoint):
        if tuple(t.shape) != shape:
            raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
        if t.device.index != device:
            raise ValueError(f"{name} is on cuda:{t.device.index}, the call's device is cuda:{device}")
        return _Kept(_Matrix(None, 0), _Packed(t.codes.data_ptr(), t.exponents.data_ptr()))
    return _Kept(_matrix(t, name, dtype, shape, device), _Packed(None, None))


def _bias(t, name, n, device):
    if t is None:
        return None
    _need(t, torch.float32, name, device)
    if t.numel() != n or t.dim() != 1:
        raise ValueError(f"{name} must be [{n}]")
    return t.data_ptr()


def _layer_type(t, name):
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise TypeError(f"{name} must be a torch tensor of two dimensions")
    if t.dtype not in _LAYER_TYPES:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    return t.dtype


def _activation(act) -> int:
    if act not in ACTIVATIONS:
        raise ValueError(f"act must be one of {', '.join(ACTIVATIONS)}")
    return ACTIVATIONS[act]


def _ref(s):
    return ctypes.byref(s) if s is not None else None


def _shapes(x, w, name):
    if w.dim() != 2 or x.shape[1] != w.shape[0]:
        raise ValueError(f"x is {list(x.shape)} and {name} {list(w.shape)}: their inner sizes differ")
    return x.shape[0], x.shape[1], w.shape[1]


def pointid_dense(layers: Layers, x: torch.Tensor, w: torch.Tensor, bias: torch.Tensor | None = None,
                  act: str = "none", residual: torch.Tensor | None = None, y: torch.Tensor | None = None,
                  save=None, stream=None) -> torch.Tensor:
    """y [m][n] = act(x [m][k] @ w [k][n] + bias) + residual.

    ``save`` (a tensor like y, or a Checkpoint) receives x @ w + bias for the backward pass."""
    dt, dev = _layer_type(x, "x"), layers.device
    m, k, n = _shapes(x, w, "w")
    code = _activation(act)
    y, out = _output(y, x, "y", dt, (m, n), dev, stream)
    _check(lib.pointid_dense(
        layers.raw, _LAYER_TYPES[dt], code, m, k, n, _ref(_matrix(x, "x", dt, (m, k), dev)),
        _ref(_matrix(w, "w", dt, (k, n), dev)), _bias(bias, "bias", n, dev),
        _ref(_matrix(residual, "residual", dt, (m, n), dev)), ctypes.byref(out),
        _ref(_kept(save, "save", dt, (m, n), dev)), _layer_stream(stream, dev)))
    return y


def pointid_dense_backward(layers: Layers, dy: torch.Tensor, x, w: torch.Tensor, z=None, act: str = "none",
                           need_dx: bool = True, need_dw: bool = True, need_db: bool = True, stream=None):
    """(dx, dw, db) of pointid_dense from dy [m][n]; None for what is not needed.

    ``x`` and ``z`` (the saved x @ w + bias) are tensors or Checkpoints; x is not needed
    without dw, z not with act "none".  db is float32 [n]."""
    dt, dev = _layer_type(dy, "dy"), layers.device
    m, n = dy.shape
    k = w.shape[0]
    code = _activation(act)

    def outputs():
        return (_output(None, dy, "dx", dt, (m, k), dev) if need_dx else (None, None),
                _output(None, dy, "dw", dt, (k, n), dev) if need_dw else (None, None),
                dy.new_empty((n,), dtype=torch.float32) if need_db else None)

    (dx, to_dx), (dw, to_dw), db = outputs() if stream is None else _make(stream, dev, outputs)
    _check(lib.pointid_dense_backward(
        layers.raw, _LAYER_TYPES[dt], code, m, k, n, _ref(_matrix(dy, "dy", dt, (m, n), dev)),
        _ref(_kept(x, "x", dt, (m, k), dev)), _ref(_matrix(w, "w", dt, (k, n), dev)),
        _ref(_kept(z, "z", dt, (m, n), dev)), _ref(to_dx), _ref(to_dw), _ptr(db),
        _layer_stream(stream, dev)))
    return dx, dw, db


def pointid_gated(layers: Layers, x: torch.Tensor, wg: torch.Tensor, wu: torch.Tensor,
                  bias_g: torch.Tensor | None = None, bias_u: torch.Tensor | None = None, act: str = "silu",
                  h: torch.Tensor | None = None, save_g=None, save_u=None, stream=None) -> torch.Tensor:
    """h [m][n] = act(x @ wg + bias_g) * (x @ wu + bias_u).

    ``save_g`` and ``save_u`` (tensors like h, or Checkpoints) receive the two factors'
    sums for the backward pass."""
    dt, dev = _layer_type(x, "x"), layers.device
    m, k, n = _shapes(x, wg, "wg")
    code = _activation(act)
    h, out = _output(h, x, "h", dt, (m, n), dev, stream)
    _check(lib.pointid_gated(
        layers.raw, _LAYER_TYPES[dt], code, m, k, n, _ref(_matrix(x, "x", dt, (m, k), dev)),
        _ref(_matrix(wg, "wg", dt, (k, n), dev)), _ref(_matrix(wu, "wu", dt, (k, n), dev)),
        _bias(bias_g, "bias_g", n, dev), _bias(bias_u, "bias_u", n, dev),
        ctypes.byref(out), _ref(_kept(save_g, "save_g", dt, (m, n), dev)),
        _ref(_kept(save_u, "save_u", dt, (m, n), dev)), _layer_stream(stream, dev)))
    return h


def pointid_gated_backward(layers: Layers, dh: torch.Tensor, x, wg: torch.Tensor, wu: torch.Tensor, g, u,
                           act: str = "silu", need_dx: bool = True, need_dw: bool = True, need_db: bool = False,
                           stream=None):
    """(dx, dwg, dwu, dbg, dbu) of pointid_gated from dh [m][n]; None for what is not needed.

    ``x``, ``g`` and ``u`` are tensors or Checkpoints."""
    dt, dev = _layer_type(dh, "dh"), layers.device
    m, n = dh.shape
    k = wg.shape[0]
    code = _activation(act)

    def outputs():
        return (_output(None, dh, "dx", dt, (m, k), dev) if need_dx else (None, None),
                *(_output(None, dh, name, dt, (k, n), dev) if need_dw else (None, None) for name in ("dwg", "dwu")),
                *(dh.new_empty((n,), dtype=torch.float32) if need_db else None for _ in range(2)))

    (dx, to_dx), (dwg, to_dwg), (dwu, to_dwu), dbg, dbu = outputs() if stream is None else _make(stream, dev, outputs)
    _check(lib.pointid_gated_backward(
        layers.raw, _LAYER_TYPES[dt], code, m, k, n, _ref(_matrix(dh, "dh", dt, (m, n), dev)),
        _ref(_kept(x, "x", dt, (m, k), dev)), _ref(_matrix(wg, "wg", dt, (k, n), dev)),
        _ref(_matrix(wu, "wu", dt, (k, n), dev)), _ref(_kept(g, "g", dt, (m, n), dev)),
        _ref(_kept(u, "u", dt, (m, n), dev)), _ref(to_dx), _ref(to_dwg), _ref(to_dwu), _ptr(dbg), _ptr(dbu), _layer_stream(stream, dev)))
    return dx, dwg, dwu, dbg, dbu


def pointid_checkpoint_save(x: torch.Tensor, out: Checkpoint | None = None, stream=None) -> Checkpoint:
    """The 8-bit checkpoint of a matrix [m][n] (float32, bfloat16 or float16)."""
    dt, dev = _layer_type(x, "x"), x.get_device()
    m, n = x.shape
    a = _matrix(x, "x", dt, (m, n), dev)
    if torch.cuda.current_device() != dev:              # there is no handle to make it so
        with torch.cuda.device(dev):
            return pointid_checkpoint_save(x, out, stream)
    if out is None:
        out = Checkpoint.__new__(Checkpoint)
        if stream is None:
            out.codes = x.new_empty((m, n), dtype=torch.uint8)
            out.exponents = out.codes.new_empty((m, -(-n // 32)))
        else:
            out.codes, out.exponents = (_empty((m, c), torch.uint8, x.device, stream) for c in (n, -(-n // 32)))
        packed = _Packed(out.codes.data_ptr(), out.exponents.data_ptr())
    else:
        packed = _kept(out, "out", dt, (m, n), dev).packed
    _check(lib.pointid_checkpoint_save(_LAYER_TYPES[dt], m, n, ctypes.byref(a), ctypes.byref(packed),
                                       _layer_stream(stream, dev)))
    return out


def pointid_checkpoint_load(saved: Checkpoint, dtype=torch.float32, out: torch.Tensor | None = None,
                            stream=None) -> torch.Tensor:
    """The values a checkpoint stands for, as a matrix [m][n] of ``dtype``."""
    m, n = saved.shape
    dt, dev = dtype if out is None else _layer_type(out, "out"), saved.codes.get_device()
    if dt not in _LAYER_TYPES:
        raise TypeError(f"dtype must be float32, bfloat16 or float16, got {dt}")
    kept = _kept(saved, "saved", dt, (m, n), dev)
    if torch.cuda.current_device() != dev:
        with torch.cuda.device(dev):
            return pointid_checkpoint_load(saved, dtype, out, stream)
    out, a = _output(out, saved.codes, "out", dt, (m, n), dev, stream)
    _check(lib.pointid_checkpoint_load(_LAYER_TYPES[dt], m, n, ctypes.byref(kept.packed), ctypes.byref(a),
                                       _layer_stream(stream, dev)))
    return out


# ---- around the layers

class Drop(NamedTuple):
    """A dropout: probability, and what its mask is made of (``step``: an int64 or uint64 device
    value that is added to the offset when the call runs)."""
    p: float
    seed: int
    offset: int = 0
    step: torch.Tensor | None = None


class Norm(NamedTuple):
    """A norm of rows, "rms" or "layer", with its parameters (float32 [n])."""
    kind: str = "rms"
    weight: torch.Tensor | None = None
    bias: torch.Tensor | None = None
    eps: float = 1e-5


class Block(NamedTuple):
    """A residual block's end: its output, and how that is added to the block's input x,
    scale x + gate * drop(norm(out)); gate float32 [n]."""
    out: torch.Tensor
    norm: Norm | None = None
    gate: torch.Tensor | None = None
    scale: float = 1.0
    drop: Drop | None = None


class Normed(NamedTuple):
    h: torch.Tensor | None
    total: torch.Tensor | None
    stats: torch.Tensor | None


class NormGradients(NamedTuple):
    dx: torch.Tensor | None
    dout: torch.Tensor | None
    dweight: torch.Tensor | None
    dbias: torch.Tensor | None
    dblock_weight: torch.Tensor | None
    dblock_bias: torch.Tensor | None
    dgate: torch.Tensor | None


class LogProbs(NamedTuple):
    logp: torch.Tensor | None
    lse: torch.Tensor
    entropy: torch.Tensor | None
    top_ids: torch.Tensor | None
    top_logp: torch.Tensor | None


def _drop(d, device):
    """The fields of a dropout."""
    if d is None:
        return 0.0, 0, 0, None
    if not 0.0 <= d.p <= 1.0:
        raise ValueError("p must be in [0, 1]")
    if not (0 <= d.seed < 1 << 64 and 0 <= d.offset < 1 << 64):
        raise ValueError("seed and offset must be in [0, 2^64)")
    step = d.step
    if step is not None:
        if not isinstance(step, torch.Tensor) or step.dtype not in (torch.int64, torch.uint64):
            raise TypeError("step must be a torch tensor of int64 or uint64")
        if step.numel() != 1 or step.get_device() != device:
            raise ValueError(f"step must be one value on cuda:{device}")
        step = step.data_ptr()
    return d.p, d.seed, d.offset, step


def _vector(t, name, n, device, dtype=torch.float32):
    """The address of a vector [n], or None."""
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == device and t.shape == (n,)
            and t.is_contiguous()):
        _need(t, dtype, name, device)                   # says what is wrong with it
        raise ValueError(f"{name} must be [{n}]")
    return t.data_ptr()


def _norm(norm, name, n, device):
    """The fields of a norm."""
    if norm is None:
        return 0, 0.0, None, None
    kind, weight, bias, eps = norm
    if kind not in NORMS:
        raise ValueError(f"{name}.kind must be one of {', '.join(NORMS)}")
    return NORMS[kind], eps, _vector(weight, name + ".weight", n, device), _vector(bias, name + ".bias", n, device)


def _block(block, dt, shape, device):
    if block is None:
        return None
    out = _matrix(block.out, "block.out", dt, shape, device)
    n = shape[1]
    return _Block(out.data, out.ld, *_norm(block.norm, "block.norm", n, device),
                  _vector(block.gate, "block.gate", n, device), block.scale, *_drop(block.drop, device))


def _scratch(size, like):
    """(the memory, its address) of a call's scratch: of its stream's, so that it can be captured."""
    if size == 0:
        return None, None
    t = torch.empty(size, dtype=torch.uint8, device=like.device)
    return t, t.data_ptr()


def _rows_of_floats(like, rows, n):
    """float32 vectors [n], in one piece of memory."""
    if rows == 1:
        return (like.new_empty((n,), dtype=torch.float32),)
    return like.new_empty((rows, n), dtype=torch.float32).unbind() if rows else ()


def _like(t, given, name, dtype, shape, device):
    """An output like t, given or made (on the stream that is current), and its descriptor."""
    if given is not None:
        return given, _matrix(given, name, dtype, shape, device)
    t = torch.empty_like(t, memory_format=torch.contiguous_format)
    return t, _Matrix(t.data_ptr(), shape[1])


def pointid_dropout(layers: Layers, x: torch.Tensor, drop: Drop, residual: torch.Tensor | None = None,
                    y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """y [m][n] = drop(x) + residual; its gradient by x is pointid_dropout(dy, drop).

    ``y`` may be x or residual itself."""
    dt, dev = _layer_type(x, "x"), layers.device
    shape = x.shape
    a, r = _matrix(x, "x", dt, shape, dev), _matrix(residual, "residual", dt, shape, dev)
    d = _Drop(*_drop(drop, dev))

    def outputs():
        return _like(x, y, "y", dt, shape, dev)

    y, out = outputs() if stream is None else _make(stream, dev, outputs)
    _check(lib.pointid_dropout(layers.raw, _LAYER_TYPES[dt], shape[0], shape[1], a, d, r, out,
                               _layer_stream(stream, dev)))
    return y


def pointid_norm(layers: Layers, x: torch.Tensor, norm: Norm | None = None, block: Block | None = None,
                 keep: bool = False, total: torch.Tensor | None = None, h: torch.Tensor | None = None,
                 stream=None) -> Normed:
    """The joint of two residual blocks: total = scale x + gate * drop(block.norm(block.out)), where there is a
    block, and h = norm(total), where there is a norm.

    Returns (h, total, stats), None for what there is not: total without a block is x itself; with
    ``keep`` the rows' statistics [m][4] are there for the backward pass.  ``total`` may be x itself."""
    dt, dev = _layer_type(x, "x"), layers.device
    m, n = shape = x.shape
    if norm is None and block is None:
        raise ValueError("neither norm nor block is given")
    if (h is not None and norm is None) or (total is not None and block is None):
        raise ValueError("h needs norm and total needs block")
    a = _matrix(x, "x", dt, shape, dev)
    after = _NormOf(*_norm(norm, "norm", n, dev)) if norm is not None else None
    end = _block(block, dt, shape, dev)

    def outputs():
        return (_like(x, total, "total", dt, shape, dev) if block is not None else (None, None),
                _like(x, h, "h", dt, shape, dev) if norm is not None else (None, None),
                x.new_empty((m, 4), dtype=torch.float32) if keep else None)

    (total, to_total), (h, to_h), stats = outputs() if stream is None else _make(stream, dev, outputs)
    _check(lib.pointid_norm(layers.raw, _LAYER_TYPES[dt], m, n, a, after, end, to_total, to_h,
                            stats.data_ptr() if keep else None, _layer_stream(stream, dev)))
    return Normed(h, total, stats)


def pointid_norm_backward(layers: Layers, dh: torch.Tensor | None, total: torch.Tensor | None,
                          stats: torch.Tensor | None, norm: Norm | None = None, block: Block | None = None,
                          dtotal: torch.Tensor | None = None, need_dx: bool = True, need_dout: bool = True,
                          need_params: bool = True, dx: torch.Tensor | None = None, stream=None) -> NormGradients:
    """Gradients of pointid_norm from those of h and total (``dtotal``), with the total (without a
    block: x) and the stats of the forward call, and its norm and block.

    Parameters' gradients are float32 [n], of those that are given.  ``dx`` may be dtotal itself."""
    if norm is None and dh is not None:
        raise ValueError("dh is the gradient of h, which there is only with norm")
    given = dh if norm is not None else dtotal
    dt, dev = _layer_type(given, "dh" if norm is not None else "dtotal"), layers.device
    m, n = shape = given.shape
    a = b = before = None
    if norm is not None:
        if total is None:
            raise ValueError("total is needed with norm")
        a, b = _matrix(dh, "dh", dt, shape, dev), _matrix(total, "total", dt, shape, dev)
        before = _NormOf(*_norm(norm, "norm", n, dev))
    c = _matrix(dtotal, "dtotal", dt, shape, dev)
    end = _block(block, dt, shape, dev)
    after = block.norm if block is not None else None
    kept = None
    if norm is not None or after is not None:
        _need(stats, torch.float32, "stats", dev)
        if stats.shape != (m, 4):
            raise ValueError(f"stats must be [{m}, 4]")
        kept = stats.data_ptr()
    wanted = [False] * 5
    if need_params:
        if norm is not None:
            wanted[0], wanted[1] = norm.weight is not None, norm.bias is not None
        if after is not None:
            wanted[2], wanted[3] = after.weight is not None, after.bias is not None
        wanted[4] = block is not None and block.gate is not None
    size = lib.pointid_norm_backward_scratch(layers.raw, m, n)

    def outputs():
        return (_like(given, dx, "dx", dt, shape, dev) if need_dx or dx is not None else (None, None),
                _like(given, None, "dout", dt, shape, dev) if need_dout and block is not None else (None, None),
                iter(_rows_of_floats(given, sum(wanted), n)), _scratch(size, given))

    (dx, to_dx), (dout, to_dout), made, (scratch, at) = outputs() if stream is None else _make(stream, dev, outputs)
    sums = [next(made) if w else None for w in wanted]
    grads = _NormGrads(to_dx and to_dx.data, to_dx.ld if to_dx else 0, to_dout and to_dout.data,
                       to_dout.ld if to_dout else 0, *[p if p is None else p.data_ptr() for p in sums])
    _check(lib.pointid_norm_backward(layers.raw, _LAYER_TYPES[dt], m, n, a, b, kept, before, end, c, grads, at, size,
                                     _layer_stream(stream, dev)))
    return NormGradients(dx, dout, *sums)


def pointid_logprobs(layers: Layers, logits: torch.Tensor, targets: torch.Tensor | None = None, scale: float = 1.0,
                     entropy: bool = False, top: int = 0, stream=None) -> LogProbs:
    """Log probabilities of z = scale logits [m][n]: (logp, lse, entropy, top_ids, top_logp), float32 [m]
    (int32 and float32 [m][top]), None for what is not asked for.

    logp: the targets' (int32 [m]; 0 for a target outside [0, n)); top: the most likely columns
    in falling order, the lowest first among equals."""
    dt, dev = _layer_type(logits, "logits"), layers.device
    m, n = logits.shape
    a = _matrix(logits, "logits", dt, (m, n), dev)
    at = _vector(targets, "targets", m, dev, torch.int32)
    if not 0 <= top <= min(64, n):
        raise ValueError("top must be in [0, 64] and at most n")
    size = lib.pointid_logprobs_scratch(layers.raw, m, n, top)

    def outputs():
        return (_rows_of_floats(logits, 1 + (at is not None) + bool(entropy), m),
                logits.new_empty((m, top), dtype=torch.int32) if top else None,
                logits.new_empty((m, top), dtype=torch.float32) if top else None, _scratch(size, logits))

    values, ids, best, (scratch, scratch_at) = outputs() if stream is None else _make(stream, dev, outputs)
    lse, h, logp = values[0], values[1] if entropy else None, values[-1] if at is not None else None
    _check(lib.pointid_logprobs(layers.raw, _LAYER_TYPES[dt], m, n, a, scale, at,
                                logp.data_ptr() if at is not None else None, lse.data_ptr(),
                                h.data_ptr() if entropy else None, top, ids.data_ptr() if top else None,
                                best.data_ptr() if top else None, scratch_at, size, _layer_stream(stream, dev)))
    return LogProbs(logp, lse, h, ids, best)


def pointid_logprobs_backward(layers: Layers, logits: torch.Tensor, lse: torch.Tensor,
                              targets: torch.Tensor | None = None, dlogp: torch.Tensor | None = None,
                              entropy: torch.Tensor | None = None, dentropy: torch.Tensor | None = None,
                              dlse: torch.Tensor | None = None, scale: float = 1.0,
                              dlogits: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The logits' gradient from those of logp, entropy and lse (float32 [m]), with the lse (and,
    for dentropy, the entropy) of the forward call.  ``dlogits`` may be logits itself."""
    dt, dev = _layer_type(logits, "logits"), layers.device
    m, n = shape = logits.shape
    a = _matrix(logits, "logits", dt, shape, dev)
    vectors = (_vector(lse, "lse", m, dev), _vector(targets, "targets", m, dev, torch.int32),
               _vector(dlogp, "dlogp", m, dev), _vector(entropy, "entropy", m, dev),
               _vector(dentropy, "dentropy", m, dev), _vector(dlse, "dlse", m, dev))

    def outputs():
        return _like(logits, dlogits, "dlogits", dt, shape, dev)

    dlogits, out = outputs() if stream is None else _make(stream, dev, outputs)
    _check(lib.pointid_logprobs_backward(layers.raw, _LAYER_TYPES[dt], m, n, a, scale, *vectors, out,
                                         _layer_stream(stream, dev)))
    return dlogits
