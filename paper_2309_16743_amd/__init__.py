"""MI355X (gfx950) online surrogate training: GPU training reservoir + MLP train step.

Thin Python binding over the C ABI of libonline_train.so (include/*.h).  The
functions below carry the C names and only marshal arguments: torch tensors
supply device pointers and HIP streams; every step of the path runs in the
library's HIP kernels.  Importing this package does not touch the GPU; the
first call loads the library and raises if it was not built.
"""
from __future__ import annotations

import ctypes as C
import operator
from typing import Optional

import numpy as np

from . import _abi
from ._abi import (OT_ACT_GELU, OT_ACT_NONE, OT_ACT_RELU, OT_ACT_SILU, OT_ADAPTERS_RELU, OT_ADAPTERS_RELU_INPUT, OT_BF16, OT_E_CLOSED, OT_E_INVAL, OT_E_STATE, OT_EMPTY, OT_FP32, OT_NOT_READY, OT_OK,
                   OT_POLICY_FIFO, OT_POLICY_FIRO, OT_POLICY_RESERVOIR, OT_SURROGATE_KEEP_GRADS, OTError,
                   check, last_error, load)

__all__ = [
    "Reservoir", "Surrogate", "reservoir_create", "reservoir_put", "reservoir_sample_batch",
    "reservoir_end_reception", "reservoir_stats", "reservoir_read_meta", "reservoir_read_rows",
    "reservoir_destroy", "surrogate_create", "surrogate_set_params", "surrogate_get_params",
    "surrogate_get_grads", "surrogate_get_adam_state", "surrogate_set_lr", "surrogate_train_step",
    "surrogate_predict", "surrogate_predict_noalloc", "surrogate_eval_loss", "surrogate_checkpoint", "surrogate_restore",
    "reservoir_checkpoint", "reservoir_restore", "surrogate_destroy", "LowRankAdapters", "GradientClip", "AdamTensors",
    "adapters_create", "adapters_forward", "adapters_backward", "adapters_destroy", "clip_create", "clip_norm",
    "clip_apply", "clip_destroy", "adam_create", "adam_step", "adam_set_lr", "adam_get_steps", "adam_set_steps",
    "adam_destroy", "DenseLayer", "GroupNorm", "Dropout", "dense_create", "dense_forward", "dense_backward",
    "dense_destroy", "norm_create", "norm_forward", "norm_backward", "norm_destroy", "dropout_create",
    "dropout_forward", "dropout_backward", "dropout_destroy", "OT_ACT_NONE", "OT_ACT_RELU", "OT_ACT_SILU",
    "OT_ACT_GELU", "OT_ADAPTERS_RELU", "OT_ADAPTERS_RELU_INPUT", "load", "last_error", "OTError",
    "OT_OK", "OT_NOT_READY", "OT_EMPTY", "OT_E_INVAL", "OT_E_CLOSED", "OT_E_STATE", "OT_FP32", "OT_BF16",
    "OT_SURROGATE_KEEP_GRADS", "OT_POLICY_RESERVOIR", "OT_POLICY_FIFO", "OT_POLICY_FIRO",
]


def _stream_handle(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _dev_ptr(t) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("expected a device tensor")
    return t.data_ptr()


def _rows(t, what: str):
    """(pointer, leading dimension) of a 2-D fp32 device tensor with unit column stride."""
    if t is None:
        return None, 0
    import torch
    if t.dtype != torch.float32 or t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{what}: expected a 2-D float32 tensor with unit column stride")
    return _dev_ptr(t), t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _checkpoint(handle, kind: str) -> np.ndarray:
    lib = load()
    n = C.c_int64()
    check(f"{kind}_checkpoint_size", getattr(lib, f"{kind}_checkpoint_size")(handle, C.byref(n)))
    buf = np.empty(n.value, np.uint8)
    check(f"{kind}_checkpoint", getattr(lib, f"{kind}_checkpoint")(handle, buf.ctypes.data, buf.nbytes))
    return buf


class Reservoir:
    """Handle of one GPU training reservoir (include/reservoir.h)."""

    def __init__(self, capacity: int, threshold: int, x_dim: int, u_dim: int, seed: int,
                 order_stream=None, policy: int = OT_POLICY_RESERVOIR):
        lib = load()
        h = C.c_void_p()
        st = None if order_stream is None else _stream_handle(order_stream)
        check("reservoir_create", lib.reservoir_create(C.byref(h), capacity, threshold, x_dim, u_dim, seed, policy,
                                                       st))
        self.policy = policy
        self._h = h
        self.capacity, self.threshold, self.x_dim, self.u_dim = capacity, threshold, x_dim, u_dim

    @property
    def handle(self):
        return self._h

    def put(self, x, u, stream=None, accepted=None) -> int:
        """Offer the rows of u (and x); returns the ticket.  accepted: device int64[1]."""
        xp, ldx = _rows(x, "x")
        up, ldu = _rows(u, "u")
        k = 0 if u is None else u.shape[0]
        t = C.c_uint64()
        check("reservoir_put", load().reservoir_put(self._h, xp, ldx, up, ldu, k, _stream_handle(stream),
                                                    _dev_ptr(accepted), C.byref(t)))
        return t.value

    def sample_batch(self, b: int, slots, x_out=None, u_out=None, stream=None):
        """Returns (status, rows drawn, ticket or None)."""
        xp, ldx = _rows(x_out, "x_out")
        up, ldu = _rows(u_out, "u_out")
        cnt = C.c_int64()
        t = C.c_uint64()
        st = check("reservoir_sample_batch",
                   load().reservoir_sample_batch(self._h, b, _stream_handle(stream), _dev_ptr(slots), xp, ldx,
                                                 up, ldu, C.byref(cnt), C.byref(t)))
        return st, cnt.value, (t.value if st == OT_OK else None)

    def end_reception(self) -> None:
        check("reservoir_end_reception", load().reservoir_end_reception(self._h))

    def slab(self):
        """(x address, ldx, u address, ldu) of the slabs: slot k's rows start at
        x + 4 ldx k and u + 4 ldu k (bytes)."""
        x, u = C.c_void_p(), C.c_void_p()
        ldx, ldu = C.c_int64(), C.c_int64()
        check("reservoir_slab", load().reservoir_slab(self._h, C.byref(x), C.byref(ldx), C.byref(u), C.byref(ldu)))
        return x.value, ldx.value, u.value, ldu.value

    def stats(self) -> dict:
        s = _abi.ReservoirStats()
        check("reservoir_stats", load().reservoir_stats(self._h, C.byref(s)))
        return {name: getattr(s, name) for name, _ in s._fields_}

    def read_meta(self):
        seen = np.empty(self.capacity, np.int32)
        ids = np.empty(self.capacity, np.int64)
        hist = np.empty(self.stats()["hist_len"], np.int64)
        check("reservoir_read_meta", load().reservoir_read_meta(self._h, seen.ctypes.data, ids.ctypes.data,
                                                                 hist.ctypes.data))
        return seen, ids, hist

    def read_rows(self, slots):
        slots = np.ascontiguousarray(slots, dtype=np.int32)
        x = np.empty((len(slots), self.x_dim), np.float32)
        u = np.empty((len(slots), self.u_dim), np.float32)
        check("reservoir_read_rows", load().reservoir_read_rows(self._h, slots.ctypes.data, len(slots),
                                                                 x.ctypes.data, u.ctypes.data))
        return x, u

    def checkpoint(self) -> np.ndarray:
        """Synchronous snapshot of the whole reservoir state as a host byte array."""
        return _checkpoint(self._h, "reservoir")

    def restore(self, blob: np.ndarray) -> None:
        b = np.ascontiguousarray(blob, dtype=np.uint8)
        check("reservoir_restore", load().reservoir_restore(self._h, b.ctypes.data, b.nbytes))

    def timing_begin(self, phases, max_calls: int) -> None:
        mask = sum(1 << _abi.RESERVOIR_PHASES.index(p) for p in phases)
        check("reservoir_timing_begin", load().reservoir_timing_begin(self._h, mask, max_calls))

    def timing_end(self) -> dict:
        """{phase: (total ms, calls)} for the phases being timed."""
        n = len(_abi.RESERVOIR_PHASES)
        ms = np.zeros(n, np.float64)
        cnt = np.zeros(n, np.int64)
        check("reservoir_timing_end", load().reservoir_timing_end(self._h, ms.ctypes.data, cnt.ctypes.data))
        return {p: (float(ms[i]), int(cnt[i])) for i, p in enumerate(_abi.RESERVOIR_PHASES) if cnt[i]}

    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h.value:
            check("reservoir_destroy", load().reservoir_destroy(self._h))
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Surrogate:
    """Handle of one MLP surrogate with Adam state (include/surrogate.h)."""

    def __init__(self, widths, precision: int = OT_FP32, lr: float = 1e-3, beta1: float = 0.9,
                 beta2: float = 0.999, eps: float = 1e-8, seed: int = 0, max_batch: int = 1024, flags: int = 0):
        lib = load()
        self.widths = tuple(int(w) for w in widths)
        arr = (C.c_int64 * len(self.widths))(*self.widths)
        h = C.c_void_p()
        check("surrogate_create", lib.surrogate_create(C.byref(h), arr, len(self.widths), precision, lr, beta1,
                                                       beta2, eps, seed, max_batch, flags))
        self._h = h
        self.precision = precision

    @property
    def handle(self):
        return self._h

    @property
    def n_layers(self) -> int:
        return len(self.widths) - 1

    def _layer_arrays(self, layer):
        return (np.empty((self.widths[layer + 1], self.widths[layer]), np.float32),
                np.empty(self.widths[layer + 1], np.float32))

    def set_params(self, layer: int, W=None, b=None) -> None:
        Wc = None if W is None else np.ascontiguousarray(W, dtype=np.float32)
        bc = None if b is None else np.ascontiguousarray(b, dtype=np.float32)
        if Wc is not None:
            assert Wc.shape == (self.widths[layer + 1], self.widths[layer])
        check("surrogate_set_params", load().surrogate_set_params(
            self._h, layer, None if Wc is None else Wc.ctypes.data, None if bc is None else bc.ctypes.data))

    def get_params(self, layer: int):
        W, b = self._layer_arrays(layer)
        check("surrogate_get_params", load().surrogate_get_params(self._h, layer, W.ctypes.data, b.ctypes.data))
        return W, b

    def get_grads(self, layer: int, weights: bool = True):
        """(dW, db) of the last step; dW is None when weights=False (the output
        layer's dW is not stored when its Adam update is fused)."""
        W, b = self._layer_arrays(layer)
        check("surrogate_get_grads", load().surrogate_get_grads(self._h, layer, W.ctypes.data if weights else None,
                                                                b.ctypes.data))
        return (W if weights else None), b

    def get_adam_state(self, layer: int):
        mW, mb = self._layer_arrays(layer)
        vW, vb = self._layer_arrays(layer)
        t = C.c_int64()
        check("surrogate_get_adam_state", load().surrogate_get_adam_state(
            self._h, layer, mW.ctypes.data, mb.ctypes.data, vW.ctypes.data, vb.ctypes.data, C.byref(t)))
        return (mW, mb), (vW, vb), t.value

    def set_lr(self, lr: float) -> None:
        check("surrogate_set_lr", load().surrogate_set_lr(self._h, lr))

    def set_device_step(self, enable: bool) -> None:
        """Adam's step counter in device memory (include/surrogate.h), so that a
        captured train step can be replayed."""
        check("surrogate_set_device_step", load().surrogate_set_device_step(self._h, 1 if enable else 0))

    def train_step(self, x, u, stream=None, loss=None) -> None:
        xp, ldx = _rows(x, "x")
        up, ldu = _rows(u, "u")
        check("surrogate_train_step", load().surrogate_train_step(
            self._h, xp, ldx, up, ldu, u.shape[0], _stream_handle(stream), _dev_ptr(loss)))

    def train_step_rows(self, x, u_addr: int, ldu: int, rows, n_rows: int, stream=None, loss=None,
                        targets_read=None) -> None:
        """Train step whose target row j is the fp32 row at device address
        u_addr + 4 ldu rows[j] (rows: int32 device tensor of x's row count,
        each in [0, n_rows)); targets_read: torch.cuda.Event recorded once the
        targets have been read."""
        import torch
        xp, ldx = _rows(x, "x")
        if rows.dtype != torch.int32 or rows.dim() != 1 or rows.shape[0] != x.shape[0] or not rows.is_contiguous():
            raise ValueError("rows: expected a contiguous int32 tensor with one index per row of x")
        ev = None
        if targets_read is not None:
            targets_read.record(torch.cuda.current_stream() if stream is None else stream)   # create the event
            ev = targets_read.cuda_event
        check("surrogate_train_step_rows", load().surrogate_train_step_rows(
            self._h, xp, ldx, u_addr, ldu, _dev_ptr(rows), n_rows, x.shape[0], _stream_handle(stream),
            _dev_ptr(loss), ev))

    def predict(self, x, y, stream=None) -> None:
        xp, ldx = _rows(x, "x")
        yp, ldy = _rows(y, "y")
        check("surrogate_predict", load().surrogate_predict(self._h, xp, ldx, x.shape[0], yp, ldy,
                                                            _stream_handle(stream)))

    def predict_noalloc(self, x, y, stream=None) -> None:
        """predict() through the entry point that allocates nothing (its
        workspace is the library's per-device scratch; see include/surrogate.h)."""
        xp, ldx = _rows(x, "x")
        yp, ldy = _rows(y, "y")
        check("surrogate_predict_noalloc", load().surrogate_predict_noalloc(self._h, xp, ldx, x.shape[0], yp, ldy,
                                                                            _stream_handle(stream)))

    def checkpoint(self) -> np.ndarray:
        """Synchronous snapshot of parameters, Adam moments and step counter."""
        return _checkpoint(self._h, "surrogate")

    def restore(self, blob: np.ndarray) -> None:
        b = np.ascontiguousarray(blob, dtype=np.uint8)
        check("surrogate_restore", load().surrogate_restore(self._h, b.ctypes.data, b.nbytes))

    def eval_loss(self, x, u, loss, stream=None) -> None:
        """Validation MSE of the current surrogate on rows x -> u into the device scalar `loss`."""
        xp, ldx = _rows(x, "x")
        up, ldu = _rows(u, "u")
        check("surrogate_eval_loss", load().surrogate_eval_loss(self._h, xp, ldx, up, ldu, x.shape[0],
                                                                _stream_handle(stream), _dev_ptr(loss)))

    def timing_begin(self, phases, max_steps: int) -> None:
        mask = sum(1 << _abi.SURROGATE_PHASES.index(p) for p in phases)
        check("surrogate_timing_begin", load().surrogate_timing_begin(self._h, mask, max_steps))

    def timing_end(self) -> dict:
        """{phase: (total ms, steps)} for the phases being timed."""
        n = len(_abi.SURROGATE_PHASES)
        ms = np.zeros(n, np.float64)
        cnt = np.zeros(n, np.int64)
        check("surrogate_timing_end", load().surrogate_timing_end(self._h, ms.ctypes.data, cnt.ctypes.data))
        return {p: (float(ms[i]), int(cnt[i])) for i, p in enumerate(_abi.SURROGATE_PHASES) if cnt[i]}

    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h.value:
            check("surrogate_destroy", load().surrogate_destroy(self._h))
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# A small call's time is the host's, so the checks below ask each tensor for each of its properties once.
def _matrix(t, rows: int, cols: int, dtype, device: int, what: str):
    """(pointer, leading dimension) of a rows x cols tensor on the device with unit column stride."""
    shape, st = t.shape, t.stride()
    if t.dtype is not dtype or len(shape) != 2 or shape[0] != rows or shape[1] != cols or (
            rows > 0 and cols > 1 and st[1] != 1):
        raise ValueError(f"{what}: expected a {rows} x {cols} {dtype} tensor with unit column stride")
    if t.get_device() != device:
        raise ValueError(f"{what}: expected a tensor on cuda:{device}")
    return t.data_ptr(), st[0] if rows > 1 else max(st[0], cols)


def _bank(t, n: int, rank: int, cols: int, dtype, device: int, what: str, of: str = "adapters"):
    """(pointer, leading dimension) of an n x rank x cols tensor on the device whose rows follow each other."""
    shape, st = t.shape, t.stride()
    if t.dtype is not dtype or len(shape) != 3 or shape[0] != n or shape[1] != rank or shape[2] != cols or (
            cols > 1 and st[2] != 1):
        raise ValueError(f"{what}: expected a {n} x {rank} x {cols} {dtype} tensor with unit column stride")
    ld = st[1] if rank > 1 else st[0] if n > 1 else max(st[0], cols)
    if n > 1 and st[0] != rank * ld:
        raise ValueError(f"{what}: the rows of successive {of} must follow each other")
    if t.get_device() != device:
        raise ValueError(f"{what}: expected a tensor on cuda:{device}")
    return t.data_ptr(), ld


def _vector(t, n: int, dtype, device: int, what: str):
    if t is None:
        return None
    shape = t.shape
    if t.dtype is not dtype or len(shape) != 1 or shape[0] != n or (n > 1 and t.stride()[0] != 1):
        raise ValueError(f"{what}: expected a contiguous {dtype} tensor of {n} values")
    if t.get_device() != device:
        raise ValueError(f"{what}: expected a tensor on cuda:{device}")
    return t.data_ptr()


def _raw_stream(stream, device: int, torch):
    """Handle of the given stream, or of the device's current one: without making a Stream object for it (1 us of a
    small call) where torch can say it."""
    if stream is None:
        current = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        return torch.cuda.current_stream(device).cuda_stream if current is None else current(device)
    return stream if isinstance(stream, int) else stream.cuda_stream


class LowRankAdapters:
    """Sizes and workspaces of a bank of low-rank adapters beside one frozen layer
    (include/adapters.h).  Tensors: x (n, in), w (out, in), down (G, rank, in), up
    (G, rank, out), ids int32 (n), bias fp32 (out), scale fp32 (G), t fp32 (n, rank)."""

    def __init__(self, in_dim: int, out_dim: int, rank: int, n_adapters: int, precision: int = OT_FP32,
                 max_rows: int = 1024):
        import torch
        h = C.c_void_p()
        check("adapters_create", load().adapters_create(C.byref(h), in_dim, out_dim, rank, n_adapters, precision,
                                                        max_rows))
        self._h = h
        self._torch, self._lib, self._device = torch, load(), torch.cuda.current_device()
        self.in_dim, self.out_dim, self.rank, self.n_adapters = in_dim, out_dim, rank, n_adapters
        self.precision = precision
        self.dtype = torch.bfloat16 if precision == OT_BF16 else torch.float32

    @property
    def handle(self):
        return self._h

    def _common(self, x, down, up, ids, scale):
        torch, dev = self._torch, self._device
        n = x.shape[0]
        g, r = self.n_adapters, self.rank
        return (n, _matrix(x, n, self.in_dim, self.dtype, dev, "x"),
                (None, 0) if down is None else _bank(down, g, r, self.in_dim, self.dtype, dev, "down"),
                _bank(up, g, r, self.out_dim, self.dtype, dev, "up"),
                _vector(ids, n, torch.int32, dev, "ids"), _vector(scale, g, torch.float32, dev, "scale"))

    def forward(self, x, w, down, up, ids, y, bias=None, scale=None, t=None, relu: bool = False, stream=None) -> None:
        """y = x W^T + bias + scale (x down^T) up per row's adapter (ids), in y's type
        (float32 or bfloat16); t receives x down^T for backward()."""
        torch, dev = self._torch, self._device
        n, xp, dp, up_, ip, sp = self._common(x, down, up, ids, scale)
        wp = _matrix(w, self.out_dim, self.in_dim, self.dtype, dev, "w")
        y_type = y.dtype
        if y_type is not torch.float32 and y_type is not torch.bfloat16:
            raise ValueError("y: expected float32 or bfloat16")
        yp = _matrix(y, n, self.out_dim, y_type, dev, "y")
        tp = (None, 0) if t is None else _matrix(t, n, self.rank, torch.float32, dev, "t")
        check("adapters_forward", self._lib.adapters_forward(
            self._h, *xp, *wp, _vector(bias, self.out_dim, torch.float32, dev, "bias"), *dp, *up_, sp, ip, n, *yp,
            OT_BF16 if y_type is torch.bfloat16 else OT_FP32, *tp, OT_ADAPTERS_RELU if relu else 0,
            _raw_stream(stream, self._device, self._torch)))

    def backward(self, x, w, down, up, ids, dy, t, ddown, dup, dx=None, scale=None, relu_input: bool = False,
                 stream=None) -> None:
        """Gradients of the bank into ddown, dup (fp32, whole) and, if given, of x into dx
        (relu_input: zero where x is not above 0); w and down may be None without dx."""
        torch, dev = self._torch, self._device
        n, xp, dp, up_, ip, sp = self._common(x, down, up, ids, scale)
        g, r = self.n_adapters, self.rank
        if dx is not None and (w is None or down is None):
            raise ValueError("dx needs w and down")
        wp = (None, 0) if w is None else _matrix(w, self.out_dim, self.in_dim, self.dtype, dev, "w")
        dyp = _matrix(dy, n, self.out_dim, self.dtype, dev, "dy")
        tp = _matrix(t, n, r, torch.float32, dev, "t")
        ddp = _bank(ddown, g, r, self.in_dim, torch.float32, dev, "ddown")
        dup_ = _bank(dup, g, r, self.out_dim, torch.float32, dev, "dup")
        dxp = (None, 0) if dx is None else _matrix(dx, n, self.in_dim, self.dtype, dev, "dx")
        check("adapters_backward", self._lib.adapters_backward(
            self._h, *xp, *wp, *dp, *up_, sp, ip, n, *dyp, *tp, *ddp, *dup_, *dxp,
            OT_ADAPTERS_RELU_INPUT if relu_input else 0, _raw_stream(stream, self._device, self._torch)))

    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h.value:
            check("adapters_destroy", load().adapters_destroy(self._h))
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _list_arrays(tensors, dtypes, counts, device: int, what: str):
    """Host array of the device addresses of a list of contiguous tensors (None: NULL entries allowed)."""
    if len(tensors) != len(counts):
        raise ValueError(f"{what}: expected {len(counts)} tensors")
    out = (C.c_void_p * len(counts))()
    for i, (t, n) in enumerate(zip(tensors, counts)):
        if t is None:
            continue
        if t.dtype != dtypes[i] or t.numel() != n or not t.is_contiguous():
            raise ValueError(f"{what}[{i}]: expected a contiguous {dtypes[i]} tensor of {n} elements")
        if n and t.get_device() != device:
            raise ValueError(f"{what}[{i}]: expected a tensor on cuda:{device}")
        out[i] = t.data_ptr() if n else None
    return out


class GradientClip:
    """A list of gradient tensors (contiguous, float32 or bfloat16) clipped by their
    global norm, in place or into the tensors `out` (include/gradients.h).  The object
    keeps the tensors."""

    def __init__(self, grads, out=None):
        import torch
        self.grads = list(grads)
        self.out = None if out is None else list(out)
        n = len(self.grads)
        counts = (C.c_int64 * n)(*[t.numel() for t in self.grads])
        types = (C.c_int32 * n)()
        for i, t in enumerate(self.grads):
            if t.dtype not in (torch.float32, torch.bfloat16):
                raise ValueError(f"grads[{i}]: expected float32 or bfloat16")
            types[i] = OT_BF16 if t.dtype == torch.bfloat16 else OT_FP32
        dtypes = [t.dtype for t in self.grads]
        self._device = torch.cuda.current_device()
        g = _list_arrays(self.grads, dtypes, counts, self._device, "grads")
        o = None if self.out is None else _list_arrays(self.out, dtypes, counts, self._device, "out")
        h = C.c_void_p()
        check("clip_create", load().clip_create(C.byref(h), n, g, o, counts, types))
        self._h = h
        self._torch, self._lib = torch, load()

    def norm(self, norm, stream=None) -> None:
        """The global norm into the device scalar `norm`."""
        check("clip_norm", self._lib.clip_norm(self._h, _scalar(norm, "norm", self._device, self._torch),
                                               _raw_stream(stream, self._device, self._torch)))

    def apply(self, max_norm: float, norm=None, stream=None) -> None:
        """Scale every tensor by min(1, max_norm / norm); the norm into `norm` (nullable)."""
        check("clip_apply", self._lib.clip_apply(self._h, max_norm, _scalar(norm, "norm", self._device, self._torch),
                                                 _raw_stream(stream, self._device, self._torch)))

    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h.value:
            check("clip_destroy", load().clip_destroy(self._h))
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _scalar(t, what: str, device: int, torch):
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.numel() != 1:
        raise ValueError(f"{what}: expected a float32 tensor of one element")
    if t.get_device() != device:
        raise ValueError(f"{what}: expected a tensor on cuda:{device}")
    return t.data_ptr()


class AdamTensors:
    """Adam over lists of contiguous fp32 tensors with their gradients clipped by the
    global norm (include/gradients.h); copies: bf16 tensors (or None) refreshed by
    each step.  The object keeps the tensors."""

    def __init__(self, params, grads, m, v, copies=None, lr: float = 1e-3, beta1: float = 0.9, beta2: float = 0.999,
                 eps: float = 1e-8, steps: int = 0):
        import torch
        self.params, self.grads, self.m, self.v = list(params), list(grads), list(m), list(v)
        self.copies = None if copies is None else list(copies)
        n = len(self.params)
        self._device = torch.cuda.current_device()
        counts = (C.c_int64 * n)(*[t.numel() for t in self.params])
        f32 = [torch.float32] * n
        arrays = []
        for name in ("params", "grads", "m", "v"):
            tensors = getattr(self, name)
            if any(t is None for t in tensors):
                raise ValueError(f"{name}: None among the tensors")
            arrays.append(_list_arrays(tensors, f32, counts, self._device, name))
        c = None
        if self.copies is not None:
            c = _list_arrays(self.copies, [torch.bfloat16] * n, counts, self._device, "copies")
        h = C.c_void_p()
        check("adam_create", load().adam_create(C.byref(h), n, *arrays, c, counts, lr, beta1, beta2, eps, steps))
        self._h = h
        self._torch, self._lib = torch, load()

    def step(self, max_norm: float = 0.0, norm=None, stream=None) -> None:
        """One step; max_norm 0: gradients as they are.  norm (nullable): the norm before
        clipping.  A norm that is not finite takes no step."""
        check("adam_step", self._lib.adam_step(self._h, max_norm, _scalar(norm, "norm", self._device, self._torch),
                                               _raw_stream(stream, self._device, self._torch)))

    def set_lr(self, lr: float) -> None:
        check("adam_set_lr", load().adam_set_lr(self._h, lr))

    def get_steps(self) -> int:
        n = C.c_int64()
        check("adam_get_steps", load().adam_get_steps(self._h, C.byref(n)))
        return n.value

    def set_steps(self, steps: int) -> None:
        check("adam_set_steps", load().adam_set_steps(self._h, steps))

    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h.value:
            check("adam_destroy", load().adam_destroy(self._h))
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class _Layer:
    """What the layers' objects share: handle, device, closing."""
    _destroy = ""

    def _open(self, create: str, *args, precision: int) -> None:
        import torch
        h = C.c_void_p()
        check(create, getattr(load(), create)(C.byref(h), *args))
        self._h = h
        self._torch, self._lib, self._device = torch, load(), torch.cuda.current_device()
        self.precision = precision
        self.dtype = torch.bfloat16 if precision == OT_BF16 else torch.float32

    @property
    def handle(self):
        return self._h

    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h.value:
            check(self._destroy, getattr(load(), self._destroy)(self._h))
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class DenseLayer(_Layer):
    """A dense layer y = act(x w^T + bias) + residual and its gradients (include/layers.h).
    Tensors: x (n, in), w (out, in), bias fp32 (out); y and residual (n, out), float32 or bfloat16
    alike; pre, dy (n, out); dx (n, in); dw fp32 (out, in); dbias fp32 (out).  activation:
    OT_ACT_*.  max_rows: rows of the largest backward (0: a layer that only serves)."""
    _destroy = "dense_destroy"

    def __init__(self, in_dim: int, out_dim: int, precision: int = OT_FP32, activation: int = OT_ACT_NONE,
                 max_rows: int = 1024):
        self._open("dense_create", in_dim, out_dim, precision, activation, max_rows, precision=precision)
        self.in_dim, self.out_dim, self.activation = in_dim, out_dim, activation

    def forward(self, x, w, y, bias=None, residual=None, pre=None, stream=None) -> None:
        """y = act(x w^T + bias) + residual; pre receives x w^T + bias for backward().  y may be the residual."""
        torch, dev = self._torch, self._device
        n = x.shape[0]
        xp = _matrix(x, n, self.in_dim, self.dtype, dev, "x")
        wp = _matrix(w, self.out_dim, self.in_dim, self.dtype, dev, "w")
        y_type = y.dtype
        if y_type is not torch.float32 and y_type is not torch.bfloat16:
            raise ValueError("y: expected float32 or bfloat16")
        yp = _matrix(y, n, self.out_dim, y_type, dev, "y")
        rp = (None, 0) if residual is None else _matrix(residual, n, self.out_dim, y_type, dev, "residual")
        pp = (None, 0) if pre is None else _matrix(pre, n, self.out_dim, self.dtype, dev, "pre")
        check("dense_forward", self._lib.dense_forward(
            self._h, *xp, *wp, _vector(bias, self.out_dim, torch.float32, dev, "bias"), *rp, n, *yp,
            OT_BF16 if y_type is torch.bfloat16 else OT_FP32, *pp, _raw_stream(stream, dev, torch)))

    def backward(self, x, w, dy, pre=None, dx=None, dw=None, dbias=None, stream=None) -> None:
        """Gradients from dy (and pre, where the layer has an activation), written whole into those of dx, dw, dbias
        that are given; x may be None without dw, w without dx."""
        torch, dev = self._torch, self._device
        n = dy.shape[0]
        if dw is not None and x is None:
            raise ValueError("dw needs x")
        if dx is not None and w is None:
            raise ValueError("dx needs w")
        if pre is None and self.activation != OT_ACT_NONE:
            raise ValueError("pre: expected what forward() stored")
        none = (None, 0)
        xp = none if x is None else _matrix(x, n, self.in_dim, self.dtype, dev, "x")
        wp = none if w is None else _matrix(w, self.out_dim, self.in_dim, self.dtype, dev, "w")
        dyp = _matrix(dy, n, self.out_dim, self.dtype, dev, "dy")
        pp = none if pre is None else _matrix(pre, n, self.out_dim, self.dtype, dev, "pre")
        dxp = none if dx is None else _matrix(dx, n, self.in_dim, self.dtype, dev, "dx")
        dwp = none if dw is None else _matrix(dw, self.out_dim, self.in_dim, torch.float32, dev, "dw")
        check("dense_backward", self._lib.dense_backward(
            self._h, *xp, *wp, n, *dyp, *pp, *dxp, *dwp, _vector(dbias, self.out_dim, torch.float32, dev, "dbias"),
            _raw_stream(stream, dev, torch)))


class GroupNorm(_Layer):
    """Group norm with an activation over channels-last data (include/layers.h).  x, y, dy and dx are
    (samples, positions, channels), or (samples, channels) with one position; weight, bias, dweight and
    dbias fp32 (channels); stats fp32 (samples, groups, 2).  activation: OT_ACT_*."""
    _destroy = "norm_destroy"

    def __init__(self, channels: int, groups: int, positions: int = 1, precision: int = OT_FP32,
                 activation: int = OT_ACT_NONE, eps: float = 1e-5, max_samples: int = 1024):
        self._open("norm_create", channels, groups, positions, precision, activation, eps, max_samples,
                   precision=precision)
        self.channels, self.groups, self.positions, self.activation = channels, groups, positions, activation

    def _rows(self, t, n: int, what: str):
        """(pointer, leading dimension) of the rows of n samples."""
        shape = t.shape
        if len(shape) == 2 and self.positions == 1:
            return _matrix(t, n, self.channels, self.dtype, self._device, what)
        return _bank(t, n, self.positions, self.channels, self.dtype, self._device, what, "samples")

    def _stats(self, t, n: int):
        if t is None:
            return None
        if t.dtype is not self._torch.float32 or tuple(t.shape) != (n, self.groups, 2) or not t.is_contiguous():
            raise ValueError(f"stats: expected a contiguous torch.float32 tensor of {n} x {self.groups} x 2 values")
        if t.get_device() != self._device:
            raise ValueError(f"stats: expected a tensor on cuda:{self._device}")
        return t.data_ptr()

    def forward(self, x, y, weight=None, bias=None, stats=None, stream=None) -> None:
        """y = act(weight (x - mean) rstd + bias); stats receives mean and rstd for backward().  y may be x."""
        torch, dev, c = self._torch, self._device, self.channels
        n = x.shape[0]
        check("norm_forward", self._lib.norm_forward(
            self._h, *self._rows(x, n, "x"), _vector(weight, c, torch.float32, dev, "weight"),
            _vector(bias, c, torch.float32, dev, "bias"), n, *self._rows(y, n, "y"), self._stats(stats, n),
            _raw_stream(stream, dev, torch)))

    def backward(self, x, stats, dy, weight=None, bias=None, dx=None, dweight=None, dbias=None, stream=None) -> None:
        """Gradients from dy and the forward's stats, written whole into those of dx, dweight, dbias that are
        given.  dx may be dy."""
        torch, dev, c = self._torch, self._device, self.channels
        n = x.shape[0]
        check("norm_backward", self._lib.norm_backward(
            self._h, *self._rows(x, n, "x"), _vector(weight, c, torch.float32, dev, "weight"),
            _vector(bias, c, torch.float32, dev, "bias"), n, self._stats(stats, n), *self._rows(dy, n, "dy"),
            *((None, 0) if dx is None else self._rows(dx, n, "dx")), _vector(dweight, c, torch.float32, dev, "dweight"),
            _vector(dbias, c, torch.float32, dev, "dbias"), _raw_stream(stream, dev, torch)))


class Dropout(_Layer):
    """Dropout whose mask comes from a counter (seed, site, step, row, column) and is never stored
    (include/layers.h).  x, residual, y, dy, dx: (rows, columns).  step: an int, or a device int64 tensor of
    one element, read when the kernel runs (so that replays of a captured call take masks of
    their own)."""
    _destroy = "dropout_destroy"

    def __init__(self, p: float, seed: int, site: int = 0, precision: int = OT_FP32):
        if not 0 <= seed < 1 << 64 or not 0 <= site < 1 << 32:
            raise ValueError("seed: expected a value of 64 bits, site: one of 32")
        self._open("dropout_create", p, seed, site, precision, precision=precision)
        self.p, self.seed, self.site = p, seed, site

    def _step(self, step):
        """(host part, device part)."""
        if not hasattr(step, "data_ptr"):
            step = operator.index(step)
            if not 0 <= step < 1 << 32:
                raise ValueError("step: expected a value of 32 bits")
            return step, None
        if step.dtype is not self._torch.int64 or step.numel() != 1:
            raise ValueError("step: expected an int or an int64 tensor of one element")
        if step.get_device() != self._device:
            raise ValueError(f"step: expected a tensor on cuda:{self._device}")
        return 0, step.data_ptr()

    def forward(self, x, y, step, residual=None, stream=None) -> None:
        """y = residual + (x / (1 - p) where it is kept).  y may be x or the residual."""
        n, cols = x.shape
        dev = self._device
        xp, yp = _matrix(x, n, cols, self.dtype, dev, "x"), _matrix(y, n, cols, self.dtype, dev, "y")
        rp = (None, 0) if residual is None else _matrix(residual, n, cols, self.dtype, dev, "residual")
        check("dropout_forward", self._lib.dropout_forward(self._h, *xp, *rp, n, cols, *yp, *self._step(step),
                                                           _raw_stream(stream, dev, self._torch)))

    def backward(self, dy, dx, step, stream=None) -> None:
        """dx = dy / (1 - p) where forward() of the same step kept x.  dx may be dy."""
        n, cols = dy.shape
        dev = self._device
        dyp, dxp = _matrix(dy, n, cols, self.dtype, dev, "dy"), _matrix(dx, n, cols, self.dtype, dev, "dx")
        check("dropout_backward", self._lib.dropout_backward(self._h, *dyp, n, cols, *dxp, *self._step(step),
                                                             _raw_stream(stream, dev, self._torch)))


# ---- C-named entry points (argument marshalling only) ----------------------------
def reservoir_create(capacity, threshold, x_dim, u_dim, seed, policy=OT_POLICY_RESERVOIR,
                     order_stream=None) -> Reservoir:
    return Reservoir(capacity, threshold, x_dim, u_dim, seed, order_stream, policy)


def reservoir_put(r: Reservoir, x, u, stream=None, accepted=None) -> int:
    return r.put(x, u, stream, accepted)


def reservoir_sample_batch(r: Reservoir, b, slots, x_out=None, u_out=None, stream=None):
    return r.sample_batch(b, slots, x_out, u_out, stream)


def reservoir_end_reception(r: Reservoir) -> None:
    r.end_reception()


def reservoir_stats(r: Reservoir) -> dict:
    return r.stats()


def reservoir_read_meta(r: Reservoir):
    return r.read_meta()


def reservoir_read_rows(r: Reservoir, slots):
    return r.read_rows(slots)


def reservoir_destroy(r: Reservoir) -> None:
    r.close()


def surrogate_create(widths, precision=OT_FP32, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, seed=0,
                     max_batch=1024, flags=0) -> Surrogate:
    return Surrogate(widths, precision, lr, beta1, beta2, eps, seed, max_batch, flags)


def surrogate_set_params(s: Surrogate, layer, W=None, b=None) -> None:
    s.set_params(layer, W, b)


def surrogate_get_params(s: Surrogate, layer):
    return s.get_params(layer)


def reservoir_checkpoint(r: Reservoir) -> np.ndarray:
    return r.checkpoint()


def reservoir_restore(r: Reservoir, blob) -> None:
    r.restore(blob)


def surrogate_checkpoint(s: Surrogate) -> np.ndarray:
    return s.checkpoint()


def surrogate_restore(s: Surrogate, blob) -> None:
    s.restore(blob)


def surrogate_eval_loss(s: Surrogate, x, u, loss, stream=None):
    return s.eval_loss(x, u, loss, stream)


def surrogate_get_grads(s: Surrogate, layer):
    return s.get_grads(layer)


def surrogate_get_adam_state(s: Surrogate, layer):
    return s.get_adam_state(layer)


def surrogate_set_lr(s: Surrogate, lr) -> None:
    s.set_lr(lr)


def surrogate_train_step(s: Surrogate, x, u, stream=None, loss=None) -> None:
    s.train_step(x, u, stream, loss)


def surrogate_predict(s: Surrogate, x, y, stream=None) -> None:
    s.predict(x, y, stream)


def surrogate_predict_noalloc(s: Surrogate, x, y, stream=None) -> None:
    s.predict_noalloc(x, y, stream)


def surrogate_destroy(s: Surrogate) -> None:
    s.close()


def adapters_create(in_dim, out_dim, rank, n_adapters, precision=OT_FP32, max_rows=1024) -> LowRankAdapters:
    return LowRankAdapters(in_dim, out_dim, rank, n_adapters, precision, max_rows)


def adapters_forward(a: LowRankAdapters, x, w, down, up, ids, y, bias=None, scale=None, t=None, relu=False,
                     stream=None) -> None:
    a.forward(x, w, down, up, ids, y, bias, scale, t, relu, stream)


def adapters_backward(a: LowRankAdapters, x, w, down, up, ids, dy, t, ddown, dup, dx=None, scale=None,
                      relu_input=False, stream=None) -> None:
    a.backward(x, w, down, up, ids, dy, t, ddown, dup, dx, scale, relu_input, stream)


def adapters_destroy(a: LowRankAdapters) -> None:
    a.close()


def clip_create(grads, out=None) -> GradientClip:
    return GradientClip(grads, out)


def clip_norm(c: GradientClip, norm, stream=None) -> None:
    c.norm(norm, stream)


def clip_apply(c: GradientClip, max_norm, norm=None, stream=None) -> None:
    c.apply(max_norm, norm, stream)


def clip_destroy(c: GradientClip) -> None:
    c.close()


def adam_create(params, grads, m, v, copies=None, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8,
                steps=0) -> AdamTensors:
    return AdamTensors(params, grads, m, v, copies, lr, beta1, beta2, eps, steps)


def adam_step(a: AdamTensors, max_norm=0.0, norm=None, stream=None) -> None:
    a.step(max_norm, norm, stream)


def adam_set_lr(a: AdamTensors, lr) -> None:
    a.set_lr(lr)


def adam_get_steps(a: AdamTensors) -> int:
    return a.get_steps()


def adam_set_steps(a: AdamTensors, steps) -> None:
    a.set_steps(steps)


def adam_destroy(a: AdamTensors) -> None:
    a.close()


def dense_create(in_dim, out_dim, precision=OT_FP32, activation=OT_ACT_NONE, max_rows=1024) -> DenseLayer:
    return DenseLayer(in_dim, out_dim, precision, activation, max_rows)


def dense_forward(d: DenseLayer, x, w, y, bias=None, residual=None, pre=None, stream=None) -> None:
    d.forward(x, w, y, bias, residual, pre, stream)


def dense_backward(d: DenseLayer, x, w, dy, pre=None, dx=None, dw=None, dbias=None, stream=None) -> None:
    d.backward(x, w, dy, pre, dx, dw, dbias, stream)


def dense_destroy(d: DenseLayer) -> None:
    d.close()


def norm_create(channels, groups, positions=1, precision=OT_FP32, activation=OT_ACT_NONE, eps=1e-5,
                max_samples=1024) -> GroupNorm:
    return GroupNorm(channels, groups, positions, precision, activation, eps, max_samples)


def norm_forward(d: GroupNorm, x, y, weight=None, bias=None, stats=None, stream=None) -> None:
    d.forward(x, y, weight, bias, stats, stream)


def norm_backward(d: GroupNorm, x, stats, dy, weight=None, bias=None, dx=None, dweight=None, dbias=None,
                  stream=None) -> None:
    d.backward(x, stats, dy, weight, bias, dx, dweight, dbias, stream)


def norm_destroy(d: GroupNorm) -> None:
    d.close()


def dropout_create(p, seed, site=0, precision=OT_FP32) -> Dropout:
    return Dropout(p, seed, site, precision)


def dropout_forward(d: Dropout, x, y, step, residual=None, stream=None) -> None:
    d.forward(x, y, step, residual, stream)


def dropout_backward(d: Dropout, dy, dx, step, stream=None) -> None:
    d.backward(dy, dx, step, stream)


def dropout_destroy(d: Dropout) -> None:
    d.close()
