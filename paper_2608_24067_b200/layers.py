"""Thin Python binding of the dense operators in ``include/som.h``: a linear layer with its epilogue, routing to experts,
the experts' products, and their gradients.

Argument marshalling only, like ``som``: the library computes, PyTorch supplies memory and streams, and there is no
fallback.  Matrices are 2-d CUDA tensors whose rows are contiguous (``stride(1) == 1``); rows may lie further apart.

The calls leave no autograd history, also where their inputs require a gradient: what they return is detached, and the gradients
come from the ``*_backward`` calls (``examples/experts_on_map.py`` chains them; an ``autograd.Function`` around a pair of calls makes
them part of a graph).
"""
from __future__ import annotations

import ctypes

import torch

from .som import SOM_OK, SomError, load_library

# the current stream's address without building a Stream object (2 us a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)

_TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
_SCORES = {"softmax": 0, "sigmoid": 1}
_PRODUCTS = {"forward": 0, "dz": 1, "dz of experts": 2, "dx": 3, "dw": 4, "route": 5}
_TILES = {"128x128": 0, "128x256": 1, "256x256": 2, "warp a token": 0, "four lanes a token": 1}


def _elsewhere(t, index, name):
    """Raises: t is not on the handle's device, GPU `index`."""
    if not t.is_cuda:
        raise TypeError("%s must be a CUDA tensor" % name)
    raise ValueError("%s is on %s, the handle on cuda:%d" % (name, t.device, index))


def _matrix(t, rows, cols, dtype, index, name):
    """(address, distance of rows) of a [rows][cols] tensor on GPU `index`."""
    if t.get_device() != index:
        _elsewhere(t, index, name)
    if t.dtype is not dtype:
        raise TypeError("%s must be a 2-d CUDA tensor of %s with contiguous rows" % (name, dtype))
    if t.shape != (rows, cols):
        raise ValueError("%s must have shape %s, not %s" % (name, (rows, cols), tuple(t.shape)))
    far, near = t.stride()
    if near != 1 and cols > 1:
        raise TypeError("%s must be a 2-d CUDA tensor of %s with contiguous rows" % (name, dtype))
    return t.data_ptr(), far if rows > 1 else cols


def _whole(t, shape, dtype, index, name):
    """Address of a contiguous tensor on GPU `index`; 0 for None."""
    if t is None:
        return 0
    if t.get_device() != index:
        _elsewhere(t, index, name)
    if t.dtype is not dtype or not t.is_contiguous():
        raise TypeError("%s must be a contiguous CUDA tensor of %s" % (name, dtype))
    if t.shape != shape:
        raise ValueError("%s must have shape %s, not %s" % (name, shape, tuple(t.shape)))
    return t.data_ptr()


def _code(table, key, name):
    try:
        return table[key]
    except KeyError:
        raise ValueError("%s must be one of %s" % (name, sorted(str(k) for k in table))) from None


class Layers:
    """Handle of the dense operators on one device (``som_layers_create``): workspace and status.

    Calls on one handle must not overlap, neither on the GPU (issue them on one stream or order the streams) nor on the host: one
    thread at a time, as a call may grow the workspace.  Calls run on the current
    stream, or on ``stream``: the caller orders that stream behind what writes the inputs, and what reads the outputs behind it."""

    def __init__(self, device=None):
        self._lib = load_library()
        self._h = ctypes.c_void_p()
        self.device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        with torch.cuda.device(self.device):
            rc = self._lib.som_layers_create(ctypes.byref(self._h))
        if rc != SOM_OK:
            self._h = ctypes.c_void_p()
            raise SomError(rc, "som_layers_create")

    def _check(self, rc: int, where: str):
        if rc != SOM_OK:
            raise SomError(rc, where, self._lib.som_layers_last_cuda_error(self._h))

    def _on(self, stream, call, *args, **kw):
        """call(*args, **kw) on `stream`.  Its outputs are that stream's memory: memory of the current stream may have work before it
        that was queued when it belonged to another tensor.  And neither what the call is given nor what it returns is handed
        out again before both streams are done with it."""
        if stream.device != self.device:
            raise ValueError("the stream is on %s, the handle on %s" % (stream.device, self.device))
        before = torch.cuda.current_stream(self.device)
        with torch.cuda.stream(stream):
            out = call(*args, **kw)
        for t in (*args, *kw.values()):
            if isinstance(t, torch.Tensor):
                t.record_stream(stream)
        for t in out.values() if isinstance(out, dict) else (out,):
            t.record_stream(before)
        return out

    def _stream(self, stream=None) -> int:
        if stream is not None:
            return stream.cuda_stream
        if _raw_stream is not None:
            return _raw_stream(self.device.index)
        return torch.cuda.current_stream(self.device).cuda_stream

    def _half(self, x):
        """The type code of x, which has to be a 16-bit matrix on the handle's device."""
        if not isinstance(x, torch.Tensor) or x.dtype not in (torch.float16, torch.bfloat16) or x.dim() != 2:
            raise TypeError("x must be a 2-d float16 or bfloat16 CUDA tensor")
        if x.device != self.device:
            raise ValueError("x is on %s, the handle on %s" % (x.device, self.device))
        return _TYPES[x.dtype]

    def _unit(self, x, weight, bias, gated):
        """What linear and its gradient share: type, T, D, F and the rows of weight, addresses."""
        kind = self._half(x)
        T, D = x.shape
        if weight.dim() != 2:
            raise ValueError("weight must be 2-d")
        rows, on = weight.shape[0], self.device.index
        if gated and rows % 2:
            raise ValueError("a gated weight has an even number of rows")
        xp, ldx = _matrix(x, T, D, x.dtype, on, "x")
        return (kind, T, D, rows // 2 if gated else rows, rows, xp, ldx, _whole(weight, (rows, D), x.dtype, on, "weight"),
                0 if bias is None else _whole(bias, (rows,), x.dtype, on, "bias"))

    def linear(self, x, weight, bias=None, residual=None, act="none", gated=False, out=None, stream=None):
        """som_linear: act(x weight^T + bias) + residual; gated: weight's first half of rows is activated and multiplies
        the products of the second.  Returns [T, F]."""
        if stream is not None:
            return self._on(stream, self.linear, x, weight, bias, residual, act, gated, out)
        kind, T, D, F, rows, xp, ldx, wp, bp = self._unit(x, weight, bias, gated)
        if out is None:
            out = x.new_empty((T, F))
            yp, ldy = out.data_ptr(), F
        else:
            yp, ldy = _matrix(out, T, F, x.dtype, self.device.index, "out")
        rp, ldr = (0, 0) if residual is None else _matrix(residual, T, F, x.dtype, self.device.index, "residual")
        rc = self._lib.som_linear(self._h, kind, _code(_ACTS, act, "act"), bool(gated), T, D, F, xp, ldx, wp, bp, rp, ldr, yp, ldy,
                                  self._stream())
        if rc:
            self._check(rc, "som_linear")
        return out

    def linear_backward(self, x, weight, dy, bias=None, act="none", gated=False, stream=None):
        """som_linear_backward: {"dx", "dweight"} and, with a bias, "dbias" (the residual's gradient is dy)."""
        if stream is not None:
            return self._on(stream, self.linear_backward, x, weight, dy, bias, act, gated)
        kind, T, D, F, rows, xp, ldx, wp, bp = self._unit(x, weight, bias, gated)
        gp, ldg = _matrix(dy, T, F, x.dtype, self.device.index, "dy")
        out = {"dx": x.new_empty((T, D)), "dweight": x.new_empty((rows, D))}
        if bias is not None:
            out["dbias"] = x.new_empty((rows,))
        rc = self._lib.som_linear_backward(self._h, kind, _code(_ACTS, act, "act"), bool(gated), T, D, F, xp, ldx, wp, bp, gp, ldg,
                                           out["dx"].data_ptr(), out["dweight"].data_ptr(),
                                           out["dbias"].data_ptr() if bias is not None else 0, self._stream())
        if rc:
            self._check(rc, "som_linear_backward")
        return out

    def _logits(self, logits):
        """Type code, T, E, address and distance of rows."""
        if not isinstance(logits, torch.Tensor) or logits.dim() != 2:
            raise TypeError("logits must be a 2-d CUDA tensor")
        kind = _code(_TYPES, logits.dtype, "logits' type")
        if logits.device != self.device:
            raise ValueError("logits are on %s, the handle on %s" % (logits.device, self.device))
        T, E = logits.shape
        return (kind, T, E, *_matrix(logits, T, E, logits.dtype, self.device.index, "logits"))

    def route(self, logits, k, score="softmax", bias=None, groups=1, top_groups=1, group_best=1, renorm=True, scale=1.0,
              stream=None):
        """som_route: {"weights" fp32 [T, k], "indices" int32 [T, k], "counts" int32 [E]}."""
        if stream is not None:
            return self._on(stream, self.route, logits, k, score, bias, groups, top_groups, group_best, renorm, scale)
        kind, T, E, lp, ld = self._logits(logits)
        new = logits.new_empty
        weights, indices, counts = new((T, k), dtype=torch.float32), new((T, k), dtype=torch.int32), new((E,), dtype=torch.int32)
        rc = self._lib.som_route(self._h, kind, _code(_SCORES, score, "score"), T, E, k, lp, ld,
                                 0 if bias is None else _whole(bias, (E,), torch.float32, self.device.index, "bias"), groups, top_groups, group_best,
                                 bool(renorm), scale, weights.data_ptr(), indices.data_ptr(), counts.data_ptr(), self._stream())
        if rc:
            self._check(rc, "som_route")
        return {"weights": weights, "indices": indices, "counts": counts}

    def route_backward(self, logits, indices, dweights, score="softmax", renorm=True, scale=1.0, stream=None):
        """som_route_backward: the logits' gradient [T, E]."""
        if stream is not None:
            return self._on(stream, self.route_backward, logits, indices, dweights, score, renorm, scale)
        kind, T, E, lp, ld = self._logits(logits)
        k = indices.shape[-1]
        out = logits.new_empty((T, E))
        rc = self._lib.som_route_backward(self._h, kind, _code(_SCORES, score, "score"), T, E, k, lp, ld,
                                          _whole(indices, (T, k), torch.int32, self.device.index, "indices"),
                                          _whole(dweights, (T, k), torch.float32, self.device.index, "dweights"), bool(renorm), scale,
                                          out.data_ptr(), self._stream())
        if rc:
            self._check(rc, "som_route_backward")
        return out

    def _experts(self, x, indices, weights, w1, w2, b1, b2, gated):
        kind = self._half(x)
        if w1.dim() != 3 or w2.dim() != 3 or indices.dim() != 2:
            raise ValueError("w1 and w2 must be 3-d, indices 2-d")
        T, D = x.shape
        E, rows = w1.shape[:2]
        if gated and rows % 2:
            raise ValueError("a gated w1 has an even number of rows")
        I = rows // 2 if gated else rows
        k = indices.shape[1]
        t, wt, on = x.dtype, weights.dtype, self.device.index
        if wt is not torch.float32 and wt is not t:
            raise TypeError("weights must be float32 or of x's type")
        xp, ldx = _matrix(x, T, D, t, on, "x")
        return kind, T, E, k, D, I, rows, (xp, ldx, _whole(indices, (T, k), torch.int32, on, "indices"),
                                           _whole(weights, (T, k), wt, on, "weights"), _TYPES[wt],
                                           _whole(w1, (E, rows, D), t, on, "w1"), _whole(b1, (E, rows), t, on, "b1"),
                                           _whole(w2, (E, D, I), t, on, "w2"), _whole(b2, (E, D), t, on, "b2"))

    def experts(self, x, indices, weights, w1, w2, b1=None, b2=None, residual=None, act="silu", gated=True, out=None, stream=None):
        """som_experts: residual + sum over a token's experts of weight * (w2 act(w1 x + b1) + b2).  Returns [T, D]."""
        if stream is not None:
            return self._on(stream, self.experts, x, indices, weights, w1, w2, b1, b2, residual, act, gated, out)
        kind, T, E, k, D, I, rows, p = self._experts(x, indices, weights, w1, w2, b1, b2, gated)
        if out is None:
            out = x.new_empty((T, D))
            yp, ldy = out.data_ptr(), D
        else:
            yp, ldy = _matrix(out, T, D, x.dtype, self.device.index, "out")
        rp, ldr = (0, 0) if residual is None else _matrix(residual, T, D, x.dtype, self.device.index, "residual")
        rc = self._lib.som_experts(self._h, kind, _code(_ACTS, act, "act"), bool(gated), T, E, k, D, I, *p, rp, ldr, yp, ldy,
                                   self._stream())
        if rc:
            self._check(rc, "som_experts")
        return out

    def experts_backward(self, x, indices, weights, w1, w2, dy, b1=None, b2=None, act="silu", gated=True, stream=None):
        """som_experts_backward: {"dx", "dweights", "dw1", "dw2"} and, with biases, "db1", "db2"."""
        if stream is not None:
            return self._on(stream, self.experts_backward, x, indices, weights, w1, w2, dy, b1, b2, act, gated)
        kind, T, E, k, D, I, rows, p = self._experts(x, indices, weights, w1, w2, b1, b2, gated)
        gp, ldg = _matrix(dy, T, D, x.dtype, self.device.index, "dy")
        new = x.new_empty
        out = {"dx": new((T, D)), "dweights": weights.new_empty((T, k)), "dw1": new((E, rows, D)), "dw2": new((E, D, I))}
        if b1 is not None:
            out["db1"] = new((E, rows))
        if b2 is not None:
            out["db2"] = new((E, D))
        rc = self._lib.som_experts_backward(self._h, kind, _code(_ACTS, act, "act"), bool(gated), T, E, k, D, I, *p, gp, ldg,
                                            out["dx"].data_ptr(), out["dweights"].data_ptr(), out["dw1"].data_ptr(),
                                            out["db1"].data_ptr() if b1 is not None else 0, out["dw2"].data_ptr(),
                                            out["db2"].data_ptr() if b2 is not None else 0, self._stream())
        if rc:
            self._check(rc, "som_experts_backward")
        return out

    def device_flags(self, stream=None) -> int:
        """som_layers_device_flags: status of what earlier calls skipped on the device (0 = nothing); synchronises."""
        return int(self._lib.som_layers_device_flags(self._h, self._stream(stream)))

    def launch_count(self) -> int:
        return int(self._lib.som_layers_launch_count(self._h))

    def rounds(self, product, tiles) -> int:
        """som_layers_rounds: the most rounds of this form that a block made for this product (or "route") so far, 0 = none."""
        return int(self._lib.som_layers_rounds(self._h, _code(_PRODUCTS, product, "product"), _code(_TILES, tiles, "tiles")))

    def destroy(self):
        if self._h:
            self._lib.som_layers_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass
