"""Thin Python binding of the dense operators in ``include/som.h``: a linear layer with its epilogue, routing to experts,
the experts' products, layer norm, and their gradients; AdamW over many tensors; matrices in 4 bits and the linear layer on them.

Argument marshalling only, like ``som``: the library computes, PyTorch supplies memory and streams, and there is no
fallback.  Matrices are 2-d CUDA tensors whose rows are contiguous (``stride(1) == 1``); rows may lie further apart.

The calls leave no autograd history, also where their inputs require a gradient: what they return is detached, and the gradients
come from the ``*_backward`` calls (``examples/experts_on_map.py`` chains them; an ``autograd.Function`` around a pair of calls makes
them part of a graph).  Neither do ``AdamW``'s steps, which write the parameters' memory as it is.
"""
from __future__ import annotations

import array
import ctypes
import operator

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


class Fp4Matrix:
    """A matrix in 4 bits (``Layers.quantize_fp4``): ``codes`` uint8 [rows, D / 2], two values a byte, and ``scales``, the blocks' powers of
    two, uint8 in the order that ``som.h`` gives.  Both may be stored and put together again."""

    def __init__(self, codes, scales):
        if codes.dim() != 2 or codes.dtype is not torch.uint8 or scales.dtype is not torch.uint8:
            raise TypeError("codes and scales must be uint8, codes 2-d")
        self.codes, self.scales = codes, scales
        self.shape = (codes.shape[0], 2 * codes.shape[1])

    def record_stream(self, stream):
        self.codes.record_stream(stream)
        self.scales.record_stream(stream)


def _scale_bytes(rows, D):
    """som_fp4_scale_bytes"""
    return (rows + 127) // 128 * ((D + 255) // 256) * 1024


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
            if isinstance(t, (torch.Tensor, Fp4Matrix)):
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

    def _norm(self, x, weight, bias):
        """What norm and its gradient share: type codes, T, D, addresses."""
        if not isinstance(x, torch.Tensor) or x.dim() != 2:
            raise TypeError("x must be a 2-d CUDA tensor")
        kind, t, on = _code(_TYPES, x.dtype, "x's type"), x.dtype, self.device.index
        T, D = x.shape
        wt = weight.dtype if weight is not None else bias.dtype if bias is not None else t
        if wt is not torch.float32 and wt is not t:
            raise TypeError("weight and bias must be float32 or of x's type")
        return (kind, T, D, *_matrix(x, T, D, t, on, "x"), _whole(weight, (D,), wt, on, "weight"), _whole(bias, (D,), wt, on, "bias"), _TYPES[wt], wt)

    def norm(self, x, weight=None, bias=None, residual=None, eps=1e-5, out=None, stream=None):
        """som_norm: layer norm of the rows of x, or of x + residual.  Returns [T, D]; with a residual {"y", "sum"}, the sum being what
        was normed, in x's type.  x: float32, float16 or bfloat16; weight and bias of that type or float32."""
        if stream is not None:
            return self._on(stream, self.norm, x, weight, bias, residual, eps, out)
        kind, T, D, xp, ldx, wp, bp, wt, _ = self._norm(x, weight, bias)
        if out is None:
            out = x.new_empty((T, D))
            yp, ldy = out.data_ptr(), D
        else:
            yp, ldy = _matrix(out, T, D, x.dtype, self.device.index, "out")
        rp, ldr, sp, total = 0, 0, 0, None
        if residual is not None:
            rp, ldr = _matrix(residual, T, D, x.dtype, self.device.index, "residual")
            total = x.new_empty((T, D))
            sp = total.data_ptr()
        rc = self._lib.som_norm(self._h, kind, T, D, xp, ldx, wp, bp, wt, rp, ldr, eps, sp, D, yp, ldy, self._stream())
        if rc:
            self._check(rc, "som_norm")
        return out if residual is None else {"y": out, "sum": total}

    def norm_backward(self, x, weight, dy, bias=None, dsum=None, eps=1e-5, stream=None):
        """som_norm_backward: {"dx"} and, with them, "dweight" and "dbias".  x is what was normed (with a residual: the sum), dsum the
        gradient that the sum got from elsewhere; dx is x's and the residual's gradient alike."""
        if stream is not None:
            return self._on(stream, self.norm_backward, x, weight, dy, bias, dsum, eps)
        kind, T, D, xp, ldx, wp, _, wt, wtype = self._norm(x, weight, bias)
        gp, ldg = _matrix(dy, T, D, x.dtype, self.device.index, "dy")
        sp, lds = (0, 0) if dsum is None else _matrix(dsum, T, D, x.dtype, self.device.index, "dsum")
        out = {"dx": x.new_empty((T, D))}
        if weight is not None:
            out["dweight"] = x.new_empty((D,), dtype=wtype)
        if bias is not None:
            out["dbias"] = x.new_empty((D,), dtype=wtype)
        rc = self._lib.som_norm_backward(self._h, kind, T, D, xp, ldx, wp, wt, gp, ldg, sp, lds, eps, out["dx"].data_ptr(),
                                         out["dweight"].data_ptr() if weight is not None else 0,
                                         out["dbias"].data_ptr() if bias is not None else 0, self._stream())
        if rc:
            self._check(rc, "som_norm_backward")
        return out

    def _fp4(self, q, rows, D, name):
        """Addresses of a matrix in 4 bits."""
        if not isinstance(q, Fp4Matrix):
            raise TypeError("%s must be an Fp4Matrix" % name)
        if D % 32 or not D:
            raise ValueError("%s must have columns in blocks of 32" % name)
        on = self.device.index
        return _whole(q.codes, (rows, D // 2), torch.uint8, on, name), _whole(q.scales, (_scale_bytes(rows, D),), torch.uint8, on, name)

    def quantize_fp4(self, x, stream=None):
        """som_fp4_quantize: x (float32, float16 or bfloat16, columns in blocks of 32) in 4 bits.  Returns an Fp4Matrix."""
        if stream is not None:
            return self._on(stream, self.quantize_fp4, x)
        if not isinstance(x, torch.Tensor) or x.dim() != 2:
            raise TypeError("x must be a 2-d CUDA tensor")
        kind = _code(_TYPES, x.dtype, "x's type")
        T, D = x.shape
        xp, ldx = _matrix(x, T, D, x.dtype, self.device.index, "x")
        if D % 32 or not D:
            raise ValueError("x must have columns in blocks of 32")
        codes, scales = x.new_empty((T, D // 2), dtype=torch.uint8), x.new_empty((_scale_bytes(T, D),), dtype=torch.uint8)
        rc = self._lib.som_fp4_quantize(self._h, kind, T, D, xp, ldx, codes.data_ptr(), scales.data_ptr(), self._stream())
        if rc:
            self._check(rc, "som_fp4_quantize")
        return Fp4Matrix(codes, scales)

    def values_fp4(self, q, dtype=torch.bfloat16, stream=None):
        """som_fp4_values: what an Fp4Matrix stands for, in `dtype` (exact in float32 and bfloat16)."""
        if stream is not None:
            return self._on(stream, self.values_fp4, q, dtype)
        if not isinstance(q, Fp4Matrix):
            raise TypeError("q must be an Fp4Matrix")
        T, D = q.shape
        kind = _code(_TYPES, dtype, "dtype")
        cp, sp = self._fp4(q, T, D, "q")
        out = q.codes.new_empty((T, D), dtype=dtype)
        rc = self._lib.som_fp4_values(self._h, kind, T, D, cp, sp, out.data_ptr(), D, self._stream())
        if rc:
            self._check(rc, "som_fp4_values")
        return out

    def linear_fp4(self, x, weight, bias=None, residual=None, act="none", gated=False, out=None, stream=None):
        """som_fp4_linear: ``linear`` with x, quantised within the call, and weight (an Fp4Matrix) in 4 bits.  Returns [T, F] of x's type."""
        if stream is not None:
            return self._on(stream, self.linear_fp4, x, weight, bias, residual, act, gated, out)
        kind = self._half(x)
        if not isinstance(weight, Fp4Matrix):
            raise TypeError("weight must be an Fp4Matrix")
        T, D = x.shape
        rows, on, t = weight.shape[0], self.device.index, x.dtype
        if gated and rows % 2:
            raise ValueError("a gated weight has an even number of rows")
        F = rows // 2 if gated else rows
        xp, ldx = _matrix(x, T, D, t, on, "x")
        cp, sp = self._fp4(weight, rows, D, "weight")
        if out is None:
            out = x.new_empty((T, F))
            yp, ldy = out.data_ptr(), F
        else:
            yp, ldy = _matrix(out, T, F, t, on, "out")
        rp, ldr = (0, 0) if residual is None else _matrix(residual, T, F, t, on, "residual")
        rc = self._lib.som_fp4_linear(self._h, kind, _code(_ACTS, act, "act"), bool(gated), T, D, F, xp, ldx, cp, sp,
                                      _whole(bias, (rows,), t, on, "bias"), rp, ldr, yp, ldy, self._stream())
        if rc:
            self._check(rc, "som_fp4_linear")
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


class _Tensor(ctypes.Structure):
    """som_adamw_tensor"""
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("copy", ctypes.c_void_p), ("m", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("exponents", ctypes.c_void_p), ("n", ctypes.c_int64), ("number", ctypes.c_uint32), ("first_chunk", ctypes.c_uint32)]


class _Step(ctypes.Structure):
    """som_adamw_step"""
    _fields_ = [("rate", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double), ("decay", ctypes.c_double),
                ("step", ctypes.c_int64), ("rate_at", ctypes.c_void_p), ("step_at", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("seed", ctypes.c_uint32)]


# of many tensors, by map(): a loop over the same checks takes up to twice the time
_address, _numel, _contiguous, _gpu = torch.Tensor.data_ptr, torch.Tensor.numel, torch.Tensor.is_contiguous, torch.Tensor.get_device
_dtype, _shape = operator.attrgetter("dtype"), operator.attrgetter("shape")


class AdamW:
    """AdamW over many tensors (``som_adamw``): it keeps their moments, in 32 bits or in 8, and ``step`` moves all of them in one launch (one for
    each combination of types, and for each 500 tensors).

    params: contiguous CUDA tensors (float32, float16 or bfloat16) on the handle's device that share no memory; copies: for each float32
    parameter a 16-bit tensor that gets its new value, or None.  Both keep their memory: a step refuses one whose memory, type or size was
    exchanged (``p.data = ...``, ``Module.half``), and a new optimiser takes over with ``state`` and ``load``.  The moments are zeroed on the current stream.  The first step has number 1."""

    def __init__(self, layers, params, copies=None, bits=32):
        if bits not in (8, 32):
            raise ValueError("bits must be 8 or 32")
        self._layers, self.bits, self.params, self.steps = layers, bits, tuple(params), 0
        self.copies = (None,) * len(self.params) if copies is None else tuple(copies)
        if len(self.copies) != len(self.params):
            raise ValueError("copies must be as many as params")
        on, spans, groups = layers.device.index, [], {}
        for i, (p, c) in enumerate(zip(self.params, self.copies)):
            _code(_TYPES, p.dtype, "a parameter's type")
            _whole(p, p.shape, p.dtype, on, "params[%d]" % i)
            spans.append((p.data_ptr(), p.data_ptr() + p.numel() * p.element_size()))
            if c is not None:
                if p.dtype is not torch.float32 or c.dtype not in (torch.float16, torch.bfloat16):
                    raise TypeError("a copy is a 16-bit tensor beside a float32 parameter")
                _whole(c, p.shape, c.dtype, on, "copies[%d]" % i)
                spans.append((c.data_ptr(), c.data_ptr() + c.numel() * c.element_size()))
            groups.setdefault((p.dtype, None if c is None else c.dtype), []).append(i)
        spans = sorted(s for s in spans if s[0] < s[1])
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            raise ValueError("params and copies must not share memory")
        if bits == 32:
            self._m = [torch.zeros_like(p, dtype=torch.float32) for p in self.params]
            self._v = [torch.zeros_like(p, dtype=torch.float32) for p in self.params]
            self._exponents = [None] * len(self.params)
        else:
            self._m = [torch.zeros_like(p, dtype=torch.uint8) for p in self.params]
            self._v = [torch.zeros_like(p, dtype=torch.uint8) for p in self.params]
            self._exponents = [p.new_zeros((2, -(-p.numel() // 256)), dtype=torch.uint8) for p in self.params]
        self._groups = []
        # what the tables say of the parameters and their copies
        self._written = [t for t in (*self.params, *self.copies) if t is not None]
        self._homes = [list(map(f, self._written)) for f in (_address, _dtype, _numel)]
        # where moments() puts the values: pieces of one tensor, each on 16 bytes
        self._places, self._all = [], 0
        for p in self.params:
            self._places.append((p.shape, p.stride(), self._all))
            self._all += -(-p.numel() // 8) * 8
        for (pt, ct), which in groups.items():
            table = (_Tensor * len(which))()
            for t, i in zip(table, which):
                p, c, e = self.params[i], self.copies[i], self._exponents[i]
                t.param, t.copy, t.m, t.v = p.data_ptr(), 0 if c is None else c.data_ptr(), self._m[i].data_ptr(), self._v[i].data_ptr()
                t.exponents, t.n, t.number = 0 if e is None else e.data_ptr(), p.numel(), i
            # the gradients' addresses in it, and their shapes
            column = memoryview(table).cast("B").cast("Q")[_Tensor.grad.offset // 8::ctypes.sizeof(_Tensor) // 8]
            self._groups.append((pt, -1 if ct is None else _TYPES[ct], which, table, column, [self.params[i].shape for i in which]))

    def _record(self, stream, more=()):
        for t in (*self.params, *self.copies, *self._m, *self._v, *self._exponents, *more):
            if t is not None:
                t.record_stream(stream)

    def step(self, grads, rate=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, decay=0.01, step=None, scale=None, seed=None, stream=None):
        """som_adamw: one step.  grads: as params, contiguous, float32 or 16 bits (beside 16-bit parameters their type); parameters of one type
        have gradients of one type.  rate: a number, or a float32 CUDA tensor of one element; step: its number, by default one more than the
        last, or an int64 CUDA tensor of one element; scale: None, or a float32 CUDA tensor of one element that multiplies the gradients (where
        it is an infinity or NaN the step changes no tensor, but counts: the host does not learn of it, and a caller who does gives ``step``).
        seed: of the random bits that round 8-bit moments, by default the step's number."""
        L = self._layers
        if stream is not None:
            if stream.device != L.device:
                raise ValueError("the stream is on %s, the handle on %s" % (stream.device, L.device))
            with torch.cuda.stream(stream):
                self.step(grads, rate, beta1, beta2, eps, decay, step, scale, seed)
            return self._record(stream, [*grads, *(t for t in (rate, step, scale) if isinstance(t, torch.Tensor))])
        if len(grads) != len(self.params):
            raise ValueError("there must be as many grads as params")
        on, mine = L.device.index, self._written
        address, dtype, numel = self._homes
        if list(map(_address, mine)) != address or list(map(_dtype, mine)) != dtype or list(map(_numel, mine)) != numel or not all(map(_contiguous, mine)):
            raise ValueError("the memory of a parameter or copy was exchanged after the optimiser was made")
        how = _Step(beta1=beta1, beta2=beta2, eps=eps, decay=decay)
        if isinstance(rate, torch.Tensor):
            how.rate_at = _whole(rate.view(1) if rate.dim() == 0 else rate, (1,), torch.float32, on, "rate")
        else:
            how.rate = rate
        if isinstance(step, torch.Tensor):
            how.step_at = _whole(step.view(1) if step.dim() == 0 else step, (1,), torch.int64, on, "step")
        else:
            how.step = step = self.steps + 1 if step is None else int(step)
            if step < 1:
                raise ValueError("step must be at least 1")
        if scale is not None:
            how.scale = _whole(scale.view(1) if scale.dim() == 0 else scale, (1,), torch.float32, on, "scale")
        how.seed = (seed if seed is not None else 0 if isinstance(step, torch.Tensor) else step) & 0xFFFFFFFF
        kinds = []
        for pt, _, which, _, column, shapes in self._groups:  # all is checked before anything is changed
            some = [grads[i] for i in which]
            gt = some[0].dtype
            if gt is not torch.float32 and (gt is not pt and pt is not torch.float32 or gt not in _TYPES):
                raise TypeError("gradients must be float32 or 16 bits, beside 16-bit parameters of their type")
            if list(map(_dtype, some)) != [gt] * len(some) or list(map(_shape, some)) != shapes or list(map(_gpu, some)) != [on] * len(some) or not all(map(_contiguous, some)):
                for g, shape, i in zip(some, shapes, which):
                    _whole(g, shape, gt, on, "grads[%d]" % i)
            column[:] = array.array("Q", map(_address, some))
            kinds.append(_TYPES[gt])
        for (pt, ct, which, table, _, _), gt in zip(self._groups, kinds):
            rc = L._lib.som_adamw(L._h, _TYPES[pt], gt, ct, self.bits, len(table), table, ctypes.byref(how), L._stream())
            if rc:
                L._check(rc, "som_adamw")
        if not isinstance(step, torch.Tensor):
            self.steps = step

    def moments(self, stream=None):
        """The moments as two lists of tensors of the parameters' shapes: with bits=32 the moments themselves (float32), with bits=8 their
        values (som_adamw_moments, bfloat16, which holds them exactly)."""
        if self.bits == 32:
            return list(self._m), list(self._v)
        L = self._layers
        if stream is not None:
            if stream.device != L.device:
                raise ValueError("the stream is on %s, the handle on %s" % (stream.device, L.device))
            before = torch.cuda.current_stream(L.device)
            with torch.cuda.stream(stream):
                out = self.moments()
            self._record(stream)
            for t in (*out[0], *out[1]):
                t.record_stream(before)
            return out
        m, v = torch.empty(self._all, dtype=torch.bfloat16, device=L.device), torch.empty(self._all, dtype=torch.bfloat16, device=L.device)
        for _, _, which, table, _, _ in self._groups:
            to, mp, vp = ctypes.c_void_p * len(which), m.data_ptr(), v.data_ptr()
            rc = L._lib.som_adamw_moments(L._h, len(table), table, to(*[mp + 2 * self._places[i][2] for i in which]),
                                          to(*[vp + 2 * self._places[i][2] for i in which]), L._stream())
            if rc:
                L._check(rc, "som_adamw_moments")
        return [m.as_strided(*place) for place in self._places], [v.as_strided(*place) for place in self._places]

    def state(self):
        """What ``load`` takes, for a checkpoint: the moments' own memory, with bits=8 as pairs of codes and exponents."""
        if self.bits == 32:
            return list(self._m), list(self._v)
        return tuple([(c, e[k]) for c, e in zip(codes, self._exponents)] for k, codes in enumerate((self._m, self._v)))

    def load(self, m, v, steps=0):
        """Takes over moments as ``state`` gives them, and the number of steps made."""
        if len(m) != len(self.params) or len(v) != len(self.params):
            raise ValueError("there must be as many moments as params")
        for k, (mine, given) in enumerate(((self._m, m), (self._v, v))):
            for i, (to, x) in enumerate(zip(mine, given)):
                code, e = x if self.bits == 8 else (x, None)
                if code.dtype is not to.dtype or code.numel() != to.numel():
                    raise ValueError("moment %d must have %d elements of %s" % (i, to.numel(), to.dtype))
                if e is not None and (e.dtype is not torch.uint8 or e.numel() != self._exponents[i][k].numel()):
                    raise ValueError("moment %d must have %d exponents" % (i, self._exponents[i][k].numel()))
        for k, (mine, given) in enumerate(((self._m, m), (self._v, v))):
            for i, (to, x) in enumerate(zip(mine, given)):
                code, e = x if self.bits == 8 else (x, None)
                to.copy_(code.reshape(to.shape))
                if e is not None:
                    self._exponents[i][k].copy_(e.reshape(-1))
        self.steps = int(steps)
