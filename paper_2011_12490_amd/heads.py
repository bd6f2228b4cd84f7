"""Operators that train a mixture of heads (include/derf.h, "Operators of training").

Samples are routed to their heads and back, the heads' layers run on the sorted
rows, and AdamW updates the weights: a training step of the decomposition of
Sec. 3.2 is

    r = route(ids, num_heads)                  # ids [T, k]: each sample's heads
    x0 = dispatch(x, r)
    y0 = linear(x0, w0, b0, r.offsets, relu=True)
    y1 = linear(y0, w1, b1, r.offsets)
    out = combine(y1, r, weights)              # weights [T, k]
    ...                                        # dout: the loss's gradient
    dy1, dweights = combine_backward(dout, y1, r, weights)
    dy0, dw1, db1 = linear_backward(dy1, y0, w1, r.offsets)
    dx0, dw0, db0 = linear_backward(dy0, x0, w0, r.offsets, y=y0)
    dx = dispatch_backward(dx0, r)
    optimizer.step()

gated and gated_backward take the place of linear in heads of gated layers, lookup brings
the samples' rows of a table (a code for each image) and lookup_backward their gradients,
and Muon takes hidden layers' weights where AdamW takes the rest.

Argument checks and marshalling only; all work is done by libderf.so, on torch's
current stream of the tensors' device.  Tensors are float32 or bfloat16, of any
row stride (the layers': below 2^21 elements), on one GPU; what does not fit, and
what the library itself refuses, raises ValueError before any GPU work.  An out=
tensor shares no memory with the call's other tensors (gated layers, lookups and
orthogonalise check that).  No autograd graph is recorded: while autograd records
(torch.is_grad_enabled()), a tensor that requires a gradient is refused, but for the
optimizer's, since its gradient would be lost; a tensor with a forward-mode tangent is
refused everywhere, for the same reason.
"""
from __future__ import annotations

import ctypes
import functools
from typing import List, NamedTuple, Optional, Sequence

import torch
from torch.autograd import forward_ad

from . import derf

MAX_TOP_K = 16
MOMENT_BLOCK = 256  # values of an 8-bit moment that share a scale
ACTIVATIONS = {"silu": 0, "gelu": 1, "relu": 2, "sigmoid": 3}  # derf_activation
_PRECISION = {torch.float32: derf.DERF_PREC_FP32, torch.bfloat16: derf.DERF_PREC_BF16}


class Routing(NamedTuple):
    """Where (sample, slot) pairs lie when sorted by head (derf_route): offsets
    int32 [num_heads + 1], pair int32 [T * k], row int32 [T, k]."""
    offsets: torch.Tensor
    pair: torch.Tensor
    row: torch.Tensor
    num_heads: int


class Refused(derf.DerfError, ValueError):
    """Arguments that the library refuses (DERF_ERR_INVALID_ARG)."""


def _check(status: int, name: str) -> None:
    if status != derf.DERF_OK:
        raise (Refused if status == derf.DERF_ERR_INVALID_ARG else derf.DerfError)(status, name)


_entry = {}  # entry points by name


def _call(name: str, device: torch.device, *args) -> None:
    """Call an entry point with the device's current stream as its last argument."""
    f = _entry.get(name)
    if f is None:
        f = _entry[name] = getattr(derf.lib(), name)
    index = device.index
    stream = torch._C._cuda_getCurrentRawStream(index)  # without the Stream object
    if torch._C._cuda_getDevice() == index:
        status = f(*args, stream)
    else:
        with torch.cuda.device(index):
            status = f(*args, stream)
    if status != derf.DERF_OK:
        _check(status, name)


@functools.lru_cache(maxsize=256)
def _workspace_bytes(name: str, *sizes: int) -> int:
    return getattr(derf.lib(), name)(*sizes)


def _ptr(x: Optional[torch.Tensor]):
    return None if x is None else x.data_ptr()


def _no_graph(x, name) -> None:
    """Refuse a tensor that requires a gradient, which autograd would silently not get."""
    if torch.is_grad_enabled():
        raise ValueError("%s requires a gradient and autograd would not see it: detach it or call under "
                         "torch.no_grad()" % name)


def _no_tangent(x, name) -> None:
    """Refuse a tensor with a forward-mode tangent, which the results would be without."""
    if forward_ad.unpack_dual(x).tangent is not None:
        raise ValueError("%s has a forward-mode tangent, which the result would not have: pass its primal" % name)


def _not_negated(x, name) -> None:
    """Refuse a view whose sign torch has yet to change (the imaginary part of a conjugate): its
    memory holds other values.  Only single values a row pass the checks of strides so."""
    if x.is_neg():
        raise ValueError("%s is a lazily negated view: call resolve_neg() on it" % name)


def _array(x, name, dtype, shape, device=None, leaf=False) -> None:
    """Check a contiguous GPU array of a given type and shape; leaf: autograd may follow it.
    device: a GPU, but for an optimizer's tensors (leaf)."""
    if not isinstance(x, torch.Tensor):
        raise ValueError("%s must be a torch tensor" % name)
    if ((device is None or leaf) and not x.is_cuda) or (device is not None and x.device != device):
        raise ValueError("%s must be a tensor on %s" % (name, device or "a GPU"))
    if x.dtype != dtype:
        raise ValueError("%s must be %s, got %s" % (name, dtype, x.dtype))
    if x.shape != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(x.shape)))
    if not x.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if shape and shape[-1] == 1 and x.numel() == 1:
        _not_negated(x, name)
    if x.requires_grad and not leaf:
        _no_graph(x, name)
    if forward_ad._current_level >= 0:  # tangents are there within a level only
        _no_tangent(x, name)


def _rows(x, name, shape=None, dtype=None, device=None) -> int:
    """Check an array of rows (elements of a row side by side, rows any distance
    apart that does not make them overlap); returns that distance.  device: a GPU."""
    if not isinstance(x, torch.Tensor):
        raise ValueError("%s must be a torch tensor" % name)
    if x.device != device if device is not None else not x.is_cuda:
        raise ValueError("%s must be a tensor on %s" % (name, device or "a GPU"))
    if x.dtype not in _PRECISION or (dtype is not None and x.dtype != dtype):
        raise ValueError("%s must be %s, got %s" % (name, dtype or "float32 or bfloat16", x.dtype))
    size = x.shape
    if len(size) != 2 or size[1] < 1 or (shape is not None and size != shape):
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape) if shape else "[rows, dim]",
                                                           tuple(size)))
    stride, step = x.stride()
    if step != 1 and size[1] > 1:
        raise ValueError("%s: the elements of a row must lie side by side" % name)
    if size[1] == 1:
        _not_negated(x, name)
    if x.requires_grad:
        _no_graph(x, name)
    if forward_ad._current_level >= 0:
        _no_tangent(x, name)
    if size[0] <= 1:  # no next row
        return size[1]
    if stride < size[1]:
        raise ValueError("%s: rows overlap" % name)
    return stride


def _out_rows(out, name, rows, dim, like):
    if out is None:
        return like.new_empty((rows, dim)), dim
    return out, _rows(out, name, (rows, dim), like.dtype, like.device)


def _out_array(out, name, shape, device):
    if out is None:
        return torch.empty(shape, dtype=torch.float32, device=device)
    _array(out, name, torch.float32, shape, device)
    return out


def _workspace(need: int, device):
    return torch.empty((need,), dtype=torch.uint8, device=device) if need else None


def _routing(routing, device):
    if not isinstance(routing, Routing):
        raise ValueError("routing must be a Routing")
    row = routing.row
    if not isinstance(row, torch.Tensor) or row.dim() != 2:
        raise ValueError("routing.row must be a tensor [T, k]")
    if row.dtype != torch.int32 or row.device != device or not row.is_contiguous():
        raise ValueError("routing.row must be a contiguous int32 tensor on %s" % device)
    return row.shape


def route(ids: torch.Tensor, num_heads: int) -> Routing:
    """Sort the pairs of ids (int32 [T, k]) stably by head; an id outside
    [0, num_heads) is a pair without a head."""
    if not isinstance(ids, torch.Tensor) or ids.dim() != 2:
        raise ValueError("ids must be a tensor [T, k]")
    _array(ids, "ids", torch.int32, ids.shape)
    T, k = ids.shape
    need = _workspace_bytes("derf_route_workspace", T, k, num_heads)
    if need < 0:
        raise ValueError("invalid sizes: %d samples, %d pairs each, %d heads" % (T, k, num_heads))
    dev = ids.device
    offsets, pair, row = ids.new_empty((num_heads + 1,)), ids.new_empty((T * k,)), torch.empty_like(ids)
    ws = _workspace(need, dev)
    _call("derf_route", dev, ids.data_ptr(), T, k, num_heads, offsets.data_ptr(), pair.data_ptr(),
          row.data_ptr(), _ptr(ws), need)
    return Routing(offsets, pair, row, num_heads)


def dispatch(x: torch.Tensor, routing: Routing, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Samples' rows [T, D] in the heads' order [T * k, D]; zero without a head."""
    stride = _rows(x, "x")
    T, k = _routing(routing, x.device)
    if x.shape[0] != T:
        raise ValueError("x has %d rows, the routing %d samples" % (x.shape[0], T))
    out, out_stride = _out_rows(out, "out", T * k, x.shape[1], x)
    _call("derf_dispatch", x.device, x.data_ptr(), stride, routing.row.data_ptr(), T, k, x.shape[1],
          _PRECISION[x.dtype], out.data_ptr(), out_stride)
    return out


def combine(rows: torch.Tensor, routing: Routing, weights: Optional[torch.Tensor] = None,
            out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Rows [T * k, D] back to their samples, summed with weights (float32
    [T, k]; None: ones) over the pairs that have a head."""
    stride = _rows(rows, "rows")
    T, k = _routing(routing, rows.device)
    if rows.shape[0] != T * k:
        raise ValueError("%d rows, the routing has %d" % (rows.shape[0], T * k))
    if weights is not None:
        _array(weights, "weights", torch.float32, (T, k), rows.device)
    out, out_stride = _out_rows(out, "out", T, rows.shape[1], rows)
    _call("derf_combine", rows.device, rows.data_ptr(), stride, _ptr(weights), routing.row.data_ptr(),
          T, k, rows.shape[1], _PRECISION[rows.dtype], out.data_ptr(), out_stride)
    return out


def dispatch_backward(dout: torch.Tensor, routing: Routing,
                      out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of dispatch: each sample's sum over its pairs' rows."""
    return combine(dout, routing, None, out)


def combine_backward(dout: torch.Tensor, rows: Optional[torch.Tensor], routing: Routing,
                     weights: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                     out_weights: Optional[torch.Tensor] = None):
    """Gradients of combine: (drows [T * k, D], dweights [T, k]).  rows None: no
    gradient of the weights is taken, and dweights is None."""
    stride = _rows(dout, "dout")
    T, k = _routing(routing, dout.device)
    if dout.shape[0] != T:
        raise ValueError("dout has %d rows, the routing %d samples" % (dout.shape[0], T))
    D, rows_stride = dout.shape[1], 0
    if rows is not None:
        rows_stride = _rows(rows, "rows", (T * k, D), dout.dtype, dout.device)
        out_weights = _out_array(out_weights, "out_weights", (T, k), dout.device)
    elif out_weights is not None:
        raise ValueError("out_weights needs rows")
    if weights is not None:
        _array(weights, "weights", torch.float32, (T, k), dout.device)
    out, out_stride = _out_rows(out, "out", T * k, D, dout)
    _call("derf_combine_backward", dout.device, dout.data_ptr(), stride, _ptr(rows), rows_stride,
          _ptr(weights), routing.row.data_ptr(), T, k, D, _PRECISION[dout.dtype], out.data_ptr(),
          out_stride, _ptr(out_weights))
    return out, out_weights


def _layer(w, offsets, like):
    if not isinstance(w, torch.Tensor) or w.dim() != 3:
        raise ValueError("weight must be a tensor [heads, fan_out, fan_in]")
    _array(w, "weight", like.dtype, w.shape, like.device)
    K, O, I = w.shape
    _array(offsets, "offsets", torch.int32, (K + 1,), like.device)
    return K, O, I


def linear(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor],
           offsets: torch.Tensor, relu: bool = False,
           out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Every head's layer on its rows: y[r] = act(weight[h] @ x[r] + bias[h]) for
    offsets[h] <= r < offsets[h + 1], zero from offsets[-1] on.  weight
    [heads, fan_out, fan_in] of x's type, bias float32 [heads, fan_out] or None."""
    stride = _rows(x, "x")
    K, O, I = _layer(weight, offsets, x)
    if x.shape[1] != I:
        raise ValueError("x has rows of %d, the layer takes %d" % (x.shape[1], I))
    if bias is not None:
        _array(bias, "bias", torch.float32, (K, O), x.device)
    out, out_stride = _out_rows(out, "out", x.shape[0], O, x)
    _call("derf_heads_linear", x.device, x.data_ptr(), stride, weight.data_ptr(), _ptr(bias),
          offsets.data_ptr(), x.shape[0], K, I, O, int(bool(relu)), _PRECISION[x.dtype],
          out.data_ptr(), out_stride)
    return out


def linear_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor,
                    offsets: torch.Tensor, y: Optional[torch.Tensor] = None,
                    need_dx: bool = True, out_x: Optional[torch.Tensor] = None,
                    out_weight: Optional[torch.Tensor] = None,
                    out_bias: Optional[torch.Tensor] = None):
    """Gradients of linear: (dx, dweight, dbias); y: the layer's output where it
    had a ReLU.  dweight [heads, fan_out, fan_in] and dbias [heads, fan_out] are
    float32; need_dx False (a first layer): dx is None and not computed."""
    dy_stride = _rows(dy, "dy")
    K, O, I = _layer(weight, offsets, dy)
    R = dy.shape[0]
    if dy.shape[1] != O:
        raise ValueError("dy has rows of %d, the layer gives %d" % (dy.shape[1], O))
    x_stride = _rows(x, "x", (R, I), dy.dtype, dy.device)
    y_stride = 0 if y is None else _rows(y, "y", (R, O), dy.dtype, dy.device)
    dx_stride = 0
    if need_dx:
        out_x, dx_stride = _out_rows(out_x, "out_x", R, I, dy)
    elif out_x is not None:
        raise ValueError("out_x without need_dx")
    out_weight = _out_array(out_weight, "out_weight", (K, O, I), dy.device)
    out_bias = _out_array(out_bias, "out_bias", (K, O), dy.device)
    prec = _PRECISION[dy.dtype]
    need = _workspace_bytes("derf_heads_linear_workspace", R, K, I, O, int(y is not None), prec)
    if need < 0:
        raise ValueError("invalid sizes: %d rows, %d heads of %d to %d" % (R, K, I, O))
    ws = _workspace(need, dy.device)
    _call("derf_heads_linear_backward", dy.device, dy.data_ptr(), dy_stride, x.data_ptr(), x_stride,
          weight.data_ptr(), _ptr(y), y_stride, offsets.data_ptr(), R, K, I, O, prec, _ptr(out_x),
          dx_stride, out_weight.data_ptr(), out_bias.data_ptr(), _ptr(ws), need)
    return out_x, out_weight, out_bias


def _gated_layer(w, offsets, like, act):
    if not isinstance(w, torch.Tensor) or w.dim() != 4 or w.shape[1] != 2:
        raise ValueError("weight must be a tensor [heads, 2, fan_out, fan_in]")
    _array(w, "weight", like.dtype, w.shape, like.device)
    K, _, O, I = w.shape
    _array(offsets, "offsets", torch.int32, (K + 1,), like.device)
    if act not in ACTIVATIONS:
        raise ValueError("act is %r, not one of %s" % (act, ", ".join(ACTIVATIONS)))
    return K, O, I


def gated(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor],
          offsets: torch.Tensor, act: str = "silu", keep: bool = False,
          out: Optional[torch.Tensor] = None, out_pre: Optional[torch.Tensor] = None):
    """Every head's gated layer on its rows: (y, pre) with y[r] = act(g) * u, g = weight[h, 0] @
    x[r] + bias[h, 0] and u = weight[h, 1] @ x[r] + bias[h, 1], zero from offsets[-1] on.
    weight [heads, 2, fan_out, fan_in] of x's type, bias float32 [heads, 2, fan_out] or
    None; act one of ACTIVATIONS.  pre [R, 2 * fan_out], g then u, is what the gradients
    need: with keep (or out_pre), else None."""
    stride = _rows(x, "x")
    K, O, I = _gated_layer(weight, offsets, x, act)
    if x.shape[1] != I:
        raise ValueError("x has rows of %d, the layer takes %d" % (x.shape[1], I))
    if bias is not None:
        _array(bias, "bias", torch.float32, (K, 2, O), x.device)
    out, out_stride = _out_rows(out, "out", x.shape[0], O, x)
    pre_stride = 0
    if keep or out_pre is not None:
        out_pre, pre_stride = _out_rows(out_pre, "out_pre", x.shape[0], 2 * O, x)
    _call("derf_heads_gated", x.device, x.data_ptr(), stride, weight.data_ptr(), _ptr(bias),
          offsets.data_ptr(), x.shape[0], K, I, O, ACTIVATIONS[act], _PRECISION[x.dtype],
          out.data_ptr(), out_stride, _ptr(out_pre), pre_stride)
    return out, out_pre


def gated_backward(dy: torch.Tensor, pre: torch.Tensor, x: torch.Tensor, weight: torch.Tensor,
                   offsets: torch.Tensor, act: str = "silu", need_dx: bool = True,
                   out_x: Optional[torch.Tensor] = None, out_weight: Optional[torch.Tensor] = None,
                   out_bias: Optional[torch.Tensor] = None):
    """Gradients of gated at the gates and ups that it kept: (dx, dweight, dbias).
    dweight [heads, 2, fan_out, fan_in] is of the weights' type (its factors carry that
    type's rounding), dbias [heads, 2, fan_out] float32; need_dx False: dx is None and
    not computed."""
    dy_stride = _rows(dy, "dy")
    K, O, I = _gated_layer(weight, offsets, dy, act)
    R = dy.shape[0]
    if dy.shape[1] != O:
        raise ValueError("dy has rows of %d, the layer gives %d" % (dy.shape[1], O))
    pre_stride = _rows(pre, "pre", (R, 2 * O), dy.dtype, dy.device)
    x_stride = _rows(x, "x", (R, I), dy.dtype, dy.device)
    dx_stride = 0
    if need_dx:
        out_x, dx_stride = _out_rows(out_x, "out_x", R, I, dy)
    elif out_x is not None:
        raise ValueError("out_x without need_dx")
    if out_weight is None:
        out_weight = torch.empty_like(weight, requires_grad=False)
    else:
        _array(out_weight, "out_weight", weight.dtype, weight.shape, dy.device)
    out_bias = _out_array(out_bias, "out_bias", (K, 2, O), dy.device)
    prec = _PRECISION[dy.dtype]
    need = _workspace_bytes("derf_heads_gated_workspace", R, K, I, O, prec)
    if need < 0:
        raise ValueError("invalid sizes: %d rows, %d heads of %d to 2 x %d" % (R, K, I, O))
    ws = _workspace(need, dy.device)
    _call("derf_heads_gated_backward", dy.device, dy.data_ptr(), dy_stride, pre.data_ptr(), pre_stride,
          x.data_ptr(), x_stride, weight.data_ptr(), offsets.data_ptr(), R, K, I, O, ACTIVATIONS[act],
          prec, _ptr(out_x), dx_stride, out_weight.data_ptr(), out_bias.data_ptr(), _ptr(ws), need)
    return out_x, out_weight, out_bias


def lookup(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0,
           out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Rows of a table [V, D] picked by ids (int32 [T]): out[t] = scale * table[ids[t]], zero
    where an id is outside [0, V)."""
    stride = _rows(table, "table")
    V, D = table.shape
    if V < 1:
        raise ValueError("table has no rows")
    if not isinstance(ids, torch.Tensor) or ids.dim() != 1:
        raise ValueError("ids must be a tensor [T]")
    _array(ids, "ids", torch.int32, ids.shape, table.device)
    out, out_stride = _out_rows(out, "out", ids.shape[0], D, table)
    _call("derf_lookup", table.device, table.data_ptr(), stride, ids.data_ptr(), ids.shape[0], V, D,
          scale, _PRECISION[table.dtype], out.data_ptr(), out_stride)
    return out


def lookup_backward(dout: torch.Tensor, ids: torch.Tensor, num_rows: int, scale: float = 1.0,
                    out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of lookup in the table, float32 [num_rows, D]: each row's samples summed, times
    scale; zero without any.  Samples go in a fixed order, so the sums repeat bit for bit."""
    stride = _rows(dout, "dout")
    T, D = dout.shape
    _array(ids, "ids", torch.int32, (T,), dout.device)
    need = _workspace_bytes("derf_lookup_workspace", T, num_rows, D)
    if need < 0:
        raise ValueError("invalid sizes: %d samples, %d rows of %d" % (T, num_rows, D))
    out = _out_array(out, "out", (num_rows, D), dout.device)
    ws = _workspace(need, dout.device)
    _call("derf_lookup_backward", dout.device, dout.data_ptr(), stride, ids.data_ptr(), T, num_rows, D,
          scale, _PRECISION[dout.dtype], out.data_ptr(), _ptr(ws), need)
    return out


class AdamW:
    """AdamW over lists of tensors, in one launch a step (derf_adamw_create).

    params and grads: contiguous float32 or bfloat16 tensors of one GPU; the
    gradients are read from these tensors at every step, so a program writes them
    in place.  copies: bfloat16 tensors (or None in the place of one) that
    receive the updated parameters rounded.  state_bits 32 keeps the moments in
    float32; 8 in e4m3 with a float32 scale for each 256 values, the second
    moment as its square root.  Moments start at zero unless given (m, v and, in
    8 bits, m_scale, v_scale: lists like params, used in place)."""

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor],
                 lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8,
                 weight_decay: float = 0.01, state_bits: int = 32, copies=None, m=None, v=None,
                 m_scale=None, v_scale=None):
        self.handle = None
        if state_bits not in (8, 32):
            raise ValueError("state_bits is %r, not 8 or 32" % (state_bits,))
        self.params, self.grads = list(params), list(grads)
        if not self.params or len(self.params) != len(self.grads):
            raise ValueError("need parameters and as many gradients")
        self.lr, self.betas, self.eps, self.weight_decay = lr, tuple(betas), eps, weight_decay
        self.state_bits, self.steps = state_bits, 0
        self.copies = self._list(copies, "copies") if copies is not None else [None] * len(self.params)
        for i, (p, g, c) in enumerate(zip(self.params, self.grads, self.copies)):
            for name, x in (("params", p), ("grads", g)):
                if not isinstance(x, torch.Tensor) or x.dtype not in _PRECISION:
                    raise ValueError("%s[%d] must be a float32 or bfloat16 tensor" % (name, i))
                _array(x, "%s[%d]" % (name, i), x.dtype, p.shape, self.params[0].device, leaf=True)
            if c is not None:
                _array(c, "copies[%d]" % i, torch.bfloat16, p.shape, self.params[0].device, leaf=True)
        self.device = self.params[0].device
        state = torch.float32 if state_bits == 32 else torch.float8_e4m3fn
        self.m, self.v = self._state(m, "m", state), self._state(v, "v", state)
        self.m_scale = self.v_scale = None
        if state_bits == 8:
            self.m_scale = self._state(m_scale, "m_scale", torch.float32, MOMENT_BLOCK)
            self.v_scale = self._state(v_scale, "v_scale", torch.float32, MOMENT_BLOCK)
        elif m_scale is not None or v_scale is not None:
            raise ValueError("scales belong to 8-bit moments")
        table = (derf.derf_adamw_tensor * len(self.params))()
        for i, (p, g, c) in enumerate(zip(self.params, self.grads, self.copies)):
            ptr = [x.data_ptr() for x in (p, g, self.m[i], self.v[i])]
            ptr += [0, 0] if state_bits == 32 else [self.m_scale[i].data_ptr(), self.v_scale[i].data_ptr()]
            table[i] = derf.derf_adamw_tensor(*ptr, 0 if c is None else c.data_ptr(), p.numel(),
                                              _PRECISION[p.dtype], _PRECISION[g.dtype])
        handle = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            _check(derf.lib().derf_adamw_create(
                ctypes.byref(handle), ctypes.cast(table, ctypes.c_void_p), len(self.params),
                state_bits), "derf_adamw_create")
        self.handle = handle

    def _list(self, given, name) -> List:
        given = list(given)
        if len(given) != len(self.params):
            raise ValueError("%s: one for each parameter" % name)
        return given

    def _state(self, given, name, dtype, block=1) -> List[torch.Tensor]:
        counts = [-(-p.numel() // block) for p in self.params]
        if given is None:
            return [torch.zeros((n,), dtype=torch.uint8 if dtype.itemsize == 1 else dtype,
                                device=self.device).view(dtype) for n in counts]
        given = self._list(given, name)
        for i, (x, n) in enumerate(zip(given, counts)):
            _array(x, "%s[%d]" % (name, i), dtype, (n,) if block > 1 else getattr(x, "shape", ()), self.device, leaf=True)
            if x.numel() != n:
                raise ValueError("%s[%d] holds %d values, %d needed" % (name, i, x.numel(), n))
        return given

    def step(self, step: Optional[int] = None, grad_scale: Optional[torch.Tensor] = None) -> None:
        """One step, number `step` (None: one more than the last).  grad_scale:
        float32 [1] on the GPU, a factor on every gradient.  Not while the stream
        is being captured: a graph would repeat this step's number and rate, so it
        raises; capture the rest of a training step and call this beside the replay."""
        if self.handle is None:
            raise ValueError("the optimizer is closed")
        if grad_scale is not None:
            _array(grad_scale, "grad_scale", torch.float32, (1,), self.device, leaf=True)
        step = self.steps + 1 if step is None else int(step)
        _call("derf_adamw_step", self.device, self.handle, self.lr, self.betas[0], self.betas[1],
              self.eps, self.weight_decay, step, _ptr(grad_scale))
        self.steps = step

    def moments(self, i: int):
        """The first moment and the square root of the second of parameter i, in float32."""
        if self.state_bits == 32:
            return self.m[i], self.v[i].sqrt()
        n = self.params[i].numel()
        spread = lambda s: s.repeat_interleave(MOMENT_BLOCK)[:n]  # noqa: E731
        return (self.m[i].float().reshape(-1) * spread(self.m_scale[i]),
                self.v[i].float().reshape(-1) * spread(self.v_scale[i]))

    def close(self):
        if self.handle is not None and self.handle.value:
            derf.derf_adamw_destroy(self.handle)
        self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def orthogonalise(x: torch.Tensor, iterations: int = 5, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x's matrices (the last two dimensions) with their singular values brought near 1 and
    their directions kept (derf_orthogonalise): float32 through products of 22 bits, about
    as exactly as the iteration in float32, bfloat16 through products of 11 bits (22 where a
    side is below 8).  x: contiguous, [fan_out, fan_in] or
    [heads, fan_out, fan_in]; out: x, or another tensor of its shape and type."""
    if not isinstance(x, torch.Tensor) or x.dim() not in (2, 3) or x.dtype not in _PRECISION:
        raise ValueError("x must be a float32 or bfloat16 tensor [fan_out, fan_in] or [heads, fan_out, fan_in]")
    _array(x, "x", x.dtype, x.shape)
    K, (O, I) = (x.shape[0] if x.dim() == 3 else 1), x.shape[-2:]
    prec = _PRECISION[x.dtype]
    need = _workspace_bytes("derf_orthogonalise_workspace", K, O, I, prec)
    if need < 0:
        raise ValueError("invalid sizes: %d matrices of %d x %d" % (K, O, I))
    if out is None:
        out = torch.empty_like(x)
    else:
        _array(out, "out", x.dtype, x.shape, x.device)
    ws = _workspace(need, x.device)
    _call("derf_orthogonalise", x.device, x.data_ptr(), K, O, I, iterations, prec, out.data_ptr(), _ptr(ws), need)
    return out


class Muon:
    """Steps along orthogonalised directions over lists of weight tensors (derf_muon_create).

    params and grads: contiguous float32 or bfloat16 tensors [fan_out, fan_in] or [heads,
    fan_out, fan_in] of one GPU, each matrix orthogonalised for itself; the gradients are
    read from these tensors at every step.  copies: bfloat16 tensors (or None in the place
    of one) that receive the updated parameters rounded.  m: the momentum, float32 tensors
    of the parameters' shapes, used in place; zeros unless given.  The optimizer holds its
    workspace until close(): about 5 to 17 bytes a value of the matrices of one padded
    shape, at most 8 GiB (or what one matrix needs), beside torch's allocator; none for
    matrices of up to 64 x 512 or 128 x 128.  Its steps go on one stream, or are waited for.  Biases and other vectors
    belong to AdamW."""

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], lr: float = 0.02,
                 momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0, iterations: int = 5,
                 copies=None, m=None):
        self.handle = None
        self.params, self.grads = list(params), list(grads)
        if not self.params or len(self.params) != len(self.grads):
            raise ValueError("need parameters and as many gradients")
        for name, given in (("copies", copies), ("m", m)):
            if given is not None and len(given) != len(self.params):
                raise ValueError("%s: one for each parameter" % name)
        self.lr, self.momentum, self.nesterov = lr, momentum, bool(nesterov)
        self.weight_decay, self.iterations = weight_decay, iterations
        self.copies = list(copies) if copies is not None else [None] * len(self.params)
        first = self.params[0]
        if not isinstance(first, torch.Tensor):
            raise ValueError("params[0] must be a torch tensor")
        self.device = first.device
        for i, (p, g, c) in enumerate(zip(self.params, self.grads, self.copies)):
            for name, x in (("params", p), ("grads", g)):
                if not isinstance(x, torch.Tensor) or x.dtype not in _PRECISION or x.dim() not in (2, 3):
                    raise ValueError("%s[%d] must be a float32 or bfloat16 tensor of matrices" % (name, i))
                _array(x, "%s[%d]" % (name, i), x.dtype, p.shape, self.device, leaf=True)
            if c is not None:
                _array(c, "copies[%d]" % i, torch.bfloat16, p.shape, self.device, leaf=True)
        if m is None:
            self.m = [torch.zeros(p.shape, dtype=torch.float32, device=self.device) for p in self.params]
        else:
            self.m = list(m)
            for i, (p, x) in enumerate(zip(self.params, self.m)):
                _array(x, "m[%d]" % i, torch.float32, p.shape, self.device, leaf=True)
        table = (derf.derf_muon_tensor * len(self.params))()
        for i, (p, g, c) in enumerate(zip(self.params, self.grads, self.copies)):
            table[i] = derf.derf_muon_tensor(p.data_ptr(), g.data_ptr(), self.m[i].data_ptr(), _ptr(c),
                                             p.shape[0] if p.dim() == 3 else 1, p.shape[-2], p.shape[-1],
                                             _PRECISION[p.dtype], _PRECISION[g.dtype])
        handle = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            _check(derf.lib().derf_muon_create(ctypes.byref(handle), ctypes.cast(table, ctypes.c_void_p),
                                               len(self.params)), "derf_muon_create")
        self.handle = handle

    def step(self, grad_scale: Optional[torch.Tensor] = None) -> None:
        """One step.  grad_scale: float32 [1] on the GPU, a factor on every gradient.  Not while
        the stream is being captured (a graph would repeat this step's rate): it raises."""
        if self.handle is None:
            raise ValueError("the optimizer is closed")
        if grad_scale is not None:
            _array(grad_scale, "grad_scale", torch.float32, (1,), self.device, leaf=True)
        _call("derf_muon_step", self.device, self.handle, self.lr, self.momentum, int(self.nesterov),
              self.weight_decay, self.iterations, _ptr(grad_scale))

    def close(self):
        if self.handle is not None and self.handle.value:
            derf.derf_muon_destroy(self.handle)
        self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
