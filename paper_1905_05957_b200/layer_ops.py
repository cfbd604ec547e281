"""Layers in 16-bit floats and what stands between layers, for the networks whose gradients the workers compress: products with bias,
activation and residual in their epilogue, norms around a residual connection, and dropout.  Argument marshalling over the C ABI
(include/dsq.h); PyTorch supplies memory and streams.

As with the 8-bit layers the calls stand outside autograd: a result carries no gradient, backward() gives a layer's.  What backward() needs is
kept by reference: the inputs of a training forward may not be changed before it.
"""
from __future__ import annotations

import ctypes as C
import math

import torch

from . import matrix_ops as _m
from .binding import (ACTIVATIONS, DS_F16_FORWARD, DS_F16_INPUTS, DS_F16_WEIGHTS, DS_F32, DS_NORM_LAYER, DS_NORM_MAX_COLS, DS_NORM_RMS,
                      ds_f16_product, ds_norm_args, fast_call, fast_struct_call, load_library)
from .matrix_ops import _DTYPES, _check, _current, _dev_status, _empty, _matrix, _out, _raw_stream, _vector

_HALVES = {torch.bfloat16: _DTYPES[torch.bfloat16], torch.float16: _DTYPES[torch.float16]}
_NORMS = {"rms": DS_NORM_RMS, "layer": DS_NORM_LAYER}
_call = _struct = _matmul_at = _slope_at = _pack_at = _norm_at = _norm_back_at = _dropout_at = None


def _load():
    """Looks the library's functions up once."""
    global _call, _struct, _matmul_at, _slope_at, _pack_at, _norm_at, _norm_back_at, _dropout_at
    _struct, at = fast_struct_call()
    _matmul_at, _slope_at, _norm_at, _norm_back_at = (at[n] for n in ("ds_f16_matmul", "ds_f16_slope", "ds_norm_forward", "ds_norm_backward"))
    _call, at = fast_call()
    _pack_at, _dropout_at = at["ds_f16_pack"], at["ds_dropout"]


def _half(t: torch.dtype, what: str) -> int:
    code = _HALVES.get(t)
    if code is None:
        raise TypeError(f"{what}: bfloat16 or float16 expected, got {t}")
    return code


def _activation(name: str) -> int:
    code = ACTIVATIONS.get(name)
    if code is None:
        raise ValueError(f"activation: one of {', '.join(ACTIVATIONS)} expected, got {name!r}")
    return code


def _like(t: torch.Tensor, rows: int, cols: int, dtype: torch.dtype, device, what: str) -> tuple[torch.Tensor, int]:
    """t as rows of consecutive entries, and the distance between them; it has to be [rows, cols] of dtype on device."""
    if t.dtype is not dtype:
        raise TypeError(f"{what}: {dtype} expected, got {t.dtype}")
    if t.shape != (rows, cols) or t.device != device:
        raise ValueError(f"{what}: a matrix {(rows, cols)} on {device} expected, got {tuple(t.shape)} on {t.device}")
    t, _, _, ld, _ = _matrix(t, what)
    return t, ld


def _on_boundary(p: int, ld: int, rows: int) -> bool:
    return p % 16 == 0 and (rows <= 1 or ld % 8 == 0)


def _packed(x: torch.Tensor, ld: int, dtype: torch.dtype, index: int) -> tuple[torch.Tensor, int]:
    """A copy of a matrix in 16 bits, on 16-byte rows."""
    r, c = x.shape
    pitch = max(8, (c + 7) // 8 * 8)
    out = _empty((r, pitch), dtype=dtype, device=x.device)
    rc = _call(_pack_at, x.data_ptr(), _m._dtype(x.dtype, "x"), r, c, ld, out.data_ptr(), _half(dtype, "dtype"), pitch, _raw_stream(index))
    if rc:
        _check(rc, "ds_f16_pack")
    return out[:, :c], pitch


def _product(layout: int, dt: int, m: int, n: int, k: int, a: int, lda: int, b: int, ldb: int, bias, act: int, res, ldr: int, z, ldz: int, out: int, odt: int,
             ldo: int, index: int, device):
    rows_a, rows_b = (k if layout == DS_F16_WEIGHTS else m), (n if layout == DS_F16_FORWARD else k)
    ws, size = None, 0
    if not (_on_boundary(a, lda, rows_a) and _on_boundary(b, ldb, rows_b)):
        args = ds_f16_product(dt, layout, m, n, k, a, lda, b, ldb, 0, 0, 0, 0, 0, 0, out, odt, ldo, 0, 0, 0)
        size = load_library().ds_f16_matmul_workspace(C.byref(args))
        ws = _empty(size, dtype=torch.uint8, device=device)
    rc = _struct(_matmul_at, _raw_stream(index), dt, layout, m, n, k, a, lda, b, ldb, bias, act, res, ldr, z, ldz, out, odt, ldo,
                 ws.data_ptr() if size else None, size, _dev_status(index))
    if rc:
        _check(rc, "ds_f16_matmul")


def linear16(x: torch.Tensor, w: torch.Tensor, bias: torch.Tensor | None = None, activation: str = "none", residual: torch.Tensor | None = None,
             out_dtype: torch.dtype | None = None, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """act(x W^T + bias) + residual for x [tokens, k], w [n, k] and residual [tokens, n] in bfloat16 or float16 and bias [n] in float32; sums and
    epilogue in 32 bits, one rounding at the end.  activation: none, relu, gelu, gelu_tanh or silu.  The result has x's type or is float32 (out_dtype, or out's).  `out` may be
    the residual itself, and may not overlap anything else.  Weights whose rows start on 16-byte boundaries are read where they lie, others are copied at
    every call (Linear16 copies them once)."""
    if stream is not None:
        with torch.cuda.stream(stream):      # what is allocated here belongs to the stream that uses it
            return linear16(x, w, bias, activation, residual, out_dtype, out)
    return _forward(x, w, bias, _activation(activation), residual, out_dtype, out, False)[0]


def _forward(x, w, bias, act, residual, out_dtype, out, keep_z):
    if _struct is None:
        _load()
    dt = _half(x.dtype, "x")
    x, m, k, ldx, device = _matrix(x, "x")
    n = w.shape[0]
    w, ldw = _like(w, n, k, x.dtype, device, "w")
    index = device.index
    if index != _current():                  # the library works on the current device
        with torch.cuda.device(device):
            return _forward(x, w, bias, act, residual, out_dtype, out, keep_z)
    bp = None if bias is None else _vector(bias, n, "bias", device)
    rp, ldr = None, 0
    if residual is not None:
        residual, ldr = _like(residual, m, n, x.dtype, device, "residual")
        rp = residual.data_ptr()
    if out is not None:
        ldo, odt = _out(out, m, n, device), _DTYPES.get(out.dtype)
    else:
        out = _empty((m, n), dtype=out_dtype or x.dtype, device=device)
        ldo, odt = n, _DTYPES.get(out.dtype)
    if odt != dt and odt != DS_F32:
        raise TypeError(f"out: {x.dtype} or float32 expected, got {out.dtype}")
    z, ldz = None, 0
    if keep_z:
        ldz = (n + 7) // 8 * 8
        z = _empty((m, ldz), dtype=x.dtype, device=device)[:, :n]
    if m and n:
        _product(DS_F16_FORWARD, dt, m, n, k, x.data_ptr(), ldx, w.data_ptr(), ldw, bp, act, rp, ldr, None if z is None else z.data_ptr(), ldz, out.data_ptr(),
                 odt, ldo, index, device)
    return out, z


class Linear16:
    """A linear layer y = act(x W^T + bias) + residual in 16-bit floats.

    W [out, in]: bfloat16 or float16, used where it lies if its rows start on 16-byte boundaries, else copied; or float32 (a slice of a model of the step),
    copied as `dtype` (bfloat16 unless given).  Call set_weight() after every change of W.  The bias is float32.  forward(x, training=True) keeps x and, with an activation,
    x W^T + bias in 16 bits for the gradients."""

    def __init__(self, weight: torch.Tensor, bias: torch.Tensor | None = None, activation: str = "none", dtype: torch.dtype | None = None, stream=None):
        self.activation, self._act = activation, _activation(activation)
        self.bias, self._dtype = bias, dtype
        self.set_weight(weight, stream)

    def set_weight(self, weight: torch.Tensor, stream=None):
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.set_weight(weight)
        if _struct is None:
            _load()
        _m._dtype(weight.dtype, "weight")
        weight, r, _, ld, device = _matrix(weight, "weight")
        dtype = self._dtype or (torch.bfloat16 if weight.dtype is torch.float32 else weight.dtype)
        _half(dtype, "dtype")
        if self.bias is not None:
            _vector(self.bias, r, "bias", device)
        if device.index != _current():
            with torch.cuda.device(device):
                return self.set_weight(weight)
        if weight.dtype is not dtype or not _on_boundary(weight.data_ptr(), ld, r):
            weight, ld = _packed(weight, ld, dtype, device.index)
        self.weight, self._device = weight, device
        self._x = self._z = None
        self._stream = self._saved_on = _raw_stream(device.index)      # where the allocator takes the tensors to be in use

    def _used(self, saved: bool):
        """Tells the allocator of the current stream: dropped before that has run, the layer's memory is kept until it has."""
        raw = _raw_stream(self._device.index)
        if raw != self._stream:
            self.weight.record_stream(torch.cuda.current_stream(self._device))
            if self.bias is not None:
                self.bias.record_stream(torch.cuda.current_stream(self._device))
            self._stream = raw
        if saved and raw != self._saved_on:
            for t in (self._x, self._z):
                if t is not None:
                    t.record_stream(torch.cuda.current_stream(self._device))
            self._saved_on = raw

    def forward(self, x: torch.Tensor, residual: torch.Tensor | None = None, training: bool = False, out_dtype: torch.dtype | None = None,
                out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.forward(x, residual, training, out_dtype, out)
        if x.device != self._device:
            raise ValueError(f"x on {x.device}, the weights on {self._device}")
        if self._device.index != _current():
            with torch.cuda.device(self._device):
                return self.forward(x, residual, training, out_dtype, out)
        self._used(False)
        if training:
            _half(x.dtype, "x")
            x, m, k, ldx, _ = _matrix(x, "x")
            if m and k and not _on_boundary(x.data_ptr(), ldx, m):      # once, for this product and for the gradient of the weights
                x = _packed(x, ldx, x.dtype, self._device.index)[0]
        y, z = _forward(x, self.weight, self.bias, self._act, residual, out_dtype, out, training and self._act != 0)
        if training:
            self._x, self._z, self._saved_on = x, z, _raw_stream(self._device.index)
        return y

    def backward(self, dy: torch.Tensor, grad_dtype: torch.dtype | None = None, dw: torch.Tensor | None = None, db: torch.Tensor | None = None,
                 need_dx: bool = True, stream=None):
        """(dx, dw, db) of the last training forward; the gradient of the residual is dy itself; db is None for a layer without bias, dx if it is not wanted.
        dw and db have grad_dtype (the type of x unless given, or float32) or are given: [out, in] and [out] views of a gradient row of DoubleSqueeze, for instance.
        dy has the type of x; its product with the activation's slope is rounded to that type before the products, db is summed before."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.backward(dy, grad_dtype, dw, db, need_dx)
        if self._x is None:
            raise RuntimeError("backward needs a forward with training=True before it")
        x, z, device = self._x, self._z, self._device
        index, dt = device.index, _HALVES[x.dtype]
        if index != _current():
            with torch.cuda.device(device):
                return self.backward(dy, grad_dtype, dw, db, need_dx)
        (m, k), n = x.shape, self.weight.shape[0]
        dy, lddy = _like(dy, m, n, x.dtype, device, "dy")
        grad_dtype = grad_dtype or x.dtype
        if dw is None:
            dw, ldo = _empty((n, k), dtype=grad_dtype, device=device), k
        else:
            ldo = _out(dw, n, k, device)
        if self.bias is None:
            db = None
        elif db is None:
            db = _empty(n, dtype=grad_dtype, device=device)
        elif db.shape != (n,) or db.device != device or not db.is_contiguous():
            raise ValueError(f"db: {n} contiguous values on {device} expected, got {tuple(db.shape)} on {db.device}")
        for g, what in ((dw, "dw"), (db, "db")):
            if g is not None and g.dtype is not x.dtype and g.dtype is not torch.float32:
                raise TypeError(f"{what}: {x.dtype} or float32 expected, got {g.dtype}")
        self._used(True)
        raw = _raw_stream(index)
        dz, lddz = dy, lddy
        if self._act or db is not None:
            size = load_library().ds_f16_slope_workspace(m, n) if db is not None else 0
            ws = _empty(size, dtype=torch.uint8, device=device) if size else None
            if self._act:
                lddz = (n + 7) // 8 * 8
                dz = _empty((m, lddz), dtype=x.dtype, device=device)[:, :n]
            rc = _struct(_slope_at, raw, dt, m, n, dy.data_ptr(), lddy, None if z is None else z.data_ptr(), 0 if z is None else z.stride(0), self._act,
                         dz.data_ptr() if self._act else None, lddz, None if db is None else db.data_ptr(), 0 if db is None else _DTYPES[db.dtype],
                         ws.data_ptr() if size else None, size)
            if rc:
                _check(rc, "ds_f16_slope")
        if need_dx and m and n and not _on_boundary(dz.data_ptr(), lddz, m):      # once, for both products
            dz, lddz = _packed(dz, lddz, x.dtype, index)
        dx = None
        if need_dx:
            dx = _empty((m, k), dtype=x.dtype, device=device)
            if m and k:
                _product(DS_F16_INPUTS, dt, m, k, n, dz.data_ptr(), lddz, self.weight.data_ptr(), self.weight.stride(0), None, 0, None, 0, None, 0, dx.data_ptr(), dt, k,
                         index, device)
        if n and k:
            _product(DS_F16_WEIGHTS, dt, n, k, m, dz.data_ptr(), lddz, x.data_ptr(), x.stride(0), None, 0, None, 0, None, 0, dw.data_ptr(), _DTYPES[dw.dtype], ldo, index,
                     device)
        return dx, dw, db


def _threshold(p: float) -> int:
    """A probability in 65536ths."""
    if not 0 <= p < 1:
        raise ValueError(f"p: a probability of at least 0 and below 1 expected, got {p}")
    t = math.floor(p * 65536 + 0.5)
    if t > 65535:
        raise ValueError(f"p: {p} drops all but less than one entry in 65536")
    return t


def _word(v: int, what: str) -> int:
    if not 0 <= v < 1 << 32:
        raise ValueError(f"{what}: a whole number of 32 bits expected, got {v}")
    return v


def dropout(x: torch.Tensor, p: float, seed: int, step: int = 0, layer: int = 0, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """x with each entry dropped with probability p (to the nearest 65536th) and the others divided by the probability that they stay.  The mask is a function
    of (seed, layer, step, row, column) alone: the same call on the gradient of the result gives the gradient of x.  `out` may be x itself."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return dropout(x, p, seed, step, layer, out)
    if _struct is None:
        _load()
    dt = _m._dtype(x.dtype, "x")
    x, r, c, ld, device = _matrix(x, "x")
    index = device.index
    if index != _current():
        with torch.cuda.device(device):
            return dropout(x, p, seed, step, layer, out)
    if out is None:
        out, ldo = _empty((r, c), dtype=x.dtype, device=device), c
    elif out.dtype is not x.dtype:
        raise TypeError(f"out: {x.dtype} expected, got {out.dtype}")
    else:
        ldo = _out(out, r, c, device)
    rc = _call(_dropout_at, x.data_ptr(), dt, r, c, ld, out.data_ptr(), ldo, _threshold(p), seed & 0xFFFFFFFFFFFFFFFF, _word(layer, "layer"), _word(step, "step"),
               _raw_stream(index))
    if rc:
        _check(rc, "ds_dropout")
    return out


class ResidualNorm:
    """What stands between two blocks of a network: from the output y of one and the residual stream x

        h = residual_scale x + D(gate * post(y)),    n = pre(h)

    the stream and the input of the next.  post and pre are RMS ("rms") or layer norms ("layer") over a row, each there if it has a weight, with an optional bias;
    gate [cols] or [groups, cols] multiplies rows by entry (the rows are `groups` equal runs: one for each sequence, say); D is dropout with probability p, drawn as
    dropout() draws it.  All parameters are float32 and are used where they lie; the arithmetic is in 32 bits, h and n are rounded once.  y and n have one type
    (float32, bfloat16, float16), x and h the same or float32."""

    def __init__(self, norm: str = "rms", post_weight: torch.Tensor | None = None, post_bias: torch.Tensor | None = None, gate: torch.Tensor | None = None,
                 pre_weight: torch.Tensor | None = None, pre_bias: torch.Tensor | None = None, residual_scale: float = 1.0, eps: float = 1e-5, p: float = 0.0,
                 seed: int = 0, layer: int = 0):
        if norm not in _NORMS:
            raise ValueError(f"norm: one of {', '.join(_NORMS)} expected, got {norm!r}")
        if (post_bias is not None and post_weight is None) or (pre_bias is not None and pre_weight is None):
            raise ValueError("a norm with a bias needs a weight")
        if not eps >= 0:
            raise ValueError(f"eps: not below 0 expected, got {eps}")
        self._norm, self._scale, self._eps = _NORMS[norm], float(residual_scale), float(eps)
        self._drop = (_threshold(p), seed & 0xFFFFFFFFFFFFFFFF, _word(layer, "layer"))
        self._tensors = {"post_weight": post_weight, "post_bias": post_bias, "gate": gate, "pre_weight": pre_weight, "pre_bias": pre_bias}
        given = [t for t in self._tensors.values() if t is not None]
        self.cols = given[0].shape[-1] if given else None
        self._device = device = given[0].device if given else None
        if given and not given[0].is_cuda:
            raise ValueError("parameters: CUDA tensors expected: there is no CPU path")
        self._groups = 0
        if gate is not None:
            if gate.dim() == 2:
                self._groups = gate.shape[0]
            elif gate.dim() == 1:
                self._groups = 1
            if not self._groups:
                raise ValueError(f"gate: [cols] or [groups, cols] expected, got {tuple(gate.shape)}")
        at = {name: None if t is None else _vector(t.reshape(-1) if name == "gate" and t.is_contiguous() else t,
                                                   self.cols * self._groups if name == "gate" else self.cols, name, device) for name, t in self._tensors.items()}
        self._params = (at["post_weight"], at["post_bias"], at["gate"], self._groups, at["pre_weight"], at["pre_bias"], self._scale, self._eps, *self._drop)
        self._stream = None if device is None else _raw_stream(device.index)
        self._saved = None

    def _used(self, saved=()):
        """Tells the allocator of the current stream, on which parameters and what is kept are about to be used."""
        device = self._device if self._device is not None else saved[0].device
        raw = _raw_stream(device.index)
        if raw != self._stream:
            if self._stream is not None:
                for t in (*self._tensors.values(), *saved):
                    if t is not None:
                        t.record_stream(torch.cuda.current_stream(device))
            self._stream = raw

    def forward(self, y: torch.Tensor, x: torch.Tensor | None = None, step: int = 0, training: bool = False, need_h: bool = True, h: torch.Tensor | None = None,
                n: torch.Tensor | None = None, stream=None):
        """(h, n); n is None without a pre norm, h if it is not wanted.  They are written to h and n where those are given, which may be x or y themselves
        (but not in a training forward, whose inputs backward() reads).  `step` enters the random bits alone."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.forward(y, x, step, training, need_h, h, n)
        if _struct is None:
            _load()
        dt = _m._dtype(y.dtype, "y")
        y, rows, cols, ldy, device = _matrix(y, "y")
        index = device.index
        if self.cols is not None and (cols != self.cols or device != self._device):
            raise ValueError(f"y: rows of {self.cols} on {self._device} expected, got {cols} on {device}")
        if not 0 < cols <= DS_NORM_MAX_COLS:
            raise ValueError(f"y: rows of 1 to {DS_NORM_MAX_COLS} entries expected, got {cols}")
        if self._groups and rows % self._groups:
            raise ValueError(f"y: {rows} rows are not {self._groups} equal runs")
        if index != _current():
            with torch.cuda.device(device):
                return self.forward(y, x, step, training, need_h, h, n)
        xp, ldx, sdt, stype = None, 0, dt, y.dtype
        if x is not None:
            if x.dtype is not y.dtype and x.dtype is not torch.float32:
                raise TypeError(f"x: {y.dtype} or float32 expected, got {x.dtype}")
            x, ldx = _like(x, rows, cols, x.dtype, device, "x")
            xp, stype = x.data_ptr(), x.dtype
            sdt = _DTYPES[stype]
        pre = self._params[4] is not None
        if not need_h and not pre:
            raise ValueError("nothing to compute")
        if h is not None:
            if x is None and h.dtype is torch.float32:
                stype, sdt = torch.float32, DS_F32
            if h.dtype is not stype:
                raise TypeError(f"h: {stype} expected, got {h.dtype}")
            ldh = _out(h, rows, cols, device)
        elif need_h:
            h, ldh = _empty((rows, cols), dtype=stype, device=device), cols
        else:
            ldh = 0
        ldn = 0
        if not pre:
            if n is not None:
                raise ValueError("n: there is no pre norm")
        elif n is not None:
            if n.dtype is not y.dtype:
                raise TypeError(f"n: {y.dtype} expected, got {n.dtype}")
            ldn = _out(n, rows, cols, device)
        else:
            n, ldn = _empty((rows, cols), dtype=y.dtype, device=device), cols
        if self._device is not None:
            self._used()
        stats = None
        if training:
            stats = _empty((rows, 4), dtype=torch.float32, device=device)
            for o in (h, n):
                if o is not None and rows and any(i is not None and i.data_ptr() == o.data_ptr() for i in (x, y)):
                    raise ValueError("a training forward may not write over its inputs")
        rc = _struct(_norm_at, _raw_stream(index), dt, sdt, rows, cols, self._norm, y.data_ptr(), ldy, xp, ldx, *self._params, _word(step, "step"),
                     None if stats is None else stats.data_ptr(), None if h is None else h.data_ptr(), ldh, None if n is None else n.data_ptr(), ldn)
        if rc:
            _check(rc, "ds_norm_forward")
        if training:
            self._saved = (y, ldy, x, ldx, stats, step, stype)
            if self._device is None:
                self._stream = _raw_stream(index)
        return h, n

    def backward(self, dh: torch.Tensor | None = None, dn: torch.Tensor | None = None, need_dx: bool = True, out: dict | None = None, stream=None):
        """(dy, dx, gradients) of the last training forward, from the gradients of h and / or n (one that is left out is zero).  `gradients` has a float32 tensor for every
        parameter that was given, under its name; `out` may give tensors to write some of them to (views of a gradient row of DoubleSqueeze, for instance)."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.backward(dh, dn, need_dx, out)
        if self._saved is None:
            raise RuntimeError("backward needs a forward with training=True before it")
        y, ldy, x, ldx, stats, step, stype = self._saved
        (rows, cols), device = y.shape, y.device
        index = device.index
        if index != _current():
            with torch.cuda.device(device):
                return self.backward(dh, dn, need_dx, out)
        if dh is None and dn is None:
            raise ValueError("the gradient of h or of n expected")
        dhp = dnp = None
        lddh = lddn = 0
        if dh is not None:
            dh, lddh = _like(dh, rows, cols, stype, device, "dh")
            dhp = dh.data_ptr()
        if dn is not None:
            if self._params[4] is None:
                raise ValueError("dn: there is no pre norm")
            dn, lddn = _like(dn, rows, cols, y.dtype, device, "dn")
            dnp = dn.data_ptr()
        out = out or {}
        unknown = [k for k in out if self._tensors.get(k) is None]
        if unknown:
            raise ValueError(f"out: no parameter {', '.join(map(str, unknown))}")
        grads, at = {}, []
        for name, t in self._tensors.items():
            if t is None:
                at.append(None)
                continue
            g = out.get(name)
            if g is None:
                g = _empty(t.shape, dtype=torch.float32, device=device)
            elif g.dtype is not torch.float32 or g.shape != t.shape or g.device != device or not g.is_contiguous():
                raise ValueError(f"out[{name!r}]: contiguous float32 values {tuple(t.shape)} on {device} expected")
            grads[name] = g
            at.append(g.data_ptr())
        self._used((y, x, stats))
        dy = _empty((rows, cols), dtype=y.dtype, device=device)
        dx = _empty((rows, cols), dtype=stype, device=device) if x is not None and need_dx else None
        members = [_DTYPES[y.dtype], _DTYPES[stype], rows, cols, self._norm, y.data_ptr(), ldy, None if x is None else x.data_ptr(), ldx, *self._params, step, stats.data_ptr(),
                   None, 0, None, 0, dhp, lddh, dnp, lddn, None if dx is None else dx.data_ptr(), cols, dy.data_ptr(), cols, *at]
        size = load_library().ds_norm_backward_workspace(C.byref(ds_norm_args(*(0 if v is None else v for v in members))))
        ws = _empty(size, dtype=torch.uint8, device=device) if size else None
        rc = _struct(_norm_back_at, _raw_stream(index), *members, ws.data_ptr() if size else None, size)
        if rc:
            _check(rc, "ds_norm_backward")
        return dy, dx, grads
