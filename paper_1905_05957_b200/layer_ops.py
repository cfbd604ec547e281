"""Layers in 16-bit floats and what stands between layers, for the networks whose gradients the workers compress: products with bias,
activation and residual in their epilogue, norms around a residual connection, and dropout.  Argument marshalling over the C ABI
(include/dsq.h); PyTorch supplies memory and streams.

As with the 8-bit layers the calls stand outside autograd: a result carries no gradient, backward() gives a layer's.  What backward() needs is
kept by reference: the inputs of a training forward may not be changed before it.
"""
from __future__ import annotations

import math

import torch

from . import matrix_ops as _m
from .binding import (ACTIVATIONS, DS_F16_FORWARD, DS_F16_INPUTS, DS_F16_WEIGHTS, DS_F32, DS_NORM_LAYER, DS_NORM_MAX_COLS, DS_NORM_RMS,
                      fast_call, fast_struct_call, load_library)
from .matrix_ops import _DTYPES, _check, _current, _dev_status, _raw_stream, _status, _stream_of

_HALVES = {torch.bfloat16: _DTYPES[torch.bfloat16], torch.float16: _DTYPES[torch.float16]}
_NORMS = {"rms": DS_NORM_RMS, "layer": DS_NORM_LAYER}
_like_of, _F32 = torch.empty_like, torch.float32
_WIDE = 4096                 # columns above which a row's parts wait for one another
_SLOPE_ROWS = 2097120        # rows that the gradient through an activation, or a bias's, takes at most
_NOTHING = (None,) * 13      # the members of ds_norm_args that the forward pass does not read
_call = _struct = _size = _matmul_at = _matmul_ws = _slope_at = _slope_ws = _pack_at = _norm_at = _norm_back_at = _norm_back_ws = _dropout_at = None


def _load():
    """Looks the library's functions up once.  _struct comes last: who sees it, on whichever thread, sees the others."""
    global _call, _struct, _size, _matmul_at, _matmul_ws, _slope_at, _slope_ws, _pack_at, _norm_at, _norm_back_at, _norm_back_ws, _dropout_at
    struct, _size, at = fast_struct_call()
    _matmul_at, _slope_at, _norm_at, _norm_back_at = (at[n] for n in ("ds_f16_matmul", "ds_f16_slope", "ds_norm_forward", "ds_norm_backward"))
    _matmul_ws, _norm_back_ws, _slope_ws = at["ds_f16_matmul_workspace"], at["ds_norm_backward_workspace"], load_library().ds_f16_slope_workspace
    _call, at = fast_call()
    _pack_at, _dropout_at = at["ds_f16_pack"], at["ds_dropout"]
    _struct = struct


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


def _rows(t: torch.Tensor, what: str) -> tuple[torch.Tensor, int, int, int, int]:
    """t as rows of consecutive entries; rows, columns, the distance between rows, the device's index."""
    shape, index = t.shape, t.get_device()
    if index < 0:
        raise ValueError(f"{what}: a CUDA tensor expected: there is no CPU path")
    if len(shape) != 2:
        raise ValueError(f"{what}: a matrix expected, got {len(shape)} dimensions")
    r, c = shape
    ld, step = t.stride()
    if (c > 1 and step != 1) or (r > 1 and ld < c):
        t, ld = t.contiguous(), c
    return t, r, c, (ld if r > 1 else c), index


def _like(t: torch.Tensor, rows: int, cols: int, dtype: torch.dtype, index: int, what: str) -> tuple[torch.Tensor, int]:
    """t as rows of consecutive entries, and the distance between them; it has to be [rows, cols] of dtype on that device."""
    if t.dtype is not dtype:
        raise TypeError(f"{what}: {dtype} expected, got {t.dtype}")
    if t.shape != (rows, cols) or t.get_device() != index:
        raise ValueError(f"{what}: a matrix {(rows, cols)} on cuda:{index} expected, got {tuple(t.shape)} on {t.device}")
    ld, step = t.stride()
    if (cols > 1 and step != 1) or (rows > 1 and ld < cols):
        return t.contiguous(), cols
    return t, (ld if rows > 1 else cols)


def _given(out: torch.Tensor, rows: int, cols: int, index: int, what: str) -> int:
    """The distance between the rows of a given output."""
    if out.shape != (rows, cols) or out.get_device() != index:
        raise ValueError(f"{what}: a matrix {(rows, cols)} on cuda:{index} expected, got {tuple(out.shape)} on {out.device}")
    ld, step = out.stride()
    if (cols > 1 and step != 1) or (rows > 1 and ld < cols):
        raise ValueError(f"{what}: rows of consecutive entries expected")
    return ld if rows > 1 else cols


def _floats(v: torch.Tensor, n: int, index: int, what: str) -> int:
    """The address of n contiguous float32 values on that device."""
    if v.dtype is not _F32 or v.shape != (n,) or not v.is_contiguous():
        raise ValueError(f"{what}: {n} contiguous float32 values expected, got {v.dtype} {tuple(v.shape)}")
    if v.get_device() != index:
        raise ValueError(f"{what}: on {v.device}, the others on cuda:{index}")
    return v.data_ptr()


def _on_boundary(p: int, ld: int, rows: int) -> bool:
    return p % 16 == 0 and (rows <= 1 or ld % 8 == 0)


def _pitch(cols: int) -> int:
    """Entries between the rows of what the products' operands are copied to: whole lines of 128 bytes (rows that start on other boundaries of 16 bytes span a line more:
    4096 x 4096 x 4104 takes 114 us so, and 88 on lines)."""
    return (cols + 63) // 64 * 64 or 64


def _packed(x: torch.Tensor, r: int, c: int, ld: int, dtype: torch.dtype, index: int) -> tuple[torch.Tensor, int]:
    """A copy of a matrix in 16 bits, on rows of whole lines: [rows, pitch], and the pitch."""
    pitch = _pitch(c)
    out = x.new_empty((r, pitch), dtype=dtype)
    rc = _call(_pack_at, x.data_ptr(), _DTYPES[x.dtype], r, c, ld, out.data_ptr(), _HALVES[dtype], pitch, _raw_stream(index))
    if rc:
        _check(rc, "ds_f16_pack")
    return out, pitch


def _product(layout: int, dt: int, m: int, n: int, k: int, a: int, lda: int, b: int, ldb: int, bias, act: int, res, ldr: int, z, ldz: int, out: int, odt: int,
             ldo: int, index: int, raw: int, like: torch.Tensor):
    ws = address = None
    size = 0
    if (a | b) & 15 or (lda | ldb) & 7:      # perhaps an operand has to be copied
        size = _size(_matmul_ws, dt, layout, m, n, k, a, lda, b, ldb, bias, act, res, ldr, z, ldz, out, odt, ldo)
        if size:
            ws = like.new_empty(size // 2)
            address = ws.data_ptr()
    status = _status.get(index)
    rc = _struct(_matmul_at, raw, dt, layout, m, n, k, a, lda, b, ldb, bias, act, res, ldr, z, ldz, out, odt, ldo, address, size,
                 status[1] if status else _dev_status(index))
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
    return _forward(x, w, bias, _activation(activation), residual, out_dtype, out)


def _forward(x, w, bias, act, residual, out_dtype, out):
    if _struct is None:
        _load()
    dtype = x.dtype
    if dtype not in _HALVES:
        _half(dtype, "x")
    x, m, k, ldx, index = _rows(x, "x")
    n = w.shape[0]
    w, ldw = _like(w, n, k, dtype, index, "w")
    if index != _current():                  # the library works on the current device
        with torch.cuda.device(index):
            return _forward(x, w, bias, act, residual, out_dtype, out)
    return _multiply(x, m, k, ldx, w, n, ldw, bias, act, residual, out_dtype, out, False, index, _raw_stream(index))[0]


def _multiply(x, m, k, ldx, w, n, ldw, bias, act, residual, out_dtype, out, keep_z, index, raw):
    """out and z of x and w whose first entries are those of [m, k] and [n, k] matrices of one type."""
    dtype = x.dtype
    dt = _HALVES[dtype]
    bp = None if bias is None else _floats(bias, n, index, "bias")
    rp, ldr = None, 0
    if residual is not None:
        residual, ldr = _like(residual, m, n, dtype, index, "residual")
        rp = residual.data_ptr()
    if out is not None:
        ldo, odt = _given(out, m, n, index, "out"), _DTYPES.get(out.dtype)
    elif out_dtype is None:
        out, ldo, odt = (x.new_empty((m, n)) if residual is None else _like_of(residual)), n, dt
    else:
        out, ldo, odt = x.new_empty((m, n), dtype=out_dtype), n, _DTYPES.get(out_dtype)
    if odt != dt and odt != DS_F32:
        raise TypeError(f"out: {dtype} or float32 expected, got {out.dtype}")
    z, zp, ldz = None, None, 0
    if keep_z:
        ldz = _pitch(n)
        z = x.new_empty((m, ldz))
        zp = z.data_ptr()
    if m and n:
        _product(DS_F16_FORWARD, dt, m, n, k, x.data_ptr(), ldx, w.data_ptr(), ldw, bp, act, rp, ldr, zp, ldz, out.data_ptr(), odt, ldo, index, raw, x)
    return out, z


class Linear16:
    """A linear layer y = act(x W^T + bias) + residual in 16-bit floats.

    W [out, in]: bfloat16 or float16, used where it lies if its rows start on 16-byte boundaries, else copied; or float32 (a slice of a model of the step),
    copied as `dtype` (bfloat16 unless given).  Call set_weight() after every change of W (the layer keeps the memory that W had then, even if W gets other).
    The bias is float32.  forward(x, training=True) keeps x and, with an activation, x W^T + bias in 16 bits for the gradients; with an activation or a bias
    it takes up to 2097120 tokens."""

    def __init__(self, weight: torch.Tensor, bias: torch.Tensor | None = None, activation: str = "none", dtype: torch.dtype | None = None, stream=None):
        self.activation, self._act = activation, _activation(activation)
        self._bias, self._dtype = bias, dtype
        self.set_weight(weight, stream)

    @property
    def bias(self) -> torch.Tensor | None:
        return self._bias

    @bias.setter
    def bias(self, bias: torch.Tensor | None):
        self._bias, self._bias_on = bias, {}

    def set_weight(self, weight: torch.Tensor, stream=None):
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.set_weight(weight)
        if _struct is None:
            _load()
        if weight.dtype not in _DTYPES:
            _m._dtype(weight.dtype, "weight")
        weight, r, c, ld, index = _rows(weight, "weight")
        dtype = self._dtype or (torch.bfloat16 if weight.dtype is torch.float32 else weight.dtype)
        if dtype not in _HALVES:
            _half(dtype, "dtype")
        if self.bias is not None:
            _floats(self.bias, r, index, "bias")
        if index != _current():
            with torch.cuda.device(index):
                return self.set_weight(weight)
        if weight.dtype is not dtype or not _on_boundary(weight.data_ptr(), ld, r):
            weight, ld = _packed(weight, r, c, ld, dtype, index)
        else:
            weight = weight.detach()             # its memory as it is now, whatever becomes of the caller's tensor
        # the weights, perhaps on longer rows, and what backward() reads: x, likewise, and z
        self._w, self._ldw, self.shape, self._index = weight, ld, torch.Size((r, c)), index
        self._x = self._z = None
        self._rows_of_x = self._ldx = 0
        # the streams on which the allocator takes the tensors to be in use, by their handles; the caller's may belong to any
        self._on, self._saved_on, self._bias_on = set(), set(), {}      # (the bias's address with each: it may get other storage)

    @property
    def weight(self) -> torch.Tensor:
        """The weights as the products read them."""
        return self._w[:, :self.shape[1]]

    def _used(self) -> int:
        """The current stream's handle.  Tells the allocator of a stream that uses the weights for the first time: dropped before it has run, their memory is
        kept until it has."""
        raw = _raw_stream(self._index)
        if raw not in self._on:
            self._w.record_stream(_stream_of(self._index, raw))
            self._on.add(raw)
        return raw

    def forward(self, x: torch.Tensor, residual: torch.Tensor | None = None, training: bool = False, out_dtype: torch.dtype | None = None,
                out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.forward(x, residual, training, out_dtype, out)
        index = self._index
        if x.get_device() != index:
            raise ValueError(f"x on {x.device}, the weights on cuda:{index}")
        if index != _current():
            with torch.cuda.device(index):
                return self.forward(x, residual, training, out_dtype, out)
        raw, w, (n, k) = self._used(), self._w, self.shape
        dtype = w.dtype
        if x.dtype is not dtype:
            raise TypeError(f"x: {dtype} expected, got {x.dtype}")
        x, m, c, ldx, _ = _rows(x, "x")
        if c != k:
            raise ValueError(f"x has {c} columns, the weights {k}")
        if training and m > _SLOPE_ROWS and (self._act or self.bias is not None):
            raise ValueError(f"x: at most {_SLOPE_ROWS} rows expected in training with an activation or a bias, got {m}")
        if training:
            if m and k and not _on_boundary(x.data_ptr(), ldx, m):      # once, for this product and for the gradient of the weights
                x, ldx = _packed(x, m, k, ldx, dtype, index)
            else:
                x.record_stream(_stream_of(index, raw))
        y, z = _multiply(x, m, k, ldx, w, n, self._ldw, self._bias, self._act, residual, out_dtype, out, training and self._act != 0, index, raw)
        if self._bias is not None and self._bias_on.get(raw) != self._bias.data_ptr():
            self._bias.record_stream(_stream_of(index, raw))
            self._bias_on[raw] = self._bias.data_ptr()
        if training:
            self._x, self._rows_of_x, self._ldx, self._z, self._saved_on, self._x_was = x, m, ldx, z, {raw}, (x.data_ptr(), x.shape)
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
        x, z, index, act = self._x, self._z, self._index, self._act
        dtype = self._w.dtype
        dt = _HALVES[dtype]
        if (x.data_ptr(), x.shape) != self._x_was or x.dtype is not dtype:
            raise RuntimeError("x has other memory than in the training forward")
        if index != _current():
            with torch.cuda.device(index):
                return self.backward(dy, grad_dtype, dw, db, need_dx)
        m, (n, k) = self._rows_of_x, self.shape
        dy, lddy = _like(dy, m, n, dtype, index, "dy")
        grad_dtype = grad_dtype or dtype
        if dw is None:
            dw, ldo = x.new_empty((n, k), dtype=grad_dtype), k
        else:
            ldo = _given(dw, n, k, index, "dw")
        if self.bias is None:
            db = None
        elif db is None:
            db = x.new_empty(n, dtype=grad_dtype)
        elif db.shape != (n,) or db.get_device() != index or not db.is_contiguous():
            raise ValueError(f"db: {n} contiguous values on cuda:{index} expected, got {tuple(db.shape)} on {db.device}")
        for g, what in ((dw, "dw"), (db, "db")):
            if g is not None and g.dtype is not dtype and g.dtype is not torch.float32:
                raise TypeError(f"{what}: {dtype} or float32 expected, got {g.dtype}")
        raw = self._used()
        if raw not in self._saved_on:
            for t in (x, z):
                if t is not None:
                    t.record_stream(_stream_of(index, raw))
            self._saved_on.add(raw)
        dz, lddz, buf = dy.data_ptr(), lddy, None
        if act or db is not None:
            # dz, and behind it what the sums need
            ldn = _pitch(n)
            at = 2 * m * ldn if act else 0
            size = _slope_ws(m, n) if db is not None else 0
            buf = x.new_empty((at + size + 1) // 2 + 8)
            base = buf.data_ptr()
            rc = _struct(_slope_at, raw, dt, m, n, dz, lddy, None if z is None else z.data_ptr(), ldn, act, base if act else None, ldn,
                         None if db is None else db.data_ptr(), 0 if db is None else _DTYPES[db.dtype], base + at if size else None, size)
            if rc:
                _check(rc, "ds_f16_slope")
            if act:
                dz, lddz = base, ldn
        if need_dx and m and n and not _on_boundary(dz, lddz, m):      # once, for both products
            buf, lddz = _packed(dy, m, n, lddz, dtype, index)
            dz = buf.data_ptr()
        dx = None
        if need_dx:
            dx = x.new_empty((m, k))
            if m and k:
                _product(DS_F16_INPUTS, dt, m, k, n, dz, lddz, self._w.data_ptr(), self._ldw, None, 0, None, 0, None, 0, dx.data_ptr(), dt, k, index, raw, x)
        if n and k:
            _product(DS_F16_WEIGHTS, dt, n, k, m, dz, lddz, x.data_ptr(), self._ldx, None, 0, None, 0, None, 0, dw.data_ptr(), _DTYPES[dw.dtype], ldo, index, raw, x)
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
    x, r, c, ld, index = _rows(x, "x")
    if index != _current():
        with torch.cuda.device(index):
            return dropout(x, p, seed, step, layer, out)
    if out is None:
        out, ldo = _like_of(x), c
    elif out.dtype is not x.dtype:
        raise TypeError(f"out: {x.dtype} expected, got {out.dtype}")
    else:
        ldo = _given(out, r, c, index, "out")
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
    dropout() draws it.  All parameters are float32 and are used where they lie at each call (a tensor may get other storage between two of them, of the same length and on the same
    device); the arithmetic is in 32 bits, h and n are rounded once.  y and n have one type (float32, bfloat16, float16), x and h the same or float32."""

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
        self._rest = (self._scale, self._eps, _threshold(p), seed & 0xFFFFFFFFFFFFFFFF, _word(layer, "layer"))
        self._saved, self._saved_on = None, set()      # what backward() reads, and the streams that use it
        self._tensors = {"post_weight": post_weight, "post_bias": post_bias, "gate": gate, "pre_weight": pre_weight, "pre_bias": pre_bias}
        self._given = [v for v in ((0, "post_weight", post_weight), (1, "post_bias", post_bias), (2, "gate", gate), (3, "pre_weight", pre_weight), (4, "pre_bias", pre_bias))
                       if v[2] is not None]
        self.cols = self._index = None
        if self._given:
            _, name, t = self._given[0]
            self.cols, self._index = t.shape[-1] if t.dim() else 0, t.get_device()
            if self._index < 0:
                raise ValueError(f"{name}: a CUDA tensor expected: there is no CPU path")
        self._look()

    def _members(self) -> tuple:
        """The members of ds_norm_args from post_w to layer.  The parameters are looked at in every call: their storage may be another since the last one."""
        index = self._index
        for t, at, shape in self._seen:
            if t.data_ptr() != at or t.shape != shape or t.dtype is not _F32 or not t.is_contiguous() or t.get_device() != index:
                return self._look()
        return self._at

    def _look(self) -> tuple:
        at, groups, cols, index = [None] * 5, 0, self.cols, self._index
        for i, name, t in self._given:
            if i == 2:
                if not 1 <= t.dim() <= 2 or t.shape[-1] != cols or not t.numel() or t.dtype is not _F32 or not t.is_contiguous() or t.get_device() != index:
                    raise ValueError(f"gate: [cols] or [groups, cols] contiguous float32 values beside the others expected, got {t.dtype} {tuple(t.shape)} on {t.device}")
                groups = t.shape[0] if t.dim() == 2 else 1
                at[2] = t.data_ptr()
            else:
                at[i] = _floats(t, cols, index, name)
        self._seen = [(t, at[i], t.shape) for i, _, t in self._given]
        self._on = set()                         # the streams on which the allocator takes these parameters to be in use, by their handles: they may belong to any
        self._at = (at[0], at[1], at[2], groups, at[3], at[4], *self._rest)
        return self._at

    def _used(self, index: int) -> tuple[int, torch.cuda.Stream]:
        """The current stream's handle, and the stream.  Tells the allocator of one that uses the parameters for the first time: dropped before it has run,
        their memory is kept until it has."""
        raw = _raw_stream(index)
        stream = _stream_of(index, raw)
        if raw not in self._on:
            for t, _, _ in self._seen:
                t.record_stream(stream)
            self._on.add(raw)
        return raw, stream

    def forward(self, y: torch.Tensor, x: torch.Tensor | None = None, step: int = 0, training: bool = False, need_h: bool = True, h: torch.Tensor | None = None,
                n: torch.Tensor | None = None, stream=None):
        """(h, n); n is None without a pre norm, h if it is not wanted.  They are written to h and n where those are given, which may be x or y themselves
        (but not in a training forward, whose inputs backward() reads).  `step` enters the random bits alone."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.forward(y, x, step, training, need_h, h, n)
        if _struct is None:
            _load()
        dtype = y.dtype
        dt = _DTYPES.get(dtype)
        if dt is None:
            _m._dtype(dtype, "y")
        y, rows, cols, ldy, index = _rows(y, "y")
        if cols != self.cols and self.cols is not None or index != self._index and self._index is not None:
            raise ValueError(f"y: rows of {self.cols} on cuda:{self._index} expected, got {cols} on cuda:{index}")
        if not 0 < cols <= DS_NORM_MAX_COLS:
            raise ValueError(f"y: rows of 1 to {DS_NORM_MAX_COLS} entries expected, got {cols}")
        if index != _current():
            with torch.cuda.device(index):
                return self.forward(y, x, step, training, need_h, h, n)
        params = self._members()
        if params[3] and rows % params[3]:
            raise ValueError(f"y: {rows} rows are not {params[3]} equal runs")
        xp, ldx, sdt, stype = None, 0, dt, dtype
        if x is not None:
            stype = x.dtype
            if stype is not dtype and stype is not torch.float32:
                raise TypeError(f"x: {dtype} or float32 expected, got {stype}")
            x, ldx = _like(x, rows, cols, stype, index, "x")
            xp, sdt = x.data_ptr(), _DTYPES[stype]
        pre = params[4] is not None
        hp, ldh = None, 0
        if h is not None:
            if x is None and h.dtype is torch.float32:
                stype, sdt = torch.float32, DS_F32
            if h.dtype is not stype:
                raise TypeError(f"h: {stype} expected, got {h.dtype}")
            ldh = _given(h, rows, cols, index, "h")
            hp = h.data_ptr()
        elif need_h:
            h, ldh = _like_of(y if x is None else x), cols
            hp = h.data_ptr()
        elif not pre:
            raise ValueError("nothing to compute")
        np_, ldn = None, 0
        if not pre:
            if n is not None:
                raise ValueError("n: there is no pre norm")
        else:
            if n is None:
                n, ldn = _like_of(y), cols
            elif n.dtype is not dtype:
                raise TypeError(f"n: {dtype} expected, got {n.dtype}")
            else:
                ldn = _given(n, rows, cols, index, "n")
            np_ = n.data_ptr()
        raw, current = self._used(index)
        stats = sp = None
        yp, status = y.data_ptr(), _status.get(index)
        if training:
            stats = y.new_empty((rows, 4), dtype=torch.float32)
            sp = stats.data_ptr()
            if rows and (hp in (xp, yp) and hp or np_ in (xp, yp) and np_):
                raise ValueError("a training forward may not write over its inputs")
        rc = _struct(_norm_at, raw, dt, sdt, rows, cols, self._norm, yp, ldy, xp, ldx, *params, _word(step, "step"), sp, hp, ldh, np_, ldn,
                     *_NOTHING, (status[1] if status else _dev_status(index)) if cols > _WIDE else None)
        if rc:
            _check(rc, "ds_norm_forward")
        if training:
            y.record_stream(current)
            if x is not None:
                x.record_stream(current)
            self._saved, self._saved_on = (y, ldy, x, ldx, stats, step, stype, yp, xp, y.shape, dtype), {raw}
        return h, n

    def backward(self, dh: torch.Tensor | None = None, dn: torch.Tensor | None = None, need_dx: bool = True, out: dict | None = None, stream=None):
        """(dy, dx, gradients) of the last training forward, from the gradients of h and / or n (one that is left out is zero).  `gradients` has a float32 tensor for every
        parameter that was given, under its name; `out` may give tensors to write some of them to (views of a gradient row of DoubleSqueeze, for instance)."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.backward(dh, dn, need_dx, out)
        if self._saved is None:
            raise RuntimeError("backward needs a forward with training=True before it")
        y, ldy, x, ldx, stats, step, stype, yp, xp, shape, dtype = self._saved
        (rows, cols), index = shape, stats.get_device()
        if y.data_ptr() != yp or y.shape != shape or y.dtype is not dtype or x is not None and (x.data_ptr() != xp or x.shape != shape or x.dtype is not stype):
            raise RuntimeError("y or x has other memory than in the training forward")
        if index != _current():
            with torch.cuda.device(index):
                return self.backward(dh, dn, need_dx, out)
        if dh is None and dn is None:
            raise ValueError("the gradient of h or of n expected")
        params = self._members()
        if params[3] and rows % params[3]:
            raise ValueError(f"gate: {rows} rows are not {params[3]} equal runs")
        dhp = dnp = None
        lddh = lddn = 0
        if dh is not None:
            dh, lddh = _like(dh, rows, cols, stype, index, "dh")
            dhp = dh.data_ptr()
        if dn is not None:
            if params[4] is None:
                raise ValueError("dn: there is no pre norm")
            dn, lddn = _like(dn, rows, cols, dtype, index, "dn")
            dnp = dn.data_ptr()
        grads, at = {}, []
        for name, t in self._tensors.items():
            if t is None:
                if out and name in out:
                    raise ValueError(f"out: there is no {name}")
                at.append(None)
                continue
            g = out.get(name) if out else None
            if g is None:
                g = _like_of(t)
            elif g.dtype is not torch.float32 or g.shape != t.shape or g.get_device() != index or not g.is_contiguous():
                raise ValueError(f"out[{name!r}]: contiguous float32 values {tuple(t.shape)} on cuda:{index} expected")
            grads[name] = g
            at.append(g.data_ptr())
        if out and any(name not in self._tensors for name in out):
            raise ValueError(f"out: parameters are {', '.join(self._tensors)}")
        raw, current = self._used(index)
        if raw not in self._saved_on:         # what was kept is dropped at the earliest when this stream is done with it
            for t in (y, x, stats):
                if t is not None:
                    t.record_stream(current)
            self._saved_on.add(raw)
        dy, dx = _like_of(y), None
        if x is not None and need_dx:
            dx = _like_of(x)
        members = [_DTYPES[dtype], _DTYPES[stype], rows, cols, self._norm, yp, ldy, xp, ldx, *params, step, stats.data_ptr(),
                   None, 0, None, 0, dhp, lddh, dnp, lddn, None if dx is None else dx.data_ptr(), cols, dy.data_ptr(), cols, *at,
                   _dev_status(index) if cols > _WIDE else None]
        size = _size(_norm_back_ws, *members)
        ws = stats.new_empty((size + 3) // 4) if size else None
        rc = _struct(_norm_back_at, raw, *members, ws.data_ptr() if size else None, size)
        if rc:
            _check(rc, "ds_norm_backward")
        return dy, dx, grads
