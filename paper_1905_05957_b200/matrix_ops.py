"""Operators on matrices beside the DoubleSqueeze step: layer products in 8-bit integers, whose gradients the workers
compress, and the orthogonalised update that moves the model by what comes back.  Argument marshalling over the C ABI
(include/dsq.h); PyTorch supplies memory and streams.
"""
from __future__ import annotations

import ctypes as C
import math

import torch

from .binding import (DS_BF16, DS_DEV_MMA_TIMEOUT, DS_F16, DS_F32, DS_NEED_BUFFERS, DS_OK, DS_ORTH_NESTEROV, DsqError, ds_orth_config,
                      load_library)

_DTYPES = {torch.float32: DS_F32, torch.bfloat16: DS_BF16, torch.float16: DS_F16}


def _dtype(t: torch.dtype, what: str) -> int:
    if t not in _DTYPES:
        raise TypeError(f"{what}: float32, bfloat16 or float16 expected, got {t}")
    return _DTYPES[t]


def _check(rc: int, what: str):
    if rc != DS_OK:
        raise DsqError(rc, what, load_library().ds_last_error().decode())


def _stream(t: torch.Tensor, stream) -> int:
    return (stream if stream is not None else torch.cuda.current_stream(t.device)).cuda_stream


def _need_cuda(*tensors):
    for t in tensors:
        if t is not None and not t.is_cuda:
            raise ValueError("CUDA tensors expected: there is no CPU path")
        if t is not None and t.device != tensors[0].device:
            raise ValueError("tensors on different devices")


def _matrix(x: torch.Tensor, what: str) -> tuple[torch.Tensor, int]:
    """x as rows of consecutive entries, and the distance between rows."""
    if x.dim() != 2:
        raise ValueError(f"{what}: a matrix expected, got {x.dim()} dimensions")
    if x.shape[1] > 1 and x.stride(1) != 1 or x.shape[0] > 1 and x.stride(0) < x.shape[1]:
        x = x.contiguous()
    return x, (x.stride(0) if x.shape[0] > 1 else x.shape[1])


def _vector(v: torch.Tensor | None, n: int, what: str):
    if v is not None and (v.dtype != torch.float32 or v.shape != (n,) or not v.is_contiguous()):
        raise ValueError(f"{what}: {n} contiguous float32 values expected, got {v.dtype} {tuple(v.shape)}")


_status: dict = {}


def _dev_status(device: torch.device) -> torch.Tensor:
    """The device word in which products report waits that ran out (one per device, kept)."""
    if device not in _status:
        _status[device] = torch.zeros(1, dtype=torch.int32, device=device)
    return _status[device]


def device_status(device: str | torch.device = "cuda") -> int:
    """DS_DEV_* flags of the matrix operators on a device; 0 unless one of them failed.  Waits for the device."""
    device = torch.device(device)
    if device.index is None:
        device = torch.device(device.type, torch.cuda.current_device())
    return int(_dev_status(device).item())


class Int8Matrix:
    """Codes [rows, cols] (int8) with one float32 scale per row: row r stands for codes[r] * scale[r].
    Rows must start on 16-byte boundaries (int8_quantize gives such; pack() copies into such)."""

    __slots__ = ("codes", "scale")

    def __init__(self, codes: torch.Tensor, scale: torch.Tensor):
        if codes.dtype != torch.int8 or codes.dim() != 2 or (codes.shape[1] > 1 and codes.stride(1) != 1):
            raise ValueError("codes: a row-major int8 matrix expected")
        _vector(scale, codes.shape[0], "scale")
        _need_cuda(codes, scale)
        self.codes, self.scale = codes, scale

    @property
    def shape(self):
        return self.codes.shape

    @property
    def ld(self) -> int:
        r, c = self.codes.shape
        return self.codes.stride(0) if r > 1 else (c + 15) // 16 * 16

    @classmethod
    def empty(cls, rows: int, cols: int, device) -> "Int8Matrix":
        pitch = max(16, (cols + 15) // 16 * 16)
        return cls(torch.empty(rows, pitch, dtype=torch.int8, device=device)[:, :cols],
                   torch.empty(rows, dtype=torch.float32, device=device))

    @classmethod
    def pack(cls, codes: torch.Tensor, scale: torch.Tensor) -> "Int8Matrix":
        """A copy of any int8 matrix with its rows on 16-byte boundaries."""
        m = cls.empty(*codes.shape, codes.device)
        m.codes.copy_(codes)
        m.scale.copy_(scale)
        return m

    def dequantize(self) -> torch.Tensor:
        return self.codes.float() * self.scale[:, None]


def int8_quantize(x: torch.Tensor, rows: bool = True, cols: bool = False, col_sum: bool = False, stream=None):
    """Codes of a matrix by rows (Int8Matrix [rows, cols]), by columns (transposed: Int8Matrix [cols, rows]) and its column
    sums, in that order; one thing asked for is returned by itself, several as a tuple."""
    if not (rows or cols or col_sum):
        raise ValueError("nothing to compute")
    _need_cuda(x)
    dt = _dtype(x.dtype, "x")
    x, ld = _matrix(x, "x")
    r, c = x.shape
    lib = load_library()
    by_r = Int8Matrix.empty(r, c, x.device) if rows else None
    by_c = Int8Matrix.empty(c, r, x.device) if cols else None
    total = torch.empty(c, dtype=torch.float32, device=x.device) if col_sum else None
    ws = None
    if cols or col_sum:
        ws = torch.empty(lib.ds_i8_quantize_workspace(r, c, int(col_sum)), dtype=torch.uint8, device=x.device)
    _check(lib.ds_i8_quantize(x.data_ptr(), dt, r, c, ld,
                              by_r.codes.data_ptr() if rows else None, by_r.ld if rows else 0, by_r.scale.data_ptr() if rows else None,
                              by_c.codes.data_ptr() if cols else None, by_c.ld if cols else 0, by_c.scale.data_ptr() if cols else None,
                              None if total is None else total.data_ptr(), None if ws is None else ws.data_ptr(),
                              0 if ws is None else ws.numel(), _stream(x, stream)), "ds_i8_quantize")
    got = [v for v in (by_r, by_c, total) if v is not None]
    return got[0] if len(got) == 1 else tuple(got)


def _out(out, shape, dtype, device):
    if out is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if tuple(out.shape) != tuple(shape) or (out.shape[1] > 1 and out.stride(1) != 1) or (out.shape[0] > 1 and out.stride(0) < out.shape[1]):
        raise ValueError(f"out: a row-major matrix {tuple(shape)} expected, got {tuple(out.shape)}")
    return out


def int8_matmul(a: Int8Matrix, b: Int8Matrix, bias: torch.Tensor | None = None, out_dtype: torch.dtype = torch.bfloat16,
                out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """a b^T (+ bias): [a rows, b rows], the sums exact in 32-bit integers."""
    if a.shape[1] != b.shape[1]:
        raise ValueError(f"lengths differ: {a.shape[1]} and {b.shape[1]}")
    m, n, k = a.shape[0], b.shape[0], a.shape[1]
    _vector(bias, n, "bias")
    _need_cuda(a.codes, b.codes, bias, out)
    out = _out(out, (m, n), out_dtype, a.codes.device)
    ldo = out.stride(0) if m > 1 else n
    _check(load_library().ds_i8_matmul(a.codes.data_ptr(), a.ld, a.scale.data_ptr(), b.codes.data_ptr(), b.ld, b.scale.data_ptr(),
                                       None if bias is None else bias.data_ptr(), m, n, k, out.data_ptr(), _dtype(out.dtype, "out"), ldo,
                                       _dev_status(out.device).data_ptr(), _stream(out, stream)), "ds_i8_matmul")
    return out


def int8_linear(x: torch.Tensor, w: Int8Matrix, bias: torch.Tensor | None = None, out_dtype: torch.dtype | None = None,
                out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """x W^T (+ bias) for weights quantised before: x [tokens, k] is quantised by rows on the way."""
    _need_cuda(x, w.codes, bias, out)
    dt = _dtype(x.dtype, "x")
    x, ld = _matrix(x, "x")
    m, k = x.shape
    n = w.shape[0]
    if w.shape[1] != k:
        raise ValueError(f"x has {k} columns, the weights {w.shape[1]}")
    _vector(bias, n, "bias")
    out = _out(out, (m, n), out_dtype or x.dtype, x.device)
    lib = load_library()
    ws = torch.empty(max(16, lib.ds_i8_linear_workspace(m, k)), dtype=torch.uint8, device=x.device)
    _check(lib.ds_i8_linear(x.data_ptr(), dt, m, k, ld, w.codes.data_ptr(), w.ld, w.scale.data_ptr(),
                            None if bias is None else bias.data_ptr(), n, out.data_ptr(), _dtype(out.dtype, "out"),
                            out.stride(0) if m > 1 else n, ws.data_ptr(), ws.numel(), _dev_status(x.device).data_ptr(),
                            _stream(x, stream)), "ds_i8_linear")
    return out


class Int8Linear:
    """A linear layer y = x W^T (+ bias) whose three products run in 8-bit integers.

    W [out, in] (float32, bfloat16 or float16) is quantised by rows for the forward product and by columns for the gradient
    of the inputs; call set_weight() after every change of W.  forward(x, training=True) keeps the column codes of x (one byte
    an entry) for the gradient of the weights."""

    def __init__(self, weight: torch.Tensor, bias: torch.Tensor | None = None, training: bool = True, stream=None):
        self.bias = bias
        self.set_weight(weight, training, stream)

    def set_weight(self, weight: torch.Tensor, training: bool = True, stream=None):
        if training:
            self.by_rows, self.by_cols = int8_quantize(weight, rows=True, cols=True, stream=stream)
        else:
            self.by_rows, self.by_cols = int8_quantize(weight, stream=stream), None
        self._x_cols = None

    def forward(self, x: torch.Tensor, training: bool = False, out_dtype: torch.dtype | None = None, stream=None) -> torch.Tensor:
        if not training:
            return int8_linear(x, self.by_rows, self.bias, out_dtype, stream=stream)
        rows, self._x_cols = int8_quantize(x, rows=True, cols=True, stream=stream)
        return int8_matmul(rows, self.by_rows, self.bias, out_dtype or x.dtype, stream=stream)

    def backward(self, dy: torch.Tensor, dx_dtype: torch.dtype | None = None, dw_dtype: torch.dtype = torch.float32,
                 dw: torch.Tensor | None = None, stream=None):
        """(dx, dw, db) of the last training forward; db is None for a layer without bias.  `dw` may be a [out, in] view of
        a gradient row of DoubleSqueeze."""
        if self._x_cols is None or self.by_cols is None:
            raise RuntimeError("backward needs a forward with training=True before it")
        if dy.dim() != 2 or dy.shape != (self._x_cols.shape[1], self.by_rows.shape[0]):
            raise ValueError(f"dy: {(self._x_cols.shape[1], self.by_rows.shape[0])} expected, got {tuple(dy.shape)}")
        got = int8_quantize(dy, rows=True, cols=True, col_sum=self.bias is not None, stream=stream)
        dx = int8_matmul(got[0], self.by_cols, out_dtype=dx_dtype or dy.dtype, stream=stream)
        dw = int8_matmul(got[1], self._x_cols, out_dtype=dw_dtype, out=dw, stream=stream)
        return dx, dw, got[2] if self.bias is not None else None


class OrthUpdate:
    """Momentum and Newton-Schulz orthogonalisation for `batch` matrices [rows, cols] (the Muon optimiser's update).

    A plan for one shape: it owns the workspace, not the momentum.  `stride`: elements between the matrices in g, momentum
    and x (0: rows * cols).  `scale` multiplies the model update; the default is sqrt(max(1, rows / cols))."""

    def __init__(self, rows: int, cols: int, batch: int = 1, momentum: float = 0.95, nesterov: bool = True,
                 coef: tuple[float, float, float] = (3.4445, -4.7750, 2.0315), steps: int = 5, eps: float = 1e-7,
                 scale: float | None = None, stride: int = 0, device: str | torch.device = "cuda"):
        if not torch.cuda.is_available():
            raise RuntimeError("paper_1905_05957_b200 needs a CUDA device; there is no CPU path")
        self.lib = load_library()
        self.rows, self.cols, self.batch, self.stride = rows, cols, batch, stride or rows * cols
        if scale is None:
            scale = math.sqrt(max(1.0, rows / cols)) if cols > 0 else 1.0
        self.cfg = ds_orth_config(rows, cols, batch, steps, *coef, momentum, eps, scale, DS_ORTH_NESTEROV if nesterov else 0, 0, stride)
        size = C.c_size_t(0)
        rc = self.lib.ds_orth_create(C.byref(self.cfg), None, C.byref(size), None, None)
        if rc != DS_NEED_BUFFERS:
            raise DsqError(rc, "ds_orth_create (size query)")
        self.workspace = torch.zeros(size.value, dtype=torch.uint8, device=device)
        self.device = self.workspace.device
        self.dev_status = torch.zeros(4, dtype=torch.int32, device=device)
        h = C.c_void_p()
        _check(self.lib.ds_orth_create(C.byref(self.cfg), self.workspace.data_ptr(), C.byref(size), self.dev_status.data_ptr(),
                                       C.byref(h)), "ds_orth_create")
        self.handle = h

    def _span(self, t: torch.Tensor | None, what: str, dtypes) -> int | None:
        """t holds the matrices `stride` apart: a contiguous tensor of at least (batch - 1) * stride + rows * cols entries."""
        if t is None:
            return None
        need = (self.batch - 1) * self.stride + self.rows * self.cols
        if t.dtype not in dtypes or t.device != self.device or not t.is_contiguous() or t.numel() < need:
            raise ValueError(f"{what}: at least {need} contiguous entries of {dtypes} on {self.device} expected, "
                             f"got {t.numel()} of {t.dtype} on {t.device}")
        return t.data_ptr()

    def update(self, g: torch.Tensor, momentum: torch.Tensor | None = None, out: torch.Tensor | None = None,
               out_dtype: torch.dtype | None = torch.bfloat16, x: torch.Tensor | None = None, gamma: float = 0.0, decay: float = 0.0,
               stream=None) -> torch.Tensor | None:
        """One update.  momentum (float32) is advanced in place.  Returns the orthogonalised update [batch, rows, cols] in
        `out` or a new tensor of out_dtype (None: not wanted).  x (float32): also x = x (1 - gamma decay) - gamma scale update."""
        if out is None and out_dtype is not None:
            out = torch.empty(self.batch, self.rows, self.cols, dtype=out_dtype, device=self.device)
        if out is not None and (out.dtype not in (torch.float32, torch.bfloat16) or not out.is_contiguous()
                                or out.numel() != self.batch * self.rows * self.cols or out.device != self.device):
            raise ValueError("out: a contiguous float32 or bfloat16 tensor [batch, rows, cols] expected")
        gp = self._span(g, "g", tuple(_DTYPES))
        mp = self._span(momentum, "momentum", (torch.float32,))
        xp = self._span(x, "x", (torch.float32,))
        _check(self.lib.ds_orth_update(self.handle, gp, _DTYPES[g.dtype], mp, None if out is None else out.data_ptr(),
                                       DS_F32 if out is None else _DTYPES[out.dtype], xp, gamma, decay,
                                       _stream(g, stream)), "ds_orth_update")
        return out

    def timed_out(self) -> bool:
        """Whether a product of this plan ever gave up waiting (DS_DEV_MMA_TIMEOUT).  Waits for the device."""
        return bool(int(self.dev_status[0].item()) & DS_DEV_MMA_TIMEOUT)

    def close(self):
        if getattr(self, "handle", None):
            self.lib.ds_orth_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
