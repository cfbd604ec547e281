"""Operators on matrices beside the DoubleSqueeze step: layer products in 8-bit integers, whose gradients the workers
compress, and the orthogonalised update that moves the model by what comes back.  Argument marshalling over the C ABI
(include/dsq.h); PyTorch supplies memory and streams.

The calls stand outside autograd, like the rest of the package: a result carries no gradient, whatever its arguments require.
Int8Linear.backward gives a layer's gradients.
"""
from __future__ import annotations

import ctypes as C
import math

import torch

from .binding import (DS_BF16, DS_DEV_MMA_TIMEOUT, DS_F16, DS_F32, DS_NEED_BUFFERS, DS_OK, DS_ORTH_NESTEROV, DsqError, ds_orth_config,
                      fast_call,
                      load_library)

_DTYPES = {torch.float32: DS_F32, torch.bfloat16: DS_BF16, torch.float16: DS_F16}
_raw_stream = torch._C._cuda_getCurrentRawStream
_current = torch._C._cuda_getDevice
_empty = torch.empty
_call = _quantize_at = _matmul_at = _linear_at = _quantize_ws = _linear_ws = None


def _load():
    """Looks the library's functions up once: the calls below are short enough for every look-up to show."""
    global _call, _quantize_at, _matmul_at, _linear_at, _quantize_ws, _linear_ws
    lib = load_library()
    _call, address = fast_call()
    _quantize_at, _matmul_at, _linear_at = (address[n] for n in ("ds_i8_quantize", "ds_i8_matmul", "ds_i8_linear"))
    _quantize_ws, _linear_ws = lib.ds_i8_quantize_workspace, lib.ds_i8_linear_workspace


def _dtype(t: torch.dtype, what: str) -> int:
    code = _DTYPES.get(t)
    if code is None:
        raise TypeError(f"{what}: float32, bfloat16 or float16 expected, got {t}")
    return code


def _check(rc: int, what: str):
    if rc != DS_OK:
        raise DsqError(rc, what, load_library().ds_last_error().decode())


def _matrix(x: torch.Tensor, what: str) -> tuple[torch.Tensor, int, int, int, torch.device]:
    """x as rows of consecutive entries; rows, columns, the distance between rows, the device."""
    if not x.is_cuda:
        raise ValueError(f"{what}: a CUDA tensor expected: there is no CPU path")
    shape = x.shape
    if len(shape) != 2:
        raise ValueError(f"{what}: a matrix expected, got {len(shape)} dimensions")
    r, c = shape
    ld, step = x.stride()
    if (c > 1 and step != 1) or (r > 1 and ld < c):
        x = x.contiguous()
        ld = c
    return x, r, c, (ld if r > 1 else c), x.device


def _vector(v: torch.Tensor | None, n: int, what: str, device) -> int | None:
    """The address of n contiguous float32 values on `device`, or None."""
    if v is None:
        return None
    if v.dtype is not torch.float32 or v.shape != (n,) or not v.is_contiguous():
        raise ValueError(f"{what}: {n} contiguous float32 values expected, got {v.dtype} {tuple(v.shape)}")
    if v.device != device:
        raise ValueError(f"{what}: on {v.device}, the others on {device}")
    return v.data_ptr()


_streams: dict = {}    # (device index, handle) -> the stream


def _stream_of(index: int, raw: int) -> torch.cuda.Stream:
    """The current stream, whose handle is raw."""
    stream = _streams.get((index, raw))
    if stream is None:
        stream = _streams[index, raw] = torch.cuda.current_stream(index)
    return stream


_status: dict = {}     # device index -> (word in which products report waits that ran out, its address)


def _dev_status(index: int) -> int | None:
    """The address of the device's status word, made when codes or products are first asked for.  None while a graph is captured on a
    device that has none yet: it cannot be made then, and the captured products report nothing."""
    entry = _status.get(index)
    if entry is None:
        if torch.cuda.is_current_stream_capturing():
            return None
        word = torch.zeros(1, dtype=torch.int32, device=torch.device("cuda", index))
        torch.cuda.synchronize(index)          # cleared before any stream's product may set it
        entry = _status[index] = (word, word.data_ptr())
    return entry[1]


def device_status(device: str | torch.device = "cuda") -> int:
    """DS_DEV_* flags of the matrix operators on a device; 0 unless one of them failed.  (Products captured into a graph before any
    call of these operators on the device do not report.)  Waits for the device."""
    device = torch.device(device)
    index = torch.cuda.current_device() if device.index is None else device.index
    _dev_status(index)
    torch.cuda.synchronize(index)              # products on other streams, too
    return int(_status[index][0].item())


class Int8Matrix:
    """Codes [rows, cols] (int8, from -127 to 127) with one float32 scale per row: row r stands for codes[r] * scale[r].
    Rows must start on 16-byte boundaries (int8_quantize gives such; pack() copies into such)."""

    __slots__ = ("rows", "cols", "ld", "device", "codes_ptr", "scale_ptr", "_codes", "_scale", "stream")

    def __init__(self, codes: torch.Tensor, scale: torch.Tensor):
        if codes.dtype is not torch.int8 or not codes.is_cuda:
            raise ValueError("codes: a row-major int8 matrix on a CUDA device expected: there is no CPU path")
        r, c = codes.shape
        ld, step = codes.stride()
        if c > 1 and step != 1:
            raise ValueError("codes: a row-major int8 matrix expected")
        device = codes.device
        self.rows, self.cols, self.device = r, c, device
        self.ld = ld if r > 1 else (c + 15) // 16 * 16
        self._codes, self._scale = codes, scale
        self.stream = None                           # the last one on which the allocator takes the memory to be in use: the caller's may belong to any
        self.codes_ptr, self.scale_ptr = codes.data_ptr(), _vector(scale, r, "scale", device)

    @classmethod
    def _within(cls, buf: torch.Tensor, base: int, at: int, scale_at: int, rows: int, cols: int, ld: int, device, stream: int) -> "Int8Matrix":
        """Codes and scales at two offsets of one byte buffer whose address is `base`; views are made when asked for."""
        m = cls.__new__(cls)
        m.rows, m.cols, m.ld, m.device = rows, cols, ld, device
        m.codes_ptr, m.scale_ptr, m.stream = base + at, base + scale_at, stream
        m._codes, m._scale = (buf, at), (buf, scale_at)
        return m

    def used_on(self, stream: int):
        """Tells the allocator of the current stream, on which the matrix is about to be used: dropped before that has run, its memory is
        kept until it has."""
        current = _stream_of(self.device.index, stream)
        for t in (self._codes, self._scale):
            (t[0] if isinstance(t, tuple) else t).record_stream(current)
        self.stream = stream

    @property
    def codes(self) -> torch.Tensor:
        if isinstance(self._codes, tuple):
            buf, at = self._codes
            self._codes = buf.view(torch.int8).as_strided((self.rows, self.cols), (self.ld, 1), at)
        return self._codes

    @property
    def scale(self) -> torch.Tensor:
        if isinstance(self._scale, tuple):
            buf, at = self._scale
            self._scale = buf[at:at + 4 * self.rows].view(torch.float32)
        return self._scale

    @property
    def shape(self):
        return torch.Size((self.rows, self.cols))

    @classmethod
    def pack(cls, codes: torch.Tensor, scale: torch.Tensor) -> "Int8Matrix":
        """A copy of any int8 matrix with its rows on 16-byte boundaries."""
        r, c = codes.shape
        out = _empty(r, max(16, (c + 15) // 16 * 16), dtype=torch.int8, device=codes.device)[:, :c]
        out.copy_(codes)
        return cls(out, scale.to(torch.float32, copy=True))

    def dequantize(self) -> torch.Tensor:
        return self.codes.float() * self.scale[:, None]


def int8_quantize(x: torch.Tensor, rows: bool = True, cols: bool = False, col_sum: bool = False, stream=None):
    """Codes of a matrix by rows (Int8Matrix [rows, cols]), by columns (transposed: Int8Matrix [cols, rows]) and its column
    sums, in that order; one thing asked for is returned by itself, several as a tuple."""
    if not (rows or cols or col_sum):
        raise ValueError("nothing to compute")
    if stream is not None:
        with torch.cuda.stream(stream):      # what is allocated here belongs to the stream that uses it
            return int8_quantize(x, rows, cols, col_sum)
    if _call is None:
        _load()
    dt = _dtype(x.dtype, "x")
    x, r, c, ld, device = _matrix(x, "x")
    index = device.index
    if index != _current():                  # the library works on the current device
        with torch.cuda.device(device):
            return int8_quantize(x, rows, cols, col_sum)
    # one buffer: codes, scales, sums, and at its end what only the call itself uses
    ldr, ldc = (c + 15) // 16 * 16 or 16, (r + 15) // 16 * 16 or 16
    at_c = r * ldr if rows else 0
    at_rs = at_c + (c * ldc if cols else 0)
    at_cs = at_rs + (4 * ldc if rows else 0)
    at_sum = at_cs + (4 * ldr if cols else 0)
    at_ws = at_sum + (4 * ldr if col_sum else 0)
    ws = _quantize_ws(r, c, 1 if col_sum else 0) if cols or col_sum else 0
    buf = _empty(at_ws + ws + 16, dtype=torch.uint8, device=device)
    base = buf.data_ptr()
    if index not in _status:
        _dev_status(index)
    raw = _raw_stream(index)
    rc = _call(_quantize_at, x.data_ptr(), dt, r, c, ld, base if rows else 0, ldr, base + at_rs if rows else 0,
               base + at_c if cols else 0, ldc, base + at_cs if cols else 0, base + at_sum if col_sum else 0,
               base + at_ws if ws else 0, ws, raw)
    if rc:
        _check(rc, "ds_i8_quantize")
    got = []
    if rows:
        got.append(Int8Matrix._within(buf, base, 0, at_rs, r, c, ldr, device, raw))
    if cols:
        got.append(Int8Matrix._within(buf, base, at_c, at_cs, c, r, ldc, device, raw))
    if col_sum:
        got.append(buf[at_sum:at_sum + 4 * c].view(torch.float32))
    return got[0] if len(got) == 1 else tuple(got)


def _out(out: torch.Tensor, m: int, n: int, device) -> int:
    """The distance between the rows of a given output."""
    if out.shape != (m, n) or out.device != device:
        raise ValueError(f"out: a matrix {(m, n)} on {device} expected, got {tuple(out.shape)} on {out.device}")
    ld, step = out.stride()
    if (n > 1 and step != 1) or (m > 1 and ld < n):
        raise ValueError("out: rows of consecutive entries expected")
    return ld if m > 1 else n


def int8_matmul(a: Int8Matrix, b: Int8Matrix, bias: torch.Tensor | None = None, out_dtype: torch.dtype = torch.bfloat16,
                out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """a b^T (+ bias): [a rows, b rows], the sums exact in 32-bit integers."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return int8_matmul(a, b, bias, out_dtype, out)
    if _call is None:
        _load()
    m, n, k, device = a.rows, b.rows, a.cols, a.device
    if b.cols != k:
        raise ValueError(f"lengths differ: {k} and {b.cols}")
    if b.device != device:
        raise ValueError(f"matrices on {device} and {b.device}")
    index = device.index
    if index != _current():
        with torch.cuda.device(device):
            return int8_matmul(a, b, bias, out_dtype, out)
    bp = None if bias is None else _vector(bias, n, "bias", device)
    if out is None:
        out, ldo = _empty((m, n), dtype=out_dtype, device=device), n
    else:
        ldo = _out(out, m, n, device)
    raw = _raw_stream(index)
    if a.stream != raw:
        a.used_on(raw)
    if b.stream != raw:
        b.used_on(raw)
    rc = _call(_matmul_at, a.codes_ptr, a.ld, a.scale_ptr, b.codes_ptr, b.ld, b.scale_ptr, bp, m, n, k, out.data_ptr(),
               _dtype(out.dtype, "out"), ldo, _dev_status(index), raw)
    if rc:
        _check(rc, "ds_i8_matmul")
    return out


def int8_linear(x: torch.Tensor, w: Int8Matrix, bias: torch.Tensor | None = None, out_dtype: torch.dtype | None = None,
                out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """x W^T (+ bias) for weights quantised before: x [tokens, k] is quantised by rows on the way.  No gradient flows back through it.
    `out` may not overlap x."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return int8_linear(x, w, bias, out_dtype, out)
    if _call is None:
        _load()
    dt = _dtype(x.dtype, "x")
    x, m, k, ld, device = _matrix(x, "x")
    n = w.rows
    if w.cols != k:
        raise ValueError(f"x has {k} columns, the weights {w.cols}")
    if w.device != device:
        raise ValueError(f"x on {device}, the weights on {w.device}")
    index = device.index
    if index != _current():
        with torch.cuda.device(device):
            return int8_linear(x, w, bias, out_dtype, out)
    bp = None if bias is None else _vector(bias, n, "bias", device)
    if out is not None:
        ldo, odt = _out(out, m, n, device), _dtype(out.dtype, "out")
        if m and n and k:      # with few tokens some blocks still read x when others store
            first, last = x.data_ptr(), x.data_ptr() + ((m - 1) * ld + k) * x.element_size()
            if out.data_ptr() < last and first < out.data_ptr() + ((m - 1) * ldo + n) * out.element_size():
                raise ValueError("out: overlaps x")
    elif out_dtype is None:
        out, ldo, odt = x.new_empty((m, n)), n, dt
    else:
        out, ldo, odt = _empty((m, n), dtype=out_dtype, device=device), n, _dtype(out_dtype, "out")
    size = _linear_ws(m, k, n)
    ws = _empty(size, dtype=torch.uint8, device=device) if size else None
    raw = _raw_stream(index)
    if w.stream != raw:
        w.used_on(raw)
    rc = _call(_linear_at, x.data_ptr(), dt, m, k, ld, w.codes_ptr, w.ld, w.scale_ptr, bp, n, out.data_ptr(), odt, ldo,
               ws.data_ptr() if size else None, size, _dev_status(index), raw)
    if rc:
        _check(rc, "ds_i8_linear")
    return out


class Int8Linear:
    """A linear layer y = x W^T (+ bias) whose three products run in 8-bit integers.

    W [out, in] (float32, bfloat16 or float16) is quantised by rows for the forward product and by columns for the gradient
    of the inputs; call set_weight() after every change of W.  The bias is float32.  forward(x, training=True) keeps the column codes of x (one byte
    an entry) for the gradient of the weights."""

    def __init__(self, weight: torch.Tensor, bias: torch.Tensor | None = None, training: bool = True, stream=None):
        self._bias, self._on = bias, {}
        self.set_weight(weight, training, stream)

    @property
    def bias(self) -> torch.Tensor | None:
        return self._bias

    @bias.setter
    def bias(self, bias: torch.Tensor | None):
        self._bias, self._on = bias, {}

    def set_weight(self, weight: torch.Tensor, training: bool = True, stream=None):
        if training:
            self.by_rows, self.by_cols = int8_quantize(weight, rows=True, cols=True, stream=stream)
        else:
            self.by_rows, self.by_cols = int8_quantize(weight, stream=stream), None
        self._x_cols = None

    def forward(self, x: torch.Tensor, training: bool = False, out_dtype: torch.dtype | None = None, stream=None) -> torch.Tensor:
        if not training:
            y = int8_linear(x, self.by_rows, self._bias, out_dtype, stream=stream)
        else:
            rows, self._x_cols = int8_quantize(x, rows=True, cols=True, stream=stream)
            y = int8_matmul(rows, self.by_rows, self._bias, out_dtype or x.dtype, stream=stream)
        if self._bias is not None:
            index = self.by_rows.device.index
            raw = _raw_stream(index) if stream is None else stream.cuda_stream
            if self._on.get(raw) != self._bias.data_ptr():      # the allocator is told of a stream that uses the bias, which may belong to any, for the first time
                self._bias.record_stream(_stream_of(index, raw) if stream is None else stream)
                self._on[raw] = self._bias.data_ptr()
        return y

    def backward(self, dy: torch.Tensor, dx_dtype: torch.dtype | None = None, dw_dtype: torch.dtype = torch.float32,
                 dw: torch.Tensor | None = None, stream=None):
        """(dx, dw, db) of the last training forward; db is None for a layer without bias.  `dw` may be a [out, in] view of
        a gradient row of DoubleSqueeze."""
        if self._x_cols is None or self.by_cols is None:
            raise RuntimeError("backward needs a forward with training=True before it")
        if dy.dim() != 2 or dy.shape != (self._x_cols.cols, self.by_rows.rows):
            raise ValueError(f"dy: {(self._x_cols.cols, self.by_rows.rows)} expected, got {tuple(dy.shape)}")
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
        self.workspace = torch.empty(size.value, dtype=torch.uint8, device=device)
        self.device = self.workspace.device
        self.dev_status = torch.zeros(4, dtype=torch.int32, device=device)
        self._last_stream = _raw_stream(self.device.index)     # where the allocator takes both to be in use
        torch.cuda.synchronize(self.device)      # cleared before a product on any stream may set it
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
        `out` or a new tensor of out_dtype (None: not wanted).  x (float32): also x = x (1 - gamma decay) - gamma scale update.
        One plan works on one stream at a time: its workspace holds the matrices between the products.  Tensors that the caller
        allocated on another stream follow PyTorch's rules (record_stream), the plan's own memory needs nothing."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.update(g, momentum, out, out_dtype, x, gamma, decay)
        if self.device.index != _current():
            with torch.cuda.device(self.device):
                return self.update(g, momentum, out, out_dtype, x, gamma, decay)
        if out is None and out_dtype is not None:
            out = torch.empty(self.batch, self.rows, self.cols, dtype=out_dtype, device=self.device)
        if out is not None and (out.dtype not in (torch.float32, torch.bfloat16) or not out.is_contiguous()
                                or out.numel() != self.batch * self.rows * self.cols or out.device != self.device):
            raise ValueError("out: a contiguous float32 or bfloat16 tensor [batch, rows, cols] expected")
        gp = self._span(g, "g", tuple(_DTYPES))
        mp = self._span(momentum, "momentum", (torch.float32,))
        xp = self._span(x, "x", (torch.float32,))
        raw = _raw_stream(self.device.index)
        if raw != self._last_stream:             # a plan that is dropped before this stream has run keeps its memory until it has
            used = torch.cuda.current_stream(self.device)
            self.workspace.record_stream(used)
            self.dev_status.record_stream(used)
            self._last_stream = raw
        _check(self.lib.ds_orth_update(self.handle, gp, _DTYPES[g.dtype], mp, None if out is None else out.data_ptr(),
                                       DS_F32 if out is None else _DTYPES[out.dtype], xp, gamma, decay, raw), "ds_orth_update")
        return out

    def timed_out(self) -> bool:
        """Whether a product of this plan ever gave up waiting (DS_DEV_MMA_TIMEOUT).  Waits for the device."""
        torch.cuda.synchronize(self.device)
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
