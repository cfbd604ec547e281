"""8-bit layer products on the GPU against plain arithmetic: codes bit for bit against the formula in 32 bits, sums exactly (they
are whole numbers), scaled results against 64 bits within the roundings the formula has."""
import numpy as np
import pytest
import torch

from paper_1905_05957_b200 import DsqError, Int8Linear, Int8Matrix, OrthUpdate, binding, int8_linear, int8_matmul, int8_quantize, matrix_ops
from paper_1905_05957_b200.matrix_ops import device_status

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U32 = 2.0 ** -24            # half a unit in the last place, relative


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _want_codes(x: torch.Tensor):
    """The formula in numpy, 32 bits, one operation at a time; rows."""
    v = x.float().cpu().numpy()
    if v.shape[1] == 0:
        return np.zeros(v.shape, np.int8), np.zeros(v.shape[0], np.float32)
    with np.errstate(all="ignore"):
        top = np.abs(v).max(1)
        s = (top * np.float32(1 / 127)).astype(np.float32)
        s[s < np.float32(2.0 ** -126)] = 0
        inv = np.where(s > 0, np.float32(1) / s, 0).astype(np.float32)
        bad = ~np.isfinite(top)
        s[bad], inv[bad] = np.nan, 0
        q = np.rint(np.nan_to_num(v * inv[:, None], nan=0.0))
    return q.astype(np.int8), s


def _check_codes(m: Int8Matrix, x: torch.Tensor):
    q, s = _want_codes(x)
    assert np.array_equal(m.codes.cpu().numpy(), q)
    assert np.array_equal(m.scale.cpu().numpy(), s, equal_nan=True)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 17), (3, 16), (5, 31), (130, 257), (64, 1024), (129, 4100), (2, 20_011), (700, 63)])
def test_codes_by_rows_and_columns(dtype, rows, cols):
    x = (torch.randn(rows, cols, device="cuda", generator=_gen(rows * 31 + cols)) * 3).to(dtype)
    _check_codes(int8_quantize(x), x)
    by_r, by_c, total = int8_quantize(x, rows=True, cols=True, col_sum=True)
    _check_codes(by_r, x)
    _check_codes(by_c, x.T)
    _check_codes(int8_quantize(x, rows=False, cols=True), x.T)
    only = int8_quantize(x, rows=False, col_sum=True)
    assert torch.equal(only, total)                     # the same order of additions whatever else is asked for
    # a sum of `rows` terms in any order of two levels: (64 / 8 + 8 + rows / 64) roundings of partial sums at most
    bound = (16 + rows / 64 + 1) * U32 * x.double().abs().sum(0)
    assert ((total.double() - x.double().sum(0)).abs() <= bound + 1e-30).all()


def test_codes_of_views_and_odd_pitches():
    g = _gen(5)
    store = torch.randn(70, 301, device="cuda", generator=g)
    for x in (store[:, :300], store[:, 1:200], store[3:40, 7:8], store.T, store.T[5:9], store[::2, 4:100], store.to(BF16)[:, 3:60]):
        by_r, by_c = int8_quantize(x, rows=True, cols=True)
        _check_codes(by_r, x)
        _check_codes(int8_quantize(x), x)
        _check_codes(by_c, x.T)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(5, 31), (40, 24), (333, 500), (600, 1000), (257, 1153), (1000, 72)])
def test_codes_into_wider_matrices_leave_what_lies_between(dtype, rows, cols):
    x = (torch.randn(rows, cols, device="cuda", generator=_gen(rows + cols)) * 3).to(dtype)
    end_r, end_c = (cols + 15) // 16 * 16, (rows + 15) // 16 * 16      # the codes' ends, by rows and by columns
    for with_cols in (False, True):
        q = torch.full((rows, end_r + 208), 77, dtype=torch.int8, device="cuda")
        qt = torch.full((cols, end_c + 208), 77, dtype=torch.int8, device="cuda")
        s, st = torch.empty(rows, device="cuda"), torch.empty(cols, device="cuda")
        lib = binding.load_library()
        size = lib.ds_i8_quantize_workspace(rows, cols, 0)
        ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        code = {F32: 0, BF16: 1}[dtype]
        by_cols = (qt.data_ptr(), qt.stride(0), st.data_ptr()) if with_cols else (None, 0, None)
        assert lib.ds_i8_quantize(x.data_ptr(), code, rows, cols, cols, q.data_ptr(), q.stride(0), s.data_ptr(), *by_cols, None,
                                  ws.data_ptr(), size, torch.cuda.current_stream().cuda_stream) == 0
        _check_codes(Int8Matrix(q[:, :cols], s), x)
        assert (q[:, cols:end_r] == 0).all() and (q[:, end_r:] == 77).all()
        if with_cols:
            _check_codes(Int8Matrix(qt[:, :rows], st), x.T)
            assert (qt[:, rows:end_c] == 0).all() and (qt[:, end_c:] == 77).all()
        else:
            assert (qt == 77).all()


def test_lines_of_zeros_tiny_infinite_and_nan():
    x = torch.randn(9, 40, device="cuda", generator=_gen(9))
    x[1] = 0
    x[2] = 1e-42                   # the scale would be subnormal
    x[3, 5] = float("inf")
    x[4, 6] = float("nan")
    x[5] = 3.4e38
    x[6] *= 1e-36
    x[7, 3] = -float("inf")
    x[:, 11] = 0
    by_r, by_c = int8_quantize(x, rows=True, cols=True)
    _check_codes(by_r, x)
    _check_codes(by_c, x.T)
    _check_codes(int8_quantize(x), x)
    assert by_r.scale[1] == 0 and by_r.scale[2] == 0 and by_c.scale[11] == 0
    assert torch.isnan(by_r.scale[[3, 4, 7]]).all() and torch.isnan(by_c.scale[[3, 5, 6]]).all()
    w = int8_quantize(torch.randn(33, 40, device="cuda", generator=_gen(10)))
    y = int8_matmul(by_r, w, out_dtype=F32)
    assert torch.isnan(y[[3, 4, 7]]).all() and (y[[1, 2]] == 0).all() and torch.isfinite(y[[0, 6, 8]]).all()
    # from left to right, each operation rounded: what passes the largest number of 32 bits on the way is infinite
    want = (by_r.codes.double() @ w.codes.double().T).float() * by_r.scale[:, None] * w.scale[None, :]
    assert torch.isinf(want[5]).any() and torch.equal(y.nan_to_num(nan=7.0), want.nan_to_num(nan=7.0))
    y = int8_linear(x, w, out_dtype=F32)
    assert torch.isnan(y[[3, 4, 7]]).all() and (y[[1, 2]] == 0).all()


def _random_codes(rows, cols, seed, extreme=False):
    g = _gen(seed)
    q = torch.randint(-127, 128, (rows, cols), device="cuda", generator=g, dtype=torch.int8)
    if extreme:
        q = torch.where(q > 0, 127, 127).to(torch.int8)
    return Int8Matrix.pack(q, torch.rand(rows, device="cuda", generator=g) + 0.5)


def _want_product(a, b, bias):
    s = a.codes.double() @ b.codes.double().T                # whole numbers below 2^53: exact
    y = s * a.scale.double()[:, None] * b.scale.double()[None, :]
    return y if bias is None else y + bias.double()


def _check_product(y, a, b, bias):
    want = _want_product(a, b, bias)
    if y.dtype != F32:         # the 32-bit result, rounded once
        full = int8_matmul(a, b, bias, out_dtype=F32)
        assert torch.equal(y, full.to(y.dtype))
        y = full
    # conversion of the sum, two multiplications, one addition
    plain = want if bias is None else want - bias.double()
    bound = 3.01 * U32 * plain.abs() + 2.01 * U32 * want.abs() + 1e-30
    err = (y.double() - want).abs()
    assert (err <= bound).all(), (float((err - bound).max()), int((err > bound).sum()), tuple(y.shape))


@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 8, 16), (1, 40, 4097), (2, 129, 33), (7, 100, 1000), (8, 64, 512), (9, 65, 512), (16, 300, 4096),
                                   (17, 257, 700), (33, 16, 64), (64, 640, 2048), (65, 31, 130), (127, 128, 127), (128, 256, 128), (129, 257, 129),
                                   (300, 500, 1001), (1000, 72, 333), (513, 1030, 770), (2048, 1537, 96)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_products(m, n, k, dtype):
    a, b = _random_codes(m, k, 1), _random_codes(n, k, 2)
    bias = torch.randn(n, device="cuda", generator=_gen(3)) * 100 if (m + n) % 2 else None
    _check_product(int8_matmul(a, b, bias, out_dtype=dtype), a, b, bias)
    assert device_status() == 0


def test_products_at_the_largest_length_do_not_overflow():
    k = binding.DS_I8_MAX_K
    a, b = _random_codes(3, k, 1, extreme=True), _random_codes(130, k, 2, extreme=True)
    _check_product(int8_matmul(a, b, out_dtype=F32), a, b, None)
    b.codes[::2] *= -1
    _check_product(int8_matmul(a, b, out_dtype=F32), a, b, None)


def test_product_into_strided_and_odd_outputs_and_fp16():
    a, b = _random_codes(140, 200, 1), _random_codes(70, 200, 2)
    bias = torch.randn(71, device="cuda", generator=_gen(3))[1:]       # starts 4 bytes past a boundary
    store = torch.full((141, 91), -7.0, device="cuda")
    out = store[1:, 3:73]
    assert int8_matmul(a, b, bias, out=out) is out
    _check_product(out, a, b, bias)
    assert (store[0] == -7).all() and (store[:, :3] == -7).all() and (store[:, 73:] == -7).all()
    _check_product(int8_matmul(a, b, out_dtype=F16), a, b, None)


def test_empty_products():
    a, b = _random_codes(5, 0, 1), _random_codes(300, 0, 2)
    bias = torch.randn(300, device="cuda", generator=_gen(3))
    assert torch.equal(int8_matmul(a, b, bias, out_dtype=F32), bias.expand(5, 300))
    assert (int8_matmul(a, b) == 0).all()
    a, b = _random_codes(0, 64, 1), _random_codes(30, 64, 2)
    assert int8_matmul(a, b).shape == (0, 30) and int8_matmul(b, a).shape == (30, 0)
    x = torch.empty(0, 64, device="cuda")
    assert int8_linear(x, b).shape == (0, 30)
    by_r, by_c, total = int8_quantize(x, rows=True, cols=True, col_sum=True)
    assert by_r.shape == (0, 64) and by_c.shape == (64, 0) and (by_c.scale == 0).all() and (total == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("m", [1, 2, 3, 4, 5, 8, 9, 16, 24, 33, 64, 100, 200])
@pytest.mark.parametrize("n,k", [(130, 300), (1024, 2048), (47, 8200)])
def test_linear_equals_quantise_and_multiply(dtype, m, n, k):
    """int8_linear has forms of its own for few tokens: the codes are the same whole numbers, so the results agree bit for bit."""
    g = _gen(m * 7 + n)
    x = (torch.randn(m, k, device="cuda", generator=g) * 2).to(dtype)
    if m > 2:
        x[1] = 0
    w = int8_quantize(torch.randn(n, k, device="cuda", generator=g))
    w.codes.as_strided((n, w.ld), (w.ld, 1))[:, k:] = 99    # what lies between the rows is not read into the sums
    bias = torch.randn(n, device="cuda", generator=g) if n != 130 else None
    y = int8_linear(x, w, bias)
    assert torch.equal(y, int8_matmul(int8_quantize(x), w, bias, out_dtype=dtype))
    _check_product(int8_linear(x, w, bias, out_dtype=F32), int8_quantize(x), w, bias)
    assert device_status() == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,k,n", [(1, 5, 3), (64, 48, 80), (257, 130, 65), (1000, 333, 514)])
def test_layer_forward_and_gradients(m, k, n, dtype):
    g = _gen(m)
    x = torch.randn(m, k, device="cuda", generator=g).to(dtype)
    w = torch.randn(n, k, device="cuda", generator=g) / k ** 0.5
    bias = torch.randn(n, device="cuda", generator=g)
    dy = (torch.randn(m, n, device="cuda", generator=g) * 1e-3).to(dtype)
    layer = Int8Linear(w, bias)
    y = layer.forward(x, training=True)
    dx, dw, db = layer.backward(dy)
    assert y.dtype == dx.dtype == dtype and dw.dtype == F32

    def rows(v):
        q, s = _want_codes(v)
        return Int8Matrix.pack(torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda())

    _check_product(y, rows(x), rows(w), bias)
    _check_product(dx, rows(dy), rows(w.T), None)
    _check_product(dw, rows(dy.T), rows(x.T), None)
    assert ((db.double() - dy.double().sum(0)).abs() <= (17 + m / 64) * U32 * dy.double().abs().sum(0)).all()
    # a row of the flat gradient of a step takes dw in place
    flat = torch.zeros(2, 10 + n * k, device="cuda")
    view = flat[1, 10:].view(n, k)
    layer.forward(x, training=True)
    layer.backward(dy, dw=view)
    assert torch.equal(view, dw) and (flat[0] == 0).all() and (flat[1, :10] == 0).all()
    assert torch.equal(layer.forward(x), y)                 # the serving form of the same layer


def test_gradients_against_differences():
    """The loss sum(dy * (x W^T + b)) is linear in each argument: its differences along a direction must equal the products with
    the gradients up to the error of the codes, half a step of the scale for every entry."""
    g = _gen(77)
    m, k, n = 96, 160, 64
    x = torch.randn(m, k, device="cuda", generator=g)
    w = torch.randn(n, k, device="cuda", generator=g) / k ** 0.5
    b = torch.randn(n, device="cuda", generator=g)
    dy = torch.randn(m, n, device="cuda", generator=g)

    def loss(x_, w_, b_):
        return float((dy.double() * (x_.double() @ w_.double().T + b_.double())).sum())

    layer = Int8Linear(w, b)
    layer.forward(x, training=True)
    dx, dw, db = layer.backward(dy)
    for which, grad in ((0, dx), (1, dw), (2, db)):
        args = [x, w, b]
        t = torch.randn(args[which].shape, device="cuda", generator=g)
        up, down = list(args), list(args)
        up[which], down[which] = args[which].double() + 1e-3 * t, args[which].double() - 1e-3 * t
        diff = (loss(*up) - loss(*down)) / 2e-3
        got = float((grad.double() * t.double()).sum())
        # each gradient entry is a sum of L products of codes; an operand's codes are off by at most half a step, s / 2, so
        # entry (i, j) is off by at most sum_l (|u_il| t_j / 2 + |v_jl| s_i / 2 + s_i t_j / 4)
        if which == 0:
            u, v = dy, w.T
        elif which == 1:
            u, v = dy.T, x.T
        else:
            assert abs(diff - got) <= 1e-6 * float((dy.double().abs() @ t.double().abs()).sum())
            continue
        su, sv = u.abs().amax(1).double() / 127, v.abs().amax(1).double() / 127
        off = (u.double().abs().sum(1)[:, None] * sv[None] + v.double().abs().sum(1)[None] * su[:, None]) / 2 + u.shape[1] * su[:, None] * sv[None] / 4
        assert abs(diff - got) <= float((off * t.double().abs()).sum()) * 1.001
        # and those errors are random: the sum stays near their root of squares (eight times it is past any chance)
        assert abs(diff - got) <= 8 * float((off * t.double()).square().sum().sqrt())


def test_other_streams_and_many_calls_in_a_row():
    g = _gen(4)
    w = int8_quantize(torch.randn(512, 768, device="cuda", generator=g))
    xs = [torch.randn(m, 768, device="cuda", generator=g).to(BF16) for m in (1, 40, 300)]
    want = [int8_linear(x, w) for x in xs]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = [[int8_linear(x, w) for x in xs] for _ in range(20)]
    s.synchronize()
    assert all(torch.equal(y, z) for r in got for y, z in zip(r, want))


def test_a_given_stream_owns_what_the_call_allocates():
    """Calls on a stream that is behind, while the current stream allocates and overwrites: the calls' workspaces and results must
    not be handed to it."""
    g = _gen(14)
    x = torch.randn(300, 512, device="cuda", generator=g)
    w0 = torch.randn(256, 512, device="cuda", generator=g)
    dy = torch.randn(300, 256, device="cuda", generator=g)
    plain = Int8Linear(w0)
    want = plain.forward(x, training=True), *plain.backward(dy)[:2], plain.forward(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        busy = torch.randn(4096, 4096, device="cuda")
        for _ in range(20):
            busy = torch.sin(busy)
    layer = Int8Linear(w0, stream=s)
    y = layer.forward(x, training=True, stream=s)
    dx, dw, _ = layer.backward(dy, stream=s)
    z = layer.forward(x, stream=s)
    for _ in range(50):
        for n in (300 * 256, 300 * 512, 256 * 512, 200_000, 500_000):
            torch.full((n,), -1, dtype=torch.uint8, device="cuda") if n % 2 else torch.full((n,), float("nan"), device="cuda")
    s.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((y, dx, dw, z), want))


def test_tensors_of_another_device_make_it_current(monkeypatch):
    """The library works on the current device: a call whose tensors lie elsewhere changes to theirs and back.  What the calls take
    for the current device is made up here, so that one device shows it."""
    x = torch.randn(20, 64, device="cuda", generator=_gen(21))
    w = int8_quantize(x)
    update = OrthUpdate(20, 64)
    calls = (lambda: int8_quantize(x).codes, lambda: int8_matmul(w, w), lambda: int8_linear(x, w), lambda: update.update(x))
    want = [f() for f in calls]
    here, entered = torch.cuda.current_device(), []

    class Device(torch.cuda.device):
        def __enter__(self):
            entered.append(self.idx)
            return super().__enter__()

    monkeypatch.setattr(torch.cuda, "device", Device)
    for f, y in zip(calls, want):
        entered.clear()
        monkeypatch.setattr(matrix_ops, "_current", lambda: entered[-1] if entered else here + 1)
        assert torch.equal(f(), y)
        assert entered == [here]


def test_linear_in_a_captured_graph():
    g = _gen(6)
    w = int8_quantize(torch.randn(256, 512, device="cuda", generator=g))
    x = torch.randn(3, 512, device="cuda", generator=g)
    y = torch.empty(3, 256, device="cuda")
    int8_linear(x, w, out=y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        int8_linear(x, w, out=y)
    x.copy_(torch.randn(3, 512, device="cuda", generator=g))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, int8_matmul(int8_quantize(x), w, out_dtype=F32))


def test_refusals():
    lib = binding.load_library()
    x = torch.randn(8, 64, device="cuda")
    w = int8_quantize(torch.randn(16, 64, device="cuda"))
    with pytest.raises(TypeError):
        int8_quantize(x.double())
    with pytest.raises(ValueError):
        int8_quantize(x.cpu())
    with pytest.raises(ValueError):
        int8_quantize(x[0])
    with pytest.raises(ValueError):
        int8_quantize(x, rows=False)
    with pytest.raises(ValueError):
        int8_matmul(int8_quantize(x[:, :32]), w)
    with pytest.raises(ValueError):
        int8_linear(x, w, bias=torch.zeros(15, device="cuda"))
    with pytest.raises(ValueError):
        int8_linear(x, w, out=torch.zeros(8, 15, device="cuda"))
    with pytest.raises(ValueError):
        Int8Matrix(w.codes, w.scale[:-1])
    with pytest.raises(RuntimeError):
        Int8Linear(torch.randn(4, 8, device="cuda")).backward(torch.randn(2, 4, device="cuda"))
    with pytest.raises(DsqError) as e:                       # rows of codes that do not start on 16 bytes
        int8_linear(x[:, :40].contiguous(), Int8Matrix(w.codes[:, :40].contiguous(), w.scale))
    assert e.value.code == binding.DS_ERR_ALIGN
    p, big = x.data_ptr(), binding.DS_I8_MAX_K + 16
    args = (w.codes.data_ptr(), w.ld, w.scale.data_ptr(), None, 16, p, 0, 16, p, 1 << 20, None, None)
    assert lib.ds_i8_linear(p, 7, 8, 64, 64, *args) == binding.DS_ERR_INVALID_ARG            # no such type
    assert lib.ds_i8_linear(p, 0, 8, 64, 32, *args) == binding.DS_ERR_INVALID_ARG            # rows overlap
    assert lib.ds_i8_linear(p + 2, 0, 8, 64, 64, *args) == binding.DS_ERR_ALIGN
    assert lib.ds_i8_linear(p, 0, 8, big, big, *args) == binding.DS_ERR_UNSUPPORTED
    small = args[:9] + (16, None, None)
    assert lib.ds_i8_linear(p, 0, 64, 64, 64, *small) == binding.DS_ERR_BUFFER_TOO_SMALL
    q = torch.zeros(8, 64, dtype=torch.int8, device="cuda")
    assert lib.ds_i8_quantize(p, 0, 8, 64, 64, q.data_ptr(), 64, None, None, 0, None, None, None, 0, None) == binding.DS_ERR_INVALID_ARG
    assert lib.ds_i8_quantize(p, 0, 8, 64, 64, q.data_ptr(), 72, p, None, 0, None, None, None, 0, None) == binding.DS_ERR_ALIGN
    assert lib.ds_i8_quantize(p, 0, 8, 64, 64, None, 0, None, q.data_ptr(), 16, p, None, None, 0, None) == binding.DS_ERR_INVALID_ARG
    torch.cuda.synchronize()
