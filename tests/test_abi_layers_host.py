"""Host-side checks of the C ABI of the 16-bit layer, the norms and dropout that need no GPU: structures, workspace sizes, and refusals, which come before
anything is launched."""
import ctypes as C
import re

import pytest

from paper_1905_05957_b200 import binding as b
from paper_1905_05957_b200 import build as libbuild

P, FAR = 0x10000, 0x100000000          # addresses that are never read: every call below returns first
INVALID, ALIGN, SMALL, UNSUPPORTED = b.DS_ERR_INVALID_ARG, b.DS_ERR_ALIGN, b.DS_ERR_BUFFER_TOO_SMALL, b.DS_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return b.load_library()


@pytest.mark.parametrize("name,kind", sorted(b._STRUCT_CALLS.items()))
def test_structures_agree_with_the_header(name, kind):
    """The members by name and order, each of 64 bits."""
    text = open(libbuild.CSRC + "/../../include/dsq.h").read()
    body = re.search(r"typedef struct \{([^{}]*)\} %s;" % kind.__name__, text).group(1)
    names = [re.sub(r"[*\s]", "", m) for line in body.split(";") for m in re.sub(r"^\s*(const\s+)?(void|float|double|uint64_t|uint32_t)\b", "", line.strip()).split(",") if m.strip()]
    assert names == [f[0] for f in kind._fields_] and C.sizeof(kind) == 8 * len(names)


def test_struct_calls(lib):
    call, size, at = b.fast_struct_call()
    zero = [0] * len(b.ds_norm_args._fields_)
    assert call(at["ds_norm_forward"], None, *zero) == INVALID                          # no columns
    zero[3] = 8
    zero[15], zero[16] = 1.0, 1e-5
    assert call(at["ds_norm_forward"], None, *zero) == b.DS_OK                          # no rows
    zero[16] = -1.0
    assert call(at["ds_norm_forward"], None, *zero) == INVALID                          # floats arrive as doubles
    product = list(PRODUCT.values())
    product[6] = 65
    assert size(at["ds_f16_matmul_workspace"], *product) == 40 * 64 * 2 and size(at["ds_f16_matmul_workspace"], 1) == 0
    assert size(at["ds_norm_backward_workspace"], *zero) == 0
    if getattr(call, "__name__", "") == "call_struct":
        for bad in ((), (1,), (at["ds_f16_matmul_workspace"], "x")):
            with pytest.raises(TypeError):
                size(*bad)
        for bad in ((), (1, 2), (1, 2, *range(65)), (at["ds_norm_forward"], None, "x")):
            with pytest.raises(TypeError):
                call(*bad)


def test_a_second_thread_sees_all_functions_or_none(lib, monkeypatch):
    from paper_1905_05957_b200 import layer_ops
    seen = []
    for name in ("fast_struct_call", "fast_call"):
        real = getattr(b, name)
        monkeypatch.setattr(layer_ops, name, lambda real=real: (seen.append(layer_ops._struct), real())[1])
    monkeypatch.setattr(layer_ops, "_struct", None)
    layer_ops._load()
    assert seen == [None, None] and layer_ops._struct is not None and layer_ops._dropout_at is not None


def _args(kind, values, **kw):
    values = {**values, **kw}
    return kind(**{k: v for k, v in values.items() if v is not None})


PRODUCT = dict(dtype=1, layout=0, m=40, n=24, k=64, a=P, lda=64, b=2 * P, ldb=64, bias=None, activation=0, residual=None, ldr=0, z=None, ldz=0, out=FAR, out_dtype=1, ldo=24,
               workspace=None, workspace_bytes=0, dev_status=None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=0), INVALID), (dict(dtype=3), INVALID), (dict(layout=3), INVALID), (dict(activation=5), INVALID), (dict(out_dtype=2), INVALID), (dict(out_dtype=7), INVALID),
    (dict(m=(1 << 30) + 1), INVALID), (dict(k=1 << 40), INVALID), (dict(a=None), INVALID), (dict(b=None), INVALID), (dict(out=None), INVALID), (dict(lda=63), INVALID),
    (dict(ldb=32), INVALID), (dict(ldo=23), INVALID), (dict(residual=P * 9, ldr=20), INVALID), (dict(z=P * 9, ldz=20), INVALID), (dict(out=FAR + 1), ALIGN), (dict(a=P + 1), ALIGN),
    (dict(bias=P + 2), ALIGN), (dict(dev_status=P + 2), ALIGN), (dict(out=P), INVALID), (dict(out=2 * P + 128), INVALID), (dict(z=FAR, ldz=24), INVALID),
    (dict(residual=FAR, ldr=32), INVALID), (dict(residual=FAR + 2, ldr=24), INVALID), (dict(residual=FAR, ldr=24, out_dtype=0), INVALID), (dict(bias=FAR), INVALID),
    (dict(lda=65), INVALID), (dict(lda=65, workspace=FAR * 2, workspace_bytes=16), SMALL), (dict(a=P + 2, workspace=FAR * 2 + 8, workspace_bytes=1 << 20), ALIGN),
    (dict(lda=65, workspace=FAR, workspace_bytes=1 << 20), INVALID), (dict(m=0), b.DS_OK), (dict(n=0), b.DS_OK),
    (dict(layout=1, lda=63), INVALID), (dict(layout=1, ldb=23), INVALID), (dict(layout=2, lda=39), INVALID), (dict(layout=2, ldb=23), INVALID),
], ids=str)
def test_product_refusals(lib, kw, code):
    assert lib.ds_f16_matmul(C.byref(_args(b.ds_f16_product, PRODUCT, **kw)), None) == code


def test_product_workspace(lib):
    def size(**kw):
        return lib.ds_f16_matmul_workspace(C.byref(_args(b.ds_f16_product, PRODUCT, **kw)))
    assert size() == 0 and size(k=63, lda=64, ldb=64) == 0
    assert size(lda=65) == 40 * 64 * 2 and size(b=P + 2) == 24 * 64 * 2 and size(a=P + 2, ldb=65) == 64 * 64 * 2
    assert size(layout=2, lda=41) == 64 * 64 * 2 and size(layout=1, ldb=25) == 64 * 64 * 2      # rows of whole lines
    assert size(m=1, lda=7) == 0                                                      # a single row has no pitch
    assert size(m=9, lda=65) == size(m=16, a=P + 2) == 0 and size(m=18, lda=65) == 18 * 64 * 2      # few tokens are read where they lie
    assert size(m=9, ldb=65) == 24 * 64 * 2
    assert lib.ds_f16_matmul(None, None) == INVALID and lib.ds_f16_matmul_workspace(None) == 0


def test_product_workspace_of_few_tokens(lib):
    """Short rows are read where they lie, long ones are copied; two groups of tokens only where CTAs take W in a round."""
    def size(**kw):
        return lib.ds_f16_matmul_workspace(C.byref(_args(b.ds_f16_product, PRODUCT, **{**dict(m=8, k=2040, lda=2041, ldb=2040), **kw})))
    assert size() == size(m=16) == size(m=1, a=P + 2) == 0
    assert size(k=2048, lda=2049, ldb=2048) == 8 * 2048 * 2 and size(m=1, k=2048, a=P + 2, ldb=2048) == 2048 * 2 and size(m=8, k=2048, lda=2048, ldb=2048) == 0
    assert size(m=16, n=1 << 20) == 16 * 2048 * 2 and size(m=8, n=1 << 20) == 0


SLOPE = dict(dtype=1, rows=100, cols=64, dy=P, lddy=64, z=FAR, ldz=64, activation=2, dz=2 * FAR, lddz=64, sum=3 * FAR, sum_dtype=0, workspace=4 * FAR, workspace_bytes=1 << 20)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=0), INVALID), (dict(activation=9), INVALID), (dict(sum_dtype=2), INVALID), (dict(dy=None), INVALID), (dict(z=None), INVALID), (dict(activation=0), INVALID),
    (dict(dz=None, sum=None), INVALID), (dict(lddy=63), INVALID), (dict(ldz=63), INVALID), (dict(lddz=63), INVALID), (dict(dy=P + 1), ALIGN), (dict(sum=FAR * 3 + 2), ALIGN),
    (dict(dz=P + 128), INVALID), (dict(dz=FAR, lddz=72), INVALID), (dict(sum=P), INVALID), (dict(workspace=None), INVALID), (dict(workspace=P + 8), ALIGN),
    (dict(workspace_bytes=511), SMALL), (dict(workspace=FAR), INVALID), (dict(rows=65536 * 64), UNSUPPORTED), (dict(rows=(1 << 30) + 1), INVALID), (dict(cols=0), b.DS_OK),
], ids=str)
def test_slope_refusals(lib, kw, code):
    assert lib.ds_f16_slope(C.byref(_args(b.ds_f16_slope_args, SLOPE, **kw)), None) == code


def test_pack_refusals(lib):
    def pack(x=P, dtype=0, rows=10, cols=20, ld=20, out=FAR, odt=1, ldo=24):
        return lib.ds_f16_pack(x, dtype, rows, cols, ld, out, odt, ldo, None)
    assert pack(rows=0) == pack(cols=0) == b.DS_OK
    for kw in (dict(dtype=3), dict(odt=0), dict(x=None), dict(out=None), dict(ld=19), dict(ldo=16), dict(out=P), dict(rows=1 << 31)):
        assert pack(**kw) == INVALID
    for kw in (dict(x=P + 2), dict(out=FAR + 8), dict(ldo=28)):
        assert pack(**kw) == ALIGN


NORM = dict(dtype=1, stream_dtype=0, rows=12, cols=64, norm=1, y=FAR, ldy=64, x=2 * FAR, ldx=64, post_w=P, post_b=P, gate=P, groups=3, pre_w=P, pre_b=P, residual_scale=1.0,
            eps=1e-5, threshold=0, seed=1, layer=0, step=0, stats=3 * FAR)
FORWARD = dict(NORM, h=4 * FAR, ldh=64, n=5 * FAR, ldn=64)
BACKWARD = dict(NORM, dh=4 * FAR, lddh=64, dn=5 * FAR, lddn=64, dx=6 * FAR, lddx=64, dy=7 * FAR, lddy=64, d_post_w=8 * FAR, d_post_b=9 * FAR, d_gate=10 * FAR, d_pre_w=11 * FAR,
                d_pre_b=12 * FAR, workspace=13 * FAR, workspace_bytes=1 << 30)
BOTH = [(dict(dtype=3), INVALID), (dict(stream_dtype=2), INVALID), (dict(norm=2), INVALID), (dict(cols=0), INVALID), (dict(cols=32769), UNSUPPORTED), (dict(rows=(1 << 30) + 1), INVALID),
        (dict(groups=5), INVALID), (dict(groups=0), INVALID), (dict(gate=None), INVALID), (dict(post_w=None), INVALID), (dict(pre_w=None), INVALID), (dict(eps=-1.0), INVALID),
        (dict(eps=float("nan")), INVALID), (dict(threshold=65536), INVALID), (dict(layer=1 << 32), INVALID), (dict(step=1 << 32), INVALID), (dict(y=None), INVALID),
        (dict(ldy=63), INVALID), (dict(ldx=63), INVALID), (dict(y=FAR + 1), ALIGN), (dict(x=FAR * 2 + 2), ALIGN), (dict(gate=P + 2), ALIGN), (dict(stats=3 * FAR + 8), ALIGN)]


@pytest.mark.parametrize("kw,code", BOTH + [
    (dict(h=None, n=None), INVALID), (dict(n=None), INVALID), (dict(pre_w=None, pre_b=None), INVALID), (dict(ldh=60), INVALID), (dict(ldn=60), INVALID), (dict(h=5 * FAR), INVALID),
    (dict(h=2 * FAR + 256), INVALID), (dict(h=FAR), INVALID), (dict(n=2 * FAR), INVALID), (dict(h=2 * FAR, ldh=72), INVALID), (dict(stats=FAR), INVALID), (dict(rows=0), b.DS_OK),
], ids=str)
def test_forward_refusals(lib, kw, code):
    assert lib.ds_norm_forward(C.byref(_args(b.ds_norm_args, FORWARD, **kw)), None) == code


@pytest.mark.parametrize("kw,code", BOTH + [
    (dict(dh=None, dn=None), INVALID), (dict(stats=None), INVALID), (dict(lddh=60), INVALID), (dict(lddn=60), INVALID), (dict(lddx=60), INVALID), (dict(lddy=60), INVALID),
    (dict(x=None), INVALID), (dict(dx=7 * FAR), INVALID), (dict(dx=4 * FAR + 256), INVALID), (dict(dy=4 * FAR), INVALID), (dict(dy=3 * FAR), INVALID), (dict(d_gate=4 * FAR), INVALID),
    (dict(d_pre_w=12 * FAR), INVALID), (dict(d_post_w=P), INVALID), (dict(workspace=None), INVALID), (dict(workspace=13 * FAR + 8), ALIGN), (dict(workspace_bytes=64), SMALL),
    (dict(workspace=7 * FAR), INVALID), (dict(pre_w=None, pre_b=None), INVALID),
], ids=str)
def test_backward_refusals(lib, kw, code):
    assert lib.ds_norm_backward(C.byref(_args(b.ds_norm_args, BACKWARD, **kw)), None) == code


def test_the_pitch_of_a_single_row_is_not_read(lib):
    """In place over the residual, dy or z whatever it is: what is refused is the misaligned address that is looked at after that."""
    one = dict(m=1, residual=FAR, ldr=7, ldo=24, a=P + 1)
    assert lib.ds_f16_matmul(C.byref(_args(b.ds_f16_product, PRODUCT, **one)), None) == ALIGN
    assert lib.ds_f16_matmul(C.byref(_args(b.ds_f16_product, PRODUCT, **dict(one, residual=FAR + 16))), None) == INVALID
    for kw in (dict(dz=P, lddz=7), dict(dz=FAR, lddz=0)):
        assert lib.ds_f16_slope(C.byref(_args(b.ds_f16_slope_args, SLOPE, rows=1, workspace=4 * FAR + 8, **kw)), None) == ALIGN
    assert lib.ds_f16_slope(C.byref(_args(b.ds_f16_slope_args, SLOPE, rows=1, workspace=4 * FAR + 8, dz=P + 64)), None) == INVALID


VECTORS = dict(post_w=20 * FAR, post_b=21 * FAR, gate=22 * FAR, pre_w=23 * FAR, pre_b=24 * FAR)


@pytest.mark.parametrize("name", VECTORS)
def test_outputs_over_parameters_are_refused(lib, name):
    """CTAs read them at times of their own: an output there would be read by some of them."""
    at = VECTORS[name] + 4 * 16
    for out in ("h", "n", "stats"):
        assert lib.ds_norm_forward(C.byref(_args(b.ds_norm_args, FORWARD, **VECTORS, **{out: at})), None) == INVALID
    for out in ("dx", "dy"):
        assert lib.ds_norm_backward(C.byref(_args(b.ds_norm_args, BACKWARD, **VECTORS, **{out: at})), None) == INVALID


def test_backward_workspace(lib):
    """Sums of each CTA, for each parameter whose gradient is wanted, and of each unit of a gate's rows; none that nothing asks for."""
    def size(**kw):
        return lib.ds_norm_backward_workspace(C.byref(_args(b.ds_norm_args, BACKWARD, **kw)))
    assert size(rows=0) == 0 and size(norm=7) == 0
    bare = dict(d_post_w=None, d_post_b=None, d_gate=None, d_pre_w=None, d_pre_b=None)
    assert size(**bare) == 0
    one = size(rows=30000, **dict(bare, d_pre_w=11 * FAR))
    assert one > 0 and one % (4 * 64) == 0 and size(rows=30000, **dict(bare, d_pre_w=11 * FAR, d_pre_b=12 * FAR)) == 2 * one
    assert size(rows=1200, groups=1200, **dict(bare, d_gate=10 * FAR)) == 0            # whole gates go straight to their place


def test_dropout_refusals(lib):
    def drop(x=P, dtype=0, rows=10, cols=16, ldx=16, out=FAR, ldo=16, threshold=100):
        return lib.ds_dropout(x, dtype, rows, cols, ldx, out, ldo, threshold, 1, 0, 0, None)
    assert drop(rows=0) == drop(cols=0) == b.DS_OK
    for kw in (dict(dtype=-1), dict(dtype=3), dict(threshold=65536), dict(x=None), dict(out=None), dict(ldx=15), dict(ldo=15), dict(out=P + 64), dict(out=P, ldo=24), dict(rows=1 << 31)):
        assert drop(**kw) == INVALID
    for kw in (dict(x=P + 2), dict(out=FAR + 1), dict(dtype=1, x=P + 1)):
        assert drop(**kw) == ALIGN
