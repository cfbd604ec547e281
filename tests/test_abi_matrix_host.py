"""Host-side checks of the matrix operators' C ABI that need no GPU: struct sizes, workspace sizes, and refusals, which come
before anything is launched."""
import ctypes as C
import os
import subprocess
import sys

import pytest

from paper_1905_05957_b200 import binding as b
from paper_1905_05957_b200 import build as libbuild

P = 0x10000          # an address that is never read: every call below returns first


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return b.load_library()


def test_struct_and_call_extension(lib):
    assert C.sizeof(b.ds_orth_config) == 56
    call, address = b.fast_call()
    # the extension and ctypes call the same function with the same arguments
    assert call(address["ds_i8_matmul"], P, 64, P, P, 64, P, None, 0, 5, 64, P, 1, 5, P, None) == b.DS_OK
    assert call(address["ds_i8_matmul"], P, 64, P, P, 64, P, None, 4, 5, 64, P, 9, 5, P, None) == b.DS_ERR_INVALID_ARG
    with pytest.raises(TypeError):
        call()
    with pytest.raises(TypeError):
        call(address["ds_i8_matmul"], *range(19))
    with pytest.raises(TypeError):
        call("address")


def test_workspace_sizes(lib):
    assert lib.ds_i8_linear_workspace(1, 2048, 2048) == 0                       # a single token is one launch
    assert lib.ds_i8_linear_workspace(100, 1000, 64) == 100 * 1008 + 4 * 128    # codes, then scales
    assert lib.ds_i8_linear_workspace(7, 100_000, 64) == 7 * 100_000 + 4 * 64
    w = lib.ds_i8_quantize_workspace(1000, 300, 0)
    assert w >= 4 * 1300 and lib.ds_i8_quantize_workspace(1000, 300, 1) == w + 4 * 16 * 300


def _quantize(lib, **kw):
    a = dict(x=P, dtype=0, rows=8, cols=64, ld=64, q=P, ldq=64, scale=P, qt=None, ldqt=0, scale_t=None, col_sum=None, ws=None, ws_bytes=0)
    a.update(kw)
    return lib.ds_i8_quantize(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), b.DS_ERR_INVALID_ARG), (dict(ld=63), b.DS_ERR_INVALID_ARG), (dict(x=None), b.DS_ERR_INVALID_ARG),
    (dict(scale=None), b.DS_ERR_INVALID_ARG), (dict(q=None), b.DS_ERR_INVALID_ARG), (dict(q=None, scale=None), b.DS_ERR_INVALID_ARG),
    (dict(ldq=48), b.DS_ERR_INVALID_ARG), (dict(ldq=72), b.DS_ERR_ALIGN), (dict(q=P + 8), b.DS_ERR_ALIGN), (dict(x=P + 2), b.DS_ERR_ALIGN),
    (dict(qt=P, scale_t=P, ldqt=16), b.DS_ERR_INVALID_ARG), (dict(qt=P, scale_t=P, ldqt=16, ws=P, ws_bytes=16), b.DS_ERR_BUFFER_TOO_SMALL),
    (dict(qt=P, scale_t=P, ldqt=16, ws=P + 4, ws_bytes=1 << 20), b.DS_ERR_ALIGN), (dict(rows=(1 << 30) + 1), b.DS_ERR_INVALID_ARG),
])
def test_quantiser_refusals(lib, kw, code):
    assert _quantize(lib, **kw) == code


def _matmul(lib, **kw):
    a = dict(a=P, lda=64, sa=P, b=P, ldb=64, sb=P, bias=None, m=4, n=5, k=64, out=P, dtype=0, ldo=5, status=P)
    a.update(kw)
    return lib.ds_i8_matmul(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=-1), b.DS_ERR_INVALID_ARG), (dict(ldo=4), b.DS_ERR_INVALID_ARG), (dict(k=b.DS_I8_MAX_K + 1), b.DS_ERR_UNSUPPORTED),
    (dict(a=None), b.DS_ERR_INVALID_ARG), (dict(sb=None), b.DS_ERR_INVALID_ARG), (dict(out=None), b.DS_ERR_INVALID_ARG),
    (dict(lda=32), b.DS_ERR_INVALID_ARG), (dict(ldb=72), b.DS_ERR_ALIGN), (dict(b=P + 1), b.DS_ERR_ALIGN), (dict(out=P + 1), b.DS_ERR_ALIGN),
    (dict(bias=P + 2), b.DS_ERR_ALIGN), (dict(m=0), b.DS_OK), (dict(n=0, ldo=0), b.DS_OK),
])
def test_product_refusals(lib, kw, code):
    assert _matmul(lib, **kw) == code


def test_linear_refusals(lib):
    def linear(**kw):
        a = dict(x=P, dtype=0, rows=64, k=64, ldx=64, w=P, ldw=64, sw=P, bias=None, n=5, out=P, odt=0, ldo=5, ws=P, size=1 << 20, status=P)
        a.update(kw)
        return lib.ds_i8_linear(*a.values(), None)

    assert linear(ws=None) == b.DS_ERR_INVALID_ARG
    assert linear(ws=P + 4) == b.DS_ERR_ALIGN
    assert linear(size=64) == b.DS_ERR_BUFFER_TOO_SMALL
    assert linear(k=b.DS_I8_MAX_K + 1) == b.DS_ERR_UNSUPPORTED
    for kw in (dict(x=None), dict(w=None), dict(sw=None), dict(out=None), dict(ldx=32), dict(ldo=4), dict(dtype=5), dict(odt=5)):
        assert linear(rows=2, ws=None, **kw) == b.DS_ERR_INVALID_ARG          # the one-launch form makes its own checks
    for kw in (dict(w=P + 8), dict(ldw=72), dict(x=P + 2), dict(out=P + 2), dict(sw=P + 1)):
        assert linear(rows=2, ws=None, **kw) == b.DS_ERR_ALIGN
    assert linear(rows=0, ws=None) == b.DS_OK


def test_orth_plans(lib):
    cfg = b.ds_orth_config(300, 200, 2, 5, 3.4445, -4.775, 2.0315, 0.95, 1e-7, 1.0, 1, 0, 0)
    size, h = C.c_size_t(0), C.c_void_p()
    assert lib.ds_orth_create(C.byref(cfg), None, C.byref(size), None, None) == b.DS_NEED_BUFFERS
    # X twice in two halves, A and B, in 16 bits
    assert size.value >= 2 * (4 * 2 * 200 * 300 + 2 * 2 * 200 * 200)
    assert lib.ds_orth_create(C.byref(cfg), P, C.byref(size), P, C.byref(h)) == b.DS_OK
    assert lib.ds_orth_update(h, None, 0, None, P, 0, None, 0.0, 0.0, None) == b.DS_ERR_INVALID_ARG
    assert lib.ds_orth_update(h, P, 0, P, None, 0, None, 0.0, 0.0, None) == b.DS_ERR_INVALID_ARG       # nothing to write
    assert lib.ds_orth_update(h, P, 0, None, P, 2, None, 0.0, 0.0, None) == b.DS_ERR_INVALID_ARG       # no such output type
    assert lib.ds_orth_update(h, P, 0, P + 2, P, 0, None, 0.0, 0.0, None) == b.DS_ERR_ALIGN
    assert lib.ds_orth_update(h, P, 0, None, None, 0, P, float("nan"), 0.0, None) == b.DS_ERR_INVALID_ARG
    assert lib.ds_orth_destroy(h) == b.DS_OK
    assert lib.ds_orth_create(C.byref(cfg), P + 16, C.byref(size), P, C.byref(h)) == b.DS_ERR_ALIGN
    assert lib.ds_orth_create(C.byref(cfg), P, C.byref(C.c_size_t(64)), P, C.byref(h)) == b.DS_ERR_BUFFER_TOO_SMALL
    assert lib.ds_orth_create(C.byref(cfg), P, C.byref(size), None, C.byref(h)) == b.DS_ERR_INVALID_ARG
    for field, value in (("rows", 0), ("cols", (1 << 20) + 1), ("batch", 0), ("batch", 70_000), ("steps", 0), ("a", float("inf")),
                         ("momentum", float("nan")), ("eps", -1.0), ("flags", 2), ("reserved", 1), ("stride", 59_999)):
        bad = b.ds_orth_config.from_buffer_copy(cfg)
        setattr(bad, field, value)
        assert lib.ds_orth_create(C.byref(bad), None, C.byref(size), None, None) == b.DS_ERR_INVALID_ARG, field


def test_a_host_without_a_device_gets_a_status():
    """In a process of its own that sees no device: calls of every form end with the CUDA error as their status."""
    code = """
import ctypes as C
from paper_1905_05957_b200 import binding as b
lib, P = b.load_library(), 0x10000
for m, n, k in ((4, 64, 64), (40, 64, 64), (100, 64, 64), (100, 64, 0), (5000, 5000, 256)):
    print(lib.ds_i8_matmul(P, 256, P, P, 256, P, None, m, n, k, P, 0, n, P, None))
for rows in (2, 100):
    print(lib.ds_i8_linear(P, 0, rows, 64, 64, P, 64, P, None, 64, P, 0, 64, P, 1 << 20, P, None))
print(lib.ds_i8_quantize(P, 0, 8, 64, 64, P, 64, P, P, 16, P, None, P, 1 << 20, None))
for m, n in ((48, 100), (300, 500), (4096, 4096)):
    cfg = b.ds_orth_config(m, n, 1, 5, 3.4445, -4.775, 2.0315, 0.95, 1e-7, 1.0, 1, 0, 0)
    size, h = C.c_size_t(0), C.c_void_p()
    assert lib.ds_orth_create(C.byref(cfg), None, C.byref(size), None, None) == b.DS_NEED_BUFFERS
    assert lib.ds_orth_create(C.byref(cfg), P, C.byref(size), P, C.byref(h)) == b.DS_OK
    print(lib.ds_orth_update(h, P, 0, None, P, 0, None, 0.0, 0.0, None))
"""
    env = dict(os.environ, CUDA_VISIBLE_DEVICES="", PYTHONPATH=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    got = subprocess.run([sys.executable, "-c", code], env=env, capture_output=True, text=True)
    assert got.returncode == 0, got.stderr[-500:]
    assert [int(v) for v in got.stdout.split()] == [b.DS_ERR_CUDA] * 11


def test_a_host_without_a_c_compiler(lib, tmp_path, monkeypatch):
    """The library is built without the extension, and the calls go through ctypes to the same functions."""
    missing = str(tmp_path / "dsq_call.so")
    monkeypatch.setattr(libbuild, "CALL_LIB", missing)
    monkeypatch.setenv("CC", str(tmp_path / "no-such-compiler"))
    assert libbuild.build_call() is None and libbuild.build() == libbuild.LIB
    monkeypatch.setattr(libbuild.sysconfig, "get_paths", lambda: {"include": str(tmp_path)})      # no Python.h
    monkeypatch.setenv("CC", "gcc")
    assert libbuild.build_call() is None and libbuild.build() == libbuild.LIB and not os.path.exists(missing)
    monkeypatch.setattr(b, "CALL_LIB", missing)
    monkeypatch.setattr(b, "_call", None)
    call, address = b.fast_call()
    assert call(address["ds_i8_matmul"], P, 64, P, P, 64, P, None, 0, 5, 64, P, 1, 5, P, None) == b.DS_OK
    assert call(address["ds_i8_matmul"], P, 64, P, P, 64, P, None, 4, 5, 64, P, 9, 5, P, None) == b.DS_ERR_INVALID_ARG
    assert call(address["ds_i8_linear"], P, 0, 0, 64, 64, P, 64, P, None, 5, P, 0, 5, 0, 0, P, 0) == b.DS_OK
    assert call(address["ds_i8_quantize"], P, 3, 8, 64, 64, P, 64, P, 0, 0, 0, 0, 0, 0, 0) == b.DS_ERR_INVALID_ARG


def test_the_extension_names_its_interpreter():
    assert os.path.basename(libbuild.CALL_LIB) == "dsq_call" + libbuild.sysconfig.get_config_var("EXT_SUFFIX")


@pytest.mark.parametrize("rows", [2, 64])
def test_linear_refuses_before_it_launches(lib, rows):
    """Both forms: a refusal of the product's arguments comes before the quantiser is launched (without a device: before its launch fails)."""
    def linear(**kw):
        a = dict(x=P, dtype=0, rows=rows, k=64, ldx=64, w=P, ldw=64, sw=P, bias=None, n=5, out=P, odt=0, ldo=5, ws=P, size=1 << 20, status=P)
        a.update(kw)
        return lib.ds_i8_linear(*a.values(), None)

    for kw in (dict(x=None), dict(w=None), dict(sw=None), dict(out=None), dict(ldx=32), dict(ldw=48), dict(ldo=4), dict(dtype=5), dict(odt=5),
               dict(n=(1 << 30) + 1, ldo=1 << 31)):
        assert linear(**kw) == b.DS_ERR_INVALID_ARG, kw
    for kw in (dict(w=P + 8), dict(ldw=72), dict(x=P + 2), dict(out=P + 2), dict(sw=P + 1), dict(bias=P + 2), dict(status=P + 1)):
        assert linear(**kw) == b.DS_ERR_ALIGN, kw
