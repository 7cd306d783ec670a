"""Host-side checks of the layer operators: every refusal comes before any
pointer or device is touched, so the pointers below are never dereferenced."""

import ctypes
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

from paper_2009_04509_amd import build as B  # noqa: E402

NULL = ctypes.c_void_p(0)
FAKE = ctypes.c_void_p(0x10000)
BF16, FP32 = 1, 0


@pytest.fixture(scope="module")
def b():
    from paper_2009_04509_amd import binding
    return binding


def mat(b, at=0x20000, ld=64):
    return ctypes.byref(b._Matrix(at, ld))


def kept(b, at=0x20000, ld=64, codes=None, exponents=None):
    return ctypes.byref(b._Kept(b._Matrix(at, ld), b._Packed(codes, exponents)))


def dense(b, layers=FAKE, dtype=BF16, act=0, m=4, k=64, n=64, x="", w="", bias=None, residual=None, y="", z=None):
    x, w, y = (mat(b) if v == "" else v for v in (x, w, y))
    return b.lib.pointid_dense(layers, dtype, act, m, k, n, x, w, bias, residual, y, z, NULL)


def test_create_refusals(b):
    out = ctypes.c_void_p(0x1234)
    assert b.lib.pointid_layers_create(0, None) == b.POINTID_EINVAL
    if not torch.cuda.is_available():
        assert b.lib.pointid_layers_create(0, ctypes.byref(out)) == b.POINTID_ENODEV
        assert out.value is None
    assert b.lib.pointid_layers_destroy(NULL) == b.POINTID_OK
    assert b.lib.pointid_layers_trim(NULL, 0, None) == b.POINTID_EINVAL


@pytest.mark.parametrize("case, word", [
    (dict(layers=NULL), "layers"),
    (dict(act=5), "act"), (dict(act=-1), "act"),
    (dict(m=-1), "m must"), (dict(m=1 << 31), "m must"),
    (dict(k=0), "k and n"), (dict(n=0), "k and n"), (dict(k=(1 << 20) + 1), "k and n"), (dict(n=(1 << 20) + 1), "k and n"),
    (dict(x=None), "x is NULL"), (dict(w=None), "w is NULL"), (dict(y=None), "y is NULL"),
    (dict(bias=ctypes.c_void_p(0x20002)), "bias"),
])
def test_dense_refusals(b, case, word):
    assert dense(b, **case) == b.POINTID_EINVAL
    assert word in b.pointid_last_error()


def test_dtype_is_unsupported(b):
    for dtype in (3, -1, 9):
        assert dense(b, dtype=dtype) == b.POINTID_EUNSUPPORTED
        assert b.lib.pointid_checkpoint_save(dtype, 1, 1, mat(b), ctypes.byref(b._Packed(1, 1)), NULL) == \
            b.POINTID_EUNSUPPORTED


def test_matrix_refusals(b):
    for name in ("x", "w", "y", "residual"):
        assert dense(b, **{name: mat(b, ld=63)}) == b.POINTID_EINVAL and name in b.pointid_last_error()
        assert dense(b, **{name: mat(b, at=0x20001)}) == b.POINTID_EINVAL and "aligned" in b.pointid_last_error()
        assert dense(b, dtype=FP32, **{name: mat(b, at=0x20002)}) == b.POINTID_EINVAL
        assert dense(b, m=1 << 30, k=1 << 20, n=1 << 20, **{name: mat(b, ld=1 << 62)}) == b.POINTID_EINVAL


def test_kept_refusals(b):
    assert dense(b, z=kept(b, codes=1, exponents=1)) == b.POINTID_EINVAL and "both" in b.pointid_last_error()
    assert dense(b, z=kept(b, at=None)) == b.POINTID_EINVAL
    assert dense(b, z=kept(b, at=None, codes=1)) == b.POINTID_EINVAL and "keep_z" in b.pointid_last_error()


def test_no_rows_is_a_no_op(b):
    assert dense(b, m=0, x=None, w=None, y=None) == b.POINTID_OK
    assert b.lib.pointid_gated(FAKE, BF16, 2, 0, 64, 64, None, None, None, None, None, None, None, None, NULL) == \
        b.POINTID_OK
    assert b.lib.pointid_checkpoint_save(BF16, 0, 5, None, None, NULL) == b.POINTID_OK
    assert b.lib.pointid_checkpoint_load(BF16, 0, 5, None, None, NULL) == b.POINTID_OK


def test_backward_refusals(b):
    def call(act=1, dy="", x="", w="", z="", dx="", dw="", db=None):
        dy, w, dx, dw = (mat(b) if v == "" else v for v in (dy, w, dx, dw))
        x, z = (kept(b) if v == "" else v for v in (x, z))
        return b.lib.pointid_dense_backward(FAKE, BF16, act, 4, 64, 64, dy, x, w, z, dx, dw, db, NULL)
    for name in ("dy", "x", "w", "z"):
        assert call(**{name: None}) == b.POINTID_EINVAL and name in b.pointid_last_error()
    assert call(z=kept(b, at=None, codes=1)) == b.POINTID_EINVAL
    assert call(db=ctypes.c_void_p(3)) == b.POINTID_EINVAL
    assert call(dx=mat(b, ld=1)) == b.POINTID_EINVAL and "dx" in b.pointid_last_error()


def test_gated_backward_refusals(b):
    def call(m=4, dh="", x="", wg="", wu="", g="", u="", dx="", dwg="", dwu=""):
        dh, wg, wu, dx, dwg, dwu = (mat(b) if v == "" else v for v in (dh, wg, wu, dx, dwg, dwu))
        x, g, u = (kept(b) if v == "" else v for v in (x, g, u))
        return b.lib.pointid_gated_backward(FAKE, BF16, 2, m, 64, 64, dh, x, wg, wu, g, u, dx, dwg, dwu, None, None, NULL)
    for name in ("dh", "x", "wg", "wu", "g", "u"):
        assert call(**{name: None}) == b.POINTID_EINVAL and name in b.pointid_last_error()
    assert call(dwg=None) == b.POINTID_EINVAL and "both" in b.pointid_last_error()
    assert call(dwu=None) == b.POINTID_EINVAL
    assert call(u=kept(b, at=None, codes=1, exponents=1)) == b.POINTID_EINVAL and "alike" in b.pointid_last_error()


def test_checkpoint_refusals(b):
    ok = ctypes.byref(b._Packed(1, 1))
    for fn, order in ((b.lib.pointid_checkpoint_save, 1), (b.lib.pointid_checkpoint_load, -1)):
        def call(rows, cols, m, c):
            return fn(BF16, rows, cols, *((m, c)[::order]), NULL)
        assert call(-1, 4, mat(b), ok) == b.POINTID_EINVAL
        assert call(2, 0, mat(b), ok) == b.POINTID_EINVAL
        assert call(2, (1 << 20) + 1, mat(b), ok) == b.POINTID_EINVAL
        assert call(2, 65, mat(b), ok) == b.POINTID_EINVAL
        assert call(2, 64, None, ok) == b.POINTID_EINVAL
        assert call(2, 64, mat(b), None) == b.POINTID_EINVAL
        assert call(2, 64, mat(b), ctypes.byref(b._Packed(1, None))) == b.POINTID_EINVAL


def test_binding_refusals(b):
    """What the binding checks before the call: types, devices, shapes, strides."""
    layers = b.Layers(FAKE, 0)
    layers.close = lambda: None
    x = torch.zeros((2, 4), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device"):
        b.pointid_dense(layers, x, torch.zeros((4, 8), dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="inner"):
        b.pointid_dense(layers, x, torch.zeros((5, 8), dtype=torch.bfloat16))
    with pytest.raises(TypeError):
        b.pointid_dense(layers, x.double(), x)
    with pytest.raises(TypeError):
        b.pointid_dense(layers, x[0], x)
    with pytest.raises(ValueError, match="act"):
        b.pointid_dense(layers, x, torch.zeros((4, 8), dtype=torch.bfloat16), act="tanh")
    with pytest.raises(ValueError):
        b.Checkpoint(torch.zeros((2, 40), dtype=torch.uint8), torch.zeros((2, 2), dtype=torch.uint8))
    layers._raw = None


@pytest.mark.parametrize("sanitize", ["address", "thread"])
def test_refusals_under_sanitizer(sanitize):
    if os.environ.get("POINTID_LIB"):
        pytest.skip("already in a child process")
    lib, rt = B.library_path(sanitize), B.sanitizer_runtime(sanitize)
    if not os.path.exists(lib) or rt is None:
        pytest.skip("the sanitized build or its runtime is not there")
    env = dict(os.environ, POINTID_LIB=lib, LD_PRELOAD=rt, UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1",
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1", TSAN_OPTIONS="halt_on_error=1:report_signal_unsafe=0")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider", __file__], cwd=ROOT, env=env,
                       capture_output=True, text=True, timeout=600)
    out = r.stdout + r.stderr
    assert r.returncode == 0 and "Sanitizer" not in out and "runtime error:" not in out, out[-4000:]
