"""Host-side checks of dropout, the norms at a residual joint and log probabilities: every refusal
comes before any pointer or device is touched, so the pointers below are never dereferenced."""

import ctypes
import math
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
AT = 0x20000


@pytest.fixture(scope="module")
def b():
    from paper_2009_04509_amd import binding
    return binding


def mat(b, at=AT, ld=64):
    return b._Matrix(at, ld)


def dropout(b, layers=FAKE, dtype=BF16, m=4, n=64, x="", drop="", residual=None, y=""):
    x, y = (mat(b) if v == "" else v for v in (x, y))
    return b.lib.pointid_dropout(layers, dtype, m, n, x, b._Drop(0.5, 1, 2, None) if drop == "" else drop, residual, y, NULL)


def refused(b, rc, word):
    assert rc == b.POINTID_EINVAL and word in b.pointid_last_error(), b.pointid_last_error()


@pytest.mark.parametrize("case, word", [
    (dict(layers=NULL), "layers"), (dict(m=-1), "m must"), (dict(m=(1 << 28) + 1), "m must"), (dict(n=0), "n must"),
    (dict(n=(1 << 20) + 1), "n must"), (dict(x=None), "x is NULL"), (dict(y=None), "y is NULL"), (dict(drop=None), "drop"),
])
def test_dropout_refusals(b, case, word):
    refused(b, dropout(b, **case), word)


def test_dropout_arguments(b):
    for p in (-0.1, 1.1, math.nan):
        refused(b, dropout(b, drop=b._Drop(p, 1, 2, None)), "p must")
    refused(b, dropout(b, drop=b._Drop(0.5, 1, 2, 0x1004)), "step")
    for name in ("x", "residual", "y"):
        refused(b, dropout(b, **{name: mat(b, ld=63)}), name)
        refused(b, dropout(b, **{name: mat(b, at=AT + 1)}), "aligned")
    assert dropout(b, m=0, x=None, y=None) == b.POINTID_OK
    for dtype in (3, -1):
        assert dropout(b, dtype=dtype) == b.POINTID_EUNSUPPORTED


def norm(b, layers=FAKE, dtype=BF16, m=4, n=64, x="", norm="", block="", total="", h="", stats=None):
    x, total, h = (mat(b) if v == "" else v for v in (x, total, h))
    norm = b._NormOf(1, 1e-5, None, None) if norm == "" else norm
    return b.lib.pointid_norm(layers, dtype, m, n, x, norm, blk(b) if block == "" else block, total, h, stats, NULL)


def blk(b, at=AT, ld=64, kind=1, eps=1e-5, weight=None, bias=None, gate=None, scale=1.0, p=0.0, step=None):
    return b._Block(at, ld, kind, eps, weight, bias, gate, scale, p, 1, 2, step)


def test_norm_refusals(b):
    for case, word in ((dict(layers=NULL), "layers"), (dict(m=-1), "m must"), (dict(n=1 << 21), "n must"), (dict(x=None), "x is"),
                       (dict(total=None, h=None), "neither"), (dict(norm=None), "both or neither"),
                       (dict(h=None), "both or neither"), (dict(block=None), "without a block"),
                       (dict(block=blk(b, at=None)), "out is NULL"), (dict(block=blk(b, kind=3)), "kind"),
                       (dict(block=blk(b, eps=-1.0)), "eps"), (dict(block=blk(b, scale=math.inf)), "scale"),
                       (dict(block=blk(b, p=2.0)), "p must"), (dict(block=blk(b, gate=AT + 2)), "gate"),
                       (dict(block=blk(b, weight=AT + 2)), "after"), (dict(norm=b._NormOf(7, 0, None, None)), "kind"),
                       (dict(norm=b._NormOf(2, math.nan, None, None)), "eps"), (dict(norm=b._NormOf(2, math.inf, None, None)), "eps"),
                       (dict(norm=b._NormOf(1, 0, AT + 1, None)), "aligned"), (dict(stats=ctypes.c_void_p(AT + 4)), "stats"),
                       (dict(total=mat(b, ld=3)), "total"), (dict(h=mat(b, at=AT + 1)), "aligned"), (dict(x=mat(b, ld=3)), "x:")):
        refused(b, norm(b, **case), word)
    assert norm(b, m=0, x=None, total=None, h=None) == b.POINTID_OK
    assert norm(b, dtype=3) == b.POINTID_EUNSUPPORTED


def test_norm_backward_refusals(b):
    def call(layers=FAKE, dtype=BF16, m=4, n=64, dh="", total="", stats=AT, norm="", block="", dtotal="", grads="", scratch=None):
        dh, total, dtotal = (mat(b) if v == "" else v for v in (dh, total, dtotal))
        norm = b._NormOf(1, 1e-5, None, None) if norm == "" else norm
        grads = b._NormGrads(AT, 64, AT, 64, AT, AT, AT, AT, AT) if grads == "" else grads
        return b.lib.pointid_norm_backward(layers, dtype, m, n, dh, total, stats, norm, blk(b) if block == "" else block, dtotal,
                                           grads, scratch, 0, NULL)
    sums = dict(norm=b._NormGrads(None, 0, None, 0, AT, None, None, None, None),
                after=b._NormGrads(None, 0, None, 0, None, None, AT, None, None),
                gate=b._NormGrads(None, 0, None, 0, None, None, None, None, AT),
                odd=b._NormGrads(None, 0, None, 0, AT + 2, None, None, None, None))
    for case, word in ((dict(layers=NULL), "layers"), (dict(grads=None), "grads"), (dict(dh=None), "dh"), (dict(total=None), "total"),
                       (dict(stats=None), "stats"), (dict(stats=AT + 4), "stats"), (dict(norm=None, grads=sums["norm"]), "without norm"),
                       (dict(block=None), "without a block"), (dict(block=None, grads=sums["gate"]), "without a block"),
                       (dict(block=blk(b, kind=0), grads=sums["after"]), "after the block"),
                       (dict(block=blk(b, at=None)), "out is NULL"), (dict(grads=sums["odd"]), "aligned"),
                       (dict(block=blk(b, kind=0, at=None), grads=sums["gate"]), "out is NULL"),
                       (dict(norm=None, dtotal=None, grads=b._NormGrads(AT, 64)), "neither"),
                       (dict(grads=b._NormGrads(AT, 3)), "dx"), (dict(grads=b._NormGrads(None, 0, AT, 3)), "dout"),
                       (dict(scratch=ctypes.c_void_p(AT + 16)), "scratch"), (dict(n=0), "n must")):
        refused(b, call(**case), word)
    assert call(dtype=4) == b.POINTID_EUNSUPPORTED
    assert call(grads=b._NormGrads()) == b.POINTID_OK                   # nothing is wanted
    assert call(m=0, dh=None, total=None, stats=None, grads=b._NormGrads(AT, 64)) == b.POINTID_OK
    assert b.lib.pointid_norm_backward_scratch(NULL, 4, 64) == 0


def logprobs(b, layers=FAKE, dtype=BF16, m=4, n=64, logits="", scale=1.0, targets=AT, logp=AT, lse=AT, entropy=AT, top=3,
             top_ids=AT, top_logp=AT, scratch=None):
    logits = mat(b) if logits == "" else logits
    return b.lib.pointid_logprobs(layers, dtype, m, n, logits, scale, targets, logp, lse, entropy, top, top_ids, top_logp,
                                  scratch, 0, NULL)


def test_logprobs_refusals(b):
    for case, word in ((dict(layers=NULL), "layers"), (dict(logits=None), "logits"), (dict(scale=0.0), "scale"),
                       (dict(scale=-1.0), "scale"), (dict(scale=math.nan), "scale"), (dict(scale=math.inf), "scale"),
                       (dict(top=-1), "top must"), (dict(top=65), "top must"), (dict(n=2), "top must"),
                       (dict(targets=None), "targets"), (dict(top_ids=None), "top_ids"), (dict(top_logp=None), "top_ids or"),
                       (dict(logp=None, lse=None, entropy=None, top=0), "no output"), (dict(lse=AT + 2), "aligned"),
                       (dict(targets=AT + 2), "targets"), (dict(top_ids=AT + 1), "top_ids"), (dict(logits=mat(b, ld=5)), "logits"),
                       (dict(scratch=ctypes.c_void_p(AT + 8)), "scratch"), (dict(m=-2), "m must")):
        refused(b, logprobs(b, **case), word)
    assert logprobs(b, dtype=7) == b.POINTID_EUNSUPPORTED
    assert logprobs(b, m=0, logits=None) == b.POINTID_OK
    assert b.lib.pointid_logprobs_scratch(NULL, 4, 64, 3) == 0


def test_logprobs_backward_refusals(b):
    def call(layers=FAKE, dtype=BF16, m=4, n=64, logits="", scale=1.0, lse=AT, targets=AT, dlogp=AT, entropy=AT, dentropy=AT,
             dlse=AT, dlogits=""):
        logits, dlogits = (mat(b) if v == "" else v for v in (logits, dlogits))
        return b.lib.pointid_logprobs_backward(layers, dtype, m, n, logits, scale, lse, targets, dlogp, entropy, dentropy, dlse,
                                               dlogits, NULL)
    for case, word in ((dict(layers=NULL), "layers"), (dict(logits=None), "logits"), (dict(dlogits=None), "dlogits"),
                       (dict(lse=None), "lse"), (dict(dlogp=None, dentropy=None, dlse=None), "no gradient"),
                       (dict(targets=None), "targets"), (dict(entropy=None), "entropy"), (dict(scale=0.0), "scale"),
                       (dict(dlogits=mat(b, ld=1)), "dlogits"), (dict(dlse=AT + 1), "aligned"), (dict(targets=AT + 3), "targets")):
        refused(b, call(**case), word)
    assert call(dtype=3) == b.POINTID_EUNSUPPORTED
    assert call(m=0, logits=None, dlogits=None, lse=None) == b.POINTID_OK


def test_binding_refusals(b):
    """What the binding checks before the call: types, devices, shapes, strides."""
    layers = b.Layers(FAKE, 0)
    layers.close = lambda: None
    x = torch.zeros((2, 8))
    with pytest.raises(ValueError, match="device"):
        b.pointid_dropout(layers, x, b.Drop(0.5, 1))
    with pytest.raises(TypeError):
        b.pointid_dropout(layers, x.double(), b.Drop(0.5, 1))
    with pytest.raises(ValueError, match="neither"):
        b.pointid_norm(layers, x)
    with pytest.raises(ValueError, match="h needs norm"):
        b.pointid_norm(layers, x, b.Norm(), total=x)
    with pytest.raises(ValueError, match="kind"):
        b._norm(b.Norm("batch"), "norm", 8, 0)
    with pytest.raises(ValueError, match="device"):
        b._norm(b.Norm("rms", x[0]), "norm", 8, 0)
    for drop in (b.Drop(1.5, 0), b.Drop(0.5, -1), b.Drop(0.5, 1 << 64), b.Drop(0.5, 0, 1 << 64)):
        with pytest.raises(ValueError):
            b._drop(drop, 0)
    with pytest.raises(TypeError):
        b._drop(b.Drop(0.5, 0, 0, torch.zeros(1)), 0)
    with pytest.raises(ValueError, match="step"):
        b._drop(b.Drop(0.5, 0, 0, torch.zeros(1, dtype=torch.int64)), 0)
    with pytest.raises(ValueError, match="device"):
        b.pointid_logprobs(layers, x)
    with pytest.raises(ValueError, match="device"):
        b.pointid_logprobs_backward(layers, x, x[:, 0])
    with pytest.raises(TypeError):
        b._vector(torch.zeros(2, dtype=torch.int64), "targets", 2, 0, torch.int32)
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
