"""GPU: norms of rows of one value, of rows whose values differ by little beside their mean, and of rows
whose sums pass fp32's range."""

import pytest
import torch

import around64 as A

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
EPS = 1e-5


@pytest.fixture(scope="module")
def pid():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2009_04509_amd import binding
    return binding


@pytest.fixture(scope="module")
def layers(pid):
    h = pid.pointid_layers_create(0)
    yield h
    h.close()


# of every kernel: 16 lanes and whole waves a row, whole and ragged ends, shared parameters, two pieces, read again
SIZES = [(4, 5), (4, 100), (70000, 100), (4, 1001), (4, 5280), (4200, 5280), (4, 6145), (4, 12000), (4, 16383), (4, 20000)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m, n", SIZES)
def test_rows_of_one_value(pid, layers, dtype, m, n):
    """Nothing is left of the mean: h is the bias, at a joint too."""
    values = torch.tensor([1000.0, -0.1, 4096.0, 255.0], device=DEV).to(A.DT[dtype])
    x = values.repeat(m // 4).view(-1, 1).expand(m, n).contiguous()
    b = torch.randn(n, device=DEV)
    want = b.to(A.DT[dtype]).expand(m, n)
    norm = pid.Norm("layer", torch.full((n,), 3.0, device=DEV), b)
    got = pid.pointid_norm(layers, x, norm, keep=True)
    assert torch.equal(got.h, want) and torch.equal(got.stats[:, 2], x[:, 0].float())
    got = pid.pointid_norm(layers, torch.zeros_like(x), norm, pid.Block(x), keep=True)
    assert torch.equal(got.total, x) and torch.equal(got.h, want)
    got = pid.pointid_norm(layers, torch.zeros_like(x), None, pid.Block(x, norm), keep=True)
    assert torch.equal(got.total, want) and torch.equal(got.stats[:, 0], x[:, 0].float())


@pytest.mark.parametrize("m, n", SIZES)
def test_the_mean_is_rounded_once(pid, layers, m, n):
    """fp32 rows of 1e4 and a deviation of 1: the mean is off by its own rounding, 2^-24 of it, and by that
    of the values' differences from it, which is nothing beside."""
    g = torch.Generator(device=DEV).manual_seed(n)
    x = torch.randn((m, n), generator=g, device=DEV) + 1e4
    got = pid.pointid_norm(layers, x, pid.Norm("layer", eps=EPS), keep=True)
    mean = x.double().mean(1)
    # the differences' sum is a tree of at most 40 + n / 64 terms in turn: A.depth(n) E of their mean size, 0.8
    tol = 1e4 * 1.001 * 2.0 ** -24 + 2 * A.depth(n) * A.E
    assert ((got.stats[:, 2].double() - mean).abs() <= tol).all()
    u = (x.double() - got.stats[:, 2:3].double()) * got.stats[:, 3:4].double()
    assert ((got.h.double() - u).abs() <= 4 * A.E * u.abs() + 1e-12).all()
    var = (x.double() - mean.view(-1, 1)).square().mean(1) + EPS
    # each difference is exact but for the mean's own rounding, whose square counts
    assert ((got.stats[:, 3].double() * var.sqrt() - 1).abs() <= A.depth(n) * A.E + tol * tol / var).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [100, 1001, 12000, 20000])
def test_sums_past_the_range(pid, layers, dtype, n):
    """Of squares: 0 times the weight, whatever the mean; of a layer norm's values: NaN.  The next rows are theirs."""
    x = torch.randn((6, n), device=DEV)
    x[0] = torch.where(torch.arange(n, device=DEV) % 2 == 0, 1e30, -1e30)
    x[1] = 1e30 + 1e28 * x[1].clamp(-1, 1)
    x[2] = 3e38
    x = x.to(A.DT[dtype])
    w, b = (torch.randn(n, device=DEV) for _ in range(2))
    for kind in ("rms", "layer"):
        h = pid.pointid_norm(layers, x, pid.Norm(kind, w, b)).h
        assert torch.equal(h[:2], b.to(h.dtype).expand(2, n)), kind
        assert h[2].isnan().all() if kind == "layer" else torch.equal(h[2], b.to(h.dtype))
        assert torch.equal(h[3:], pid.pointid_norm(layers, x[3:], pid.Norm(kind, w, b)).h)
