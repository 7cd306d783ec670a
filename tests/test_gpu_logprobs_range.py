"""GPU: log probabilities where the log of the sum of exponentials is large: masks of a type's lowest
value or of -1e9 in every column, logits times a scale past fp32's range;
and the gradients of rows of nothing.

fp32 keeps lse to 2^-24 of itself, so that past 2^24 or so ln of a sum is lost in it: the gradient is
that of z_j = scale x_j rounded to fp32 (past its range to its largest finite values) and of lse as it stands,
p_j = e^(z_j - lse), which is 1 where z_j is the row's largest."""

import math

import pytest
import torch

import around64 as A

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
INF = math.inf
MOST = torch.finfo(torch.float32).max


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


def rows_of_large_values(dtype, n, m):
    """m rows: ends of the type's range and mask values in every column, in all but one, and beside -inf."""
    t = torch.finfo(A.DT[dtype])
    x = A.rand(A.gen(n), m, n, dtype=dtype)
    at = n // 2
    mask = -1e4 if dtype == "fp16" else -1e9
    x[0] = t.min
    x[1] = t.max
    x[2] = t.min
    x[2, at] = t.max
    x[3] = -INF
    x[3, at] = t.min
    x[4] = mask
    x[5] = -INF
    x[6] = -mask
    x[7, at] = t.max
    x[8] = mask
    x[8, at] = 1.5
    x[9] = (x[9].double() * 1e-3 - mask).to(x.dtype)
    targets = torch.full((m,), at, dtype=torch.int32)
    targets[8] = (at + 1) % n
    return x, targets, at


def rounded_logits(x, scale):
    """scale x in fp32, at its largest finite values past the range (in 64 bits)."""
    z = (x.double() * float(torch.tensor(scale))).float().double()
    return torch.where(torch.isinf(z) & torch.isfinite(x), z.sign() * MOST, z)


def check(pid, layers, dtype, m, n, scale):
    x, targets, at = rows_of_large_values(dtype, n, m)
    X, t = x.to(DEV), targets.to(DEV)
    got = pid.pointid_logprobs(layers, X, t, scale, entropy=True, top=2)
    want = A.logprobs64(x.double(), float(torch.tensor(scale)), targets, 2)
    assert torch.equal(got.top_ids.long().cpu(), want["top_ids"][0])
    lse, tol = want["lse"]
    lse = torch.where(torch.isfinite(lse), lse.clamp(-MOST, MOST), lse)
    A.near(got.lse, lse, A.rounded(lse, tol, "fp32"), "lse")
    # what lies below fp32's range is minus infinity in it
    for name in ("logp", "entropy"):
        v, tol = want[name]
        v = torch.where(v < -MOST, -INF, v)
        A.near(got[got._fields.index(name)], v, A.rounded(v, tol, "fp32"), name)

    # of the gradient: z less lse rounded once, its product with 1 / ln 2, and 2^q, as E each; then the formula
    l = got.lse.double().cpu().view(-1, 1)
    empty = l == -INF
    d = torch.where(empty, -INF, rounded_logits(x, scale) - l)
    p = d.exp()
    finite = torch.where(p > 0, d, 0.0)
    # (below 2^10 the kernels may leave z unrounded, or round its factors)
    size = rounded_logits(x, scale).abs().nan_to_num(posinf=0) + l.abs().nan_to_num(posinf=0)
    near_lse = torch.where(l.abs() < 1024, 4 * A.E * size, 0.0)
    tp = p * (6 * A.E + 3 * A.E * finite.abs() + torch.where(p > 0, near_lse, 0.0))
    g = A.gen(n + 1)
    dlogp, dh, dl = (torch.randn(m, generator=g) for _ in range(3))
    h = got.entropy.double().cpu()
    one = torch.zeros_like(p)
    one[torch.arange(m), targets.long()] = 1.0
    one[empty[:, 0]] = 0.0
    for use in ((1, 0, 0), (1, 1, 1)):
        a, b, c = (v.double().view(-1, 1) * u for u, v in zip(use, (dlogp, dh, dl)))
        dx = pid.pointid_logprobs_backward(
            layers, X, got.lse, t, dlogp.to(DEV), got.entropy if use[1] else None, dh.to(DEV) if use[1] else None,
            dl.to(DEV) if use[2] else None, scale=scale)
        hh = h.view(-1, 1)
        on = c - a - b * (finite + hh)
        size = c.abs() + a.abs() + (b * (finite.abs() + hh.abs())).abs()
        s = float(torch.tensor(scale))
        v = (p * on + one * a) * s
        tol = (tp * size + p * (4 * A.E * size + b.abs() * tp / p.clamp(min=1e-300)) + 2 * A.E * (one * a).abs()) * s
        tol = tol + 2 * A.E * v.abs()
        if dtype == "fp16":                            # to the nearest: from 65520 on an infinity
            v = torch.where(v.abs() - tol >= 65520, v.sign() * INF, v)
        A.near(dx, v, A.rounded(v, tol, dtype), f"dlogits {use}")


SIZES = [(12, 3), (12, 70), (12, 500), (12, 900), (1100, 2500), (12, 40000)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m, n", SIZES)
@pytest.mark.parametrize("scale", [1.0, 0.7])
def test_large_lse(pid, layers, dtype, m, n, scale):
    check(pid, layers, dtype, m, n, scale)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m, n", SIZES)
@pytest.mark.parametrize("scale", [1.25, 2.0 ** 64])
def test_past_the_range(pid, layers, dtype, m, n, scale):
    """An lse that fp32 does not reach is its largest finite value, never that of a row of nothing."""
    check(pid, layers, dtype, m, n, scale)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("n", [3, 70, 900, 40000])
def test_rows_of_nothing_have_no_gradient(pid, layers, dtype, n):
    """Their lse is minus infinity; what a loss makes of it (a penalty of lse^2: an infinity, or a NaN) does
    not reach the logits."""
    x = A.rand(A.gen(n), 4, n, dtype=dtype)
    x[1] = -INF
    x[3] = -INF
    t = torch.tensor([0, 1, -1, n - 1], dtype=torch.int32, device=DEV)
    X = x.to(DEV)
    got = pid.pointid_logprobs(layers, X, t, entropy=True)
    good = torch.ones(4, device=DEV)
    for bad in (-INF, INF, math.nan):
        d = good.clone()
        d[1::2] = bad
        for args in ((d, None, None, None), (None, got.entropy, d, None), (None, None, None, d), (d, got.entropy, d, d)):
            dx = pid.pointid_logprobs_backward(layers, X, got.lse, t if args[0] is not None else None, *args)
            assert (dx[1::2] == 0).all() and torch.isfinite(dx).all(), (bad, dx[1::2])
            same = pid.pointid_logprobs_backward(layers, X, got.lse, t if args[0] is not None else None,
                                                 *(good if v is d else v for v in args))
            assert torch.equal(dx[::2], same[::2])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [3, 70, 900, 40000])
@pytest.mark.parametrize("scale", [0.25, 2.0 ** -64])
def test_columns_further_apart_than_the_range(pid, layers, dtype, n, scale):
    """Logits whose difference passes fp32's range, their log probability not."""
    t = torch.finfo(A.DT[dtype])
    x = A.rand(A.gen(n), 3, n, dtype=dtype)
    x[:, 0], x[:, 1] = t.max, t.min
    x[1, 2] = -INF
    targets = torch.tensor([1, 2, 0], dtype=torch.int32)
    got = pid.pointid_logprobs(layers, x.to(DEV), targets.to(DEV), scale, entropy=True, top=3)
    want = A.logprobs64(x.double(), scale, targets, 3)
    for name in ("lse", "logp", "entropy", "top_logp"):
        A.near(got[got._fields.index(name)], want[name][0], A.rounded(*want[name], "fp32"), name)
    low = pid.pointid_logprobs(layers, x.to(DEV), torch.ones(3, dtype=torch.int32, device=DEV), scale)
    v, tol = A.logprobs64(x.double(), scale, torch.ones(3, dtype=torch.int32), 0)["logp"]
    A.near(low.logp, v, A.rounded(v, tol, "fp32"), "logp of the lowest")
