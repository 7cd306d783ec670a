"""Layer operators at the ends of their ranges: infinities beside large values, infinities
at the end of a few rows, row pitches that pass 32 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


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


def same_kind(y, z):
    """The infinities and NaNs of the 64-bit result z in y."""
    assert torch.equal(y.isnan(), z.isnan())
    assert torch.equal(y.isinf(), z.isinf()) and torch.equal(y[z.isinf()], z[z.isinf()])


@pytest.mark.parametrize("m", [3, 40])
@pytest.mark.parametrize("form", ["forward", "dx", "dw"])
def test_fp32_infinities_times_large_values(pid, layers, m, form):
    """No part of an infinity may meet a part of the other value with a sign of its own."""
    g = torch.Generator().manual_seed(21)
    k, n = 36, 68
    left, right = torch.randn((m, k), generator=g), torch.randn((k, n), generator=g)
    right = right.sign() * (1e5 + 300 * torch.rand((k, n), generator=g))
    left[0, 3], left[1, 5], left[2, 7] = float("inf"), -float("inf"), float("nan")
    right[3, 4], right[5, 6] = float("inf"), -float("inf")       # inf inf and -inf -inf
    z = left.double() @ right.double()
    a, b = left.to(DEV), right.to(DEV)
    if form == "forward":
        y = pid.pointid_dense(layers, a, b)
    elif form == "dx":                                           # dy [m][k] . w^T
        y = pid.pointid_dense_backward(layers, a, None, b.t().contiguous(), need_dw=False, need_db=False)[0]
    else:                                                        # x^T . dy
        y = pid.pointid_dense_backward(layers, b, a.t().contiguous(), torch.empty((m, n), device=DEV),
                                       need_dx=False, need_db=False)[1]
    same_kind(y.double().cpu(), z)


@pytest.mark.parametrize("form", ["forward", "dx", "dw"])
def test_fp32_values_above_the_largest_bf16(pid, layers, form):
    """Finite values that round to an infinity in 16 bits, beside an infinity or not."""
    g = torch.Generator().manual_seed(24)
    m, k, n = 40, 36, 68
    left, right = torch.randn((m, k), generator=g), torch.randn((k, n), generator=g) * 2.0 ** -10
    left[3, 5], left[4, 6], left[5, 7] = 3.4028e38, -3.4e38, 3.39e38
    left[6, 1] = float("inf")
    z = left.double() @ right.double()
    a, b = left.to(DEV), right.to(DEV)
    if form == "forward":
        y = pid.pointid_dense(layers, a, b)
    elif form == "dx":
        y = pid.pointid_dense_backward(layers, a, None, b.t().contiguous(), need_dw=False, need_db=False)[0]
    else:
        y = pid.pointid_dense_backward(layers, b, a.t().contiguous(), torch.empty((m, n), device=DEV),
                                       need_dx=False, need_db=False)[1]
    y = y.double().cpu()
    same_kind(y, z)
    here = z.isfinite()
    # 6 k products of parts, each sum rounded to 2^-23 of the magnitudes at most
    bound = (left.double().abs() @ right.double().abs()) * (6 * k * 2.0 ** -23)
    assert ((y - z).abs() <= bound)[here].all()


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("k", [1, 63, 513, 700])
def test_an_infinity_at_the_end_of_few_rows(pid, layers, dtype, k):
    """What stands past the last inner index is nothing, not that of the last value."""
    g = torch.Generator().manual_seed(22)
    m, n = 2, 33                                                 # odd: 16-bit weights are streamed too
    x, w = torch.randn((m, k), generator=g).to(DT[dtype]), torch.randn((k, n), generator=g).to(DT[dtype])
    x[0, k - 1] = float("inf")
    same_kind(pid.pointid_dense(layers, x.to(DEV), w.to(DEV)).double().cpu(), x.double() @ w.double())


@pytest.mark.parametrize("dtype", DT)
def test_few_rows_and_weights_far_apart(pid, layers, dtype):
    """Weights whose rows lie 2^30 bytes and more apart."""
    k, n, pitch = 9, 40, (1 << 28) + 8
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("not enough device memory")
    g = torch.Generator().manual_seed(23)
    w = torch.empty((k * pitch,), dtype=DT[dtype], device=DEV).view(k, pitch)[:, 3:3 + n]
    w.copy_(torch.randn((k, n), generator=g))
    for m in (1, 5):
        x = torch.randn((m, k), generator=g).to(DT[dtype]).to(DEV)
        z = x.double() @ w.double()
        y = pid.pointid_dense(layers, x, w)
        # a sum of 9 products, each of 3 exact parts or exact, and one rounding
        bound = (x.double().abs() @ w.double().abs()) * (2.0 ** -19 + torch.finfo(DT[dtype]).eps / 2)
        assert ((y.double() - z).abs() <= bound).all()
