"""GPU: log probabilities, entropy and the most likely columns, and the logits' gradient,
against their definitions in 64 bits (tolerances: see around64)."""

import math

import pytest
import torch

import around64 as A

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
INF = math.inf


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


def check(pid, layers, x, targets, scale, top, dtype, what=""):
    """Both passes of logits x on the host; their results."""
    m, n = x.shape
    t = None if targets is None else targets.to(DEV)
    X = x.to(DEV)
    got = pid.pointid_logprobs(layers, X, t, scale, entropy=True, top=top)
    want = A.logprobs64(x.double(), float(torch.tensor(scale)), targets, top)
    assert (got.logp is None) == (targets is None) and (got.top_ids is None) == (top == 0)
    for name, (v, tol) in want.items():
        g = getattr(got, name)
        if name == "top_ids":
            assert torch.equal(g.long().cpu(), v), f"top_ids {what}"
        else:
            A.near(g, v, A.rounded(v, tol, "fp32"), f"{name} {what}")
    g = A.gen(n)
    dlogp, dh, dl = (torch.randn(m, generator=g) for _ in range(3))
    lse, h = got.lse.double().cpu(), got.entropy.double().cpu()
    for use in ((1, 0, 0), (1, 1, 1), (0, 1, 0), (0, 0, 1)):
        if use[0] and targets is None:
            continue
        args = [v if u else None for u, v in zip(use, (dlogp, dh, dl))]
        dx = pid.pointid_logprobs_backward(layers, X, got.lse, t if use[0] else None, *(
            None if v is None else v.to(DEV) for v in (args[0], got.entropy if use[1] else None, args[1], args[2])), scale=scale)
        v, tol = A.logprobs_back64(x.double(), float(torch.tensor(scale)), lse, targets if use[0] else None,
                                   *(None if v is None else v.double() for v in (args[0], h if use[1] else None, args[1], args[2])))
        A.near(dx, v, A.rounded(v, tol, dtype), f"dlogits {use} {what}")
    return got


# rows of a few columns, about a wave's 512 and a block's 2048, and split ones
SIZES = [(1, 1), (2, 2), (700, 3), (5, 8), (3, 9), (40, 64), (9, 65), (130, 200), (4, 511), (6, 513), (3, 2049), (2, 5000),
         (1, 8191), (1, 65537), (3, 131072)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m, n", SIZES)
def test_logprobs(pid, layers, dtype, m, n):
    g = A.gen(m * 31 + n)
    for scale, top, banned in ((1.0, min(n, 5), 0.0), (0.7, min(n, 64), 0.1), (1.5, 0, 0.5), (1.0, 1, 0.0)):
        x = A.rand(g, m, n, dtype=dtype, scale=3.0)
        targets = torch.randint(0, n, (m,), generator=g, dtype=torch.int32)
        if banned:
            x = torch.where(torch.rand((m, n), generator=g) < banned, -INF, x)
            targets[::3] = torch.tensor([-1, n, -100, 2 ** 31 - 1], dtype=torch.int32).repeat(m)[:targets[::3].numel()]
        check(pid, layers, x, targets, scale, top, dtype, f"scale {scale} top {top}")


@pytest.mark.parametrize("n", [7, 300, 3000, 70000])
@pytest.mark.parametrize("order", ["equal", "rising", "falling", "few values", "threads"])
def test_top_of_ordered_rows(pid, layers, n, order):
    """Orders that go with the threads' own columns, and rows of equals: the lowest column first."""
    i = torch.arange(n)
    x = {"equal": torch.zeros(n), "rising": i / 8, "falling": -i / 8.0, "few values": (i * 7919 % 3).float(),
         "threads": (i // 8 % 256).float() * 100 + (i // 2048)}[order].repeat(3, 1)
    x[1] = -x[1]
    x[2] = torch.where(i % 5 == 0, x[2], -INF)
    for top in (1, 20, 64):
        got = pid.pointid_logprobs(layers, x.to(DEV), top=min(top, n))
        ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(got.top_ids.long().cpu(), ids), (order, top)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("m, n", [(3, 300), (1100, 3000), (3, 70000), (520, 20000)])
def test_top_of_few_values(pid, layers, dtype, m, n):
    """Rows of 16-bit values with many equals, of either sign, by every kernel that chooses them."""
    g = A.gen(n)
    x = torch.randint(-20, 3, (m, n), generator=g).double() * torch.rand((m, 1), generator=g, dtype=torch.float64)
    x[1] = torch.where(torch.rand(n, generator=g) < 0.9, -INF, x[1])
    x = x.to(A.DT[dtype])
    for top in (1, 7, 64):
        got = pid.pointid_logprobs(layers, x.to(DEV), top=top)
        ids = torch.sort(x.double() + 0.0, dim=1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(got.top_ids.long().cpu(), ids), top


def test_the_widest_rows(pid, layers):
    """More pieces than 16 bits count, by one block a row."""
    m, n = 520, 1 << 20
    x = torch.zeros((m, n), dtype=torch.bfloat16, device=DEV)
    at = torch.arange(m, device=DEV) * 2003 + 7
    x[torch.arange(m, device=DEV), at] = 2
    x[:, -1] = 1
    got = pid.pointid_logprobs(layers, x, top=4)
    want = torch.stack([at, torch.full_like(at, n - 1), torch.zeros_like(at), torch.ones_like(at)], 1)
    assert torch.equal(got.top_ids.long(), want)
    lse = math.log(n - 2 + math.e + math.exp(2))
    assert (got.lse - lse).abs().max() < 1e-5


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m, n", [(2, 100), (2, 9000), (1100, 5000), (520, 9000)])
def test_nans_of_both_kinds_hide_nothing(pid, layers, dtype, m, n):
    """A quiet and a signalling NaN right after a row's largest value, in the same thread's columns."""
    x = A.rand(A.gen(n), m, n, dtype=dtype)
    best = torch.arange(m) * 13 % (n - 8) // 8 * 8
    rows = torch.arange(m)
    x[rows, best] = 9.0
    bits = x.view(torch.int16 if dtype != "fp32" else torch.int32)
    nan = {"bf16": (0x7FC0, 0x7F81), "fp16": (0x7E00, 0x7C01), "fp32": (0x7FC00000, 0x7F800001)}[dtype]
    for kind in (0, 1):
        bits[rows, best + 1] = nan[kind]
        got = pid.pointid_logprobs(layers, x.to(DEV), entropy=True, top=2)
        assert torch.equal(got.top_ids[:, 0].long().cpu(), best)
        second = torch.where(torch.isnan(x), -INF, x.double())
        second[rows, best] = -INF
        assert torch.equal(got.top_ids[:, 1].long().cpu(), second.max(1).values.view(-1, 1).eq(second).int().argmax(1))
        assert got.lse.isnan().all() and got.entropy.isnan().all() and got.top_logp.isnan().all()


def test_zeros_of_both_signs_are_equal(pid, layers):
    x = torch.zeros((1, 600), device=DEV)
    x[0, :300] = -0.0
    assert pid.pointid_logprobs(layers, x, top=4).top_ids.tolist() == [[0, 1, 2, 3]]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("n", [3, 70, 900, 40000])
def test_masked_rows(pid, layers, dtype, n):
    """Rows with nothing left, with one column left, at the type's lowest value, wholly and in part."""
    lowest = torch.finfo(A.DT[dtype]).min
    x = A.rand(A.gen(n), 6, n, dtype=dtype)
    x[0] = -INF
    x[1] = -INF
    x[1, n // 2] = 1.5
    x[2] = lowest
    x[3, 1:] = lowest
    x[4, :-1] = -INF
    targets = torch.tensor([1, n // 2, 2, 0, 0, 1], dtype=torch.int32)
    got = check(pid, layers, x, targets, 1.0, min(n, 4), dtype)
    assert got.lse[0] == -INF and got.logp[0] == -INF and got.entropy[0] == 0
    assert got.top_ids[0].tolist() == list(range(min(n, 4))) and (got.top_logp[0] == -INF).all()
    assert got.logp[1] == 0 and got.entropy[1] == 0 and got.logp[4] == -INF
    if dtype != "fp32":                                        # equal probabilities
        assert abs(got.entropy[2].item() - math.log(n)) < 1e-5


@pytest.mark.parametrize("n", [5, 700, 50000])
def test_infinities_and_nans(pid, layers, n):
    x = torch.randn((4, n), generator=A.gen(1))
    x[0, n // 3] = INF
    x[1, n // 2] = math.nan
    x[2] = math.nan
    t = torch.zeros(4, dtype=torch.int32, device=DEV)
    got = pid.pointid_logprobs(layers, x.to(DEV), t, entropy=True, top=3)
    assert got.lse[:3].isnan().all() and got.logp[:3].isnan().all() and got.entropy[:3].isnan().all()
    assert got.top_logp[:3].isnan().all() and torch.isfinite(got.lse[3])
    assert got.top_ids[0, 0] == n // 3 and got.top_ids[2].tolist() == [0, 1, 2] and n // 2 not in got.top_ids[1].tolist()
    alone = pid.pointid_logprobs(layers, x[3:].to(DEV), t[3:], entropy=True, top=3)
    assert torch.equal(alone.top_ids[0], got.top_ids[3])
    dx = pid.pointid_logprobs_backward(layers, x.to(DEV), got.lse, t, torch.ones(4, device=DEV))
    assert dx[:3].isnan().all() and torch.isfinite(dx[3]).all()


def test_large_values(pid, layers):
    """Logits of 1e4 that differ by little: nothing overflows."""
    x = (torch.randn((4, 1000), generator=A.gen(3)) + 1e4).float()
    check(pid, layers, x, torch.arange(4, dtype=torch.int32), 1.0, 10, "fp32")
    check(pid, layers, -x, torch.arange(4, dtype=torch.int32), 1.0, 10, "fp32")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [3, 45, 1000, 9001])
def test_pitches_and_in_place(pid, layers, dtype, n):
    m = 19
    big = A.rand(A.gen(n), m, n + 9, dtype=dtype)
    t = torch.arange(m, dtype=torch.int32) % n
    g = torch.randn(m, generator=A.gen(2)).to(DEV)
    for shift in (0, 1, 4):
        cut = slice(shift, shift + n)
        B = big.to(DEV)
        got = pid.pointid_logprobs(layers, B[:, cut], t.to(DEV), top=2, entropy=True)
        want = A.logprobs64(big[:, cut].double(), 1.0, t, 2)
        A.near(got.logp, want["logp"][0], A.rounded(*want["logp"], "fp32"), "logp")
        assert torch.equal(got.top_ids.long().cpu(), want["top_ids"][0])
        dx = pid.pointid_logprobs_backward(layers, B[:, cut], got.lse, t.to(DEV), g)
        v, tol = A.logprobs_back64(big[:, cut].double(), 1.0, got.lse.double().cpu(), t, g.double().cpu(), None, None, None)
        A.near(dx, v, A.rounded(v, tol, dtype), "dlogits")
        place = pid.pointid_logprobs_backward(layers, B[:, cut], got.lse, t.to(DEV), g, dlogits=B[:, cut])
        assert torch.equal(place, dx)
        assert torch.equal(B[:, :shift].cpu(), big[:, :shift]) and torch.equal(B[:, shift + n:].cpu(), big[:, shift + n:])


def test_only_what_is_asked_for(pid, layers):
    x = torch.randn((7, 90), device=DEV)
    got = pid.pointid_logprobs(layers, x)
    assert got.logp is None and got.entropy is None and got.top_ids is None and got.top_logp is None
    full = pid.pointid_logprobs(layers, x, torch.zeros(7, dtype=torch.int32, device=DEV), entropy=True, top=3)
    assert torch.equal(got.lse, full.lse)
    empty = pid.pointid_logprobs(layers, x[:0], torch.zeros(0, dtype=torch.int32, device=DEV), entropy=True, top=3)
    assert empty.logp.shape == empty.lse.shape == empty.entropy.shape == (0,) and empty.top_ids.shape == (0, 3)
    assert pid.pointid_logprobs_backward(layers, x[:0], empty.lse, dlse=empty.lse).shape == (0, 90)


@pytest.mark.parametrize("m, n", [(1, 50000), (3, 700), (300, 100)])
def test_captured(pid, layers, m, n):
    x = torch.randn((m, n), device=DEV)
    t = torch.zeros(m, dtype=torch.int32, device=DEV)
    g = torch.ones(m, device=DEV)

    def step():
        got = pid.pointid_logprobs(layers, x, t, top=5, entropy=True)
        return (*got, pid.pointid_logprobs_backward(layers, x, got.lse, t, g))

    step()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    outs = []
    for graph in graphs:
        with torch.cuda.graph(graph):
            outs.append(step())
    for i in range(3):
        x.normal_()
        t.fill_(i)
        want = [v.clone() for v in step()]
        for graph, out in zip(graphs, outs):
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_the_same_bits_and_rows_alone(pid, layers):
    x = torch.randn((600, 3000), device=DEV)
    a = pid.pointid_logprobs(layers, x, entropy=True, top=7)
    b = pid.pointid_logprobs(layers, x, entropy=True, top=7)
    assert all(torch.equal(p, q) for p, q in zip(a[1:], b[1:]))


def test_rows_past_32_bits_of_elements(pid, layers):
    m, n = 33000, 131072                                       # 4.3e9 elements of 16 bits
    x = torch.zeros((m, n), dtype=torch.bfloat16, device=DEV)
    x[-1, 77] = 5
    t = torch.full((m,), 77, dtype=torch.int32, device=DEV)
    got = pid.pointid_logprobs(layers, x, t, top=2)
    assert got.top_ids[-1].tolist() == [77, 0] and got.top_ids[0].tolist() == [0, 1]
    assert abs(got.logp[-1].item() - (5 - math.log(n - 1 + math.exp(5)))) < 1e-5
    assert abs(got.logp[0].item() + math.log(n)) < 1e-5
    dx = pid.pointid_logprobs_backward(layers, x, got.lse, t, torch.ones(m, device=DEV), dlogits=x)
    assert abs(dx[-1, 77].item() - (1 - math.exp(got.logp[-1].item()))) < 4e-3 and dx[0, 77] == 1


def test_a_first_split_without_candidates(pid, layers):
    """A split row whose first half is masked."""
    x = torch.randn((1, 100000), device=DEV)
    x[0, :60000] = -INF
    got = pid.pointid_logprobs(layers, x, top=64)
    assert torch.equal(got.top_ids.long()[0], torch.sort(x[0], descending=True, stable=True).indices[:64])
