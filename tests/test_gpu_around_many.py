"""GPU: dropout, the joint and log probabilities over so many rows that a block has several in turn:
the mask of each row, the sums over all of them, the choice of the likeliest columns by one wave, rows
alone, and matrices past the last-level cache whose rows lie off every boundary.  Against the
definitions in 64 bits (tolerances: see around64)."""

import math

import pytest
import torch

import around64 as A

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
EPS = 1e-5
SEED, OFFSET = 0x0123456789ABCDEF, (3 << 32) + 5


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


def factor_of(rows, cols, p):
    """drop's factors of the given rows."""
    threshold = math.floor(p * 65536 + 0.5)
    bits = torch.cat([A.drop_bits(1, cols, SEED, OFFSET, first_row=r) for r in rows])
    return torch.where(bits >= threshold, 65536 / (65536 - threshold), 0.0).double()


class Joint:
    """A joint's inputs, on the device."""

    def __init__(self, pid, dtype, m, n, before, after, p, pad=0):
        g = torch.Generator(device=DEV).manual_seed(m + n)

        def matrix():
            big = torch.randn((m, n + pad), generator=g, device=DEV).to(A.DT[dtype])
            return big[:, pad // 2:pad // 2 + n]

        def params(kind):
            w, b = (torch.randn(n, generator=g, device=DEV) for _ in range(2))
            return w, b if kind == "layer" else None

        self.dtype, self.m, self.n, self.before, self.after, self.p = dtype, m, n, before, after, p
        self.x, self.o, self.dh, self.dt = (matrix() for _ in range(4))
        (self.wb, self.bb), (self.wa, self.ba) = params(before), params(after)
        if not after:
            self.wa = None
        self.gate, self.scale = torch.randn(n, generator=g, device=DEV), 0.5
        self.norm = pid.Norm(before, self.wb, self.bb, EPS)
        self.block = pid.Block(self.o, pid.Norm(after, self.wa, self.ba, EPS) if after else None, self.gate, self.scale,
                               pid.Drop(p, SEED, OFFSET) if p else None)

    def check_forward(self, got, rows):
        def f(t):
            return None if t is None else t[rows].double().cpu() if t.dim() == 2 else t.double().cpu()

        factor = factor_of(rows, self.n, self.p) if self.p else None
        t, tt = A.total64(f(self.x), f(self.o), self.after, EPS, f(self.wa), f(self.ba), f(self.gate), self.scale, factor)[:2]
        u, tu = A.norm64(self.before, EPS, t, tt)[:2]
        h, th = A.affine64(u, tu, f(self.wb), f(self.bb))
        A.near(got.total[rows], t, A.rounded(t, tt, self.dtype), "total")
        A.near(got.h[rows], h, A.rounded(h, th, self.dtype), "h")

    def check_backward(self, back, total, stats, rows=None):
        """Of all rows (the sums too), or of some."""
        def f(t):
            return None if t is None else (t if rows is None or t.dim() == 1 else t[rows]).double().cpu()

        at = range(self.m) if rows is None else rows
        factor = None
        if self.p:
            factor = factor_of(at, self.n, self.p) if rows is not None else A.drop_factor(self.m, self.n, self.p, SEED, OFFSET)
        want = A.back64(f(self.dh), f(total), f(self.o), f(stats), self.before, self.after, f(self.wb), f(self.wa), f(self.ba),
                        f(self.gate), self.scale, factor, f(self.dt))
        given = {"dx": True, "dout": True, "dweight": True, "dbias": self.bb is not None, "dblock_weight": bool(self.after),
                 "dblock_bias": self.ba is not None, "dgate": True}
        for name, there in given.items():
            g = getattr(back, name)
            if not there:
                assert g is None, name
                continue
            v, tol = want[name]
            if name in ("dx", "dout"):
                A.near(g if rows is None else g[rows], v, A.rounded(v, tol, self.dtype), name)
            elif rows is None:
                A.near(g, v, A.rounded(v, tol, "fp32"), name)


KINDS = [("rms", "rms"), ("layer", "layer"), ("layer", None)]


# more sets of rows than blocks: parameters in shared memory and not, two pieces a thread, rows read again
@pytest.mark.parametrize("dtype, m, n", [(d, m, n) for d in ("bf16", "fp16", "fp32") for m, n in (
    (4200, 4096), (70000, 40), (9000, 520), (8400, 1003))] + [("bf16", 66000, 8200), ("bf16", 66000, 16392)])
def test_masks_of_many_rows_forward(pid, layers, dtype, m, n):
    rows = sorted({0, 1, 5, m // 3, m // 2, m // 2 + 1, m - 257, m - 2, m - 1})
    for before, after in KINDS[:1] if m * n > 1 << 28 else KINDS:
        j = Joint(pid, dtype, m, n, before, after, 0.2)
        j.check_forward(pid.pointid_norm(layers, j.x, j.norm, j.block), rows)


@pytest.mark.parametrize("m, n", [(3000, 1000), (20000, 40), (1100, 2600), (600, 6200), (800, 9000)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_masks_and_sums_of_many_rows_backward(pid, layers, dtype, m, n):
    for before, after in KINDS:
        j = Joint(pid, dtype, m, n, before, after, 0.2)
        got = pid.pointid_norm(layers, j.x, j.norm, j.block, keep=True)
        back = pid.pointid_norm_backward(layers, j.dh, got.total, got.stats, j.norm, j.block, dtotal=j.dt)
        j.check_backward(back, got.total, got.stats)


@pytest.mark.parametrize("n", [3, 40, 300, 513, 3000, 4096])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_of_logits_alone(pid, layers, dtype, n):
    """Where a row alone is not split either, its results are the same bits among others."""
    m = 600
    x = A.rand(A.gen(n), m, n, dtype=dtype, scale=3.0).to(DEV)
    t = (torch.arange(m, device=DEV) * 7 % n).int()
    top = min(n, 9)
    got = pid.pointid_logprobs(layers, x, t, entropy=True, top=top)
    for r in (0, 1, 17, 333, m - 1):
        one = pid.pointid_logprobs(layers, x[r:r + 1], t[r:r + 1], entropy=True, top=top)
        assert all(torch.equal(a, b[r:r + 1]) for a, b in zip(one, got)), r


@pytest.mark.parametrize("n", [520, 3000, 8192])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_ordered_rows_by_one_wave(pid, layers, dtype, n):
    """More than 1024 rows: a wave has a row of its own.  Orders that go with its threads' columns give more
    candidates than its list holds."""
    m, i = 1100, torch.arange(n, device=DEV)
    x = torch.stack([(i // 8 % 64).float() * 8 + i // 512, -(i // 8 % 64).float() * 8 - i // 512, torch.zeros(n, device=DEV),
                     (i // 8).float() / 4, -(i // 8).float() / 4]).repeat(m // 5, 1).to(A.DT[dtype])
    want = torch.sort(x.double(), dim=1, descending=True, stable=True)
    for top in (1, 8, 64):
        got = pid.pointid_logprobs(layers, x, top=top)
        assert torch.equal(got.top_ids.long(), want.indices[:, :top]), top


# matrices of 384 MB and more together, rows of odd widths at odd pitches between columns of NaN
PAD = 3


def between(m, n, dtype=torch.bfloat16):
    big = torch.full((m, n + 2 * PAD), math.nan, dtype=dtype, device=DEV)
    return big, big[:, PAD:PAD + n]


def untouched(big):
    return bool(torch.isnan(big[:, :PAD]).all() and torch.isnan(big[:, -PAD:]).all())


def test_dropout_past_the_cache_off_every_boundary(pid, layers):
    m, n = 16385, 8191
    g = torch.Generator(device=DEV).manual_seed(1)
    (bx, x), (br, r), (by, y) = (between(m, n) for _ in range(3))
    x.copy_(torch.randn((m, n), generator=g, device=DEV))
    r.copy_(torch.randn((m, n), generator=g, device=DEV))
    for place in (y, r):
        rows = [0, 1, 2, 8000, m - 2, m - 1]
        v = A.dropped(x[rows].double().cpu(), factor_of(rows, n, 0.3))
        w = v + r[rows].double().cpu()
        assert pid.pointid_dropout(layers, x, pid.Drop(0.3, SEED, OFFSET), residual=r, y=place) is place
        A.near(place[rows], w, A.rounded(w, 2 * A.E * v.abs() + A.E * (v.abs() + w.abs()), "bf16"), "y")
        assert torch.isfinite(place).all() and untouched(bx) and untouched(br) and untouched(by)
    assert torch.equal(r, y)


def test_the_joint_past_the_cache_off_every_boundary(pid, layers):
    m, n = 16385, 4095
    j = Joint(pid, "bf16", m, n, "rms", "layer", 0.1, pad=2 * PAD)
    rows = [0, 1, 7, 9000, m - 2, m - 1]
    (bt, t), (bh, h), (bd, d) = (between(m, n) for _ in range(3))
    got = pid.pointid_norm(layers, j.x, j.norm, j.block, keep=True, total=t, h=h)
    j.check_forward(got, rows)
    assert torch.isfinite(t).all() and torch.isfinite(h).all() and untouched(bt) and untouched(bh)
    back = pid.pointid_norm_backward(layers, j.dh, t, got.stats, j.norm, j.block, dtotal=j.dt, dx=d)
    j.check_backward(back, t, got.stats, rows)
    assert torch.isfinite(d).all() and torch.isfinite(back.dout).all() and untouched(bd)
    d.copy_(j.dt)
    place = pid.pointid_norm_backward(layers, j.dh, t, got.stats, j.norm, j.block, dtotal=d, dx=d)
    assert torch.equal(place.dx, pid.pointid_norm_backward(layers, j.dh, t, got.stats, j.norm, j.block, dtotal=j.dt).dx)
    assert untouched(bd) and torch.equal(place.dout, back.dout)


def test_logits_past_the_cache_off_every_boundary(pid, layers):
    m, n = 6401, 32003
    g = torch.Generator(device=DEV).manual_seed(2)
    bx, x = between(m, n)
    x.copy_(torch.randn((m, n), generator=g, device=DEV) * 3)
    t = torch.randint(0, n, (m,), generator=g, device=DEV, dtype=torch.int32)
    dlogp, dh = (torch.randn(m, generator=g, device=DEV) for _ in range(2))
    got = pid.pointid_logprobs(layers, x, t, entropy=True)
    rows = [0, 1, 3000, m - 2, m - 1]
    by, y = between(m, n)

    def f(v):
        return v[rows].double().cpu()

    v, tol = A.logprobs_back64(f(x), 1.0, f(got.lse), t[rows].cpu(), f(dlogp), f(got.entropy), f(dh), None)
    for place, big in ((y, by), (x, bx)):
        pid.pointid_logprobs_backward(layers, x, got.lse, t, dlogp, got.entropy, dh, dlogits=place)
        A.near(place[rows], v, A.rounded(v, tol, "bf16"), "dlogits")
        assert torch.isfinite(place).all() and untouched(big)
    assert torch.equal(x, y)
