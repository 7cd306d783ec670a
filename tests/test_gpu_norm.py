"""GPU: the norms at the joint of two residual blocks, forward and backward, against their
definitions in 64 bits (tolerances: see around64)."""

import math

import pytest
import torch

import around64 as A

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
EPS = 1e-5
# (before, after, biases, gate, scale, p)
FORMS = [("rms", None, False, False, 1.0, 0.0), ("layer", None, True, True, 0.5, 0.0),
         ("rms", "rms", False, True, 1.0, 0.25), ("layer", "layer", True, True, -1.5, 0.1),
         (None, "rms", True, False, 1.0, 0.0), ("layer", "rms", False, False, 2.0, 0.5), (None, None, False, True, 1.0, 0.5)]


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


class Joint:
    """Inputs of one joint on the host, and the calls' arguments on the device."""

    def __init__(self, pid, dtype, m, n, form, seed=0, columns=None):
        self.pid, self.dtype, self.m, self.n, self.form = pid, dtype, m, n, form
        self.before, self.after, biases, gate, self.scale, self.p = form
        g = A.gen(seed + m * 7919 + n)
        self.x, self.o, self.dh, self.dt = (A.rand(g, m, n, dtype=dtype) for _ in range(4))
        if columns is not None:
            self.x, self.o = columns(self.x), columns(self.o)
        f = [torch.randn(n, generator=g) for _ in range(5)]
        self.wb, self.wa, self.gate = f[0], f[1] if self.after else None, f[2] if gate else None
        self.bb, self.ba = (f[3] if biases else None, f[4] if biases and self.after else None)
        self.seed, self.offset = 77, 1 << 35
        self.factor = A.drop_factor(m, n, self.p, self.seed, self.offset) if self.p else None

    def dev(self, t):
        return None if t is None else t.to(DEV)

    def norm(self):
        return self.pid.Norm(self.before, self.dev(self.wb), self.dev(self.bb), EPS) if self.before else None

    def block(self, out=None):
        after = self.pid.Norm(self.after, self.dev(self.wa), self.dev(self.ba), EPS) if self.after else None
        drop = self.pid.Drop(self.p, self.seed, self.offset) if self.p else None
        return self.pid.Block(self.dev(self.o) if out is None else out, after, self.dev(self.gate), self.scale, drop)

    def f64(self, t):
        return None if t is None else t.double()

    def want(self):
        """{name: (value, bound)} of the forward call, and the statistics"""
        f = self.f64
        t, tt, _, mean_a, r_a = A.total64(f(self.x), f(self.o), self.after, EPS, f(self.wa), f(self.ba), f(self.gate),
                                          self.scale, self.factor)
        out = {"total": (t, tt)}
        stats = torch.tensor([0.0, 1.0, 0.0, 1.0], dtype=torch.float64).repeat(self.m, 1)
        if self.after:
            stats[:, 0:1], stats[:, 1:2] = mean_a, r_a
        if self.before:
            u, tu, mean, r = A.norm64(self.before, EPS, t, tt)
            stats[:, 2:3], stats[:, 3:4] = mean, r
            out["h"] = A.affine64(u, tu, f(self.wb), f(self.bb))
        return out, stats

    def check_forward(self, got, what=""):
        want, stats = self.want()
        for name, (v, tol) in want.items():
            A.near(getattr(got, name), v, A.rounded(v, tol, self.dtype), f"{name} {what}")
        return stats

    def check_backward(self, got, stats, t, dt=True, what=""):
        f = self.f64
        want = A.back64(f(self.dh), f(t) if self.before else None, f(self.o), f(stats), self.before, self.after, f(self.wb),
                        f(self.wa), f(self.ba), f(self.gate), self.scale, self.factor, f(self.dt) if dt else None)
        given = {"dx": 1, "dout": 1, "dweight": self.before, "dbias": self.before and self.bb is not None,
                 "dblock_weight": self.after, "dblock_bias": self.ba is not None, "dgate": self.gate is not None}
        for name, there in given.items():
            g = getattr(got, name)
            if not there:
                assert g is None, name
                continue
            v, tol = want[name]
            A.near(g, v, A.rounded(v, tol, self.dtype if name in ("dx", "dout") else "fp32"), f"{name} {what}")


# one row to many; widths about the pieces of 8, the waves' 512, and the kernels' widest
SIZES = [(1, 1), (1, 8), (2, 9), (3, 64), (5, 127), (7, 512), (300, 513), (33, 1031), (70, 2048), (3, 4097), (2, 8200),
         (9, 16384), (2, 16392), (2, 33001)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m, n", SIZES)
def test_forward_and_backward(pid, layers, dtype, m, n):
    for i, form in enumerate(FORMS):
        j = Joint(pid, dtype, m, n, form, seed=i)
        got = pid.pointid_norm(layers, j.dev(j.x), j.norm(), j.block(), keep=True)
        stats = j.check_forward(got, str(form))
        tol = 1e-3 if n < 4 else 1e-4                          # a look; h holds them to their bounds
        assert torch.allclose(got.stats.double().cpu(), stats, rtol=tol, atol=1e-3), form
        t = got.total.cpu() if j.before else None
        dt = i % 3 != 1 or not j.before
        back = pid.pointid_norm_backward(layers, j.dev(j.dh) if j.before else None, got.total if j.before else None,
                                         got.stats, j.norm(), j.block(), dtotal=j.dev(j.dt) if dt else None)
        j.check_backward(back, got.stats.cpu(), t, dt, str(form))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("m, n", [(4100, 8192), (4097, 7000), (6, 8192), (4100, 6145), (70000, 40), (9000, 520),
                                  (4100, 3587), (4200, 4093), (70000, 13), (20000, 1001)])
def test_many_rows_and_the_widest_that_are_held(pid, layers, dtype, m, n):
    """With every parameter: what a block keeps in shared memory is largest.  The last rows and all
    column sums are checked."""
    for form in (FORMS[3], FORMS[2]):
        j = Joint(pid, dtype, 6, n, form, seed=1)
        if j.p:
            j.p, j.factor = 0.0, None                       # the rows' masks are tested elsewhere
        d = torch.device(DEV)

        def many(t):
            return j.dev(t).repeat(-(-m // 6), 1)[:m].contiguous()

        x, o, dh, dt = (many(t) for t in (j.x, j.o, j.dh, j.dt))
        got = pid.pointid_norm(layers, x, j.norm(), j.block(o), keep=True)
        back = pid.pointid_norm_backward(layers, dh, got.total, got.stats, j.norm(), j.block(o), dtotal=dt)
        few = pid.pointid_norm(layers, x[:6], j.norm(), j.block(o[:6]), keep=True)
        j.check_forward(few)
        # rows alike have results alike, wherever they stand (to the rounding of sums in another order)
        rows = torch.arange(m, device=d) % 6
        assert torch.allclose(got.h.float(), few.h.float()[rows], rtol=2.0 ** -6, atol=1e-5)
        f = pid.pointid_norm_backward(layers, dh[:6], few.total, few.stats, j.norm(), j.block(o[:6]), dtotal=dt[:6])
        j.check_backward(f, few.stats.cpu(), few.total.cpu())
        for a, b in ((back.dx, f.dx), (back.dout, f.dout)):
            assert torch.allclose(a.float(), b.float()[rows], rtol=2.0 ** -6, atol=2.0 ** -6)
        times = torch.bincount(rows, minlength=6).double()
        for name, k in (("dweight", 0), ("dblock_weight", 1), ("dgate", 2)):
            parts = []
            for i in range(6):
                one = pid.pointid_norm_backward(layers, dh[i:i + 1], few.total[i:i + 1], few.stats[i:i + 1], j.norm(),
                                                j.block(o[i:i + 1]), dtotal=dt[i:i + 1])
                parts.append(getattr(one, name).double() * times[i])
            parts = torch.stack(parts)
            # fp32 sums of m terms in a tree of partial sums of at most m / 256 + 64 in turn
            tol = parts.abs().sum(0) * (m / 256 + 64) * A.E + 1e-5 * parts.abs().sum(0)
            assert ((getattr(back, name).double() - parts.sum(0)).abs() <= tol).all(), name


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("n", [2, 7, 9, 15, 127, 129, 505, 515, 1001, 4090, 8191, 8195, 16383])
def test_rows_that_end_inside_a_piece(pid, layers, dtype, n):
    """Every matrix between columns of NaN, total in x's place and dx in dtotal's: nothing of what is beside
    a row is taken or written."""
    def inside(t):
        big = torch.full((t.shape[0], n + 11), float("nan"), dtype=A.DT[dtype], device=DEV)
        big[:, 5:5 + n] = t.to(DEV)
        return big, big[:, 5:5 + n]

    def around_is_untouched(big):
        assert torch.isnan(big[:, :5]).all() and torch.isnan(big[:, 5 + n:]).all()

    for i, form in enumerate(FORMS):
        j = Joint(pid, dtype, 5, n, form, seed=i)
        (bx, x), (bo, o), (bdh, dh), (bdt, dt) = (inside(t) for t in (j.x, j.o, j.dh, j.dt))
        bh, h = inside(torch.zeros(5, n))
        got = pid.pointid_norm(layers, x, j.norm(), j.block(o), total=x, h=h if j.before else None, keep=True)
        j.check_forward(got, str(form))
        back = pid.pointid_norm_backward(layers, dh if j.before else None, x if j.before else None, got.stats, j.norm(),
                                         j.block(o), dtotal=dt, dx=dt)
        j.check_backward(back, got.stats.cpu(), got.total.cpu() if j.before else None, True, str(form))
        for big in (bx, bo, bdh, bdt, bh):
            around_is_untouched(big)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_a_norm_alone(pid, layers, dtype, kind):
    for m, n in ((1, 5), (40, 136), (3, 2500)):
        j = Joint(pid, dtype, m, n, (kind, None, True, False, 1.0, 0.0))
        got = pid.pointid_norm(layers, j.dev(j.x), j.norm(), keep=True)
        assert got.total is None
        u, tu, mean, r = A.norm64(kind, EPS, j.x.double(), torch.zeros((m, n), dtype=torch.float64))
        v, tol = A.affine64(u, tu, j.wb.double(), j.bb.double())
        A.near(got.h, v, A.rounded(v, tol, dtype), "h")
        back = pid.pointid_norm_backward(layers, j.dev(j.dh), j.dev(j.x), got.stats, j.norm())
        want = A.back64(j.dh.double(), j.x.double(), None, got.stats.double().cpu(), kind, None, j.wb.double(), None, None,
                        None, 1.0, None, None)
        for name in ("dx", "dweight", "dbias"):
            v, tol = want[name]
            A.near(getattr(back, name), v, A.rounded(v, tol, dtype if name == "dx" else "fp32"), name)
        assert back.dout is None and back.dgate is None and back.dblock_weight is None


@pytest.mark.parametrize("m, n", [(3, 40), (9000, 40), (5000, 264), (2500, 1200), (9000, 2050), (40, 9000)])
def test_only_what_is_asked_for(pid, layers, m, n):
    """Every output alone, over enough rows for each block to have several, is what it is with the
    others; and what is not there is nowhere written."""
    g = A.gen(m + n)
    x, o, dh, dt = (A.rand(g, m, n).to(DEV) for _ in range(4))
    w = torch.randn(n, generator=g).to(DEV)
    norm, block = pid.Norm("rms", w), pid.Block(o, pid.Norm("layer", w, w), w, 0.5, pid.Drop(0.1, 1))
    full = pid.pointid_norm(layers, x, norm, block, keep=True)
    M = [pid._Matrix(v.data_ptr(), n) for v in (x, torch.empty_like(x), torch.empty_like(x))]
    total, h = torch.empty_like(x), torch.empty_like(x)
    fields, end = pid._NormOf(*pid._norm(norm, "norm", n, 0)), pid._block(block, torch.bfloat16, x.shape, 0)
    stream = torch.cuda.current_stream().cuda_stream
    T, H = pid._Matrix(total.data_ptr(), n), pid._Matrix(h.data_ptr(), n)
    assert pid.lib.pointid_norm(layers.raw, 1, m, n, M[0], fields, end, None, H, None, stream) == pid.POINTID_OK
    assert pid.lib.pointid_norm(layers.raw, 1, m, n, M[0], None, end, T, None, None, stream) == pid.POINTID_OK
    assert torch.equal(total, full.total) and torch.equal(h, full.h)
    every = pid.pointid_norm_backward(layers, dh, full.total, full.stats, norm, block, dtotal=dt)
    outs = ("dx", "dout", "dweight", "dblock_weight", "dblock_bias", "dgate")
    made = {k: torch.empty_like(getattr(every, k)) for k in outs}
    for k in outs:
        grads = pid._NormGrads()
        setattr(grads, k, made[k].data_ptr())
        grads.ld_dx = grads.ld_dout = n
        assert pid.lib.pointid_norm_backward(layers.raw, 1, m, n, pid._Matrix(dh.data_ptr(), n),
                                             pid._Matrix(full.total.data_ptr(), n), full.stats.data_ptr(), fields, end,
                                             pid._Matrix(dt.data_ptr(), n), grads, None, 0, stream) == pid.POINTID_OK
        if k in ("dx", "dout"):
            assert torch.equal(made[k], getattr(every, k)), k
        else:
            # which sums a block keeps may change how many rows it takes, and so the order of the sums
            assert torch.allclose(made[k], getattr(every, k), rtol=1e-3, atol=1e-3 * m ** 0.5), k
    back = pid.pointid_norm_backward(layers, dh, full.total, full.stats, norm, block, dtotal=dt, need_dx=False)
    assert back.dx is None and torch.equal(back.dout, every.dout) and torch.equal(back.dgate, every.dgate)
    back = pid.pointid_norm_backward(layers, dh, full.total, full.stats, norm, block, dtotal=dt, need_dout=False)
    assert back.dout is None and torch.equal(back.dx, every.dx) and torch.equal(back.dweight, every.dweight)


def test_no_parameters(pid, layers):
    """weights and biases that are not given are ones and zeros, and have no gradients"""
    x, o = (torch.randn((20, 100), device=DEV) for _ in range(2))
    ones, zeros = torch.ones(100, device=DEV), torch.zeros(100, device=DEV)
    a = pid.pointid_norm(layers, x, pid.Norm("layer"), pid.Block(o, pid.Norm("layer")), keep=True)
    full = pid.Norm("layer", ones, zeros)
    b = pid.pointid_norm(layers, x, full, pid.Block(o, full, ones), keep=True)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    da = pid.pointid_norm_backward(layers, x, a.total, a.stats, pid.Norm("layer"), pid.Block(o, pid.Norm("layer")))
    db = pid.pointid_norm_backward(layers, x, a.total, a.stats, full, pid.Block(o, full, ones))
    assert torch.equal(da.dx, db.dx) and torch.equal(da.dout, db.dout) and all(v is None for v in da[2:])
    assert all(v is not None for v in db[2:])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [40, 83, 1200])
def test_pitches_offsets_and_in_place(pid, layers, dtype, n):
    m = 29
    j = Joint(pid, dtype, m, n, ("layer", "rms", True, True, 0.5, 0.25))
    plain = pid.pointid_norm(layers, j.dev(j.x), j.norm(), j.block(), keep=True)
    back = pid.pointid_norm_backward(layers, j.dev(j.dh), plain.total, plain.stats, j.norm(), j.block(), dtotal=j.dev(j.dt))
    j.check_forward(plain)

    def wide(t, shift):
        big = torch.full((m, n + 11), 7.0, dtype=t.dtype, device=DEV)
        big[:, shift:shift + n] = t
        return big

    for shift in (1, 3):
        x, o, total, h, dh, dt = (wide(t, shift) for t in (j.x, j.o, j.x, j.x, j.dh, j.dt))
        cut = slice(shift, shift + n)
        got = pid.pointid_norm(layers, x[:, cut], j.norm(), j.block(o[:, cut]), keep=True, total=total[:, cut], h=h[:, cut])
        j.check_forward(got, "pitched")
        for big in (total, h):
            assert (big[:, :shift] == 7).all() and (big[:, shift + n:] == 7).all()
        got = pid.pointid_norm(layers, x[:, cut], j.norm(), j.block(o[:, cut]), total=x[:, cut])      # in place
        j.check_forward(got, "in place")
        grads = pid.pointid_norm_backward(layers, dh[:, cut], plain.total, plain.stats, j.norm(), j.block(o[:, cut]),
                                          dtotal=dt[:, cut], dx=dt[:, cut])
        j.check_backward(grads, plain.stats.cpu(), plain.total.cpu(), what="in place")
        assert (dt[:, :shift] == 7).all() and (dt[:, shift + n:] == 7).all()
    assert torch.equal(back.dx, pid.pointid_norm_backward(layers, j.dev(j.dh), plain.total, plain.stats, j.norm(), j.block(),
                                                          dtotal=j.dev(j.dt), need_dout=False, need_params=False).dx)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_a_mean_far_from_zero(pid, layers, dtype):
    """A layer norm of rows whose mean is 200 times their deviation: the squares are of what is left."""
    for n in (100, 2048, 20000):
        j = Joint(pid, dtype, 6, n, ("layer", "layer", True, False, 1.0, 0.0), columns=lambda t: (t.double() + 200).to(t.dtype))
        j.check_forward(pid.pointid_norm(layers, j.dev(j.x), j.norm(), j.block()), f"n {n}")


def test_zeros_infinities_and_nans(pid, layers):
    x = torch.randn((6, 72), device=DEV)
    x[0] = 0
    x[1, 5] = math.inf
    x[2, 7] = math.nan
    h = pid.pointid_norm(layers, x, pid.Norm("rms")).h
    assert (h[0] == 0).all() and h[2].isnan().all() and h[1, 5].isnan() and (h[1, :5] == 0).all()
    good = pid.pointid_norm(layers, x[3:], pid.Norm("rms")).h
    assert torch.equal(h[3:], good)
    h = pid.pointid_norm(layers, x, pid.Norm("layer")).h
    assert (h[0] == 0).all() and h[1].isnan().all() and h[2].isnan().all() and torch.isfinite(h[3:]).all()


@pytest.mark.parametrize("n", [72, 9000])
def test_statistics_of_norms_that_are_not_there_are_not_read(pid, layers, n):
    for form, absent in ((("rms", None, False, True, 1.0, 0.0), slice(0, 2)), ((None, "layer", True, True, 1.0, 0.0), slice(2, 4))):
        j = Joint(pid, "bf16", 40, n, form)
        got = pid.pointid_norm(layers, j.dev(j.x), j.norm(), j.block(), keep=True)
        stats = got.stats.clone()
        stats[:, absent] = math.nan
        back = pid.pointid_norm_backward(layers, j.dev(j.dh) if j.before else None, got.total if j.before else None, stats,
                                         j.norm(), j.block(), dtotal=j.dev(j.dt))
        j.check_backward(back, got.stats.cpu(), got.total.cpu() if j.before else None, what=str(form))


@pytest.mark.parametrize("n", [8, 100, 2048, 9000, 20000])
def test_infinities_that_are_dropped(pid, layers, n):
    """A block's output that is an infinity or NaN where it is dropped: nothing of it arrives, nor in
    the gate's gradient."""
    m, p = 24, 0.5
    keep = A.drop_factor(m, n, p, 9, 4) > 0
    g = A.gen(n)
    x, dt = (torch.randn((m, n), generator=g).to(DEV) for _ in range(2))
    o = torch.randn((m, n), generator=g)
    bad = torch.where(keep, o, torch.where(torch.arange(n) % 2 == 0, math.nan, -math.inf))
    gate = torch.randn(n, generator=g).to(DEV)
    for norm in (None, pid.Norm("rms")):
        results = []
        for out in (o, bad):
            block = pid.Block(out.to(DEV), None, gate, 1.0, pid.Drop(p, 9, 4))
            got = pid.pointid_norm(layers, x, norm, block, keep=True)
            back = pid.pointid_norm_backward(layers, dt if norm else None, got.total if norm else None, got.stats, norm, block,
                                             dtotal=dt)
            results.append([got.total, back.dx, back.dout, back.dgate] + ([got.h] if norm else []))
        assert all(torch.equal(a, b) and torch.isfinite(a).all() for a, b in zip(*results))


def test_no_rows(pid, layers):
    x = torch.empty((0, 24), device=DEV)
    norm = pid.Norm("rms", torch.ones(24, device=DEV), torch.ones(24, device=DEV))
    got = pid.pointid_norm(layers, x, norm, pid.Block(x, norm, torch.ones(24, device=DEV)), keep=True)
    assert got.h.shape == got.total.shape == (0, 24)
    back = pid.pointid_norm_backward(layers, x, got.total, got.stats, norm, pid.Block(x, norm, torch.ones(24, device=DEV)))
    assert all((v == 0).all() and v.shape == (24,) for v in back[2:])


def test_the_same_bits(pid, layers):
    j = Joint(pid, "bf16", 3000, 1000, ("rms", "layer", True, True, 1.0, 0.1))
    got = pid.pointid_norm(layers, j.dev(j.x), j.norm(), j.block(), keep=True)
    args = (j.dev(j.dh), got.total, got.stats, j.norm(), j.block(), j.dev(j.dt))
    first = pid.pointid_norm_backward(layers, *args)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, pid.pointid_norm_backward(layers, *args)))
    # and a row's results do not depend on the others
    cut = pid.pointid_norm(layers, j.dev(j.x)[:5], j.norm(), j.block(j.dev(j.o)[:5]))
    assert torch.equal(cut.h, got.h[:5])


@pytest.mark.parametrize("m, n", [(5, 300), (700, 1031)])
def test_captured(pid, layers, m, n):
    """Two graphs, each with scratch of its own, replayed in turn with eager calls between."""
    j = [Joint(pid, "bf16", m, n, ("rms", "rms", True, True, 1.0, 0.1), seed=s) for s in (1, 2)]

    def step(k):
        got = pid.pointid_norm(layers, k.X, k.norm_, k.block_, keep=True)
        return (*got, *pid.pointid_norm_backward(layers, k.DH, got.total, got.stats, k.norm_, k.block_, dtotal=k.DT))

    runs = []
    for k in j:
        k.X, k.DH, k.DT, k.norm_, k.block_ = j[0].dev(k.x), k.dev(k.dh), k.dev(k.dt), k.norm(), k.block()
        want = [v.clone() for v in step(k)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(k)
        runs.append((graph, out, want))
    for _ in range(3):
        for graph, out, want in runs:
            for v in out:
                v.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want))
        assert all(torch.equal(a, b) for a, b in zip(step(j[0]), runs[0][2]))


def test_caller_scratch(pid, layers):
    """Memory of the caller's own: enough of it gives the same bits, too little is refused."""
    j = Joint(pid, "bf16", 500, 264, ("rms", None, False, False, 1.0, 0.0))
    x, dh, w = j.dev(j.x), j.dev(j.dh), j.dev(j.wb)
    stats = pid.pointid_norm(layers, x, j.norm(), keep=True).stats
    need = pid.lib.pointid_norm_backward_scratch(layers.raw, 500, 264)
    outs = []
    for scratch, size, status in ((None, 0, 0), (torch.empty(need, dtype=torch.uint8, device=DEV), need, 0),
                                  (torch.empty(need, dtype=torch.uint8, device=DEV), 16, pid.POINTID_EINVAL)):
        dx, dw = torch.zeros_like(x), torch.zeros(264, device=DEV)
        grads = pid._NormGrads(dx.data_ptr(), 264, None, 0, dw.data_ptr(), None, None, None, None)
        rc = pid.lib.pointid_norm_backward(layers.raw, 1, 500, 264, pid._Matrix(dh.data_ptr(), 264), pid._Matrix(x.data_ptr(), 264),
                                           stats.data_ptr(), pid._NormOf(1, EPS, w.data_ptr(), None), None, None, grads,
                                           scratch.data_ptr() if scratch is not None else None, size,
                                           torch.cuda.current_stream().cuda_stream)
        assert rc == status
        outs.append((dx, dw))
    assert all(torch.equal(a, b) for a, b in zip(outs[0], outs[1]))
    assert "scratch" in pid.pointid_last_error()


def test_rows_past_32_bits_of_elements(pid, layers):
    m, n = (1 << 20) + 3, 4096                                # past 2^32 elements
    x = torch.ones((m, n), dtype=torch.bfloat16, device=DEV)
    x[-2:, ::2] = -3
    w = torch.ones(n, device=DEV)
    got = pid.pointid_norm(layers, x, pid.Norm("layer", w), pid.Block(x, None, None, 1.0), keep=True)
    assert (got.h[:-2] == 0).all() and (got.total[-2:, 0] == -6).all()
    want = A.norm64("layer", EPS, x[-2:].double().cpu() * 2, torch.zeros((2, n), dtype=torch.float64))[0]
    assert (got.h[-2:].double().cpu() - want).abs().max() < 0.01
