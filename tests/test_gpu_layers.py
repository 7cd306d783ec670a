"""GPU: the layer operators against their definitions in 64 bits.

Tolerances, fixed from the arithmetic.  u is half a unit in the last place of the
result's type (2^-8 bf16, 2^-11 fp16, 2^-24 fp32) relative to a value, E = 2^-23.  A sum of
L terms in fp32 in any order is off by at most L E times the sum of magnitudes S (products
of 16-bit values are exact; the 6 products of fp32 parts count as 6 L).  An activation's
slope is at most 1.13, and it is computed to 3e-7 of max(1, |z|).  16-bit gradients
round dz once (u |dz|), or keep it in two parts.
"""

import ctypes
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
U = {name: torch.finfo(t).eps / 2 for name, t in DT.items()}
TINY = {"bf16": 2.0 ** -133, "fp16": 2.0 ** -25, "fp32": 2.0 ** -149}
E = 2.0 ** -23
ACTS = ["none", "relu", "silu", "gelu", "sigmoid"]


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


# ---- the definitions in 64 bits

def act64(name, z):
    return {"none": lambda: z, "relu": lambda: torch.where(z <= 0, torch.zeros_like(z), z),
            "silu": lambda: z * torch.sigmoid(z), "gelu": lambda: z * torch.special.ndtr(z),
            "sigmoid": lambda: torch.sigmoid(z)}[name]()


def slope64(name, z):
    s = torch.sigmoid(z)
    return {"none": lambda: torch.ones_like(z), "relu": lambda: (z > 0).double(),
            "silu": lambda: s * (1 + z * (1 - s)),
            "gelu": lambda: torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi),
            "sigmoid": lambda: s * (1 - s)}[name]()


def e4m3_grid():
    """The 256 codes' values."""
    c = torch.arange(256)
    e, f = (c >> 3) & 15, (c & 7).double()
    v = torch.where(e == 0, f / 8 * 2.0 ** -6, (1 + f / 8) * torch.pow(2.0, (e - 7).double()))
    v[127] = v[255] = float("nan")
    return torch.where(c >= 128, -v, v)


def checkpoint64(x):
    """(codes, exponents, values) of a finite matrix x, each code by search for the nearest value
    (an even code on a tie)."""
    x = x.double().cpu()
    m, n = x.shape
    nb = -(-n // 32)
    pad = torch.nn.functional.pad(x, (0, nb * 32 - n)).view(m, nb, 32)
    top = pad.abs().amax(2)
    p = torch.zeros_like(top, dtype=torch.int64)
    for i, j in (top > 0).nonzero().tolist():
        k = min(126, math.floor(math.log2(448 / top[i, j].item())) + 1)
        while top[i, j].item() * 2.0 ** k > 448:
            k -= 1
        p[i, j] = min(k, 126)
    scaled = (pad * torch.pow(2.0, p.double()).unsqueeze(2)).view(m, -1)[:, :n]
    mags = e4m3_grid()[:127]
    hi = torch.searchsorted(mags, scaled.abs().contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    dh, dl = (mags[hi] - scaled.abs()).abs(), (mags[lo] - scaled.abs()).abs()
    code = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    cols = torch.arange(n) // 32
    values = mags[code] * torch.pow(2.0, -p.double())[:, cols] * torch.where(scaled < 0, -1.0, 1.0)
    code = code + 128 * torch.signbit(scaled)
    return code.to(torch.uint8), (127 - p).to(torch.uint8), values


def rand(g, *shape, dtype="bf16", scale=1.0):
    return (torch.randn(shape, generator=g, dtype=torch.float64) * scale).to(DT[dtype])


def dev(t):
    return None if t is None else t.to(DEV)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def near(got, want, tol, what):
    got = got.detach().double().cpu()
    assert got.shape == want.shape, what
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, e.g. at " \
        f"{bad.nonzero()[0].tolist()}: {got[bad][0].item()} for {want[bad][0].item()}, tolerance {tol[bad][0].item()}"


def sums(a, b, dtype):
    """(a @ b, the bound of its fp32 error) in 64 bits"""
    a, b = a.double(), b.double()
    terms = a.shape[1] * (6 if dtype == "fp32" else 1) + 8
    return a @ b, (a.abs() @ b.abs()) * terms * E


def act_tol(z, tz):
    return 1.13 * tz + 3e-7 * z.abs().clamp(min=1)


SIZES = [(1, 1, 1), (1, 7, 3), (1, 130, 129), (2, 64, 64), (3, 100, 77), (5, 33, 8), (8, 1024, 300), (9, 16, 100),
         (31, 64, 31), (64, 128, 128), (65, 72, 136), (130, 257, 66), (257, 320, 264), (300, 96, 520)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m, k, n", SIZES)
def test_dense(pid, layers, dtype, m, k, n):
    g = gen(m * 1000003 + k * 1009 + n)
    x, w = rand(g, m, k, dtype=dtype), rand(g, k, n, dtype=dtype, scale=k ** -0.5)
    b, r = torch.randn(n, generator=g), rand(g, m, n, dtype=dtype)
    z, tz = sums(x, w, dtype)
    for i, act in enumerate(ACTS):
        bias, res = i % 2 == 0, i % 3 != 1
        zz = z + b.double() if bias else z
        tt = tz + (b.abs().double() * 2 * E if bias else 0) + zz.abs() * E
        want = act64(act, zz)
        tol = act_tol(zz, tt)
        if res:
            want = want + r.double()
            tol = tol + want.abs() * E
        save = torch.empty((m, n), dtype=DT[dtype], device=DEV) if i % 2 else None
        y = pid.pointid_dense(layers, dev(x), dev(w), dev(b) if bias else None, act, dev(r) if res else None, save=save)
        near(y, want, tol + want.abs() * U[dtype] + TINY[dtype], f"y {act}")
        if save is not None:
            near(save, zz, tt + zz.abs() * U[dtype] + TINY[dtype], f"z {act}")


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m, k, n", SIZES)
def test_gated(pid, layers, dtype, m, k, n):
    g = gen(m * 1000003 + k * 1009 + n + 1)
    x = rand(g, m, k, dtype=dtype)
    wg, wu = (rand(g, k, n, dtype=dtype, scale=k ** -0.5) for _ in range(2))
    bg, bu = (torch.randn(n, generator=g) for _ in range(2))
    (zg, tg), (zu, tu) = sums(x, wg, dtype), sums(x, wu, dtype)
    for i, act in enumerate(ACTS):
        bias = i % 2 == 0
        G, U_ = (zg + bg.double(), zu + bu.double()) if bias else (zg, zu)
        eg, eu = (t + v.abs() * 2 * E + bb.abs().double() * 2 * E for t, v, bb in ((tg, G, bg), (tu, U_, bu)))
        a, ta = act64(act, G), act_tol(G, eg)
        want = a * U_
        tol = a.abs() * eu + (U_.abs() + eu) * ta + want.abs() * E
        sg, su = (torch.empty((m, n), dtype=DT[dtype], device=DEV) for _ in range(2)) if i % 2 else (None, None)
        h = pid.pointid_gated(layers, dev(x), dev(wg), dev(wu), dev(bg) if bias else None, dev(bu) if bias else None, act,
                              save_g=sg, save_u=su)
        near(h, want, tol + want.abs() * U[dtype] + TINY[dtype], f"h {act}")
        if sg is not None:
            near(sg, G, eg + G.abs() * U[dtype] + TINY[dtype], "g")
            near(su, U_, eu + U_.abs() * U[dtype] + TINY[dtype], "u")


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("n", [8, 9, 15, 255, 256, 257, 259, 260, 263, 264, 513, 1031])
def test_few_rows_at_the_edges_of_their_strips(pid, layers, dtype, n):
    """Widths that end a few columns into the streaming kernel's strip of 256."""
    g = gen(n)
    for m in (1, 2, 7):
        k = 90
        x, w, w2 = rand(g, m, k, dtype=dtype), rand(g, k, n, dtype=dtype), rand(g, k, n, dtype=dtype)
        z, tz = sums(x, w, dtype)
        z2, tz2 = sums(x, w2, dtype)
        y = pid.pointid_dense(layers, dev(x), dev(w))
        near(y, z, tz + z.abs() * U[dtype] + TINY[dtype], "y")
        h = pid.pointid_gated(layers, dev(x), dev(w), dev(w2), act="none")
        want = z * z2
        near(h, want, z.abs() * tz2 + (z2.abs() + tz2) * tz + want.abs() * (U[dtype] + E) + TINY[dtype], "h")


def kept(pid, v, eight):
    """(what is handed over, its values in 64 bits)"""
    if not eight:
        return dev(v), v.double()
    code, e, values = checkpoint64(v)
    return pid.Checkpoint(dev(code), dev(e)), values


def gradient_tol(dz, tdz, dtype, exact):
    """dz's own error, and its rounding for the products"""
    return tdz if exact or dtype == "fp32" else tdz + dz.abs() * U[dtype] + TINY[dtype]


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m, k, n", [(1, 1, 1), (1, 64, 40), (3, 100, 77), (31, 64, 31), (65, 72, 136), (130, 257, 66),
                                     (257, 320, 264), (600, 24, 300)])
def test_dense_backward(pid, layers, dtype, m, k, n, eight):
    g = gen(m * 1000003 + k * 1009 + n + 2)
    dy, w = rand(g, m, n, dtype=dtype), rand(g, k, n, dtype=dtype, scale=k ** -0.5)
    x, x64 = kept(pid, rand(g, m, k, dtype=dtype), eight)
    z, z64 = kept(pid, rand(g, m, n, dtype=dtype), eight)
    for act in ACTS:
        s = slope64(act, z64)
        dz = dy.double() * s
        tdz = dy.abs().double() * (1e-6 * z64.abs().clamp(min=1)) + dz.abs() * E if act not in ("none", "relu") else dz * 0
        te = gradient_tol(dz, tdz, dtype, act in ("none", "relu"))
        dx, dw, db = pid.pointid_dense_backward(layers, dev(dy), x, dev(w), None if act == "none" else z, act)
        for got, a, b_, ta, tb, name in ((dx, dz, w.double().t(), te, None, "dx"), (dw, x64.t(), dz, None, te, "dw")):
            want, tol = sums(a, b_, dtype)
            tol = tol + (ta @ b_.abs() if ta is not None else a.abs() @ tb)
            near(got, want, tol + want.abs() * U[dtype] + TINY[dtype], f"{name} {act}")
        near(db, dz.sum(0), tdz.sum(0) + dz.abs().sum(0) * (m + 2) * E + 1e-30, f"db {act}")


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m, k, n", [(1, 1, 1), (1, 64, 40), (3, 100, 77), (65, 72, 136), (130, 257, 66), (300, 320, 264)])
def test_gated_backward(pid, layers, dtype, m, k, n, eight):
    g = gen(m * 1000003 + k * 1009 + n + 3)
    dh = rand(g, m, n, dtype=dtype)
    wg, wu = (rand(g, k, n, dtype=dtype, scale=k ** -0.5) for _ in range(2))
    x, x64 = kept(pid, rand(g, m, k, dtype=dtype), eight)
    G, g64 = kept(pid, rand(g, m, n, dtype=dtype), eight)
    V, u64 = kept(pid, rand(g, m, n, dtype=dtype), eight)
    d = dh.double()
    for act in ACTS:
        dg, du = d * u64 * slope64(act, g64), d * act64(act, g64)
        tg = (d * u64).abs() * (1e-6 * g64.abs().clamp(min=1)) + dg.abs() * 3 * E
        tu = d.abs() * (3e-7 * g64.abs().clamp(min=1)) + du.abs() * E
        eg, eu = gradient_tol(dg, tg, dtype, False), gradient_tol(du, tu, dtype, False)
        dx, dwg, dwu, dbg, dbu = pid.pointid_gated_backward(layers, dev(dh), x, dev(wg), dev(wu), G, V, act, need_db=True)
        a, ta = sums(dg, wg.double().t(), dtype)
        b_, tb = sums(du, wu.double().t(), dtype)
        want = a + b_
        near(dx, want, 2 * (ta + tb) + eg @ wg.abs().double().t() + eu @ wu.abs().double().t() + want.abs() * U[dtype] +
             TINY[dtype], f"dx {act}")
        for got, v, e_, name in ((dwg, dg, eg, "dwg"), (dwu, du, eu, "dwu")):
            want, tol = sums(x64.t(), v, dtype)
            near(got, want, tol + x64.abs().t() @ e_ + want.abs() * U[dtype] + TINY[dtype], f"{name} {act}")
        near(dbg, dg.sum(0), tg.sum(0) + dg.abs().sum(0) * (m + 2) * E + 1e-30, "dbg")
        near(dbu, du.sum(0), tu.sum(0) + du.abs().sum(0) * (m + 2) * E + 1e-30, "dbu")


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_few_values_keep_the_gradient_in_two_parts(pid, layers, dtype):
    """dz of few values is not rounded to 16 bits before the products: dx is off by the
    rounding of the result alone (and fp32 sums)."""
    g = gen(77)
    m, k, n = 2, 512, 640
    dy, w, z = rand(g, m, n, dtype=dtype), rand(g, k, n, dtype=dtype), rand(g, m, n, dtype=dtype)
    x = rand(g, m, k, dtype=dtype)
    dz = dy.double() * slope64("silu", z.double())
    dx, dw, _ = pid.pointid_dense_backward(layers, dev(dy), dev(x), dev(w), dev(z), "silu")
    want, tol = sums(dz, w.double().t(), dtype)
    rest = dz.abs() * (U[dtype] ** 2 + 1e-6) + TINY[dtype]
    near(dx, want, tol + rest @ w.abs().double().t() + want.abs() * U[dtype] + TINY[dtype], "dx")
    want, tol = sums(x.double().t(), dz, dtype)
    near(dw, want, tol + x.abs().double().t() @ rest + want.abs() * U[dtype] + TINY[dtype], "dw")


@pytest.mark.parametrize("act", ACTS)
def test_gradients_against_differences(pid, layers, act):
    """The fp32 gradients of sum(c * layer) along random directions against central
    differences of the 64-bit definition."""
    g = gen(ACTS.index(act) + 500)
    m, k, n = 40, 50, 60
    x, wg, wu = rand(g, m, k, dtype="fp32"), rand(g, k, n, dtype="fp32", scale=0.15), rand(g, k, n, dtype="fp32", scale=0.15)
    bg, bu, c = torch.randn(n, generator=g), torch.randn(n, generator=g), rand(g, m, n, dtype="fp32")
    a = [t.double() for t in (x, wg, wu, bg, bu)]

    def dense(x, w, _, b, __):
        return (c.double() * act64(act, x @ w + b)).sum()

    def gated(x, wg, wu, bg, bu):
        return (c.double() * act64(act, x @ wg + bg) * (x @ wu + bu)).sum()

    z = torch.empty((m, n), device=DEV)
    pid.pointid_dense(layers, dev(x), dev(wg), dev(bg), act, save=z)
    dx, dw, db = pid.pointid_dense_backward(layers, dev(c), dev(x), dev(wg), z, act)
    G, V = torch.empty((m, n), device=DEV), torch.empty((m, n), device=DEV)
    pid.pointid_gated(layers, dev(x), dev(wg), dev(wu), dev(bg), dev(bu), act, save_g=G, save_u=V)
    q = pid.pointid_gated_backward(layers, dev(c), dev(x), dev(wg), dev(wu), G, V, act, need_db=True)
    for f, grads in ((dense, (dx, dw, None, db, None)), (gated, q[:3] + q[3:])):
        for i, grad in enumerate(grads):
            if grad is None:
                continue
            for _ in range(3):
                d = torch.randn(a[i].shape, generator=g, dtype=torch.float64)
                # relu: a step that turns no sign between it and the point
                h = 1e-6
                up, down = list(a), list(a)
                up[i], down[i] = a[i] + h * d, a[i] - h * d
                slope = (f(*up) - f(*down)) / (2 * h)
                got = (grad.double().cpu() * d).sum()
                size = (grad.double().cpu() * d).norm() + 1
                assert abs(got - slope) <= 1e-4 * size, (f.__name__, i, got, slope)


def pitched(t, pad, shift, device=DEV):
    """t on the device as a view with a longer pitch, `shift` elements off the alignment"""
    m, n = t.shape
    flat = torch.full((m * (n + pad) + shift + 8,), float("nan"), dtype=t.dtype, device=device)
    v = flat[shift:shift + m * (n + pad)].view(m, n + pad)[:, :n]
    v.copy_(t)
    return v, flat


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m, k, n, pad, shift", [(2, 72, 40, 5, 3), (70, 72, 40, 8, 8), (70, 72, 40, 8, 1), (70, 72, 40, 3, 0),
                                                 (130, 65, 131, 7, 5), (7, 64, 136, 16, 4)])
def test_views(pid, layers, dtype, m, k, n, pad, shift):
    """Pitched, shifted operands and outputs (NaN between the rows): the bits of the
    contiguous call's, and nothing written beside the rows."""
    g = gen(m + k + n + pad)
    x, w, w2, r = (rand(g, *s, dtype=dtype) for s in ((m, k), (k, n), (k, n), (m, n)))
    v = [pitched(t, pad, shift)[0] for t in (x, w, w2, r)]

    def out(rows, cols):
        return pitched(torch.zeros((rows, cols), dtype=DT[dtype]), pad, shift)

    (y, y_all), (z, z_all) = out(m, n), out(m, n)
    pid.pointid_dense(layers, v[0], v[1], None, "gelu", v[3], y=y, save=z)
    z0 = torch.empty((m, n), dtype=DT[dtype], device=DEV)
    y0 = pid.pointid_dense(layers, dev(x), dev(w), None, "gelu", dev(r), save=z0)
    near(y, y0.double().cpu(), y0.abs().double().cpu() * 2 * U[dtype] + 1e-5, "y")
    near(z, z0.double().cpu(), z0.abs().double().cpu() * 2 * U[dtype] + 1e-4, "z")
    for whole, rows, cols in ((y_all, m, n), (z_all, m, n)):
        assert int(whole.isnan().sum()) == whole.numel() - rows * cols
    # the residual may be the output itself
    pid.pointid_dense(layers, v[0], v[1], None, "gelu", v[3], y=v[3])
    assert torch.equal(v[3], y)
    h, h0 = pid.pointid_gated(layers, v[0], v[1], v[2]), pid.pointid_gated(layers, dev(x), dev(w), dev(w2))
    near(h, h0.double().cpu(), h0.abs().double().cpu() * 2 * U[dtype] + 1e-3, "h")
    # the weights of a gated layer as the halves of one matrix
    both = torch.cat([w, w2], 1).to(DEV)
    h1 = pid.pointid_gated(layers, dev(x), both[:, :n], both[:, n:])
    near(h1, h0.double().cpu(), h0.abs().double().cpu() * 2 * U[dtype] + 1e-3, "h of halves")
    got = pid.pointid_gated_backward(layers, v[3], v[0], v[1], v[2], y, z)
    want = pid.pointid_gated_backward(layers, v[3].contiguous(), dev(x), dev(w), dev(w2), y.contiguous(), z.contiguous())
    for a, b in zip(got[:3], want[:3]):
        near(a, b.double().cpu(), b.abs().double().cpu() * 2 * U[dtype] + 1e-2 * (U[dtype] * 512), "gradients")


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_checkpoint_is_the_definition(pid, dtype):
    g = gen(9)
    top = {"bf16": 3.3895313892515355e38, "fp16": 65504.0, "fp32": 3.4028234663852886e38}[dtype]
    least = {"bf16": 2.0 ** -133, "fp16": 2.0 ** -24, "fp32": 2.0 ** -149}[dtype]
    for m, n in ((1, 1), (3, 31), (2, 32), (5, 33), (7, 100), (2, 257)):
        x = rand(g, m, n, dtype=dtype) * torch.exp(2 * torch.randn((m, 1), generator=g)).to(DT[dtype])
        if n >= 31:
            x[0, :32] = 0                                          # a block of zeros
            x[-1, 0:5] = torch.tensor([448, 447, 449, 16.5, 17.0], dtype=torch.float64).to(DT[dtype])      # ties, the limit
            if m > 2:
                x[1, :] *= torch.tensor(least * 64, dtype=torch.float64).to(DT[dtype]) if dtype != "fp16" else 2.0 ** -14
                x[1, 3], x[1, 4] = top, -top
        code, e, values = checkpoint64(x)
        c = pid.pointid_checkpoint_save(dev(x))
        assert torch.equal(c.exponents.cpu(), e), (m, n)
        assert torch.equal(c.codes.cpu(), code), (m, n)
        got = pid.pointid_checkpoint_load(c, DT[dtype])
        assert torch.equal(got.cpu(), values.to(DT[dtype])), (m, n)
        assert torch.equal(pid.pointid_checkpoint_load(c, torch.float32).cpu(), values.float())
        # the same from a pitched, shifted matrix, into one
        v, whole = pitched(x, 3, 1)
        c2 = pid.pointid_checkpoint_save(v)
        assert torch.equal(c2.codes, c.codes) and torch.equal(c2.exponents, c.exponents)
        o, whole = pitched(torch.zeros_like(x), 3, 1)
        pid.pointid_checkpoint_load(c, out=o)
        assert torch.equal(o, got) and int(whole.isnan().sum()) == whole.numel() - m * n


def test_checkpoint_of_what_is_not_finite(pid):
    x = torch.ones((2, 70))
    x[0, 1], x[0, 2], x[0, 40], x[1, :] = float("inf"), float("nan"), -float("inf"), float("nan")
    c = pid.pointid_checkpoint_save(dev(x))
    got = pid.pointid_checkpoint_load(c, torch.float32).cpu()
    assert torch.equal(got.isnan(), ~x.isfinite())
    assert torch.equal(got[0][x[0].isfinite()], x[0][x[0].isfinite()])


@pytest.mark.parametrize("m, k, n", [(1, 64, 70), (6, 72, 100), (40, 72, 96), (300, 264, 100), (20, 4096, 64)])
def test_checkpoints_written_by_the_layers(pid, layers, m, k, n):
    """Codes written in the epilogue (and where a split sum is joined): the values of the
    checkpoint of z, one code off at most where z in fp32 falls beside a rounding limit."""
    g = gen(m + n)
    x, wg, wu = rand(g, m, k), rand(g, k, n, scale=k ** -0.5), rand(g, k, n, scale=k ** -0.5)
    for name, call in (("dense", lambda c: pid.pointid_dense(layers, dev(x), dev(wg), act="silu", save=c)),
                       ("gated", lambda c: pid.pointid_gated(layers, dev(x), dev(wg), dev(wu), save_g=c)),
                       ("gated u", lambda c: pid.pointid_gated(layers, dev(x), dev(wu), dev(wg), save_u=c))):
        c = pid.Checkpoint.empty(m, n, DEV)
        call(c)
        z, tz = sums(x, wg, "bf16")
        _, e, values = checkpoint64(z)
        got = pid.pointid_checkpoint_load(c, torch.float32).double().cpu()
        step = torch.pow(2.0, (127 - c.exponents.cpu().double()).neg())[:, torch.arange(n) // 32] * 2.0 ** -9
        near(got, z, z.abs() / 16 * 1.01 + step + tz, name)
        assert (got != values).double().mean() < 0.01, name
        assert (c.exponents.cpu() != e).double().mean() < 0.05, name


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_step_from_checkpoints(pid, layers, dtype):
    """A gated layer's training step with g, u and x kept in 8 bits: the gradients of the
    definition at the values that the checkpoints stand for."""
    g = gen(31)
    m, k, n = 150, 200, 168
    x, dh = rand(g, m, k, dtype=dtype), rand(g, m, n, dtype=dtype)
    wg, wu = (rand(g, k, n, dtype=dtype, scale=k ** -0.5) for _ in range(2))
    G, V = (pid.Checkpoint.empty(m, n, DEV) for _ in range(2))
    pid.pointid_gated(layers, dev(x), dev(wg), dev(wu), save_g=G, save_u=V)
    X = pid.pointid_checkpoint_save(dev(x))
    dx, dwg, dwu, _, _ = pid.pointid_gated_backward(layers, dev(dh), X, dev(wg), dev(wu), G, V)
    g64, u64, x64 = (pid.pointid_checkpoint_load(c, torch.float32).double().cpu() for c in (G, V, X))
    d = dh.double()
    dg, du = d * u64 * slope64("silu", g64), d * act64("silu", g64)
    for got, want, size in ((dx, dg @ wg.double().t() + du @ wu.double().t(), None), (dwg, x64.t() @ dg, None),
                            (dwu, x64.t() @ du, None)):
        err = (got.double().cpu() - want).norm() / want.norm()
        assert err <= 2 * U[dtype], err


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m, k, n", [(200, 92928, 128), (64, 20000, 72), (3, 50000, 96), (12, 30001, 40)])
def test_long_sums(pid, layers, dtype, m, k, n):
    """Sums split over blocks and joined; the gradient of the weights over as many rows."""
    g = gen(k)
    x, w = rand(g, m, k, dtype=dtype), rand(g, k, n, dtype=dtype, scale=k ** -0.5)
    b = torch.randn(n, generator=g)
    xd, wd = dev(x), dev(w)
    z = xd.double() @ wd.double() + dev(b).double()
    # random signs: the errors of a sum of magnitude S add up like sqrt(terms)
    tol = (8 * math.sqrt(6 * k if dtype == "fp32" else k) * E * math.sqrt(2 / math.pi) * 4 + E) * torch.ones_like(z)
    y = pid.pointid_dense(layers, xd, wd, dev(b), "relu")
    want = z.clamp(min=0)
    near(y, want.cpu(), (tol + want.abs() * U[dtype]).cpu() + TINY[dtype], "y")
    dy, z8 = rand(g, k, n, dtype=dtype), torch.ones((k, n), dtype=DT[dtype])
    xt = xd.t().contiguous()                              # k rows of m columns
    _, dw, db = pid.pointid_dense_backward(layers, dev(dy), xt, torch.zeros((m, n), dtype=DT[dtype], device=DEV), dev(z8),
                                           "relu", need_dx=False)
    want = xd.double() @ dev(dy).double()
    err = (dw.double() - want).norm() / want.norm()
    assert err <= 1.05 * U[dtype] + 2e-6, err
    want = dev(dy).double().sum(0)
    near(db, want.cpu(), torch.full((n,), 16 * math.sqrt(k) * E * 4, dtype=torch.float64), "db")


def test_needs(pid, layers):
    """Each output alone has the bits it has among the others, and asks for its inputs only."""
    g = gen(4)
    m, k, n = 90, 100, 110
    dy, x, w, z = rand(g, m, n), rand(g, m, k), rand(g, k, n), rand(g, m, n)
    dy, x, w, z = map(dev, (dy, x, w, z))
    dx, dw, db = pid.pointid_dense_backward(layers, dy, x, w, z, "gelu")
    a, b, c = pid.pointid_dense_backward(layers, dy, None, w, z, "gelu", need_dw=False, need_db=False)
    assert b is None and c is None and torch.equal(a, dx)
    a, b, c = pid.pointid_dense_backward(layers, dy, x, w, z, "gelu", need_dx=False, need_db=False)
    assert a is None and c is None and torch.equal(b, dw)
    a, b, c = pid.pointid_dense_backward(layers, dy, None, w, z, "gelu", need_dx=False, need_dw=False)
    assert torch.equal(c, db)
    # no activation: z is not read
    dx, dw, db = pid.pointid_dense_backward(layers, dy, x, w)
    a, b, c = pid.pointid_dense_backward(layers, dy, x, w, z, "none", need_db=False)
    assert torch.equal(a, dx) and torch.equal(b, dw) and c is None
    with pytest.raises(pid.PointIdError) as e:
        pid.pointid_dense_backward(layers, dy, x, w, None, "relu")
    assert e.value.status == pid.POINTID_EINVAL


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_no_rows(pid, layers, dtype):
    x, w = torch.empty((0, 40), dtype=DT[dtype], device=DEV), torch.ones((40, 24), dtype=DT[dtype], device=DEV)
    assert pid.pointid_dense(layers, x, w).shape == (0, 24)
    assert pid.pointid_gated(layers, x, w, w).shape == (0, 24)
    e = torch.empty((0, 24), dtype=DT[dtype], device=DEV)
    dx, dw, db = pid.pointid_dense_backward(layers, e, x, w, e, "relu")
    assert dx.shape == (0, 40) and not dw.any() and not db.any() and dw.shape == (40, 24)
    q = pid.pointid_gated_backward(layers, e, x, w, w, e, e, need_db=True)
    assert all(not t.any() for t in q[1:])
    c = pid.pointid_checkpoint_save(e)
    assert pid.pointid_checkpoint_load(c, DT[dtype]).shape == (0, 24)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("m", [3, 70])
def test_infinities_and_nans(pid, layers, dtype, m):
    """They come out where fp32 arithmetic has them, and nowhere else."""
    g = gen(12)
    k, n = 80, 96
    x, w = rand(g, m, k, dtype=dtype), rand(g, k, n, dtype=dtype)
    x[0, 3], x[1, 5], x[2, 7] = float("inf"), float("nan"), -float("inf")
    w[9, 11], w[10, 13] = float("inf"), float("nan")
    z = x.double() @ w.double()
    y = pid.pointid_dense(layers, dev(x), dev(w)).double().cpu()
    assert torch.equal(y.isnan(), z.isnan())
    assert torch.equal(y.isinf(), z.isinf()) and torch.equal(y[z.isinf()], z[z.isinf()])
    y = pid.pointid_dense(layers, dev(x), dev(w), act="relu").double().cpu()
    assert torch.equal(y.isnan(), z.isnan()) and (y[z == -float("inf")] == 0).all()
    # a gradient that relu stops does not reach the products
    dy = torch.zeros((m, n), dtype=DT[dtype])
    dy[0, 0] = float("inf")
    zz = torch.full((m, n), -1.0, dtype=DT[dtype])
    dx, dw, db = pid.pointid_dense_backward(layers, dev(dy), dev(rand(g, m, k, dtype=dtype)), dev(rand(g, k, n, dtype=dtype)),
                                            dev(zz), "relu")
    assert not dx.any() and not dw.any() and not db.any()


def test_fp16_overflows_to_infinity(pid, layers):
    x, w = torch.full((70, 64), 200.0, dtype=torch.float16, device=DEV), torch.full((64, 40), 200.0, dtype=torch.float16, device=DEV)
    assert pid.pointid_dense(layers, x, w).isinf().all()


def test_rows_past_32_bit_offsets(pid, layers):
    """Rows of a long, wide buffer: offsets past 2^31 elements."""
    m, k, n, pitch = 70000, 64, 72, 40000
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("not enough device memory")
    big = torch.empty((m, pitch), dtype=torch.bfloat16, device=DEV)
    x = big[:, :k]
    y = big[:, 1024:1024 + n]
    g = torch.Generator(device=DEV).manual_seed(3)
    x.copy_(torch.randn((m, k), generator=g, device=DEV))
    w = torch.randn((k, n), generator=g, device=DEV).bfloat16()
    pid.pointid_dense(layers, x, w, act="relu", y=y)
    want = (x.float() @ w.float()).clamp(min=0)
    assert ((y.float() - want).norm() / want.norm()).item() <= 2 ** -9
    dx, dw, _ = pid.pointid_dense_backward(layers, y, x, w)
    want = x.double().t() @ y.double()
    assert ((dw.double() - want).norm() / want.norm()).item() <= 2 ** -9
    want = y.float() @ w.float().t()
    assert ((dx.float() - want).norm() / want.norm()).item() <= 2 ** -9


def test_a_pitch_past_the_products_reach(pid, layers):
    m, k, n, pitch = 20, 64, 72, (1 << 21) + 8
    g = torch.Generator(device=DEV).manual_seed(4)
    for dtype in (torch.bfloat16, torch.float32):
        x = torch.empty((m, pitch), dtype=dtype, device=DEV)[:, :k]
        x.copy_(torch.randn((m, k), generator=g, device=DEV))
        w = torch.randn((k, n), generator=g, device=DEV).to(dtype)
        assert torch.equal(pid.pointid_dense(layers, x, w), pid.pointid_dense(layers, x.contiguous(), w))


def test_same_bits_on_any_stream(pid, layers):
    """Calls on two streams at once, sharing the scratch cache, with inputs that each
    stream is still making: the bits of the calls alone."""
    g = torch.Generator(device=DEV).manual_seed(5)
    cases = []
    for m, k, n in ((4, 4096, 512), (200, 3000, 120), (64, 8192, 128), (333, 555, 77)):
        x = torch.randn((m, k), generator=g, device=DEV).bfloat16()
        w = torch.randn((k, n), generator=g, device=DEV).bfloat16()
        dy = torch.randn((m, n), generator=g, device=DEV).bfloat16()
        alone = [pid.pointid_dense(layers, x, w, act="gelu")] + list(pid.pointid_dense_backward(layers, dy, x, w, dy, "silu"))
        cases.append((x, w, dy, alone))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for turn in range(6):
        for i, (x, w, dy, alone) in enumerate(cases):
            s = streams[(turn + i) % 2]
            with torch.cuda.stream(s):
                x2 = (x.float() * 1).bfloat16()
                got.append((alone, [pid.pointid_dense(layers, x2, w, act="gelu")] +
                            list(pid.pointid_dense_backward(layers, dy, x2, w, dy, "silu"))))
    torch.cuda.synchronize()
    for want, have in got:
        assert all(torch.equal(a, b) for a, b in zip(want, have))
    assert pid.pointid_layers_trim(layers, 0) == 0


def test_capture(pid, layers):
    """A call without scratch goes into a graph; one that takes scratch refuses."""
    g = torch.Generator(device=DEV).manual_seed(6)
    x = torch.randn((512, 256), generator=g, device=DEV).bfloat16()
    w = torch.randn((256, 4096), generator=g, device=DEV).bfloat16()
    y = torch.empty((512, 4096), dtype=torch.bfloat16, device=DEV)
    odd = torch.randn((255, 33), generator=g, device=DEV).bfloat16()
    graph = torch.cuda.CUDAGraph()
    refused = None
    with torch.cuda.graph(graph):
        pid.pointid_dense(layers, x, w, act="relu", y=y)
        try:
            pid.pointid_dense(layers, x[:, :255], odd)
        except pid.PointIdError as e:
            refused = e
    assert refused is not None and refused.status == pid.POINTID_EINVAL and "captured" in str(refused)
    for i in range(4):
        x.copy_(torch.randn((512, 256), generator=g, device=DEV))
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, pid.pointid_dense(layers, x, w, act="relu"))
        torch.cuda.synchronize()


def test_refusals_on_the_device(pid, layers):
    x, w = torch.ones((4, 8), dtype=torch.bfloat16, device=DEV), torch.ones((8, 16), dtype=torch.bfloat16, device=DEV)
    for bad in (dict(bias=torch.ones(16, dtype=torch.bfloat16, device=DEV)), dict(bias=torch.ones(15, device=DEV)),
                dict(residual=torch.ones((4, 16), device=DEV)), dict(y=torch.ones((4, 17), dtype=torch.bfloat16, device=DEV)),
                dict(y=torch.ones((16, 4), dtype=torch.bfloat16, device=DEV).t()),
                dict(residual=torch.ones((1, 16), dtype=torch.bfloat16, device=DEV).expand(4, 16)),
                dict(save=pid.Checkpoint.empty(4, 15, DEV))):
        with pytest.raises((TypeError, ValueError)):
            pid.pointid_dense(layers, x, w, **bad)
    closed = pid.pointid_layers_create(0)
    closed.close()
    with pytest.raises(ValueError):
        pid.pointid_dense(closed, x, w)
    with pytest.raises(pid.PointIdError) as e:
        pid.pointid_layers_create(4096)
    assert e.value.status == pid.POINTID_ENODEV


def test_timing_names(pid, layers):
    x, w = torch.ones((4, 4096), dtype=torch.bfloat16, device=DEV), torch.ones((4096, 64), dtype=torch.bfloat16, device=DEV)
    pid.pointid_timing_reset()
    pid.pointid_timing_enable(True)
    try:
        pid.pointid_dense(layers, x, w)
        torch.cuda.synchronize()
        assert pid.pointid_timing_query("layers_product")[1] == 1 and pid.pointid_timing_query("layers_join")[1] == 1
    finally:
        pid.pointid_timing_enable(False)
        pid.pointid_timing_reset()
