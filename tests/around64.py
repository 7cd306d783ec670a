"""The operators around the layers in 64 bits, with the bounds of what fp32 arithmetic may be off.

u is half a unit in the last place of the result's type relative to a value (2^-8 bf16, 2^-11
fp16, 2^-24 fp32), E = 2^-23 bounds one fp32 operation by twice its rounding.  A tree of partial
sums of at most D terms in turn is off by at most D E of the sum of magnitudes.
"""

import math

import numpy as np
import torch

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
U = {name: torch.finfo(t).eps / 2 for name, t in DT.items()}
TINY = {"bf16": 2.0 ** -133, "fp16": 2.0 ** -25, "fp32": 2.0 ** -149}
E = 2.0 ** -23


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rand(g, *shape, dtype="bf16", scale=1.0):
    return (torch.randn(shape, generator=g, dtype=torch.float64) * scale).to(DT[dtype])


def near(got, want, tol, what):
    """Every value within its tolerance; a NaN or infinity only where there is the same."""
    got, tol = got.detach().double().cpu(), torch.as_tensor(tol, dtype=torch.float64).expand(want.shape)
    assert got.shape == want.shape, what
    odd = ~torch.isfinite(want)
    same = (got == want) | (got.isnan() & want.isnan())
    bad = torch.where(odd, ~same, ~((got - want).abs() <= tol))
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, e.g. at " \
        f"{bad.nonzero()[0].tolist()}: {got[bad][0].item()} for {want[bad][0].item()}, tolerance {tol[bad][0].item()}"


def rounded(want, tol, dtype):
    """The tolerance of a value that is rounded to a type at the end."""
    return tol + (want.abs() + tol) * U[dtype] + TINY[dtype]


# ---- random bits and dropout

def philox(counter, key):
    """Philox4x32-10, plain whole numbers of any size."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def drop_bits(rows, cols, seed, offset, first_row=0):
    """The 16 random bits of each element, [rows][cols]."""
    low = np.uint64(0xFFFFFFFF)
    shift = np.uint64(32)
    groups = -(-cols // 8)
    c = [np.broadcast_to(np.arange(groups, dtype=np.uint64), (rows, groups)),
         np.broadcast_to(np.arange(first_row, first_row + rows, dtype=np.uint64)[:, None], (rows, groups)),
         np.full((rows, groups), offset & 0xFFFFFFFF, np.uint64), np.full((rows, groups), offset >> 32, np.uint64)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> shift) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> shift) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    halves = [(w >> np.uint64(16 * h)) & np.uint64(0xFFFF) for w in c for h in (0, 1)]
    bits = np.stack(halves, 2).reshape(rows, -1)[:, :cols]
    return torch.from_numpy(bits.astype(np.int64))


def drop_factor(rows, cols, p, seed, offset):
    """0, or one over the share that is kept."""
    threshold = math.floor(p * 65536 + 0.5)
    keep = drop_bits(rows, cols, seed, offset) >= threshold
    return torch.where(keep, 65536 / (65536 - threshold) if threshold < 65536 else 0.0, 0.0).double()


def dropped(v, factor):
    """What is dropped is 0, whatever it was."""
    return torch.where(factor > 0, v * factor, 0.0)


# ---- norms.  A value goes with the bound of its error: (v, tv).

def depth(n):
    """Terms in turn of a row's sum: each thread's, of at least 64, and the tree over them."""
    return 40 + n / 64


def norm64(kind, eps, v, tv):
    """(u, its bound, mean, 1 / deviation)"""
    n = v.shape[1]
    D = depth(n)
    mean, tmean = torch.zeros_like(v[:, :1]), torch.zeros_like(v[:, :1])
    if kind == "layer":
        mean = v.mean(1, keepdim=True)
        tmean = tv.mean(1, keepdim=True) + (D + 2) * E * v.abs().mean(1, keepdim=True)
    d = v - mean
    td = tv + tmean + E * (v.abs() + d.abs())
    square = (d * d).mean(1, keepdim=True)
    tsquare = (2 * d.abs() * td + td * td).mean(1, keepdim=True) + (D + 4) * E * square
    if kind == "layer":            # what shifts every d alike adds nothing of first order
        t = tv + E * (v.abs() + d.abs())
        tsquare = (2 * d.abs() * t + td * td).mean(1, keepdim=True) + (D + 4) * E * square
    r = (square + eps) ** -0.5
    tr = r * (tsquare / (square + eps) + 4 * E)
    return d * r, td * r + (d.abs() + td) * tr + 2 * E * (d * r).abs(), mean, r


def affine64(u, tu, w, b):
    if w is not None:
        u, tu = u * w, tu * w.abs() + E * (u * w).abs()
    if b is not None:
        u, tu = u + b, tu + E * (u.abs() + (u + b).abs())
    return u, tu


def total64(x, o, after, eps, wa, ba, gate, scale, factor):
    """(t, its bound, of the norm after the block: v, mean, r)"""
    v, tv, mean, r = o, torch.zeros_like(o), None, None
    if after:
        v, tv, mean, r = norm64(after, eps, o, tv)
        v, tv = affine64(v, tv, wa, ba)
    plain = v
    if factor is not None:
        v, tv = dropped(v, factor), dropped(tv + 2 * E * v.abs(), factor)
    if gate is not None:
        v, tv = v * gate, tv * gate.abs() + E * (v * gate).abs()
    t = scale * x + v
    return t, tv + 2 * E * ((scale * x).abs() + v.abs() + t.abs()), plain, mean, r


def back64(dh, t, o, stats, before, after, wb, wa, ba, gate, scale, factor, dt):
    """{name: (gradient, bound)} from the statistics that the kernel is given too."""
    out = {}
    ref = t if t is not None else dt
    m, n = ref.shape
    D, rows = depth(n), (m + 16) * E
    d, td = (dt, torch.zeros_like(dt)) if dt is not None else (torch.zeros_like(t), torch.zeros_like(t))

    def column(name, a, ta):
        out[name] = a.sum(0), ta.sum(0) + rows * a.abs().sum(0)

    def through(kind, f, tf, u, r):
        """f - u mean(f u) - [layer] mean(f), times r"""
        mu, tmu = (f * u).mean(1, keepdim=True), (tf * u.abs() + (D + 6) * E * (f * u).abs()).mean(1, keepdim=True)
        m1, tm1 = torch.zeros_like(mu), torch.zeros_like(mu)
        if kind == "layer":
            m1, tm1 = f.mean(1, keepdim=True), (tf + (D + 4) * E * f.abs()).mean(1, keepdim=True)
        g = r * (f - u * mu - m1)
        return g, r * (tf + u.abs() * tmu + 2 * E * (u * mu).abs() + tm1 + 4 * E * (f.abs() + (u * mu).abs() + m1.abs()))

    if before:
        u, r = (t - stats[:, 2:3]) * stats[:, 3:4], stats[:, 3:4]
        tu = 2 * E * u.abs()
        e = dh * wb if wb is not None else dh
        g, tg = through(before, e, E * e.abs(), u, r)
        d, td = d + g, td + tg + E * (d.abs() + g.abs())
        column("dweight", dh * u, dh.abs() * tu + E * (dh * u).abs())
        column("dbias", dh, torch.zeros_like(dh))
    out["dx"] = scale * d, abs(scale) * td + E * (scale * d).abs()
    if factor is not None:
        d, td = dropped(d, factor), dropped(td + 2 * E * d.abs(), factor)
    q, tq = (d * gate, td * gate.abs() + E * (d * gate).abs()) if gate is not None else (d, td)
    if after:
        u, r = (o - stats[:, 0:1]) * stats[:, 1:2], stats[:, 1:2]
        tu = 2 * E * u.abs()
        column("dblock_weight", q * u, tq * u.abs() + q.abs() * tu + E * (q * u).abs())
        column("dblock_bias", q, tq)
        f, tf = (q * wa, tq * wa.abs() + E * (q * wa).abs()) if wa is not None else (q, tq)
        out["dout"] = through(after, f, tf, u, r)
        v, tv = affine64(u, tu, wa, ba)
    else:
        out["dout"] = q, tq
        v, tv = o, torch.zeros_like(q)
    if gate is not None:
        column("dgate", d * v, td * v.abs() + d.abs() * tv + E * (d * v).abs())
    return out


# ---- log probabilities

def logprobs64(x, scale, targets, top):
    """{name: (values, bound)} of finite logits and masked (minus infinity) ones."""
    m, n = x.shape
    z = x * scale
    most = z.amax(1, keepdim=True)
    empty = most[:, 0] == -math.inf
    d = torch.where(empty.view(-1, 1), -math.inf, z - most)
    e = d.exp()
    s = e.sum(1)
    p = e / s.view(-1, 1)
    low = torch.where(e > 0, d, 0.0).abs()
    spread = (p * low).sum(1)
    # of s: the sums, each column's exponent and its rescalings
    D = depth(n)
    ts = (2 * D + 10 + 8 * spread) * E
    ln = s.log()
    lse = most[:, 0] + ln
    tln = ts + 2 * E * (1 + ln.abs())
    out = {"lse": (lse, tln + 3 * E * (most[:, 0].abs() + ln.abs() + lse.abs()))}
    w = (p * low).sum(1)
    tw = (2 * D + 10) * E * w + (p * low * (8 * E * (1 + low))).sum(1) + ts * w
    out["entropy"] = ln + w, tln + tw + 3 * E * (ln.abs() + w)
    if targets is not None:
        has = (targets >= 0) & (targets < n)
        dt = d.gather(1, torch.where(has, targets, 0).long().view(-1, 1))[:, 0]
        out["logp"] = torch.where(has, dt - ln, 0.0), torch.where(has, tln + 4 * E * (dt.abs() + ln.abs()), 0.0)
    if top:
        ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :top]
        dt = d.gather(1, ids)
        out["top_ids"] = ids, torch.zeros_like(dt)
        out["top_logp"] = dt - ln.view(-1, 1), tln.view(-1, 1) + 4 * E * (dt.abs() + ln.abs().view(-1, 1))
    for name, (v, t) in out.items():
        if name in ("top_ids",):
            continue
        v[empty] = 0.0 if name == "entropy" else -math.inf
        t[~torch.isfinite(v)] = 0.0
        if name == "entropy":
            t[empty] = 0.0
        if name == "logp":
            v[~has], t[~has] = 0.0, 0.0
    return out


def logprobs_back64(x, scale, lse, targets, dlogp, entropy, dentropy, dlse):
    """(gradient, bound) from the lse and entropy that the kernel is given too."""
    m, n = x.shape
    z, l = x * scale, lse.view(-1, 1)
    empty = l == -math.inf
    logp = torch.where(empty, -math.inf, z - l)
    p = logp.exp()
    finite = torch.where(p > 0, logp, 0.0)
    a = torch.where(p > 0, 2 * E * (z.abs() + l.abs()), 0.0)
    tp = p * (a + 5 * E + 3 * E * finite.abs())
    zero = torch.zeros((m, 1), dtype=torch.float64)
    has = (targets >= 0) & (targets < n) if targets is not None else torch.zeros(m, dtype=torch.bool)
    g = torch.where(has, dlogp, 0.0).view(-1, 1) if dlogp is not None else zero
    gl = dlse.view(-1, 1) if dlse is not None else zero
    gh, h = (dentropy.view(-1, 1), entropy.view(-1, 1)) if dentropy is not None else (zero, zero)
    c = gl - g - gh * (finite + h)
    tc = 3 * E * (gl.abs() + g.abs() + (gh * (finite + h)).abs()) + gh.abs() * (a + 2 * E * (finite.abs() + h.abs()))
    d = p * c
    td = tp * c.abs() + p * tc + E * d.abs()
    if has.any():
        one = torch.zeros_like(d)
        one[has.nonzero()[:, 0], targets[has].long()] = 1.0
        d = d + one * g
        td = td + E * one * (g.abs() + d.abs())
    d, td = torch.where(empty, 0.0, d * scale), torch.where(empty, 0.0, td * scale + E * (d * scale).abs())
    return d, td
