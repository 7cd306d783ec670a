"""Performance cases of the operators around the layers in a training step: norms at the
joint of two residual blocks, dropout, and log probabilities as the loss, with their gradients.

A case is one use of one operator (``op``) on matrices of ``dtype``, m rows of n columns:

``norm``               t = scale x + gate * drop(N_a(o)),  h = N_b(t)   (o: a block's output;
                       N_a: the norm after the block, N_b: the one before the next)
``norm_backward``      gradients of x, o and every parameter from those of h and t
``dropout``            y = drop(x) + r
``logprobs``           of each row's logits: log probability of its target, log of the sum of
                       exponentials, entropy, the ``top`` most likely columns
``logprobs_backward``  the logits' gradient from those of the log probabilities and entropies

Norms: "rms" x / sqrt(mean(x^2) + eps) * weight, or "layer" (x - mean) / sqrt(var + eps) *
weight + bias.  drop keeps an element with the 16 bits that Philox4x32-10 gives for its row and
column (counter: column / 8, row, offset; key: seed) if they are at least round(p 2^16), and
divides by the share that it keeps.
"""

from __future__ import annotations

import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
EPS = 1e-5
IGNORED = -100                      # the target of a row that has none


def _norm_case(name, op, dtype, m, n, before="rms", after="rms", gate=True, scale=1.0, p=0.0):
    return {"name": name, "op": op, "dtype": dtype, "m": m, "n": n, "before": before, "after": after, "gate": gate,
            "scale": scale, "p": p}


def _dropout_case(name, dtype, m, n, p, residual):
    return {"name": name, "op": "dropout", "dtype": dtype, "m": m, "n": n, "p": p, "residual": residual}


def _logprobs_case(name, op, dtype, m, n, scale=1.0, banned=0.0, ignored=0.0, top=0, entropy=True, pad=0):
    return {"name": name, "op": op, "dtype": dtype, "m": m, "n": n, "scale": scale, "banned": banned,
            "ignored": ignored, "top": top, "entropy": entropy, "pad": pad}


def listed():
    return [
        # one row at the joint of two blocks: serving one request at a time
        _norm_case("norm_row_bf16", "norm", "bf16", 1, 8192, gate=False),
        # a full batch at such a joint, forward: both norms, a gate and a scaled residual
        _norm_case("norm_16384_bf16", "norm", "bf16", 16384, 4096, scale=0.5),
        # a job's batch of an odd width, dropout on the block's output, no norm after it
        _norm_case("norm_1693_fp32", "norm", "fp32", 1693, 1031, before="layer", after="none", gate=False, p=0.1),
        # the gradients at the joint over a full batch, with dropout: seven results
        _norm_case("norm_backward_16384_bf16", "norm_backward", "bf16", 16384, 4096, scale=0.5, p=0.1),
        # the same over a job's batch of rows as long as a patch, layer norms
        _norm_case("norm_backward_1693_fp16", "norm_backward", "fp16", 1693, 2304, before="layer", after="layer"),
        # dropout and the residual of a full batch: the largest pass
        _dropout_case("dropout_16384_bf16", "bf16", 16384, 8192, 0.1, True),
        # dropout of a client's request, odd width
        _dropout_case("dropout_235_fp32", "fp32", 235, 1031, 0.5, False),
        # one row of many classes with its 20 likeliest: serving one request at a time
        _logprobs_case("logprobs_row_bf16", "logprobs", "bf16", 1, 131072, scale=1.25, top=20),
        # a batch over many classes: some banned, some rows without a target
        _logprobs_case("logprobs_4096_bf16", "logprobs", "bf16", 4096, 65536, banned=0.02, ignored=0.05, top=8),
        # the three classes of an event's hits, beside the Michel output in rows of four
        _logprobs_case("logprobs_classes_fp32", "logprobs", "fp32", 50000, 3, top=1, pad=1),
        # the loss's gradient over many classes, with an entropy term
        _logprobs_case("logprobs_backward_4096_bf16", "logprobs_backward", "bf16", 4096, 65536, banned=0.02,
                       ignored=0.05),
        # the same over a job's batch, single precision, an odd number of classes
        _logprobs_case("logprobs_backward_1693_fp32", "logprobs_backward", "fp32", 1693, 32003, ignored=0.05,
                       entropy=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_backward", "norm_backward", "dropout", "logprobs", "logprobs",
                     "logprobs_backward"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    widest, most = (131072, 1 << 28) if op.startswith("logprobs") else (16384, 1 << 26)
    while True:
        m = _log_int(rng, 1, 16384 if op[0] != "l" else 50000)
        n = _log_int(rng, 3 if op[0] == "l" else 16, widest)
        if rng.random() < 0.5 and n > 8:           # widths of real layers are mostly even
            n = (n + 15) // 16 * 16
        if m * n * SIZE[dtype] <= 2 * most:
            break
    p = rng.choice([0.0, 0.05, 0.1, 0.25, 0.5])
    if op.startswith("norm"):
        case = _norm_case("", op, dtype, m, n, rng.choice(["rms", "layer"]), rng.choice(["none", "rms", "layer"]),
                          rng.random() < 0.5, rng.choice([1.0, 1.0, 0.5, 1.5]), p if rng.random() < 0.5 else 0.0)
    elif op == "dropout":
        case = _dropout_case("", dtype, m, n, p, rng.random() < 0.5)
    else:
        case = _logprobs_case("", op, dtype, m, n, rng.choice([1.0, 1.0, 0.7, 1.25]),
                              rng.choice([0.0, 0.02]) if n >= 64 else 0.0, rng.choice([0.0, 0.05]),
                              min(n // 2, rng.choice([0, 1, 5, 8, 20, 32])) if op == "logprobs" else 0,
                              rng.random() < 0.7, rng.choice([0, 0, 1, 8]))
    del case["name"]
    return case


# ---- inputs

def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    m, n, dt = case["m"], case["n"], DTYPES[case["dtype"]]

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    s = {"case": case, "seed": seed * 0x9E3779B97F4A7C15 % (1 << 64), "offset": seed + (1 << 33)}
    if case["op"] == "dropout":
        s["x"] = randn(m, n).clamp_(min=0).to(dt)                       # out of a ReLU
        s["r"] = randn(m, n).to(dt) if case["residual"] else None
        return s
    if case["op"].startswith("logprobs"):
        # most columns unlikely, a few of every row likely
        x = randn(m, n + case["pad"]) * 2
        x += (torch.rand(x.shape, generator=g, device="cuda") < 4 / n).float() * 8
        target = torch.randint(0, n, (m,), generator=g, device="cuda", dtype=torch.int32)
        if case["banned"]:
            held = x.gather(1, target.long().view(-1, 1))
            x.masked_fill_(torch.rand(x.shape, generator=g, device="cuda") < case["banned"], -math.inf)
            x.scatter_(1, target.long().view(-1, 1), held)
        if case["ignored"]:
            target.masked_fill_(torch.rand(m, generator=g, device="cuda") < case["ignored"], IGNORED)
        s["logits"], s["target"] = x.to(dt)[:, :n], target
        if case["op"] == "logprobs_backward":
            # as the forward pass left them
            lse, entropy = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
            for a in range(0, m, 1024):
                z = s["logits"][a:a + 1024].double() * case["scale"]
                l = torch.logsumexp(z, 1)
                lse[a:a + 1024] = l
                d = z - l.view(-1, 1)
                entropy[a:a + 1024] = -(d.exp() * d.clamp(min=-800)).sum(1)
            s["lse"], s["entropy"] = lse, entropy
            # the mean over the rows that have a target, some rows weighted; a bonus for entropy
            # (fp16: times the loss's scale, which keeps small gradients in the type's range)
            unit = (16384.0 if case["dtype"] == "fp16" else 1.0) / m
            s["dlogp"] = -(0.5 + torch.rand(m, generator=g, device="cuda")) * unit
            s["dentropy"] = torch.full((m,), -0.01 * unit, device="cuda") if case["entropy"] else None
        return s
    # the residual stream has grown: rows and some columns of differing magnitude
    columns = torch.exp(0.5 * randn(n))
    x = randn(m, n) * torch.exp(0.5 * randn(m, 1)) * columns
    o = randn(m, n) * torch.exp(0.5 * randn(m, 1)) + (0.3 if case["after"] == "layer" else 0.0)

    def params(kind):
        return (1 + 0.2 * randn(n), 0.1 * randn(n) if kind == "layer" else None) if kind != "none" else (None, None)

    s["x"], s["o"] = x.to(dt), o.to(dt)
    s["wa"], s["ba"] = params(case["after"])
    s["wb"], s["bb"] = params(case["before"])
    s["gate"] = 0.5 * randn(n) if case["gate"] else None
    if case["op"] == "norm_backward":
        # as the forward pass left them: the sum and each norm's mean and 1 / deviation
        s["t"] = (x.mul_(case["scale"]).add_(o)).to(dt)
        del s["x"]
        s["dh"], s["dt"] = randn(m, n).to(dt), randn(m, n).to(dt)
        stats = torch.zeros((m, 4), device="cuda")
        for i, (kind, v) in enumerate(((case["after"], s["o"]), (case["before"], s["t"]))):
            if kind == "none":
                continue
            v = v.double()
            if kind == "layer":
                stats[:, 2 * i] = v.mean(1)
                v -= v.mean(1, keepdim=True)
            stats[:, 2 * i + 1] = (v.square().mean(1) + EPS).rsqrt()
        s["stats"] = stats
    return s


# ---- the operators in their plain form, in 32 bits

def _drop_factor(s):
    """What drop multiplies each element by: 0, or one over the share that is kept."""
    m, n, p = s["case"]["m"], s["case"]["n"], s["case"]["p"]
    threshold = math.floor(p * 65536 + 0.5)
    low = (1 << 32) - 1
    # 32-bit words in 64 bits; products wrap, their upper words are masked
    c0 = torch.arange(-(-n // 8), device="cuda").view(1, -1).expand(m, -1)
    c1 = torch.arange(m, device="cuda").view(-1, 1)
    c2, c3 = s["offset"] & low, s["offset"] >> 32
    k0, k1 = s["seed"] & low, s["seed"] >> 32
    c2, c3 = torch.full_like(c1, c2), torch.full_like(c1, c3)
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    bits = torch.stack([h for c in (c0, c1, c2, c3) for h in (c & 0xFFFF, c >> 16)], 2).view(m, -1)[:, :n]
    return (bits >= threshold).float() * (65536 / (65536 - threshold) if threshold < 65536 else 0.0)


def _normed(kind, v):
    """(v less its mean, 1 / deviation) by rows."""
    if kind == "layer":
        v = v - v.sum(1, keepdim=True) / v.shape[1]
    return v, 1 / torch.sqrt((v * v).sum(1, keepdim=True) / v.shape[1] + EPS)


def _normed_back(kind, e, unit, r):
    """The gradient of v from e, that of unit = (v - mean) r."""
    back = e - unit * ((e * unit).sum(1, keepdim=True) / e.shape[1])
    if kind == "layer":
        back = back - e.sum(1, keepdim=True) / e.shape[1]
    return back * r


def _plain_norm(s):
    c, dt = s["case"], DTYPES[s["case"]["dtype"]]
    v = s["o"].float()
    if c["after"] != "none":
        v, r = _normed(c["after"], v)
        v = v * r * s["wa"]
        if s["ba"] is not None:
            v = v + s["ba"]
    if c["p"]:
        v = v * _drop_factor(s)
    t = s["x"].float() * c["scale"] + (v * s["gate"] if c["gate"] else v)
    h, r = _normed(c["before"], t)
    h = h * r * s["wb"]
    return [t.to(dt), (h + s["bb"] if s["bb"] is not None else h).to(dt)]


def _plain_norm_backward(s):
    c, dt = s["case"], DTYPES[s["case"]["dtype"]]
    dh, unit = s["dh"].float(), (s["t"].float() - s["stats"][:, 2:3]) * s["stats"][:, 3:4]
    dwb, dbb = (dh * unit).sum(0), dh.sum(0) if s["bb"] is not None else None
    d = s["dt"].float() + _normed_back(c["before"], dh * s["wb"], unit, s["stats"][:, 3:4])
    dx = (d * c["scale"]).to(dt)
    v = s["o"].float()
    if c["p"]:
        d = d * _drop_factor(s)
    dwa = dba = dgate = None
    if c["after"] != "none":
        unit = (v - s["stats"][:, 0:1]) * s["stats"][:, 1:2]
        v = unit * s["wa"]
        if s["ba"] is not None:
            v = v + s["ba"]
    if c["gate"]:
        dgate = (d * v).sum(0)
        d = d * s["gate"]
    if c["after"] != "none":
        dwa, dba = (d * unit).sum(0), d.sum(0) if s["ba"] is not None else None
        d = _normed_back(c["after"], d * s["wa"], unit, s["stats"][:, 1:2])
    return [v for v in (dx, d.to(dt), dwb, dbb, dwa, dba, dgate) if v is not None]


def _plain_logprobs(s):
    c = s["case"]
    x, n = s["logits"].float(), c["n"]
    z = x * c["scale"]
    most = z.amax(1, keepdim=True)
    e = torch.exp(z - most)
    total = e.sum(1, keepdim=True)
    lse = (most + torch.log(total)).view(-1)
    there = s["target"] >= 0
    at = torch.where(there, s["target"], 0).long().view(-1, 1)
    outs = [torch.where(there, z.gather(1, at).view(-1) - lse, 0.0), lse]
    if c["entropy"]:
        d = torch.where(e > 0, z - most, 0.0)
        outs.append(torch.log(total.view(-1)) - (e * d).sum(1) / total.view(-1))
    if c["top"]:
        # whole numbers in the order of the values, each with its column: the lowest first among equals
        bits = x.contiguous().view(torch.int32)
        key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * (1 << 20)
        key += (1 << 20) - 1 - torch.arange(n, device="cuda")
        ids = (1 << 20) - 1 - (torch.topk(key, c["top"], 1).values & ((1 << 20) - 1))
        outs += [ids.int(), z.gather(1, ids) - lse.view(-1, 1)]
    return outs


def _plain_logprobs_backward(s):
    c = s["case"]
    logp = s["logits"].float() * c["scale"] - s["lse"].view(-1, 1)
    p = torch.exp(logp)
    there = s["target"] >= 0
    dlogp = torch.where(there, s["dlogp"], 0.0).view(-1, 1)
    d = -p * dlogp
    if c["entropy"]:
        d = d - p * torch.where(p > 0, logp + s["entropy"].view(-1, 1), 0.0) * s["dentropy"].view(-1, 1)
    d.scatter_add_(1, torch.where(there, s["target"], 0).long().view(-1, 1), dlogp)
    return [(d * c["scale"]).to(DTYPES[c["dtype"]])]


def _plain(s):
    op = s["case"]["op"]
    if op == "dropout":
        y = s["x"].float() * _drop_factor(s)
        return [(y + s["r"].float() if s["r"] is not None else y).to(s["x"].dtype)]
    return {"norm": _plain_norm, "norm_backward": _plain_norm_backward, "logprobs": _plain_logprobs,
            "logprobs_backward": _plain_logprobs_backward}[op](s)


# ---- the framework's operators

_handles = {}


def _layers(device):
    """The program's handle on a device."""
    if device not in _handles:
        from paper_2009_04509_amd import binding
        _handles[device] = (binding, binding.pointid_layers_create(device))
    return _handles[device]


def _own(s):
    c = s["case"]
    op = c["op"]
    pid, layers = _layers((s["logits"] if "logits" in s else s["o"] if "o" in s else s["x"]).get_device())
    if op == "dropout":
        return [pid.pointid_dropout(layers, s["x"], pid.Drop(c["p"], s["seed"], s["offset"]), residual=s["r"])]
    if op == "logprobs":
        got = pid.pointid_logprobs(layers, s["logits"], s["target"], scale=c["scale"], entropy=c["entropy"],
                                   top=c["top"])
        return [v for v in (got.logp, got.lse, got.entropy, got.top_ids, got.top_logp) if v is not None]
    if op == "logprobs_backward":
        return [pid.pointid_logprobs_backward(layers, s["logits"], s["lse"], s["target"], s["dlogp"],
                                              s["entropy"] if c["entropy"] else None, s["dentropy"],
                                              scale=c["scale"])]
    before = pid.Norm(c["before"], s["wb"], s["bb"], EPS)
    block = pid.Block(s["o"], pid.Norm(c["after"], s["wa"], s["ba"], EPS) if c["after"] != "none" else None, s["gate"],
                      c["scale"], pid.Drop(c["p"], s["seed"], s["offset"]) if c["p"] else None)
    if op == "norm":
        got = pid.pointid_norm(layers, s["x"], before, block)
        return [got.total, got.h]
    got = pid.pointid_norm_backward(layers, s["dh"], s["t"], s["stats"], before, block, dtotal=s["dt"])
    return [v for v in (got.dx, got.dout, got.dweight, got.dbias, got.dblock_weight, got.dblock_bias, got.dgate)
            if v is not None]


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    """Bytes: inputs read and outputs written once.  Operations: those of the formulas, each
    exponential and each random word's share counted as one."""
    m, n, es = case["m"], case["n"], SIZE[case["dtype"]]
    op = case["op"]
    if op == "dropout":
        return {"bytes": (3 if case["residual"] else 2) * es * m * n, "flops": 8 * m * n}
    if op == "logprobs":
        return {"bytes": m * (es * n + 4 + 4 * (2 + case["entropy"]) + 8 * case["top"]), "flops": 6 * m * n}
    if op == "logprobs_backward":
        return {"bytes": m * (2 * es * n + 4 + 4 * (2 + 2 * case["entropy"])), "flops": (4 + 3 * case["entropy"]) * m * n}
    normed = (case["before"] != "none") + (case["after"] != "none")
    params = sum({"none": 0, "rms": 1, "layer": 2}[case[k]] for k in ("before", "after")) + case["gate"]
    if op == "norm":
        return {"bytes": 4 * es * m * n + 4 * n * params, "flops": (6 * normed + 3 + 8 * (case["p"] > 0)) * m * n}
    return {"bytes": 6 * es * m * n + 16 * m + 8 * n * params, "flops": (14 * normed + 6 + 8 * (case["p"] > 0)) * m * n}


# ---- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    m, n, op = case["m"], case["n"], case["op"]

    def kept():
        """The share that drop leaves of each element, its random words by multiplication in
        two halves of 16 bits."""
        limit = int(case["p"] * 65536 + 0.5)
        if limit == 0:
            return 1.0
        mask = 0xFFFFFFFF

        def product(word, factor):
            upper, lower = word * (factor >> 16), word * (factor & 0xFFFF)
            middle = (upper & 0xFFFF) * 65536 + lower
            return (upper >> 16) + (middle >> 32), middle & mask

        groups = (n + 7) // 8
        col, row = torch.meshgrid(torch.arange(groups, device="cuda"), torch.arange(m, device="cuda"), indexing="ij")
        word = [col, row, torch.full_like(col, s["offset"] % 2 ** 32), torch.full_like(col, s["offset"] // 2 ** 32)]
        for i in range(10):
            key = [(s["seed"] % 2 ** 32 + i * 0x9E3779B9) % 2 ** 32, (s["seed"] // 2 ** 32 + i * 0xBB67AE85) % 2 ** 32]
            (h0, l0), (h1, l1) = product(word[0], 0xD2511F53), product(word[2], 0xCD9E8D57)
            word = [h1 ^ word[1] ^ key[0], l1, h0 ^ word[3] ^ key[1], l0]
        out = torch.empty((groups * 8, m), dtype=torch.float64, device="cuda")
        for i in range(8):
            out[i::8] = ((word[i // 2] >> (16 * (i % 2))) % 65536 >= limit).double()
        return out[:n].T * (65536 / (65536 - limit))

    def f64(name):
        return s[name].double() if s.get(name) is not None else None

    if op == "dropout":
        y = kept() * f64("x")
        return [y + f64("r") if case["residual"] else y]
    if op == "logprobs":
        logits = f64("logits")
        lse = torch.logsumexp(logits * case["scale"], dim=1)
        rows = torch.arange(m, device="cuda")
        there = s["target"] != IGNORED
        logp = torch.zeros(m, dtype=torch.float64, device="cuda")
        logp[there] = logits[rows[there], s["target"][there].long()] * case["scale"] - lse[there]
        outs = [logp, lse]
        if case["entropy"]:
            h = torch.empty(m, dtype=torch.float64, device="cuda")
            for a in range(0, m, 1024):
                h[a:a + 1024] = torch.special.entr(torch.softmax(logits[a:a + 1024] * case["scale"], dim=1)).sum(dim=1)
            outs.append(h)
        if case["top"]:
            ids = torch.empty((m, case["top"]), dtype=torch.int32, device="cuda")
            values = torch.empty((m, case["top"]), dtype=torch.float64, device="cuda")
            for a in range(0, m, 1024):
                v, i = torch.sort(logits[a:a + 1024], dim=1, descending=True, stable=True)
                ids[a:a + 1024], values[a:a + 1024] = i[:, :case["top"]], v[:, :case["top"]]
            outs += [ids, values * case["scale"] - lse[:, None]]
        return outs
    if op == "logprobs_backward":
        d = torch.empty((m, n), dtype=torch.float64, device="cuda")
        for a in range(0, m, 1024):
            b = min(a + 1024, m)
            z = s["logits"][a:b].double() * case["scale"]
            p = torch.softmax(z, dim=1)
            weight = torch.where(s["target"][a:b] != IGNORED, s["dlogp"][a:b].double(), 0.0)
            d[a:b] = -weight[:, None] * p
            if case["entropy"]:
                # dH / dz_j = -p_j (log p_j + H)
                part = torch.special.entr(p)
                d[a:b] += s["dentropy"][a:b].double()[:, None] * (part - p * part.sum(dim=1, keepdim=True))
            rows = (s["target"][a:b] != IGNORED).nonzero()[:, 0]
            d[a + rows, s["target"][a:b][rows].long()] += weight[rows]
        return [d * case["scale"]]

    def standard(kind, v):
        """(the normed rows without their parameters, 1 / deviation)"""
        if kind == "layer":
            r = 1 / torch.sqrt(torch.var(v, dim=1, correction=0, keepdim=True) + EPS)
            return (v - torch.mean(v, dim=1, keepdim=True)) * r, r
        r = 1 / torch.sqrt(torch.mean(v ** 2, dim=1, keepdim=True) + EPS)
        return v * r, r

    def affine(unit, w, b):
        return unit if w is None else unit * w if b is None else unit * w + b

    factor = kept()
    gate = f64("gate") if case["gate"] else 1.0
    a_unit, a_r = standard(case["after"], f64("o")) if case["after"] != "none" else (f64("o"), None)
    branch = affine(a_unit, f64("wa"), f64("ba"))
    if op == "norm":
        t = case["scale"] * f64("x") + branch * factor * gate
        return [t, affine(standard(case["before"], t)[0], f64("wb"), f64("bb"))]

    def jacobian(kind, e, unit, r):
        """e times the norm's Jacobian, which is symmetric: the identity less its share along
        the normed row (and along the ones)."""
        out = e - unit * torch.mean(unit * e, dim=1, keepdim=True)
        return r * (out - torch.mean(e, dim=1, keepdim=True) if kind == "layer" else out)

    b_unit, b_r = standard(case["before"], f64("t"))
    dh = f64("dh")
    dt = f64("dt") + jacobian(case["before"], dh * f64("wb"), b_unit, b_r)
    outs = [dt * case["scale"], None, torch.sum(dh * b_unit, dim=0)]
    if s["bb"] is not None:
        outs.append(torch.sum(dh, dim=0))
    db = dt * factor * gate
    if case["after"] != "none":
        outs[1] = jacobian(case["after"], db * f64("wa"), a_unit, a_r)
        outs.append(torch.sum(db * a_unit, dim=0))
        if s["ba"] is not None:
            outs.append(torch.sum(db, dim=0))
    else:
        outs[1] = db
    if case["gate"]:
        outs.append(torch.sum(dt * factor * branch, dim=0))
    return outs
