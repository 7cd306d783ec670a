"""Performance cases of the layer operators: dense and gated layers, forward and
backward, and 8-bit activation checkpoints.

A case is one use of one operator (``op``) on matrices of ``dtype``, m rows of k inputs
and n outputs (weights [k][n], as everywhere in this repository):

``dense``           y = act(x W + b) + r
``dense_backward``  dx, dW and db from dy, x, W and the saved z = x W + b
``gated``           h = act(x Wg + bg) * (x Wu + bu)
``gated_backward``  dx, dWg, dWu, dbg, dbu from dh, x, Wg, Wu and the saved g, u
``gated_step``      a gated layer's part of a training step: forward with g, u and x
                    saved in 8 bits, then the backward pass from them
``checkpoint``      a matrix saved in 8 bits and loaded again

``saved`` says what the backward pass reads: the activations in their own type
("type") or 8-bit checkpoints ("8bit": blocks of 32 along a row share a power of two).
"""

from __future__ import annotations

import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
BLOCK = 32
FC1_IN = 92928                      # the network's first dense layer: 92,928 -> 128
PIXELS = 2304                       # of a 48 x 48 patch


def _case(name, op, dtype, m, k, n, act="none", bias=True, residual=False, saved="type"):
    return {"name": name, "op": op, "dtype": dtype, "m": m, "k": k, "n": n, "act": act, "bias": bias,
            "residual": residual, "saved": saved}


def listed():
    return [
        # the network's second dense layer over one client's request: the smallest call
        _case("fc2_235_fp32", "dense", "fp32", 235, 128, 32, "relu"),
        # its first dense layer over the same request: a long sum for few outputs
        _case("fc1_235_bf16", "dense", "bf16", 235, FC1_IN, 128, "relu"),
        # one row through a square layer with its residual: serving one request at a time
        _case("dense_row_fp16", "dense", "fp16", 1, 8192, 8192, bias=False, residual=True),
        # a full batch through a hidden layer: bias, activation and residual at once
        _case("dense_16384_bf16", "dense", "bf16", 16384, 4096, 4096, "gelu", residual=True),
        # gradients of the first dense layer over a job's batch
        _case("fc1_backward_1693_fp16", "dense_backward", "fp16", 1693, FC1_IN, 128, "relu"),
        # a layer over flattened patches with odd sizes, its activations kept in 8 bits
        _case("dense_backward_8bit_bf16", "dense_backward", "bf16", 1693, PIXELS, 1031, "silu", saved="8bit"),
        # a few rows through a gated layer: serving a handful of requests
        _case("gated_rows_bf16", "gated", "bf16", 4, 4096, 12288, "silu", bias=False),
        # a client's request through a gated layer over patches, odd width, single precision
        _case("gated_235_fp32", "gated", "fp32", 235, PIXELS, 1021, "gelu"),
        # the gradients of such a layer over a job's batch, single precision
        _case("gated_backward_1693_fp32", "gated_backward", "fp32", 1693, 1024, 2048, "silu"),
        # the largest: a gated layer's whole training step with 8-bit checkpoints
        _case("gated_step_8192_bf16", "gated_step", "bf16", 8192, 4096, 8192, "silu", bias=False, saved="8bit"),
        # the checkpoint alone, of a full batch's activations and of a small ragged one
        _case("checkpoint_16384_bf16", "checkpoint", "bf16", 16384, 0, 8192, bias=False),
        _case("checkpoint_235_fp16", "checkpoint", "fp16", 235, 0, 1031, bias=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["dense", "dense", "dense_backward", "gated", "gated_backward", "gated_step", "checkpoint"])
    dtype = rng.choice(["bf16", "fp16"] if op == "gated_step" else ["bf16", "bf16", "fp16", "fp32"])
    most = 2 * 8192 * 4096 * 8192 if dtype != "fp32" else 2 * 8192 * 4096 * 2048
    while True:
        m = _log_int(rng, 1, 16384)
        k = FC1_IN if op.startswith("dense") and rng.random() < 0.1 else _log_int(rng, 16, 8192)
        n = _log_int(rng, 16, 12288)
        if rng.random() < 0.5:                     # widths of real layers are mostly even
            k, n = (k + 15) // 16 * 16, (n + 15) // 16 * 16
        cost = {"dense": 1, "dense_backward": 2, "gated": 2, "gated_backward": 4, "gated_step": 6, "checkpoint": 0}[op]
        if cost * m * k * n <= most and k * n <= 1 << 26 and m * k <= 1 << 28:
            break
    act = rng.choice(["relu", "silu", "gelu", "sigmoid"]) if op.startswith("gated") else \
        rng.choice(["none", "relu", "silu", "gelu", "sigmoid"])
    # a step reads back checkpoints made from its own sums: without the column sums in
    # fp32, which would show every value that fell on the other side of an 8-bit rounding
    bias = op != "gated_step" and op != "checkpoint" and rng.random() < 0.6
    saved = "8bit" if op == "gated_step" or (op.endswith("backward") and rng.random() < 0.5) else "type"
    case = _case("", op, dtype, m, 0 if op == "checkpoint" else k, n, "none" if op == "checkpoint" else act, bias,
                 op == "dense" and rng.random() < 0.5, saved)
    del case["name"]
    return case


# ---- inputs

def _two_to(power):
    """2^power in 32 bits, for whole powers from -126 to 127, from the number's bits: exact."""
    return ((power.int() + 127) << 23).view(torch.float32)


def _checkpoint(x):
    """(q, e): the e4m3 codes [m][n] and biased exponents [m][ceil(n / 32)] of x."""
    m, n = x.shape
    nb = -(-n // BLOCK)
    v = torch.nn.functional.pad(x.float(), (0, nb * BLOCK - n)).view(m, nb, BLOCK)
    f, e = torch.frexp(v.abs().amax(2))
    k = torch.where(f == 0, torch.zeros_like(e), torch.where(f <= 0.875, 9 - e, 8 - e)).clamp(max=126)
    q = (v * _two_to(k).unsqueeze(2)).to(torch.float8_e4m3fn).view(m, nb * BLOCK)[:, :n]
    return q.contiguous().view(torch.uint8), (127 - k).to(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    m, k, n, dt = case["m"], case["k"], case["n"], DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(dt)

    def bias():
        return (torch.rand(n, generator=g, device="cuda") - 0.5) * 0.2 if case["bias"] else None

    s = {"case": case}
    if case["op"] == "checkpoint":
        # activations: rows of differing magnitude, stretches that a ReLU left at zero
        x = torch.randn((m, n), generator=g, device="cuda")
        x *= torch.exp(torch.randn((m, 1), generator=g, device="cuda"))
        dead = torch.rand((m, -(-n // BLOCK)), generator=g, device="cuda") < 0.1
        s["x"] = x.masked_fill_(dead.repeat_interleave(BLOCK, 1)[:, :n], 0.0).to(dt)
        return s
    gated, back = case["op"].startswith("gated"), not case["op"] in ("dense", "gated")
    eight = case["saved"] == "8bit" and case["op"] != "gated_step"
    # half of a layer's inputs come out of a ReLU as zeros
    x = normal(m, k).clamp_(min=0) if not gated else normal(m, k)
    s["x"] = _checkpoint(x) if eight else x
    for name in (("wg", "wu") if gated else ("w",)):
        s[name] = normal(k, n, scale=math.sqrt((1.0 if gated else 2.0) / k))
    if case["op"] in ("dense", "gated"):
        for name in (("bg", "bu") if gated else ("b",)):
            s[name] = bias()
    if case["residual"]:
        s["r"] = normal(m, n)
    if back:
        s["dy"] = normal(m, n)
        if case["op"] != "gated_step":
            for name in (("g", "u") if gated else ("z",)):
                z = normal(m, n)
                s[name] = _checkpoint(z) if eight else z
    return s


# ---- the operators in their plain form, in 32 bits

def _act(name, z):
    if name == "relu":
        return torch.where(z <= 0, torch.zeros_like(z), z)
    if name == "sigmoid":
        return 1 / (1 + torch.exp(-z))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_slope(name, z):
    if name == "relu":
        return (z > 0).float()
    if name == "sigmoid":
        t = 1 / (1 + torch.exp(-z))
        return t * (1 - t)
    if name == "silu":
        t = 1 / (1 + torch.exp(-z))
        return t * (1 + z * (1 - t))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def _values(saved):
    """The 32-bit values of what was saved: a matrix, or an 8-bit checkpoint (q, e)."""
    if not isinstance(saved, tuple):
        return saved.float()
    q, e = saved
    scale = _two_to(e.int() - 127).repeat_interleave(BLOCK, 1)[:, :q.shape[1]]
    return q.view(torch.float8_e4m3fn).float() * scale


def _plain(s):
    c = s["case"]
    op, act, dt = c["op"], c["act"], DTYPES[c["dtype"]]
    if op == "checkpoint":
        return [_values(_checkpoint(s["x"])).to(dt)]
    if op == "dense":
        z = s["x"].float() @ s["w"].float()
        y = _act(act, z + s["b"] if c["bias"] else z)
        return [(y + s["r"].float() if c["residual"] else y).to(dt)]
    if op == "dense_backward":
        x, w = _values(s["x"]), s["w"].float()
        dz = s["dy"].float() * _act_slope(act, _values(s["z"]))
        return [(dz @ w.t()).to(dt), (x.t() @ dz).to(dt)] + ([dz.sum(0)] if c["bias"] else [])
    x, wg, wu = _values(s["x"]), s["wg"].float(), s["wu"].float()
    outs = []
    if op in ("gated", "gated_step"):
        g, u = x @ wg, x @ wu
        if op == "gated" and c["bias"]:
            g, u = g + s["bg"], u + s["bu"]
        outs.append((_act(act, g) * u).to(dt))
        if op == "gated":
            return outs
        x, g, u = _values(_checkpoint(s["x"])), _values(_checkpoint(g)), _values(_checkpoint(u))
    else:
        g, u = _values(s["g"]), _values(s["u"])
    dh = s["dy"].float()
    dg, du = dh * u * _act_slope(act, g), dh * _act(act, g)
    outs += [(dg @ wg.t() + du @ wu.t()).to(dt), (x.t() @ dg).to(dt), (x.t() @ du).to(dt)]
    return outs + ([dg.sum(0), du.sum(0)] if c["bias"] else [])


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
    op, act = c["op"], c["act"]
    x = s["x"]
    device = (x[0] if isinstance(x, tuple) else x).device
    pid, layers = _layers(device.index or 0)

    def saved(v):
        return pid.Checkpoint(*v) if isinstance(v, tuple) else v

    if op == "checkpoint":
        return [pid.pointid_checkpoint_load(pid.pointid_checkpoint_save(x), x.dtype)]
    if op == "dense":
        return [pid.pointid_dense(layers, x, s["w"], s["b"], act, residual=s.get("r"))]
    if op == "dense_backward":
        dx, dw, db = pid.pointid_dense_backward(layers, s["dy"], saved(x), s["w"], saved(s["z"]), act,
                                                need_db=c["bias"])
        return [dx, dw] + ([db] if c["bias"] else [])
    if op == "gated":
        return [pid.pointid_gated(layers, x, s["wg"], s["wu"], s["bg"], s["bu"], act)]
    outs = []
    if op == "gated_step":
        g, u = (pid.Checkpoint.empty(c["m"], c["n"], device) for _ in range(2))
        outs.append(pid.pointid_gated(layers, x, s["wg"], s["wu"], act=act, save_g=g, save_u=u))
        x = pid.pointid_checkpoint_save(x)
    else:
        x, g, u = saved(x), saved(s["g"]), saved(s["u"])
    dx, dwg, dwu, dbg, dbu = pid.pointid_gated_backward(layers, s["dy"], x, s["wg"], s["wu"], g, u, act,
                                                        need_db=c["bias"])
    return outs + [dx, dwg, dwu] + ([dbg, dbu] if c["bias"] else [])


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    """Bytes: inputs read and outputs written once.  Operations: those of the products,
    and of a checkpoint the scaling and rounding of each value."""
    m, k, n, es = case["m"], case["k"], case["n"], SIZE[case["dtype"]]
    eight = case["saved"] == "8bit"

    def kept(rows, cols):
        return rows * (cols + -(-cols // BLOCK)) if eight else es * rows * cols

    op = case["op"]
    if op == "checkpoint":
        return {"bytes": 2 * es * m * n + 2 * m * (n + -(-n // BLOCK)), "flops": 4 * m * n}
    if op == "dense":
        return {"bytes": es * (m * k + k * n + (2 if case["residual"] else 1) * m * n) + 4 * n * case["bias"],
                "flops": 2 * m * k * n}
    if op == "dense_backward":
        return {"bytes": es * (m * n + 2 * k * n + m * k) + kept(m, k) + kept(m, n) + 4 * n * case["bias"],
                "flops": 4 * m * k * n}
    if op == "gated":
        return {"bytes": es * (m * k + 2 * k * n + m * n) + 8 * n * case["bias"], "flops": 4 * m * k * n}
    if op == "gated_backward":
        return {"bytes": es * (m * n + 4 * k * n + m * k) + kept(m, k) + 2 * kept(m, n) + 8 * n * case["bias"],
                "flops": 8 * m * k * n}
    return {"bytes": es * (2 * m * k + 4 * k * n + 2 * m * n), "flops": 12 * m * k * n}


# ---- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    op, name = case["op"], case["act"]
    d = {"x": None}
    d.update((key, v.double()) for key, v in s.items() if isinstance(v, torch.Tensor))

    def times_two_to(v, power):
        return v * ((power.long() + 1023) << 52).view(torch.float64)

    def grid(v):
        """v on the 8-bit grid of its blocks: the largest magnitude of a block scaled by
        the largest power of two that leaves it within 448, then 4 significant bits, and
        no finer than 2^-9."""
        rows, cols = v.shape
        out = torch.empty_like(v)
        whole = cols // BLOCK * BLOCK
        for a, b, width in ((0, whole, BLOCK), (whole, cols, cols - whole)):
            if a == b:
                continue
            t = v[:, a:b].reshape(rows, -1, width)
            top = t.abs().max(dim=2, keepdim=True).values
            # 448 / top = f 2^e with f in [1/2, 1): the exponent of the power below it
            power = torch.frexp(448.0 / top.clamp(min=2.0 ** -140)).exponent - 1
            t = torch.where(top > 0, times_two_to(t, power.clamp(max=126)), t)
            step = times_two_to(torch.ones_like(t), torch.frexp(t).exponent.clamp(min=-5) - 4)
            back = times_two_to(torch.round(t / step) * step, -power.clamp(max=126))
            out[:, a:b] = torch.where(top > 0, back, torch.zeros_like(back)).reshape(rows, b - a)
        return out

    def decode(q, e):
        sign = 1.0 - 2.0 * (q >> 7).double()
        low, high = (q & 7).double(), ((q >> 3) & 15).int()
        mag = torch.where(high == 0, low / 8 * 2.0 ** -6, times_two_to(1 + low / 8, high - 7))
        cols = torch.arange(q.shape[1], device=q.device) // BLOCK
        return sign * times_two_to(mag, e.int()[:, cols] - 127)

    for key, v in s.items():
        if isinstance(v, tuple):
            d[key] = decode(*v)
    if op == "checkpoint":
        return [grid(d["x"])]

    def sigma(z):
        return torch.sigmoid(z)

    def phi(z):
        return torch.special.ndtr(z)

    f = {"none": lambda z: z, "relu": lambda z: z.clamp(min=0), "sigmoid": sigma, "silu": lambda z: z * sigma(z),
         "gelu": lambda z: z * phi(z)}[name]
    slope = {"none": torch.ones_like, "relu": lambda z: torch.heaviside(z, torch.zeros_like(z)),
             "sigmoid": lambda z: sigma(z) * sigma(-z), "silu": lambda z: sigma(z) + z * sigma(z) * sigma(-z),
             "gelu": lambda z: phi(z) + z * torch.exp(-z.square() / 2) * (2 * math.pi) ** -0.5}[name]
    if op == "dense":
        y = f(torch.mm(d["x"], d["w"]) + d.get("b", 0.0))
        return [y + d["r"] if "r" in d else y]
    if op == "dense_backward":
        dz = slope(d["z"]) * d["dy"]
        outs = [torch.mm(dz, d["w"].T), torch.mm(d["x"].T, dz)]
        return outs + [dz.sum(dim=0)] if case["bias"] else outs
    outs = []
    if op != "gated_backward":
        g = torch.mm(d["x"], d["wg"]) + d.get("bg", 0.0)
        u = torch.mm(d["x"], d["wu"]) + d.get("bu", 0.0)
        outs = [f(g) * u]
        if op == "gated":
            return outs
        d["g"], d["u"], d["x"] = grid(g), grid(u), grid(d["x"])
    dg, du = slope(d["g"]) * d["u"] * d["dy"], f(d["g"]) * d["dy"]
    outs += [torch.mm(dg, d["wg"].T) + torch.mm(du, d["wu"].T), torch.mm(d["x"].T, dg), torch.mm(d["x"].T, du)]
    return outs + [dg.sum(dim=0), du.sum(dim=0)] if case["bias"] else outs
