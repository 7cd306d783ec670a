"""A small patch classifier trained with the library's layers.

    python -m paper_2009_04509_amd.patch_head [--steps N] [--batch B] [--dtype bf16|fp16|fp32] [--kept 8bit|type]
                                             [--block plain|normed] [--dropout P]

The classifier has the heads of the network of paper §2.2 (softmax over track, shower and
none, a sigmoid for Michel) on a dense layer over the patch's 2,304 pixels and a gated
block with its residual, in place of the convolution and the wide first layer:

    a1  = relu(x w1 + b1)
    h   = silu(a1 wg) * (a1 wu)
    a2  = h wd + bd + a1
    out = a2 wo + bo

Every layer and gradient is one call of the library.  With ``kept="8bit"`` what the backward pass
reads (x, z1, a1, g, u, h, a2) is kept in 8-bit checkpoints: the pre-activations are
written so by the forward layers themselves.  Only the loss over the 4 outputs and the
update of the parameters are torch.

``--block normed`` has norms and dropout around the gated block, and the softmax branch's
loss and its gradient by the library's log probabilities (NormedPatchHead).
"""

from __future__ import annotations

import math

import torch

from . import binding as pid

PIXELS = 48 * 48
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def draw_patches(n: int, generator: torch.Generator, device) -> tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(patches [n][2304], class [n], michel [n]): noise; a straight line of charge through
    the centre (track, class 0); a spray of short lines from it (shower, class 1; half
    of them short and bright: Michel); nothing (class 2)."""
    r = torch.arange(48, device=device, dtype=torch.float32) - 24
    yy, xx = r.view(1, 48, 1), r.view(1, 1, 48)

    def uniform(lo, hi, *shape):
        return lo + (hi - lo) * torch.rand(shape, generator=generator, device=device)

    kind = torch.randint(0, 3, (n,), generator=generator, device=device)
    michel = (kind == 1) & (torch.rand((n,), generator=generator, device=device) < 0.5)
    image = torch.randn((n, 48, 48), generator=generator, device=device) * 0.3
    lines = 5
    angle = uniform(0, 2 * math.pi, n, lines)
    angle[:, 1:] = angle[:, :1] + (angle[:, 1:] - math.pi) * 0.25
    for i in range(lines):
        c, s = torch.cos(angle[:, i]).view(n, 1, 1), torch.sin(angle[:, i]).view(n, 1, 1)
        along, across = xx * c + yy * s, xx * s - yy * c
        ridge = torch.exp(-0.5 * across * across)
        if i == 0:
            image += ridge * (kind == 0).view(n, 1, 1) * 2
        reach = torch.where(michel, 8.0, 20.0).view(n, 1, 1)
        ray = ridge * ((along > 0) & (along < reach))
        image += ray * (kind == 1).view(n, 1, 1) * torch.where(michel, 2.0, 1.0).view(n, 1, 1)
    return image.view(n, PIXELS), kind, michel.float()


class PatchHead:
    """Parameters in fp32, their copies in the layers' type, momentum, and one training step."""

    def __init__(self, device: int = 0, hidden: int = 512, gated: int = 1536, dtype: str = "bf16", kept: str = "8bit",
                 seed: int = 0):
        self.layers = pid.pointid_layers_create(device)
        self.device = torch.device("cuda", device)
        self.dtype = DTYPES[dtype]
        self.eight = kept == "8bit"
        g = torch.Generator(device=self.device).manual_seed(seed)

        def normal(rows, cols, gain):
            return torch.randn((rows, cols), generator=g, device=self.device) * math.sqrt(gain / rows)

        self.master = {"w1": normal(PIXELS, hidden, 2.0), "wg": normal(hidden, gated, 1.0), "wu": normal(hidden, gated, 1.0),
                       "wd": normal(gated, hidden, 1.0), "wo": normal(hidden, 4, 1.0)}
        for name, n in (("b1", hidden), ("bd", hidden), ("bo", 4)):
            self.master[name] = torch.zeros(n, device=self.device)
        self.momentum = {k: torch.zeros_like(v) for k, v in self.master.items()}
        self._copy()

    def _copy(self):
        self.p = {k: v.to(self.dtype) if k[0] == "w" else v for k, v in self.master.items()}

    def _keep(self, m, n):
        """Where a layer puts its pre-activation."""
        return pid.Checkpoint.empty(m, n, self.device) if self.eight else \
            torch.empty((m, n), dtype=self.dtype, device=self.device)

    def _kept(self, x):
        return pid.pointid_checkpoint_save(x) if self.eight else x

    def forward(self, x: torch.Tensor, train: bool = False):
        """Outputs [m][4] of patches [m][2304], and with ``train`` what backward() needs."""
        L, p, m = self.layers, self.p, x.shape[0]
        hidden, gated = p["wg"].shape
        z1 = self._keep(m, hidden) if train else None
        g, u = (self._keep(m, gated) if train else None for _ in range(2))
        a1 = pid.pointid_dense(L, x, p["w1"], p["b1"], "relu", save=z1)
        h = pid.pointid_gated(L, a1, p["wg"], p["wu"], act="silu", save_g=g, save_u=u)
        a2 = pid.pointid_dense(L, h, p["wd"], p["bd"], residual=a1)
        out = pid.pointid_dense(L, a2, p["wo"], p["bo"])
        if not train:
            return out
        return out, {"x": self._kept(x), "z1": z1, "a1": self._kept(a1), "g": g, "u": u, "h": self._kept(h),
                     "a2": self._kept(a2)}

    def backward(self, dout: torch.Tensor, k: dict) -> dict:
        """Gradients of every parameter from the outputs' gradient."""
        L, p = self.layers, self.p
        da2, dwo, dbo = pid.pointid_dense_backward(L, dout, k["a2"], p["wo"])
        dh, dwd, dbd = pid.pointid_dense_backward(L, da2, k["h"], p["wd"])
        da1, dwg, dwu, _, _ = pid.pointid_gated_backward(L, dh, k["a1"], p["wg"], p["wu"], k["g"], k["u"], "silu")
        da1 += da2                                   # the residual's
        _, dw1, db1 = pid.pointid_dense_backward(L, da1, k["x"], p["w1"], k["z1"], "relu", need_dx=False)
        return {"w1": dw1, "b1": db1, "wg": dwg, "wu": dwu, "wd": dwd, "bd": dbd, "wo": dwo, "bo": dbo}

    @staticmethod
    def loss(out: torch.Tensor, kind: torch.Tensor, michel: torch.Tensor):
        """(mean loss, its gradient by the outputs): cross entropy of the softmax over the
        first three plus that of the sigmoid of the fourth."""
        o = out.float()
        logp = torch.log_softmax(o[:, :3], 1)
        s = torch.sigmoid(o[:, 3])
        n = o.shape[0]
        value = -logp.gather(1, kind.view(-1, 1)).mean() - (michel * torch.nn.functional.logsigmoid(o[:, 3]) +
                                                            (1 - michel) * torch.nn.functional.logsigmoid(-o[:, 3])).mean()
        d = torch.empty_like(o)
        d[:, :3] = logp.exp()
        d[:, :3].scatter_add_(1, kind.view(-1, 1), torch.full((n, 1), -1.0, device=o.device))
        d[:, 3] = s - michel
        return value, d / n

    def step(self, x: torch.Tensor, kind: torch.Tensor, michel: torch.Tensor, rate: float = 0.05,
             momentum: float = 0.9) -> torch.Tensor:
        """One step of gradient descent; the loss before it (a device value)."""
        out, kept = self.forward(x.to(self.dtype), train=True)
        value, d = self.loss(out, kind, michel)
        scale = 1024.0                               # keeps the gradients of a batch inside fp16's range
        for name, grad in self.backward((d * scale).to(self.dtype), kept).items():
            self.momentum[name].mul_(momentum).add_(grad.float(), alpha=1 / scale)
            self.master[name].add_(self.momentum[name], alpha=-rate)
        self._copy()
        return value


class NormedPatchHead(PatchHead):
    """The classifier with norms (root mean square) before and after the gated block, a gate on its
    output, and dropout as in paper §2.2 after the dense layer and on the block's output:

        a1  = drop(relu(x w1 + b1))
        n1  = norm(a1, s1)
        h   = silu(n1 wg) * (n1 wu)
        t   = a1 + gate * drop(norm(h wd + bd, sa))
        n2  = norm(t, s2)
        out = n2 wo + bo

    The norms read what they need for their gradients in its own type.  The masks are made again
    in the backward pass, from the step's number."""

    def __init__(self, device: int = 0, hidden: int = 512, gated: int = 1536, dtype: str = "bf16", kept: str = "8bit",
                 seed: int = 0, dropout: float = 0.1):
        super().__init__(device, hidden, gated, dtype, kept, seed)
        self.p_drop, self.seed, self.steps = dropout, seed, 0
        for name, value in (("s1", 1.0), ("sa", 1.0), ("s2", 1.0), ("gate", 0.5)):
            self.master[name] = torch.full((hidden,), value, device=self.device)
            self.momentum[name] = torch.zeros_like(self.master[name])
        self._copy()

    def _drop(self, i: int):
        """The step's i-th mask."""
        return pid.Drop(self.p_drop, self.seed, 2 * self.steps + i)

    def forward(self, x: torch.Tensor, train: bool = False):
        L, p, m = self.layers, self.p, x.shape[0]
        hidden, gated = p["wg"].shape
        z1 = self._keep(m, hidden) if train else None
        g, u = (self._keep(m, gated) if train else None for _ in range(2))
        a1 = pid.pointid_dense(L, x, p["w1"], p["b1"], "relu", save=z1)
        if train:
            a1 = pid.pointid_dropout(L, a1, self._drop(0), y=a1)
        first = pid.pointid_norm(L, a1, pid.Norm("rms", p["s1"]), keep=train)
        h = pid.pointid_gated(L, first.h, p["wg"], p["wu"], act="silu", save_g=g, save_u=u)
        o = pid.pointid_dense(L, h, p["wd"], p["bd"])
        block = pid.Block(o, pid.Norm("rms", p["sa"]), p["gate"], drop=self._drop(1) if train else None)
        joint = pid.pointid_norm(L, a1, pid.Norm("rms", p["s2"]), block, keep=train)
        out = pid.pointid_dense(L, joint.h, p["wo"], p["bo"])
        if not train:
            return out
        return out, {"x": self._kept(x), "z1": z1, "a1": a1, "first": first.stats, "n1": self._kept(first.h), "g": g, "u": u,
                     "h": self._kept(h), "block": block, "joint": joint, "n2": self._kept(joint.h)}

    def backward(self, dout: torch.Tensor, k: dict) -> dict:
        L, p = self.layers, self.p
        dn2, dwo, dbo = pid.pointid_dense_backward(L, dout, k["n2"], p["wo"])
        j = pid.pointid_norm_backward(L, dn2, k["joint"].total, k["joint"].stats, pid.Norm("rms", p["s2"]), k["block"])
        dh, dwd, dbd = pid.pointid_dense_backward(L, j.dout, k["h"], p["wd"])
        dn1, dwg, dwu, _, _ = pid.pointid_gated_backward(L, dh, k["n1"], p["wg"], p["wu"], k["g"], k["u"], "silu")
        # the residual's gradient joins that through the norm, in its own memory
        f = pid.pointid_norm_backward(L, dn1, k["a1"], k["first"], pid.Norm("rms", p["s1"]), dtotal=j.dx, dx=j.dx)
        da1 = pid.pointid_dropout(L, f.dx, self._drop(0), y=f.dx)
        _, dw1, db1 = pid.pointid_dense_backward(L, da1, k["x"], p["w1"], k["z1"], "relu", need_dx=False)
        return {"w1": dw1, "b1": db1, "wg": dwg, "wu": dwu, "wd": dwd, "bd": dbd, "wo": dwo, "bo": dbo, "s1": f.dweight,
                "sa": j.dblock_weight, "s2": j.dweight, "gate": j.dgate}

    def loss_and_gradient(self, out: torch.Tensor, kind: torch.Tensor, michel: torch.Tensor, scale: float):
        """(mean loss, its gradient by the outputs times ``scale``, in their type)"""
        n = out.shape[0]
        kind = kind.to(torch.int32)
        got = pid.pointid_logprobs(self.layers, out[:, :3], kind)
        z = out[:, 3].float()
        value = -got.logp.mean() - (michel * torch.nn.functional.logsigmoid(z) +
                                    (1 - michel) * torch.nn.functional.logsigmoid(-z)).mean()
        d = torch.empty_like(out)
        each = torch.full((n,), -scale / n, device=out.device)
        pid.pointid_logprobs_backward(self.layers, out[:, :3], got.lse, kind, each, dlogits=d[:, :3])
        d[:, 3] = (torch.sigmoid(z) - michel) * (scale / n)
        return value, d

    def step(self, x: torch.Tensor, kind: torch.Tensor, michel: torch.Tensor, rate: float = 0.05,
             momentum: float = 0.9) -> torch.Tensor:
        out, kept = self.forward(x.to(self.dtype), train=True)
        scale = 1024.0
        value, d = self.loss_and_gradient(out, kind, michel, scale)
        grads = self.backward(d, kept)
        self.steps += 1
        for name, grad in grads.items():
            self.momentum[name].mul_(momentum).add_(grad.float(), alpha=1 / scale)
            self.master[name].add_(self.momentum[name], alpha=-rate)
        self._copy()
        return value


def main(argv=None):
    import argparse
    ap = argparse.ArgumentParser(description="Train a small patch classifier with the library's layers.")
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--batch", type=int, default=1693)
    ap.add_argument("--dtype", choices=sorted(DTYPES), default="bf16")
    ap.add_argument("--kept", choices=["8bit", "type"], default="8bit")
    ap.add_argument("--block", choices=["plain", "normed"], default="plain")
    ap.add_argument("--dropout", type=float, default=0.1, help="of --block normed")
    a = ap.parse_args(argv)
    model = PatchHead(dtype=a.dtype, kept=a.kept) if a.block == "plain" else \
        NormedPatchHead(dtype=a.dtype, kept=a.kept, dropout=a.dropout)
    g = torch.Generator(device=model.device).manual_seed(1)
    for i in range(a.steps):
        value = model.step(*draw_patches(a.batch, g, model.device))
        if i % 20 == 0 or i == a.steps - 1:
            print(f"step {i:4d}: loss {value.item():.4f}", flush=True)
    x, kind, michel = draw_patches(4096, g, model.device)
    out = model.forward(x.to(model.dtype)).float()
    right = (out[:, :3].argmax(1) == kind).float().mean().item()
    found = ((out[:, 3] > 0) == (michel > 0)).float().mean().item()
    print(f"{a.dtype}, activations kept in {a.kept}: class right on {100 * right:.1f} %, Michel on {100 * found:.1f} % of 4096 "
          "new patches", flush=True)
    return right, found


if __name__ == "__main__":
    main()
