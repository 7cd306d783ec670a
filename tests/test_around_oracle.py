"""The 64-bit definitions that the operators around the layers are tested against: the random
words against published ones, the gradients against differences and automatic differentiation."""

import math

import pytest
import torch

import around64 as A


def test_random_words():
    """The test vectors published with the generator: counter and key of zeros, of ones, of digits of pi."""
    assert A.philox([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert A.philox([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert A.philox([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]) == \
        [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_bits_are_the_words_halves():
    seed, offset = 0x0123456789ABCDEF, 0xFEDCBA9876543210
    bits = A.drop_bits(5, 21, seed, offset)
    for row, col in ((0, 0), (0, 1), (3, 7), (4, 8), (2, 20)):
        w = A.philox([col // 8, row, offset & 0xFFFFFFFF, offset >> 32], [seed & 0xFFFFFFFF, seed >> 32])
        assert bits[row, col] == (w[col % 8 // 2] >> (16 * (col % 2))) & 0xFFFF


def test_dropout_keeps_its_share():
    for p in (0.1, 0.5, 0.9):
        kept = (A.drop_factor(500, 200, p, 7, 3) > 0).double().mean().item()
        assert abs(kept - (1 - p)) < 5 * math.sqrt(p * (1 - p) / 100000)


@pytest.mark.parametrize("before", [None, "rms", "layer"])
@pytest.mark.parametrize("after", [None, "rms", "layer"])
def test_norm_gradients(before, after):
    g = A.gen(5)
    m, n, eps = 4, 11, 1e-3
    x, o, dh, dt = (torch.randn((m, n), generator=g, dtype=torch.float64) for _ in range(4))
    wb, bb, wa, ba, gate = (torch.randn(n, generator=g, dtype=torch.float64) for _ in range(5))
    factor = A.drop_factor(m, n, 0.3, 1, 2)
    leaves = {"x": x, "out": o, "weight": wb, "bias": bb, "block_weight": wa, "block_bias": ba, "gate": gate}

    def loss(v):
        t = A.total64(v["x"], v["out"], after, eps, v["block_weight"], v["block_bias"], v["gate"], 0.7, factor)[0]
        y = (t * dt).sum()
        if before:
            h = A.norm64(before, eps, t, torch.zeros_like(t))[0] * v["weight"] + v["bias"]
            y = y + (h * dh).sum()
        return y

    t, _, _, mean_a, r_a = A.total64(x, o, after, eps, wa, ba, gate, 0.7, factor)
    stats = torch.zeros((m, 4), dtype=torch.float64)
    stats[:, 1] = stats[:, 3] = 1
    if after:
        stats[:, 0:1], stats[:, 1:2] = mean_a, r_a
    if before:
        stats[:, 2:3], stats[:, 3:4] = A.norm64(before, eps, t, torch.zeros_like(t))[2:]
    got = A.back64(dh, t, o, stats, before, after, wb, wa, ba, gate, 0.7, factor, dt)
    wanted = {k: v.clone().requires_grad_() for k, v in leaves.items()}
    loss(wanted).backward()
    for name, leaf in leaves.items():
        if name in ("weight", "bias") and not before or name.startswith("block") and not after:
            continue
        grad = got["d" + name][0]
        torch.testing.assert_close(grad, wanted[name].grad, rtol=1e-10, atol=1e-10)
        # central differences of a few of them
        for i in range(0, leaf.numel(), 7):
            v = {k: t.clone() for k, t in leaves.items()}
            step = 1e-5
            v[name].view(-1)[i] += step
            up = loss(v)
            v[name].view(-1)[i] -= 2 * step
            assert abs((up - loss(v)) / (2 * step) - grad.reshape(-1)[i]) < 1e-6


def test_logprobs_gradients():
    g = A.gen(6)
    m, n, scale = 3, 9, 1.3
    x = torch.randn((m, n), generator=g, dtype=torch.float64)
    t = torch.tensor([4, -1, 8])
    dlogp, dh, dl = (torch.randn(m, generator=g, dtype=torch.float64) for _ in range(3))

    def loss(v):
        logp = torch.log_softmax(v * scale, 1)
        entropy = -(logp.exp() * logp).sum(1)
        chosen = torch.stack([logp[i, k] if k >= 0 else logp.new_zeros(()) for i, k in enumerate(t.tolist())])
        return (chosen * dlogp + entropy * dh + torch.logsumexp(v * scale, 1) * dl).sum()

    fwd = A.logprobs64(x, scale, t, 4)
    logp = torch.log_softmax(x * scale, 1)
    torch.testing.assert_close(fwd["entropy"][0], -(logp.exp() * logp).sum(1))
    torch.testing.assert_close(fwd["top_logp"][0], logp.topk(4, 1).values)
    got, _ = A.logprobs_back64(x, scale, fwd["lse"][0], t, dlogp, fwd["entropy"][0], dh, dl)
    v = x.clone().requires_grad_()
    loss(v).backward()
    torch.testing.assert_close(got, v.grad, rtol=1e-10, atol=1e-12)
    for i in range(0, m * n, 4):
        a, b = x.clone(), x.clone()
        a.view(-1)[i] += 1e-5
        b.view(-1)[i] -= 1e-5
        assert abs((loss(a) - loss(b)) / 2e-5 - got.reshape(-1)[i]) < 1e-7
