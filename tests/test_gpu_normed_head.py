"""GPU: the layers with norms, dropout and log probabilities together, in the training of a small
patch classifier: one step's loss and gradients against 64-bit automatic differentiation of its
formulas with the same masks, and that the command runs."""

import pytest
import torch

import around64 as A

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def head():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2009_04509_amd import patch_head
    return patch_head


# rounding of every activation and gradient on the way to 2^-9 (bf16), 2^-12 (fp16) of it, about
# 14 of them in turn on a path, the norms' gradients being differences of their size at most; fp32
# by its sums.  8-bit checkpoints: 2^-4 of a value at most, 2^-5 on average, averaged over 300 rows.
@pytest.mark.parametrize("dtype, kept, tol", [("fp32", "type", 2e-5), ("bf16", "type", 0.05), ("fp16", "type", 0.007),
                                              ("bf16", "8bit", 0.12), ("fp32", "8bit", 0.12)])
def test_gradients_of_a_step(head, dtype, kept, tol):
    m, hidden, p_drop = 300, 72, 0.25
    model = head.NormedPatchHead(hidden=hidden, gated=200, dtype=dtype, kept=kept, seed=3, dropout=p_drop)
    model.steps = 5
    g = torch.Generator(device=model.device).manual_seed(4)
    x, kind, michel = head.draw_patches(m, g, model.device)
    x = x.to(model.dtype)
    out, k = model.forward(x, train=True)
    value, d = model.loss_and_gradient(out, kind, michel, 64.0)
    grads = model.backward(d, k)
    p = {n: v.double().cpu().requires_grad_() for n, v in model.p.items()}
    masks = [A.drop_factor(m, hidden, p_drop, 3, 10 + i) for i in range(2)]

    def norm(v, w):
        return v * (v.square().mean(1, keepdim=True) + 1e-5) ** -0.5 * w

    a1 = torch.relu(x.double().cpu() @ p["w1"] + p["b1"]) * masks[0]
    n1 = norm(a1, p["s1"])
    h = torch.nn.functional.silu(n1 @ p["wg"]) * (n1 @ p["wu"])
    t = a1 + p["gate"] * (norm(h @ p["wd"] + p["bd"], p["sa"]) * masks[1])
    o = norm(t, p["s2"]) @ p["wo"] + p["bo"]
    want = torch.nn.functional.cross_entropy(o[:, :3], kind.cpu()) + \
        torch.nn.functional.binary_cross_entropy_with_logits(o[:, 3], michel.double().cpu())
    want.backward()
    assert abs(value.item() - want.item()) <= max(tol, 1e-5) * abs(want.item())
    assert set(grads) == set(p)
    for name, grad in grads.items():
        err = (grad.double().cpu() / 64 - p[name].grad).norm() / p[name].grad.norm()
        assert err <= tol, (name, err.item())


@pytest.mark.parametrize("dtype, kept", [("bf16", "8bit"), ("fp16", "type"), ("fp32", "type")])
def test_the_command_runs(head, dtype, kept):
    right, found = head.main(["--steps", "4", "--batch", "300", "--dtype", dtype, "--kept", kept, "--block", "normed"])
    assert 0 <= right <= 1 and 0 <= found <= 1


def test_without_training_nothing_is_dropped(head):
    model = head.NormedPatchHead(hidden=64, gated=96, dtype="fp32", kept="type", dropout=0.5)
    x = head.draw_patches(50, torch.Generator(device=model.device).manual_seed(1), model.device)[0]
    assert torch.equal(model.forward(x), model.forward(x))
    a, _ = model.forward(x, train=True)
    model.steps += 1
    assert not torch.equal(a, model.forward(x, train=True)[0])
