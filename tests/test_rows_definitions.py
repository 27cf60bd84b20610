"""The definitions that the operators on node rows are held to, in 64 bits: their gradients against differences and against reverse
differentiation, and the bounds against what 32-bit arithmetic of another order is off by."""
import pytest
import torch

from _rows import GatedFF, ResidualNorm, act


def rand(*shape, scale=1.0, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed + sum(shape))) * scale


@pytest.mark.parametrize("name", ["sigmoid", "silu", "gelu"])
def test_gated_ff_gradients(name):
    x, Wg, Wu, Wd = rand(5, 6), rand(6, 9, seed=1), rand(6, 9, seed=2), rand(9, 4)
    bg, bu, bd, dy = rand(9, seed=3), rand(9, seed=4), rand(4), rand(5, 4, seed=5)
    got = GatedFF(x, Wg, Wu, Wd, bg, bu, bd, name).backward(dy)
    leaves = [v.double().requires_grad_(True) for v in (x, Wg, Wu, Wd, bg, bu, bd)]
    f = lambda x, Wg, Wu, Wd, bg, bu, bd: (act(name, x @ Wg + bg) * (x @ Wu + bu)) @ Wd + bd  # noqa: E731
    assert torch.autograd.gradcheck(f, leaves)
    f(*leaves).backward(dy.double())
    for v, q in zip(leaves, ("dX", "dWg", "dWu", "dWd", "dbg", "dbu", "dbd")):
        assert torch.allclose(v.grad, got[q][0], rtol=1e-12, atol=1e-12), q


@pytest.mark.parametrize("post", [None, "rms", "layer"])
@pytest.mark.parametrize("pre", ["rms", "layer"])
@pytest.mark.parametrize("gated", [True, False])
def test_residual_norm_gradients(post, pre, gated):
    F, eps = 7, 1e-2
    R, B, gate, dR, dZ = (rand(4, F, seed=s) for s in range(5))
    gate = gate if gated else None
    scale, w_post, b_post, w_pre, b_pre = (rand(F, seed=s) for s in range(5))
    if post is None:
        w_post = b_post = None

    def unit(kind, x):
        if kind == "layer":
            x = x - x.mean(1, keepdim=True)
        return x if kind is None else x / (x.square().mean(1, keepdim=True) + eps).sqrt()

    given = {"R": R, "B": B, "gate": gate, "scale": scale, "w_post": w_post, "b_post": b_post, "w_pre": w_pre, "b_pre": b_pre}
    leaves = {q: v.double().requires_grad_(True) for q, v in given.items() if v is not None}

    def f(*at):
        v = dict(zip(leaves, at))
        p = unit(post, v["B"])
        if post is not None:
            p = p * v["w_post"] + v["b_post"]
        r = v["R"] + v["scale"] * (torch.sigmoid(v["gate"]) if gated else 1.0) * p
        return r, unit(pre, r) * v["w_pre"] + v["b_pre"]

    assert torch.autograd.gradcheck(f, list(leaves.values()))
    r, z = f(*leaves.values())
    torch.autograd.backward([r, z], [dR.double(), dZ.double()])
    want = ResidualNorm(B, gate, post, pre, scale, w_post, b_post, w_pre, b_pre, eps)
    ahead = want.forward(R)
    assert torch.allclose(ahead["R_out"][0], r) and torch.allclose(ahead["Z"][0], z)
    back = want.backward(r.detach(), dR, dZ)
    assert set(back) == {"d" + q for q in leaves}
    for q, v in leaves.items():
        assert torch.allclose(v.grad, back["d" + q][0], rtol=1e-10, atol=1e-12), q


def test_bounds_hold_for_plain_32_bit_arithmetic():
    """The forms as float32 torch operations stay within the bounds as well, and not by orders of magnitude only."""
    x, Wg, Wu, Wd = rand(50, 40), rand(40, 70, seed=1), rand(40, 70, seed=2), rand(70, 30)
    y, bound = GatedFF(x, Wg, Wu, Wd, None, None, None, "silu").forward()
    err = ((act("silu", x @ Wg) * (x @ Wu)) @ Wd).double() - y
    assert bool((err.abs() <= bound).all()) and float((bound / y.abs().mean()).max()) < 1e-3
    R, B = rand(50, 64), rand(50, 64, seed=1)
    z, bound = ResidualNorm(B, None, "layer", "layer", None, None, None, None, None, 1e-5).forward(R)["Z"]
    ln = torch.nn.functional.layer_norm
    err = ln(R + ln(B, (64,), eps=1e-5), (64,), eps=1e-5).double() - z
    assert bool((err.abs() <= bound).all()) and float(bound.max()) < 1e-3
