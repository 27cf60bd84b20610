"""The operators on node rows as a model uses them, around an aggregation: norm, aggregation, norms with gate and residual scale, gated
feed-forward block, norms; and back through all of it with the transposed frame."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_gated_ff import pipad  # noqa: E402,F401

EPS = 1e-5
VECTORS = ("w0", "s1", "w1", "b1", "v1", "c1", "s2", "w2", "v2")
MATRICES = ("Wg", "Wu", "Wd")


def graph(n, k, seed):
    """Directed snapshots, rows without edges and one that everything points to among them; also dense, normalised, in 64 bits."""
    rng = np.random.default_rng(seed)
    snaps, dense = [], []
    base = rng.random((n, n)) < 6 / n
    for _ in range(k):
        a = (base & (rng.random((n, n)) < 0.9)) | (rng.random((n, n)) < 0.5 / n)
        a[:, 0], a[3] = True, False
        np.fill_diagonal(a, False)
        snaps.append((torch.from_numpy(np.concatenate([[0], a.sum(1).cumsum()]).astype(np.int32)).cuda(), torch.from_numpy(np.nonzero(a)[1].astype(np.int32)).cuda()))
        d = 1.0 / np.sqrt(1.0 + a.sum(1))
        dense.append(torch.from_numpy(d[:, None] * (a + np.eye(n)) * d).cuda())
    return snaps, dense


def layer(pipad, frame, back, R, gate, p, dR2, dZ2, layout):  # noqa: F811
    """One layer and its gradients, as a training program writes them."""
    _, z0 = pipad.residual_norm(R, pre="rms", w_pre=p["w0"], eps=EPS)
    a = pipad.frame_aggregate(frame, z0)
    r1, z1 = pipad.residual_norm(R, a, gate, post="layer", pre="rms", scale=p["s1"], w_post=p["w1"], b_post=p["b1"], w_pre=p["v1"], eps=EPS)
    f = pipad.gated_ff(z1, p["Wg"], p["Wu"], p["Wd"], p["bg"], p["bu"], p["bd"])
    r2, z2 = pipad.residual_norm(r1, f, post="rms", pre="layer", scale=p["s2"], w_post=p["w2"], w_pre=p["v2"], b_pre=p["c1"], eps=EPS)
    d2 = pipad.residual_norm_backward(r2, dR2, dZ2, f, post="rms", pre="layer", scale=p["s2"], w_post=p["w2"], w_pre=p["v2"], eps=EPS)
    df = pipad.gated_ff_backward(z1, d2.dB, p["Wg"], p["Wu"], p["Wd"], p["bg"], p["bu"])
    d1 = pipad.residual_norm_backward(r1, d2.dR, df.dX, a, gate, post="layer", pre="rms", scale=p["s1"], w_post=p["w1"], b_post=p["b1"], w_pre=p["v1"],
                                      eps=EPS)
    d0 = pipad.residual_norm_backward(R, d1.dR, pipad.frame_aggregate(back, d1.dB), pre="rms", w_pre=p["w0"], eps=EPS)
    grads = {"w0": d0.dw_pre, "s1": d1.dscale, "w1": d1.dw_post, "b1": d1.db_post, "v1": d1.dw_pre, "s2": d2.dscale, "w2": d2.dw_post, "v2": d2.dw_pre,
             "c1": d2.db_pre, "Wg": df.dWg, "Wu": df.dWu, "Wd": df.dWd, "bg": df.dbg, "bu": df.dbu, "bd": df.dbd}
    return r2, z2, d0.dR, d1.dgate, grads


def reference(dense, R, gate, p, dR2, dZ2):
    """The same in 64 bits, [k, n, F], by reverse differentiation."""
    p = {q: v.double().requires_grad_(True) for q, v in p.items()}
    R, gate = R.double().requires_grad_(True), gate.double().requires_grad_(True)

    def unit(kind, x):
        x = x - x.mean(-1, keepdim=True) if kind == "layer" else x
        return x / (x.square().mean(-1, keepdim=True) + EPS).sqrt()

    a = torch.stack([m @ z for m, z in zip(dense, unit("rms", R) * p["w0"])])
    r1 = R + p["s1"] * torch.sigmoid(gate) * (unit("layer", a) * p["w1"] + p["b1"])
    z1 = unit("rms", r1) * p["v1"]
    f = (torch.nn.functional.silu(z1 @ p["Wg"] + p["bg"]) * (z1 @ p["Wu"] + p["bu"])) @ p["Wd"] + p["bd"]
    r2 = r1 + p["s2"] * unit("rms", f) * p["w2"]
    z2 = unit("layer", r2) * p["v2"] + p["c1"]
    torch.autograd.backward([r2, z2], [dR2.double(), dZ2.double()])
    return r2.detach(), z2.detach(), R.grad, gate.grad, {q: v.grad for q, v in p.items()}


def parameters(gen, F, hidden):
    p = {q: torch.randn(F, device="cuda", generator=gen) * 0.3 + (q[0] in "wv") for q in VECTORS}
    p.update({q: torch.randn((F, hidden), device="cuda", generator=gen) / F ** 0.5 for q in MATRICES[:2]})
    p["Wd"] = torch.randn((hidden, F), device="cuda", generator=gen) / hidden ** 0.5
    p.update({q: torch.randn(c, device="cuda", generator=gen) * 0.1 for q, c in (("bg", hidden), ("bu", hidden), ("bd", F))})
    return p


@pytest.mark.parametrize("n,k,F,hidden", [(90, 2, 24, 64), (301, 3, 64, 171), (40, 5, 130, 50)])
@pytest.mark.parametrize("layout", ["list", "wide"])
def test_layer_and_its_gradients(pipad, n, k, F, hidden, layout):  # noqa: F811
    """Each of the seven calls is off by at most some 5e-7 of its result in the 2-norm (about four roundings of 2^-24 that add up as their
    squares do); a norm passes on at most twice what reaches it here, so 7 x 2^2 x 5e-7 = 1.4e-5 covers the chain."""
    snaps, dense = graph(n, k, n)
    gen = torch.Generator(device="cuda").manual_seed(n)
    p = parameters(gen, F, hidden)
    R, gate, dR2, dZ2 = (torch.randn((k, n, F), device="cuda", generator=gen) for _ in range(4))
    form = (lambda x: x.transpose(0, 1).contiguous()) if layout == "wide" else (lambda x: list(x.unbind(0)))
    frame = pipad.frame_build_overlap(snaps, validate=True)
    back = pipad.frame_transpose(frame)
    got = layer(pipad, frame, back, form(R), form(gate), p, form(dR2), form(dZ2), layout)
    want = reference(dense, R, gate, p, dR2, dZ2)
    for q in range(4):
        x = got[q].transpose(0, 1) if layout == "wide" else torch.stack(got[q])
        assert float((x - want[q]).norm() / want[q].norm()) < 1.4e-5, q
    assert set(got[4]) == set(want[4])
    for q, v in want[4].items():
        assert float((got[4][q] - v).norm() / v.norm()) < 1.4e-5, q
    frame.close()
    back.close()


def test_layer_recorded_into_a_graph(pipad):  # noqa: F811
    n, k, F, hidden = 500, 3, 32, 96
    snaps, _ = graph(n, k, 1)
    gen = torch.Generator(device="cuda").manual_seed(1)
    p = parameters(gen, F, hidden)
    R, gate, dR2, dZ2 = ([torch.randn((n, F), device="cuda", generator=gen) for _ in range(k)] for _ in range(4))
    frame = pipad.frame_build_overlap(snaps)
    back = pipad.frame_transpose(frame)

    def flat(out):
        return [*out[0], *out[1], *out[2], *out[3], *out[4].values()]

    def run():
        return flat(layer(pipad, frame, back, R, gate, p, dR2, dZ2, "list"))

    run()
    torch.cuda.synchronize()
    graph_ = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph_):
        outs = run()
    for replay in range(3):
        for x in (*R, *gate, p["Wg"]):
            x.normal_(0, 0.5, generator=gen)
        want = run()
        torch.cuda.synchronize()
        for o in outs:
            o.fill_(float("nan"))
        graph_.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, outs)), replay
    frame.close()
    back.close()
