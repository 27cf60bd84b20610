"""The norms around a block with its gate and residual scale, and their gradients, against their definition in 64 bits, element by
element, within bounds derived from the roundings (_rows.py)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from _rows import LAYOUTS, ResidualNorm, fill_with, room, stacked, untouched, within  # noqa: E402
from test_gpu_gated_ff import pipad  # noqa: E402,F401

EPS = 1e-5


def rows(gen, layout, n, k, F, scale=1.0):
    return fill_with(room(layout, n, k, F)[1], torch.randn((k, n, F), device="cuda", generator=gen) * scale)


def vectors(gen, F, post, pre, bias, scale=True):
    v = lambda: torch.randn(F, device="cuda", generator=gen)  # noqa: E731
    return {"scale": v() if scale else None, "w_post": v() if post else None, "b_post": v() if post and bias else None,
            "w_pre": v() if pre else None, "b_pre": v() if pre and bias else None}


def check(pipad, n, k, F, post, pre, gated=True, block=True, layout="list", bias=True, learnt=True, seed=0, in_place=False):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(seed + n + 31 * F)
    R = rows(gen, layout, n, k, F)
    B, gate = rows(gen, layout, n, k, F, 2.0) if block else None, rows(gen, layout, n, k, F, 3.0) if gated else None
    v = vectors(gen, F, post, pre, bias, block) if learnt else dict.fromkeys(("scale", "w_post", "b_post", "w_pre", "b_pre"))
    ops = [None if x is None else stacked(x) for x in (B, gate)]
    want = ResidualNorm(*ops, post, pre, *v.values(), EPS)
    ahead = want.forward(stacked(R))
    outs = {q: room(layout, n, k, F) for q in ("R_out", "Z", "dR", "dB", "dgate")}
    if in_place and block:
        outs["R_out"] = fill_with(outs["R_out"][1], torch.stack(list(R) if isinstance(R, list) else list(R.unbind(1)))), outs["R_out"][1]
        given = outs["R_out"][1]
    else:
        given = R
    r, z = pipad.residual_norm(given, B, gate, post=post, pre=pre, **v, eps=EPS, R_out=outs["R_out"][1] if block else None, Z=outs["Z"][1] if pre else None)
    within(stacked(r), *ahead["R_out"], "R_out")
    if pre:
        within(stacked(z), *ahead["Z"], "Z")
        assert untouched(*outs["Z"])
    else:
        assert z is None
    if block and not in_place:
        assert untouched(*outs["R_out"])
    dR, dZ = rows(gen, layout, n, k, F, 0.1), rows(gen, layout, n, k, F, 0.1) if pre else None
    back = want.backward(stacked(r), stacked(dR), None if dZ is None else stacked(dZ))
    if in_place:
        fill_with(outs["dR"][1], torch.stack(list(dR) if isinstance(dR, list) else list(dR.unbind(1))))
        dR = outs["dR"][1]
    v.pop("b_pre")
    got = pipad.residual_norm_backward(r, dR, dZ, B, gate, post=post, pre=pre, **v, eps=EPS, dR=outs["dR"][1], dB=outs["dB"][1] if block else None,
                                       dgate=outs["dgate"][1] if gated else None)
    for q, value in got._asdict().items():
        assert (value is not None) == (q in back), q
        if value is not None:
            matrix = q in ("dR", "dB", "dgate")
            within(stacked(value) if matrix else value, *back[q], q)
            if matrix:
                assert untouched(*outs[q])


@pytest.mark.parametrize("post", [None, "rms", "layer"])
@pytest.mark.parametrize("pre", [None, "rms", "layer"])
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("F", [1, 5, 64, 100])
def test_every_form(pipad, post, pre, gated, F):  # noqa: F811
    check(pipad, 43, 2, F, post, pre, gated)
    check(pipad, 43, 2, F, post, pre, gated, bias=False, in_place=True)
    check(pipad, 9, 1, F, post, pre, gated, learnt=False)


@pytest.mark.parametrize("F", [1, 2, 3, 4, 6, 7, 8, 9, 16, 17, 32, 33, 64, 65, 127, 128, 129, 253, 256, 257, 511, 512, 513, 1000, 1023, 1024, 1025, 1028, 2000, 4095, 4096])
@pytest.mark.parametrize("layout", ["list", "odd"])
def test_every_width(pipad, F, layout):  # noqa: F811
    check(pipad, 70, 2, F, "layer", "rms", layout=layout)


@pytest.mark.parametrize("F", [1, 2, 3, 4, 5, 8, 10, 12, 13, 16, 20, 24, 25, 30, 32, 40, 48, 49, 60, 64, 80, 96, 97, 110, 128, 190])
@pytest.mark.parametrize("n,k", [(1, 1), (259, 3), (2100, 1)])
def test_rows_that_share_a_wave(pipad, F, n, k):  # noqa: F811
    check(pipad, n, k, F, "rms", "layer", layout="odd")


@pytest.mark.parametrize("pre", ["rms", "layer"])
@pytest.mark.parametrize("F", [3, 64, 200, 1500])
def test_before_a_first_block(pipad, F, pre):  # noqa: F811
    check(pipad, 300, 1, F, None, pre, gated=False, block=False)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("n,k,F", [(1, 1, 64), (1, 32, 20), (3, 5, 64), (33, 2, 128), (257, 4, 30), (600, 1, 16)])
def test_every_layout_and_number_of_rows(pipad, layout, n, k, F):  # noqa: F811
    check(pipad, n, k, F, "rms", "layer", layout=layout)


def test_one_of_the_results_or_gradients(pipad):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(7)
    n, k, F = 90, 2, 36
    R, B, gate, dR, dZ = (rows(gen, "list", n, k, F) for _ in range(5))
    v = vectors(gen, F, "rms", "layer", True)
    kw = dict(post="rms", pre="layer", eps=EPS)
    r, z = pipad.residual_norm(R, B, gate, **kw, **v)
    assert all(torch.equal(x, y) for x, y in zip(pipad.residual_norm(R, B, gate, post="rms", pre=None, eps=EPS, **{**v, "w_pre": None, "b_pre": None})[0], r))
    v.pop("b_pre")
    zero = [torch.zeros_like(x) for x in R]
    for given, same in (((dR, None), (dR, zero)), ((None, dZ), (zero, dZ))):
        x, y = (pipad.residual_norm_backward(r, *g, B, gate, **kw, **v) for g in (given, same))
        for p, q in zip(x, y):
            assert all(torch.equal(s, t) for s, t in zip(p, q))
    every, some = pipad.residual_norm_backward(r, dR, dZ, B, gate, **kw, **v), pipad.residual_norm_backward(r, dR, dZ, B, gate, **kw, **v, vectors=False)
    assert all(torch.equal(s, t) for q in range(3) for s, t in zip(every[q], some[q])) and some[3:] == (None,) * 5
    empty = [torch.empty((0, F), device="cuda")] * 2
    got = pipad.residual_norm_backward(empty, empty, empty, empty, empty, **kw, **v)
    assert all(bool((g == 0).all()) for g in got[3:]) and pipad.residual_norm(empty, empty, empty, **kw)[1][1].shape == (0, F)


def test_rows_at_the_edges(pipad):  # noqa: F811
    """Rows of zeros, of equal values, of huge and tiny values; a row that is not finite spoils itself alone."""
    F = 64
    R = torch.randn((8, 1, F), device="cuda")
    R[0], R[1], R[2], R[3] = 0.0, 5.0, R[2] * 1e15, R[3] * 1e-30
    _, z = pipad.residual_norm(R, pre="layer", eps=EPS)
    assert bool((z[0] == 0).all()) and bool((z[1].abs() <= 5 * 2.0 ** -22 / EPS ** 0.5).all())
    want = torch.nn.functional.layer_norm(R.double(), (F,), eps=EPS)
    assert bool((z[2:].double() - want[2:]).abs().max() < 1e-5)
    _, z = pipad.residual_norm(R, pre="rms", eps=EPS)
    assert bool((z[0] == 0).all()) and float((z[2].norm() - 8.0).abs()) < 1e-4 and bool(z.isfinite().all())
    for bad in (float("inf"), float("nan")):
        R2 = R.clone()
        R2[5, 0, 7] = bad
        _, z2 = pipad.residual_norm(R2, pre="rms", eps=EPS)
        others = [0, 1, 2, 3, 4, 6, 7]
        assert torch.equal(z[others], z2[others]) and not bool(z2[5, 0, 7].isfinite())
    gate = torch.full((8, 1, F), -float("inf"), device="cuda")  # a closed gate: the block is not heard, and hears nothing
    r, _ = pipad.residual_norm(R, R.clone(), gate, post=None, pre="rms")
    assert torch.equal(r, R)
    d = pipad.residual_norm_backward(r, torch.ones_like(R), None, R.clone(), gate, post=None, pre="rms")
    assert bool((d.dB == 0).all()) and bool((d.dgate == 0).all()) and bool((d.dscale == 0).all())
    gate.fill_(float("inf"))
    r, _ = pipad.residual_norm(R, R.clone(), gate, post=None, pre="rms")
    assert torch.equal(r, R + R)


@pytest.mark.parametrize("n,F", [(2, 64), (5000, 48), (3000, 1200)])
def test_same_bits_again_on_another_stream_and_in_a_graph(pipad, n, F):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(8)
    R, B, gate, dR, dZ = (rows(gen, "list", n, 2, F) for _ in range(5))
    v = vectors(gen, F, "layer", "rms", True)
    back = {q: x for q, x in v.items() if q != "b_pre"}

    def both(stream=None):
        r, z = pipad.residual_norm(R, B, gate, post="layer", pre="rms", **v, stream=stream)
        d = pipad.residual_norm_backward(R, dR, dZ, B, gate, post="layer", pre="rms", **back, stream=stream)
        return [*r, *z, *d.dR, *d.dB, *d.dgate, *d[3:]]

    want = both()
    torch.cuda.synchronize()
    got = both(torch.cuda.Stream())
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = both()
    for replay in range(3):
        for x in (*R, *dZ):
            x.normal_(generator=gen)
        want = both()
        torch.cuda.synchronize()
        for o in outs:
            o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, outs)), replay


def test_workspace_is_all_that_is_written(pipad):  # noqa: F811
    lib = pipad.load_library()
    gen = torch.Generator(device="cuda").manual_seed(9)
    for n, k, F in ((1, 1, 7), (4000, 3, 64), (30000, 1, 2), (500, 2, 3000), (90, 32, 9)):
        need = ctypes.c_size_t()
        assert lib.pipad_residual_norm_workspace(F, n, k, ctypes.byref(need)) == 0
        ops = [rows(gen, "list", n, k, F) for _ in range(5)]
        seen = []
        for fill in (0, 255):
            ws = torch.full((need.value + 4096,), fill, dtype=torch.uint8, device="cuda")
            seen.append(pipad.residual_norm_backward(*ops, post="rms", workspace=ws[:need.value])[3:])
            assert bool((ws[need.value:] == fill).all())
        assert all(torch.equal(x, y) for x, y in zip(*seen))
        with pytest.raises(pipad.PipadError) as why:
            pipad.residual_norm_backward(*ops, post="rms", workspace=ws[:need.value - 16])
        assert why.value.status == -6


def test_rows_past_32_bit_offsets(pipad):  # noqa: F811
    n, F = 35_000_000, 128
    gen = torch.Generator(device="cuda").manual_seed(10)
    R, B, dZ = (torch.zeros((n, F), device="cuda") for _ in range(3))
    some = torch.cat([torch.arange(a, a + 40, device="cuda") for a in (0, 2 ** 31 // F - 20, 2 ** 32 // F - 20, n - 40)])
    for x in (R, B, dZ):
        x[some] = torch.randn((some.numel(), F), device="cuda", generator=gen)
    want = ResidualNorm(B[some], None, "rms", "layer", None, None, None, None, None, EPS)
    r, z = pipad.residual_norm([R], [B], post="rms", pre="layer", eps=EPS)
    ahead = want.forward(R[some])
    within(r[0][some], *ahead["R_out"], "R_out")
    within(z[0][some], *ahead["Z"], "Z")
    d = pipad.residual_norm_backward(r, None, [dZ], [B], post="rms", pre="layer", eps=EPS)
    back = want.backward(r[0][some], None, dZ[some])
    within(d.dR[0][some], *back["dR"], "dR")
    within(d.dB[0][some], *back["dB"], "dB")
    within(d.dw_post, *back["dw_post"], "dw_post")


def test_more_rows_than_a_launch_has_threads_for(pipad):  # noqa: F811
    """A workgroup has 16 rows of 33 columns, and a launch fewer than 2^32 threads along x: 2^24 workgroups are more than one launch."""
    n, F = (1 << 28) + 77, 33
    gen = torch.Generator(device="cuda").manual_seed(12)
    R, Z = torch.zeros((n, F), device="cuda"), torch.full((n, F), 7.0, device="cuda")
    some = torch.cat([torch.arange(a, a + 40, device="cuda") for a in (0, (1 << 26) - 20, (1 << 27) - 20, (1 << 28) - 20, n - 40)])
    R[some] = torch.randn((some.numel(), F), device="cuda", generator=gen)
    pipad.residual_norm([R], pre="layer", eps=EPS, Z=[Z])
    want = ResidualNorm(None, None, None, "layer", None, None, None, None, None, EPS)
    within(Z[some], *want.forward(R[some])["Z"], "Z")
    assert float(Z.sum(1).abs().max()) < 1e-3 and not bool((Z == 7.0).all(1).any())
