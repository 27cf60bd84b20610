"""The gated feed-forward block and its gradients against their definition in 64 bits, element by element, within bounds derived from
the roundings (_rows.py)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from _rows import LAYOUTS, GatedFF, fill_with, room, stacked, untouched, within  # noqa: E402


@pytest.fixture(scope="module")
def pipad():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2301_00391_amd as p
    p.load_library()
    return p


def weights(gen, F, hidden, Fo, bias, pad=0):
    def w(r, c):
        return (torch.randn((r, c + pad), device="cuda", generator=gen) / r ** 0.5)[:, :c]
    b = [torch.randn(c, device="cuda", generator=gen) * 0.3 if bias else None for c in (hidden, hidden, Fo)]
    return [w(F, hidden), w(F, hidden), w(hidden, Fo)], b


def operands(gen, layout, n, k, F, scale=1.0, spread=False):
    whole, x = room(layout, n, k, F)
    v = torch.randn((k, n, F), device="cuda", generator=gen) * scale
    if spread:  # (magnitudes from 2^-20 to 2^10 within a row)
        v *= torch.exp2(torch.randint(-20, 11, (k, n, F), device="cuda", generator=gen).float())
    return whole, fill_with(x, v)


def check(pipad, n, k, F, hidden, Fo, activation, layout="list", bias=True, pad=0, seed=0, spread=False):
    gen = torch.Generator(device="cuda").manual_seed(seed + n + 31 * F + 7 * hidden + Fo)
    W, b = weights(gen, F, hidden, Fo, bias, pad)
    _, X = operands(gen, layout, n, k, F, spread=spread)
    _, dY = operands(gen, layout, n, k, Fo, 0.1)
    whole_y, Y = room(layout, n, k, Fo)
    whole_dx, dX = room(layout, n, k, F)
    want = GatedFF(stacked(X), *W, *b, activation)
    pipad.gated_ff(X, *W, *b, activation=activation, Y=Y)
    within(stacked(Y), *want.forward(), "Y")
    assert untouched(whole_y, Y)
    got = pipad.gated_ff_backward(X, dY, *W, *b[:2], activation=activation, dX=dX)
    for q, (value, bound) in want.backward(stacked(dY)).items():
        g = getattr(got, q)
        within(stacked(g) if q == "dX" else g, value, bound, q)
    assert untouched(whole_dx, dX)


WIDTHS = [(1, 1, 1), (2, 8, 2), (6, 16, 6), (7, 33, 5), (16, 43, 16), (16, 64, 17), (31, 32, 33), (32, 128, 32), (33, 90, 100), (60, 31, 64),
          (64, 171, 64), (64, 256, 64), (65, 100, 128), (100, 77, 31), (128, 341, 100), (128, 65, 128), (129, 40, 3), (3, 40, 129), (200, 130, 256),
          (256, 70, 200), (256, 40, 256), (140, 20, 60), (90, 50, 161), (300, 33, 20), (17, 1000, 290), (257, 40, 300), (320, 70, 257)]


@pytest.mark.parametrize("activation", ["sigmoid", "gelu", "silu"])
@pytest.mark.parametrize("F,hidden,Fo", WIDTHS)
def test_every_width(pipad, F, hidden, Fo, activation):
    check(pipad, 131, 2, F, hidden, Fo, activation, layout="padded" if F % 2 else "list", bias=activation != "gelu")


@pytest.mark.parametrize("n,k", [(1, 1), (1, 32), (2, 1), (3, 7), (5, 1), (15, 1), (16, 1), (17, 1), (31, 1), (32, 1), (33, 1), (63, 2), (64, 1), (127, 1), (128, 1),
                                 (129, 3), (511, 1), (700, 32)])
@pytest.mark.parametrize("F,hidden,Fo", [(16, 43, 16), (64, 100, 60), (150, 64, 40), (270, 64, 20)])
def test_every_number_of_rows(pipad, n, k, F, hidden, Fo):
    check(pipad, n, k, F, hidden, Fo, "silu")


@pytest.mark.parametrize("activation", ["silu", "gelu", "sigmoid"])
@pytest.mark.parametrize("F,hidden,Fo", [(1, 97, 1), (16, 129, 40), (40, 250, 20), (33, 97, 100), (100, 160, 97), (70, 300, 250), (200, 128, 130), (256, 257, 256), (150, 97, 5)])
@pytest.mark.parametrize("n,k,layout", [(257, 1, "list"), (100, 3, "padded"), (33, 32, "list")])
def test_every_width_of_four_or_more_hidden_tiles(pipad, F, hidden, Fo, activation, n, k, layout):
    check(pipad, n, k, F, hidden, Fo, activation, layout=layout, bias=activation != "gelu")


@pytest.mark.parametrize("F,hidden,Fo", [(257, 33, 20), (290, 160, 300), (530, 130, 40), (40, 130, 530), (700, 97, 260), (1100, 40, 3), (600, 257, 1060)])
@pytest.mark.parametrize("n,k", [(2100, 1), (70, 31), (512, 1), (513, 1)])
def test_rows_of_more_than_256_columns(pipad, F, hidden, Fo, n, k):
    check(pipad, n, k, F, hidden, Fo, "silu", layout="padded" if F % 4 else "list")


@pytest.mark.parametrize("rows", [255, 256, 257, 4095, 4096, 4097, 8191, 8192, 8193, 16383, 16384, 16385])
@pytest.mark.parametrize("F,hidden,Fo", [(16, 96, 16), (16, 97, 16), (40, 97, 150), (150, 97, 40)])
def test_rows_on_both_sides_of_a_choice(pipad, rows, F, hidden, Fo):
    check(pipad, rows, 1, F, hidden, Fo, "silu")


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("F,hidden,Fo,pad", [(16, 40, 16, 0), (64, 96, 64, 3), (30, 50, 70, 1), (160, 40, 140, 4), (260, 40, 30, 4), (30, 33, 300, 0)])
def test_every_layout(pipad, layout, F, hidden, Fo, pad):
    check(pipad, 77, 3, F, hidden, Fo, "gelu", layout=layout, pad=pad)


@pytest.mark.parametrize("F,hidden,Fo", [(20, 50, 20), (64, 128, 64), (128, 60, 90)])
def test_products_keep_the_last_bits_over_a_wide_range_of_magnitudes(pipad, F, hidden, Fo):
    check(pipad, 200, 1, F, hidden, Fo, "sigmoid", spread=True)


@pytest.mark.parametrize("rows", [300, 17000])
@pytest.mark.parametrize("F,hidden,Fo", [(20, 100, 20), (64, 128, 64), (128, 130, 90), (250, 99, 100)])
def test_products_keep_the_last_bits_in_every_kernel(pipad, rows, F, hidden, Fo):
    check(pipad, rows, 1, F, hidden, Fo, "sigmoid", spread=True)


@pytest.mark.parametrize("F,hidden,Fo", [(16, 40, 16), (64, 90, 64), (130, 40, 20), (256, 40, 20), (20, 40, 300)])
def test_relu_has_no_slope_at_zero(pipad, F, hidden, Fo):
    """Small whole numbers: G is exact, with many zeros, so its sign is no matter of rounding."""
    gen = torch.Generator(device="cuda").manual_seed(F)
    whole = lambda *s: torch.randint(-1, 2, s, device="cuda", generator=gen).float()  # noqa: E731
    X, dY = [whole(150, F) for _ in range(2)], [whole(150, Fo) for _ in range(2)]
    Wg, Wu, Wd = whole(F, hidden), whole(F, hidden), whole(hidden, Fo)
    want = GatedFF(stacked(X), Wg, Wu, Wd, None, None, None, "relu")
    assert bool((want.G == 0).any())
    assert torch.equal(stacked(pipad.gated_ff(X, Wg, Wu, Wd, activation="relu")).double(), want.forward()[0])
    got = pipad.gated_ff_backward(X, dY, Wg, Wu, Wd, activation="relu")
    for q, (value, bound) in want.backward(stacked(dY)).items():
        within(stacked(got.dX) if q == "dX" else getattr(got, q), value, bound, q)


def test_empty_and_partial_results(pipad):
    gen = torch.Generator(device="cuda").manual_seed(1)
    W, b = weights(gen, 10, 20, 12, True)
    X, dY = [torch.empty((0, 10), device="cuda")] * 3, [torch.empty((0, 12), device="cuda")] * 3
    assert pipad.gated_ff(X, *W, *b)[2].shape == (0, 12)
    got = pipad.gated_ff_backward(X, dY, *W, *b[:2])
    assert all(bool((g == 0).all()) for g in got[1:]) and got.dWd.shape == (20, 12)
    X, dY = torch.randn((50, 2, 10), device="cuda"), torch.randn((50, 2, 12), device="cuda")
    every = pipad.gated_ff_backward(X, dY, *W, *b[:2])
    for keywords, there in (({"rows_grad": False}, range(1, 7)), ({"weights": False}, (0, 4, 5, 6)), ({"biases": False}, range(4)),
                            ({"weights": False, "biases": False}, (0,))):
        some = pipad.gated_ff_backward(X, dY, *W, *b[:2], **keywords)
        for q, (x, y) in enumerate(zip(some, every)):
            assert (x is None) == (q not in there) and (x is None or torch.equal(x, y))


def test_rows_do_not_see_each_other(pipad):
    """A row that is not finite spoils itself alone, whatever shares its tile."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    for n, F, hidden, Fo in ((1, 64, 50, 64), (5, 64, 50, 64), (300, 64, 50, 64), (300, 64, 150, 64), (900, 150, 150, 140), (900, 150, 50, 140), (900, 300, 50, 40)):
        W, b = weights(gen, F, hidden, Fo, True)
        X, dY = torch.randn((n, 3, F), device="cuda", generator=gen), torch.randn((n, 3, Fo), device="cuda", generator=gen)
        for bad in (float("inf"), float("nan"), -float("inf")):
            X2, dY2 = X.clone(), dY.clone()
            X2[n // 2, 1, 3] = bad
            keep = torch.ones((n, 3), dtype=torch.bool, device="cuda")
            keep[n // 2, 1] = False
            y, y2 = pipad.gated_ff(X, *W, *b), pipad.gated_ff(X2, *W, *b)
            assert torch.equal(y[keep], y2[keep]) and not bool(y2[n // 2, 1].isfinite().any())
            dY2[n // 2, 1, 2] = bad
            d, d2 = pipad.gated_ff_backward(X, dY, *W, *b[:2]).dX, pipad.gated_ff_backward(X2, dY2, *W, *b[:2]).dX
            assert torch.equal(d[keep], d2[keep]) and not bool(d2[n // 2, 1].isfinite().any())


@pytest.mark.parametrize("n,k", [(1, 1), (9, 2), (3000, 3)])
def test_same_bits_again_on_another_stream_and_in_a_graph(pipad, n, k):
    gen = torch.Generator(device="cuda").manual_seed(3)
    F, hidden, Fo = 64, 100, 48
    W, b = weights(gen, F, hidden, Fo, True)
    X, dY = [torch.randn((n, F), device="cuda", generator=gen) for _ in range(k)], [torch.randn((n, Fo), device="cuda", generator=gen) for _ in range(k)]

    def both(stream=None):
        return [*pipad.gated_ff(X, *W, *b, stream=stream), *pipad.gated_ff_backward(X, dY, *W, *b[:2], stream=stream)[1:],
                *pipad.gated_ff_backward(X, dY, *W, *b[:2], stream=stream).dX]

    want = both()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = both(side)  # (tensors of the current stream, work on another one)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = both()
        graphs.append((graph, outs))
    for replay in range(3):
        for x in X:
            x.normal_(generator=gen)
        want = both()
        torch.cuda.synchronize()
        for graph, outs in graphs:
            for o in outs:
                o.fill_(float("nan"))
            graph.replay()
        torch.cuda.synchronize()
        for _, outs in graphs:
            assert all(torch.equal(x, y) for x, y in zip(want, outs)), replay


def test_workspace_is_all_that_is_written(pipad):
    """The workspace of the size that is asked for, with a guard behind it, whatever it held before."""
    from paper_2301_00391_amd import rows
    lib = pipad.load_library()
    gen = torch.Generator(device="cuda").manual_seed(4)
    for n, k, F, hidden, Fo in ((1, 1, 64, 256, 64), (4, 2, 30, 50, 7), (900, 3, 64, 171, 60), (7000, 3, 64, 171, 60), (300, 2, 140, 33, 150), (1200, 2, 140, 33, 150), (1200, 2, 260, 33, 150)):
        W, b = weights(gen, F, hidden, Fo, True)
        X, dY = [torch.randn((n, F), device="cuda", generator=gen) for _ in range(k)], [torch.randn((n, Fo), device="cuda", generator=gen) for _ in range(k)]
        block = rows._ff_struct(rows._Rows(X, "X"), F, *W, *b, "silu")[0]
        for backward in (0, 1):
            need = ctypes.c_size_t()
            assert lib.pipad_gated_ff_workspace(block, n, k, backward, ctypes.byref(need)) == 0
            seen = []
            for fill in (0, 255):
                ws = torch.full((need.value + 4096,), fill, dtype=torch.uint8, device="cuda")
                part = ws[:need.value]
                if backward:
                    d = pipad.gated_ff_backward(X, dY, *W, *b[:2], workspace=part)
                    seen.append([*d.dX, *d[1:]])
                else:
                    seen.append(pipad.gated_ff(X, *W, *b, workspace=part))
                assert bool((ws[need.value:] == fill).all())
            assert all(torch.equal(x, y) for x, y in zip(*seen))
            with pytest.raises(pipad.PipadError) as why:
                if backward:
                    pipad.gated_ff_backward(X, dY, *W, *b[:2], workspace=ws[:need.value - 16])
                else:
                    pipad.gated_ff(X, *W, *b, workspace=ws[:need.value - 16])
            assert why.value.status == -6


def test_rows_past_32_bit_offsets(pipad):
    """Matrices of more than 2^32 elements: the rows at both ends and around 2^31 and 2^32 elements."""
    n, F, hidden = 35_000_000, 128, 24
    gen = torch.Generator(device="cuda").manual_seed(5)
    W, b = weights(gen, F, hidden, 4, True)
    X, dY = torch.zeros((n, F), device="cuda"), torch.zeros((n, 4), device="cuda")
    some = torch.cat([torch.arange(a, a + 40, device="cuda") for a in (0, 2 ** 31 // F - 20, 2 ** 32 // F - 20, n - 40)])
    X[some] = torch.randn((some.numel(), F), device="cuda", generator=gen)
    dY[some] = torch.randn((some.numel(), 4), device="cuda", generator=gen)
    want = GatedFF(X[some], *W, *b, "silu")
    within(pipad.gated_ff([X], *W, *b)[0][some], *want.forward(), "Y")
    got, back = pipad.gated_ff_backward([X], [dY], *W, *b[:2]), want.backward(dY[some])
    within(got.dX[0][some], *back["dX"], "dX")
    for q in ("dWg", "dWu", "dWd"):  # (the other rows' terms are exact zeros)
        within(getattr(got, q), *back[q], q)


@pytest.mark.parametrize("rows,F,hidden,Fo", [(300_000, 64, 64, 64), (120_007, 128, 90, 100), (2_000_003, 16, 32, 16)])
def test_many_rows(pipad, rows, F, hidden, Fo):
    """Sums over many rows: within 2e-6 of the definition, in the 2-norm (random signs: errors of a long chain of additions grow with its
    root: 2^-24 times the root of some 2^14 additions between a chain's start and the parts' sums is 8e-6 at worst, half of it on average
    as the sum grows, a third of that as roundings are spread evenly)."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    W, b = weights(gen, F, hidden, Fo, True)
    X, dY = torch.randn((rows, F), device="cuda", generator=gen), torch.randn((rows, Fo), device="cuda", generator=gen)
    got = pipad.gated_ff_backward([X], [dY], *W, *b[:2], activation="gelu")
    y = pipad.gated_ff([X], *W, *b, activation="gelu")[0]
    want = GatedFF(X, *W, *b, "gelu")
    assert float((y - want.forward()[0]).norm() / want.forward()[0].norm()) < 1e-6
    for q, (value, _) in want.backward(dY).items():
        g = got.dX[0] if q == "dX" else getattr(got, q)
        assert float((g - value).norm() / value.norm()) < 2e-6, q


def test_tensors_that_do_not_fit(pipad):
    gen = torch.Generator(device="cuda").manual_seed(6)
    W, b = weights(gen, 8, 20, 6, True)
    X, dY = torch.zeros((5, 2, 8), device="cuda"), torch.zeros((5, 2, 6), device="cuda")
    wrong = [lambda: pipad.gated_ff(X, W[0].cpu(), *W[1:], *b), lambda: pipad.gated_ff(X, *W[:2], W[2].cpu(), *b), lambda: pipad.gated_ff(X, *W, b[0].cpu(), *b[1:]),
             lambda: pipad.gated_ff(X, W[0].double(), *W[1:]), lambda: pipad.gated_ff(X, W[0].T, *W[1:]), lambda: pipad.gated_ff(X, W[0], W[1][:, :10], W[2]),
             lambda: pipad.gated_ff(X, *W, b[2]), lambda: pipad.gated_ff(X, *W, activation="tanh"), lambda: pipad.gated_ff(X, *W, activation=None),
             lambda: pipad.gated_ff(X, *W, Y=X), lambda: pipad.gated_ff(X, *W, Y=[dY[:, 0]]), lambda: pipad.gated_ff(X, *W, Y=dY.cpu()),
             lambda: pipad.gated_ff(X, *W, Y=dY[:4]), lambda: pipad.gated_ff(X[:, :, ::2], W[0][:4], W[1][:4], W[2]),
             lambda: pipad.gated_ff(X.half(), *W), lambda: pipad.gated_ff(X, *W, workspace=torch.zeros(1 << 20)),
             lambda: pipad.gated_ff_backward(X, X, *W), lambda: pipad.gated_ff_backward(X, dY.cpu(), *W),
             lambda: pipad.residual_norm(X, X.cpu()), lambda: pipad.residual_norm(X, X[:, :, :4]), lambda: pipad.residual_norm(X, X, dY),
             lambda: pipad.residual_norm(X, pre="batch"), lambda: pipad.residual_norm(X, w_pre=b[0]), lambda: pipad.residual_norm(X, X, scale=torch.zeros(8))]
    for call in wrong:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: pipad.residual_norm(X, gate=X), lambda: pipad.residual_norm(X, scale=torch.zeros(8, device="cuda")), lambda: pipad.residual_norm(X, pre=None),
                 lambda: pipad.residual_norm_backward(X), lambda: pipad.gated_ff_backward(X, dY, *W, rows_grad=False, weights=False, biases=False),
                 lambda: pipad.gated_ff(X, *W, workspace=torch.zeros(1, device="cuda"))):
        with pytest.raises(pipad.PipadError):
            call()


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("n,k", [(1, 1), (40, 3), (0, 2), (70, 32)])
def test_same_bits_with_and_without_the_native_half(pipad, monkeypatch, layout, n, k):
    from paper_2301_00391_amd import binding
    gen = torch.Generator(device="cuda").manual_seed(11)
    F, hidden, Fo = 20, 50, 12
    W, b = weights(gen, F, hidden, Fo, True, 1)
    ops = [operands(gen, layout, n, k, F)[1] for _ in range(5)]
    dY = operands(gen, layout, n, k, Fo)[1]
    v = [torch.randn(F, device="cuda", generator=gen) for _ in range(5)]
    seen, host = [], binding._host
    assert host is not None
    made = []

    class Seen:
        def __getattr__(self, name):
            return lambda *args: made.append(getattr(host, name)(*args)) or made[-1]

    for half in (Seen(), None):
        monkeypatch.setattr(binding, "_host", half)
        outs = [room(layout, n, k, F)[1] for _ in range(6)]
        Y = room(layout, n, k, Fo)[1]
        pipad.gated_ff(ops[0], *W, *b, Y=Y)
        d = pipad.gated_ff_backward(ops[0], dY, *W, *b[:2], dX=outs[0])
        some = pipad.gated_ff_backward(ops[0], dY, *W, *b[:2], rows_grad=False, weights=False)
        pipad.residual_norm(ops[0], ops[1], ops[2], post="rms", pre="layer", scale=v[0], w_post=v[1], b_post=v[2], w_pre=v[3], b_pre=v[4], R_out=outs[1], Z=outs[2])
        e = pipad.residual_norm_backward(outs[1], ops[3], ops[4], ops[1], ops[2], post="rms", pre="layer", scale=v[0], w_post=v[1], b_post=v[2], w_pre=v[3],
                                         dR=outs[3], dB=outs[4], dgate=outs[5])
        less = pipad.residual_norm_backward(outs[1], ops[3], None, ops[1], post="rms", pre="layer", dR=outs[3], dB=outs[4], biases=False)
        torch.cuda.synchronize()
        seen.append([stacked(Y), *map(stacked, outs), *d[1:], *some[4:], *e[3:], less.dscale, less.dw_post, less.dw_pre])
        assert some[:4] == (None,) * 4 and less.db_post is None and less.db_pre is None and less.dgate is None
    assert all(torch.equal(x, y) for x, y in zip(*seen))
    assert len(made) == 6 and all(m is not None for m in made)


def test_weights_of_more_values_than_a_launch_has_threads_for(pipad):
    """One row, so that every gradient is a product of two vectors; 64 values a workgroup of 256 threads: 2^30 of them are 2^32 threads."""
    F, hidden, Fo = 17000, 22000, 15000
    gen = torch.Generator(device="cuda").manual_seed(13)
    W, _ = weights(gen, F, hidden, Fo, False)
    assert 2 * F * hidden + hidden * Fo > 1 << 30
    X, dY = torch.randn((1, F), device="cuda", generator=gen), torch.randn((1, Fo), device="cuda", generator=gen)
    got = pipad.gated_ff_backward([X], [dY], *W, rows_grad=False)
    G, U = ((X.double() @ w.double())[0] for w in W[:2])
    dH = (W[2].double() @ dY[0].double())
    s = torch.sigmoid(G)
    # Sums of 2^14 products of random signs, a root of it times their size off by 2^-22 each at most (2^-22 for both factors, 2^-24 for the
    # additions): some 1e-6 of the sums' own size on average, 1e-5 at the worst of 2^14 of them.
    for name, g, want in (("dWg", got.dWg, torch.outer(X[0].double(), dH * U * s * (1 + G * (1 - s)))), ("dWu", got.dWu, torch.outer(X[0].double(), dH * G * s)),
                          ("dWd", got.dWd, torch.outer(G * s * U, dY[0].double()))):
        error = float((g - want).norm() / want.norm())
        assert error < 1e-5, (name, error)
        del want
