"""The gated feed-forward block and the gradient of X on weights whose columns differ in size: a column of the result is the product of its own column of
weights, whatever the others hold."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from _rows import GatedFF, within  # noqa: E402
from _spread import LIMIT, LIMIT_GRADIENT, check_columns, powers  # noqa: E402
from test_gpu_gated_ff import pipad, weights  # noqa: E402,F401

#: rows, F, hidden, Fo: one of each kernel, on both sides of their rules
KERNELS = [(256, 64, 256, 64), (257, 64, 256, 64), (300, 20, 60, 20), (300, 200, 130, 150), (17_000, 64, 130, 60), (17_000, 16, 43, 16), (17_000, 200, 130, 150),
           (400, 300, 130, 40), (600, 300, 130, 40), (600, 40, 130, 300), (2_000, 520, 70, 530)]


def case(rows, F, hidden, Fo, bias=False, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed + rows + F + hidden + Fo)
    W, b = weights(gen, F, hidden, Fo, bias)
    return gen, W, b, torch.randn((rows, F), device="cuda", generator=gen), torch.randn((rows, Fo), device="cuda", generator=gen)


@pytest.mark.parametrize("rows,F,hidden,Fo", KERNELS)
def test_columns_of_y_have_a_scale_of_their_own(pipad, rows, F, hidden, Fo):  # noqa: F811
    gen, (Wg, Wu, Wd), _, X, _ = case(rows, F, hidden, Fo)
    y = pipad.gated_ff([X], Wg, Wu, Wd)[0]
    d = powers(gen, Fo, -60, 20)
    assert torch.equal(pipad.gated_ff([X], Wg, Wu, Wd * d)[0], y * d)
    want = GatedFF(X, Wg, Wu, Wd * d, None, None, None, "silu").forward()
    within(y * d, *want, "Y")
    check_columns(y * d, want[0], 0, LIMIT["Y"], "Y")


@pytest.mark.parametrize("value", [1e9, 1e30, float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("rows,F,hidden,Fo", KERNELS)
def test_a_huge_weight_is_one_column_s_matter(pipad, rows, F, hidden, Fo, value):  # noqa: F811
    _, W, b, X, _ = case(rows, F, hidden, Fo, True)
    y = pipad.gated_ff([X], *W, *b)[0]
    W[2][hidden // 2, 5] = value
    y2, others = pipad.gated_ff([X], *W, *b)[0], [c for c in range(Fo) if c != 5]
    assert torch.equal(y[:, others], y2[:, others])
    if abs(value) < 1e38:
        check_columns(y2[:, 5:6], GatedFF(X, *W, *b, "silu").forward()[0][:, 5:6], 0, LIMIT["Y"], "Y")
    else:
        assert not bool(y2[:, 5].isfinite().any())


@pytest.mark.parametrize("rows,F,hidden,Fo", KERNELS)
def test_columns_of_dx_have_a_scale_of_their_own(pipad, rows, F, hidden, Fo):  # noqa: F811
    """Every second column of X is 0, so that G and U do not see these rows of Wg and Wu, and dX sees them in a column each."""
    gen, (Wg, Wu, Wd), _, X, dY = case(rows, F, hidden, Fo)
    X[:, ::2] = 0.0
    d = torch.ones(F, device="cuda")
    d[::2] = powers(gen, (F + 1) // 2, -60)
    run = lambda Wg, Wu: pipad.gated_ff_backward([X], [dY], Wg, Wu, Wd, weights=False, biases=False).dX[0]  # noqa: E731
    dx, dx2 = run(Wg, Wu), run(Wg * d[:, None], Wu * d[:, None])
    assert torch.equal(dx2, dx * d)
    want = GatedFF(X, Wg * d[:, None], Wu * d[:, None], Wd, None, None, None, "silu").backward(dY)["dX"]
    within(dx2, *want, "dX")
    check_columns(dx2, want[0], 0, LIMIT_GRADIENT, "dX")


@pytest.mark.parametrize("value", [1e9, 1e30])
@pytest.mark.parametrize("rows,F,hidden,Fo", KERNELS)
def test_a_huge_weight_is_one_column_of_dx_s_matter(pipad, rows, F, hidden, Fo, value):  # noqa: F811
    """Of a hidden column that Y does not see (a row of zeros in Wd), so that dG and dU of it are 0."""
    _, (Wg, Wu, Wd), (bg, bu, _), X, dY = case(rows, F, hidden, Fo, True)
    h = hidden // 2
    Wd[h] = 0.0
    run = lambda: pipad.gated_ff_backward([X], [dY], Wg, Wu, Wd, bg, bu, weights=False, biases=False).dX[0]  # noqa: E731
    dx = run()
    Wg[4, h], Wu[6, h] = value, -value
    dx2, others = run(), [f for f in range(F) if f not in (4, 6)]
    assert torch.equal(dx[:, others], dx2[:, others])


@pytest.mark.parametrize("rows,F,hidden,Fo", KERNELS)
def test_hidden_columns_have_a_scale_of_their_own(pipad, rows, F, hidden, Fo):  # noqa: F811
    """Wu's columns and Wd's rows times powers of two that cancel: floats give the same Y and dX, bit by bit."""
    gen, (Wg, Wu, Wd), _, X, dY = case(rows, F, hidden, Fo)
    d = powers(gen, hidden, -12, 12)
    Wu, Wd = Wu * d, Wd / d[:, None]
    want = GatedFF(X, Wg, Wu, Wd, None, None, None, "gelu")
    y, (value, bound) = pipad.gated_ff([X], Wg, Wu, Wd, activation="gelu")[0], want.forward()
    within(y, value, bound, "Y")
    check_columns(y, value, 0, LIMIT["Y"], "Y")
    dx, (value, bound) = pipad.gated_ff_backward([X], [dY], Wg, Wu, Wd, activation="gelu", weights=False, biases=False).dX[0], want.backward(dY)["dX"]
    within(dx, value, bound, "dX")
    check_columns(dx, value, 0, LIMIT_GRADIENT, "dX")


@pytest.mark.parametrize("rows,F,hidden,Fo", KERNELS)
def test_columns_of_x_that_weights_make_up_for(pipad, rows, F, hidden, Fo):  # noqa: F811
    """X's columns and Wg's and Wu's rows times powers of two that cancel."""
    gen, (Wg, Wu, Wd), _, X, dY = case(rows, F, hidden, Fo)
    d = powers(gen, F, -12, 12)
    X, Wg, Wu = X * d, Wg / d[:, None], Wu / d[:, None]
    want = GatedFF(X, Wg, Wu, Wd, None, None, None, "sigmoid")
    y, (value, bound) = pipad.gated_ff([X], Wg, Wu, Wd, activation="sigmoid")[0], want.forward()
    within(y, value, bound, "Y")
    check_columns(y, value, 0, LIMIT["Y"], "Y")
    dx, (value, bound) = pipad.gated_ff_backward([X], [dY], Wg, Wu, Wd, activation="sigmoid", weights=False, biases=False).dX[0], want.backward(dY)["dX"]
    within(dx, value, bound, "dX")
    check_columns(dx, value, 0, LIMIT_GRADIENT, "dX")


@pytest.mark.parametrize("rows,F,hidden,Fo", KERNELS)
def test_every_kernel_keeps_the_bits(pipad, rows, F, hidden, Fo):  # noqa: F811
    """Columns of about one size, with biases: errors in the 2-norm, for each choice of kernels."""
    for activation in ("silu", "gelu", "sigmoid", "relu"):
        _, W, b, X, dY = case(rows, F, hidden, Fo, True)
        want = GatedFF(X, *W, *b, activation)
        check_columns(pipad.gated_ff([X], *W, *b, activation=activation)[0], want.forward()[0], 0, LIMIT["Y"], "Y")
        if activation != "relu":  # (whose slope jumps where G changes sign)
            dx = pipad.gated_ff_backward([X], [dY], *W, *b[:2], activation=activation, weights=False, biases=False).dX[0]
            check_columns(dx, want.backward(dY)["dX"][0], 0, LIMIT_GRADIENT, "dX")


@pytest.mark.parametrize("rows,F,hidden,Fo", KERNELS)
def test_large_hidden_values_and_small_weights(pipad, rows, F, hidden, Fo):  # noqa: F811
    """H of 1e35 and more, where floats end at 3e38, and weights that bring Y and dX back: what lies between has to stay inside, too."""
    _, (Wg, Wu, Wd), _, X, dY = case(rows, F, hidden, Fo)
    Wg, Wu, Wd = Wg * 1e18, Wu * 1e17, Wd * 1e-30
    want = GatedFF(X, Wg, Wu, Wd, None, None, None, "relu")
    check_columns(pipad.gated_ff([X], Wg, Wu, Wd, activation="relu")[0], want.forward()[0], 0, LIMIT["Y"], "Y")
    Wg, Wu, Wd = Wg * 1e-48, Wu * 1e-17, Wd * 1e30  # dU of 1e35, dG of 1e35, of weights of 1e-30
    Wu = Wu * 1e-30
    dy = dY * 1e35
    bg, bu = torch.ones(hidden, device="cuda"), torch.ones(hidden, device="cuda")
    want = GatedFF(X, Wg, Wu, Wd, bg, bu, None, "silu").backward(dy)["dX"][0]
    check_columns(pipad.gated_ff_backward([X], [dy], Wg, Wu, Wd, bg, bu, weights=False, biases=False).dX[0], want, 0, LIMIT_GRADIENT, "dX")
