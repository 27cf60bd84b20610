"""The gradients of the gated feed-forward block's weights on operands whose columns, or rows, differ in size: a row of dWg belongs to a column of X, a column
of it to a hidden column, a column of dWd to one of dY, and none of them sees the others."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from _rows import GatedFF, within  # noqa: E402
from _spread import LIMIT_GRADIENT, check_columns, powers  # noqa: E402
from test_gpu_gated_ff import pipad  # noqa: E402,F401
from test_gpu_gated_ff_columns import case  # noqa: E402

#: rows, F, hidden, Fo: every number of tiles of columns that there is a kernel for, four and eight waves, rows of more than 256 columns
KERNELS = [(300, 16, 43, 16), (300, 20, 60, 64), (300, 64, 256, 64), (3_000, 64, 171, 20), (700, 128, 60, 100), (700, 40, 70, 120), (700, 120, 70, 40), (700, 200, 130, 250),
           (700, 200, 70, 30), (700, 30, 70, 200), (700, 100, 70, 200), (700, 200, 70, 100), (700, 50, 70, 200), (700, 200, 70, 50), (600, 300, 130, 40), (700, 40, 130, 300),
           (513, 300, 70, 310)]


def compare(pipad, X, dY, W, b, activation, along, least=0.0):  # noqa: F811
    """Each element within its bound, and in the 2-norm the columns (0) and rows (1) of a gradient that `along` names: those whose entries are of about one
    size.  Where entries differ by 2^20 one of them is the norm, a single sum of random signs, and such a sum comes out at a hundredth of its terms' size in
    one case of a hundred, with the error of its terms."""
    got, want = pipad.gated_ff_backward([X], [dY], *W, *b, activation=activation, rows_grad=False), GatedFF(X, *W, *b, None, activation).backward(dY)
    for q, (value, bound) in want.items():
        if q != "dX":
            within(getattr(got, q), value, bound + least, q)
    for q, dims in along.items():
        for dim in dims:
            check_columns(getattr(got, q), want[q][0], dim, LIMIT_GRADIENT, q)


EVERY = {"dWg": (0, 1), "dWu": (0, 1), "dWd": (0, 1)}


@pytest.mark.parametrize("rows,F,hidden,Fo", KERNELS)
def test_columns_of_x(pipad, rows, F, hidden, Fo):  # noqa: F811
    gen, W, b, X, dY = case(rows, F, hidden, Fo, True)
    compare(pipad, X * powers(gen, F, -28), dY, W, b[:2], "silu", {"dWg": (1,), "dWu": (1,), "dWd": (0, 1)})


@pytest.mark.parametrize("rows,F,hidden,Fo", KERNELS)
def test_columns_of_x_that_weights_make_up_for(pipad, rows, F, hidden, Fo):  # noqa: F811
    gen, (Wg, Wu, Wd), b, X, dY = case(rows, F, hidden, Fo, True)
    d = powers(gen, F, -12, 12)
    compare(pipad, X * d, dY, (Wg / d[:, None], Wu / d[:, None], Wd), b[:2], "sigmoid", {"dWg": (1,), "dWu": (1,), "dWd": (0, 1)})


@pytest.mark.parametrize("rows,F,hidden,Fo", KERNELS)
def test_columns_of_dy(pipad, rows, F, hidden, Fo):  # noqa: F811
    gen, W, b, X, dY = case(rows, F, hidden, Fo, True)
    compare(pipad, X, dY * powers(gen, Fo, -28), W, b[:2], "gelu", {"dWg": (0, 1), "dWu": (0, 1), "dWd": (0,)})


@pytest.mark.parametrize("rows,F,hidden,Fo", KERNELS)
def test_hidden_columns(pipad, rows, F, hidden, Fo):  # noqa: F811
    gen, (Wg, Wu, Wd), _, X, dY = case(rows, F, hidden, Fo)
    d, e = powers(gen, hidden, -40), powers(gen, hidden, -12, 12)
    compare(pipad, X, dY, (Wg, Wu * d, Wd * e[:, None]), (None, None), "silu", {"dWg": (0,), "dWu": (0,), "dWd": (1,)})


@pytest.mark.parametrize("rows,F,hidden,Fo", KERNELS)
def test_rows_of_small_gradients_that_alone_have_a_feature(pipad, rows, F, hidden, Fo):  # noqa: F811
    """Every row has one of X's columns, and rows of the same column have gradients of the same size: 2^-28 to 1, side by side in every tile."""
    gen, W, b, X, dY = case(rows, F, hidden, Fo, True)
    at = torch.arange(rows, device="cuda") % F
    one = torch.zeros_like(X)
    one[torch.arange(rows, device="cuda"), at] = X[:, 0]
    # (X's values differ as well, so that terms differ by more than 2^-29 in all: those have 2^-51 of the largest, twice for dG and for what is added up)
    compare(pipad, one, dY * powers(gen, F, -28)[at][:, None], W, b[:2], "silu", {}, least=2.0 ** -50 * 3 * float((X[:, 0].abs() * dY.norm(dim=1)).max()))


@pytest.mark.parametrize("value", [1e9, 1e30, float("inf"), float("nan")])
@pytest.mark.parametrize("rows,F,hidden,Fo", KERNELS)
def test_a_huge_weight_is_one_hidden_column_s_matter(pipad, rows, F, hidden, Fo, value):  # noqa: F811
    _, W, b, X, dY = case(rows, F, hidden, Fo, True)
    h = hidden // 2
    others = [c for c in range(hidden) if c != h]
    run = lambda: pipad.gated_ff_backward([X], [dY], *W, *b[:2], rows_grad=False)  # noqa: E731
    want = run()
    for q, at in ((0, (3, h)), (1, (3, h)), (2, (h, 3))):
        before = float(W[q][at])
        W[q][at] = value
        got = run()
        W[q][at] = before
        for name in ("dWg", "dWu"):
            assert torch.equal(getattr(got, name)[:, others], getattr(want, name)[:, others]), (q, name)
        for name in ("dWd", "dbg", "dbu"):
            assert torch.equal(getattr(got, name)[others], getattr(want, name)[others]), (q, name)


@pytest.mark.parametrize("rows,F,hidden,Fo", KERNELS)
def test_every_kernel_keeps_the_bits(pipad, rows, F, hidden, Fo):  # noqa: F811
    for activation in ("silu", "gelu", "sigmoid"):
        _, W, b, X, dY = case(rows, F, hidden, Fo, True)
        compare(pipad, X, dY, W, b[:2], activation, EVERY)
