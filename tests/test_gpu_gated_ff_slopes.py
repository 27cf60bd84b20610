"""The slopes of the activations where a gate is wide open or closed, relative to the slope itself."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from _rows import U, stacked, within  # noqa: E402
from test_gpu_gated_ff import pipad  # noqa: E402,F401


@pytest.mark.parametrize("gate", [-80.0, -30.0, -20.0, -12.0, -5.0, -0.5, 0.5, 5.0, 12.0, 16.0, 20.0, 30.0, 80.0])
@pytest.mark.parametrize("activation", ["sigmoid", "silu"])
@pytest.mark.parametrize("rows,hidden", [(40, 64), (300, 128), (20_000, 128), (600, 300)])
def test_slopes_keep_their_bits(pipad, rows, hidden, activation, gate):  # noqa: F811
    """X = 0, so that G and U are their biases exactly; dH = 1, Wg the unit matrix and Wu 0, so that a row of dX is the slope times U, and dbg is
    the number of rows times it.  U is 1, or where sigmoid's slope is small beside sigmoid a power of two that brings dG to dU's size: the
    two share a scale."""
    X, dY = torch.zeros((rows, 1, hidden), device="cuda"), torch.ones((rows, 1, 1), device="cuda")
    Wg, Wu, Wd = torch.eye(hidden, device="cuda"), torch.zeros((hidden, hidden), device="cuda"), torch.ones((hidden, 1), device="cuda")
    bg, bu = torch.full((hidden,), gate, device="cuda"), torch.full((hidden,), 2.0 ** round(max(gate, 0.0) / math.log(2)) if activation == "sigmoid" else 1.0, device="cuda")
    got = pipad.gated_ff_backward(X, dY, Wg, Wu, Wd, bg, bu, activation=activation)
    g = bg.double()
    s, rest = torch.sigmoid(g), torch.sigmoid(-g)  # (1 - s is not rest in 64 bits, either)
    slope = s * rest if activation == "sigmoid" else s * (1 + g * rest)
    # What the slope is the sum of: one exponential's argument is rounded (its rounding comes out times the argument), twelve more roundings and the
    # products' pieces, off by 4 U each of two; sums of equal values over 32 rows, with what they lose carried on, and over the parts 64 more.
    parts = bu.double() * (slope.abs() if activation == "sigmoid" else s + (g * s * rest).abs())
    slope = slope * bu.double()
    bound = (2 * abs(gate) + 32) * U * parts + 1e-37
    within(stacked(got.dX), slope.expand(rows, hidden), bound.expand(rows, hidden), "dX")
    within(got.dbg, rows * slope, rows * (bound + 64 * U * parts), "dbg")
