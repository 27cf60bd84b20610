"""The gradients of the vectors that all rows share, as sums over many rows."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from _rows import U  # noqa: E402
from test_gpu_gated_ff import pipad  # noqa: E402,F401


@pytest.mark.parametrize("F,lanes,per_lane", [(2, 1, 2), (4, 1, 4), (14, 8, 2), (16, 4, 4), (34, 16, 3), (126, 32, 4), (128, 32, 4), (256, 64, 4), (300, 64, 8), (302, 64, 8),
                                              (600, 64, 16), (1500, 256, 16), (1502, 256, 16)])
def test_equal_terms(pipad, F, lanes, per_lane):  # noqa: F811
    """Rows of +1 and -1 by turns under eps = 0 are their own norms, and equal gradients c of R_out and Z then have no mean along them: g = 2 c, exactly,
    and every sum is one of equal terms, as many a lane as 2048 workgroups leave it.  c is 1 and a little less than half of the last step that a sum of
    1 has beyond half of them: a plain chain of additions loses that each time, terms / 4 U in all.  A sum that carries what it rounds off is off by 2 U, one
    of chains of 64 by 64 U and 1 U for each chain; the sums of lanes and workgroups are equal numbers, two at a time, and exact, but for three
    columns a lane, whose 2048 workgroups are no power of two of rows: 21 additions at most."""
    terms = 256 if per_lane <= 4 else 1024
    n = 2048 * (256 // lanes) * terms
    c = 1.0 + terms * 2.0 ** -25 - 2.0 ** -23
    rows = torch.ones((n, F), device="cuda")
    rows[:, 1::2] = -1.0
    d = torch.full((n, F), c, device="cuda")
    assert float(d[0, 0]) == c
    got = pipad.residual_norm_backward([rows], [d], [d], [rows], post="rms", pre="rms", eps=0.0, dR=[torch.empty_like(d)], dB=[torch.empty_like(d)])
    assert bool((got.dR[0] == 2 * c).all())
    sign, most = rows[0].double(), (2 if per_lane <= 4 else 64 + terms / 64) + 21
    assert most < terms / 4
    for q, want in (("dscale", 2 * c * n * sign), ("dw_post", 2 * c * n * sign), ("db_post", 2 * c * n * sign.abs()), ("dw_pre", c * n * sign),
                    ("db_pre", c * n * sign.abs())):
        off = float(((getattr(got, q).double() - want).abs() / want.abs()).max())
        assert off <= most * U, (q, off / U, most)
