"""What the tests of products over columns of different size notice: an operand that keeps 16 bits of its row's, or its block's, largest value."""
import pytest
import torch

from _rows import GatedFF
from _spread import LIMIT, LIMIT_GRADIENT, columns_off, powers


def rounded(x, largest, bits=16):
    step = torch.exp2(torch.ceil(torch.log2(largest)) - bits)
    return torch.round(x / step) * step


@pytest.mark.parametrize("operand,dim,result", [("X", 0, "dWg"), ("X", 0, "dWu"), ("Wd", 0, "Y"), ("Wg", 1, "dX"), ("dY", 0, "dWd"), ("Wu", 0, "dWd"),
                                                ("Wd", 1, "dWg")])
def test_an_operand_of_16_bits_is_noticed(operand, dim, result):
    """Columns (rows, dim = 1) of the operand at 2^-20 to 1 of the others, which is 16 bits for the largest and none for the smallest."""
    gen = torch.Generator().manual_seed(3)
    rand = lambda *s: torch.randn(s, generator=gen, dtype=torch.float64)  # noqa: E731
    F, hidden, Fo, rows = 20, 64, 24, 150
    v = {"X": rand(rows, F), "Wg": rand(F, hidden) / F ** 0.5, "Wu": rand(F, hidden) / F ** 0.5, "Wd": rand(hidden, Fo) / hidden ** 0.5, "dY": rand(rows, Fo)}
    d = powers(gen, v[operand].shape[1 - dim], -20, device="cpu").double()
    for q in ("Wg", "Wu") if operand == "Wg" else (operand,):  # (a column of dX sees both)
        v[q] = v[q] * (d if dim == 0 else d[:, None])

    def results(v):
        block = GatedFF(v["X"], v["Wg"], v["Wu"], v["Wd"], None, None, None, "silu")
        return {"Y": block.forward()[0], **{q: g for q, (g, _) in block.backward(v["dY"]).items()}}

    want = results(v)
    got = results({**v, operand: rounded(v[operand], v[operand].abs().amax(dim=1, keepdim=True) if operand in ("X", "dY") else v[operand].abs().max())})
    along = 1 if operand in ("X", "Wu") else 0
    off = columns_off(got[result], want[result], along)
    assert float(off.max()) > 100 * LIMIT.get(result, LIMIT_GRADIENT)
    same = results(v)
    assert all(float(columns_off(same[q], want[q], 0).max()) == 0 for q in ("Y", "dX", "dWg", "dWd"))
