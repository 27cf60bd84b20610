"""Helpers of the tests of products whose operands differ in size from column to column: a product of floats does not notice, since a result sees its
own column alone.  Errors are taken column by column, relative to the column's own size (2-norm)."""
import torch

#: Relative error of a column of Y, and of a gradient.  Operands are held to 2^-22 of themselves, 2^-24 on average and with random signs; G, U and H
#: (backward dH, dG, dU as well) come one after the other from two such operands each, and sums of 32-bit floats add as much again: some six to
#: sixteen roundings of 2^-24, added like random numbers below 4 x 2^-24 = 2.4e-7, four times which for few rows that share a large one.
LIMIT = {"Y": 1e-6}
LIMIT_GRADIENT = 2e-6


def powers(gen, count, low, high=0, device="cuda"):
    """Powers of two from 2^low to 2^high, both among them, in any order."""
    e = torch.randint(low, high + 1, (count,), device=device, generator=gen).float()
    if count > 1:
        e[0], e[-1] = low, high
    return torch.exp2(e)


def columns_off(got, want, dim):
    """Error of each column (dim = 0) or row (1) relative to it; columns that are zeros have to be."""
    size, off = want.norm(dim=dim), (got.double() - want).norm(dim=dim)
    return torch.where(size > 0, off / size.clamp(min=1e-300), torch.where(off > 0, torch.full_like(off, float("inf")), off))


def check_columns(got, want, dim, limit, what):
    off = columns_off(got, want, dim)
    assert bool((off <= limit).all()), f"{what}: {int((~(off <= limit)).sum())} of {off.numel()} beyond {limit:.1e}, worst {float(off.nan_to_num(nan=1e30).max()):.3g}"
