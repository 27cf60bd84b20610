"""Limits of the operators on node rows that the binding has to see itself; no GPU is needed to be refused."""
import pytest

torch = pytest.importorskip("torch")

import paper_2301_00391_amd as pipad  # noqa: E402

TOO_LARGE = -4


@pytest.mark.parametrize("n", [1 << 31, (1 << 32) + 5])
@pytest.mark.parametrize("listed", [False, True])
def test_more_rows_than_an_int32_counts(n, listed):
    """Refused as too large, not taken for the rows that the low 32 bits count (nothing is read: memory of one value stands for the rows)."""
    x = torch.zeros(1, 1).expand(n, 1)
    x = [x] if listed else x.unsqueeze(1)
    w = torch.zeros(1, 1)
    for call in (lambda: pipad.residual_norm(x), lambda: pipad.residual_norm_backward(x, None, x), lambda: pipad.gated_ff(x, w, w, w),
                 lambda: pipad.gated_ff_backward(x, x, w, w, w)):
        with pytest.raises(pipad.PipadError) as why:
            call()
        assert why.value.status == TOO_LARGE
