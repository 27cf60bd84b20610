"""The gated feed-forward block on few rows of many hidden and many result columns: more than a workgroup has threads for, and more than LDS
holds."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_gated_ff import check, pipad  # noqa: E402,F401


@pytest.mark.parametrize("rows", [1, 5, 256, 257])
@pytest.mark.parametrize("F,hidden,Fo", [(20, 1023, 7), (20, 1024, 7), (20, 1025, 7), (33, 2050, 40), (7, 8192, 5), (7, 8193, 5), (300, 1500, 20)])
def test_many_hidden_columns(pipad, rows, F, hidden, Fo):  # noqa: F811
    check(pipad, rows, 1, F, hidden, Fo, "silu")


@pytest.mark.parametrize("F,hidden,Fo", [(20, 40, 1023), (20, 40, 1024), (20, 1100, 1025), (2048, 40, 2060), (2049, 40, 30), (3, 1030, 8192), (3, 1030, 8193),
                                         (3, 50, 8200)])
def test_many_result_columns(pipad, F, hidden, Fo):  # noqa: F811
    check(pipad, 3, 2, F, hidden, Fo, "gelu")
