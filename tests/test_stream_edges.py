"""Arguments of dropout and of the join with the residual stream at the ends of
their ranges (no GPU needed)."""
import pytest

from paper_2401_11202_amd import partir as P
from tests.test_stream_checks import A, _never_launch, bwd, join  # noqa: F401

MOST = 2 ** 63 - 1


@pytest.mark.parametrize("rows", [16, 17, 2 ** 40, MOST - 16, MOST - 14, MOST])
def test_a_gate_row_for_any_count_of_rows(rows):
    """One gate row for all: 160 bytes, whatever lies behind them is another's."""
    assert join(rows=rows) == "PARTIR_E_HIP" and bwd(rows=rows) == "PARTIR_E_HIP"
    assert join(rows=rows, H=A[3]) == "PARTIR_E_LAYOUT" and join(rows=rows, N=A[3]) == "PARTIR_E_LAYOUT"
    assert bwd(rows=rows, dgate=A[5]) == "PARTIR_E_LAYOUT" and bwd(rows=rows, dgate=A[3]) == "PARTIR_E_LAYOUT"
    assert bwd(rows=rows, dgpost=A[11]) == "PARTIR_E_LAYOUT"
    ws = P.lib().partir_residual_norm_backward_workspace
    assert ws(16, 40, rows) == ws(16, 40, 16)
