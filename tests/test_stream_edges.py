"""Arguments of dropout and of the join with the residual stream at the ends of
their ranges (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2401_11202_amd import partir as P
from tests.test_stream_checks import A, NULL, _never_launch, bwd, drop, join, status  # noqa: F401

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


@pytest.mark.parametrize("row0", [2 ** 32 - 15, 2 ** 32, MOST - 16, MOST - 15, MOST])
def test_rows_numbered_past_their_range(row0):
    assert drop(row0=row0) == join(row0=row0) == bwd(row0=row0) == "PARTIR_E_SHAPE"


@pytest.mark.parametrize("row0", [-1, 2 ** 32 + 1, 2 ** 64, 2 ** 64 + 1, -2 ** 64 + 5])
def test_the_binding_passes_no_other_row_on(row0):
    x, y, s = torch.zeros(16, 40), torch.zeros(16, 40, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int64)
    for call in (lambda: P.dropout(x, 0.5, s, row0=row0), lambda: P.residual_norm(x, y, p=0.5, seed=s, row0=row0),
                 lambda: P.residual_norm_backward(x, y, x, y, p=0.5, seed=s, row0=row0)):
        assert status(call) == "PARTIR_E_SHAPE"


@pytest.mark.parametrize("T", [16, 0])
@pytest.mark.parametrize("gain", ["post", "pre"])
def test_a_gain_of_1_has_no_gradient(gain, T):
    none = {"g" + gain: NULL}
    assert bwd(T=T, **none) == "PARTIR_E_UNSUPPORTED"
    assert bwd(T=T, **none, **{"dg" + gain: NULL}) == "PARTIR_E_HIP"
    assert bwd(T=T, **{"dg" + gain: NULL}) == "PARTIR_E_HIP"


@pytest.mark.parametrize("T,D,want", [(2 ** 30 - 64, 128, "PARTIR_E_HIP"), (2 ** 30 - 63, 128, "PARTIR_E_SHAPE"), (2 ** 30 - 1, 128, "PARTIR_E_SHAPE"),
                                      (8191, 2 ** 24, "PARTIR_E_HIP"), (8192, 2 ** 24, "PARTIR_E_SHAPE")])
def test_the_largest_launch_of_dropout(T, D, want):
    """A launch is fewer than 2^32 threads: at most 2^24 - 1 workgroups of 256, each for 1024 groups of eight columns."""
    assert drop(T=T, D=D, ldx=D, ldy=D, R=NULL, ldr=0, Y=ctypes.c_void_p(1 << 50)) == want
