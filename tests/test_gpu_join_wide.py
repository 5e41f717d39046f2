"""The join with the residual stream where its other GPU tests do not reach: counts of
a gate's rows at the end of their range.  Tolerances are those of
tests/test_gpu_residual_norm.py."""
import sys

import pytest
import torch

from paper_2401_11202_amd import partir as P
from tests.gpu_common import say
from tests.test_gpu_residual_norm import close, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [300, 10 ** 6, sys.maxsize - 1, sys.maxsize, 2 ** 64 + 7])
def test_one_gate_row_for_any_count_of_rows(rows):
    say(f"residual_norm gate_rows={rows}")
    T, D = 300, 264
    dev, ref, kw, j = make(T, D, ("f32", "bf16", True, -1, True, 0.2, 0.5, True))
    kw["gate_rows"] = rows
    h, n = P.residual_norm(dev["X"], dev["Y"], **kw)
    close(h, j.h, j.h_size, "H")
    close(n, j.n, j.n_size, "N")
    gains = tuple(torch.full((r, D) if r else (D,), float("nan"), device="cuda") for r in (0, 1, 0))
    got = P.residual_norm_backward(dev["X"], dev["Y"], dev["dH"], dev["dN"], gain_out=gains, **kw)
    want = j.backward(ref["dH"], ref["dN"])
    for k, g in zip(("dX", "dY", "dg_post", "dgate", "dg_pre"), got):
        close(g, *want[k], k)
