"""The join with the residual stream where its other GPU tests do not reach: counts of
a gate's rows at the end of their range, rows above 8192 columns in several workgroups,
offsets past 32 bits.  Tolerances are those of tests/test_gpu_residual_norm.py."""
import sys

import pytest
import torch

from paper_2401_11202_amd import partir as P
from tests.gpu_common import say
from tests.test_gpu_residual_norm import FORMS, close, make

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


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("T,D", [(70, 8200), (40, 12288), (131, 16384)])
def test_gradients_of_wide_rows_by_several_workgroups(T, D, form):
    """Sixteen columns a lane, with workgroups' partial sums, and a gate's rows in chunks
    of several workgroups as well as a team's several gate rows."""
    say(f"residual_norm_backward T={T} D={D} {form}")
    dev, ref, kw, j = make(T, D, form)
    got = dict(zip(("dX", "dY", "dg_post", "dgate", "dg_pre"), P.residual_norm_backward(dev["X"], dev["Y"], dev["dH"], dev["dN"], **kw)))
    for k, (g, size) in j.backward(ref["dH"], ref["dN"]).items():
        if got[k] is None:
            assert k in ("dg_post", "dg_pre") and kw["g_" + k[3:]] is None
            continue
        close(got[k], g, size, k)
    assert (got["dgate"] is None) == (kw["gate"] is None)


@pytest.mark.parametrize("T,D,ld", [(33000, 1032, 2 ** 16), (70, 8200, 2 ** 24)])
def test_offsets_past_32_bits(T, D, ld):
    """Everything as columns of rows of up to 2^24 values: the same results in every bit as from dense rows."""
    say(f"residual_norm and dropout T={T} D={D} leading dim {ld}")
    g = torch.Generator(device="cuda").manual_seed(5)
    dense = [torch.randn(T, D, generator=g, device="cuda") for _ in range(4)]
    wide = torch.empty(T, ld, device="cuda")
    assert (T - 1) * ld * 4 > 2 ** 32
    X, Y, dH, dN, h, n, d = cols = [wide[:, 8 * (i + 1) + i * D:8 * (i + 1) + (i + 1) * D] for i in range(7)]
    for c, t in zip(cols, dense):
        c.copy_(t)
    gain = torch.rand(D, generator=g, device="cuda")
    gate = torch.rand(-(-T // 11), D, generator=g, device="cuda")
    seed = torch.tensor([5, 6], device="cuda")
    kw = dict(g_post=gain, post_norm=True, gate=gate, gate_rows=11, g_pre=gain, p=0.3, seed=seed)
    want = P.residual_norm(*dense[:2], **kw)
    got = P.residual_norm(X, Y, out=h, norm_out=n, **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(P.dropout(X, 0.3, seed, residual=Y, out=d), P.dropout(dense[0], 0.3, seed, residual=dense[1]))
    want = P.residual_norm_backward(*dense, **kw)
    got = P.residual_norm_backward(X, Y, dH, dN, out=(h, n), **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("T,D", [(3, 24), (700, 512), (1501, 1000), (90, 5120), (60, 9000)])
def test_gradients_repeat_whatever_workspace_and_outputs_held(T, D, form):
    """Sums of a workgroup's rows, of a team's gate rows and of the parts: each is written before it is read."""
    say(f"residual_norm_backward T={T} D={D} {form}")
    dev, ref, kw, j = make(T, D, form)
    args = dev["X"], dev["Y"], dev["dH"], dev["dN"]
    first = P.residual_norm_backward(*args, **kw)
    ws = torch.empty(P.lib().partir_residual_norm_backward_workspace(T, D, kw["gate_rows"] or 0), dtype=torch.uint8, device="cuda")
    for fill in (255, 0, 127):                     # NaN, 0, 3e38
        outs = [None if t is None else torch.full_like(t, float("nan")) for t in first]
        ws.fill_(fill)
        P.residual_norm_backward(*args, out=outs[:2], gain_out=outs[2:], workspace=ws, **kw)
        assert all(a is b is None or torch.equal(a, b) for a, b in zip(outs, first))
