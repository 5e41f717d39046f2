"""Clipping of very many tensors: the partial sums of the tables are added to a
few before the scaling launches read them.  Tolerances as in
tests/test_gpu_grad_norm.py."""
import ctypes

import pytest
import torch

from paper_2401_11202_amd import partir as P
from tests.gpu_common import say
from tests.test_gpu_grad_norm import check

F, B = torch.float32, torch.bfloat16


def views(n, seed):
    """n neighbouring tensors of 0 to 40 values, of both types in turn, and two large ones among them."""
    g = torch.Generator().manual_seed(seed)
    sizes = torch.randint(0, 41, (n,), generator=g).tolist()
    sizes[1], sizes[n // 2] = 300_001, 200_003
    flat = {k: torch.randn(sum(sizes[i::2]), generator=g).cuda().to(k) for i, k in enumerate((F, B))}
    at, ts = dict.fromkeys(flat, 0), []
    for i, s in enumerate(sizes):
        k = (F, B)[i % 2]
        ts.append(flat[k][at[k]:at[k] + s])
        at[k] += s
    return ts


@pytest.mark.gpu
@pytest.mark.parametrize("n", [2040, 2049, 5000, 20000])
def test_norm_and_clip_of_many_tensors(n):
    say(f"clip {n} tensors")
    ts = views(n, n)
    check(ts, 0.5, out=[torch.full_like(t, 9.0) for t in ts])
    check(ts, 1e9)
    check(ts, 0.25)


@pytest.mark.gpu
def test_many_tensors_replayed():
    ts = views(3000, 1)
    out, norm = [torch.empty_like(t) for t in ts], torch.empty((), device="cuda")
    ws = torch.empty(P.lib().partir_grad_norm_workspace(3000), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.clip_grad_norm(ts, 2.0, out=out, norm=norm, workspace=ws)
    for _ in range(3):
        ts[1].mul_(1.5)
        g.replay()
        torch.cuda.synchronize()
        want = [torch.empty_like(t) for t in ts]
        n = P.clip_grad_norm(ts, 2.0, out=want)
        assert torch.equal(n, norm) and all(torch.equal(a, b) for a, b in zip(want, out))


@pytest.mark.parametrize("n", [1, 144, 145, 288, 289, 100000, 2 ** 24])
def test_workspace_holds_the_partials_and_their_sums(n, monkeypatch):
    """A float64 for each of 2048 workgroups of each table of 144 tensors, and
    256 more where those are too many for every workgroup to add."""
    parts = -(-n // 144) * 2048
    need = P.lib().partir_grad_norm_workspace(n)
    assert need == 8 * (parts + (256 if parts > 2048 else 0))
    if n > 1000:
        return
    monkeypatch.setenv("PARTIR_FAIL_LAUNCH", "1")
    ptrs, numel, dts = (ctypes.c_void_p * n)(*[0x100000 + 4096 * i for i in range(n)]), (ctypes.c_int64 * n)(*[9] * n), (ctypes.c_int * n)()
    call = lambda b: P.STATUS[P.lib().partir_clip_grad_norm(ptrs, ptrs, numel, dts, n, 1.0, 0x10000, 0x20000, b, None)]  # noqa: E731
    assert dts[0] == P.F32
    assert call(need) == "PARTIR_E_HIP" and call(need - 1) == "PARTIR_E_WORKSPACE"
