"""GPU parity of grad_norm and clip_grad_norm against fp64.

Tolerances.  Squares of float32 and bf16 values are exact in float64 and their
sum is off by less than 2^-40, so the norm is off by its rounding to float32,
half a step 2^-24 (2^-23 granted); above float32's range it is infinite.  A
scaled value is a float64 product rounded to float32 (2^-24) and, in bf16, once
more (2^-8); below float32's normal range both types step by 2^-133 or less, so
that half a step is at most 2^-134 (bf16) and 2^-150 (float32)."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as OO
from paper_2401_11202_amd import partir as P
from tests.gpu_common import host, say

pytestmark = pytest.mark.gpu
STEP = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134}
REL = {torch.float32: 2.0 ** -23 + 2.0 ** -24, torch.bfloat16: 2.0 ** -8 + 2.0 ** -22}


def tensors(sizes, kinds, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(n, generator=g, device="cuda") * scale).to(k) for n, k in zip(sizes, kinds)]


def check(ts, max_norm, **kw):
    before = [host(t) for t in ts]
    n, ref = OO.clip(before, max_norm)
    alone = float(P.grad_norm(ts))
    out = kw.get("out") or ts
    got = float(P.clip_grad_norm(ts, max_norm, **kw))
    assert alone == got and (abs(got - n) <= 2.0 ** -23 * n if n < 3.4e38 else got == np.inf)
    for o, r, b in zip(out, ref, before):
        assert (np.abs(host(o) - r) <= REL[o.dtype] * np.abs(r) + STEP[o.dtype]).all()
        if n <= max_norm:
            assert (host(o) == b).all()


F, B = torch.float32, torch.bfloat16
LISTS = [([1], [F]), ([1], [B]), ([0, 3, 0], [F, B, F]), ([8192], [F]), ([16384], [B]), ([8193, 16385, 7], [F, B, B]),
         ([100003, 1, 65536, 3], [B, F, F, B]), ([5] * 300, [F, B, F] * 100), ([3_000_001, 4096], [F, B])]


@pytest.mark.parametrize("sizes,kinds", LISTS, ids=[f"{len(s)}x{max(s)}" for s, _ in LISTS])
def test_norm_and_clip(sizes, kinds):
    say(f"clip {len(sizes)} tensors, the largest of {max(sizes)}")
    for max_norm in (0.5, 1e9):
        check(tensors(sizes, kinds, 3), max_norm)                      # in place
        ts = tensors(sizes, kinds, 4)
        check(ts, max_norm, out=[torch.full_like(t, 9.0) for t in ts])
    ts = tensors(sizes, kinds, 3)
    assert float(P.clip_grad_norm(ts, 0.0)) > 0 and all(bool((t == 0).all()) for t in ts)


def test_no_tensors():
    assert float(P.grad_norm([])) == 0.0 and float(P.clip_grad_norm([], 1.0)) == 0.0
    e = torch.empty((3, 0), device="cuda")
    assert float(P.clip_grad_norm([e], 1.0)) == 0.0


@pytest.mark.parametrize("kind", [F, B])
def test_views_of_a_bucket_at_every_alignment(kind):
    """Neighbouring views of odd sizes: each is scaled once, what lies between stays."""
    sizes = [1, 7, 8, 9, 31, 33000, 2, 8191, 16383, 5]
    flat = torch.randn(sum(sizes) + 2 * len(sizes), device="cuda").to(kind)
    before, at, views = flat.clone(), 1, []
    for n in sizes:
        views.append(flat[at:at + n])
        at += n + 1
    gaps = torch.ones_like(flat, dtype=torch.bool)
    for v in views:
        gaps[v.storage_offset():v.storage_offset() + v.numel()] = False
    check(views, 1.0)
    assert torch.equal(flat[gaps], before[gaps])
    other = torch.zeros(flat.numel() + 8, device="cuda", dtype=kind)   # outputs at other alignments than their inputs
    outs = [other[v.storage_offset() + 3:v.storage_offset() + 3 + v.numel()] for v in views]
    check(views, 1e-2, out=outs)


def test_large_and_small_values_keep_their_norm():
    check([torch.full((1000,), 3e37, device="cuda"), torch.full((10,), 1e-30, device="cuda")], 1.0)
    check([torch.full((4096,), 1e-30, device="cuda")], 1e-33)
    check([torch.full((70000,), 2.0 ** -130, device="cuda")], 1.0)     # below the normal range


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_norm_that_is_not_finite_scales_nothing(bad):
    ts = tensors([9000, 17], [F, B], 5)
    ts[0][8999] = bad
    before = [t.clone() for t in ts]
    out = [torch.zeros_like(t) for t in ts]
    n = float(P.clip_grad_norm(ts, 1.0, out=out))
    assert n != n if bad != bad else n == float("inf")
    P.clip_grad_norm(ts, 1.0)
    for t, o, b in zip(ts, out, before):
        assert torch.equal(t.nan_to_num(1.5), b.nan_to_num(1.5)) and torch.equal(o.nan_to_num(1.5), b.nan_to_num(1.5))


def test_replayed_graph_and_exact_repeats():
    ts = tensors([70001, 500, 12], [F, B, F], 6)
    out = [torch.empty_like(t) for t in ts]
    norm = torch.empty((), device="cuda")
    ws = torch.empty(P.lib().partir_grad_norm_workspace(3), dtype=torch.uint8, device="cuda")
    P.clip_grad_norm(ts, 2.0, out=out, norm=norm, workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.clip_grad_norm(ts, 2.0, out=out, norm=norm, workspace=ws)
    for i in range(3):
        ts[0].mul_(1.7)
        g.replay()
        torch.cuda.synchronize()
        want = [torch.empty_like(t) for t in ts]
        n = P.clip_grad_norm(ts, 2.0, out=want)
        assert torch.equal(n, norm) and all(torch.equal(a, b) for a, b in zip(want, out))
