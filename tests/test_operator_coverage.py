"""Which kernels and loops the sizes of the GPU tests reach, by the host's
rules, and what the relative bound of the gradients sees (no GPU needed)."""
import numpy as np
import pytest

from oracle import operators_oracle as OO
from paper_2401_11202_amd import partir as P
from tests import test_gpu_cross_loops as L
from tests import test_gpu_operator_runs as R
from tests.gpu_common import TOL_REL_FRO, rel_fro

DH, CUS = 128, 256


def forward(B, Sq, Sk, Hq, Hk, *_):
    """(waves over rows, key groups) of the forward kernel, as its launch chooses."""
    rows = Hq // Hk * Sq
    if rows <= 32:
        return 1, 4
    grid = B * Hk * -(-rows // 128) * P.plan_cross_attention(B, Sq, Sk, Hq, Hk)["n_virtual_shards"]
    return 4, 2 if grid <= CUS else 1


def test_the_forward_tests_reach_every_kernel():
    assert {forward(*s) for s in L.MANY_ROWS} == {(4, 1)}
    assert {forward(*s) for s in L.LONG_KEYS} == {(4, 2), (1, 4)}
    # every place in the ring of three 32-key blocks is the last one of some sequence
    blocks = {-(-n // 32) for _, _, Sk, _, _, lens in L.MANY_ROWS for n in (lens or [Sk])}
    assert {n % 3 for n in blocks if n > 3} == {0, 1, 2} and {0, 1, 2, 3} <= blocks
    for B, Sq, Sk, Hq, Hk, _ in L.MANY_ROWS:   # a grid that no parts are asked for
        assert B * Hk * -(-Hq // Hk * Sq // 128) > CUS
    assert {B * Hk % 8 == 0 for B, _, _, _, Hk, _ in L.MANY_ROWS} == {True, False}


def test_the_gradient_tests_stream_many_tiles():
    """Without parts a workgroup takes every tile of 64 rows of its key head."""
    for shapes, one_pass in ((L.ONE_PASS, True), (L.TWO_PASSES, False)):
        for B, Sq, Sk, Hq, Hk, _ in shapes:
            assert (Sk <= 128) == one_pass
            assert P.plan_cross_attention_backward(B, Sq, Sk, Hq, Hk)["n_virtual_shards"] == 1
            assert -(-Hq // Hk * Sq // 64) >= 6
        assert {16 % (Hq // Hk) == 0 for _, _, _, Hq, Hk, _ in shapes} == {True, False}   # rows by steps, and divided
    assert any(P.plan_cross_attention_backward(*s[:5])["n_virtual_shards"] > 1 for s in L.LONG_KEYS)


def test_the_run_tests_take_more_than_one_block_or_chunk():
    for cases, grid in ((R.ROTARY, 8192), (R.NORM, 2048), (R.GRADIENTS, 1024)):
        for T, *_ in cases:
            assert -(-T // 16) > grid
    for sizes, kinds in R.CHUNKS:
        assert len(sizes) <= 144 and sum(-(-n * k.itemsize // 32768) for n, k in zip(sizes, kinds)) > 2 * 2048


@pytest.mark.parametrize("Sq,Sk,Hq,Hk", [(100, 4100, 2, 1), (1, 4096, 16, 16), (200, 300, 2, 1), (64, 257, 1, 1)])
def test_the_relative_bound_sees_a_wrong_rowsum(Sq, Sk, Hq, Hk):
    """Gradients with D left out, halved, doubled or negated are past the bound
    in dQ or dK at the sizes at which the GPU's are held to it."""
    rng = np.random.default_rng(Sq)
    q, g = rng.standard_normal((2, Sq, Hq * DH))
    k, v = rng.standard_normal((2, Sk, Hk * DH))
    ref = OO.cross_attention_backward(q, k, v, g, 1, Sq, Sk, Hq, Hk)
    for factor in (0.0, 0.5, 2.0, -1.0):
        dq, dk = np.zeros_like(q), np.zeros_like(k)
        for h in range(Hq):
            c, e = slice(h * DH, (h + 1) * DH), slice(h // (Hq // Hk) * DH, (h // (Hq // Hk) + 1) * DH)
            s = q[:, c] @ k[:, e].T * DH ** -0.5
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            dp = g[:, c] @ v[:, e].T
            ds = p * (dp - factor * (p * dp).sum(1, keepdims=True)) * DH ** -0.5
            dq[:, c] = ds @ k[:, e]
            dk[:, e] += ds.T @ q[:, c]
        worst = max(rel_fro(dq, ref[0]), rel_fro(dk, ref[1]))
        assert worst > 2 * TOL_REL_FRO, factor
