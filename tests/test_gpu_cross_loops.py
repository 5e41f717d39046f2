"""cross_attention at sizes where a workgroup streams many tiles: the forward
kernel of many rows (a ring of three stages), the one-pass gradients and the
dK / dV pass without parts, against the fp64 oracle.

Tolerances: elementwise as in tests/test_gpu_cross_attention.py.  Those bounds
add absolute values over the keys, so that with many keys they let a wrong
rowsum D through; the error of each result relative to its whole size
(Frobenius) is held too.  Its parts are the roundings to bf16 of the weights,
of dS, of O within D and of the result, each at most 2^-8 of its value; over many
terms of either sign they add in quadrature, to at most 2^-7 = 0.8e-2, below the
framework's bound for chained products (tests/gpu_common.py).  With a single key
dS is 0 and so are dQ and dK: nothing to be relative to."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as OO
from paper_2401_11202_amd import partir as P
from tests.gpu_common import TOL_REL_FRO, host, rel_fro, say
from tests.test_gpu_cross_attention import bounds, check, make

pytestmark = pytest.mark.gpu
DH = 128
NAMES = ("O", "lse", "dQ", "dK", "dV")


def run(B, Sq, Sk, Hq, Hk, lens=None, wid=0):
    say(f"cross_attention B={B} Sq={Sq} Sk={Sk} heads {Hq}/{Hk} lens={lens}")
    Q, K, V, dO, q, k, v, g = make(B, Sq, Sk, Hq, Hk, lens, wid)
    ln = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    n = [Sk] * B if lens is None else lens
    kw = dict(B=B, Sq=Sq, Sk=Sk, n_heads=Hq, n_kv_heads=Hk, k_lens=ln)
    O, lse = P.cross_attention_train(Q, K, V, **kw)
    assert torch.equal(P.cross_attention(Q, K, V, **kw), O)
    got = (O, lse, *P.cross_attention_backward(Q, K, V, O, dO, lse, **kw))
    for x, y in zip(got[2:], P.cross_attention_backward(Q, K, V, O, dO, lse, **kw)):
        assert torch.equal(x, y)
    ro, rl = OO.cross_attention(q, k, v, B, Sq, Sk, Hq, Hk, n)
    refs = (ro, rl, *OO.cross_attention_backward(q, k, v, g, B, Sq, Sk, Hq, Hk, n))
    for name, x, r, b in zip(NAMES, got, refs, bounds(q, k, v, g, ro, B, Sq, Sk, Hq, Hk, n, DH ** -0.5)):
        check(name, x, r, b)
        if name != "lse" and (max(n) > 1 or name in ("O", "dV")):
            err = rel_fro(host(x), r)
            say(f"    {name}: relative error {err:.2e}")
            assert err < TOL_REL_FRO, name
    for b in range(B):
        pad = slice(b * Sk + n[b], (b + 1) * Sk)
        assert not got[3][pad].any() and not got[4][pad].any()
    # in the queries' place: the same bits
    assert P.cross_attention(Q, K, V, out=Q, **kw) is Q and torch.equal(Q, O)


# more than 256 workgroups of 128 rows; keys of one block of 32 to ten, whole and not
MANY_ROWS = [(2, 2100, Sk, 8, 8, None) for Sk in (1, 31, 33, 65, 97, 300)] + [
    (2, 2100, 300, 8, 8, [300, 161]), (2, 2100, 70, 8, 8, [0, 33]), (3, 2304, 130, 5, 5, [96, 130, 0]),
    (2, 1840, 200, 9, 3, [200, 127]), (1, 4200, 1000, 32, 8, [937])]


@pytest.mark.parametrize("B,Sq,Sk,Hq,Hk,lens", MANY_ROWS)
def test_many_rows(B, Sq, Sk, Hq, Hk, lens):
    run(B, Sq, Sk, Hq, Hk, lens, wid=Sq + Sk)


# up to 128 keys, more (sequence, key head)s than half of the compute units: every workgroup takes all its rows
ONE_PASS = [(17, 400, 77, 8, 8, None), (17, 330, 128, 8, 8, [128, 0, 1] + [31 * i % 129 for i in range(14)]),
            (9, 150, 90, 45, 15, [90 - 7 * b for b in range(9)]), (33, 130, 40, 16, 4, None)]


@pytest.mark.parametrize("B,Sq,Sk,Hq,Hk,lens", ONE_PASS)
def test_gradients_in_one_pass_over_many_tiles(B, Sq, Sk, Hq, Hk, lens):
    run(B, Sq, Sk, Hq, Hk, lens, wid=Sq + Sk)


# above 128 keys, more key blocks than half of the compute units
TWO_PASSES = [(17, 450, 200, 8, 8, None), (6, 450, 700, 8, 8, [700, 513, 1, 0, 699, 256]), (15, 150, 200, 27, 9, [200 - 13 * b for b in range(15)]),
              (16, 512, 1200, 16, 4, [1200 - 61 * b for b in range(16)])]


@pytest.mark.parametrize("B,Sq,Sk,Hq,Hk,lens", TWO_PASSES)
def test_gradients_in_two_passes_over_many_tiles(B, Sq, Sk, Hq, Hk, lens):
    run(B, Sq, Sk, Hq, Hk, lens, wid=Sq + Sk)


# the key axis of dQ in parts, D from O, where a wrong D is a few percent of the result
LONG_KEYS = [(1, 100, 4100, 2, 1, None), (2, 1, 4096, 8, 8, None), (2, 200, 300, 4, 2, [300, 257]), (1, 64, 257, 2, 2, None)]


@pytest.mark.parametrize("B,Sq,Sk,Hq,Hk,lens", LONG_KEYS)
def test_rowsums_over_long_keys(B, Sq, Sk, Hq, Hk, lens):
    run(B, Sq, Sk, Hq, Hk, lens, wid=Sq + Sk)
