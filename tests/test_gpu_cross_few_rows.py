"""cross_attention of few query rows (up to 32 of a key head): the weights are
held to 2^-16, so the output is off by little more than its own rounding.

Tolerance: with A = P |V| and e the relative error of a weight before its
rounding (2^-14 and 2^-16 of scale |Q||K|^T, as in
tests/test_gpu_cross_attention.py), (2^-16 + e) A and 2^-8 |O| for the result's
rounding.  A single rounding of the weights to bf16 would add 2^-8 A at most,
which over few keys is past it."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as OO
from paper_2401_11202_amd import partir as P
from tests.gpu_common import host, say
from tests.test_gpu_cross_attention import make

pytestmark = pytest.mark.gpu
U, DH = 2.0 ** -8, 128


@pytest.mark.parametrize("B,Sq,Sk,Hq,Hk,lens", [
    (32, 1, 3, 8, 2, None), (8, 1, 40, 32, 1, None), (4, 8, 77, 8, 2, [77, 31, 0, 5]), (16, 32, 20, 2, 2, None),
    (2, 5, 130, 12, 2, [130, 2]), (3, 1, 2000, 16, 16, [2000, 64, 7])])
def test_weights_keep_more_than_bf16(B, Sq, Sk, Hq, Hk, lens):
    say(f"cross_attention of few rows B={B} Sq={Sq} Sk={Sk} heads {Hq}/{Hk} lens={lens}")
    Q, K, V, _, q, k, v, _ = make(B, Sq, Sk, Hq, Hk, lens, Sk)
    kw = dict(B=B, Sq=Sq, Sk=Sk, n_heads=Hq, n_kv_heads=Hk)
    got = host(P.cross_attention(Q, K, V, k_lens=None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda"), **kw))
    n = [Sk] * B if lens is None else lens
    ref, _ = OO.cross_attention(q, k, v, B, Sq, Sk, Hq, Hk, n)
    A, _ = OO.cross_attention(q, k, np.abs(v), B, Sq, Sk, Hq, Hk, n)
    norms = lambda x: np.sqrt((x.reshape(x.shape[0], -1, DH) ** 2).sum(-1)).max()  # noqa: E731  |Q||K|^T is at most their product
    e = 2.0 ** -14 + 2.0 ** -16 * DH ** -0.5 * norms(q) * norms(k)
    err = np.abs(got - ref) - (2.0 ** -16 + e) * A - U * np.abs(ref)
    say(f"    largest error past its bound {err.max():.2e}")
    assert err.max() <= 0.0
