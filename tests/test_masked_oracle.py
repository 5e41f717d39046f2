"""Pins of the masked attention oracle (no GPU needed): single cases by hand, the
unmasked case against another evaluator, gradients against differences."""
import math

import numpy as np
import pytest

from oracle import masked_oracle as MO
from oracle import operators_oracle as OO


def test_visible_keys():
    see, pos = MO.visible(1, 3, 5, k_lens=[9, 4], q_starts=[0, 1], prefix_lens=[0, 3])
    assert (pos == [1, 2, 3]).all()
    assert see.astype(int).tolist() == [[1, 1, 1, 0, 0], [1, 1, 1, 0, 0], [1, 1, 1, 1, 0]]
    see, _ = MO.visible(0, 2, 4, q_docs=[7, -1], k_docs=[7, -1, 7, 7])      # positions 2 and 3
    assert see.astype(int).tolist() == [[1, 0, 1, 0], [0, 1, 0, 0]]
    see, _ = MO.visible(0, 3, 2, q_lens=[2])                                # positions -1, 0, 1; the last one padding
    assert see.astype(int).tolist() == [[0, 0], [1, 0], [0, 0]]


def test_one_key_two_keys():
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(2, 128)), rng.normal(size=(2, 128)), rng.normal(size=(2, 128))
    O, lse = MO.attention(q, k, v, 1, 2, 2, 1, 1, cap=1.5, slopes=[0.25])
    assert np.allclose(O[0], v[0], atol=1e-15)
    z = [1.5 * math.tanh(float(q[1] @ k[j]) / math.sqrt(128) / 1.5) - 0.25 * (1 - j) for j in range(2)]
    w = [math.exp(t) for t in z]
    assert np.allclose(O[1], (w[0] * v[0] + w[1] * v[1]) / sum(w), atol=1e-14)
    assert abs(lse[1, 0] - math.log2(sum(w))) < 1e-14


def test_without_masks_it_is_cross_attention():
    rng = np.random.default_rng(1)
    Q, dO = rng.normal(size=(10, 512)), rng.normal(size=(10, 512))
    K, V = rng.normal(size=(14, 256)), rng.normal(size=(14, 256))
    a = MO.attention(Q, K, V, 2, 5, 7, 4, 2, causal=False, k_lens=[7, 3], dO=dO)
    b = (*OO.cross_attention(Q, K, V, 2, 5, 7, 4, 2, [7, 3]), *OO.cross_attention_backward(Q, K, V, dO, 2, 5, 7, 4, 2, [7, 3]))
    for x, y in zip(a, b):
        assert np.allclose(x, y, atol=1e-12)


@pytest.mark.parametrize("kw", [dict(cap=0.7), dict(slopes=[0.3, -0.1]), dict(cap=2.0, slopes=[0.5, 0.1], prefix_lens=[2]),
                                dict(q_docs=[0, 0, 1, 1], k_docs=[0, 0, 1, 1]), dict(q_lens=[3], k_lens=[3])])
def test_gradients_against_differences(kw):
    rng = np.random.default_rng(2)
    dh = 8
    v = {"Q": rng.normal(size=(4, 2 * dh)), "K": rng.normal(size=(4, dh)), "V": rng.normal(size=(4, dh))}
    dO = rng.normal(size=(4, 2 * dh))
    loss = lambda **k: (MO.attention(**{**v, **k}, B=1, Sq=4, Sk=4, Hq=2, Hk=1, dh=dh, **kw)[0] * dO).sum()  # noqa: E731
    g = dict(zip("QKV", MO.attention(**v, B=1, Sq=4, Sk=4, Hq=2, Hk=1, dh=dh, dO=dO, **kw)[2:]))
    for n in "QKV":
        for i in np.ndindex(v[n].shape):
            e = np.zeros(v[n].shape)
            e[i] = 1e-5
            assert abs((loss(**{n: v[n] + e}) - loss(**{n: v[n] - e})) / 2e-5 - g[n][i]) < 1e-8, (n, i)
