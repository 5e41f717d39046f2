"""Pins of the oracle of dropout and of the join with the residual stream (no GPU
needed): the generator's published test vectors, its statistics, gradients
against differences."""
import numpy as np
import pytest

from oracle import stream_oracle as SO


@pytest.mark.parametrize("counter,key,want", [   # the known answers published with the generator, ten rounds
    ((0, 0, 0, 0), (0, 0), "6627e8d5 e169c58d bc57ac4c 9b00dbd8"),
    ((2 ** 32 - 1,) * 4, (2 ** 32 - 1,) * 2, "408f276d 41c83b0e a20bc7c6 6d5451fd"),
    ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), "d16cfe09 94fdcceb 5001e420 24126ea1"),
])
def test_generator(counter, key, want):
    assert " ".join(f"{int(w):08x}" for w in SO.philox(counter, key)) == want


@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.9, 1.0])
def test_share_kept(p):
    f = SO.factors(400, 500, p, (77, 3))
    kept = (f != 0).mean()
    assert abs(kept - (1 - p)) <= 5 * np.sqrt(p * (1 - p) / f.size) + 2.0 ** -17    # five deviations, and the step of p
    if kept:
        assert np.ptp(f[f != 0]) == 0 and abs(f.mean() - 1) <= 5 * np.sqrt(p / (1 - p) / f.size) + 1e-5 if p < 1 else True


def test_mask_depends_on_the_place_alone():
    whole = SO.factors(60, 43, 0.4, (5, 2 ** 40 + 9), row0=1000)
    assert (SO.factors(20, 17, 0.4, (5, 2 ** 40 + 9), row0=1030) == whole[30:50, :17]).all()
    for other in ((6, 2 ** 40 + 9), (5, 2 ** 41 + 9), (5 + 2 ** 32, 2 ** 40 + 9), (5, 2 ** 40 + 10)):
        assert (SO.factors(60, 43, 0.4, other, row0=1000) != whole).mean() > 0.3


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("next_norm", [False, True])
def test_join_gradients_against_differences(post, next_norm):
    rng = np.random.default_rng(1)
    T, D, rows = 5, 8, 2
    v = {"x": rng.normal(size=(T, D)), "y": rng.normal(size=(T, D)), "g_post": rng.normal(size=D), "gate": rng.normal(size=(3, D)),
         "g_pre": rng.normal(size=D)}
    f = SO.factors(T, D, 0.3, (1, 2))
    dh, dn = rng.normal(size=(T, D)), rng.normal(size=(T, D))

    def join(**k):
        return SO.Join(**{**v, **k}, post=post, gate_rows=rows, scale=0.7, f=f, eps=1e-3)

    def loss(**k):
        j = join(**k)
        return (j.h * dh).sum() + ((j.n * dn).sum() if next_norm else 0.0)

    g = join().backward(dh, dn if next_norm else None)
    for name, leaf in (("dX", "x"), ("dY", "y"), ("dg_post", "g_post"), ("dgate", "gate"), ("dg_pre", "g_pre")):
        if name not in g:
            continue
        for i in np.ndindex(v[leaf].shape):
            e = np.zeros(v[leaf].shape)
            e[i] = 1e-5
            num = (loss(**{leaf: v[leaf] + e}) - loss(**{leaf: v[leaf] - e})) / 2e-5
            assert abs(num - g[name][0][i]) <= 1e-7 * (1 + g[name][1][i]), (name, i)
