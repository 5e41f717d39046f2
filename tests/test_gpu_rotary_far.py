"""Rotary at positions far past 2^31, which int64 positions reach: the angle is
formed in float64, its 1 / (2 pi), its product with the frequency and that with
the position each off by half a step, 2^-53, and a position past 2^53 by as
much: within 2^-51 of the angle in all.  The rest as in tests/test_gpu_rotary.py."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as OO
from paper_2401_11202_amd import inputs as I
from paper_2401_11202_amd import partir as P
from tests.gpu_common import say
from tests.test_gpu_rotary import close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("far", [2 ** 31, 2 ** 35, 2 ** 42])
@pytest.mark.parametrize("sign", [1, -1])
def test_far_positions(far, sign):
    T, H, dh = 64, 2, 64
    say(f"rotary at positions of {sign} x {far}")
    x, f = I.gaussian(340, 0, (T, H * dh), 1.0, "f32"), OO.frequencies(dh)
    pos = sign * (far + np.random.default_rng(1).integers(0, far // 2, T))
    got, _ = P.rotary(x.to_device(), None, torch.from_numpy(f).cuda(), d_head=dh, positions=torch.from_numpy(pos).cuda())
    angle = np.repeat((np.abs(pos)[:, None] * f)[:, None, :], 2, 1).reshape(T, H, 1, dh // 2)   # half pairs: twice a head
    slack = np.broadcast_to(2.0 ** -20 + 2.0 ** -51 * angle, (T, H, 2, dh // 2)).reshape(T, H * dh)
    close(got, OO.rotary(x.f64(), pos, f, dh), OO.pair_size(x.f64(), dh // 2, dh), slack, "f32", "Q")
