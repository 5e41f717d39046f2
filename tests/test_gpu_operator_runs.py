"""The rotary, norm and clipping kernels at sizes where a workgroup takes more
than one unit of its work: further blocks of tokens behind the first, runs of
several chunks that cross from one tensor to the next.

Tolerances as in tests/test_gpu_rotary.py and tests/test_gpu_grad_norm.py; a
gain gradient adds up to 6 rows a lane, 64 row groups and 1024 workgroups here,
under 128 additions deep: 2^-16 of the sum of its terms' sizes, as there."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as OO
from paper_2401_11202_amd import inputs as I
from paper_2401_11202_amd import partir as P
from tests.gpu_common import host, say
from tests.test_gpu_grad_norm import check as check_clip
from tests.test_gpu_rotary import close

pytestmark = pytest.mark.gpu

# blocks are of 16 tokens at most, grids of 8192 (rotation), 2048 (with the norm) and 1024 (gradients) workgroups at most
ROTARY = [(16 * 8192 + 16 * 9 + 5, 1, 0, 8, 8, "bf16", False), (2 * 16 * 8192 + 3, 1, 1, 16, 12, "f32", True)]
NORM = [(2 * 16 * 2048 + 37, 1, 1, 64, 64, "bf16", False), (16 * 2048 + 1, 1, 0, 24, 6, "f32", True)]
GRADIENTS = [(3 * 16 * 1024 + 21, 1, 1, 64, 64, "bf16", False), (16 * 1024 + 1, 2, 0, 24, 6, "f32", True)]


def gaussians(T, Hq, Hk, dh, dtype, wid):
    return [None if h == 0 else I.gaussian(330, 2 * wid + i, (T, h * dh), 1.0, dtype) for i, h in enumerate((Hq, Hk))]


def device(ts):
    return [None if t is None else t.to_device() for t in ts]


@pytest.mark.parametrize("T,Hq,Hk,dh,rd,dtype,inter", ROTARY)
def test_rotary_of_many_tokens(T, Hq, Hk, dh, rd, dtype, inter):
    say(f"rotary T={T} H={Hq}+{Hk} dh={dh} rd={rd} {dtype}")
    x, f, S = gaussians(T, Hq, Hk, dh, dtype, 0), OO.frequencies(rd), 5000
    got = P.rotary(*device(x), torch.from_numpy(f).cuda(), d_head=dh, S=S, interleaved=inter)
    for i in range(2):
        if x[i] is not None:
            ref = OO.rotary(x[i].f64(), np.arange(T) % S, f, dh, interleaved=inter)
            close(got[i], ref, OO.pair_size(x[i].f64(), rd // 2, dh, inter), 2.0 ** -20, dtype, "QK"[i])


@pytest.mark.parametrize("T,Hq,Hk,dh,rd,dtype,inter", NORM)
def test_norm_of_many_tokens(T, Hq, Hk, dh, rd, dtype, inter):
    say(f"qk_norm_rotary T={T} H={Hq}+{Hk} dh={dh} rd={rd} {dtype}")
    x, f, S = gaussians(T, Hq, Hk, dh, dtype, 1), OO.frequencies(rd), 5000
    g = [I.gaussian(331, i, (dh,), 1.0, "f32") for i in range(2)]
    got = P.qk_norm_rotary(*device(x), *device(g), torch.from_numpy(f).cuda(), d_head=dh, S=S, interleaved=inter)
    for i in range(2):
        if x[i] is not None:
            v, pos = x[i].f64(), np.arange(T) % S
            size = OO.pair_size(OO.head_norm(v, g[i].f64(), dh, 1e-6)[0], rd // 2, dh, inter)
            close(got[i], OO.qk_norm_rotary(v, g[i].f64(), pos, f, dh, 1e-6, interleaved=inter), size, 2.0 ** -18, dtype, "QK"[i])


@pytest.mark.parametrize("T,Hq,Hk,dh,rd,dtype,inter", GRADIENTS)
def test_norm_gradients_of_many_tokens(T, Hq, Hk, dh, rd, dtype, inter):
    say(f"qk_norm_rotary_backward T={T} H={Hq}+{Hk} dh={dh} rd={rd} {dtype}")
    x, dy, f, S = gaussians(T, Hq, Hk, dh, dtype, 2), gaussians(T, Hq, Hk, dh, dtype, 3), OO.frequencies(rd), 5000
    g = [I.gaussian(331, i, (dh,), 1.0, "f32") for i in range(2)]
    got = P.qk_norm_rotary_backward(*device(x), *device(dy), *device(g), torch.from_numpy(f).cuda(), d_head=dh, S=S, interleaved=inter)
    for i in range(2):
        if x[i] is None:
            continue
        v, d = x[i].f64(), dy[i].f64()
        dx, dg = OO.qk_norm_rotary_backward(v, g[i].f64(), d, np.arange(T) % S, f, dh, 1e-6, interleaved=inter)
        h, r = np.abs(v).reshape(T, -1, dh), OO.head_norm(v, None, dh, 1e-6)[1]
        dn = OO.pair_size(d, rd // 2, dh, inter).reshape(T, -1, dh) + np.abs(d).reshape(T, -1, dh)
        u = dn * np.abs(g[i].f64())
        terms = r * u + h * r ** 3 * (h * u).mean(-1, keepdims=True)
        close(got[i], dx, terms.reshape(T, -1), 2.0 ** -17, dtype, "d" + "QK"[i])
        close(got[2 + i], dg, (dn * h * r).sum((0, 1)), 2.0 ** -16, "f32", "dg" + "qk"[i])


# chunks are of 32 KiB, at most 2048 workgroups share a table of up to 144 tensors
F, B = torch.float32, torch.bfloat16
CHUNKS = [([9_000_001, 8_000_003, 77, 12_345_679, 16_000_000, 1, 5_000_000], [F, B, F, F, B, B, F])]


@pytest.mark.parametrize("sizes,kinds", CHUNKS)
@pytest.mark.parametrize("apart", [False, True])
def test_clipping_in_runs_of_chunks(sizes, kinds, apart):
    say(f"clip {sum(sizes)} values, out of place {apart}")
    g = torch.Generator(device="cuda").manual_seed(7)
    flat = {k: torch.randn(sum(n for n, kk in zip(sizes, kinds) if kk is k), generator=g, device="cuda").to(k) for k in (F, B)}
    at, ts = dict.fromkeys(flat, 0), []
    for n, k in zip(sizes, kinds):           # neighbours in a bucket, of odd sizes
        ts.append(flat[k][at[k]:at[k] + n])
        at[k] += n
    check_clip(ts, 0.5, **({"out": [torch.full_like(t, 9.0) for t in ts]} if apart else {}))
