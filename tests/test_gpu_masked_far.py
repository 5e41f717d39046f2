"""Masked attention where its other GPU tests do not reach: keys and values whose
offsets pass 32 bits."""
import pytest
import torch

from paper_2401_11202_amd import inputs as I
from paper_2401_11202_amd import partir as P
from tests.gpu_common import say
from tests.test_gpu_masked_attention import DH, FORMS, form

pytestmark = pytest.mark.gpu


def tensors(wid, Tq, Tk, cq, ck):
    return [I.gaussian(wid, i, (n, c), 1.0).to_device() for i, (n, c) in enumerate(((Tq, cq), (Tk, ck), (Tk, ck), (Tq, cq)))]


@pytest.mark.parametrize("B,Sq,Sk", [(1, 1, 70000), (2, 1, 33000), (1, 300, 70000), (2, 2500, 2500)])
def test_offsets_past_32_bits(B, Sq, Sk):
    """Keys and values (and the queries of a training step) as columns of rows of up to
    2^24 values: the same results in every bit as from dense ones."""
    Hq, Hk, f = 4, 2, form(FORMS[3], 4)
    ld = 2 ** 20 if B * Sk < 2 ** 13 else 2 ** 16
    Q, K, V, dO = tensors(72, B * Sq, B * Sk, Hq * DH, Hk * DH)
    wide = torch.empty(B * Sk, ld, dtype=torch.bfloat16, device="cuda")
    assert (B * Sk - 1) * ld * 2 > 2 ** 32 and (B * Sk - 1) * ld > 2 ** 31
    say(f"masked_attention B={B} Sq={Sq} Sk={Sk} leading dim {ld}")
    k, v = wide[:, 8:8 + Hk * DH], wide[:, ld - Hk * DH:]
    k.copy_(K)
    v.copy_(V)
    q, g = Q, dO
    if Sq == Sk:
        q, g = wide[:, 1024:1024 + Hq * DH], wide[:, 2048:2048 + Hq * DH]
        q.copy_(Q)
        g.copy_(dO)
    kw = dict(B=B, Sq=Sq, Sk=Sk, n_heads=Hq, n_kv_heads=Hk, slopes=torch.tensor(f["slopes"], device="cuda"), cap=f["cap"])
    O, lse = P.masked_attention_train(Q, K, V, **kw)
    o, l = P.masked_attention_train(q, k, v, **kw)
    assert torch.equal(o, O) and torch.equal(l, lse)
    want = P.masked_attention_backward(Q, K, V, O, dO, lse, **kw)
    out = None
    if Sq == Sk:
        out = tuple(wide[:, 4096 * (i + 1):4096 * (i + 1) + t.shape[1]] for i, t in enumerate(want))
    got = P.masked_attention_backward(q, k, v, o, g, l, out=out, **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
