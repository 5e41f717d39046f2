"""Masked attention where its other GPU tests do not reach: documents behind the 4096th
query, caches whose offsets pass 32 bits, and calls that find other things in their
workspace and outputs.  Tolerances are those of tests/test_gpu_masked_attention.py."""
import numpy as np
import pytest
import torch

from paper_2401_11202_amd import inputs as I
from paper_2401_11202_amd import partir as P
from tests.gpu_common import say
from tests.test_gpu_masked_attention import DH, FORMS, form, packed, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lengths", [(4000, 96, 104, 100), (3500, 700, 100), (65, 4031, 1, 199), (4095, 2, 203)])
@pytest.mark.parametrize("down", [False, True])
def test_gradients_of_documents_behind_the_4096th_query(lengths, down):
    """dK and dV look at 64 blocks of 64 queries at a time: documents on both sides of the 4096th query, and across it."""
    S = sum(lengths)
    ids = np.repeat(np.arange(len(lengths)), lengths)
    run(1, S, S, 1, 1, dict(q_docs=-ids if down else ids, k_docs=-ids if down else ids), wid=70)


def test_gradients_of_documents_of_queries_in_several_pieces_of_the_keys():
    """More queries than keys, whose documents lie in another order than the keys': the queries of a key block are far apart."""
    Sq, Sk = 4500, 400
    rng = np.random.default_rng(8)
    q = np.repeat(rng.permutation(30), 150)
    k = np.repeat(np.arange(40), 10)
    run(1, Sq, Sk, 1, 1, dict(causal=False, q_docs=q, k_docs=k), wid=71)


def tensors(wid, Tq, Tk, cq, ck):
    return [I.gaussian(wid, i, (n, c), 1.0).to_device() for i, (n, c) in enumerate(((Tq, cq), (Tk, ck), (Tk, ck), (Tq, cq)))]


@pytest.mark.parametrize("B,Sq,Sk,Hq,Hk,ld", [(1, 1, 70000, 4, 2, 2 ** 16), (2, 1, 33000, 4, 2, 2 ** 16), (1, 300, 70000, 4, 2, 2 ** 16),
                                              (2, 2500, 2500, 4, 2, 2 ** 20), (1, 2900, 2900, 3, 1, 2 ** 20), (2, 128, 128, 4, 2, 2 ** 24),
                                              (2, 128, 128, 3, 1, 2 ** 24), (1, 300, 300, 2, 2, 2 ** 24), (1, 270, 270, 3, 1, 2 ** 24),
                                              (1, 1, 200, 8, 2, 2 ** 24)])
def test_offsets_past_32_bits(B, Sq, Sk, Hq, Hk, ld):
    """Keys and values (and the queries and gradients of a training step) as columns of
    rows of up to 2^24 values: the same results in every bit as from dense ones."""
    f = form(FORMS[3], Hq)
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


@pytest.mark.parametrize("B,Sq,Sk,Hq,Hk,docs,ragged", [(16, 1, 2047, 32, 8, 0, True), (1, 509, 4096, 32, 8, 0, False), (2, 2048, 2048, 16, 16, 300, False),
                                                      (2, 1500, 1500, 32, 8, 0, True), (3, 333, 333, 12, 4, 0, True), (3, 100, 100, 12, 4, 30, True)])
@pytest.mark.parametrize("f", [FORMS[1], FORMS[2]])
def test_results_repeat_whatever_workspace_and_outputs_held(B, Sq, Sk, Hq, Hk, docs, ragged, f):
    say(f"masked_attention B={B} Sq={Sq} Sk={Sk} heads {Hq}/{Hk} docs={docs} ragged={ragged} {f}")
    Q, K, V, dO = tensors(73, B * Sq, B * Sk, Hq * DH, Hk * DH)
    f = form(f, Hq)
    kw = dict(B=B, Sq=Sq, Sk=Sk, n_heads=Hq, n_kv_heads=Hk, cap=f.get("cap", 0.0))
    if "slopes" in f:
        kw["slopes"] = torch.tensor(f["slopes"], device="cuda")
    if docs:
        kw["q_docs"] = kw["k_docs"] = torch.tensor(packed(B, Sk, docs), dtype=torch.int32, device="cuda")
    if ragged:
        kw["k_lens"] = torch.tensor([Sk - (b * Sk) // (B + 1) for b in range(B)], dtype=torch.int32, device="cuda")
        if Sq == Sk:
            kw["q_lens"] = kw["k_lens"]
    O, lse = P.masked_attention_train(Q, K, V, **kw)
    first = [O, lse, *P.masked_attention_backward(Q, K, V, O, dO, lse, **kw)]
    need = max(P.plan_masked_attention(B, Sq, Sk, Hq, Hk, docs=bool(docs))["workspace_bytes"],
               P.plan_masked_attention_backward(B, Sq, Sk, Hq, Hk, docs=bool(docs))["workspace_bytes"])
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    for fill in (255, 0, 127):                     # NaN, 0, 3e38
        outs = [t.clone().fill_(float("nan")) for t in first]
        ws.fill_(fill)
        P.masked_attention_train(Q, K, V, out=outs[0], lse=outs[1], workspace=ws, **kw)
        ws.fill_(fill)
        P.masked_attention_backward(Q, K, V, outs[0], dO, outs[1], out=tuple(outs[2:]), workspace=ws, **kw)
        assert all(torch.equal(a, b) for a, b in zip(outs, first))
