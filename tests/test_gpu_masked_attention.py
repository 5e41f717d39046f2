"""GPU parity of masked attention (forward, training forward, gradients) against
the fp64 oracle.

Tolerances are those of tests/test_gpu_cross_attention.py with what the changed
scores add to a weight's relative error e: a cap's tanh is formed as 1 - 2 r, r = 1 /
(1 + 2^x), where exp2, the sum and the reciprocal leave 2^-22 each of numbers up to
1, so z is off by 2^-20 of the cap at most; the bias is a product and a sum, 2^-22
of the largest; the cap's derivative 4 r (1 - r) is off by 2^-19.  Weights below
2^-126, the least that float32 and bf16 hold, are 0 (a bias of 600 gives 10^-260):
2^-125 is added to every weight's error; a gradient below 2^-126 is rounded to
bf16's steps there, 2^-133."""
import math

import numpy as np
import pytest
import torch

from oracle import masked_oracle as MO
from paper_2401_11202_amd import inputs as I
from paper_2401_11202_amd import partir as P
from tests.gpu_common import host, say
from tests.test_gpu_cross_attention import check

pytestmark = pytest.mark.gpu
DH = 128


def clamp(lens, B, S):
    return [S] * B if lens is None else [max(0, min(int(n), S)) for n in lens]


def packed(B, S, mean, seed=0):
    """Documents one after the other in every row."""
    rng = np.random.default_rng(seed)
    out = []
    for _ in range(B):
        row = np.repeat(np.arange(S), rng.integers(1, 2 * mean, size=S))[:S]
        out.append(row)
    return np.concatenate(out)


def make(B, Sq, Sk, Hq, Hk, mask, wid, qscale=1.0):
    """Device tensors as columns of fused projections, NaN behind the lengths, and their fp64 values."""
    QG = I.gaussian(500, wid, (B * Sq, 2 * Hq * DH), qscale)
    KV = I.gaussian(501, wid, (B * Sk, 2 * Hk * DH), 1.0)
    qg, kv = QG.to_device(), KV.to_device()
    for b, n in enumerate(clamp(mask.get("k_lens"), B, Sk)):
        kv[b * Sk + n:(b + 1) * Sk] = float("nan")
    for b, n in enumerate(clamp(mask.get("q_lens"), B, Sq)):
        qg[b * Sq + n:(b + 1) * Sq] = float("nan")
    a, c = QG.f64(), KV.f64()
    dev = (qg[:, :Hq * DH], kv[:, :Hk * DH], kv[:, Hk * DH:], qg[:, Hq * DH:])
    return dev, (a[:, :Hq * DH], c[:, :Hk * DH], c[:, Hk * DH:], a[:, Hq * DH:])


def device_mask(mask):
    out = {}
    for k, v in mask.items():
        if k == "slopes":
            out[k] = torch.tensor(np.asarray(v), dtype=torch.float32, device="cuda")
        elif k in ("causal", "cap"):
            out[k] = v
        else:
            out[k] = torch.tensor(np.asarray(v), dtype=torch.int64, device="cuda").to(torch.int32)
    return out


def run(B, Sq, Sk, Hq, Hk, mask=None, scale=None, wid=0, qscale=1.0, backward=True):
    mask = dict(mask or {})
    say(f"masked_attention B={B} Sq={Sq} Sk={Sk} heads {Hq}/{Hk} scale={scale} "
        f"{ {k: (v if np.size(v) < 9 else 'array') for k, v in mask.items()} }")
    (Q, K, V, dO), (q, k, v, g) = make(B, Sq, Sk, Hq, Hk, mask, wid, qscale)
    dm = device_mask(mask)
    if "slopes" in mask:
        mask["slopes"] = np.asarray(mask["slopes"], np.float32).astype(np.float64)
    kw = dict(B=B, Sq=Sq, Sk=Sk, n_heads=Hq, n_kv_heads=Hk, scale=0.0 if scale is None else scale, **dm)
    O, lse = P.masked_attention_train(Q, K, V, **kw)
    assert torch.equal(P.masked_attention(Q, K, V, **kw), O)
    refs = MO.attention(q, k, v, B, Sq, Sk, Hq, Hk, scale, dO=g, **mask)
    bound = MO.bounds(q, k, v, g, refs[0], B, Sq, Sk, Hq, Hk, scale, **mask)
    check("O", O, refs[0], bound[0])
    check("lse", lse, refs[1], bound[1])
    assert bool((O.float().reshape(B * Sq, Hq, DH)[lse == -math.inf] == 0).all())
    if not backward:
        return
    grads = P.masked_attention_backward(Q, K, V, O, dO, lse, **kw)
    again = P.masked_attention_backward(Q, K, V, O, dO, lse, **kw)
    for name, x, y, r, bd in zip(("dQ", "dK", "dV"), grads, again, refs[2:], bound[2:]):
        assert torch.equal(x, y), name
        check(name, x, r, bd + 2.0 ** -133)


@pytest.mark.parametrize("S", [1, 2, 31, 32, 33, 64, 65, 127, 129, 200, 257, 330])
@pytest.mark.parametrize("Hq,Hk", [(2, 2), (4, 1), (3, 1)])
def test_causal_self_attention(S, Hq, Hk):
    run(2, S, S, Hq, Hk, wid=S)


@pytest.mark.parametrize("Sq,Sk", [(1, 1), (1, 70), (5, 200), (33, 100), (100, 333), (130, 130), (70, 40), (200, 3)])
@pytest.mark.parametrize("Hq,Hk", [(4, 1), (6, 2), (1, 1)])
def test_queries_at_the_end_of_the_keys(Sq, Sk, Hq, Hk):
    """More queries than keys: the first ones see none."""
    run(1, Sq, Sk, Hq, Hk, wid=Sq + Sk)


FORMS = [dict(cap=2.0), dict(cap=50.0), dict(slopes=True), dict(cap=5.0, slopes=True)]


def form(f, Hq):
    f = dict(f)
    if f.pop("slopes", None):
        f["slopes"] = [2.0 ** (-4.0 * (h + 1) / Hq) for h in range(Hq)]
    return f


@pytest.mark.parametrize("f", FORMS)
@pytest.mark.parametrize("B,Sq,Sk,Hq,Hk", [(1, 1, 300, 8, 2), (2, 3, 90, 4, 4), (2, 150, 150, 4, 2), (1, 400, 400, 2, 1), (1, 60, 700, 6, 1),
                                           (3, 290, 290, 8, 8)])
def test_changed_scores(B, Sq, Sk, Hq, Hk, f):
    run(B, Sq, Sk, Hq, Hk, form(f, Hq), wid=Sq)


@pytest.mark.parametrize("f", [{}, *FORMS])
@pytest.mark.parametrize("causal", [True, False])
def test_documents(f, causal):
    B, S = 2, 390
    ids = packed(B, S, 60)
    run(B, S, S, 4, 2, dict(form(f, 4), causal=causal, q_docs=ids, k_docs=ids), wid=3)


@pytest.mark.parametrize("kind", ["random", "one key each", "apart", "long", "ends of 64", "signed"])
def test_documents_in_any_order(kind):
    B, S = 2, 320
    rng = np.random.default_rng(4)
    q = {"random": rng.integers(0, 5, B * S), "one key each": np.arange(B * S), "apart": np.zeros(B * S), "long": np.repeat([3, 9, 9, 4], B * S // 4),
         "ends of 64": np.arange(B * S) // 64, "signed": rng.choice([-2 ** 31, 2 ** 31 - 1, -1, 0], B * S)}[kind]
    k = np.ones(B * S) if kind == "apart" else q
    run(B, S, S, 3, 1, dict(q_docs=q, k_docs=k), wid=5)
    run(B, S, S, 2, 2, dict(causal=False, q_docs=q, k_docs=k), wid=6)


def test_documents_of_another_sequence():
    """Queries and keys with document numbers of their own, queries behind the prompt."""
    rng = np.random.default_rng(6)
    run(2, 40, 500, 4, 1, dict(q_docs=np.repeat([1, 2, 3, 9], 20), k_docs=np.sort(rng.integers(0, 4, (2, 500)), 1).reshape(-1)), wid=8)


@pytest.mark.parametrize("S,lens,prefix", [(200, [200, 77, 0], [30, 0, 10]), (300, [1, 300, 129], [1, 300, 64]), (130, [65, 64, 63], [63, 64, 65]),
                                           (520, [520, 257, 256], [255, 256, 257])])
@pytest.mark.parametrize("f", [{}, FORMS[3]])
def test_padded_batches_with_prefixes(S, lens, prefix, f):
    run(3, S, S, 4, 2, dict(form(f, 4), k_lens=lens, q_lens=lens, prefix_lens=prefix), wid=S)


@pytest.mark.parametrize("f", [{}, *FORMS])
@pytest.mark.parametrize("B,Sq,Sk,Hq,Hk,lens", [(4, 1, 900, 8, 2, [900, 1, 0, 433]), (3, 4, 200, 4, 4, [4, 100, 200]), (2, 70, 300, 6, 2, [300, 71])])
def test_new_tokens_over_a_ragged_cache(B, Sq, Sk, Hq, Hk, lens, f):
    run(B, Sq, Sk, Hq, Hk, dict(form(f, Hq), k_lens=lens, q_starts=[n - Sq for n in lens]), wid=Sk, backward=Sq < 5)


@pytest.mark.parametrize("mask", [dict(q_starts=[-2 ** 31, 2 ** 31 - 1]), dict(q_starts=[-100, 1000]), dict(k_lens=[-5, 2 ** 31 - 1]),
                                  dict(q_lens=[-1, 2 ** 30]), dict(prefix_lens=[-7, 2 ** 31 - 1]), dict(k_lens=[0, 0]), dict(q_lens=[0, 0]),
                                  dict(causal=False, q_lens=[90, 3], k_lens=[2, 140])])
def test_numbers_out_of_their_range(mask):
    ref = dict(mask)
    run(2, 150, 150, 2, 1, ref, wid=9)


@pytest.mark.parametrize("B,Sq,Sk,Hq,Hk", [(1, 1, 5000, 4, 1), (2, 1, 4096, 8, 8), (1, 3, 9001, 2, 2), (1, 100, 4100, 2, 1), (1, 1100, 1100, 2, 1),
                                           (2, 900, 900, 1, 1)])
@pytest.mark.parametrize("f", [{}, FORMS[3]])
def test_axes_in_parts(B, Sq, Sk, Hq, Hk, f):
    p, q = P.plan_masked_attention(B, Sq, Sk, Hq, Hk), P.plan_masked_attention_backward(B, Sq, Sk, Hq, Hk)
    assert p["n_virtual_shards"] > 1 or q["n_virtual_shards"] > 1
    run(B, Sq, Sk, Hq, Hk, form(f, Hq), wid=Sk + Sq)
    if Sq == Sk:
        ids = packed(B, Sq, 200)
        run(B, Sq, Sk, Hq, Hk, dict(form(f, Hq), q_docs=ids, k_docs=ids), wid=Sk + Sq)


@pytest.mark.parametrize("B,S,Hq,Hk", [(9, 500, 8, 8), (7, 450, 20, 4)])
@pytest.mark.parametrize("f", [{}, FORMS[3]])
def test_grids_without_parts(B, S, Hq, Hk, f):
    """Enough workgroups that the forward takes whole axes, with heads of whole rounds of the XCDs and without."""
    assert P.plan_masked_attention(B, S, S, Hq, Hk)["n_virtual_shards"] == 1
    ids = packed(B, S, 150)
    run(B, S, S, Hq, Hk, dict(form(f, Hq), q_docs=ids, k_docs=ids), wid=S)


@pytest.mark.parametrize("B,S,Hq,Hk", [(33, 130, 8, 8), (43, 97, 9, 3), (65, 161, 4, 4), (67, 143, 6, 2)])
@pytest.mark.parametrize("f", [{}, *FORMS])
def test_many_short_sequences(B, S, Hq, Hk, f):
    """The kernels of many workgroups in every form, without documents, on ragged batches."""
    lens = [S - (37 * b) % (S + 1) for b in range(B)]
    run(B, S, S, Hq, Hk, dict(form(f, Hq), k_lens=lens, q_lens=lens), wid=S)


@pytest.mark.parametrize("B,Sq,Sk,Hq,Hk", [(3, 64, 64, 4, 2), (2, 128, 128, 8, 1), (260, 20, 20, 1, 1), (130, 45, 33, 6, 2), (1, 300, 127, 6, 1),
                                           (270, 90, 100, 3, 1), (2, 5, 97, 12, 4), (3, 400, 1, 2, 1)])
@pytest.mark.parametrize("f", [{}, *FORMS])
def test_up_to_128_keys(B, Sq, Sk, Hq, Hk, f):
    """All gradients in one launch: ragged queries and keys, prefixes; then documents, in one piece each and not."""
    if Sq == Sk:
        lens = [S - (7 * b) % (S + 1) for b, S in enumerate([Sk] * B)]
        run(B, Sq, Sk, Hq, Hk, dict(form(f, Hq), k_lens=lens, q_lens=lens, prefix_lens=[n // 3 for n in lens]), wid=Sk)
    else:
        run(B, Sq, Sk, Hq, Hk, dict(form(f, Hq), q_lens=[Sq - (11 * b) % (Sq + 1) for b in range(B)], q_starts=[(5 * b) % 9 - 3 for b in range(B)]),
            wid=Sk)
    q, k = packed(B, Sq, 9), packed(B, Sk, 9)
    run(B, Sq, Sk, Hq, Hk, dict(form(f, Hq), q_docs=q, k_docs=k), wid=Sk + 1)
    run(B, Sq, Sk, Hq, Hk, dict(form(f, Hq), causal=False, q_docs=q % 3, k_docs=k % 3), wid=Sk + 1)


@pytest.mark.parametrize("scale,qscale", [(1.0, 1.0), (0.02, 1.0), (1.0, 4.0)])
@pytest.mark.parametrize("cap", [0.0, 30.0])
def test_scales_from_flat_to_one_hot(scale, qscale, cap):
    run(2, 180, 180, 4, 2, dict(cap=cap), scale, 77, qscale)


@pytest.mark.parametrize("slope", [0.0, -0.5, 30.0])
def test_slopes_of_any_size(slope):
    run(1, 300, 300, 2, 2, dict(slopes=[slope, slope / 3]), wid=12)


def test_capped_scores_at_their_ends():
    """Scores far past the cap: every weight alike; and a cap far above them: as without one."""
    Q, K = (torch.randn(64, 128, device="cuda").to(torch.bfloat16) * 1000 for _ in range(2))
    V = torch.randn(64, 128, device="cuda").to(torch.bfloat16)
    kw = dict(B=1, Sq=64, Sk=64, n_heads=1)
    O, lse = P.masked_attention_train(Q, K, V, causal=False, cap=2.0 ** -10, **kw)
    assert bool(((lse - 6).abs() < 2.0 ** -8).all())
    assert bool(((O.float() - V.float().mean(0)).abs() < 2.0 ** -6).all())
    Q, K = Q / 1000, K / 1000
    a, b = P.masked_attention(Q, K, V, cap=1024.0, **kw), P.masked_attention(Q, K, V, **kw)
    assert bool(((a.float() - b.float()).abs() <= 2.0 ** -6 * (1 + b.float().abs())).all())


def test_far_positions():
    """Queries millions of positions behind their keys: distances that float32 does not hold as two positions."""
    run(2, 140, 140, 2, 1, dict(causal=False, slopes=[2.0 ** -20, -(2.0 ** -21)], q_starts=[2 ** 25 + 3, -(2 ** 26) + 5]), wid=13)


def test_many_documents():
    """As many documents as the list of runs holds, and one more."""
    for n in (4096, 4097):
        ids = n - np.arange(n)
        run(1, n, n, 1, 1, dict(q_docs=ids, k_docs=ids), wid=14, backward=False)
    ids = np.arange(1500) // 2
    run(1, 1500, 1500, 1, 1, dict(q_docs=ids, k_docs=ids), wid=15)


@pytest.mark.parametrize("S", [1, 60, 130, 300])
@pytest.mark.parametrize("f", [dict(cap=1000.0), dict(cap=1000.0, slopes=True), {}])
def test_rows_of_one_key_have_no_gradient(S, f):
    """dS = P (dP - D) is 0 with one key, whatever P: D = P dP / P.  dP and D are
    float32 sums of the same 128 products, a product and a division, below 2^-20 of
    |dO| |V|^T; that P is off by 2^-20 of the cap must not show."""
    say(f"masked_attention S={S} {f}")
    B, H = 3, 2
    (Q, K, V, dO), (q, k, v, g) = make(B, S, S, H, H, {}, 50 + S)
    ids = torch.arange(B * S, device="cuda", dtype=torch.int32)
    kw = dict(B=B, Sq=S, Sk=S, n_heads=H, q_docs=ids, k_docs=ids, **device_mask(form(f, H)))
    O, lse = P.masked_attention_train(Q, K, V, **kw)
    dq, dk, _ = P.masked_attention_backward(Q, K, V, O, dO, lse, **kw)
    ds = 2.0 ** -20 * np.repeat((np.abs(g) * np.abs(v)).reshape(B * S, H, DH).sum(-1), DH, axis=1) * DH ** -0.5
    for name, got, x in (("dQ", dq, k), ("dK", dk, q)):
        past = np.abs(host(got)) - 1.01 * ds * np.abs(x)
        say(f"    {name}: largest error past its bound {past.max():.2e}")
        assert past.max() <= 0, name


def test_very_many_sequences():
    """More sequences than a launch has workgroups of 1024 threads.  One key: a query
    that sees it has weight 1, so O = V and dV = dO in every bit; dS = P (dP - D) is 0
    but for the errors of P and D, 2^-20 each of dP, and |dP| <= 128 * 6^2 with values
    up to 6."""
    B = 2 ** 22 + 3
    say(f"masked_attention B={B}")
    torch.manual_seed(0)
    Q, K, V, dO = (torch.randn(B, DH, device="cuda", dtype=torch.bfloat16).clamp_(-6, 6) for _ in range(4))
    kd = torch.arange(B, device="cuda", dtype=torch.int32)
    seen = kd % 3 != 1
    qd = torch.where(seen, kd, kd + 1)
    kw = dict(B=B, Sq=1, Sk=1, n_heads=1, q_docs=qd, k_docs=kd)
    O, lse = P.masked_attention_train(Q, K, V, **kw)
    assert torch.equal(O, V * seen[:, None]) and torch.equal(lse[:, 0] == -math.inf, ~seen)
    dq, dk, dv = P.masked_attention_backward(Q, K, V, O, dO, lse, **kw)
    assert torch.equal(dv, dO * seen[:, None])
    for g in (dq, dk):
        assert not g[~seen].any() and float(g.abs().max()) <= 2 * 2.0 ** -20 * (DH * 36) * 6 * DH ** -0.5


def test_nothing_to_do():
    e = torch.zeros(0, 256, device="cuda", dtype=torch.bfloat16)
    x = torch.randn(6, 256, device="cuda").to(torch.bfloat16)
    ids = torch.zeros(6, device="cuda", dtype=torch.int32)
    O, lse = P.masked_attention_train(x, e, e, B=2, Sq=3, Sk=0, n_heads=2)
    assert not O.any() and bool((lse == -math.inf).all())
    assert not P.masked_attention(x, e, e, B=2, Sq=3, Sk=0, n_heads=2, q_docs=ids, k_docs=ids[:0]).any()
    dq, dk, dv = P.masked_attention_backward(x, e, e, O, x, lse, B=2, Sq=3, Sk=0, n_heads=2)
    assert not dq.any() and dk.shape == (0, 256)
    assert P.masked_attention(e, x, x, B=2, Sq=0, Sk=3, n_heads=2).shape == (0, 256)
    lse0 = torch.zeros(0, 2, device="cuda")
    dq, dk, dv = P.masked_attention_backward(e, x, x, e, e, lse0, B=2, Sq=0, Sk=3, n_heads=2)
    assert not dk.any() and not dv.any()


def test_output_in_the_queries_place_and_gradients_into_views():
    S, Hq, Hk = 150, 4, 2
    (Q, K, V, dO), _ = make(2, S, S, Hq, Hk, {}, 40)
    kw = dict(B=2, Sq=S, Sk=S, n_heads=Hq, n_kv_heads=Hk, cap=9.0)
    O, lse = P.masked_attention_train(Q, K, V, **kw)
    g = P.masked_attention_backward(Q, K, V, O, dO, lse, **kw)
    wide = torch.full((2 * S, (Hq + 2 * Hk) * DH + 8), 3.0, device="cuda", dtype=torch.bfloat16)
    out = (wide[:, :Hq * DH], wide[:, Hq * DH:(Hq + Hk) * DH], wide[:, (Hq + Hk) * DH:-8])
    P.masked_attention_backward(Q, K, V, O, dO, lse, out=out, **kw)
    assert all(torch.equal(a, b) for a, b in zip(out, g)) and bool((wide[:, -8:] == 3).all())
    assert P.masked_attention(Q, K, V, out=Q, **kw) is Q and torch.equal(Q, O)


def test_a_captured_step_reads_its_masks_at_every_replay():
    B, S, Hq, Hk = 2, 260, 4, 2
    (Q, K, V, dO), _ = make(B, S, S, Hq, Hk, {}, 41)
    ids = torch.tensor(packed(B, S, 50), dtype=torch.int32, device="cuda")
    lens = torch.tensor([260, 100], dtype=torch.int32, device="cuda")
    kw = dict(B=B, Sq=S, Sk=S, n_heads=Hq, n_kv_heads=Hk, cap=20.0, q_docs=ids, k_docs=ids, k_lens=lens, q_lens=lens)

    def step():
        O, lse = P.masked_attention_train(Q, K, V, **kw)
        return [O, lse, *P.masked_attention_backward(Q, K, V, O, dO, lse, **kw)]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for r in range(3):
        lens.copy_(torch.tensor([260 - 70 * r, 100 + 50 * r], dtype=torch.int32))
        ids.copy_(torch.tensor(packed(B, S, 30 + 40 * r, r), dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, step()):
            assert torch.equal(a, b)


def test_a_captured_step_of_short_sequences():
    """The one launch for all gradients, which must leave the gradients of rows that a shorter batch no longer has at 0."""
    B, S, Hq, Hk = 3, 120, 4, 1
    (Q, K, V, dO), _ = make(B, S, S, Hq, Hk, {}, 44)
    ids = torch.tensor(packed(B, S, 30), dtype=torch.int32, device="cuda")
    lens = torch.tensor([120, 100, 3], dtype=torch.int32, device="cuda")
    kw = dict(B=B, Sq=S, Sk=S, n_heads=Hq, n_kv_heads=Hk, cap=20.0, q_docs=ids, k_docs=ids, k_lens=lens, q_lens=lens)

    def step():
        O, lse = P.masked_attention_train(Q, K, V, **kw)
        return [O, lse, *P.masked_attention_backward(Q, K, V, O, dO, lse, **kw)]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for r in range(4):
        lens.copy_(torch.tensor([120 - 40 * r, 30 * r, 7 + r], dtype=torch.int32))
        ids.copy_(torch.tensor(packed(B, S, 5 + 20 * r, r), dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, step()):
            assert torch.equal(a, b)
        assert not outs[2].reshape(B, S, -1)[1, 30 * r:].any()


@pytest.mark.parametrize("S", [110, 700])
def test_two_graphs_share_a_workspace(S):
    """Each call writes what it reads of a workspace."""
    Hq, Hk = 4, 1
    ws = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    graphs, steps = [], []
    for i, mean in enumerate((20, 90)):
        (Q, K, V, dO), _ = make(2, S, S, Hq, Hk, {}, 46 + i)
        ids = torch.tensor(packed(2, S, mean, i), dtype=torch.int32, device="cuda")
        kw = dict(B=2, Sq=S, Sk=S, n_heads=Hq, n_kv_heads=Hk, q_docs=ids, k_docs=ids)

        def step(Q=Q, K=K, V=V, dO=dO, kw=kw, ws=ws):
            O, lse = P.masked_attention_train(Q, K, V, workspace=ws, **kw)
            return [O, lse, *P.masked_attention_backward(Q, K, V, O, dO, lse, workspace=ws, **kw)]

        steps.append(step)
        step()
        torch.cuda.synchronize()
        graphs.append((torch.cuda.CUDAGraph(), []))
        with torch.cuda.graph(graphs[-1][0]):
            graphs[-1][1].extend(step())
    want = [[x.clone() for x in s(ws=None)] for s in steps]
    for _ in range(3):
        for graph, outs in graphs:
            for x in outs:
                x.fill_(7)
            ws.fill_(255)
            graph.replay()
        torch.cuda.synchronize()
        for (_, outs), w in zip(graphs, want):
            assert all(torch.equal(a, b) for a, b in zip(outs, w))


def test_two_streams_at_once():
    ids = torch.tensor(packed(2, 500, 100), dtype=torch.int32, device="cuda")
    cases = []
    for i, m in enumerate((dict(cap=30.0), dict(q_docs=ids, k_docs=ids))):
        (Q, K, V, dO), _ = make(2, 500, 500, 4, 2, {}, 42 + i)
        cases.append((Q, K, V, dO, dict(B=2, Sq=500, Sk=500, n_heads=4, n_kv_heads=2, **m)))

    def step(Q, K, V, dO, kw, stream=None):
        O, lse = P.masked_attention_train(Q, K, V, stream=stream, **kw)
        return [O, lse, *P.masked_attention_backward(Q, K, V, O, dO, lse, stream=stream, **kw)]

    want = [step(*c) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = [step(*c, stream=s) for c, s in zip(cases, streams)]
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(g, w))
