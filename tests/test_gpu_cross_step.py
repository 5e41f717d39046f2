"""The operators together, as a training step and a serving step use them: a
cross attention layer with normed, rotated queries and keys -- projections,
norms with the rotation, attention over the encoder's states, the output
projection, every gradient back to the weights, and their clipping -- against
autograd in fp64 on the CPU.

Tolerance: chained products round several bf16 intermediates; the error of each
result relative to its whole size stays within the framework's bound for such
chains (tests/gpu_common.py)."""
import numpy as np
import pytest
import torch

from paper_2401_11202_amd import inputs as I
from paper_2401_11202_amd import partir as P
from tests.gpu_common import TOL_REL_FRO, host, rel_fro, say

pytestmark = pytest.mark.gpu
B, Sq, Sk, D, Hq, Hk, DH = 2, 24, 41, 512, 4, 2, 128
LENS = [41, 17]


def layer64(x, states, W, g, f, lens, dY):
    """Output and gradients of the layer by autograd in fp64."""
    leaf = {k: torch.from_numpy(v).requires_grad_() for k, v in dict(W, gq=g[0], gk=g[1]).items()}
    x, states, dY = (torch.from_numpy(t) for t in (x, states, dY))

    def heads(t, gain, S):
        t = t.reshape(B, S, -1, DH)
        t = t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6) * gain
        z = torch.polar(torch.ones(1, dtype=torch.float64), torch.outer(torch.arange(S, dtype=torch.float64), f))[None, :, None]
        z = torch.complex(t[..., :DH // 2], t[..., DH // 2:]) * z
        return torch.cat((z.real, z.imag), -1)

    q = heads(x @ leaf["Wq"], leaf["gq"], Sq)
    kv = states @ leaf["Wkv"]
    k = heads(kv[:, :Hk * DH], leaf["gk"], Sk)
    v = kv[:, Hk * DH:].reshape(B, Sk, Hk, DH)
    out = []
    for b in range(B):
        kk, vv = (t[b, :lens[b]].transpose(0, 1).repeat_interleave(Hq // Hk, 0) for t in (k, v))
        s = q[b].transpose(0, 1) @ kk.transpose(1, 2) / DH ** 0.5
        out.append((torch.softmax(s, -1) @ vv).transpose(0, 1).reshape(Sq, -1))
    y = torch.cat(out) @ leaf["Wo"]
    return y.detach().numpy(), {k: t.numpy() for k, t in zip(leaf, torch.autograd.grad(y, list(leaf.values()), dY))}


def test_training_step():
    say("cross attention layer: training step")
    x, states = I.gaussian(320, 0, (B * Sq, D)), I.gaussian(320, 1, (B * Sk, D))
    W = {"Wq": I.gaussian(320, 2, (D, Hq * DH), D ** -0.5), "Wkv": I.gaussian(320, 3, (D, 2 * Hk * DH), D ** -0.5),
         "Wo": I.gaussian(320, 4, (Hq * DH, D), D ** -0.5)}
    g = [I.gaussian(320, 5 + i, (DH,), 1.0, "f32") for i in range(2)]
    dY = I.gaussian(320, 7, (B * Sq, D))
    f = P.rotary_frequencies(DH)
    X, E, dYd = x.to_device(), states.to_device(), dY.to_device()
    Wd = {k: w.to_device() for k, w in W.items()}
    gq, gk = (t.to_device() for t in g)
    lens = torch.tensor(LENS, dtype=torch.int32, device="cuda")
    kw = dict(B=B, Sq=Sq, Sk=Sk, n_heads=Hq, n_kv_heads=Hk, k_lens=lens)
    # forward
    q0 = P.loop_matmul(X, Wd["Wq"], tile="N", R=2)
    kv = P.loop_matmul(E, Wd["Wkv"], tile="N", R=2)
    k0, v = kv[:, :Hk * DH], kv[:, Hk * DH:]
    q, _ = P.qk_norm_rotary(q0, None, gq, None, f, d_head=DH, S=Sq)
    k, _ = P.qk_norm_rotary(k0, None, gk, None, f, d_head=DH, S=Sk)
    o, lse = P.cross_attention_train(q, k, v, **kw)
    y = P.loop_matmul(o, Wd["Wo"], sum="K", R=2, out_dtype=torch.float32)
    # backward: every gradient of a weight is a product over the tokens
    tr = lambda t: t.t().contiguous()  # noqa: E731
    dWo = P.loop_matmul(tr(o), dYd, out_dtype=torch.float32)
    do = P.loop_matmul(dYd, Wd["Wo"], b_layout="nk")
    dkv = torch.empty_like(kv)
    dq, _, _ = P.cross_attention_backward(q, k, v, o, do, lse, out=(torch.empty_like(q), dkv[:, :Hk * DH], dkv[:, Hk * DH:]), **kw)
    dq0, _, dgq, _ = P.qk_norm_rotary_backward(q0, None, dq, None, gq, None, f, d_head=DH, S=Sq, out=(dq, None))
    dk = dkv[:, :Hk * DH]
    _, _, dgk, _ = P.qk_norm_rotary_backward(k0, None, dk, None, gk, None, f, d_head=DH, S=Sk, out=(dk, None))
    pad = lambda t: torch.nn.functional.pad(t, (0, -t.shape[1] % 8))  # noqa: E731  tokens in 16-byte runs
    dWkv = P.loop_matmul(pad(tr(E)), pad(tr(dkv)), b_layout="nk", out_dtype=torch.float32)
    dWq = P.loop_matmul(tr(X), dq0, out_dtype=torch.float32)
    grads = {"Wq": dWq, "Wkv": dWkv, "Wo": dWo, "gq": dgq, "gk": dgk}
    ry, ref = layer64(x.f64(), states.f64(), {k: w.f64() for k, w in W.items()}, [t.f64() for t in g], f.cpu(), LENS, dY.f64())
    assert rel_fro(host(y), ry) < TOL_REL_FRO
    for name, t in grads.items():
        err = rel_fro(host(t), ref[name])
        say(f"    d{name}: relative error {err:.2e}")
        assert err < TOL_REL_FRO
    before = {n: t.clone() for n, t in grads.items()}
    norm = float(P.clip_grad_norm(list(grads.values()), 1.0))
    want = np.sqrt(sum((r ** 2).sum() for r in ref.values()))
    assert abs(norm / want - 1) < TOL_REL_FRO
    for n, t in grads.items():
        assert (np.abs(host(t) - host(before[n]) / norm) <= 2.0 ** -22 * np.abs(host(t)) + 2.0 ** -140).all()


def test_single_tokens_continue_a_prompt():
    """Queries given one at a time, at their positions, see what the prompt's
    call gave them: the same keys in another grouping of the sums, both within
    the attention's rounding."""
    Q = I.gaussian(321, 0, (B * Sq, Hq * DH)).to_device()
    KV = I.gaussian(321, 1, (B * Sk, 2 * Hk * DH)).to_device()
    f = P.rotary_frequencies(DH)
    gq, gk = (I.gaussian(321, 2 + i, (DH,), 1.0, "f32").to_device() for i in range(2))
    lens = torch.tensor(LENS, dtype=torch.int32, device="cuda")
    k, _ = P.qk_norm_rotary(KV[:, :Hk * DH], None, gk, None, f, d_head=DH, S=Sk)
    kw = dict(B=B, Sk=Sk, n_heads=Hq, n_kv_heads=Hk, k_lens=lens)
    q, _ = P.qk_norm_rotary(Q, None, gq, None, f, d_head=DH, S=Sq)
    whole = P.cross_attention(q, k, KV[:, Hk * DH:], Sq=Sq, **kw)
    big = host(KV).reshape(B, Sk, 2, Hk, DH)[:, :, 1]
    for s in (0, 5, Sq - 1):
        at = torch.arange(B, device="cuda") * Sq + s
        pos = torch.full((B,), s, dtype=torch.int32, device="cuda")
        one, _ = P.qk_norm_rotary(Q[at], None, gq, None, f, d_head=DH, positions=pos)
        assert torch.equal(one, q[at])
        got = host(P.cross_attention(one, k, KV[:, Hk * DH:], Sq=1, **kw))
        # two evaluations, each within 2^-8 of sum_j p_j |v_j| <= max_j |v_j| and a rounding of 2^-8
        for b in range(B):
            top = np.repeat(np.abs(big[b, :LENS[b]]).max(0), Hq // Hk, 0).reshape(-1)
            assert (np.abs(got[b] - host(whole[at])[b]) <= 4 * 2.0 ** -8 * top).all()


def test_two_streams_at_once():
    """Two chains of every operator, one replayed from a graph and one issued on
    another stream meanwhile, give what each gives alone."""
    f = P.rotary_frequencies(DH)
    gain = I.gaussian(322, 9, (DH,), 1.0, "f32").to_device()
    lens = torch.tensor(LENS, dtype=torch.int32, device="cuda")
    sets = [[I.gaussian(322, 4 * n + i, (r, c)).to_device() for i, (r, c) in
             enumerate(((B * Sq, Hq * DH), (B * Sk, 2 * Hk * DH), (B * Sq, Hq * DH)))] for n in range(2)]

    def chain(Q, KV, dO):
        q, _ = P.qk_norm_rotary(Q, None, gain, None, f, d_head=DH, S=Sq)
        k, _ = P.rotary(KV[:, :Hk * DH], None, f, d_head=DH, S=Sk)
        kw = dict(B=B, Sq=Sq, Sk=Sk, n_heads=Hq, n_kv_heads=Hk, k_lens=lens)
        o, lse = P.cross_attention_train(q, k, KV[:, Hk * DH:], **kw)
        dq, dk, dv = P.cross_attention_backward(q, k, KV[:, Hk * DH:], o, dO, lse, **kw)
        dx, _, dg, _ = P.qk_norm_rotary_backward(Q, None, dq, None, gain, None, f, d_head=DH, S=Sq)
        clipped = [torch.empty_like(t) for t in (dx, dk, dv, dg)]
        return [o, lse, P.clip_grad_norm([dx, dk, dv, dg], 0.5, out=clipped), *clipped]
    want = [chain(*s) for s in sets]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        captured = chain(*sets[0])
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    for s in (side, other):
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for t in captured:
            t.fill_(7.0)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            g.replay()
        with torch.cuda.stream(other):
            eager = [chain(*sets[1]) for _ in range(3)]
        torch.cuda.synchronize()
        for got, ref in [(captured, want[0])] + [(e, want[1]) for e in eager]:
            for x, y in zip(got, ref):
                assert torch.equal(x, y)
