"""Performance cases of the operators around attention and the training step:
rotary positions, per-head norms of queries and keys with the rotation,
cross attention (forward, training step, single tokens) and the clipping of
gradients by their global norm.

``own`` False computes them in plain form (elementary torch operations in 32
bits, angles and long sums in 64); ``own`` True calls the framework.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def _rotary(name, T, S, Hq, Hk, dh, rd, **k):
    return dict({"op": "rotary", "T": T, "S": S, "Hq": Hq, "Hk": Hk, "dh": dh, "rd": rd, "dtype": "bf16", "interleaved": False,
                 "scaled": False, "far": 0, "train": False}, **({"name": name} if name else {}), **k)


def _norm(name, T, S, Hq, Hk, dh, rd, **k):
    return dict(_rotary(name, T, S, Hq, Hk, dh, rd), **dict({"op": "qk_norm_rotary"}, **k))


def _cross(name, B, Sq, Sk, Hq, Hk, ragged, train):
    return dict({"op": "cross_attention", "B": B, "Sq": Sq, "Sk": Sk, "Hq": Hq, "Hk": Hk, "ragged": ragged, "train": train},
                **({"name": name} if name else {}))


def _clip(name, layers, D, F, dtype, bucket, clips):
    return dict({"op": "clip_grad_norm", "layers": layers, "D": D, "F": F, "dtype": dtype, "bucket": bucket, "clips": clips},
                **({"name": name} if name else {}))


def listed():
    return [
        # one new token of each of 16 requests far into long contexts, frequencies scaled by parts
        _rotary("rotary_decode", 16, 1, 32, 8, 128, 128, far=131072, scaled=True),
        # queries and keys of the two-layer decoder's tokens (4 x 2048, 40 heads), neighbouring pairs, and their gradients
        dict(_rotary("rotary_train", 8192, 2048, 40, 40, 128, 128), interleaved=True, train=True),
        # a short ragged batch of a model that turns a part of its heads only
        _rotary("rotary_part", 1021, 1021, 12, 2, 80, 20),
        # new tokens of 7 requests, shared key heads
        _norm("qk_norm_decode", 7, 1, 32, 8, 128, 128, far=32768),
        # training step of the attention block's queries and keys (4 x 2048 tokens, 32 heads)
        _norm("qk_norm_train", 8192, 2048, 32, 32, 128, 128, train=True),
        # float32 activations, heads of 96, an odd number of tokens
        _norm("qk_norm_f32", 4099, 4099, 16, 4, 96, 96, dtype="f32", interleaved=True),
        # one new token of each of 32 requests over encoder states of up to 1501 positions
        _cross("cross_decode", 32, 1, 1501, 32, 8, 0.9, False),
        # a single request over a long document's states
        _cross("cross_decode_long", 1, 1, 131072, 32, 8, 0.0, False),
        # training over long states with shared key heads, a padded batch
        _cross("cross_train", 4, 4096, 2048, 32, 8, 0.4, True),
        # many queries over a short prompt's states (77 positions), training
        _cross("cross_train_short", 2, 4096, 77, 8, 8, 0.3, True),
        # the gradients of a small model, as views of one flat bucket for each type
        _clip("clip_bucket", 32, 250, 1001, "mixed", True, True),
        # the fp32 gradients of the two-layer decoder (D 5120, F 13824)
        _clip("clip_decoder", 2, 5120, 13824, "f32", False, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("rotary", "qk_norm_rotary", "cross_attention", "cross_attention", "clip_grad_norm"))
    if op in ("rotary", "qk_norm_rotary"):
        Hk = rng.choice((1, 2, 3, 4, 8, 12, 16))
        Hq = Hk * rng.choice((1, 1, 2, 4))
        dh = rng.choice((64, 80, 96, 128, 256))
        rd = rng.choice((dh, dh, dh // 2, 2 * rng.randint(4, dh // 2)))
        T = _log(rng, 1, 8192 * 80 * 128 // ((Hq + Hk) * dh) if (Hq + Hk) * dh > 10240 else 8192)
        S = rng.choice((T, max(1, T // 3)))
        return dict(_rotary(None, T, S, Hq, Hk, dh, rd), op=op, dtype=rng.choice(("bf16", "bf16", "f32")),
                    interleaved=rng.random() < 0.4, scaled=rng.random() < 0.4, far=rng.choice((0, 4096, 131072, 1000003)),
                    train=rng.random() < 0.5)
    if op == "cross_attention":
        Hk = rng.choice((1, 2, 4, 5, 8, 16))
        Hq = Hk * rng.choice((1, 2, 4, 8))
        if rng.random() < 0.4:   # new tokens
            B = _log(rng, 1, 64)
            return _cross(None, B, rng.choice((1, 1, 1, 2, 5)), _log(rng, 1, max(1, min(131072, 1000000 // (B * Hk)))), Hq, Hk,
                          rng.choice((0.0, 0.5, 1.0)), False)
        B = rng.randint(1, 4)
        Sq, Sk = _log(rng, 1, 4096), _log(rng, 1, 4096)
        while B * Hq * Sq * Sk > 800_000_000:
            Sq = max(1, Sq // 2)
        return _cross(None, B, Sq, Sk, Hq, Hk, rng.choice((0.0, 0.5, 1.0)), rng.random() < 0.6)
    D, bucket = 2 * _log(rng, 16, 1024), rng.random() < 0.5
    F, most = _log(rng, 17, 4 * D), 480_000_000
    layers = min(rng.randint(1, 24 if bucket else 7), max(1, most // (4 * D * D + 2 * D * F + 2 * D)))
    return _clip(None, layers, D, F, rng.choice(("f32", "bf16", "mixed")), bucket, rng.random() < 0.7)


def _lengths(c):
    """Valid encoder positions of each sequence of the batch."""
    B = c["B"]
    return [c["Sk"] - int(c["ragged"] * c["Sk"] * ((7 * b) % B) / max(1, B - 1)) for b in range(B)]


def _grad_shapes(c):
    """A decoder's gradients: four projections, the MLP's two weights, two norms' gains, a layer each."""
    D, F = c["D"], c["F"]
    return [s for _ in range(c["layers"]) for s in ((D, D), (D, D), (D, D), (D, D), (D, F), (F, D), (D,), (D,))]


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.bfloat16, scale=1.0):
        return torch.randn(*shape, generator=g, device="cuda").mul_(scale).to(dtype)

    if c["op"] in ("rotary", "qk_norm_rotary"):
        T, Hq, Hk, dh, rd = c["T"], c["Hq"], c["Hk"], c["dh"], c["rd"]
        dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        qkv = normal(T, (Hq + 2 * Hk) * dh, dtype=dt)   # the fused projection that queries and keys are columns of
        s = {"c": c, "qkv": qkv, "Q": qkv[:, :Hq * dh], "K": qkv[:, Hq * dh:(Hq + Hk) * dh], "positions": None, "magnitude": 1.0}
        if c["far"]:
            s["positions"] = torch.randint(0, c["far"], (T,), generator=g, device="cuda")
        i = np.arange(rd // 2, dtype=np.float64)
        f = 10000.0 ** (-2.0 * i / rd)
        if c["scaled"]:   # by parts: slow pairs divided by 8, fast ones kept, a ramp between (in turns over 4096 positions)
            turns = 4096 * f / (2 * math.pi)
            keep = np.clip((turns - 1.0) / (32.0 - 1.0), 0.0, 1.0)
            f = f * keep + f / 8.0 * (1.0 - keep)
            s["magnitude"] = 0.1 * math.log(8.0) + 1.0
        s["freqs"] = torch.from_numpy(f).to("cuda")
        if c["op"] == "qk_norm_rotary":
            s["gq"] = 1.0 + 0.1 * normal(dh, dtype=torch.float32)
            s["gk"] = 1.0 + 0.1 * normal(dh, dtype=torch.float32)
        if c["train"]:
            s["dQ"], s["dK"] = normal(T, Hq * dh, dtype=dt), normal(T, Hk * dh, dtype=dt)
        return s
    if c["op"] == "cross_attention":
        B, Sq, Sk, Hq, Hk = c["B"], c["Sq"], c["Sk"], c["Hq"], c["Hk"]
        kv = normal(B * Sk, 2 * Hk * 128)                # the fused projection of the encoder's states
        s = {"c": c, "Q": normal(B * Sq, Hq * 128, scale=1.5), "kv": kv, "K": kv[:, :Hk * 128], "V": kv[:, Hk * 128:],
             "lens": torch.tensor(_lengths(c), dtype=torch.int32, device="cuda") if c["ragged"] else None}
        if c["train"]:
            s["dO"] = normal(B * Sq, Hq * 128)
        return s
    shapes = _grad_shapes(c)
    kinds = [torch.bfloat16 if c["dtype"] == "bf16" or (c["dtype"] == "mixed" and len(sh) == 2 and i % 8 < 4) else torch.float32
             for i, sh in enumerate(shapes)]
    if c["bucket"]:
        numel = {k: sum(math.prod(sh) for sh, kk in zip(shapes, kinds) if kk is k) for k in set(kinds)}
        flat = {k: normal(n, dtype=k, scale=0.02) for k, n in sorted(numel.items(), key=lambda x: str(x[0]))}
        outs = {k: torch.empty_like(v) for k, v in flat.items()}
        at, grads, out = dict.fromkeys(flat, 0), [], []
        for sh, k in zip(shapes, kinds):
            n = math.prod(sh)
            grads.append(flat[k][at[k]:at[k] + n].view(sh))
            out.append(outs[k][at[k]:at[k] + n].view(sh))
            at[k] += n
        whole = [outs[k] for k in sorted(outs, key=str)]
    else:
        grads = [normal(*sh, dtype=k, scale=0.02) for sh, k in zip(shapes, kinds)]
        out = whole = [torch.empty_like(t) for t in grads]
    norm = 0.02 * math.sqrt(sum(math.prod(sh) for sh in shapes))
    return {"c": c, "grads": grads, "out": out, "whole": whole, "max_norm": norm * (0.37 if c["clips"] else 2.0)}


# ---------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------
def _angles(s):
    c = s["c"]
    T = c["T"]
    pos = s["positions"] if s["positions"] is not None else torch.arange(T, device="cuda") % c["S"]
    a = pos.double()[:, None] * s["freqs"]
    return (torch.cos(a) * s["magnitude"]).float()[:, None], (torch.sin(a) * s["magnitude"]).float()[:, None]


def _turn(x, cos, sin, c):
    """x [T, H, dh] float32 with its first rd values of each head turned."""
    rd = c["rd"]
    y = x.clone()
    if c["interleaved"]:
        a, b = x[..., 0:rd:2], x[..., 1:rd:2]
        y[..., 0:rd:2], y[..., 1:rd:2] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = x[..., :rd // 2], x[..., rd // 2:rd]
        y[..., :rd // 2], y[..., rd // 2:rd] = a * cos - b * sin, a * sin + b * cos
    return y


def _plain_rotary(s):
    c = s["c"]
    cos, sin = _angles(s)
    heads = lambda x: x.float().reshape(c["T"], -1, c["dh"])  # noqa: E731
    flat = lambda x: x.reshape(c["T"], -1).to(s["Q"].dtype)  # noqa: E731
    out = [flat(_turn(heads(s["Q"]), cos, sin, c)), flat(_turn(heads(s["K"]), cos, sin, c))]
    if c["train"]:
        out += [flat(_turn(heads(s["dQ"]), cos, -sin, c)), flat(_turn(heads(s["dK"]), cos, -sin, c))]
    return out


_EPS = 1e-6


def _plain_norm(s):
    c = s["c"]
    cos, sin = _angles(s)
    dt = s["Q"].dtype

    def forward(x, g):
        x = x.float().reshape(c["T"], -1, c["dh"])
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPS)
        return _turn(x * r * g, cos, sin, c).reshape(c["T"], -1).to(dt)

    def backward(x, g, dy):
        x, dy = (v.float().reshape(c["T"], -1, c["dh"]) for v in (x, dy))
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPS)
        dn = _turn(dy, cos, -sin, c)
        u = g * dn
        dx = r * (u - x * (r * r * (x * u).mean(-1, keepdim=True)))
        return dx.reshape(c["T"], -1).to(dt), (dn * x * r).sum((0, 1))

    out = [forward(s["Q"], s["gq"]), forward(s["K"], s["gk"])]
    if c["train"]:
        dq, dgq = backward(s["Q"], s["gq"], s["dQ"])
        dk, dgk = backward(s["K"], s["gk"], s["dK"])
        out += [dq, dk, dgq, dgk]
    return out


def _split(s, x, S, H):
    """[B S, H 128] as [B, Hk, (H / Hk) S, 128] float32: the query heads of a key head are rows beside each other."""
    c = s["c"]
    x = x.float().reshape(c["B"], S, c["Hk"], H // c["Hk"], 128)
    return x.permute(0, 2, 3, 1, 4).reshape(c["B"], c["Hk"], -1, 128)


def _join(s, x, S, H):
    c = s["c"]
    x = x.reshape(c["B"], c["Hk"], H // c["Hk"], S, 128).permute(0, 3, 1, 2, 4)
    return x.reshape(c["B"] * S, H * 128).to(torch.bfloat16)


def _plain_cross(s):
    c = s["c"]
    B, Sq, Sk, Hq, Hk = c["B"], c["Sq"], c["Sk"], c["Hq"], c["Hk"]
    scale = 128 ** -0.5
    q, k, v = _split(s, s["Q"], Sq, Hq), _split(s, s["K"], Sk, Hk), _split(s, s["V"], Sk, Hk)
    x = torch.matmul(q, k.transpose(-1, -2)) * scale
    if s["lens"] is not None:
        seen = (torch.arange(Sk, device="cuda") < s["lens"][:, None])[:, None, None]
        x = torch.where(seen, x, -math.inf)
    m = x.amax(-1, keepdim=True).clamp_min(-3.0e38)     # a sequence without keys has none
    p = torch.exp(x - m)
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    o = torch.matmul(p, v)
    if not c["train"]:
        return _join(s, o, Sq, Hq)
    lse = ((m + torch.log(total)) * math.log2(math.e)).reshape(B, Hk, Hq // Hk, Sq).permute(0, 3, 1, 2).reshape(B * Sq, Hq)
    do = _split(s, s["dO"], Sq, Hq)
    dv = torch.matmul(p.transpose(-1, -2), do)
    ds = p * (torch.matmul(do, v.transpose(-1, -2)) - (do * o).sum(-1, keepdim=True))
    dq = torch.matmul(ds, k) * scale
    dk = torch.matmul(ds.transpose(-1, -2), q) * scale
    return [_join(s, o, Sq, Hq), lse, _join(s, dq, Sq, Hq), _join(s, dk, Sk, Hk), _join(s, dv, Sk, Hk)]


def _plain_clip(s):
    norm = torch.stack([t.float().square().sum(dtype=torch.float64) for t in s["grads"]]).sum().sqrt()
    factor = torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0).float()
    for t, o in zip(s["grads"], s["out"]):
        o.copy_(t * factor if t.dtype == torch.float32 else t.float() * factor)
    return [norm.float(), *s["whole"]]


# ---------------------------------------------------------------------------
# The framework's calls
# ---------------------------------------------------------------------------
def _own(s):
    from paper_2401_11202_amd import partir
    c = s["c"]
    if c["op"] in ("rotary", "qk_norm_rotary"):
        k = dict(d_head=c["dh"], positions=s["positions"], S=c["S"], interleaved=c["interleaved"], magnitude=s["magnitude"])
        if c["op"] == "rotary":
            out = partir.rotary(s["Q"], s["K"], s["freqs"], **k)
            return [*out, *partir.rotary(s["dQ"], s["dK"], s["freqs"], inverse=True, **k)] if c["train"] else list(out)
        out = partir.qk_norm_rotary(s["Q"], s["K"], s["gq"], s["gk"], s["freqs"], eps=_EPS, **k)
        if not c["train"]:
            return list(out)
        return [*out, *partir.qk_norm_rotary_backward(s["Q"], s["K"], s["dQ"], s["dK"], s["gq"], s["gk"], s["freqs"], eps=_EPS, **k)]
    if c["op"] == "cross_attention":
        k = dict(B=c["B"], Sq=c["Sq"], Sk=c["Sk"], n_heads=c["Hq"], n_kv_heads=c["Hk"], k_lens=s["lens"])
        if not c["train"]:
            return partir.cross_attention(s["Q"], s["K"], s["V"], **k)
        o, lse = partir.cross_attention_train(s["Q"], s["K"], s["V"], **k)
        return [o, lse, *partir.cross_attention_backward(s["Q"], s["K"], s["V"], o, s["dO"], lse, **k)]
    norm = partir.clip_grad_norm(s["grads"], s["max_norm"], out=s["out"])
    return [norm, *s["whole"]]


def run(state):
    if own:
        return _own(state)
    op = state["c"]["op"]
    if op == "rotary":
        return _plain_rotary(state)
    if op == "qk_norm_rotary":
        return _plain_norm(state)
    return _plain_cross(state) if op == "cross_attention" else _plain_clip(state)


# ---------------------------------------------------------------------------
# Work, and the definitions in 64 bits
# ---------------------------------------------------------------------------
def work(case):
    c = case
    if c["op"] in ("rotary", "qk_norm_rotary"):
        values = c["T"] * (c["Hq"] + c["Hk"]) * c["dh"]
        es = 4 if c["dtype"] == "f32" else 2
        turned = 3.0 * c["T"] * (c["Hq"] + c["Hk"]) * c["rd"]
        normed = 0.0 if c["op"] == "rotary" else 4.0 * values
        flops = turned + normed + (turned + 2.5 * normed if c["train"] else 0.0)
        return {"bytes": float(values * es * (4 if c["train"] else 2) + (8 * c["T"] if c["far"] else 0) + 4 * c["rd"]), "flops": flops}
    if c["op"] == "cross_attention":
        keys = sum(_lengths(c))
        q, kv = c["B"] * c["Sq"] * c["Hq"] * 256, keys * c["Hk"] * 256
        pairs = 128.0 * c["Hq"] * c["Sq"] * keys
        if c["train"]:   # in: Q, dO, K, V; out: O, lse, dQ, dK, dV (gradients of the padding are written too)
            return {"bytes": float(4 * q + q // 64 + 2 * kv + 2 * c["B"] * c["Sk"] * c["Hk"] * 256), "flops": 14.0 * pairs}
        return {"bytes": float(2 * q + 2 * kv), "flops": 4.0 * pairs}
    n = values = 0
    for i, sh in enumerate(_grad_shapes(c)):
        m = math.prod(sh)
        n += m * (2 if c["dtype"] == "bf16" or (c["dtype"] == "mixed" and len(sh) == 2 and i % 8 < 4) else 4)
        values += m
    return {"bytes": 2.0 * n, "flops": 3.0 * values}


def _turn64(x, s):
    """The first rd values of each head as complex numbers, times magnitude e^(i theta)."""
    c = s["c"]
    T, rd = c["T"], c["rd"]
    pos = (torch.arange(T, device="cuda") % c["S"] if s["positions"] is None else s["positions"]).double()
    w = torch.polar(torch.full((T, rd // 2), float(s["magnitude"]), dtype=torch.float64, device="cuda"), torch.outer(pos, s["freqs"]))[:, None]
    head = x[..., :rd]
    if c["interleaved"]:
        z = torch.complex(head[..., 0::2], head[..., 1::2]) * w
        head = torch.stack((z.real, z.imag), -1).flatten(-2)
    else:
        lo, hi = head.chunk(2, -1)
        z = torch.complex(lo, hi) * w
        head = torch.cat((z.real, z.imag), -1)
    return torch.cat((head, x[..., rd:]), -1)


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] in ("rotary", "qk_norm_rotary"):
        q = s["Q"].double().requires_grad_(c["train"])
        k = s["K"].double().requires_grad_(c["train"])
        gains = [] if c["op"] == "rotary" else [s["gq"].double().requires_grad_(c["train"]), s["gk"].double().requires_grad_(c["train"])]
        out = []
        for i, x in enumerate((q, k)):
            x = x.reshape(c["T"], -1, c["dh"])
            if gains:
                x = gains[i] * x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["dh"] + _EPS)
            out.append(_turn64(x, s).reshape(c["T"], -1))
        if c["train"]:
            out += torch.autograd.grad(out, [q, k, *gains], [s["dQ"].double(), s["dK"].double()])
        return [x.detach() for x in out]
    if c["op"] == "cross_attention":
        B, Sq, Sk, Hq, Hk = c["B"], c["Sq"], c["Sk"], c["Hq"], c["Hk"]
        leaf = [s[n].double().requires_grad_(c["train"]) for n in ("Q", "K", "V")]
        outs, lses = [], []
        for b, n in enumerate(_lengths(c) if s["lens"] is not None else [Sk] * B):
            q = leaf[0][b * Sq:(b + 1) * Sq].reshape(Sq, Hk, Hq // Hk, 128)
            k, v = (x[b * Sk:b * Sk + n].reshape(n, Hk, 128) for x in leaf[1:])
            x = torch.einsum("qhgd,khd->hgqk", q, k) / math.sqrt(128.0)
            lses.append((torch.logsumexp(x, -1) / math.log(2.0)).permute(2, 0, 1).reshape(Sq, Hq))
            w = torch.exp(x - torch.logsumexp(x, -1, keepdim=True))
            outs.append(torch.einsum("hgqk,khd->qhgd", w, v).reshape(Sq, Hq * 128))
        o = torch.cat(outs)
        if not c["train"]:
            return o
        grads = torch.autograd.grad(o, leaf, s["dO"].double(), allow_unused=True)
        return [o.detach(), torch.cat(lses).detach(), *(torch.zeros_like(x) if d is None else d for d, x in zip(grads, leaf))]
    total = math.sqrt(math.fsum(float(torch.linalg.vector_norm(t.double())) ** 2 for t in s["grads"]))
    factor = s["max_norm"] / total if total > s["max_norm"] else 1.0
    for t, o in zip(s["grads"], s["out"]):
        o.copy_(t)
    whole = [w.double() * factor for w in s["whole"]]
    return [torch.tensor(total, dtype=torch.float64), *whole]
