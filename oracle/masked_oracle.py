"""Plain fp64 evaluation (numpy) of masked attention and its gradients.  Test
infrastructure: written from the definitions, it shares nothing with the HIP
library."""
from __future__ import annotations

import numpy as np


def visible(b, Sq, Sk, causal=True, k_lens=None, q_lens=None, q_starts=None, prefix_lens=None, q_docs=None, k_docs=None, **_):
    """[Sq, Sk]: which keys the queries of sequence b see; and the queries' positions."""
    start = Sk - Sq if q_starts is None else int(q_starts[b])
    kn = Sk if k_lens is None else min(max(int(k_lens[b]), 0), Sk)
    qn = Sq if q_lens is None else min(max(int(q_lens[b]), 0), Sq)
    pre = 0 if prefix_lens is None else int(prefix_lens[b])
    see = np.zeros((Sq, Sk), bool)
    for i in range(qn):
        for_all = np.arange(kn)
        if causal:
            for_all = for_all[(for_all <= start + i) | (for_all < pre)]
        if q_docs is not None:
            for_all = for_all[np.asarray(k_docs[b * Sk:(b + 1) * Sk])[for_all] == q_docs[b * Sq + i]]
        see[i, for_all] = True
    return see, start + np.arange(Sq)


def attention(Q, K, V, B, Sq, Sk, Hq, Hk, scale=None, cap=0.0, slopes=None, dh=128, dO=None, **mask):
    """(O, base-2 lse), and with dO also dQ, dK, dV."""
    scale = dh ** -0.5 if scale is None else scale
    O, lse = np.zeros((B * Sq, Hq * dh)), np.full((B * Sq, Hq), -np.inf)
    dQ, dK, dV = np.zeros_like(O), np.zeros((B * Sk, Hk * dh)), np.zeros((B * Sk, Hk * dh))
    for b in range(B):
        see, pos = visible(b, Sq, Sk, **mask)
        rows, keys = np.flatnonzero(see.any(1)), np.flatnonzero(see.any(0))
        if not len(rows):
            continue
        see = see[np.ix_(rows, keys)]
        for h in range(Hq):
            kh = h // (Hq // Hk)
            cq, ck = slice(h * dh, (h + 1) * dh), slice(kh * dh, (kh + 1) * dh)
            q, k, v = Q[b * Sq + rows][:, cq], K[b * Sk + keys][:, ck], V[b * Sk + keys][:, ck]
            x = scale * (q @ k.T)
            d = np.ones_like(x)
            if cap:
                t = np.tanh(x / cap)
                x, d = cap * t, 1 - t * t
            if slopes is not None:
                x = x - slopes[h] * np.abs(pos[rows][:, None] - keys[None])
            x = np.where(see, x, -np.inf)
            m = x.max(1, keepdims=True)
            p = np.exp(x - m)
            t = p.sum(1, keepdims=True)
            p /= t
            O[b * Sq + rows, cq] = p @ v
            lse[b * Sq + rows, h] = ((m + np.log(t)) / np.log(2.0))[:, 0]
            if dO is None:
                continue
            g = dO[b * Sq + rows][:, cq]
            dp = g @ v.T
            ds = p * (dp - (p * dp).sum(1, keepdims=True)) * d
            dQ[b * Sq + rows, cq] = scale * (ds @ k)
            dK[b * Sk + keys, ck] += scale * (ds.T @ q)
            dV[b * Sk + keys, ck] += p.T @ g
    return (O, lse) if dO is None else (O, lse, dQ, dK, dV)


def bounds(Q, K, V, dO, O, B, Sq, Sk, Hq, Hk, scale=None, cap=0.0, slopes=None, dh=128, u=2.0 ** -8, **mask):
    """Elementwise bounds of |error| of O, lse, dQ, dK, dV without their own rounding, when weights and dS are rounded by u."""
    scale = dh ** -0.5 if scale is None else scale
    out = [np.zeros((B * Sq, Hq * dh)), np.zeros((B * Sq, Hq)), np.zeros((B * Sq, Hq * dh)), np.zeros((B * Sk, Hk * dh)),
           np.zeros((B * Sk, Hk * dh))]
    for b in range(B):
        see, pos = visible(b, Sq, Sk, **mask)
        rows, keys = np.flatnonzero(see.any(1)), np.flatnonzero(see.any(0))
        if not len(rows):
            continue
        see = see[np.ix_(rows, keys)]
        for h in range(Hq):
            kh = h // (Hq // Hk)
            cq, ck = slice(h * dh, (h + 1) * dh), slice(kh * dh, (kh + 1) * dh)
            q, k, v, g = Q[b * Sq + rows][:, cq], K[b * Sk + keys][:, ck], V[b * Sk + keys][:, ck], dO[b * Sq + rows][:, cq]
            x = scale * (q @ k.T)
            e = 2.0 ** -14 + 2.0 ** -16 * scale * float((np.abs(q) @ np.abs(k).T).max()) + 2.0 ** -20 * cap
            d = np.ones_like(x)
            if cap:
                t = np.tanh(x / cap)
                x, d = cap * t, 1 - t * t
            if slopes is not None:
                far = abs(slopes[h]) * np.abs(pos[rows][:, None] - keys[None])
                x = x - slopes[h] * np.abs(pos[rows][:, None] - keys[None])
                e += 2.0 ** -22 * float(far.max())
            x = np.where(see, x, -np.inf)
            p = np.exp(x - x.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            p += 2.0 ** -125 / u      # float32 weights, and bf16 ones, below 2^-126 are 0: off by up to that, here times u
            A = p @ np.abs(v)
            out[0][b * Sq + rows, cq] = (u + e) * A
            out[1][b * Sq + rows, h] = 2 * e
            dD = ((2 * u + e) * np.abs(g) * A).sum(1, keepdims=True)
            D = np.abs((g * O[b * Sq + rows][:, cq]).sum(1, keepdims=True))
            size = np.abs(g @ v.T) + D
            ds = p * (d * (size * (u + 2 * e) + dD) + (2.0 ** -19 * size if cap else 0.0))
            out[2][b * Sq + rows, cq] = scale * (ds @ np.abs(k))
            out[3][b * Sk + keys, ck] += scale * (ds.T @ np.abs(q))
            out[4][b * Sk + keys, ck] += (u + e) * (p.T @ np.abs(g))
    return out
