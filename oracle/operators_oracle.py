"""Plain fp64 evaluation (numpy) of the operators beside the loop nests:
rotary positions, per-head norms with the rotation, cross attention, the
global norm of gradients.  Test infrastructure: written from the definitions,
it shares nothing with the HIP library."""
from __future__ import annotations

import numpy as np


def frequencies(rd, base=10000.0, scaling=None, factor=1.0, original_length=0, slow=1.0, fast=32.0):
    """Radians per position of each pair."""
    i = np.arange(rd // 2)
    if scaling == "base":
        base = base * factor ** (rd / (rd - 2))
    f = np.power(float(base), -2.0 * i / rd) if rd else np.zeros(0)
    if scaling == "linear":
        f = f / factor
    if scaling == "parts":
        turns = original_length * f / (2 * np.pi)
        keep = np.clip((turns - slow) / (fast - slow), 0.0, 1.0)
        f = keep * f + (1 - keep) * f / factor
    return f


def rotary(x, pos, freqs, dh, interleaved=False, magnitude=1.0, inverse=False):
    """x [T, H dh] with the first 2 len(freqs) values of each head turned."""
    T = x.shape[0]
    rd = 2 * len(freqs)
    y = np.array(x, np.float64).reshape(T, -1, dh)
    # the angle modulo a turn in extended precision, so that far positions keep all of it
    a = np.asarray(pos, np.longdouble)[:, None] * np.asarray(freqs, np.longdouble)
    two_pi = 2 * np.arctan2(np.longdouble(0), np.longdouble(-1))
    a = np.asarray(a - two_pi * np.rint(a / two_pi), np.float64)[:, None, :]
    c, s = magnitude * np.cos(a), magnitude * np.sin(a) * (-1.0 if inverse else 1.0)
    p, q = (slice(0, rd, 2), slice(1, rd, 2)) if interleaved else (slice(0, rd // 2), slice(rd // 2, rd))
    u, v = y[..., p].copy(), y[..., q].copy()
    y[..., p], y[..., q] = u * c - v * s, u * s + v * c
    return y.reshape(T, -1)


def pair_size(x, nf, dh, interleaved=False):
    """|a| + |b| at both places of a pair, |x| elsewhere: what a rotation's
    rounding errors are proportional to."""
    rd = 2 * nf
    y = np.abs(np.asarray(x, np.float64)).reshape(x.shape[0], -1, dh).copy()
    p, q = (slice(0, rd, 2), slice(1, rd, 2)) if interleaved else (slice(0, rd // 2), slice(rd // 2, rd))
    t = y[..., p] + y[..., q]
    y[..., p], y[..., q] = t, t
    return y.reshape(x.shape[0], -1)


def head_norm(x, g, dh, eps):
    """(g x r [T, H dh], r [T, H, 1]) with r = 1 / sqrt(mean(x^2) + eps) per head."""
    h = np.asarray(x, np.float64).reshape(x.shape[0], -1, dh)
    r = 1.0 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    return (h * r * (1.0 if g is None else g)).reshape(x.shape[0], -1), r


def qk_norm_rotary(x, g, pos, freqs, dh, eps, **kw):
    return rotary(head_norm(x, g, dh, eps)[0], pos, freqs, dh, **kw)


def qk_norm_rotary_backward(x, g, dy, pos, freqs, dh, eps, **kw):
    """(dx, dg) of qk_norm_rotary for the cotangent dy."""
    T = x.shape[0]
    dn = rotary(dy, pos, freqs, dh, inverse=True, **kw).reshape(T, -1, dh)
    h = np.asarray(x, np.float64).reshape(T, -1, dh)
    r = head_norm(x, g, dh, eps)[1]
    u = dn * (1.0 if g is None else g)
    dx = r * u - h * r ** 3 * (h * u).mean(-1, keepdims=True)
    return dx.reshape(T, -1), (dn * h * r).sum((0, 1))


def cross_attention(Q, K, V, B, Sq, Sk, Hq, Hk, lens=None, scale=None, dh=128):
    """(O [B Sq, Hq dh], base-2 lse [B Sq, Hq]); a sequence without keys gives 0 and -inf."""
    scale = dh ** -0.5 if scale is None else scale
    O, lse = np.zeros((B * Sq, Hq * dh)), np.full((B * Sq, Hq), -np.inf)
    for b in range(B):
        n = Sk if lens is None else int(lens[b])
        if n == 0 or Sq == 0:
            continue
        for h in range(Hq):
            kh = h // (Hq // Hk)
            q = Q[b * Sq:(b + 1) * Sq, h * dh:(h + 1) * dh]
            k, v = (x[b * Sk:b * Sk + n, kh * dh:(kh + 1) * dh] for x in (K, V))
            s = scale * (q @ k.T)
            m = s.max(1, keepdims=True)
            p = np.exp(s - m)
            t = p.sum(1, keepdims=True)
            O[b * Sq:(b + 1) * Sq, h * dh:(h + 1) * dh] = (p / t) @ v
            lse[b * Sq:(b + 1) * Sq, h] = ((m + np.log(t)) / np.log(2.0))[:, 0]
    return O, lse


def cross_attention_backward(Q, K, V, dO, B, Sq, Sk, Hq, Hk, lens=None, scale=None, dh=128):
    """(dQ, dK, dV); positions behind a sequence's length get zeros."""
    scale = dh ** -0.5 if scale is None else scale
    dQ, dK, dV = np.zeros((B * Sq, Hq * dh)), np.zeros((B * Sk, Hk * dh)), np.zeros((B * Sk, Hk * dh))
    for b in range(B):
        n = Sk if lens is None else int(lens[b])
        if n == 0 or Sq == 0:
            continue
        for h in range(Hq):
            kh = h // (Hq // Hk)
            rq, rk = slice(b * Sq, (b + 1) * Sq), slice(b * Sk, b * Sk + n)
            cq, ck = slice(h * dh, (h + 1) * dh), slice(kh * dh, (kh + 1) * dh)
            q, k, v, g = Q[rq, cq], K[rk, ck], V[rk, ck], dO[rq, cq]
            s = scale * (q @ k.T)
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            dp = g @ v.T
            ds = p * (dp - (p * dp).sum(1, keepdims=True))
            dQ[rq, cq] = scale * (ds @ k)
            dK[rk, ck] += scale * (ds.T @ q)
            dV[rk, ck] += p.T @ g
    return dQ, dK, dV


def clip(tensors, max_norm):
    """(norm, scaled tensors)"""
    n = float(np.sqrt(sum(float((np.asarray(t, np.float64) ** 2).sum()) for t in tensors)))
    f = max_norm / n if max_norm is not None and n > max_norm else 1.0
    return n, [np.asarray(t, np.float64) * f for t in tensors]
