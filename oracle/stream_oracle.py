"""Plain fp64 evaluation (numpy) of dropout and of the join of a block's output
with the residual stream.  Test infrastructure: written from the definitions, it
shares nothing with the HIP library."""
from __future__ import annotations

import numpy as np

M32 = np.uint64(0xFFFFFFFF)


def philox(counter, key, rounds=10):
    """Philox 4x32 (Salmon et al., 2011): counter 4 words (arrays of one shape), key 2; four arrays of words."""
    c = [np.asarray(v, np.uint64) for v in counter]
    k = [int(v) for v in key]
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & M32, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & M32]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def factors(T, D, p, seed, row0=0):
    """[T, D] factors of dropout: 0, or 65536 / kept."""
    key, stream = (int(v) % 2 ** 64 for v in seed)
    n = -(-D // 8)
    col, row = np.meshgrid(np.arange(n), row0 + np.arange(T))
    w = philox([col, row, np.full_like(col, stream % 2 ** 32), np.full_like(col, stream >> 32)], (key % 2 ** 32, key >> 32))
    bits = np.empty((T, n, 8), np.uint64)
    for i in range(4):
        bits[..., 2 * i], bits[..., 2 * i + 1] = w[i] & np.uint64(0xFFFF), w[i] >> np.uint64(16)
    kept = int(np.floor((1.0 - p) * 65536 + 0.5))
    return np.where(bits.reshape(T, 8 * n)[:, :D] < kept, 65536.0 / max(kept, 1), 0.0)


class Join:
    """h, n and the gradients of residual_norm, and the sizes that its rounding errors are proportional to."""

    def __init__(self, x, y, g_post=None, post=False, gate=None, gate_rows=None, g_pre=None, scale=1.0, f=1.0, eps=1e-6):
        T, D = y.shape
        self.x, self.y, self.post, self.eps = x, y, post, eps
        self.gp = np.ones(D) if g_post is None else g_post
        self.gn = np.ones(D) if g_pre is None else g_pre
        self.group = np.arange(T) // (gate_rows or max(T, 1))
        self.gate = gate
        self.gates = np.ones((T, D)) if gate is None else gate[self.group]
        self.sf = scale * f                                   # scale and dropout
        self.a = self.sf * self.gates
        self.r1 = 1 / np.sqrt((y * y).mean(1, keepdims=True) + eps) if post else np.ones((T, 1))
        self.u = y * self.r1 * self.gp if post else y
        self.h = x + self.a * self.u
        self.h_size = np.abs(x) + np.abs(self.a * self.u)
        self.r2 = 1 / np.sqrt((self.h ** 2).mean(1, keepdims=True) + eps)
        self.n = self.gn * self.h * self.r2
        self.n_size = np.abs(self.gn) * self.r2 * self.h_size

    def backward(self, dh, dn):
        """{name: (gradient, size)}"""
        m = lambda z: z.mean(1, keepdims=True)  # noqa: E731
        ab = np.abs
        dx, dx_size = (0.0, 0.0) if dh is None else (dh, ab(dh))
        out = {}
        if dn is not None:
            v = self.gn * dn
            dx = dx + self.r2 * (v - self.h * self.r2 ** 2 * m(self.h * v))
            dx_size = dx_size + self.r2 * (ab(v) + self.h_size * self.r2 ** 2 * m(self.h_size * ab(v)))
            out["dg_pre"] = ((dn * self.h * self.r2).sum(0), (ab(dn) * self.h_size * self.r2).sum(0))
        du, du_size = self.a * dx, ab(self.a) * dx_size
        if self.post:
            w, w_size = self.gp * du, ab(self.gp) * du_size
            dy = self.r1 * (w - self.y * self.r1 ** 2 * m(self.y * w))
            dy_size = self.r1 * (w_size + ab(self.y) * self.r1 ** 2 * m(ab(self.y) * w_size))
            out["dg_post"] = ((du * self.y * self.r1).sum(0), (du_size * ab(self.y) * self.r1).sum(0))
        else:
            dy, dy_size = du, du_size
        if self.gate is not None:
            t, t_size = self.sf * self.u * dx, ab(self.sf * self.u) * dx_size
            out["dgate"] = tuple(np.stack([z[self.group == g].sum(0) for g in range(len(self.gate))]) for z in (t, t_size))
        return {"dX": (dx, dx_size), "dY": (dy, dy_size), **out}
