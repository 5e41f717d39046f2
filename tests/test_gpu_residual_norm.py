"""GPU parity of dropout and of the join with the residual stream against the
fp64 oracle.

Tolerances.  An output is rounded once to its type (half a step, eps / 2 of its
value).  Before that everything is float32: a mean of D <= 16384 squares is a sum of
at most 16 terms a lane, 6 steps over the lanes and 16 over the waves, below 40
additions deep: with the root and the division 2^-18 relative.  H has that once, of
|x| + |a u|; N has H's error and its own norm's, 2^-16 of g r2 (|x| + |a u|); dX
sums terms that hold both, 2^-15 of their sizes, dY as many again, 2^-14.  The sums
over rows add to that at most 300 additions in a row (rows of a worker, parts of a
run), 2^-15: 2^-13 of the sum of their terms' sizes.  Masks are equal."""
import numpy as np
import pytest
import torch

from oracle import stream_oracle as SO
from paper_2401_11202_amd import inputs as I
from paper_2401_11202_amd import partir as P
from tests.gpu_common import host, say

pytestmark = pytest.mark.gpu
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
SLACK = {"H": 2.0 ** -18, "N": 2.0 ** -16, "dX": 2.0 ** -15, "dY": 2.0 ** -14, "dg_post": 2.0 ** -13, "dgate": 2.0 ** -13,
         "dg_pre": 2.0 ** -13}


def close(got, ref, size, what):
    assert got.shape == ref.shape, what
    err = np.abs(host(got) - ref) - HALF[got.dtype] * np.abs(ref) - SLACK[what] * size
    worst = float(err.max()) if err.size else 0.0
    say(f"    {what}: largest error past its bound {worst:.2e}")
    assert worst <= 0.0, what


def seed_of(key, stream):
    return torch.tensor([key, stream], dtype=torch.int64, device="cuda")


def padded(wid, idx, T, D, dtype, scale=1.0):
    """A [T, D] view whose rows are 8 values longer, and its values."""
    t = I.gaussian(wid, idx, (T, D + 8), scale, dtype)
    return t.to_device()[:, :D], t.f64()[:, :D]


# ---------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------
DROP = [(1, 1), (1, 8), (3, 7), (5, 9), (2, 1000), (1023, 13), (77, 512), (130, 1001), (3, 20000), (5000, 24)]


@pytest.mark.parametrize("T,D", DROP)
@pytest.mark.parametrize("x,y", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("residual", [False, True])
def test_dropout(T, D, x, y, residual):
    say(f"dropout T={T} D={D} {x} -> {y} residual={residual}")
    ld = (D + 7) // 8 * 8 + 8
    xs, rs = I.gaussian(400, T, (T, ld), 1.0, x), I.gaussian(401, T, (T, ld), 1.0, y)
    X, R = xs.to_device()[:, :D], rs.to_device()[:, :D]
    seed, p, row0 = (2 ** 62 + 12345, 2 ** 35 + 7), 0.3, 2 ** 32 - T
    f = SO.factors(T, D, p, seed, row0)
    room = torch.full((T, ld), 7.0, dtype=R.dtype, device="cuda")
    got = P.dropout(X, p, seed_of(*seed), residual=R if residual else None, row0=row0, out=room[:, :D])
    ref = f * xs.f64()[:, :D] + (rs.f64()[:, :D] if residual else 0.0)
    # a product, and a sum in float32, each a half step of itself, then the output's rounding
    err = np.abs(host(got) - ref) - HALF[got.dtype] * np.abs(ref) - 2.0 ** -22 * (np.abs(f * xs.f64()[:, :D]) + np.abs(ref))
    assert err.max() <= 0
    assert ((host(got) == 0) >= (f == 0)).all() if not residual else True
    assert bool((room[:, D:] == 7).all())


def test_dropout_shares_and_ends():
    X = torch.randn(300, 800, device="cuda")
    s = seed_of(3, 4)
    assert torch.equal(P.dropout(X, 0.0, s), X)
    assert not P.dropout(X, 1.0, s).any()
    got = P.dropout(X, 0.25, s)
    assert torch.equal(P.dropout(X, 0.25, s), got)
    assert abs(float((got == 0).float().mean()) - 0.25) < 5 * (0.25 * 0.75 / X.numel()) ** 0.5
    assert not torch.equal(P.dropout(X, 0.25, seed_of(3, 5)), got)
    assert P.dropout(X[:0], 0.25, s).shape == (0, 800)


def test_dropout_of_parts_is_that_of_the_whole():
    X = torch.randn(301, 136, device="cuda").to(torch.bfloat16)
    s = seed_of(9, 9)
    whole = P.dropout(X, 0.4, s, row0=5)
    parts = torch.cat([P.dropout(X[a:b], 0.4, s, row0=5 + a) for a, b in ((0, 100), (100, 101), (101, 301))])
    assert torch.equal(whole, parts) and torch.equal(P.dropout(X[:, :72], 0.4, s, row0=5), whole[:, :72])


def test_dropout_in_place_and_of_values_that_are_not_finite():
    X = torch.randn(65, 520, device="cuda")
    R = torch.randn(65, 520, device="cuda")
    s = seed_of(1, 2)
    want, sums = P.dropout(X, 0.5, s), P.dropout(X, 0.5, s, residual=R)
    bad = torch.where(want == 0, torch.tensor(float("nan"), device="cuda"), X)   # what is dropped may hold anything
    assert torch.equal(P.dropout(bad, 0.5, s), want)
    Y = X.clone()
    assert P.dropout(Y, 0.5, s, out=Y) is Y and torch.equal(Y, want)
    Y = R.clone()
    assert torch.equal(P.dropout(X, 0.5, s, residual=Y, out=Y), sums)


# ---------------------------------------------------------------------------
# join
# ---------------------------------------------------------------------------
SHAPES = [(1, 8), (3, 8), (9, 64), (5, 512), (7, 520), (33, 1000), (130, 1024), (64, 4096), (17, 5120), (5, 8192), (4, 8200),
          (2, 16384), (2051, 256), (1300, 2056)]
FORMS = [  # stream, block, post, gate rows (0: no gate, -1: one row for all), next, p, scale, gains
    ("f32", "bf16", False, 0, True, 0.0, 1.0, True), ("f32", "bf16", True, 3, True, 0.2, 0.5, True),
    ("bf16", "bf16", True, -1, True, 0.0, 1.0, False), ("f32", "f32", False, 1, True, 0.9, 1.0, True),
    ("bf16", "f32", True, 50, False, 0.5, -2.0, True), ("bf16", "bf16", False, 0, False, 0.1, 1.0, True),
    ("f32", "f32", True, 700, True, 0.0, 1.0, True),
]


def make(T, D, form, wid=410):
    stream, block, post, rows, nxt, p, scale, gains = form
    rows = T if rows == -1 else rows
    t = {"X": padded(wid, 0, T, D, stream, 2.0), "Y": padded(wid, 1, T, D, block), "dH": padded(wid, 2, T, D, stream),
         "dN": padded(wid, 3, T, D, block) if nxt else None}
    vec = lambda i: (lambda g: (g.to_device(), g.f64()))(I.gaussian(wid, i, (D,), 1.0, "f32"))  # noqa: E731
    t["g_post"] = vec(4) if post and gains else None
    t["g_pre"] = vec(5) if nxt and gains else None
    t["gate"] = padded(wid, 6, -(-T // rows), D, "f32") if rows else None
    seed = (11 * D + T, 2 ** 33 + D)
    dev = {k: None if v is None else v[0] for k, v in t.items()}
    ref = {k: None if v is None else v[1] for k, v in t.items()}
    kw = dict(g_post=dev["g_post"], post_norm=post, gate=dev["gate"], gate_rows=rows or None, g_pre=dev["g_pre"], next_norm=nxt,
              scale=scale, p=p, seed=seed_of(*seed) if p else None, row0=17, eps=1e-6)
    f = SO.factors(T, D, p, seed, 17) if p else 1.0
    j = SO.Join(ref["X"], ref["Y"], ref["g_post"], post, ref["gate"], rows or None, ref["g_pre"], scale, f, 1e-6)
    return dev, ref, kw, j


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("T,D", SHAPES)
def test_join(T, D, form):
    say(f"residual_norm T={T} D={D} {form}")
    dev, ref, kw, j = make(T, D, form)
    h, n = P.residual_norm(dev["X"], dev["Y"], **kw)
    assert h.dtype == dev["X"].dtype
    close(h, j.h, j.h_size, "H")
    assert (n is None) == (not kw["next_norm"])
    if n is not None:
        close(n, j.n, j.n_size, "N")


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("T,D", SHAPES)
def test_join_gradients(T, D, form):
    say(f"residual_norm_backward T={T} D={D} {form}")
    dev, ref, kw, j = make(T, D, form)
    got = dict(zip(("dX", "dY", "dg_post", "dgate", "dg_pre"), P.residual_norm_backward(dev["X"], dev["Y"], dev["dH"], dev["dN"], **kw)))
    want = j.backward(ref["dH"], ref["dN"])
    for k, (g, size) in want.items():
        if got[k] is None:      # gains of 1 have no gradient
            assert k in ("dg_post", "dg_pre") and kw["g_" + k[3:]] is None
            continue
        close(got[k], g, size, k)
    assert (got["dgate"] is None) == (kw["gate"] is None)


def test_join_gradients_of_the_norm_alone():
    """No cotangent of H, as behind the last block."""
    dev, ref, kw, j = make(40, 264, FORMS[1])
    got = P.residual_norm_backward(dev["X"], dev["Y"], None, dev["dN"], **kw)
    want = j.backward(None, ref["dN"])
    for k, g in zip(("dX", "dY", "dg_post", "dgate", "dg_pre"), got):
        close(g, *want[k], k)


@pytest.mark.parametrize("T,D", [(300, 512), (70, 1096)])
def test_join_in_place_and_into_views(T, D):
    say(f"join in place T={T} D={D}")
    dev, ref, kw, j = make(T, D, FORMS[1])
    h, n = P.residual_norm(dev["X"], dev["Y"], **kw)
    g = P.residual_norm_backward(dev["X"], dev["Y"], dev["dH"], dev["dN"], **kw)
    X, Y = dev["X"].clone(), dev["Y"].clone()
    h2, n2 = P.residual_norm(X, Y, out=X, norm_out=Y, **kw)
    assert h2 is X and torch.equal(h2, h) and torch.equal(n2, n)
    room = [torch.full((T, 2 * D + 16), 5.0, dtype=t.dtype, device="cuda") for t in (h, n)]
    P.residual_norm(dev["X"], dev["Y"], out=room[0][:, 8:8 + D], norm_out=room[1][:, D:2 * D], **kw)
    assert torch.equal(room[0][:, 8:8 + D], h) and torch.equal(room[1][:, D:2 * D], n)
    assert bool((room[0][:, 8 + D:] == 5).all()) and bool((room[0][:, :8] == 5).all()) and bool((room[1][:, :D] == 5).all())
    dH, dN = dev["dH"].clone(), dev["dN"].clone()
    g2 = P.residual_norm_backward(dev["X"], dev["Y"], dH, dN, out=(dH, dN), **kw)
    assert all(torch.equal(a, b) for a, b in zip(g, g2))
    part = P.residual_norm_backward(dev["X"], dev["Y"], dev["dH"], dev["dN"], gain_out=(None, torch.empty_like(g[3]), None), **kw)
    assert part[2] is None and part[4] is None and all(torch.equal(a, b) for a, b in zip(part, g) if a is not None)


def test_join_of_dropped_values_that_are_not_finite():
    dev, ref, kw, j = make(30, 64, ("f32", "f32", False, 4, True, 0.5, 1.0, True))
    kept = torch.from_numpy(SO.factors(30, 64, 0.5, (11 * 64 + 30, 2 ** 33 + 64), 17) != 0).cuda()
    bad = torch.where(kept, dev["Y"], float("inf"))
    for a, b in zip(P.residual_norm(dev["X"], bad, **kw), P.residual_norm(dev["X"], dev["Y"], **kw)):
        assert torch.equal(a, b)
    for a, b in zip(P.residual_norm_backward(dev["X"], bad, dev["dH"], dev["dN"], **kw),
                    P.residual_norm_backward(dev["X"], dev["Y"], dev["dH"], dev["dN"], **kw)):
        assert a is None and b is None or torch.equal(a, b)


def test_join_without_rows():
    g = torch.ones(16, device="cuda")
    x = torch.zeros(0, 16, device="cuda")
    kw = dict(g_post=g, post_norm=True, g_pre=g, p=0.5, seed=seed_of(1, 1))
    h, n = P.residual_norm(x, x, **kw)
    assert h.shape == n.shape == (0, 16)
    got = P.residual_norm_backward(x, x, x, x, gate=torch.zeros(0, 16, device="cuda"), gate_rows=3, **kw)
    assert got[3].shape == (0, 16) and not got[2].any() and not got[4].any()


def test_a_captured_run_takes_the_seed_of_its_replay():
    """Forward and gradients in a graph, replayed over new inputs and seeds with eager work between."""
    T, D = 200, 1032
    dev, ref, kw, j = make(T, D, FORMS[1])
    seed = kw["seed"]
    first = seed.clone()

    def step():
        h, n = P.residual_norm(dev["X"], dev["Y"], **kw)
        d = P.dropout(n, 0.3, seed, residual=n)
        return [h, n, d, *P.residual_norm_backward(dev["X"], dev["Y"], dev["dH"], d, **kw)]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for r in range(3):
        seed.copy_(first + r)
        dev["Y"].mul_(-1.0 if r else 1.0)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, step()):
            assert torch.equal(a, b)


def test_two_streams_at_once():
    a, b = (make(513, 776, FORMS[i]) for i in (1, 3))
    want = [[*P.residual_norm(d["X"], d["Y"], **k), *P.residual_norm_backward(d["X"], d["Y"], d["dH"], d["dN"], **k)] for d, _, k, _ in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(3):
        for i, (d, _, k, _) in enumerate((a, b)):
            got[i] = [*P.residual_norm(d["X"], d["Y"], stream=streams[i], **k),
                      *P.residual_norm_backward(d["X"], d["Y"], d["dH"], d["dN"], stream=streams[i], **k)]
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(x is None and y is None or torch.equal(x, y) for x, y in zip(g, w))
