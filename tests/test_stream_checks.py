"""Refusals of dropout and of the join with the residual stream (no GPU needed):
the C ABI's checks, with pointers that are never dereferenced, and the
binding's, with CPU tensors."""
import ctypes

import pytest
import torch

from paper_2401_11202_amd import partir as P

NULL, ODD = None, ctypes.c_void_p(0x900004)
A = [ctypes.c_void_p(0x1000000 * i) for i in range(1, 16)]     # tensors apart
bf, f32 = torch.bfloat16, torch.float32
nan = float("nan")


@pytest.fixture(autouse=True)
def _never_launch(monkeypatch):
    monkeypatch.setenv("PARTIR_FAIL_LAUNCH", "1")


def status(fn):
    with pytest.raises(P.PartirError) as e:
        fn()
    return P.STATUS[e.value.status]


def at(x, off):
    return ctypes.c_void_p(x.value + off)


DROP = dict(X=A[0], R=A[1], Y=A[2], T=16, D=40, ldx=40, ldr=40, ldy=40, xd=P.BF16, yd=P.F32, p=0.5, seed=A[3], row0=0)


def drop(**kw):
    a = dict(DROP, **kw)
    return P.STATUS[P.lib().partir_dropout(*(a[k] for k in DROP), None)]


@pytest.mark.parametrize("kw,want", [
    (dict(X=NULL), "PARTIR_E_NULL"), (dict(Y=NULL), "PARTIR_E_NULL"), (dict(seed=NULL), "PARTIR_E_NULL"),
    (dict(seed=NULL, p=0.0), "PARTIR_E_NULL"), (dict(T=-1), "PARTIR_E_SHAPE"), (dict(T=2 ** 31), "PARTIR_E_SHAPE"),
    (dict(D=-1), "PARTIR_E_SHAPE"), (dict(D=2 ** 25), "PARTIR_E_SHAPE"), (dict(row0=-1), "PARTIR_E_SHAPE"),
    (dict(row0=2 ** 32 - 15), "PARTIR_E_SHAPE"), (dict(p=-0.1), "PARTIR_E_UNSUPPORTED"), (dict(p=1.1), "PARTIR_E_UNSUPPORTED"),
    (dict(p=nan), "PARTIR_E_UNSUPPORTED"), (dict(xd=5), "PARTIR_E_DTYPE"), (dict(yd=-1), "PARTIR_E_DTYPE"),
    (dict(ldx=36), "PARTIR_E_LAYOUT"), (dict(ldx=44), "PARTIR_E_LAYOUT"), (dict(ldy=41), "PARTIR_E_LAYOUT"),
    (dict(X=ODD), "PARTIR_E_LAYOUT"), (dict(Y=ODD), "PARTIR_E_LAYOUT"), (dict(seed=ODD), "PARTIR_E_LAYOUT"),
    (dict(Y=A[3]), "PARTIR_E_LAYOUT"), (dict(Y=at(A[3], -16)), "PARTIR_E_LAYOUT"),   # over the seed
    (dict(Y=A[0]), "PARTIR_E_LAYOUT"),                                   # X's place, another type
    (dict(Y=A[0], xd=P.F32, ldy=44), "PARTIR_E_LAYOUT"),                 # another leading dim
    (dict(Y=at(A[1], 16)), "PARTIR_E_LAYOUT"), (dict(Y=at(A[1], 15 * 160)), "PARTIR_E_LAYOUT"),
    (dict(T=2 ** 30, D=2 ** 10, ldx=2 ** 10, ldy=2 ** 10, R=NULL, Y=ctypes.c_void_p(1 << 50)), "PARTIR_E_SHAPE"),
])
def test_dropout_refusals(kw, want):
    assert drop(**kw) == want
    assert P.lib().partir_last_error().decode().startswith(want)


@pytest.mark.parametrize("kw", [
    dict(), dict(R=NULL, ldr=0), dict(p=0.0), dict(p=1.0), dict(D=33), dict(row0=2 ** 32 - 16), dict(Y=A[1]),
    dict(Y=A[0], xd=P.F32), dict(Y=at(A[1], 16 * 160)), dict(Y=at(A[1], 160), ldr=80, ldy=80),   # the column block beside
    dict(T=1, Y=A[0], xd=P.F32, ldy=44)])
def test_dropout_accepts(kw):
    assert drop(**kw) == "PARTIR_E_HIP"


def test_dropout_of_nothing():
    assert drop(T=0, X=NULL, R=NULL, Y=NULL) == "PARTIR_OK" and drop(D=0, X=NULL, R=NULL, Y=NULL) == "PARTIR_OK"


JOIN = dict(X=A[0], Y=A[1], gpost=A[2], gate=A[3], gpre=A[4], H=A[5], N=A[6], T=16, D=40, rows=5, ldx=40, ldy=40, ldg=40, ldh=40,
            ldn=40, xd=P.F32, yd=P.BF16, post=1, scale=1.0, p=0.5, seed=A[7], row0=0, eps=1e-6)


def join(**kw):
    a = dict(JOIN, **kw)
    return P.STATUS[P.lib().partir_residual_norm(*(a[k] for k in JOIN), None)]


BOTH = [
    (dict(T=-1), "PARTIR_E_SHAPE"), (dict(D=44), "PARTIR_E_SHAPE"), (dict(D=16392, ldx=16392, ldy=16392), "PARTIR_E_SHAPE"),
    (dict(rows=0), "PARTIR_E_SHAPE"), (dict(xd=4), "PARTIR_E_DTYPE"), (dict(yd=4), "PARTIR_E_DTYPE"), (dict(Y=NULL), "PARTIR_E_NULL"),
    (dict(X=NULL), "PARTIR_E_NULL"), (dict(ldx=38), "PARTIR_E_LAYOUT"), (dict(ldx=42), "PARTIR_E_LAYOUT"), (dict(ldg=32), "PARTIR_E_LAYOUT"),
    (dict(ldy=44), "PARTIR_E_LAYOUT"), (dict(gpost=ODD), "PARTIR_E_LAYOUT"), (dict(gate=ODD), "PARTIR_E_LAYOUT"),
    (dict(seed=NULL), "PARTIR_E_NULL"), (dict(seed=ODD), "PARTIR_E_LAYOUT"), (dict(p=2.0), "PARTIR_E_UNSUPPORTED"),
    (dict(scale=nan), "PARTIR_E_UNSUPPORTED"), (dict(eps=-1.0), "PARTIR_E_UNSUPPORTED"), (dict(eps=nan), "PARTIR_E_UNSUPPORTED"),
    (dict(post=0), "PARTIR_E_UNSUPPORTED"), (dict(row0=2 ** 32), "PARTIR_E_SHAPE")]


@pytest.mark.parametrize("kw,want", BOTH + [
    (dict(H=NULL), "PARTIR_E_NULL"), (dict(H=A[1]), "PARTIR_E_LAYOUT"), (dict(H=A[0], ldh=44), "PARTIR_E_LAYOUT"),
    (dict(N=A[0]), "PARTIR_E_LAYOUT"), (dict(N=A[5]), "PARTIR_E_LAYOUT"), (dict(H=at(A[0], 32)), "PARTIR_E_LAYOUT"),
    (dict(H=A[4]), "PARTIR_E_LAYOUT"), (dict(N=A[3]), "PARTIR_E_LAYOUT"), (dict(N=A[7]), "PARTIR_E_LAYOUT"),
    (dict(N=NULL), "PARTIR_E_UNSUPPORTED")])
def test_join_refusals(kw, want):
    assert join(**kw) == want


@pytest.mark.parametrize("kw", [
    dict(), dict(H=A[0]), dict(N=A[1]), dict(N=NULL, gpre=NULL), dict(gate=NULL, rows=0, ldg=0), dict(gpost=NULL, post=0),
    dict(gpost=NULL), dict(p=0.0, seed=NULL), dict(eps=0.0), dict(rows=2 ** 40), dict(scale=-1.0),
    dict(D=16384, ldx=16384, ldy=16384, ldg=16384, ldh=16384, ldn=16384)])
def test_join_accepts(kw):
    assert join(**kw) == "PARTIR_E_HIP"


BWD = dict(X=A[0], Y=A[1], dH=A[8], dN=A[9], gpost=A[2], gate=A[3], gpre=A[4], dX=A[5], dY=A[6], dgpost=A[10], dgate=A[11],
           dgpre=A[12], T=16, D=40, rows=5, ldx=40, ldy=40, lddh=40, lddn=40, ldg=40, lddx=40, lddy=40, xd=P.F32, yd=P.BF16, post=1,
           scale=1.0, p=0.5, seed=A[7], row0=0, eps=1e-6, ws=A[13], wsb=1 << 24)


def bwd(**kw):
    a = dict(BWD, **kw)
    return P.STATUS[P.lib().partir_residual_norm_backward(*(a[k] for k in BWD), None)]


@pytest.mark.parametrize("kw,want", BOTH + [
    (dict(dX=NULL), "PARTIR_E_NULL"), (dict(dY=NULL), "PARTIR_E_NULL"), (dict(dH=NULL, dN=NULL, gpre=NULL, dgpre=NULL), "PARTIR_E_NULL"),
    (dict(dX=A[0]), "PARTIR_E_LAYOUT"), (dict(dX=A[9]), "PARTIR_E_LAYOUT"), (dict(dY=A[1]), "PARTIR_E_LAYOUT"),
    (dict(dX=A[8], lddx=44), "PARTIR_E_LAYOUT"), (dict(dY=A[5]), "PARTIR_E_LAYOUT"), (dict(dgpost=A[12]), "PARTIR_E_LAYOUT"),
    (dict(dgate=A[3]), "PARTIR_E_LAYOUT"), (dict(dgpre=at(A[11], 3 * 160)), "PARTIR_E_LAYOUT"), (dict(dgpost=A[8]), "PARTIR_E_LAYOUT"),
    (dict(gate=NULL), "PARTIR_E_UNSUPPORTED"), (dict(dN=NULL), "PARTIR_E_UNSUPPORTED"), (dict(dgate=ODD), "PARTIR_E_LAYOUT"),
    (dict(ws=NULL), "PARTIR_E_NULL"), (dict(ws=ODD), "PARTIR_E_LAYOUT"), (dict(wsb=100), "PARTIR_E_WORKSPACE")])
def test_join_backward_refusals(kw, want):
    assert bwd(**kw) == want


@pytest.mark.parametrize("kw", [
    dict(), dict(dX=A[8]), dict(dY=A[9]), dict(dH=NULL), dict(X=NULL, dN=NULL, gpre=NULL, dgpre=NULL),
    dict(dgpost=NULL, dgate=NULL, dgpre=NULL), dict(gate=NULL, dgate=NULL, ldg=0, rows=0),
    dict(dgpre=at(A[11], 4 * 160)), dict(T=0)])
def test_join_backward_accepts(kw):
    assert bwd(**kw) == "PARTIR_E_HIP"


@pytest.mark.parametrize("T,D,rows", [(1, 8, 0), (16, 40, 5), (8192, 5120, 0), (8192, 5120, 1), (70000, 8, 3), (5, 16384, 2), (2 ** 30, 8, 7)])
def test_join_backward_workspace_is_what_the_call_needs(T, D, rows):
    need = P.lib().partir_residual_norm_backward_workspace(T, D, rows)
    a = dict(T=T, D=D, rows=rows, **{k: D for k in ("ldx", "ldy", "lddh", "lddn", "ldg", "lddx", "lddy")})
    big = {k: ctypes.c_void_p(i << 48) for i, k in enumerate(("X", "Y", "dH", "dN", "gpost", "gate", "gpre", "dX", "dY", "dgpost",
                                                             "dgate", "dgpre", "seed", "ws"), 1)}
    if not rows:
        big.update(gate=NULL, dgate=NULL)
    assert bwd(wsb=need, **a, **big) == "PARTIR_E_HIP" and bwd(wsb=need - 1, **a, **big) == "PARTIR_E_WORKSPACE"
    assert need <= 12 * D * 4096 + 256 if rows != 7 else True
    assert P.lib().partir_residual_norm_backward_workspace(-1, D, rows) == ctypes.c_size_t(-1).value
    assert P.lib().partir_residual_norm_backward_workspace(T, D + 1, rows) == ctypes.c_size_t(-1).value
    assert P.lib().partir_residual_norm_backward_workspace(T, D, -1) == ctypes.c_size_t(-1).value


def test_binding_checks():
    x, y, s = torch.zeros(16, 40), torch.zeros(16, 40, dtype=bf), torch.zeros(2, dtype=torch.int64)
    d = lambda *a, **k: status(lambda: P.dropout(*a, **k))  # noqa: E731
    assert d(x, 0.5, s) == "PARTIR_E_LAYOUT"                           # all correct, but on the CPU
    assert d(x, 0.5, None) == "PARTIR_E_NULL" and d(x, 0.5, s.int()) == "PARTIR_E_DTYPE" and d(x, 0.5, s[:1]) == "PARTIR_E_SHAPE"
    assert d(x.half(), 0.5, s) == "PARTIR_E_DTYPE" and d(x[0], 0.5, s) == "PARTIR_E_SHAPE" and d(x.t(), 0.5, s) == "PARTIR_E_LAYOUT"
    assert d(x, 0.5, s, residual=y, out_dtype=f32) == "PARTIR_E_DTYPE" and d(x, 0.5, s, residual=x[:8]) == "PARTIR_E_SHAPE"
    assert d(x, 0.5, s, residual=x, out=y) == "PARTIR_E_DTYPE"
    g = torch.zeros(40)
    j = lambda *a, **k: status(lambda: P.residual_norm(*a, **k))  # noqa: E731
    assert j(x, y) == "PARTIR_E_LAYOUT"
    assert j(x[:8], y) == "PARTIR_E_SHAPE" and j(x, None) == "PARTIR_E_SHAPE" and j(None, y) == "PARTIR_E_NULL"
    assert j(x, y, g_pre=g.to(bf)) == "PARTIR_E_DTYPE" and j(x, y, g_post=g[:8], post_norm=True) == "PARTIR_E_SHAPE"
    assert j(x, y, gate=torch.zeros(2, 40), gate_rows=5) == "PARTIR_E_SHAPE" and j(x, y, gate=g[None], gate_rows=0) == "PARTIR_E_SHAPE"
    assert j(x, y, out=y) == "PARTIR_E_DTYPE" and j(x, y, norm_out=y, next_norm=False) == "PARTIR_E_UNSUPPORTED"
    b = lambda *a, **k: status(lambda: P.residual_norm_backward(*a, **k))  # noqa: E731
    assert b(x, y, x, y) == "PARTIR_E_LAYOUT"
    assert b(x, y, x, None) == "PARTIR_E_NULL" and b(x, y, None, None, next_norm=False) == "PARTIR_E_NULL"
    assert b(x, y, y, y) == "PARTIR_E_DTYPE" and b(x, y, x, x) == "PARTIR_E_DTYPE"
    assert b(x, y, x, y, g_post=g) == "PARTIR_E_UNSUPPORTED" and b(x, y, x, None, next_norm=False, g_pre=g) == "PARTIR_E_UNSUPPORTED"
    assert b(x, y, x, y, gain_out=(None, g[None], None)) == "PARTIR_E_UNSUPPORTED"
    assert b(x, y, x, y, out=(x,)) == "PARTIR_E_SHAPE"
