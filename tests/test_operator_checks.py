"""Refusals of the operators beside the nests (no GPU needed): the C ABI's
checks, with pointers that are never dereferenced, and the binding's, with CPU
tensors; and the frequencies of rotary positions, which the host computes."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import operators_oracle as OO
from paper_2401_11202_amd import partir as P

A, ODD, NULL = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10004), None
T1, T2, T3, T4, T5, T6, T7, T8 = (ctypes.c_void_p(0x100000 * i) for i in range(1, 9))   # tensors apart
bf, f32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _never_launch(monkeypatch):
    monkeypatch.setenv("PARTIR_FAIL_LAUNCH", "1")


def name(st):
    return P.STATUS[st]


def status(fn):
    with pytest.raises(P.PartirError) as e:
        fn()
    return P.STATUS[e.value.status]


# ---------------------------------------------------------------------------
# rotary and norms
# ---------------------------------------------------------------------------
ROT = dict(Q=T1, K=T2, Qo=T3, Ko=T4, f=A, pos=NULL, p64=0, T=16, S=16, Hq=4, Hk=2, dh=64, rd=64, ldq=256, ldk=128, ldqo=256,
           ldko=128, dt=P.BF16, inter=0, inv=0, mag=1.0)


def rotary(**kw):
    a = dict(ROT, **kw)
    return name(P.lib().partir_rotary(*(a[k] for k in ROT), None))


BAD_ROT = [
    (dict(Q=NULL), "PARTIR_E_NULL"), (dict(Ko=NULL), "PARTIR_E_NULL"), (dict(f=NULL), "PARTIR_E_NULL"),
    (dict(T=-1), "PARTIR_E_SHAPE"), (dict(T=2 ** 31), "PARTIR_E_SHAPE"), (dict(S=0), "PARTIR_E_SHAPE"),
    (dict(dh=60), "PARTIR_E_SHAPE"), (dict(dh=0), "PARTIR_E_SHAPE"), (dict(dh=264, rd=8), "PARTIR_E_SHAPE"),
    (dict(rd=63), "PARTIR_E_SHAPE"), (dict(rd=66), "PARTIR_E_SHAPE"), (dict(rd=-2), "PARTIR_E_SHAPE"),
    (dict(Hq=-1), "PARTIR_E_SHAPE"), (dict(Hq=2 ** 40), "PARTIR_E_SHAPE"), (dict(dt=7), "PARTIR_E_DTYPE"),
    (dict(ldq=248), "PARTIR_E_LAYOUT"), (dict(ldq=260), "PARTIR_E_LAYOUT"), (dict(ldk=2 ** 25), "PARTIR_E_SHAPE"),
    (dict(Q=ODD), "PARTIR_E_LAYOUT"), (dict(Ko=ODD), "PARTIR_E_LAYOUT"), (dict(f=ODD), "PARTIR_E_LAYOUT"),
    (dict(pos=ODD, p64=1), "PARTIR_E_LAYOUT"), (dict(mag=float("nan")), "PARTIR_E_UNSUPPORTED"),
    (dict(mag=float("inf")), "PARTIR_E_UNSUPPORTED"),
]
GOOD_ROT = [dict(), dict(pos=A, p64=1, S=0), dict(pos=ODD), dict(Hk=0, K=NULL, Ko=NULL, ldk=0, ldko=0), dict(rd=0, f=NULL),
            dict(rd=2), dict(dt=P.F32), dict(ldq=264, ldko=2 ** 24)]


@pytest.mark.parametrize("kw,want", BAD_ROT)
def test_rotary_refusals(kw, want):
    assert rotary(**kw) == want
    assert P.lib().partir_last_error().decode().startswith(want)


@pytest.mark.parametrize("kw", GOOD_ROT)
def test_rotary_accepts(kw):
    assert rotary(**kw) == "PARTIR_E_HIP"          # reached the launch, which is forced to fail


def test_nothing_to_do_launches_nothing():
    assert rotary(T=0, Q=NULL, K=NULL, Qo=NULL, Ko=NULL, f=NULL) == "PARTIR_OK"
    assert rotary(Hq=0, Hk=0, Q=NULL, K=NULL, Qo=NULL, Ko=NULL) == "PARTIR_OK"


NORM = dict(Q=T1, K=T2, gq=A, gk=A, Qo=T3, Ko=T4, f=A, pos=NULL, p64=0, T=16, S=16, Hq=4, Hk=2, dh=64, rd=64, ldq=256, ldk=128,
            ldqo=256, ldko=128, dt=P.BF16, inter=0, mag=1.0, eps=1e-6)
BWD = dict(Q=T1, K=T2, dQo=T3, dKo=T4, gq=A, gk=A, dQ=T5, dK=T6, dgq=T7, dgk=T8, f=A, pos=NULL, p64=0, T=16, S=16, Hq=4, Hk=2, dh=64,
           rd=64, ldq=256, ldk=128, lddqo=256, lddko=128, lddq=256, lddk=128, dt=P.BF16, inter=0, mag=1.0, eps=1e-6, ws=A,
           wsb=1 << 24)


def norm(**kw):
    a = dict(NORM, **kw)
    return name(P.lib().partir_qk_norm_rotary(*(a[k] for k in NORM), None))


def bwd(**kw):
    a = dict(BWD, **kw)
    return name(P.lib().partir_qk_norm_rotary_backward(*(a[k] for k in BWD), None))


def test_qk_norm_refusals():
    for kw, want in BAD_ROT:
        assert norm(**kw) == want, kw
    assert norm(gq=ODD) == "PARTIR_E_LAYOUT" and norm(eps=-1.0) == "PARTIR_E_UNSUPPORTED"
    assert norm(eps=float("nan")) == "PARTIR_E_UNSUPPORTED"
    for kw in ({}, dict(gq=NULL, gk=NULL), dict(eps=0.0), dict(rd=0, f=NULL)):
        assert norm(**kw) == "PARTIR_E_HIP", kw


def test_qk_norm_backward_refusals():
    need = P.lib().partir_qk_norm_rotary_backward_workspace(16, 4, 2, 64, 64, P.BF16)
    assert 0 < need <= 1 << 24
    for kw, want in ((dict(dQo=NULL), "PARTIR_E_NULL"), (dict(dK=NULL), "PARTIR_E_NULL"), (dict(lddqo=8), "PARTIR_E_LAYOUT"),
                     (dict(lddqo=-8), "PARTIR_E_LAYOUT"), (dict(dQo=ODD), "PARTIR_E_LAYOUT"), (dict(lddk=130), "PARTIR_E_LAYOUT"),
                     (dict(wsb=need - 1), "PARTIR_E_WORKSPACE"), (dict(ws=NULL), "PARTIR_E_NULL"), (dict(ws=ODD), "PARTIR_E_LAYOUT"),
                     (dict(dgq=ctypes.c_void_p(0x10002)), "PARTIR_E_LAYOUT"), (dict(eps=-1e-9), "PARTIR_E_UNSUPPORTED"),
                     (dict(wsb=need), "PARTIR_E_HIP"), (dict(dgq=NULL, dgk=NULL), "PARTIR_E_HIP"),
                     (dict(T=0, ws=NULL, wsb=0, dgq=NULL, dgk=NULL), "PARTIR_OK"), (dict(T=0, ws=NULL, wsb=0), "PARTIR_E_HIP")):
        assert bwd(**kw) == want, kw
    bad = ctypes.c_size_t(-1).value
    for a in ((-1, 4, 2, 64, 64, P.BF16), (16, 4, 2, 60, 60, P.BF16), (16, 4, 2, 64, 66, P.BF16), (16, -4, 2, 64, 64, P.BF16),
              (16, 4, 2, 64, 64, 9)):
        assert P.lib().partir_qk_norm_rotary_backward_workspace(*a) == bad
    assert P.lib().partir_qk_norm_rotary_backward_workspace(0, 4, 2, 64, 64, P.BF16) == 0


@pytest.mark.parametrize("T,Hq,Hk,dh,rd", [(1, 1, 0, 8, 8), (100000, 64, 64, 256, 2), (2 ** 30, 1, 1, 64, 64), (7, 2 ** 16, 1, 128, 128)])
def test_qk_norm_backward_workspace_is_what_the_call_needs(T, Hq, Hk, dh, rd):
    for dt in (P.BF16, P.F32):
        need = P.lib().partir_qk_norm_rotary_backward_workspace(T, Hq, Hk, dh, rd, dt)
        a = dict(T=T, Hq=Hq, Hk=Hk, dh=dh, rd=rd, ldq=Hq * dh, ldk=Hk * dh, lddqo=Hq * dh, lddko=Hk * dh, lddq=Hq * dh,
                 lddk=Hk * dh, dt=dt)
        assert bwd(wsb=need, **a) == "PARTIR_E_HIP" and bwd(wsb=need - 1, **a) == "PARTIR_E_WORKSPACE"
        assert need <= 1024 * 2 * 256 * 4


@pytest.mark.parametrize("scaling,kw", [(None, {}), ("linear", dict(factor=4.0)), ("base", dict(factor=8.0)),
                                        ("parts", dict(factor=16.0, original_length=4096)),
                                        ("parts", dict(factor=2.0, original_length=64, slow_turns=0.25, fast_turns=3.0))])
@pytest.mark.parametrize("rd", [2, 20, 64, 128, 256])
def test_rotary_frequencies(scaling, kw, rd):
    if scaling == "base" and rd == 2:
        assert status(lambda: P.rotary_frequencies(rd, scaling=scaling, device="cpu", **kw)) == "PARTIR_E_UNSUPPORTED"
        return
    got = P.rotary_frequencies(rd, base=50000.0, scaling=scaling, device="cpu", **kw).numpy()
    o = {"slow_turns": "slow", "fast_turns": "fast"}
    ref = OO.frequencies(rd, 50000.0, scaling, **{o.get(k, k): v for k, v in kw.items()})
    assert got.dtype == np.float64 and np.abs(got - ref).max() <= 1e-15 * 8
    if scaling == "base":       # the slowest pair is as with linear scaling, the fastest unchanged
        lin = OO.frequencies(rd, 50000.0, "linear", kw["factor"])
        assert got[0] == 1.0 and abs(got[-1] / lin[-1] - 1) < 1e-12
    if scaling == "parts":      # between the two, fast pairs kept and slow ones divided
        plain = OO.frequencies(rd, 50000.0)
        assert (got <= plain * (1 + 1e-15)).all() and (got >= plain / kw["factor"] * (1 - 1e-15)).all()


def test_rotary_frequencies_refusals():
    for kw in (dict(base=1.0), dict(base=float("inf")), dict(scaling="linear", factor=0.5), dict(scaling="nope"),
               dict(scaling="parts", factor=2.0), dict(scaling="parts", factor=2.0, original_length=9, slow_turns=2.0, fast_turns=1.0)):
        assert status(lambda: P.rotary_frequencies(64, device="cpu", **kw)) == "PARTIR_E_UNSUPPORTED", kw
    for rd in (63, 258):
        assert status(lambda: P.rotary_frequencies(rd, device="cpu")) == "PARTIR_E_SHAPE"


def test_rotary_binding_checks():
    q, k, f = torch.zeros(16, 256, dtype=bf), torch.zeros(16, 128, dtype=bf), torch.zeros(32, dtype=torch.float64)
    call = lambda *a, **kw: status(lambda: P.rotary(*a, **{**dict(d_head=64), **kw}))  # noqa: E731
    assert call(q, k, f) == "PARTIR_E_LAYOUT"                                   # all correct, but on the CPU
    assert call(q, k, f, d_head=48) == "PARTIR_E_SHAPE"
    assert call(q, k, f, d_head=0) == "PARTIR_E_SHAPE"
    assert call(q, k[:8], f) == "PARTIR_E_SHAPE"
    assert call(q, k.float(), f) == "PARTIR_E_DTYPE"
    assert call(q.half(), None, f) == "PARTIR_E_DTYPE"
    assert call(q, k, f.float()) == "PARTIR_E_DTYPE"
    assert call(q.t(), None, f, d_head=8) == "PARTIR_E_LAYOUT"
    assert call(q, k, f, positions=torch.zeros(15, dtype=torch.int64)) == "PARTIR_E_SHAPE"
    assert call(q, k, f, positions=torch.zeros(16)) == "PARTIR_E_DTYPE"
    assert call(q, k, f, out=(q, None)) == "PARTIR_E_SHAPE"
    assert call(q, k, f, out=(q, q)) == "PARTIR_E_SHAPE"
    assert call(q, k, f, out=(q, k.float())) == "PARTIR_E_DTYPE"
    g = torch.zeros(64)
    assert status(lambda: P.qk_norm_rotary(q, k, g[:32], g, f, d_head=64)) == "PARTIR_E_SHAPE"
    assert status(lambda: P.qk_norm_rotary(q, k, g, g.to(bf), f, d_head=64)) == "PARTIR_E_DTYPE"
    assert status(lambda: P.qk_norm_rotary(q, k, g, g, f, d_head=64)) == "PARTIR_E_LAYOUT"
    b = lambda *a, **kw: status(lambda: P.qk_norm_rotary_backward(*a, **{**dict(d_head=64), **kw}))  # noqa: E731
    assert b(q, k, q, None, g, g, f) == "PARTIR_E_NULL"
    assert b(q, k, q, q, g, g, f) == "PARTIR_E_SHAPE"
    assert b(q, k, q, k, g, g, f, gain_out=(g, g.to(bf))) == "PARTIR_E_DTYPE"
    assert b(q, k, q, k, g, g, f) == "PARTIR_E_LAYOUT"


# ---------------------------------------------------------------------------
# norm of gradients
# ---------------------------------------------------------------------------
def clip(ptrs, numel, dts, out=None, max_norm=1.0, norm=A, ws=A, wsb=1 << 24, n=None):
    k = len(ptrs)
    return name(P.lib().partir_clip_grad_norm((ctypes.c_void_p * k)(*ptrs), (ctypes.c_void_p * k)(*(out or ptrs)),
                                              (ctypes.c_int64 * k)(*numel), (ctypes.c_int * k)(*dts), k if n is None else n,
                                              max_norm, norm, ws, wsb, None))


def test_clip_refusals():
    one = ([0x20000], [100], [P.F32])
    assert clip(*one) == "PARTIR_E_HIP"
    assert clip([0x20002], [100], [P.F32]) == "PARTIR_E_LAYOUT"
    assert clip([0x20002], [100], [P.BF16]) == "PARTIR_E_HIP"
    assert clip([0x20001], [100], [P.BF16]) == "PARTIR_E_LAYOUT"
    assert clip([None], [100], [P.F32]) == "PARTIR_E_NULL"
    assert clip([None], [0], [P.F32]) == "PARTIR_E_HIP"                         # empty: the norm 0 is written
    assert clip([0x20000], [-1], [P.F32]) == "PARTIR_E_SHAPE"
    assert clip([0x20000], [1 << 41], [P.F32]) == "PARTIR_E_SHAPE"
    assert clip([0x20000], [100], [3]) == "PARTIR_E_DTYPE"
    assert clip(*one, max_norm=-1.0) == "PARTIR_E_UNSUPPORTED"
    assert clip(*one, max_norm=float("nan")) == "PARTIR_E_UNSUPPORTED"
    assert clip(*one, max_norm=float("inf")) == "PARTIR_E_HIP"
    assert clip(*one, norm=NULL) == "PARTIR_E_NULL"
    assert clip(*one, n=-1) == "PARTIR_E_SHAPE"
    need = P.lib().partir_grad_norm_workspace(1)
    assert clip(*one, wsb=need) == "PARTIR_E_HIP" and clip(*one, wsb=need - 1) == "PARTIR_E_WORKSPACE"
    assert clip(*one, ws=ODD) == "PARTIR_E_LAYOUT" and clip(*one, ws=NULL) == "PARTIR_E_NULL"
    assert P.lib().partir_grad_norm_workspace(-1) == ctypes.c_size_t(-1).value
    assert P.lib().partir_grad_norm_workspace(0) == 0


def test_overlapping_outputs_are_refused():
    two = [P.F32, P.F32]
    assert clip([0x20000, 0x20000], [100, 100], two) == "PARTIR_E_LAYOUT"       # the same tensor twice
    assert clip([0x20190, 0x20000], [100, 101], two) == "PARTIR_E_LAYOUT"       # one value shared, in either order
    assert clip([0x20000, 0x20190], [101, 100], two) == "PARTIR_E_LAYOUT"
    assert clip([0x20190, 0x20000], [100, 100], two) == "PARTIR_E_HIP"          # neighbours
    assert clip([0x20000, 0x20000], [100, 100], two, out=[0x30000, 0x40000]) == "PARTIR_E_HIP"   # read twice, written apart
    assert clip([0x20000, 0x30000], [100, 100], two, out=[0x30000, 0x40000]) == "PARTIR_E_LAYOUT"
    assert clip([0x20000], [100], [P.F32], out=[0x20004]) == "PARTIR_E_LAYOUT"  # its own input, shifted
    assert clip([0x20000, 0x20000], [100, 0], two) == "PARTIR_E_HIP"


def test_clip_binding_checks():
    t = torch.zeros(8)
    assert status(lambda: P.grad_norm([t])) == "PARTIR_E_LAYOUT"                # on the CPU
    assert status(lambda: P.grad_norm([t, None])) == "PARTIR_E_NULL"
    assert status(lambda: P.grad_norm([t.half()])) == "PARTIR_E_DTYPE"
    assert status(lambda: P.grad_norm([torch.zeros(4, 4).t()[:2]])) == "PARTIR_E_LAYOUT"
    assert status(lambda: P.clip_grad_norm([t], 1.0, out=[])) == "PARTIR_E_SHAPE"
    assert status(lambda: P.clip_grad_norm([t], 1.0, out=[t[:4]])) == "PARTIR_E_SHAPE"
    assert status(lambda: P.clip_grad_norm([t], 1.0, out=[t.to(bf)])) == "PARTIR_E_DTYPE"
    assert status(lambda: P.clip_grad_norm([t], 1.0, norm=torch.zeros(1))) == "PARTIR_E_SHAPE"


# ---------------------------------------------------------------------------
# cross attention
# ---------------------------------------------------------------------------
CROSS = dict(Q=A, K=A, V=A, O=T1, B=2, Sq=3, Sk=50, Hq=4, Hk=2, dh=128, ldq=512, ldk=256, ldv=256, ldo=512, lens=NULL, scale=0.0,
             ws=NULL, wsb=0)
CROSS_BWD = dict(Q=T1, K=T2, V=T3, O=T4, dO=T5, lse=A, dQ=T6, dK=T7, dV=T8, B=2, Sq=3, Sk=50, Hq=4, Hk=2, dh=128, ldq=512, ldk=256,
                 ldv=256, ldo=512, lddo=512, lddq=512, lddk=256, lddv=256, lens=NULL, scale=0.0, ws=A, wsb=1 << 30)


def cross(**kw):
    a = dict(CROSS, **kw)
    return name(P.lib().partir_cross_attention(*(a[k] for k in CROSS), None))


def cross_bwd(**kw):
    a = dict(CROSS_BWD, **kw)
    return name(P.lib().partir_cross_attention_backward(*(a[k] for k in CROSS_BWD), None))


BAD_CROSS = [
    (dict(Q=NULL), "PARTIR_E_NULL"), (dict(K=NULL), "PARTIR_E_NULL"), (dict(V=NULL), "PARTIR_E_NULL"),
    (dict(O=NULL), "PARTIR_E_NULL"), (dict(Q=ODD), "PARTIR_E_LAYOUT"), (dict(V=ODD), "PARTIR_E_LAYOUT"),
    (dict(B=-1), "PARTIR_E_SHAPE"), (dict(Sq=-1), "PARTIR_E_SHAPE"), (dict(Sk=2 ** 31), "PARTIR_E_SHAPE"),
    (dict(B=2 ** 20, Sk=2 ** 20), "PARTIR_E_SHAPE"), (dict(B=2 ** 16, Sq=2 ** 15, Sk=0), "PARTIR_E_SHAPE"),
    (dict(dh=64, ldq=512), "PARTIR_E_SHAPE"), (dict(Hq=0), "PARTIR_E_SHAPE"), (dict(Hk=0), "PARTIR_E_SHAPE"),
    (dict(Hk=8), "PARTIR_E_SHAPE"), (dict(Hk=3), "PARTIR_E_DIVISIBILITY"), (dict(Hq=2 ** 18, Hk=2 ** 18), "PARTIR_E_SHAPE"),
    (dict(ldq=504), "PARTIR_E_LAYOUT"), (dict(ldk=260), "PARTIR_E_LAYOUT"), (dict(ldv=2 ** 24 + 8), "PARTIR_E_SHAPE"),
    (dict(ldo=0), "PARTIR_E_LAYOUT"), (dict(lens=ctypes.c_void_p(0x10002)), "PARTIR_E_LAYOUT"),
    (dict(scale=float("nan")), "PARTIR_E_UNSUPPORTED"), (dict(scale=float("inf")), "PARTIR_E_UNSUPPORTED"),
    (dict(scale=1e-38), "PARTIR_E_UNSUPPORTED"),
]


@pytest.mark.parametrize("kw,want", BAD_CROSS)
def test_cross_attention_refusals(kw, want):
    assert cross(**kw) == want
    if "O" not in kw or kw["O"]:
        assert cross_bwd(**kw) == want


def test_cross_attention_accepts():
    for kw in ({}, dict(lens=ODD), dict(ldk=512, ldv=2 ** 24), dict(Sk=0, K=NULL, V=NULL), dict(Hk=4, ldk=512, ldv=512)):
        assert cross(**kw) == "PARTIR_E_HIP", kw
        assert cross_bwd(**dict(kw, lddk=512, lddv=512, **({"dK": NULL, "dV": NULL} if "Sk" in kw else {}))) == "PARTIR_E_HIP", kw
    assert cross(B=0, Q=NULL, K=NULL, V=NULL, O=NULL) == "PARTIR_OK"
    assert cross(Sq=0, Q=NULL, K=NULL, V=NULL, O=NULL) == "PARTIR_OK"      # no query reads a key
    assert cross_bwd(Sq=0, Q=NULL, O=NULL, dO=NULL, lse=NULL, dQ=NULL) == "PARTIR_E_HIP"    # dK, dV: zeros
    assert cross_bwd(Sq=0, Sk=0, Q=NULL, K=NULL, V=NULL, O=NULL, dO=NULL, lse=NULL, dQ=NULL, dK=NULL, dV=NULL) == "PARTIR_OK"
    for kw in (dict(lse=NULL), dict(dO=NULL), dict(dQ=NULL), dict(dK=NULL), dict(dV=NULL)):
        assert cross_bwd(**kw) == "PARTIR_E_NULL", kw
    for kw in (dict(lse=ctypes.c_void_p(0x10002)), dict(lddo=500), dict(lddq=8), dict(lddk=248), dict(dV=ODD)):
        assert cross_bwd(**kw) == "PARTIR_E_LAYOUT", kw


@pytest.mark.parametrize("B,Sq,Sk,Hq,Hk", [(2, 3, 50, 4, 2), (1, 1, 131072, 32, 8), (4, 4096, 2048, 32, 8), (2, 4096, 77, 8, 8),
                                           (1, 2 ** 20, 2 ** 20, 1, 1), (1, 1, 2 ** 30, 1, 1), (1, 2 ** 29, 1, 2, 1),
                                           (64, 1, 4097, 8, 1), (1, 700, 33, 3, 1)])
def test_cross_attention_workspace_is_what_the_call_needs(B, Sq, Sk, Hq, Hk):
    z = (B, Sq, Sk, Hq, Hk, 128)
    need, plan = P.lib().partir_cross_attention_workspace(*z), P.plan_cross_attention(B, Sq, Sk, Hq, Hk)
    assert need == plan["workspace_bytes"] and (need > 0) == (plan["n_virtual_shards"] > 1) == (plan["n_launches"] == 2)
    a = dict(B=B, Sq=Sq, Sk=Sk, Hq=Hq, Hk=Hk, ldq=Hq * 128, ldo=Hq * 128, ldk=Hk * 128, ldv=Hk * 128, ws=A)
    assert cross(wsb=need, **a) == "PARTIR_E_HIP"
    if need:
        assert cross(wsb=need - 1, **a) == "PARTIR_E_WORKSPACE" and cross(**dict(a, wsb=need, ws=NULL)) == "PARTIR_E_NULL"
    a.update(lddo=Hq * 128, lddq=Hq * 128, lddk=Hk * 128, lddv=Hk * 128)
    need = P.lib().partir_cross_attention_backward_workspace(*z)
    assert need == P.plan_cross_attention_backward(B, Sq, Sk, Hq, Hk)["workspace_bytes"]
    assert cross_bwd(wsb=need, **a) == "PARTIR_E_HIP"
    if need:
        assert cross_bwd(wsb=need - 1, **a) == "PARTIR_E_WORKSPACE"
        assert cross_bwd(**dict(a, wsb=need, ws=ODD)) == "PARTIR_E_LAYOUT"


def test_cross_attention_queries_refuse_what_the_call_refuses():
    bad = ctypes.c_size_t(-1).value
    for z in ((-1, 1, 1, 1, 1, 128), (1, 1, 1, 3, 2, 128), (1, 1, 1, 2, 2, 64), (2 ** 20, 2 ** 20, 1, 1, 1, 128)):
        assert P.lib().partir_cross_attention_workspace(*z) == bad
        assert P.lib().partir_cross_attention_backward_workspace(*z) == bad
        assert P.lib().partir_plan_cross_attention(*z, ctypes.byref(P.PlanInfo())) != 0
    assert name(P.lib().partir_plan_cross_attention(1, 1, 1, 1, 1, 128, None)) == "PARTIR_E_NULL"


def test_cross_attention_binding_checks():
    q, kv = torch.zeros(6, 512, dtype=bf), torch.zeros(100, 512, dtype=bf)
    k, v = kv[:, :256], kv[:, 256:]
    kw = dict(B=2, Sq=3, Sk=50, n_heads=4, n_kv_heads=2)
    call = lambda *a, **o: status(lambda: P.cross_attention(*a, **{**kw, **o}))  # noqa: E731
    assert call(q, k, v) == "PARTIR_E_LAYOUT"                                   # correct, but on the CPU
    assert call(q, kv, v) == "PARTIR_E_SHAPE"
    assert call(q, k, v, Sk=49) == "PARTIR_E_SHAPE"
    assert call(q, k, v, Sk=-50) == "PARTIR_E_SHAPE"
    assert call(q.float(), k, v) == "PARTIR_E_DTYPE"
    assert call(q, k, v.t().contiguous().t()) == "PARTIR_E_LAYOUT"
    assert call(q, k, v, k_lens=torch.zeros(2, dtype=torch.int64)) == "PARTIR_E_DTYPE"
    assert call(q, k, v, k_lens=torch.zeros(3, dtype=torch.int32)) == "PARTIR_E_SHAPE"
    assert call(q, k, v, out=q[:, :256]) == "PARTIR_E_SHAPE"
    lse = torch.zeros(6, 4)
    b = lambda *a, **o: status(lambda: P.cross_attention_backward(*a, **{**kw, **o}))  # noqa: E731
    assert b(q, k, v, q, q, lse) == "PARTIR_E_LAYOUT"
    assert b(q, k, v, q, q, lse[:, :2]) == "PARTIR_E_SHAPE"
    assert b(q, k, v, q, q.float(), lse) == "PARTIR_E_DTYPE"
    assert b(q, k, v, q, q, lse, out=(q, k)) == "PARTIR_E_SHAPE"
    assert b(q, k, v, q, q, lse, out=(q, k, q)) == "PARTIR_E_SHAPE"
    assert status(lambda: P.cross_attention_train(q, k, v, lse=lse.to(bf), **kw)) == "PARTIR_E_DTYPE"


# ---------------------------------------------------------------------------
# the oracle against torch's own routines in fp64
# ---------------------------------------------------------------------------
def test_oracle_against_autograd():
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    B, Sq, Sk, Hq, Hk, lens = 2, 3, 7, 4, 2, [7, 4]
    q, k, v = r(B * Sq, Hq * 128), r(B * Sk, Hk * 128), r(B * Sk, Hk * 128)
    do = r(B * Sq, Hq * 128)
    leaf = [x.clone().requires_grad_() for x in (q, k, v)]
    o = []
    for b in range(B):
        qq = leaf[0][b * Sq:(b + 1) * Sq].reshape(Sq, Hq, 128).transpose(0, 1)
        kk, vv = (x[b * Sk:b * Sk + lens[b]].reshape(-1, Hk, 128).transpose(0, 1).repeat_interleave(Hq // Hk, 0) for x in leaf[1:])
        o.append(torch.nn.functional.scaled_dot_product_attention(qq, kk, vv).transpose(0, 1).reshape(Sq, -1))
    o = torch.cat(o)
    grads = torch.autograd.grad(o, leaf, do)
    ref, _ = OO.cross_attention(q.numpy(), k.numpy(), v.numpy(), B, Sq, Sk, Hq, Hk, lens)
    assert np.abs(ref - o.detach().numpy()).max() < 1e-12
    for a, b in zip(OO.cross_attention_backward(q.numpy(), k.numpy(), v.numpy(), do.numpy(), B, Sq, Sk, Hq, Hk, lens), grads):
        assert np.abs(a - b.numpy()).max() < 1e-12
    # rotary as a complex product, the norm by autograd
    T, H, dh, rd = 5, 3, 16, 12
    x, gain, dy = r(T, H * dh), r(dh), r(T, H * dh)
    pos, f = np.arange(T) * 1000, OO.frequencies(rd)
    w = torch.polar(torch.full((T, 1, rd // 2), 1.5, dtype=torch.float64), torch.from_numpy(pos[:, None] * f)[:, None])
    for inter in (False, True):
        xl, gl = x.clone().requires_grad_(), gain.clone().requires_grad_()
        h = xl.reshape(T, H, dh)
        n = torch.nn.functional.rms_norm(h, (dh,), gl, 1e-4)
        a, b = (n[..., 0:rd:2], n[..., 1:rd:2]) if inter else (n[..., :rd // 2], n[..., rd // 2:rd])
        z = torch.complex(a, b) * w
        rot = torch.stack((z.real, z.imag), -1).flatten(-2) if inter else torch.cat((z.real, z.imag), -1)
        y = torch.cat((rot, n[..., rd:]), -1).reshape(T, -1)
        kw = dict(interleaved=inter, magnitude=1.5)
        assert np.abs(OO.qk_norm_rotary(x.numpy(), gain.numpy(), pos, f, dh, 1e-4, **kw) - y.detach().numpy()).max() < 1e-11
        dx, dg = torch.autograd.grad(y, (xl, gl), dy)
        got = OO.qk_norm_rotary_backward(x.numpy(), gain.numpy(), dy.numpy(), pos, f, dh, 1e-4, **kw)
        assert np.abs(got[0] - dx.numpy()).max() < 1e-11 and np.abs(got[1] - dg.numpy()).max() < 1e-11


def test_without_keys_the_rowsums_have_their_workspace():
    """The dq pass runs alone then and writes them."""
    need = P.lib().partir_cross_attention_backward_workspace(2, 3, 0, 4, 2, 128)
    assert need >= 2 * 3 * 4 * 4
    assert cross_bwd(Sk=0, K=NULL, V=NULL, dK=NULL, dV=NULL, ws=NULL, wsb=0) == "PARTIR_E_WORKSPACE"
    assert P.plan_cross_attention_backward(2, 3, 0, 4, 2)["n_launches"] == 1
    assert P.plan_cross_attention_backward(2, 0, 5, 4, 2)["n_launches"] == 1
    assert P.plan_cross_attention_backward(0, 3, 5, 4, 2)["n_launches"] == 0


# ---------------------------------------------------------------------------
# tensors in each other's place
# ---------------------------------------------------------------------------
def at(x):
    return ctypes.c_void_p(x)


def test_rotary_outputs_are_their_inputs_or_apart():
    apart = dict(Q=at(0x10000), K=at(0x20000), Qo=at(0x30000), Ko=at(0x40000))
    assert rotary(**apart) == "PARTIR_E_HIP"
    assert rotary(**dict(apart, Qo=apart["Q"], Ko=apart["K"])) == "PARTIR_E_HIP"            # in place
    assert rotary(**dict(apart, Qo=apart["Q"], ldqo=264)) == "PARTIR_E_LAYOUT"
    assert rotary(**dict(apart, Qo=apart["Q"], ldqo=264, T=1)) == "PARTIR_E_HIP"            # one row: no stride
    assert rotary(**dict(apart, Qo=apart["K"])) == "PARTIR_E_LAYOUT"
    assert rotary(**dict(apart, Qo=apart["Ko"])) == "PARTIR_E_LAYOUT"
    b = dict(apart, dQo=at(0x50000), dKo=at(0x60000), dQ=at(0x70000), dK=at(0x80000))
    b.pop("Qo"), b.pop("Ko")
    assert bwd(**b) == "PARTIR_E_HIP"
    assert bwd(**dict(b, dQ=b["dQo"], dK=b["dKo"])) == "PARTIR_E_HIP"
    assert bwd(**dict(b, dQ=b["dKo"])) == "PARTIR_E_LAYOUT"
    assert bwd(**dict(b, dQ=b["dQo"], lddq=512)) == "PARTIR_E_LAYOUT"


def test_a_period_below_one_is_refused():
    q, f = torch.zeros(16, 256, dtype=bf), torch.zeros(32, dtype=torch.float64)
    for S in (0, -3):
        assert rotary(S=S) == "PARTIR_E_SHAPE"
    assert status(lambda: P.rotary(q, None, [1.0], d_head=64)) == "PARTIR_E_DTYPE"
    assert status(lambda: P.rotary(q, None, f, d_head=64, positions=[0] * 16)) == "PARTIR_E_NULL"


def test_cross_attention_gradients_are_apart():
    names = ("Q", "K", "V", "O", "dO", "dQ", "dK", "dV")
    p = {n: at(0x10000 * (i + 1)) for i, n in enumerate(names)}
    assert cross_bwd(**p) == "PARTIR_E_HIP"
    for o in ("dQ", "dK", "dV"):
        for i in names:
            if i != o:
                assert cross_bwd(**dict(p, **{o: p[i]})) == "PARTIR_E_LAYOUT", (o, i)


def test_the_norm_is_apart_from_the_tensors():
    assert clip([0x20000], [100], [P.F32], norm=at(0x20000 + 396)) == "PARTIR_E_LAYOUT"
    assert clip([0x20000], [100], [P.F32], norm=at(0x20000 + 400)) == "PARTIR_E_HIP"
    assert clip([0x20000], [100], [P.F32], out=[0x30000], norm=at(0x20000)) == "PARTIR_E_LAYOUT"


def test_division_by_a_product():
    """The high product, addition and shift that the kernels divide by, as
    formed on the host, for divisors and dividends around powers of two."""
    rng = np.random.default_rng(0)
    ds = sorted({d for k in range(31) for d in (2 ** k - 1, 2 ** k, 2 ** k + 1) if d > 0} | set(rng.integers(1, 2 ** 30, 200).tolist()))
    for d in ds:
        l = max(0, int(d - 1).bit_length())
        m = (((1 << 32) * ((1 << l) - d)) // d + 1) & 0xFFFFFFFF
        n = np.unique(np.concatenate([rng.integers(0, 2 ** 31, 200), np.arange(5), 2 ** 31 - 1 - np.arange(5),
                                      np.clip(d * rng.integers(0, max(1, 2 ** 31 // d), 50) + rng.integers(-1, 2, 50), 0, 2 ** 31 - 1)])).astype(np.uint64)
        s = ((np.uint64(m) * n) >> np.uint64(32)) + n
        assert (s < 2 ** 32).all() and ((s >> np.uint64(l)) == n // np.uint64(d)).all(), d


def test_the_output_of_attention_is_its_queries_or_apart():
    assert cross(O=A, K=T2, V=T3) == "PARTIR_E_HIP"                            # in Q's place
    assert cross(O=A, K=T2, V=T3, ldo=1024) == "PARTIR_E_LAYOUT"               # with other rows
    assert cross(O=A, K=T2, V=T3, ldo=1024, B=1, Sq=1) == "PARTIR_E_HIP"       # a single row
    assert cross(O=T2, K=T2) == "PARTIR_E_LAYOUT" and cross(O=T3, V=T3) == "PARTIR_E_LAYOUT"
    assert cross(O=T2, K=T2, V=T2, Sk=0) == "PARTIR_E_HIP"                     # no key is read


def test_a_launch_holds_fewer_than_2_32_threads():
    one = dict(Sq=1, Sk=1, Hq=16, Hk=16, ldq=2048, ldk=2048, ldv=2048, ldo=2048, lddo=2048, lddq=2048, lddk=2048, lddv=2048,
               ws=A, wsb=1 << 60)
    f = lambda B: cross(B=B, **{k: v for k, v in one.items() if k in CROSS})  # noqa: E731
    assert f(2 ** 19 - 1) == "PARTIR_E_HIP" and f(2 ** 19) == "PARTIR_E_SHAPE"
    assert cross_bwd(B=2 ** 19 - 1, **one) == "PARTIR_E_HIP" and cross_bwd(B=2 ** 19, **one) == "PARTIR_E_SHAPE"
    assert cross(**dict(CROSS, B=2 ** 20, Sq=1, Sk=0, Hq=16, Hk=16, ldq=2048, ldo=2048)) == "PARTIR_E_SHAPE"


def test_plans_refuse_no_key_heads():
    for plan in (P.plan_cross_attention, P.plan_cross_attention_backward):
        assert status(lambda: plan(1, 1, 1, 4, 0)) == "PARTIR_E_SHAPE"
        assert plan(1, 1, 1, 4) == plan(1, 1, 1, 4, 4)


def test_gain_gradients_are_apart():
    g = lambda dgq, dgk: name(P.lib().partir_qk_norm_rotary_backward(  # noqa: E731
        T1, T2, T3, T4, NULL, NULL, T5, T6, dgq, dgk, A, NULL, 0, 8, 8, 2, 2, 64, 64, 128, 128, 128, 128, 128, 128, P.BF16, 0,
        1.0, 1e-6, A, 1 << 24, None))
    assert g(T7, T8) == g(T7, NULL) == g(NULL, NULL) == "PARTIR_E_HIP"
    assert g(T7, T7) == "PARTIR_E_LAYOUT"
