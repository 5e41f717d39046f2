"""Refusals of masked attention (no GPU needed): the C ABI's checks, with pointers
that are never dereferenced, and the binding's, with CPU tensors; workspaces and
plans."""
import ctypes

import pytest
import torch

from paper_2401_11202_amd import partir as P

NULL, ODD, A = None, 0x900004, 0x10000
T = [ctypes.c_void_p(0x1000000 * i) for i in range(1, 12)]     # tensors apart
bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
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


def mask_of(kw):
    m = P.AttentionMask(1)
    for k in [k for k in kw if hasattr(m, k)]:
        setattr(m, k, kw.pop(k))
    return m


FWD = dict(Q=T[0], K=T[1], V=T[2], O=T[3], lse=T[4], B=2, Sq=30, Sk=500, Hq=4, Hk=2, dh=128, ldq=512, ldk=256, ldv=256, ldo=512, mask=1,
           scale=0.0, ws=T[9], wsb=1 << 30)
BWD = dict(Q=T[0], K=T[1], V=T[2], O=T[3], dO=T[4], lse=T[5], dQ=T[6], dK=T[7], dV=T[8], B=2, Sq=30, Sk=500, Hq=4, Hk=2, dh=128, ldq=512,
           ldk=256, ldv=256, ldo=512, lddo=512, lddq=512, lddk=256, lddv=256, mask=1, scale=0.0, ws=T[9], wsb=1 << 30)


def call(fn, base, kw, drop=()):
    kw = dict(kw)
    m = mask_of(kw)
    a = dict(base, **kw)
    if a["mask"] is not NULL:
        a["mask"] = m
    return P.STATUS[getattr(P.lib(), fn)(*(a[k] for k in base if k not in drop), None)]


def train(**kw):
    return call("partir_masked_attention_train", FWD, kw)


def infer(**kw):
    return call("partir_masked_attention", FWD, kw, drop=("lse",))


def bwd(**kw):
    return call("partir_masked_attention_backward", BWD, kw)


BOTH = [
    (dict(mask=NULL), "PARTIR_E_NULL"), (dict(Q=NULL), "PARTIR_E_NULL"), (dict(K=NULL), "PARTIR_E_NULL"), (dict(V=NULL), "PARTIR_E_NULL"),
    (dict(O=NULL), "PARTIR_E_NULL"), (dict(lse=NULL), "PARTIR_E_NULL"), (dict(q_docs=A), "PARTIR_E_NULL"), (dict(k_docs=A), "PARTIR_E_NULL"),
    (dict(ws=NULL), "PARTIR_E_NULL"), (dict(B=-1), "PARTIR_E_SHAPE"), (dict(Sq=2 ** 31), "PARTIR_E_SHAPE"), (dict(Sk=-1), "PARTIR_E_SHAPE"),
    (dict(dh=64), "PARTIR_E_SHAPE"), (dict(Hq=0), "PARTIR_E_SHAPE"), (dict(Hk=8), "PARTIR_E_SHAPE"), (dict(Hk=3), "PARTIR_E_DIVISIBILITY"),
    (dict(ldq=2 ** 25), "PARTIR_E_SHAPE"), (dict(ldq=504), "PARTIR_E_LAYOUT"), (dict(ldk=260), "PARTIR_E_LAYOUT"),
    (dict(Q=ctypes.c_void_p(ODD)), "PARTIR_E_LAYOUT"), (dict(lse=ctypes.c_void_p(0x900002)), "PARTIR_E_LAYOUT"),
    (dict(ws=ctypes.c_void_p(ODD)), "PARTIR_E_LAYOUT"), (dict(wsb=100), "PARTIR_E_WORKSPACE"),
    (dict(slopes=0x10002), "PARTIR_E_LAYOUT"), (dict(k_lens=0x10001), "PARTIR_E_LAYOUT"), (dict(q_lens=0x10002), "PARTIR_E_LAYOUT"),
    (dict(q_starts=0x10002), "PARTIR_E_LAYOUT"), (dict(prefix_lens=0x10002), "PARTIR_E_LAYOUT"),
    (dict(q_docs=0x10002, k_docs=A), "PARTIR_E_LAYOUT"), (dict(q_docs=A, k_docs=0x10002), "PARTIR_E_LAYOUT"),
    (dict(cap=-1.0), "PARTIR_E_UNSUPPORTED"), (dict(cap=nan), "PARTIR_E_UNSUPPORTED"), (dict(cap=1025.0), "PARTIR_E_UNSUPPORTED"),
    (dict(cap=1e-4), "PARTIR_E_UNSUPPORTED"), (dict(cap=1.0, scale=1e30), "PARTIR_E_UNSUPPORTED"), (dict(scale=nan), "PARTIR_E_UNSUPPORTED"),
    (dict(prefix_lens=A, causal=0), "PARTIR_E_UNSUPPORTED")]


@pytest.mark.parametrize("kw,want", BOTH + [
    (dict(O=T[1]), "PARTIR_E_LAYOUT"), (dict(O=T[0], ldo=520), "PARTIR_E_LAYOUT"), (dict(O=at(T[0], 1024)), "PARTIR_E_LAYOUT"),
    (dict(O=at(T[2], 512 * 999)), "PARTIR_E_LAYOUT"), (dict(lse=T[0]), "PARTIR_E_LAYOUT"), (dict(lse=T[3]), "PARTIR_E_LAYOUT")])
def test_forward_refusals(kw, want):
    assert train(**kw) == want
    if "lse" not in kw:
        assert infer(**kw) == want


ACCEPT = [dict(), dict(causal=0), dict(cap=50.0), dict(cap=1024.0, slopes=A), dict(k_lens=A, q_lens=A, q_starts=A, prefix_lens=A),
          dict(q_docs=A, k_docs=A), dict(q_docs=A, k_docs=A, causal=0), dict(scale=0.1), dict(ldq=520, ldk=264)]


@pytest.mark.parametrize("kw", ACCEPT + [dict(O=T[0]), dict(O=at(T[1], 512), ldk=768, ldv=768, ldo=768)])
def test_forward_accepts(kw):
    assert train(**kw) == "PARTIR_E_HIP" and infer(**kw) == "PARTIR_E_HIP"     # reached the launch, which is forced to fail


@pytest.mark.parametrize("kw,want", BOTH + [
    (dict(dO=NULL), "PARTIR_E_NULL"), (dict(dQ=NULL), "PARTIR_E_NULL"), (dict(dK=NULL), "PARTIR_E_NULL"), (dict(dV=NULL), "PARTIR_E_NULL"),
    (dict(dQ=T[0]), "PARTIR_E_LAYOUT"), (dict(dQ=T[4]), "PARTIR_E_LAYOUT"), (dict(dK=T[8]), "PARTIR_E_LAYOUT"), (dict(dV=T[2]), "PARTIR_E_LAYOUT"),
    (dict(dK=at(T[6], 512)), "PARTIR_E_LAYOUT"), (dict(dV=T[5]), "PARTIR_E_LAYOUT"), (dict(lddv=252), "PARTIR_E_LAYOUT")])
def test_backward_refusals(kw, want):
    assert bwd(**kw) == want


@pytest.mark.parametrize("kw", ACCEPT + [dict(dK=at(T[6], 1024), dV=at(T[6], 1536), lddq=1024, lddk=1024, lddv=1024)])
def test_backward_accepts(kw):
    assert bwd(**kw) == "PARTIR_E_HIP"


ARRAYS = ("slopes", "k_lens", "q_lens", "q_starts", "prefix_lens", "q_docs", "k_docs")


@pytest.mark.parametrize("name", ARRAYS)
@pytest.mark.parametrize("out", ["O", "lse", "dQ", "dK", "dV"])
def test_outputs_are_apart_from_the_masks_arrays(name, out):
    """Behind the last array's end, and before the first, an output may lie."""
    m = dict({n: A for n in ARRAYS if "docs" in n} if "docs" in name else {}, causal=1)
    size = 4 * {"slopes": 4, "q_docs": 60, "k_docs": 1000}.get(name, 2)
    fwd = out in ("O", "lse")
    p = dict(FWD if fwd else BWD)[out]
    go = train if fwd else bwd
    for off, want in ((0, "PARTIR_E_LAYOUT"), (4 - size, "PARTIR_E_LAYOUT"), (-size, "PARTIR_E_HIP")):
        assert go(**{**m, name: at(p, off)}) == want, off


def test_nothing_to_do():
    for empty in (dict(B=0), dict(Sq=0)):
        assert infer(Q=NULL, K=NULL, V=NULL, O=NULL, ws=NULL, wsb=0, **empty) == "PARTIR_OK"
    n = {k: NULL for k in ("Q", "K", "V", "O", "dO", "lse", "dQ", "dK", "dV", "ws")}
    assert infer(Sq=0, k_docs=A, Q=NULL, O=NULL) == "PARTIR_OK"       # the array of no queries is NULL
    assert infer(Sk=0, q_docs=A, K=NULL, V=NULL, ws=NULL, wsb=0) == "PARTIR_E_HIP"
    assert bwd(B=0, wsb=0, **n) == "PARTIR_OK" and bwd(Sq=0, Sk=0, wsb=0, **n) == "PARTIR_OK"


SIZES = [(1, 1, 1, 1, 1), (16, 1, 4099, 32, 8), (1, 509, 8192, 32, 8), (2, 4096, 4096, 32, 8), (3, 333, 333, 12, 4), (1, 0, 50, 2, 1), (2, 50, 0, 2, 2),
         (1, 1, 2 ** 20, 1, 1), (300, 40, 40, 4, 4)]


@pytest.mark.parametrize("B,Sq,Sk,Hq,Hk", SIZES)
@pytest.mark.parametrize("docs", [False, True])
@pytest.mark.parametrize("causal", [0, 1])
def test_workspaces_are_what_the_calls_need(B, Sq, Sk, Hq, Hk, docs, causal):
    m = dict(causal=causal, **(dict(q_docs=A, k_docs=A) if docs else {}))
    far = [ctypes.c_void_p(i << 50) for i in range(1, 12)]
    dims = dict(B=B, Sq=Sq, Sk=Sk, Hq=Hq, Hk=Hk, ldq=Hq * 128, ldk=Hk * 128, ldv=Hk * 128, ldo=Hq * 128)
    L = P.lib()
    need = L.partir_masked_attention_workspace(B, Sq, Sk, Hq, Hk, 128, mask_of(dict(m)))
    a = dict(dims, Q=far[0], K=far[1], V=far[2], O=far[3], lse=far[4], ws=far[9], **m)
    launches = P.plan_masked_attention(B, Sq, Sk, Hq, Hk, causal=causal, docs=docs)
    assert launches["workspace_bytes"] == need
    assert train(wsb=need, **a) == ("PARTIR_E_HIP" if launches["n_launches"] else "PARTIR_OK")
    if need:
        assert train(wsb=need - 1, **a) == "PARTIR_E_WORKSPACE"
    need = L.partir_masked_attention_backward_workspace(B, Sq, Sk, Hq, Hk, 128, mask_of(dict(m)))
    a = dict(dims, Q=far[0], K=far[1], V=far[2], O=far[3], dO=far[4], lse=far[5], dQ=far[6], dK=far[7], dV=far[8], ws=far[9],
             lddo=Hq * 128, lddq=Hq * 128, lddk=Hk * 128, lddv=Hk * 128, **m)
    launches = P.plan_masked_attention_backward(B, Sq, Sk, Hq, Hk, causal=causal, docs=docs)
    assert launches["workspace_bytes"] == need
    assert bwd(wsb=need, **a) == ("PARTIR_E_HIP" if launches["n_launches"] else "PARTIR_OK")
    if need:
        assert bwd(wsb=need - 1, **a) == "PARTIR_E_WORKSPACE"


def test_queries_of_bad_sizes():
    bad, m = ctypes.c_size_t(-1).value, P.AttentionMask(1)
    for fn in ("partir_masked_attention_workspace", "partir_masked_attention_backward_workspace"):
        assert getattr(P.lib(), fn)(-1, 1, 1, 1, 1, 128, m) == bad and getattr(P.lib(), fn)(1, 1, 1, 3, 2, 128, m) == bad
        assert getattr(P.lib(), fn)(1, 1, 1, 1, 1, 128, None) == bad
    assert status(lambda: P.plan_masked_attention(1, 1, 1, 3, 2)) == "PARTIR_E_DIVISIBILITY"


def test_binding_checks():
    z = lambda *s, dtype=bf: torch.zeros(s, dtype=dtype)  # noqa: E731
    q, k = z(6, 512), z(10, 256)
    kw = dict(B=2, Sq=3, Sk=5, n_heads=4, n_kv_heads=2)
    call = lambda *a, **m: status(lambda: P.masked_attention(*a, **{**kw, **m}))  # noqa: E731
    assert call(q, k, k) == "PARTIR_E_LAYOUT"                                   # all correct, but on the CPU
    assert call(q, k, z(9, 256)) == "PARTIR_E_SHAPE" and call(q.float(), k, k) == "PARTIR_E_DTYPE" and call(q, None, k) == "PARTIR_E_NULL"
    assert call(q, k, k, slopes=z(3, dtype=f32)) == "PARTIR_E_SHAPE" and call(q, k, k, slopes=z(4)) == "PARTIR_E_DTYPE"
    for n in ("k_lens", "q_lens", "q_starts", "prefix_lens"):
        assert call(q, k, k, **{n: z(3, dtype=i32)}) == "PARTIR_E_SHAPE", n
        assert call(q, k, k, **{n: z(2, dtype=torch.int64)}) == "PARTIR_E_DTYPE", n
    assert call(q, k, k, q_docs=z(6, dtype=i32), k_docs=z(6, dtype=i32)) == "PARTIR_E_SHAPE"
    assert call(q, k, k, q_docs=z(6, dtype=torch.int64), k_docs=z(10, dtype=i32)) == "PARTIR_E_DTYPE"
    assert call(q, k, k, out=q.float()) == "PARTIR_E_DTYPE" and call(q, k, k, out=k) == "PARTIR_E_SHAPE"
    assert status(lambda: P.masked_attention_train(q, k, k, lse=z(6, 3, dtype=f32), **kw)) == "PARTIR_E_SHAPE"
    b = lambda *a, **m: status(lambda: P.masked_attention_backward(*a, **{**kw, **m}))  # noqa: E731
    lse = z(6, 4, dtype=f32)
    assert b(q, k, k, q, q, lse) == "PARTIR_E_LAYOUT"
    assert b(q, k, k, q, k, lse) == "PARTIR_E_SHAPE" and b(q, k, k, q, q, None) == "PARTIR_E_NULL"
    assert b(q, k, k, q, q, lse, out=(q, k)) == "PARTIR_E_SHAPE"
