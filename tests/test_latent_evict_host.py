"""Host-side checks of the latent-cache and eviction ABIs (no GPU needed): exports, workspace sizes, and the
refusals, with the documented status codes, before the device is touched; pins of their oracles."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from oracle import evict as oe
from oracle import latent as ol
from paper_2609_34653_amd import evict as ev
from paper_2609_34653_amd import latent as la
from paper_2609_34653_amd import omnitide as ot

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p
THETA = ctypes.cast((ctypes.c_double * 64)(*[0.5] * 64), P)
_BAD = (ctypes.c_double * 64)(*[float("inf")] * 64)
BAD_THETA = ctypes.cast(_BAD, P)


@pytest.fixture(scope="module")
def L():
    ev.lib()
    return la.lib()


def fake(i, off=0):
    """A distinct, never-dereferenced device address."""
    return P(0x10_0000_0000 + i * 0x100_0000_0000 + off)


@pytest.mark.parametrize("header,mod", [("omnitide_latent.h", la), ("omnitide_evict.h", ev)])
def test_exports(L, header, mod):
    text = open(os.path.join(ROOT, "include", header)).read()
    names = set(re.findall(r"^(?:int|size_t)\s+(omnitide_\w+)\(", text, re.M))
    assert names == set(mod.EXPORTS) and all(hasattr(L, n) for n in names)


# ------------------------------------------------------------------------------ latent cache

def append(L, **kw):
    a = dict(lat=fake(0), kr=fake(1), q=fake(2), dtype=0, n=10, H=16, R=512, ls=576, ks=576, qs=3200, qh=192,
             pool=fake(3), np=100, P=64, tab=fake(4), mp=20, st=fake(5), ctx=fake(6), S=4, pos=None,
             w=fake(7), eps=1e-6, th=THETA, style=0, mag=1.0, qo=fake(8), qos=9216, qoh=576, status=fake(9))
    a.update(kw)
    return L.omnitide_latent_append(*a.values(), None)


def test_append_refusals(L):
    for k in ("lat", "kr", "pool", "tab", "st", "ctx", "q", "qo"):
        assert append(L, **{k: None}) == ot.E_NULL, k
    assert append(L, dtype=2) == ot.E_DTYPE
    for bad in (dict(R=128), dict(R=576), dict(n=-1), dict(n=(1 << 24) + 1), dict(H=0), dict(H=4097),
                dict(ls=511), dict(ls=513), dict(ks=63), dict(ks=68), dict(qs=2936), dict(qh=60), dict(qh=68),
                dict(qos=8000), dict(qoh=63), dict(ls=1 << 32), dict(P=8), dict(P=512), dict(S=0), dict(mp=0),
                dict(np=0), dict(style=2), dict(mag=float("nan")), dict(th=BAD_THETA), dict(eps=-1.0),
                dict(eps=float("inf")), dict(lat=fake(0, 8)), dict(kr=fake(1, 4)), dict(qo=fake(8, 2)),
                dict(w=fake(7, 8)), dict(pool=fake(3, 8)), dict(mp=(1 << 24) + 1)):
        assert append(L, **bad) == ot.E_SHAPE, bad
    for bad in (dict(pool=fake(0)), dict(pool=fake(2)), dict(pool=fake(4)), dict(qo=fake(3)),
                dict(qo=fake(2, 16)), dict(qo=fake(2), qos=3200, qoh=192, dtype=1, ls=576), dict(qo=fake(0)),
                dict(qo=fake(2), qos=3200, qoh=64, qh=192), dict(status=fake(6)), dict(status=fake(2)),
                dict(qo=fake(7))):
        assert append(L, **bad) == ot.E_ALIAS, bad
    assert append(L, n=0) == ot.OK
    assert append(L, n=0, lat=None, kr=None, q=None, qo=None, H=0) == ot.OK


def rows(L, **kw):
    a = dict(pool=fake(0), np=100, P=64, W=576, tab=fake(1), mp=20, st=fake(2), ctx=fake(3), S=4, n=50,
             out=fake(4), os=576, status=fake(5))
    a.update(kw)
    return L.omnitide_paged_rows(*a.values(), None)


def test_rows_refusals(L):
    for k in ("pool", "tab", "st", "ctx", "out"):
        assert rows(L, **{k: None}) == ot.E_NULL, k
    for bad in (dict(W=4), dict(W=4104), dict(W=20), dict(os=568), dict(os=580), dict(n=-1),
                dict(n=(1 << 27) + 1), dict(P=12), dict(np=0), dict(S=0), dict(out=fake(4, 8))):
        assert rows(L, **bad) == ot.E_SHAPE, bad
    for bad in (dict(out=fake(0)), dict(out=fake(1)), dict(out=fake(2)), dict(out=fake(3)), dict(status=fake(4)),
                dict(status=fake(0))):
        assert rows(L, **bad) == ot.E_ALIAS, bad
    assert rows(L, n=0, out=None) == ot.OK


def decode(L, **kw):
    a = dict(q=fake(0), pool=fake(1), np=100, P=64, tab=fake(2), mp=20, ctx=fake(3), S=4, nq=1, H=16, R=512,
             scale=0.1, out=fake(4), od=0, ws=fake(5), wb=1 << 30, status=fake(6))
    a.update(kw)
    return L.omnitide_latent_decode_attn(*a.values(), None)


def test_decode_refusals(L):
    for k in ("q", "pool", "tab", "ctx", "out"):
        assert decode(L, **{k: None}) == ot.E_NULL, k
    assert decode(L, od=2) == ot.E_DTYPE
    for bad in (dict(R=64), dict(H=0), dict(nq=0), dict(H=1025), dict(nq=9, H=128), dict(nq=1 << 30, H=4),
                dict(S=1025), dict(S=0), dict(scale=float("nan")), dict(scale=2e30), dict(P=4), dict(mp=0),
                dict(S=1024, mp=1 << 19, P=64), dict(q=fake(0, 8)), dict(ws=fake(5, 8))):
        assert decode(L, **bad) == ot.E_SHAPE, bad
    assert decode(L, ws=None) == ot.E_WORKSPACE and decode(L, wb=1000) == ot.E_WORKSPACE
    for bad in (dict(out=fake(0)), dict(out=fake(1)), dict(ws=fake(1)), dict(ws=fake(4)), dict(ws=fake(3)),
                dict(status=fake(2)), dict(out=fake(2))):
        assert decode(L, **bad) == ot.E_ALIAS, bad


def test_decode_workspace(L):
    size = la.omnitide_latent_decode_workspace_bytes
    base = size(1, 1, 64, 16, 512)
    assert 0 < base < 1 << 26
    assert size(1024, 1, 1 << 24, 16, 512) == base           # whatever the batch
    assert decode(L, wb=base - 1) == ot.E_WORKSPACE
    last = 0
    for m in (1, 32, 33, 64, 65, 128, 129, 300, 512, 1024):
        assert size(1, 1, 64, m, 512) <= 1 << 28
        last = max(last, size(1, 1, 64, m, 512))
    for bad in ((0, 1, 64, 16, 512), (1025, 1, 64, 16, 512), (1, 0, 64, 16, 512), (1, 1, 0, 16, 512),
                (1, 2, 64, 513, 512), (1, 1, 64, 16, 100)):
        assert size(*bad) == 0


def test_decode_workspace_never_falls():
    size = la.omnitide_latent_decode_workspace_bytes
    for R in (256, 512):
        got = [size(1, 1, 64, m, R) for m in range(1, 1025)]
        assert got == sorted(got) and got[0] > 0
        assert all(size(1, nq, 64, 16, R) == got[16 * nq - 1] for nq in range(1, 65))
    assert size(1, 1, 64, 16, 256) < size(1, 1, 64, 16, 512)


def chunk(L, **kw):
    a = dict(q=fake(0), k=fake(1), v=fake(1, 256), kr=fake(2), ks=4096, kh=256, vs=4096, vh=256, es=576,
             st=fake(3), kst=fake(4), S=4, n=50, N=900, H=16, d=128, scale=0.1, out=fake(5), od=0,
             ws=fake(6), wb=1 << 30, status=fake(7))
    a.update(kw)
    return L.omnitide_latent_chunk_attn(*a.values(), None)


def test_chunk_refusals(L):
    for k in ("q", "k", "v", "kr", "st", "kst", "out"):
        assert chunk(L, **{k: None}) == ot.E_NULL, k
    assert chunk(L, od=-1) == ot.E_DTYPE
    for bad in (dict(d=96), dict(H=0), dict(H=4097), dict(S=0), dict(S=1025), dict(n=-1), dict(N=-1),
                dict(N=(1 << 27) + 1), dict(N=1 << 27, H=256), dict(n=1 << 24, H=17), dict(kh=120), dict(kh=132),
                dict(ks=3900), dict(vs=3900), dict(vh=100), dict(es=60), dict(es=68), dict(ks=1 << 25),
                dict(scale=float("inf")), dict(k=fake(1, 8)), dict(v=fake(1, 260)), dict(kr=fake(2, 2))):
        assert chunk(L, **bad) == ot.E_SHAPE, bad
    assert chunk(L, ws=None) == ot.E_WORKSPACE and chunk(L, wb=1000) == ot.E_WORKSPACE
    for bad in (dict(out=fake(0)), dict(out=fake(1)), dict(out=fake(2)), dict(ws=fake(2)), dict(ws=fake(5)),
                dict(status=fake(3)), dict(ws=fake(4))):
        assert chunk(L, **bad) == ot.E_ALIAS, bad
    assert chunk(L, n=0, q=None, k=None, v=None, kr=None, out=None, ws=None) == ot.OK


def test_chunk_of_padding_alone():
    """No rows at all is a call, with a workspace as large as any."""
    size = la.omnitide_latent_chunk_attn_workspace_bytes
    assert size(5, 2, 0, 4, 64) == size(5, 2, 100, 4, 64) > 0
    assert size(5, 2, -1, 4, 64) == 0


# --------------------------------------------------------------------------------- eviction

def weights(L, **kw):
    a = dict(q=fake(0), k=fake(1), np=100, P=64, tab=fake(2), mp=20, st=fake(3), ctx=fake(4), S=4, n=50, mq=20,
             Hq=32, Hkv=8, d=128, scale=0.1, decay=0.9, seen=fake(5), wi=fake(6), wo=fake(7), stride=1280,
             ws=fake(8), wb=1 << 36, status=fake(9))
    a.update(kw)
    return L.omnitide_paged_attn_weights(*a.values(), None)


def test_weights_refusals(L):
    for k in ("q", "k", "tab", "st", "ctx", "wo"):
        assert weights(L, **{k: None}) == ot.E_NULL, k
    for bad in (dict(d=96), dict(d=576), dict(d=320), dict(Hq=33), dict(Hq=4), dict(Hkv=0), dict(n=-1),
                dict(n=(1 << 24) + 1), dict(mq=0), dict(S=0), dict(S=1025), dict(P=24), dict(stride=1279),
                dict(stride=1 << 32), dict(decay=-0.5), dict(decay=float("nan")), dict(scale=float("nan")),
                dict(n=1 << 24, Hq=256), dict(q=fake(0, 8)), dict(wo=fake(7, 2)), dict(wi=fake(6, 1)),
                dict(ws=fake(8, 4)), dict(d=576, Hkv=1, Hq=4097)):
        assert weights(L, **bad) == ot.E_SHAPE, bad
    assert weights(L, ws=None) == ot.E_WORKSPACE and weights(L, wb=1000) == ot.E_WORKSPACE
    for bad in (dict(wo=fake(0)), dict(wo=fake(1)), dict(wo=fake(6, 16)), dict(ws=fake(6)), dict(ws=fake(7)),
                dict(wo=fake(5)), dict(status=fake(6)), dict(status=fake(4)), dict(ws=fake(2))):
        assert weights(L, **bad) == ot.E_ALIAS, bad
    assert weights(L, n=0, q=None, ws=None) == ot.OK


def test_weights_workspace():
    size = ev.omnitide_paged_attn_weights_workspace_bytes
    base = size(50, 4, 1280, 20, 32, 8, 128)
    assert base > 0
    for bigger in ((51, 4, 1280, 20, 32, 8, 128), (50, 5, 1280, 20, 32, 8, 128),
                   (50, 4, 1344, 20, 32, 8, 128), (5000, 40, 9000, 4000, 32, 8, 128)):
        assert size(*bigger) >= base
    for bad in ((0, 4, 1280, 20, 32, 8, 128), (50, 0, 1280, 20, 32, 8, 128), (50, 4, 0, 20, 32, 8, 128),
                (50, 4, 1280, 0, 32, 8, 128), (50, 4, 1280, 20, 32, 8, 100), (50, 4, 1280, 20, 32, 5, 128)):
        assert size(*bad) == 0


def test_weights_workspace_of_mixed_batches():
    """Partial sums are those of the tokens that there are, not of the longest chunk for every sequence; beside them
    at most the 2^30 bytes of scores that calls of few tokens keep."""
    size = ev.omnitide_paged_attn_weights_workspace_bytes
    # one chunk of 4,096 beside 1,023 single tokens: 16 + 1,023 row chunks of 8 heads of 16,384 sums
    assert size(5119, 1024, 16384, 4096, 32, 8, 128) < max(1 << 30, (16 + 1023 + 3) * 8 * 16384 * 4) + (1 << 25)
    assert size(2463, 64, 131072, 2400, 32, 8, 128) < max(1 << 30, (9 + 64 + 1) * 8 * 131072 * 4) + (1 << 25)
    # more query heads for a KV head than the way of few takes: the partial sums alone
    assert size(5119, 1024, 16384, 4096, 264, 4, 64) < (330 + 1024) * 4 * 16384 * 4 + (1 << 28)


@pytest.mark.parametrize("Hq,Hkv,d", [(32, 8, 128), (4, 1, 64), (16, 1, 576), (128, 1, 576), (65, 65, 64), (256, 2, 64)])
def test_weights_workspace_never_falls(Hq, Hkv, d):
    """In any of its lengths: a workspace for the largest calls serves every one of them, whichever way it goes."""
    size = ev.omnitide_paged_attn_weights_workspace_bytes
    T, S, M, Q = [1, 24, 192, 193, 665, 5000], [1, 7, 24, 300], [16, 256, 20096, 131072], [1, 2, 4, 8, 9, 64, 65, 4000]
    for a in T:
        for b in S:
            for c in M:
                for q in Q:
                    base = size(a, b, c, q, Hq, Hkv, d)
                    for k, more in enumerate((T, S, M, Q)):
                        at = [a, b, c, q]
                        i = more.index(at[k])
                        if i + 1 < len(more):
                            at[k] = more[i + 1]
                            assert size(*at, Hq, Hkv, d) >= base, (a, b, c, q, at)


def plan(L, **kw):
    a = dict(w=fake(0), ws=2000, ctx=fake(1), S=4, mc=1500, high=1000, budget=900, sink=4, recent=100,
             src=fake(2), ss=1000, new=fake(3), wo=fake(4), wos=1000, work=fake(5), wb=1 << 34, status=fake(6))
    a.update(kw)
    return L.omnitide_evict_plan(*a.values(), None)


def test_plan_refusals(L):
    for k in ("w", "ctx", "src", "new"):
        assert plan(L, **{k: None}) == ot.E_NULL, k
    for bad in (dict(S=0), dict(S=65536), dict(mc=0), dict(mc=(1 << 24) + 1, ws=1 << 25), dict(budget=0),
                dict(budget=1001), dict(sink=-1), dict(recent=-1), dict(sink=500, recent=401),
                dict(sink=1 << 30, recent=1 << 30, budget=1000), dict(ws=1499), dict(ss=999), dict(wos=999),
                dict(high=(1 << 24) + 1, ss=1 << 25, wos=1 << 25), dict(w=fake(0, 2)), dict(src=fake(2, 1)),
                dict(wo=fake(4, 2)), dict(work=fake(5, 8))):
        assert plan(L, **bad) == ot.E_SHAPE, bad
    for bad in (dict(src=fake(0)), dict(wo=fake(0)), dict(new=fake(1)), dict(new=fake(2)), dict(wo=fake(2)),
                dict(status=fake(1)), dict(status=fake(0))):
        assert plan(L, **bad) == ot.E_ALIAS, bad


def move(L, **kw):
    a = dict(k=fake(0), v=fake(1), np=100, P=64, H=8, d=128, tab=fake(2), mp=20, ctx=fake(3), dst=fake(4), dmp=10,
             src=fake(5), ss=600, new=fake(6), S=4, th=THETA, R=128, style=0, off=0, status=fake(7))
    a.update(kw)
    return L.omnitide_paged_compact(*a.values(), None)


def test_plan_workspace_never_falls():
    from paper_2609_34653_amd import evict as ev
    sizes = [1, 100, 4096, 4097, 8192, 16384, 16385, 70000, 131072, 131073, 140000, 262144, 262145, 300000,
             1 << 20, 1 << 24]
    for n_seq in (1, 3, 200):
        got = [ev.omnitide_evict_plan_workspace_bytes(n_seq, n) for n in sizes]
        assert got == sorted(got) and got[5] == 0 and got[6] > 0
        assert got[-1] <= ev.omnitide_evict_plan_workspace_bytes(n_seq + 1, sizes[-1])


def test_compact_refusals(L):
    for k in ("k", "tab", "ctx", "dst", "src", "new", "th"):
        assert move(L, **{k: None}) == ot.E_NULL, k
    for bad in (dict(H=0), dict(d=0), dict(H=33), dict(H=1, d=4104), dict(H=3, d=20, R=0), dict(P=10), dict(np=0),
                dict(mp=0), dict(dmp=0), dict(S=0), dict(S=65536, mp=1, dmp=1), dict(ss=0), dict(ss=1 << 32),
                dict(R=4), dict(R=20), dict(R=136, d=256, H=2), dict(off=8), dict(off=4, R=64), dict(off=-8, R=64),
                dict(style=2), dict(th=BAD_THETA), dict(k=fake(0, 8)), dict(v=fake(1, 8)),
                dict(H=2, d=12, R=8), dict(H=1 << 17, d=1 << 17)):
        assert move(L, **bad) == ot.E_SHAPE, bad
    for bad in (dict(v=fake(0)), dict(k=fake(2)), dict(k=fake(4)), dict(v=fake(5)), dict(status=fake(6)),
                dict(k=fake(3)), dict(status=fake(1))):
        assert move(L, **bad) == ot.E_ALIAS, bad


# ------------------------------------------------------------------------------ the binding

def test_bindings_refuse_what_is_no_device_tensor():
    x = torch.zeros(4, 512)
    for call in (lambda: la.omnitide_latent_append(x, x, x, x, x, x), lambda: la.omnitide_paged_rows(x, x, x, x, x),
                 lambda: la.omnitide_latent_decode_attn(x, x, x, x, 1.0, x),
                 lambda: la.omnitide_latent_chunk_attn(x, x, x, x, x, x, 1.0, x),
                 lambda: ev.omnitide_paged_attn_weights(x, x, x, x, x, 1, 1.0, x),
                 lambda: ev.omnitide_evict_plan(x, x, 1, 1, 0, 0, x, x),
                 lambda: ev.omnitide_paged_compact(x, None, x, x, x, x, x)):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    with pytest.raises(TypeError):
        la.omnitide_latent_append(1, x, x, x, x, x)


# ------------------------------------------------------------------------------ oracle pins

def test_absorbed_and_expanded_attention_agree():
    """(A c) . n = c . (A^T n), and sums of B c are B times sums of c."""
    g = np.random.default_rng(1)
    n, m, H, R, d, E = 23, 5, 3, 12, 6, 4
    c, e = g.standard_normal((n, R)), g.standard_normal((n, E))
    a, b = g.standard_normal((H, d, R)), g.standard_normal((H, d, R))
    q = g.standard_normal((m, H, d + E))
    want, _ = ol.expanded_attention(q, np.einsum("hdr,nr->nhd", a, c), np.einsum("hdr,nr->nhd", b, c), e, 0.3)
    ql = np.concatenate([np.einsum("hdr,mhd->mhr", a, q[..., :d]), q[..., d:]], -1)
    lat, _ = ol.absorbed_attention(ql, np.concatenate([c, e], 1), R, 0.3)
    assert np.allclose(np.einsum("hdr,mhr->mhd", b, lat), want, atol=1e-12)
    # one row: its value
    one, _ = ol.absorbed_attention(ql[:1], np.concatenate([c, e], 1)[:1], R, 0.3)
    assert np.allclose(one, c[:1][None])


def test_row_weights_sum_to_the_probabilities():
    g = np.random.default_rng(2)
    q, k = g.standard_normal((7, 6, 8)), g.standard_normal((19, 2, 8))
    w = oe.row_weights(q, k, 0.4)
    assert np.isclose(w.sum(), 7 * 6) and (w > 0).all()
    # the last row is seen by the last token alone
    x = 0.4 * np.einsum("hd,nhd->hn", q[6], np.repeat(k, 3, 1))
    p = np.exp(x) / np.exp(x).sum(1, keepdims=True)
    assert np.isclose(w[18], p[:, 18].sum())
    assert np.allclose(oe.row_weights(q, np.zeros_like(k), 1.0)[:13], 6 * sum(1 / (13 + i) for i in range(7)))


def test_plan_by_hand():
    w = [5.0, 0.0, 3.0, 3.0, float("nan"), 1.0, -0.0, 2.0, 0.5]
    assert oe.plan(w, 9, 4, 1, 1) == list(range(9))
    assert oe.plan(w, 8, 4, 1, 1) == [0, 2, 3, 8]
    assert oe.plan(w, 8, 3, 1, 1) == [0, 2, 8]               # a tie: the lower row
    assert oe.plan(w, 8, 8, 1, 1) == [0, 1, 2, 3, 5, 6, 7, 8]
    assert oe.plan(w, 8, 7, 0, 0) == [0, 1, 2, 3, 5, 7, 8]   # 0 and -0 alike: the lower row
    assert oe.plan([float("nan")] * 4, 3, 2, 0, 0) == [0, 1]
