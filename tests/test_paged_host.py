"""Host-side checks of the paged-cache ABI (no GPU needed): exports, the frequency table, and the
refusals, with the documented status codes, before the device is touched."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from oracle import paged as op
from paper_2609_34653_amd import omnitide as ot
from paper_2609_34653_amd import paged as pg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p


@pytest.fixture(scope="module")
def L():
    return pg.lib()


def fake(i, off=0):
    """A distinct, never-dereferenced device address."""
    return P(0x10_0000_0000 + i * 0x100_0000_0000 + off)


def test_exports(L):
    text = open(os.path.join(ROOT, "include", "omnitide_paged.h")).read()
    names = set(re.findall(r"^(?:int|size_t)\s+(omnitide_\w+)\(", text, re.M))
    assert names == set(pg.EXPORTS) and all(hasattr(L, n) for n in names)
    assert "page" in ot.status_string(pg.E_PAGES)


# ----------------------------------------------------------------------------- frequencies

@pytest.mark.parametrize("R", [2, 16, 64, 128])
@pytest.mark.parametrize("name,mode", [("plain", pg.ROPE_PLAIN), ("linear", pg.ROPE_LINEAR),
                                       ("base", pg.ROPE_BASE), ("ramp", pg.ROPE_RAMP)])
def test_rope_thetas(R, name, mode):
    if name == "base" and R == 2:
        return
    got = pg.omnitide_rope_thetas(1.0e6, R, mode, 8.0, 32768.0, 1.0, 32.0)
    want = op.scaled_thetas(1.0e6, R, name, 8.0, 32768.0, 1.0, 32.0)
    # pow and the oracle's exp of a product: a few units in the last place times ln(1e6)
    assert np.allclose(got.numpy(), want, rtol=1e-13, atol=0.0)


@pytest.mark.parametrize("bad", [dict(rope_dims=0), dict(rope_dims=3), dict(rope_dims=130),
                                 dict(rope_base=1.0), dict(rope_base=float("inf")),
                                 dict(scaling=4), dict(scaling=-1), dict(scaling=1, factor=0.5),
                                 dict(scaling=1, factor=float("nan")),
                                 dict(scaling=2, rope_dims=2, factor=2.0),
                                 dict(scaling=3, factor=2.0, original_len=0.0),
                                 dict(scaling=3, factor=2.0, original_len=9.0, ramp_slow=2.0,
                                      ramp_fast=2.0)])
def test_rope_thetas_refusals(bad):
    a = dict(rope_base=10000.0, rope_dims=64)
    a.update(bad)
    with pytest.raises(pg.OmnitideError) as e:
        pg.omnitide_rope_thetas(**a)
    assert e.value.code in (ot.E_SHAPE, ot.E_NULL)


@pytest.mark.parametrize("dims", [130, 256, 1 << 30, (1 << 32) + 64, 7, 0, -2])
def test_rope_dims_refused_as_a_size(dims):
    with pytest.raises(pg.OmnitideError) as e:
        pg.omnitide_rope_thetas(1.0e4, dims)
    assert e.value.code == ot.E_SHAPE


# -------------------------------------------------------------------------------- refusals

THETA = (ctypes.c_double * 64)(*[0.5] * 64)
BAD_THETA = (ctypes.c_double * 64)(*([0.5] * 63 + [float("nan")]))


def nr(L, **kw):
    a = dict(q=fake(0), k=fake(1), dtype=0, n=10, Hq=32, Hkv=8, d=128, qs=4096, ks=1024, pos=fake(2),
             wq=fake(3), wk=fake(4), eps=1e-6, th=ctypes.cast(THETA, P), R=128, style=0, mag=1.0,
             qo=fake(5), ko=fake(6), qos=4096, kos=1024, od=0)
    a.update(kw)
    return L.omnitide_qk_norm_rope(*a.values(), None)


def test_norm_rope_refusals(L):
    assert nr(L, q=None, k=None) == ot.E_NULL
    assert nr(L, qo=None) == ot.E_NULL and nr(L, ko=None) == ot.E_NULL
    assert nr(L, pos=None) == ot.E_NULL and nr(L, th=None) == ot.E_NULL
    assert nr(L, dtype=2) == ot.E_DTYPE and nr(L, od=5) == ot.E_DTYPE
    for bad in (dict(d=96), dict(n=-1), dict(n=(1 << 24) + 1), dict(Hq=0), dict(qs=4095),
                dict(qs=4088), dict(kos=1000), dict(R=130), dict(R=7), dict(R=12), dict(style=2),
                dict(eps=-1.0), dict(eps=float("nan")), dict(mag=float("inf")),
                dict(th=ctypes.cast(BAD_THETA, P)), dict(R=0, wq=None, wk=None), dict(q=fake(0, 8)),
                dict(ko=fake(6, 4)), dict(wq=fake(3, 2)), dict(qs=4100)):
        assert nr(L, **bad) == ot.E_SHAPE, bad
    # outputs over other arguments
    assert nr(L, qo=fake(0, 16)) == ot.E_ALIAS              # q shifted
    assert nr(L, qo=fake(0), qos=8192) == ot.E_ALIAS        # q at another stride
    assert nr(L, qo=fake(0), od=1) == ot.E_ALIAS            # in place needs one type
    assert nr(L, ko=fake(0)) == ot.E_ALIAS                  # k's output over q
    assert nr(L, ko=fake(5)) == ot.E_ALIAS                  # one buffer for both outputs
    assert nr(L, qo=fake(2)) == ot.E_ALIAS and nr(L, ko=fake(3)) == ot.E_ALIAS
    # a fused projection [q | k | v] in place: columns of one buffer do not overlap, one head more
    # of q does (n = 0: the checks alone)
    fused = dict(q=fake(0), k=fake(0, 4096 * 2), qo=fake(0), ko=fake(0, 4096 * 2), qs=6144, ks=6144,
                 qos=6144, kos=6144)
    assert nr(L, **fused, Hq=33) == ot.E_ALIAS
    assert nr(L, n=0) == ot.OK and nr(L, n=0, q=None, k=None, qo=None, ko=None) == ot.OK


def ap(L, **kw):
    a = dict(k=fake(0), v=fake(1), q=fake(2), dtype=0, n=10, Hq=32, Hkv=8, d=128, ks=1024, vs=1024,
             qs=4096, kp=fake(3), vp=fake(4), np=100, P=64, tab=fake(5), mp=20, st=fake(6),
             ctx=fake(7), S=4, pos=None, wk=fake(8), wq=fake(9), eps=1e-6, th=ctypes.cast(THETA, P),
             R=128, style=0, mag=1.0, qo=fake(10), qos=4096, status=fake(11))
    a.update(kw)
    return L.omnitide_paged_append(*a.values(), None)


def test_append_refusals(L):
    for k in ("k", "v", "kp", "vp", "tab", "st", "ctx", "qo", "q", "th"):
        assert ap(L, **{k: None}) == ot.E_NULL, k
    assert ap(L, dtype=3) == ot.E_DTYPE
    for bad in (dict(P=8), dict(P=48), dict(P=512), dict(S=0), dict(mp=0), dict(np=0), dict(d=80),
                dict(Hkv=33), dict(Hkv=0), dict(Hq=0), dict(ks=1000), dict(vs=1023), dict(qs=4000),
                dict(qos=4000), dict(n=-1), dict(R=9), dict(R=20), dict(style=5),
                dict(mp=(1 << 24) + 1), dict(S=1 << 20, mp=1 << 12), dict(kp=fake(3, 8)),
                dict(v=fake(1, 4))):
        assert ap(L, **bad) == ot.E_SHAPE, bad
    for bad in (dict(kp=fake(0)), dict(vp=fake(3)), dict(vp=fake(5)), dict(qo=fake(3)),
                dict(qo=fake(2, 16)), dict(qo=fake(2), dtype=1, ks=1024), dict(status=fake(7)),
                dict(kp=fake(2))):
        assert ap(L, **bad) == ot.E_ALIAS, bad
    assert ap(L, n=0) == ot.OK and ap(L, n=0, k=None, v=None, q=None, qo=None) == ot.OK


@pytest.mark.parametrize("d", [256, 192, 1 << 20])
@pytest.mark.parametrize("style", [0, 1])
def test_heads_and_rotations_beyond_the_table(L, d, style):
    """Head sizes that are not offered, rotated as a whole: refused before a frequency is copied (the
    launch arguments hold those of 128 dimensions)."""
    R = min(d, 256)
    theta = (ctypes.c_double * (R // 2))(*[0.5] * (R // 2))
    for r in (R, 136):
        rot = dict(th=ctypes.cast(theta, P), R=r, style=style, d=d)
        assert nr(L, qs=32 * d, ks=8 * d, qos=32 * d, kos=8 * d, **rot) == ot.E_SHAPE
        assert ap(L, ks=8 * d, vs=8 * d, qs=32 * d, qos=32 * d, **rot) == ot.E_SHAPE


def chunk(L, **kw):
    a = dict(q=fake(0), kp=fake(1), vp=fake(2), np=300, P=64, tab=fake(3), mp=270, st=fake(4),
             ctx=fake(5), S=3, n=700, Hq=32, Hkv=8, d=128, scale=0.1, out=fake(6), od=0, ws=fake(7),
             wsb=1 << 32, status=fake(8))
    a.update(kw)
    return L.omnitide_paged_chunk_attn(*a.values(), None)


def decode(L, **kw):
    a = dict(q=fake(0), kp=fake(1), vp=fake(2), np=300, P=64, tab=fake(3), mp=270, ctx=fake(5), S=3,
             nq=1, Hq=32, Hkv=8, d=128, scale=0.1, out=fake(6), od=0, ws=fake(7), wsb=1 << 32,
             status=fake(8))
    a.update(kw)
    return L.omnitide_paged_decode_attn(*a.values(), None)


@pytest.mark.parametrize("call", [chunk, decode])
def test_attention_refusals(L, call):
    for k in ("q", "kp", "vp", "tab", "ctx", "out") + (("st",) if call is chunk else ()):
        assert call(L, **{k: None}) == ot.E_NULL, k
    assert call(L, od=2) == ot.E_DTYPE
    for bad in (dict(P=8), dict(P=100), dict(S=0), dict(S=1025), dict(mp=0), dict(np=0), dict(d=96),
                dict(Hq=20), dict(Hkv=0), dict(Hkv=64, Hq=64), dict(scale=float("nan")),
                dict(mp=1 << 24, P=128), dict(q=fake(0, 8)), dict(out=fake(6, 4)),
                dict(scale=float("inf")), dict(scale=-2e30)):
        assert call(L, **bad) == ot.E_SHAPE, bad
    for bad in (dict(out=fake(0)), dict(out=fake(1)), dict(out=fake(5)), dict(status=fake(3)),
                dict(status=fake(6))):
        assert call(L, **bad) == ot.E_ALIAS, bad
    if call is chunk:
        assert chunk(L, n=-1) == ot.E_SHAPE and chunk(L, n=0) == ot.OK
        assert chunk(L, n=0, q=None, out=None) == ot.OK
    else:
        assert decode(L, nq=0) == ot.E_SHAPE and decode(L, nq=5) == ot.E_SHAPE
        assert decode(L, Hq=136, Hkv=8) == ot.E_SHAPE       # 17 query heads per KV head


def test_workspaces(L):
    size = pg.omnitide_paged_chunk_attn_workspace_bytes
    need = size(700, 3, 270 * 64, 32, 8, 128)
    if need:
        assert chunk(L, ws=None) == ot.E_WORKSPACE and chunk(L, wsb=need - 1) == ot.E_WORKSPACE
        assert chunk(L, wsb=need, out=fake(7)) == ot.E_ALIAS
    assert size(0, 3, 64, 32, 8, 128) == 0 and size(700, 3, 64, 32, 7, 128) == 0
    dsize = pg.omnitide_paged_decode_workspace_bytes
    need = dsize(3, 1, 270 * 64, 32, 8, 128)
    if need:
        assert decode(L, ws=None) == ot.E_WORKSPACE and decode(L, wsb=need - 1) == ot.E_WORKSPACE
        assert decode(L, wsb=need, out=fake(7)) == ot.E_ALIAS
    assert dsize(0, 1, 64, 32, 8, 128) == 0 and dsize(3, 5, 64, 32, 8, 128) == 0
    for hq, hkv, d in ((32, 8, 128), (4, 1, 64), (28, 4, 128), (8, 8, 64)):
        last = 0
        for ctx in (64, 500, 3000, 17000, 70000, 1 << 20):  # never falls as a size grows
            now = size(700, 3, ctx, hq, hkv, d)
            assert now >= last
            last = now
        for a, b in (((1, 1), (90, 1)), ((90, 1), (90, 9)), ((90, 9), (5000, 9)),
                     ((5000, 9), (100000, 9)), ((5000, 9), (5000, 900))):
            assert size(*a, 30000, hq, hkv, d) <= size(*b, 30000, hq, hkv, d), (a, b)
        last = 0
        for ctx in (64, 500, 3000, 17000, 70000, 1 << 20):
            now = dsize(3, 1, ctx, hq, hkv, d)
            assert now >= last
            last = now
        for a, b in ((1, 2), (2, 30), (30, 40), (40, 333), (333, 1024)):
            assert dsize(a, 1, 30000, hq, hkv, d) <= dsize(b, 1, 30000, hq, hkv, d), (a, b)


def test_binding_refusals():
    x = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):                         # not on the device
        pg.omnitide_qk_norm_rope(x, None, None, x, None)
    with pytest.raises(ValueError):
        pg.omnitide_qk_norm_rope(None, None, None, None, None)
    with pytest.raises(TypeError):
        pg.omnitide_qk_norm_rope(x.half(), None, None, x, None)


def test_tensors_off_the_current_device(monkeypatch):
    """Tensors of another device than the current one are refused."""
    class Tensor:
        device, index = "cuda:1", 1

        def get_device(self):
            return self.index
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    for stream in (None, 1234):
        with pytest.raises(ValueError, match="device 0 is the current one"):
            pg._on(Tensor(), stream)
    Tensor.index = 0
    assert pg._on(Tensor(), 1234) == 1234


class OnDevice(torch.Tensor):
    """A host tensor that says it is on device `number`."""
    is_cuda, number = property(lambda self: True), 0

    def get_device(self):
        return self.number


def far(t, number=0):
    t = t.as_subclass(OnDevice)
    t.number = number
    return t


class Calls:
    """Stands for the library: every call succeeds and touches nothing."""

    def __init__(self):
        self.made = []

    def __getattr__(self, name):
        return lambda *a: self.made.append((name, a)) or 0


def tensors(n=3, hq=4, hkv=2, d=64, pages=5, P=16):
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)      # noqa: E731
    rope = dict(q=bf(n, hq, d), k=bf(n, hkv, d), pos=i(n), q_out=bf(n, hq, d), k_out=bf(n, hkv, d),
                q_weight=bf(d), k_weight=bf(d))
    cache = dict(k_pool=bf(pages, P, hkv, d), v_pool=bf(pages, P, hkv, d), page_table=i(2, 3),
                 ctx_len=i(2), d_status=i(1))
    ws = torch.zeros(8, dtype=torch.uint8)
    append = dict(k=bf(n, hkv, d), v=bf(n, hkv, d), q_start=i(3), pos=i(n), k_weight=bf(d), q=bf(n, hq, d),
                  q_out=bf(n, hq, d), q_weight=bf(d), **cache)
    chunk = dict(q=bf(n, hq, d), q_start=i(3), out=bf(n, hq, d), workspace=ws, **cache)
    decode = dict(q=bf(2, 1, hq, d), out=bf(2, 1, hq, d), workspace=ws, **cache)
    return dict(omnitide_qk_norm_rope=rope, omnitide_paged_append=append,
                omnitide_paged_chunk_attn=chunk, omnitide_paged_decode_attn=decode)


@pytest.mark.parametrize("name", list(tensors()))
def test_one_tensor_on_another_device(monkeypatch, name):
    """Each tensor of each call in turn, and the stream: refused before the library is called; Tensor's
    subclasses are tensors."""
    calls = Calls()
    monkeypatch.setattr(pg, "_lib", calls)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 77 + dev, raising=False)
    args = {k: far(v) for k, v in tensors()[name].items()}
    call, more = getattr(pg, name), {} if "attn" not in name else dict(scale=1.0)
    call(**args, **more)
    assert calls.made.pop()[1][-1] == 77
    for k, v in args.items():
        with pytest.raises(ValueError, match="on device|current one"):
            call(**{**args, k: far(v, 1)}, **more)
        with pytest.raises(ValueError):                     # a host tensor
            call(**{**args, k: v.as_subclass(torch.Tensor)}, **more)

    class Stream:
        device, device_index, cuda_stream = "cuda:1", 1, 1234
    with pytest.raises(ValueError, match="stream"):
        call(**args, **more, stream=Stream())
    assert not calls.made
    Stream.device_index = 0
    call(**args, **more, stream=Stream())
    assert calls.made.pop()[1][-1] == 1234
