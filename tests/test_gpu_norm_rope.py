"""Norm and rotation of queries and keys, and the append to the pages, against float64.

Tolerance, per element: the rounding to the output type (half a step: eps / 2 of the value, and half of
the smallest step near zero) plus 2^-19 of the length of the normed pair (the header's bound: the sum of 128
squares in float, at most 12 roundings deep, halved by the root, with the root, quotient, two products and
eps' addition 11 x 2^-24; sine and cosine of a float fraction of a turn 2^-23.3 + 2 x 2^-23; magnitude,
product and fused product 3 x 2^-24; the angle in double 2^-21: below 2^-19 together)."""
import numpy as np
import pytest
import torch

from oracle import paged as op

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
STYLE = {"half": 0, "interleaved": 1}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_34653_amd import paged
    paged.lib()
    yield


def f64(t):
    return t.detach().cpu().double().numpy()


def assert_close(got, want, pair, R, style, dtype, where=""):
    """got, want [T, H, d]; pair: float64 normed, unrotated values."""
    eps = torch.finfo(dtype).eps
    length = np.abs(pair)
    if R:
        from oracle.rope import pair_dims
        a, b = pair_dims(R, style)
        n = np.hypot(pair[..., a], pair[..., b])
        length[..., a], length[..., b] = n, n
    tol = eps / 2 * np.abs(want) + 2.0 ** -19 * length + 1e-38
    err = np.abs(f64(got) - want)
    assert (err <= tol).all(), (where, float((err - tol).max()), float(err.max()))


def fused(T, hq, hkv, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, hq + 2 * hkv, d, generator=g) * torch.exp(
        torch.randn(T, hq + 2 * hkv, 1, generator=g))
    w = [1 + 0.3 * torch.randn(d, generator=g) for _ in range(2)]
    return x.to(dtype).cuda(), [y.to(dtype).cuda() for y in w]


@pytest.mark.parametrize("T,hq,hkv,d,dtype,out,R,style,norm", [
    (1, 32, 8, 128, BF, BF, 128, "half", "qk"),
    (5, 32, 8, 128, BF, BF, 128, "interleaved", "qk"),
    (67, 28, 4, 128, BF, BF, 64, "half", "k"),
    (67, 28, 4, 128, BF, F32, 64, "interleaved", "q"),
    (33, 14, 2, 64, F32, F32, 64, "half", "qk"),
    (33, 14, 2, 64, F32, F32, 32, "interleaved", ""),
    (130, 3, 1, 64, F32, BF, 8, "half", "qk"),
    (130, 1, 1, 128, BF, BF, 24, "half", ""),
    (9, 5, 5, 64, BF, BF, 2, "interleaved", "qk"),
    (9, 17, 3, 128, F32, F32, 6, "interleaved", "qk"),
    (40, 16, 4, 128, BF, BF, 0, "half", "qk"),
    (40, 16, 4, 64, F32, F32, 0, "half", "k"),
    (3001, 4, 1, 64, BF, BF, 64, "half", "qk"),
])
def test_norm_rope(T, hq, hkv, d, dtype, out, R, style, norm):
    from paper_2609_34653_amd import paged as pg
    x, (wq, wk) = fused(T, hq, hkv, d, dtype, T + R)
    q, k = x[:, :hq], x[:, hq:hq + hkv]
    rng = np.random.default_rng(T)
    pos = rng.integers(0, 1 << 20, T)
    pos[0], pos[-1] = 0, 2 ** 31 - 1 if T > 1 else 77777
    th = pg.omnitide_rope_thetas(1.0e6, R) if R else None
    wq = wq if "q" in norm else None
    wk = wk if "k" in norm else None
    qo = torch.full((T, hq, d), float("nan"), dtype=out, device="cuda")
    ko = torch.full((T, hkv, d), float("nan"), dtype=out, device="cuda")
    pd = torch.tensor(pos, dtype=torch.int32, device="cuda")
    pg.omnitide_qk_norm_rope(q, k, pd if R else None, qo, ko, th, STYLE[style], 1.25, wq, wk, 1e-5)
    torch.cuda.synchronize()
    for got, src, w in ((qo, q, wq), (ko, k, wk)):
        wn = None if w is None else f64(w)
        want = op.norm_rope(f64(src), wn, 1e-5, th, pos, style, 1.25)
        if w is None and not R:
            assert torch.equal(got, src.to(out))
            continue
        mag = 1.25 if R else 1.0
        assert_close(got, want, mag * op.norm_rope(f64(src), wn, 1e-5, None, pos, style), R, style,
                     out)
    # columns of the fused tensor that are no argument's stay
    assert torch.equal(x, fused(T, hq, hkv, d, dtype, T + R)[0])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("style", ["half", "interleaved"])
def test_norm_rope_in_place_one_side_and_padding(dtype, style):
    from paper_2609_34653_amd import paged as pg
    T, hq, hkv, d = 21, 12, 3, 64
    th = pg.omnitide_rope_thetas(10000.0, 32)
    x, (wq, wk) = fused(T, hq, hkv, d, dtype, 5)
    pos = torch.arange(T, dtype=torch.int32)
    pos[[0, 7, 20]] = -1                                     # padding: left as they were
    pd = pos.cuda()
    sep_q, sep_k = torch.zeros_like(x[:, :hq]).contiguous(), x[:, hq:hq + hkv].contiguous()
    sep_q.copy_(x[:, :hq])
    pg.omnitide_qk_norm_rope(x[:, :hq], None, pd, sep_q, None, th, STYLE[style], q_weight=wq)
    pg.omnitide_qk_norm_rope(None, x[:, hq:hq + hkv], pd, None, sep_k, th, STYLE[style], k_weight=wk)
    y = x.clone()
    pg.omnitide_qk_norm_rope(y[:, :hq], y[:, hq:hq + hkv], pd, y[:, :hq], y[:, hq:hq + hkv], th,
                             STYLE[style], q_weight=wq, k_weight=wk)
    torch.cuda.synchronize()
    assert torch.equal(y[:, :hq], sep_q) and torch.equal(y[:, hq:hq + hkv], sep_k)
    assert torch.equal(y[:, hq + hkv:], x[:, hq + hkv:])     # the values' columns
    pad = pos < 0
    assert torch.equal(y[pad.cuda()], x[pad.cuda()])
    assert not torch.equal(y[~pad.cuda()], x[~pad.cuda()])


@pytest.mark.parametrize("dtype,out", [(F32, F32), (F32, BF), (BF, BF)])
@pytest.mark.parametrize("eps", [0.0, 1e-6, 1e-34, 1e30])
def test_norm_over_the_range_of_float(dtype, out, eps):
    """Heads of one wave of every size from denormal numbers to the largest, whose squares float holds or
    not, beside each other; small and large weights; rotated."""
    from paper_2609_34653_amd import paged as pg
    hq, hkv, d, T = 26, 3, 64, 3
    x, (wq, wk) = fused(T, hq, hkv, d, dtype, 9)
    power = np.array([-126, -110, -100, -90, -80, -66, -60, -51, -50, -49, -45, -30, 0, 1, 30, 45, 55, 58,
                      59, 60, 61, 63, 64, 80, 100, 122])
    scale = torch.tensor(np.ldexp(1.0, np.concatenate([power, [-60, 0, 64], np.zeros(hkv, int)])),
                         dtype=torch.float32, device="cuda")[:, None]
    unit = x.float() / x.float().abs().amax(-1, keepdim=True)
    x = (unit * scale).to(dtype)
    wq, wk = (wq.float() * 2.0 ** -90).to(dtype), (wk.float() * 2.0 ** 90).to(dtype)
    q, k = x[:, :hq], x[:, hq:hq + hkv]
    th = pg.omnitide_rope_thetas(1.0e4, 32)
    pos = np.array([0, 77, 70001])
    qo = torch.full((T, hq, d), float("nan"), dtype=out, device="cuda")
    ko = torch.full((T, hkv, d), float("nan"), dtype=out, device="cuda")
    pg.omnitide_qk_norm_rope(q, k, i32(pos), qo, ko, th, 0, 1.0, wq, wk, eps)
    torch.cuda.synchronize()
    e = float(np.float32(eps))
    for got, src, w in ((qo, q, f64(wq)), (ko, k, f64(wk))):
        want = op.norm_rope(f64(src), w, e, th, pos, "half")
        plain = op.norm_rope(f64(src), w, e, None, pos, "half")
        assert_close(got, want, plain, 32, "half", out)


@pytest.mark.parametrize("dtype,out", [(F32, F32), (BF, BF)])
def test_norm_of_heads_of_unlike_values(dtype, out):
    """Pairs of tiny values beside a large one keep their bits: 2^-56 to 2^-16 beside 2^70, 2^-149 and up
    beside 2^-62, and beside 1."""
    from paper_2609_34653_amd import paged as pg
    T, h, d = 5, 9, 64
    x, (w, _) = fused(T, h, 0, d, F32, 11)
    x = x / x.abs().amax(-1, keepdim=True)
    at = torch.arange(d, device="cuda") % 32                 # both values of a pair are of one size
    x = x * torch.ldexp(torch.ones(1, device="cuda"), -16 - 2 * (at % 20))
    x[..., [3, 35]] = 1.5 * 2.0 ** 70
    x[:, 3:6] *= 2.0 ** -60                                  # sizes 2^-76..2^-114 beside 2^10
    x[:, 6:] *= 2.0 ** -72
    x[:, 6:] *= 2.0 ** -60                                   # denormal numbers beside 2^-62
    x = x.to(dtype)
    th = pg.omnitide_rope_thetas(1.0e4, d)
    pos, w = np.array([0, 1, 9, 700, 70001]), w.to(dtype)
    o = torch.full((T, h, d), float("nan"), dtype=out, device="cuda")
    pg.omnitide_qk_norm_rope(x, None, i32(pos), o, None, th, 0, 1.0, w, None, 0.0)
    torch.cuda.synchronize()
    want = op.norm_rope(f64(x), f64(w), 0.0, th, pos, "half")
    assert_close(o, want, op.norm_rope(f64(x), f64(w), 0.0, None, pos, "half"), d, "half", out)


def test_zero_tokens():
    from paper_2609_34653_amd import paged as pg
    e = torch.empty(0, 4, 64, dtype=BF, device="cuda")
    pg.omnitide_qk_norm_rope(e, e, torch.empty(0, dtype=torch.int32, device="cuda"), e.clone(),
                             e.clone(), pg.omnitide_rope_thetas(1e4, 64))


# ----------------------------------------------------------------------------------- append

def layout(ctx, P, seed, spare=2, max_pages=None):
    """Shuffled page table of sequences of ctx rows; unused entries hold garbage."""
    rng = np.random.default_rng(seed)
    need = [-(-n // P) for n in ctx]
    n_pages = sum(need) + spare
    order = rng.permutation(n_pages)
    table = np.full((len(ctx), max_pages or max(need + [1])), -77, np.int32)
    table[:, ::2] = 1 << 30
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return table, n_pages


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("ctx,new,P,hq,hkv,d,dtype,R,style,norm,with_q", [
    ([1], [1], 16, 4, 1, 64, BF, 64, "half", True, True),
    ([40, 7, 300, 9], [3, 7, 0, 1], 16, 32, 8, 128, BF, 128, "half", True, True),
    ([129, 65, 64], [65, 65, 1], 64, 28, 4, 128, BF, 64, "interleaved", False, False),
    ([500, 33], [200, 33], 32, 6, 2, 64, F32, 32, "half", True, True),
    ([257, 256, 255], [257, 2, 0], 256, 3, 3, 64, F32, 0, "half", False, True),
    ([70] * 70, [1] * 70, 128, 16, 2, 128, BF, 128, "half", False, True),
    ([3 + i % 5 for i in range(200)], [i % 4 for i in range(200)], 16, 8, 8, 64, BF, 0, "half", False,
     False),
])
def test_append(ctx, new, P, hq, hkv, d, dtype, R, style, norm, with_q):
    from paper_2609_34653_amd import paged as pg
    table, n_pages = layout(ctx, P, len(ctx))
    lead, tail = 2, 3                                        # padding tokens in front and behind
    start = np.concatenate([[0], np.cumsum(new)]) + lead
    T = int(start[-1]) + tail
    x, (wq, wk) = fused(T, hq, hkv, d, dtype, T)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    kp = torch.randn(n_pages, P, hkv, d, device="cuda").to(BF)
    vp = torch.randn(n_pages, P, hkv, d, device="cuda").to(BF)
    kw, vw = kp.clone(), vp.clone()
    qo = torch.full((T, hq, d), 7.0, dtype=BF, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    th = pg.omnitide_rope_thetas(1.0e6, R, pg.ROPE_LINEAR, 4.0) if R else None
    wq, wk = (wq, wk) if norm else (None, None)
    pg.omnitide_paged_append(k, v, kp, vp, i32(table), i32(start), i32(ctx), theta=th,
                             rope_style=STYLE[style], magnitude=0.75, k_weight=wk,
                             q=q if with_q else None, q_out=qo if with_q else None,
                             q_weight=wq if with_q else None, d_status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    page, line, tok, row = [], [], [], []
    for s in range(len(ctx)):
        for i in range(new[s]):
            r = ctx[s] - new[s] + i
            page.append(table[s, r // P])
            line.append(r % P)
            tok.append(start[s] + i)
            row.append(r)
    assert torch.equal(vp[page, line], v[tok].to(BF))
    vw[page, line] = vp[page, line]
    assert torch.equal(vp, vw)
    got = kp[page, line]
    wn = None if wk is None else f64(wk)
    if R or norm:
        want = op.norm_rope(f64(k[tok]), wn, 1e-6, th, row, style, 0.75)
        plain = op.norm_rope(f64(k[tok]), wn, 1e-6, None, row, style) * (0.75 if R else 1.0)
        assert_close(got, want, plain, R, style, BF)
    else:
        assert torch.equal(got, k[tok].to(BF))
    kw[page, line] = got
    assert torch.equal(kp, kw)                               # rows of no new token
    if with_q:
        want = op.norm_rope(f64(q[tok]), None if wq is None else f64(wq), 1e-6, th, row, style, 0.75)
        plain = op.norm_rope(f64(q[tok]), None if wq is None else f64(wq), 1e-6, None, row, style)
        assert_close(qo[tok], want, plain * (0.75 if R else 1.0), R, style, BF)
    rest = np.setdiff1d(np.arange(T), tok if with_q else [])
    assert (qo[rest] == 7.0).all()


def test_append_copies_every_bit_and_takes_positions():
    """bf16 values (and unrotated keys) are copied with their NaN payloads; pos overrides the row."""
    from paper_2609_34653_amd import paged as pg
    bits = torch.arange(64 * 64, dtype=torch.int32).remainder(65536).to(torch.int16)
    bits[:8] = torch.tensor([0x7f81, 0x7fff, -1, -127, 0x7f80, -128, 0, 1], dtype=torch.int16)
    k = bits.view(BF).view(64, 1, 64).cuda()
    kp, vp = torch.zeros(2, 4, 16, 1, 64, dtype=BF, device="cuda")
    tab, start, ctx = i32([[3, 1, 0, 2]]), i32([0, 64]), i32([64])
    pg.omnitide_paged_append(k, k, kp, vp, tab, start, ctx)
    torch.cuda.synchronize()
    order = kp.view(torch.int16)[[3, 1, 0, 2]].view(64, 64)
    assert torch.equal(order.cpu(), bits.view(64, 64))
    assert torch.equal(vp.view(torch.int16), kp.view(torch.int16))
    x = torch.randn(64, 1, 64, device="cuda").to(BF)
    pos = i32(np.arange(64) * 1000 - 5000)                   # negative positions too
    th = pg.omnitide_rope_thetas(1.0e4, 64)
    pg.omnitide_paged_append(x, x, kp, vp, tab, start, ctx, pos=pos, theta=th)
    torch.cuda.synchronize()
    want = op.norm_rope(f64(x), None, 0.0, th, f64(pos), "half")
    assert_close(kp[[3, 1, 0, 2]].view(64, 1, 64), want, f64(x), 64, "half", BF)


@pytest.mark.parametrize("what", ["page", "low", "long", "order", "past"])
def test_append_device_refusals(what):
    """A bad page id, length or offset is reported and writes nothing of the rows it concerns."""
    from paper_2609_34653_amd import omnitide as ot, paged as pg
    table, start, ctx = np.array([[0, 1], [2, 3]], np.int32), [0, 4, 8], [20, 32]
    want = pg.E_PAGES
    if what == "page":
        table[1, 1] = 4                                      # pages 0..3 exist
    elif what == "low":
        ctx[1], want = 3, ot.E_CAPACITY                      # four new tokens
    elif what == "long":
        ctx[1], want = 33, ot.E_CAPACITY                     # two pages of 16
    elif what == "order":
        start = [4, 3, 8]
    else:
        start = [0, 4, 9]                                    # eight tokens
    k = torch.ones(8, 1, 64, dtype=BF, device="cuda")
    kp, vp = torch.zeros(2, 4, 16, 1, 64, dtype=BF, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    pg.omnitide_paged_append(k, k, kp, vp, i32(table), i32(start), i32(ctx), d_status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == want
    assert (kp[2:] == 0).all() or what == "order"
    if what != "order":
        assert (kp[1, 0:4] == 1).all() and int((kp != 0).sum()) == 4 * 64


def test_append_to_one_row_by_many():
    """Sequences whose new tokens share a row of a page: each value is one of theirs, their own rows are
    whole."""
    from paper_2609_34653_amd import paged as pg
    n_seq, P, hkv, d = 300, 16, 8, 128
    table = np.stack([np.zeros(n_seq, int), 1 + np.arange(n_seq)], 1)     # page 0 is everybody's
    start, ctx = 2 * np.arange(n_seq + 1), np.full(n_seq, 17)             # rows 15 (shared) and 16 (own)
    no = torch.arange(2 * n_seq, device="cuda").to(torch.float32)
    k = no[:, None, None].expand(2 * n_seq, hkv, d).contiguous()
    kp, vp = torch.full((2, n_seq + 1, P, hkv, d), -5.0, dtype=BF, device="cuda")
    pg.omnitide_paged_append(k, -k, kp, vp, i32(table), i32(start), i32(ctx))
    torch.cuda.synchronize()
    first, own = (no[i::2].to(BF) for i in (0, 1))
    assert torch.isin(kp[0, 15], first).all() and torch.isin(vp[0, 15], -first).all()
    assert (kp[1:, 0] == own[:, None, None]).all() and (vp[1:, 0] == -own[:, None, None]).all()
    kp[0, 15], vp[0, 15], kp[1:, 0], vp[1:, 0] = -5.0, -5.0, -5.0, -5.0
    assert (kp == -5.0).all() and (vp == -5.0).all()


def test_append_leaves_what_is_not_its_own():
    """Padding rows of NaN in front and behind, and a sequence whose page is bad: neither the pools' other
    rows nor q_out see them; the tokens beside them are as without."""
    from paper_2609_34653_amd import paged as pg
    ctx, new, P, hq, hkv, d = [40, 35, 9], [3, 4, 9], 16, 8, 2, 64
    table, n_pages = layout(ctx, P, 8)
    start = np.concatenate([[0], np.cumsum(new)]) + 5
    T = int(start[-1]) + 4
    x, (wq, wk) = fused(T, hq, hkv, d, BF, 8)
    th = pg.omnitide_rope_thetas(1.0e4, d)

    def run(x, table):
        kp, vp = torch.full((2, n_pages, P, hkv, d), 2.0, dtype=BF, device="cuda")
        qo = torch.full((T, hq, d), 7.0, dtype=BF, device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        pg.omnitide_paged_append(x[:, hq:hq + hkv], x[:, hq + hkv:], kp, vp, i32(table), i32(start),
                                 i32(ctx), theta=th, k_weight=wk, q=x[:, :hq], q_out=qo, q_weight=wq,
                                 d_status=st)
        torch.cuda.synchronize()
        return kp, vp, qo, int(st.item())
    want = run(x, table)
    padded = x.clone()
    padded[:5] = float("nan")
    padded[int(start[-1]):] = float("inf")
    got = run(padded, table)
    assert got[3] == want[3] == 0 and all(torch.equal(a, b) for a, b in zip(got[:3], want[:3]))
    bad = table.copy()
    bad[1, 2] = n_pages                                      # rows 32..34: the last three of four tokens
    got = run(x, bad)
    tokens, page = slice(int(start[2]) - 3, int(start[2])), int(table[1, 2])
    for g, w, at, keep in zip(got, want, (page, page, tokens), (2.0, 2.0, 7.0)):
        w[at] = keep
        assert torch.equal(g, w)
    assert got[3] == pg.E_PAGES


def test_append_past_four_gigabytes():
    """Slots whose byte offset passes 32 bits."""
    from paper_2609_34653_amd import paged as pg
    P, hkv, d = 256, 32, 128
    n_pages = (5 << 30) // (P * hkv * d * 2)
    kp = torch.zeros(n_pages, P, hkv, d, dtype=BF, device="cuda")
    vp = torch.zeros_like(kp)
    x = torch.randn(300, hkv, d, device="cuda").to(BF)
    tab = i32([[n_pages - 1, n_pages - 2]])
    pg.omnitide_paged_append(x, x, kp, vp, tab, i32([0, 300]), i32([300]))
    torch.cuda.synchronize()
    assert torch.equal(kp[n_pages - 1], x[:256]) and torch.equal(vp[n_pages - 2, :44], x[256:])
    assert int((kp[:n_pages - 2] != 0).sum()) == 0
