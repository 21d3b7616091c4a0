"""The latent cache against float64: append, rows in one piece, attention over the latents and over expanded
keys and values.

Tolerances, per element:
  append  as tests/test_gpu_norm_rope.py: half a step of the output plus 2^-19 of the normed pair's length
          (the sum of 512 squares is 14 roundings deep, halved by the root: 13 x 2^-24 with the rest)
  attention, with S = sum_j p_j |v_j| + |out|:
          2^-8 S (that of probabilities rounded to bf16 once; they keep 16 bits, whose tests stand further down)
          + 2^-10 S (absorbed) or 2^-11 S (expanded) for the scores: products of bf16 are exact in float, the sum
          of d of them is off by at most d 2^-24 sum|q k|; sum|q k| scale <= 20 on these inputs, so a
          probability by 576 x 20 x 2^-24 = 2^-10.5 (192: 2^-12.1); the exponential and the sums add 2^-18
          + the rounding of a bf16 output, 2^-8 |out| (half a step)."""
import numpy as np
import pytest
import torch

from oracle import latent as ol
from oracle import paged as op
from tests.test_gpu_norm_rope import BF, F32, STYLE, assert_close, f64, i32, layout

pytestmark = pytest.mark.gpu

E = 64


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_34653_amd import latent
    latent.lib()
    yield


def rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def pool_of(ctx, table, n_pages, P, width, seed):
    """Pool whose rows in use are normal and whose other rows are NaN and infinities."""
    pool = torch.full((n_pages, P, width), float("nan"))
    pool[:, ::2] = float("inf")
    x = rand(seed, sum(ctx), width)
    at = 0
    for s, n in enumerate(ctx):
        r = np.arange(n)
        if n:
            pool[table[s, r // P], r % P] = x[at:at + n]
        at += n
    return pool.to(BF)


def near(got, want, spread, score, dtype):
    tol = (2.0 ** -8 + score) * spread
    if dtype == BF:
        tol = tol + torch.finfo(BF).eps / 2 * (np.abs(want) + tol)
    err = np.abs(f64(got) - want)
    assert np.isfinite(f64(got)).all()
    assert (err <= tol).all(), (float(err.max()), float((err / np.maximum(tol, 1e-30)).max()))


# ----------------------------------------------------------------------------------- append

APPENDS = [
    # ctx, new, page, heads, R, dtype, style, norm, turned
    ([1], [1], 16, 4, 512, BF, "half", True, True),
    ([40, 7, 300, 9], [3, 7, 0, 1], 16, 16, 512, BF, "interleaved", True, True),
    ([129, 65, 64], [65, 65, 1], 64, 20, 256, F32, "half", True, True),
    ([500, 33], [200, 33], 32, 3, 512, F32, "interleaved", False, True),
    ([257, 256], [257, 2], 256, 0, 256, BF, "half", True, True),
    ([70] * 70, [1] * 70, 128, 128, 512, BF, "half", False, True),
    ([1500], [1400], 16, 31, 512, F32, "half", True, True),
    ([90, 33], [80, 33], 16, 9, 512, BF, "half", False, False),
    ([90, 33], [80, 33], 16, 7, 256, F32, "half", True, False),
]


@pytest.mark.parametrize("case", range(len(APPENDS)))
def test_append(case):
    from paper_2609_34653_amd import latent as la, paged as pg
    ctx, new, P, H, R, dtype, style, norm, turned = APPENDS[case]
    table, n_pages = layout(ctx, P, case)
    start = np.concatenate([[0], np.cumsum(new)]) + 2        # padding in front and behind
    T = int(start[-1]) + 3
    kv = (rand(case, T, R + E) * torch.exp(rand(case + 50, T, 1))).to(dtype).cuda()
    q = rand(case + 1, T, max(H, 1), 128 + E).to(dtype).cuda()
    w = (1 + 0.3 * rand(case + 2, R)).to(dtype).cuda() if norm else None
    th = pg.omnitide_rope_thetas(1.0e6, E, pg.ROPE_LINEAR, 4.0) if turned else None
    pool = rand(case + 3, n_pages, P, R + E).to(BF).cuda()
    want_pool = f64(pool)
    out = torch.full((T, max(H, 1), R + E), 7.0, dtype=BF, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    pos = np.random.default_rng(case).integers(-5, 1 << 20, T) if case % 2 else None
    la.omnitide_latent_append(kv[:, :R], kv[:, R:], pool, i32(table), i32(start), i32(ctx),
                              pos=None if pos is None else i32(pos), theta=th, rope_style=STYLE[style],
                              magnitude=0.75, latent_weight=w, eps=1e-5,
                              q_rope=q[..., 128:] if H else None, q_out=out[..., R:] if H else None,
                              d_status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    page, line, tok, row = [], [], [], []
    for s, (n, m) in enumerate(zip(ctx, new)):
        for i in range(m):
            r = n - m + i
            page.append(table[s, r // P]), line.append(r % P)
            tok.append(start[s] + i), row.append(r)
    at = np.array(row) if pos is None else pos[tok]
    x, wn, mag = f64(kv)[tok], None if w is None else f64(w), 0.75 if turned else 1.0
    want = ol.latent_row(x[:, :R], x[:, R:], wn, 1e-5, th, at, style, 0.75)
    plain = ol.latent_row(x[:, :R], x[:, R:], wn, 1e-5, None, at, style)
    got = pool[page, line]
    assert_close(got[:, None, :R], want[:, None, :R], plain[:, None, :R], 0, style, BF, "latent")
    assert_close(got[:, None, R:], want[:, None, R:], mag * plain[:, None, R:], E if turned else 0, style, BF,
                 "key part")
    if dtype == BF and not norm:
        assert torch.equal(got[:, :R], kv[tok][:, :R])
    if dtype == BF and not turned:
        assert torch.equal(got[:, R:], kv[tok][:, R:])
    want_pool[page, line] = f64(got)
    assert np.array_equal(f64(pool), want_pool)              # other rows are as they were
    if H:
        qx = f64(q)[tok][..., 128:]
        assert_close(out[tok][..., R:], op.norm_rope(qx, None, 0.0, th, at, style, 0.75), mag * qx,
                     E if turned else 0, style, BF, "queries")
        other = np.setdiff1d(np.arange(T), tok)
        assert (f64(out[other]) == 7.0).all() and (f64(out[..., :R]) == 7.0).all()


def test_append_of_millions():
    """More workgroups than one dimension of a launch has: every row is there, bit for bit."""
    from paper_2609_34653_amd import latent as la
    n, P, R = (1 << 22) + 5, 256, 256
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn(n, R + E, generator=g, device="cuda", dtype=BF)
    pool = torch.zeros(-(-n // P) + 1, P, R + E, dtype=BF, device="cuda")
    pages = torch.randperm(pool.shape[0] - 1, generator=g, device="cuda").to(torch.int32)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    la.omnitide_latent_append(x[:, :R], x[:, R:], pool, pages[None], i32([0, n]), i32([n]), d_status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    assert torch.equal(pool[pages.long()].view(-1, R + E)[:n], x)
    assert not pool[-1].any()


def test_append_queries_in_place():
    from paper_2609_34653_amd import latent as la, paged as pg
    T, H, R, P = 21, 5, 256, 16
    table, n_pages = layout([T], P, 1)
    kv = rand(1, T, R + E).to(BF).cuda()
    q = rand(2, T, H, 64 + E).to(BF).cuda()
    th = pg.omnitide_rope_thetas(1.0e4, E)
    outs = []
    for qi, qo in ((q, torch.zeros(T, H, E, dtype=BF, device="cuda")), (q.clone(), None)):
        pool = torch.zeros(n_pages, P, R + E, dtype=BF, device="cuda")
        src = qi[..., 64:]
        dst = src if qo is None else qo
        la.omnitide_latent_append(kv[:, :R], kv[:, R:], pool, i32(table), i32([0, T]), i32([T]), theta=th,
                                  q_rope=src, q_out=dst)
        outs.append((dst.clone(), pool, qi))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    assert torch.equal(outs[1][2][..., :64], q[..., :64])    # the other columns


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("eps", [0.0, 1e-6, 1e-34])
def test_norm_over_the_range_of_float(dtype, eps):
    """Latents from denormal numbers to the largest, whose squares float holds or not."""
    from paper_2609_34653_amd import latent as la
    R, P = 512, 16
    power = np.array([-126, -110, -90, -66, -60, -52, -50, -45, 0, 45, 57, 59, 61, 64, 100, 118])
    T = len(power)
    x = rand(3, T, R)
    x = x / x.abs().amax(-1, keepdim=True) * torch.tensor(np.ldexp(1.0, power), dtype=F32)[:, None]
    kv = torch.cat([x, rand(4, T, E)], 1).to(dtype).cuda()
    w = (1 + 0.3 * rand(5, R)).to(dtype).cuda()
    table, n_pages = layout([T], P, 1)
    pool = torch.zeros(n_pages, P, R + E, dtype=BF, device="cuda")
    la.omnitide_latent_append(kv[:, :R], kv[:, R:], pool, i32(table), i32([0, T]), i32([T]),
                              latent_weight=w, eps=eps)
    got = pool[table[0, np.arange(T) // P], np.arange(T) % P]
    want = ol.latent_row(f64(kv)[:, :R], f64(kv)[:, R:], f64(w), float(np.float32(eps)), None,
                         np.zeros(T), "half")
    assert_close(got[:, None, :R], want[:, None, :R], want[:, None, :R], 0, "half", BF)


def test_append_refused_on_the_device():
    """Bad pages, lengths and offsets: nothing of those tokens is written, the others are."""
    from paper_2609_34653_amd import latent as la, omnitide as ot, paged as pg
    ctx, new, P, R = [40, 33, 20], [5, 3, 4], 16, 256
    start = [0, 5, 8, 12]
    kv = rand(1, 12, R + E).to(BF).cuda()
    for what in ("page", "low", "long", "order"):
        table, n_pages = layout(ctx, P, 3)
        n, st0, code = list(ctx), list(start), pg.E_PAGES
        if what == "page":
            table[1, 2] = n_pages
            lost = [7]                                       # row 32, the second of page 2
        elif what == "low":
            n[1], code, lost = 2, ot.E_CAPACITY, [5, 6, 7]
        elif what == "long":
            n[1], code, lost = table.shape[1] * P + 1, ot.E_CAPACITY, [5, 6, 7]
        else:
            st0, lost = [0, 5, 3, 12], [3, 4]
        pool = torch.full((n_pages, P, R + E), 9.0, dtype=BF, device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        la.omnitide_latent_append(kv[:, :R], kv[:, R:], pool, i32(table), i32(st0), i32(n), d_status=st)
        assert int(st.item()) == code
        written = (pool != 9.0).any(-1).sum().item()
        if what == "page":
            assert written == 12 - sum(r // P == 2 for r in (30, 31, 32))
        elif what != "order":
            assert written == 12 - len(lost)


# ------------------------------------------------------------------------------------- rows

@pytest.mark.parametrize("ctx,take,P,shape", [
    ([1], [1], 16, (576,)),
    ([300, 0, 77, 64], [300, 0, 77, 60], 16, (576,)),
    ([129, 5], [100, 5], 128, (8, 128)),
    ([70 + i % 9 for i in range(70)], [(70 + i % 9) * (i % 3 > 0) for i in range(70)], 32, (320,)),
    ([4000], [4000], 64, (8,)),
    ([513], [513], 256, (32, 128)),
])
def test_rows(ctx, take, P, shape):
    from paper_2609_34653_amd import latent as la
    table, n_pages = layout(ctx, P, len(ctx))
    width = int(np.prod(shape))
    pool = pool_of(ctx, table, n_pages, P, width, 1)
    start = np.concatenate([[0], np.cumsum(take)]) + 3
    n = int(start[-1]) + 2
    out = torch.full((n, width + 16), 5.0, dtype=BF, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    la.omnitide_paged_rows(pool.view(n_pages, P, *shape).cuda(), i32(table), i32(start), i32(ctx),
                           out[:, :width], st)
    assert int(st.item()) == 0
    want = torch.full((n, width + 16), 5.0, dtype=BF)
    for s, m in enumerate(take):
        r = np.arange(m)
        if m:
            want[start[s]:start[s] + m, :width] = pool[table[s, r // P], r % P]
    assert torch.equal(out.cpu(), want)


def test_rows_refused_on_the_device():
    from paper_2609_34653_amd import latent as la, omnitide as ot, paged as pg
    ctx, P, W = [50, 40], 16, 576
    for what in ("page", "many", "order"):
        table, n_pages = layout(ctx, P, 2)
        pool = pool_of(ctx, table, n_pages, P, W, 1)
        start, code = [0, 50, 90], pg.E_PAGES
        if what == "page":
            table[1, 1] = -1
        elif what == "many":
            start, code = [0, 50, 91], ot.E_CAPACITY
        else:
            start = [0, 50, 40]
        out = torch.full((95, W), 5.0, dtype=BF, device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        la.omnitide_paged_rows(pool.cuda(), i32(table), i32(start), i32(ctx), out, st)
        assert int(st.item()) == code
        r = np.arange(50)
        assert torch.equal(out[:50].cpu(), pool[table[0, r // P], r % P])
        if what == "page":
            assert torch.isnan(out[66:82]).all() and not torch.isnan(out[50:66]).any()
            assert not torch.isnan(out[82:90]).any() and (out[90:] == 5.0).all()
        else:
            assert (out[50:] == 5.0).all()


# ----------------------------------------------------------------------------------- decode

def decode(q, pool, table, ctx, scale, dtype, fill=0xff):
    from paper_2609_34653_amd import latent as la
    S, nq, H, W = q.shape
    out = torch.full((S, nq, H, W - E), float("nan"), dtype=dtype, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    nb = la.omnitide_latent_decode_workspace_bytes(S, nq, table.shape[1] * pool.shape[1], H, W - E)
    ws = torch.full((nb,), fill, dtype=torch.uint8, device="cuda")
    la.omnitide_latent_decode_attn(q, pool, i32(table), i32(ctx), scale, out, ws, st)
    torch.cuda.synchronize()
    return out, int(st.item())


def queries(seed, S, nq, H, R):
    return (rand(seed, S, nq, H, R + E) * (192 / (R + E)) ** 0.5).to(BF)


SCALE = 192 ** -0.5

DECODES = [
    # ctx, nq, page, heads, R, out
    ([1], 1, 16, 4, 512, F32),
    ([33], 1, 16, 16, 512, F32),
    ([777], 1, 64, 16, 512, BF),
    ([5000, 0, 63, 2048], 2, 128, 16, 512, BF),              # an idle sequence, 32 vectors
    ([129, 4, 40], 4, 16, 8, 256, F32),                      # four tokens, causal among them
    ([3001, 64, 65], 1, 32, 128, 512, F32),                  # 128 heads
    ([900, 16, 17, 1, 400], 1, 16, 20, 512, F32),            # 20 of 32 vectors
    ([300, 2], 2, 256, 24, 256, F32),                        # 48 of 64
    ([1200, 31], 3, 16, 27, 512, F32),                       # 81 of 128
    ([20 + 37 * i for i in range(70)], 1, 32, 16, 256, BF),
    ([30 + i % 50 for i in range(260)], 1, 16, 4, 512, F32),
    ([1 + i % 41 for i in range(1024)], 1, 16, 3, 256, BF),
    ([12000], 1, 64, 64, 512, BF),
    ([500, 90], 5, 16, 40, 256, F32),                        # 200 vectors: two row groups
    ([2000, 33, 700], 8, 16, 128, 512, F32),                 # 1,024: eight
    ([130, 3], 6, 32, 32, 512, F32),                         # fewer rows than tokens in one
    ([35000], 1, 16, 2, 512, F32),                           # long shares over small pages
]


@pytest.mark.parametrize("case", range(len(DECODES)))
def test_decode(case):
    from paper_2609_34653_amd import omnitide as ot
    ctx, nq, P, H, R, dtype = DECODES[case]
    table, n_pages = layout(ctx, P, case)
    pool = pool_of(ctx, table, n_pages, P, R + E, case)
    q = queries(case, len(ctx), nq, H, R)
    got, st = decode(q.cuda(), pool.cuda(), table, ctx, SCALE, dtype)
    short = [0 < n < nq for n in ctx]
    assert st == (ot.E_CAPACITY if any(short) else 0)
    for s, n in enumerate(ctx):
        if short[s]:
            assert torch.isnan(got[s]).all()                 # not written
        elif n == 0:
            assert (got[s] == 0).all()
        else:
            rows = pool[table[s, np.arange(n) // P], np.arange(n) % P].double().numpy()
            want, spread = ol.absorbed_attention(f64(q[s]), rows, R, SCALE)
            near(got[s], want, spread, 2.0 ** -10, dtype)


@pytest.mark.parametrize("H", [16, 128])
@pytest.mark.parametrize("rise", [True, False])
def test_decode_large_and_equal_scores(H, rise):
    """Scores that rise over the keys (the reference moves), then all keys alike."""
    n, R, P = 1500, 256, 32
    table, n_pages = layout([n], P, 1)
    pool = pool_of([n], table, n_pages, P, R + E, 3)
    r = np.arange(n)
    ramp = torch.linspace(-3, 3, n) if rise else torch.zeros(n)
    pool[table[0, r // P], r % P] = ramp[:, None].expand(n, R + E).to(BF)
    q = torch.full((1, 1, H, R + E), 0.5, dtype=BF)
    got, st = decode(q.cuda(), pool.cuda(), table, [n], 1.0, F32)
    assert st == 0
    rows = pool[table[0, r // P], r % P].double().numpy()
    want, spread = ol.absorbed_attention(f64(q[0]), rows, R, 1.0)
    # scores up to 480, all partial sums exact to 2^-24 x 480 x 20 steps at most: 2^-10.8
    near(got[0], want, spread, 2.0 ** -10, F32)


@pytest.mark.parametrize("H", [3, 16, 33, 64, 80])
def test_decode_reference_moves_in_any_step(H):
    """Parts of several steps whose scores rise and fall by 30 per 32 keys, the other way for every other head: all
    sums are exact (multiples of 2^-5 below 2^11), rows of one score differ in pairs of dimensions."""
    S, n, R, P = 40, 1500, 256, 32
    ctx = [n - 7 * s for s in range(S)]
    table, n_pages = layout(ctx, P, 1)
    pool = pool_of(ctx, table, n_pages, P, R + E, 3)
    rng = np.random.default_rng(5)
    q = torch.full((S, 1, H, R + E), 0.5, dtype=BF)
    q[:, :, 1::2] = -0.5
    for s in range(S):
        r = np.arange(ctx[s])
        level = rng.permutation(47)[r // 32] if s % 2 else r // 32
        x = np.repeat((level * 3 / 16)[:, None], R + E, 1)
        sign = rng.integers(-1, 2, ctx[s])[:, None] / 16
        x[:, ::2] += sign
        x[:, 1::2] -= sign
        pool[table[s, r // P], r % P] = torch.from_numpy(x).to(BF)
    got, st = decode(q.cuda(), pool.cuda(), table, ctx, 1.0, F32)
    assert st == 0
    for s in range(S):
        r = np.arange(ctx[s])
        rows = pool[table[s, r // P], r % P].double().numpy()
        want, spread = ol.absorbed_attention(f64(q[s]), rows, R, 1.0)
        near(got[s], want, spread, 2.0 ** -10, F32)


def far_pool(table, small, used):
    """A pool of 7 GiB with the pages of `small` that `table` names at its end: the pool and its table."""
    P, W = small.shape[1:3]
    n = (7 << 30) // (P * small[0, 0].numel() * 2)
    pool = torch.empty((n, *small.shape[1:]), dtype=BF, device="cuda")
    shift = n - small.shape[0]
    pool[shift:] = small
    return pool, np.where(table >= 0, table + shift, table)


def test_pages_beyond_four_gib():
    """Each call on the last pages of a large pool gives the bits that it gives on a small one."""
    from paper_2609_34653_amd import latent as la, paged as pg
    ctx, new, P, R, H = [300, 77], [40, 1], 16, 512, 40
    table, n_pages = layout(ctx, P, 3)
    small = pool_of(ctx, table, n_pages, P, R + E, 1).cuda()
    large, far = far_pool(table, small, ctx)
    assert large.numel() * 2 > 7 * 10 ** 9
    T, th = sum(new), pg.omnitide_rope_thetas(1.0e4, E)
    c, e, q = rand(1, T, R).to(BF).cuda(), rand(2, T, E).to(BF).cuda(), queries(3, 2, 1, H, R).cuda()
    got = []
    for pool, tab in ((small, table), (large, far)):
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        la.omnitide_latent_append(c, e, pool, i32(tab), i32([0, 40, 41]), i32(ctx), theta=th, d_status=st)
        out = torch.zeros(sum(ctx), R + E, dtype=BF, device="cuda")
        la.omnitide_paged_rows(pool, i32(tab), i32([0, 300, 377]), i32(ctx), out, d_status=st)
        dec, code = decode(q, pool, tab, ctx, SCALE, F32)
        assert code == 0 and int(st.item()) == 0
        got.append((out, dec))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    assert torch.isfinite(got[0][1]).all()


@pytest.mark.parametrize("scale", [-0.05, 0.0])
def test_decode_scales(scale):
    ctx, P, R = [300, 40], 16, 512
    table, n_pages = layout(ctx, P, 1)
    pool = pool_of(ctx, table, n_pages, P, R + E, 3)
    q = queries(1, 2, 2, 16, R)
    got, st = decode(q.cuda(), pool.cuda(), table, ctx, scale, F32)
    for s, n in enumerate(ctx):
        rows = pool[table[s, np.arange(n) // P], np.arange(n) % P].double().numpy()
        want, spread = ol.absorbed_attention(f64(q[s]), rows, R, scale)
        near(got[s], want, spread, 2.0 ** -10, F32)


@pytest.mark.parametrize("what", ["page", "negative", "first", "low", "long"])
@pytest.mark.parametrize("H", [16, 64])
def test_decode_refused_on_the_device(what, H):
    from paper_2609_34653_amd import omnitide as ot, paged as pg
    ctx, P, R, nq = [300, 200, 400], 16, 256, 3
    table, n_pages = layout(ctx, P, 2)
    pool = torch.nan_to_num(pool_of(ctx, table, n_pages, P, R + E, 2), posinf=1.0)
    q = queries(4, 3, nq, H, R)
    given, bad, code = table.copy(), list(ctx), pg.E_PAGES
    if what == "page":
        given[1, 12] = n_pages                               # rows 192..199: seen by all three tokens
    elif what == "negative":
        given[1, 3] = -1
    elif what == "first":
        given[1, 0] = 1 << 30
    elif what == "low":
        bad[1], code = 2, ot.E_CAPACITY
    else:
        bad[1], code = given.shape[1] * P + 1, ot.E_CAPACITY
    got, st = decode(q.cuda(), pool.cuda(), given, bad, SCALE, F32)
    assert st == code and torch.isnan(got[1]).all()
    for s in (0, 2):
        rows = pool[table[s, np.arange(ctx[s]) // P], np.arange(ctx[s]) % P].double().numpy()
        want, spread = ol.absorbed_attention(f64(q[s]), rows, R, SCALE)
        near(got[s], want, spread, 2.0 ** -10, F32)


def test_decode_bad_page_seen_by_the_last_token_alone():
    from paper_2609_34653_amd import paged as pg
    n, P, R, nq, H = 193, 16, 256, 3, 16                     # the last row alone lies in the last page
    table, n_pages = layout([n], P, 2)
    pool = pool_of([n], table, n_pages, P, R + E, 2)
    q = queries(4, 1, nq, H, R)
    given = table.copy()
    given[0, 12] = -5
    got, st = decode(q.cuda(), pool.cuda(), given, [n], SCALE, F32)
    assert st == pg.E_PAGES and torch.isnan(got[0, 2]).all()
    rows = pool[table[0, np.arange(n - 1) // P], np.arange(n - 1) % P].double().numpy()
    want, spread = ol.absorbed_attention(f64(q[0, :2]), rows, R, SCALE)
    near(got[0, :2], want, spread, 2.0 ** -10, F32)


# ------------------------------------------------------------------------------------ chunk

def chunk(q, kv, kr, start, kv_start, scale, dtype, split=None):
    from paper_2609_34653_amd import latent as la
    T, H, w = q.shape
    d = w - E
    k, v = (kv[..., :d], kv[..., d:]) if split is None else split
    out = torch.full((T, H, d), float("nan"), dtype=dtype, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    nb = la.omnitide_latent_chunk_attn_workspace_bytes(T, len(start) - 1, k.shape[0], H, d)
    ws = torch.full((nb,), 0xff, dtype=torch.uint8, device="cuda")
    la.omnitide_latent_chunk_attn(q, k, v, kr, i32(start), i32(kv_start), scale, out, ws, st)
    torch.cuda.synchronize()
    return out, int(st.item())


CHUNKS = [
    # ctx, new, heads, d, out
    ([1], [1], 4, 64, F32),
    ([601], [89], 4, 64, BF),
    ([64, 65, 63, 128], [64, 65, 63, 1], 8, 64, F32),
    ([700], [129], 20, 128, F32),
    ([2100, 90, 1300], [130, 0, 7], 16, 128, BF),            # a sequence without tokens
    ([5000, 17], [3, 17], 4, 128, F32),
    ([33 * i + 1 for i in range(20)], [min(33 * i + 1, 5 * i + 1) for i in range(20)], 3, 64, F32),
    ([40 + i for i in range(70)], [1 + i % 3 for i in range(70)], 4, 128, BF),
    ([1030], [1030], 5, 128, F32),                           # a prompt
    ([9 + i % 3 for i in range(300)], [i % 3 for i in range(300)], 2, 128, F32),
    ([900, 830], [600, 600], 8, 128, F32),
    ([700], [700], 128, 64, F32),                            # more row tiles than workgroups
    ([600, 520], [520, 300], 64, 128, BF),
    ([320, 65], [257, 65], 1, 64, F32),
    ([9300], [7], 2, 64, BF),
]


@pytest.mark.parametrize("case", range(len(CHUNKS)))
def test_chunk(case):
    ctx, new, H, d, dtype = CHUNKS[case]
    start = np.concatenate([[0], np.cumsum(new)]) + 1        # padding in front, two behind
    rows = np.concatenate([[0], np.cumsum(ctx)]) + 2
    T, N = int(start[-1]) + 2, int(rows[-1]) + 1
    kv, kr = rand(case, N, H, 2 * d), rand(case + 90, N, 512 + E)
    kv[:2] = kv[-1] = float("nan")                           # rows of no sequence
    kr[:2] = kr[-1] = float("inf")
    kv, kr, q = kv.to(BF), kr.to(BF), rand(case + 7, T, H, d + E).to(BF)
    scale = (d + E) ** -0.5
    got, st = chunk(q.cuda(), kv.cuda(), kr.cuda()[:, 512:], start, rows, scale, dtype)
    assert st == 0
    for s, (n, m) in enumerate(zip(ctx, new)):
        if m == 0:
            continue
        r, t = slice(rows[s], rows[s + 1]), slice(start[s], start[s + 1])
        want, spread = ol.expanded_attention(f64(q[t]), f64(kv[r, :, :d]), f64(kv[r, :, d:]),
                                             f64(kr[r, 512:]), scale)
        near(got[t], want, spread, 2.0 ** -11, dtype)
    assert torch.isnan(got[0]).all() and torch.isnan(got[int(start[-1]):]).all()


def test_chunk_tensors_of_their_own():
    """Keys and values as separate tensors, heads strided, a contiguous rotated part."""
    n, m, H, d = 300, 70, 6, 64
    kv, kr, q = rand(1, n, H, 2 * d).to(BF), rand(2, n, E).to(BF), rand(3, m, H, d + E).to(BF)
    a, st = chunk(q.cuda(), kv.cuda(), kr.cuda(), [0, m], [0, n], 0.1, F32)
    wide = torch.full((n, H, d + 24), float("nan"), dtype=BF, device="cuda")
    wide[..., 8:8 + d] = kv[..., :d].cuda()
    b, st2 = chunk(q.cuda(), None, kr.cuda(), [0, m], [0, n], 0.1, F32,
                   split=(wide[..., 8:8 + d], kv[..., d:].contiguous().cuda()))
    assert st == 0 and st2 == 0 and torch.equal(a, b) and torch.isfinite(a).all()


def test_chunk_rows_far_apart():
    """The largest strides, 2^24 elements, so rows beyond 4 GiB: the bits of contiguous tensors."""
    n, T, H, d = 150, 70, 2, 64
    wide = torch.empty(n, 1 << 24, dtype=BF, device="cuda")
    kv, kr = rand(1, n, H, 2 * d).to(BF).cuda(), rand(2, n, E).to(BF).cuda()
    wide[:, :H * 2 * d] = kv.view(n, -1)
    wide[:, -E:] = kr
    q = rand(3, T, H, d + E).to(BF).cuda()
    got = []
    for x, r in ((kv, kr), (wide[:, :H * 2 * d].unflatten(1, (H, 2 * d)), wide[:, -E:])):
        out, st = chunk(q, x, r, [0, T], [0, n], SCALE, F32)
        assert st == 0
        got.append(out)
    assert torch.equal(got[0], got[1]) and torch.isfinite(got[0]).all()


@pytest.mark.parametrize("rise", [True, False])
def test_chunk_large_and_equal_scores(rise):
    n, m, H, d = 1500, 40, 3, 128
    ramp = (torch.linspace(-3, 3, n) if rise else torch.zeros(n))[:, None]
    kv = torch.cat([ramp[:, None].expand(n, H, d), rand(1, n, H, d)], -1).to(BF)
    kr = ramp.expand(n, E).to(BF).contiguous()
    q = torch.full((m, H, d + E), 0.5, dtype=BF)
    got, st = chunk(q.cuda(), kv.cuda(), kr.cuda(), [0, m], [0, n], 1.0, F32)
    want, spread = ol.expanded_attention(f64(q), f64(kv[..., :d]), f64(kv[..., d:]), f64(kr), 1.0)
    assert st == 0
    near(got, want, spread, 2.0 ** -10, F32)                 # scores up to 288


@pytest.mark.parametrize("what", ["few", "rows", "beyond", "order"])
def test_chunk_refused_on_the_device(what):
    from paper_2609_34653_amd import omnitide as ot, paged as pg
    n, H, d = [90, 60], 4, 64
    kv, kr, q = rand(1, 150, H, 2 * d).to(BF), rand(2, 150, E).to(BF), rand(3, 40, H, d + E).to(BF)
    start, rows, code = [0, 20, 40], [0, 90, 150], pg.E_PAGES
    if what == "few":
        rows, code = [0, 90, 100], ot.E_CAPACITY
    elif what == "rows":
        rows = [0, 90, 80]
    elif what == "beyond":
        rows = [0, 90, 151]
    else:
        start = [0, 20, 10]
    got, st = chunk(q.cuda(), kv.cuda(), kr.cuda(), start, rows, 0.1, F32)
    assert st == code and torch.isnan(got[20:]).all()
    want, spread = ol.expanded_attention(f64(q[:20]), f64(kv[:90, :, :d]), f64(kv[:90, :, d:]),
                                         f64(kr[:90]), 0.1)
    near(got[:20], want, spread, 2.0 ** -11, F32)


@pytest.mark.parametrize("start", [[0, 7, 3, 9], [0, 5, 0, 5, 0, 5], [2, 1 << 30, 3, 4], [-3, 4, 8]], ids=len)
def test_chunk_overlapping_offsets(start):
    """A sequence that starts in front of an earlier offset has no tokens."""
    from paper_2609_34653_amd import paged as pg
    S, T, H, d = len(start) - 1, 9, 2, 64
    rows = [20 * i for i in range(S + 1)]
    kv, kr, q = rand(1, 20 * S, H, 2 * d).to(BF), rand(2, 20 * S, E).to(BF), rand(3, T, H, d + E).to(BF)
    got, st = chunk(q.cuda(), kv.cuda(), kr.cuda(), start, rows, 0.1, F32)
    assert st == pg.E_PAGES
    top, written = 0, np.zeros(T, bool)
    for s in range(S):
        a, b = start[s:s + 2]
        if a >= max(top, 0) and a < b <= T and b - a <= 20:
            r = slice(rows[s], rows[s + 1])
            want, spread = ol.expanded_attention(f64(q[a:b]), f64(kv[r, :, :d]), f64(kv[r, :, d:]),
                                                 f64(kr[r]), 0.1)
            near(got[a:b], want, spread, 2.0 ** -11, F32)
            written[a:b] = True
        top = max(top, a)
    assert torch.isnan(got[~torch.from_numpy(written)]).all()


# --------------------------------------------------------------------------------- together

def test_both_forms_over_one_cache():
    """Two chunks appended, attended to in the expanded form; the last tokens again in the absorbed
    form: both against float64, and alike."""
    from paper_2609_34653_amd import latent as la, paged as pg
    R, H, d, P = 512, 8, 128, 32
    old, new = [150, 61], [70, 33]
    ctx = [a + b for a, b in zip(old, new)]
    table, n_pages = layout(ctx, P, 1)
    pool = torch.full((n_pages, P, R + E), float("nan"), dtype=BF, device="cuda")
    th = pg.omnitide_rope_thetas(1.0e4, E)
    w = torch.ones(R, dtype=BF, device="cuda")
    a = (rand(11, H, d, R) * R ** -0.5).to(BF).cuda()        # keys, and values, from latents
    b = (rand(12, H, d, R) * R ** -0.5).to(BF).cuda()
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = None
    for lens, n in ((old, old), (new, ctx)):
        T = sum(lens)
        kv = rand(T, T, R + E).to(BF).cuda()
        q = rand(T + 1, T, H, d + E).to(BF).cuda()
        start = np.concatenate([[0], np.cumsum(lens)])
        la.omnitide_latent_append(kv[:, :R], kv[:, R:], pool, i32(table), i32(start), i32(n), theta=th,
                                  latent_weight=w, q_rope=q[..., d:], q_out=q[..., d:], d_status=st)
    rows_at = np.concatenate([[0], np.cumsum(ctx)])
    rows = torch.empty(sum(ctx), R + E, dtype=BF, device="cuda")
    la.omnitide_paged_rows(pool, i32(table), i32(rows_at), i32(ctx), rows, st)
    weight = torch.cat([a, b], 1).flatten(0, 1)              # [H * 2d, R]: the up projection
    kv = (rows[:, :R].float() @ weight.float().t()).to(BF).view(-1, H, 2 * d)
    got, status = chunk(q, kv, rows[:, R:], start, rows_at, SCALE, F32)
    assert status == 0 and int(st.item()) == 0
    for s in range(2):
        r, t = slice(rows_at[s], rows_at[s + 1]), slice(start[s], start[s + 1])
        want, spread = ol.expanded_attention(f64(q[t]), f64(kv[r, :, :d]), f64(kv[r, :, d:]),
                                             f64(rows[r, R:]), SCALE)
        near(got[t], want, spread, 2.0 ** -11, F32)
    # the last two tokens of each stream, absorbed
    last = torch.stack([q[start[s + 1] - 2:start[s + 1]] for s in range(2)])       # [S, 2, H, d + E]
    ql = torch.matmul(last[..., :d].float().unsqueeze(3), a.float()).squeeze(3)    # A^T n
    lat, status = decode(torch.cat([ql.to(BF), last[..., d:]], -1), pool, table, ctx, SCALE, F32)
    assert status == 0
    o = torch.matmul(b.float(), lat.unsqueeze(-1)).squeeze(-1)                      # B c
    both = torch.stack([got[start[s + 1] - 2:start[s + 1]] for s in range(2)])
    # the forms differ by the rounding of the expanded keys, values and absorbed queries to bf16 (2^-8 of
    # scores of about one, and of values)
    assert (o - both).abs().max() < 2.0 ** -5 and (o - both).abs().mean() < 2.0 ** -8


def test_streams_and_captured_calls():
    """A side stream, and a captured graph of append, rows and both attentions, replayed with other lengths and
    pages between eager work: every replay as the eager calls."""
    from paper_2609_34653_amd import latent as la, paged as pg
    R, H, d, P, S = 512, 16, 64, 16, 3
    lens = [[100, 33, 7], [64, 0, 90], [1, 120, 16]]
    mp = 8
    pool = rand(1, S * mp + 1, P, R + E).to(BF).cuda()
    th = pg.omnitide_rope_thetas(1.0e4, E)
    kv, q = rand(2, S, R + E).to(BF).cuda(), rand(3, S, H, R + E).to(BF).cuda()
    qc, exp = rand(4, S, H, d + E).to(BF).cuda(), rand(5, S * 128, H, 2 * d).to(BF).cuda()
    tables = [i32(np.random.default_rng(i).permutation(S * mp).reshape(S, mp)) for i in range(3)]
    table, ctx = tables[0].clone(), i32(lens[0])
    start = i32(range(S + 1))                                # (idle sequences: fewer rows than tokens)
    row_start = torch.zeros(S + 1, dtype=torch.int32, device="cuda")
    out = torch.zeros(S, 1, H, R, device="cuda")
    outc = torch.zeros(S, H, d, device="cuda")
    rows = torch.zeros(S * 128, R + E, dtype=BF, device="cuda")
    ws = torch.empty(la.omnitide_latent_decode_workspace_bytes(S, 1, mp * P, H, R), dtype=torch.uint8,
                     device="cuda")
    wc = torch.empty(la.omnitide_latent_chunk_attn_workspace_bytes(S, S, S * 128, H, d), dtype=torch.uint8,
                     device="cuda")

    def calls():
        la.omnitide_latent_append(kv[:, :R], kv[:, R:], pool, table, start, ctx, theta=th)
        la.omnitide_paged_rows(pool, table, row_start, ctx, rows)
        la.omnitide_latent_decode_attn(q.view(S, 1, H, R + E), pool, table, ctx, SCALE, out, ws)
        la.omnitide_latent_chunk_attn(qc, exp[..., :d], exp[..., d:], rows[:, R:], start, row_start, 0.1,
                                      outc, wc)

    def load(i):
        table.copy_(tables[i]), ctx.copy_(i32(lens[i]))
        row_start.copy_(i32(np.concatenate([[0], np.cumsum(lens[i])])))
        rows.zero_(), outc.zero_()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        load(0)
        calls()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls()
    for i in (1, 2, 0, 1):
        load(i)
        g.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (pool, rows, out, outc)]
        load(i)
        calls()
        torch.cuda.synchronize()
        for x, y in zip(got, (pool, rows, out, outc)):
            assert torch.equal(x, y)


# ------------------------------------------------------------------- probabilities of 16 bits
#
# Scores are whole numbers, exact in float, so what is left is, with S as above:
#   2^-16 S    each probability entered as its bf16 rounding and that of the remainder: half a step of half a step
#   2^-16 S    the exponential's argument, |x| log2(e) <= 110 on these inputs with the scale's and the fused product's
#              roundings: 110 x 1.5 x ln 2 x 2^-23 = 2^-16.2, and 2^-22 of the exponential
#   2^-15 S    sums of up to 300 products in float, above and below the line: 2 x 300 x 2^-24 = 2^-14.8 at most
# below 2^-14 S together; probabilities rounded to bf16 once are off by up to 2^-8 S.

def close_bits(got, want, spread):
    err = np.abs(f64(got) - want)
    assert np.isfinite(f64(got)).all()
    assert (err <= 2.0 ** -14 * spread).all(), float((err / np.maximum(spread, 1e-30)).max())


def whole_parts(seed, n, rise):
    """Rotated parts [n, 64] of whole numbers; rising ones move the reference in the middle of a part."""
    e = torch.randint(-2, 3, (n, E), generator=torch.Generator().manual_seed(seed)).float()
    if rise:
        e[:, 0] = torch.arange(n) // 8
    return e


def whole_queries(seed, shape, rise):
    q = torch.randint(-2, 3, (*shape, E), generator=torch.Generator().manual_seed(seed)).float()
    if rise:
        q[..., 0] = 8.0
    return q


@pytest.mark.parametrize("rise", [False, True])
@pytest.mark.parametrize("ctx,nq,H,R", [
    ([1, 2, 3, 40, 0, 300], 1, 16, 512),
    ([5, 37, 129, 290], 2, 20, 256),                         # both tiles of vectors
    ([260, 9], 1, 128, 512),                                 # two row groups
    ([7 + 3 * i for i in range(70)], 1, 4, 512),
])
def test_decode_probabilities_keep_16_bits(ctx, nq, H, R, rise):
    P = 16
    table, n_pages = layout(ctx, P, H)
    pool = pool_of(ctx, table, n_pages, P, R + E, H)
    q = torch.cat([torch.zeros(len(ctx), nq, H, R), whole_queries(H, (len(ctx), nq, H), rise)], -1).to(BF)
    for s, n in enumerate(ctx):
        r = np.arange(n)
        if n:
            pool[table[s, r // P], r % P, R:] = whole_parts(s, n, rise).to(BF)
    got, st = decode(q.cuda(), pool.cuda(), table, ctx, 0.125, F32)
    assert st == 0
    for s, n in enumerate(ctx):
        if n == 0:
            continue
        rows = pool[table[s, np.arange(n) // P], np.arange(n) % P].double().numpy()
        want, spread = ol.absorbed_attention(f64(q[s]), rows, R, 0.125)
        close_bits(got[s], want, spread)


@pytest.mark.parametrize("rise", [False, True])
@pytest.mark.parametrize("ctx,new,H,d", [
    ([1, 2, 3, 40, 300], [1, 2, 3, 7, 30], 4, 128),
    ([290, 129], [1, 129], 5, 64),
    ([280], [280], 16, 128),
])
def test_chunk_probabilities_keep_16_bits(ctx, new, H, d, rise):
    start, rows = np.concatenate([[0], np.cumsum(new)]), np.concatenate([[0], np.cumsum(ctx)])
    T, N = int(start[-1]), int(rows[-1])
    kv = rand(H, N, H, 2 * d).to(BF)
    kr = torch.cat([whole_parts(s, n, rise) for s, n in enumerate(ctx)]).to(BF)
    q = torch.cat([torch.zeros(T, H, d), whole_queries(H, (T, H), rise)], -1).to(BF)
    got, st = chunk(q.cuda(), kv.cuda(), kr.cuda(), start, rows, 0.125, F32)
    assert st == 0
    for s in range(len(ctx)):
        r, t = slice(rows[s], rows[s + 1]), slice(start[s], start[s + 1])
        want, spread = ol.expanded_attention(f64(q[t]), f64(kv[r, :, :d]), f64(kv[r, :, d:]), f64(kr[r]), 0.125)
        close_bits(got[t], want, spread)


# ----------------------------------------------------------------------- promises of the headers

@pytest.mark.parametrize("scale", [-0.05, 0.0])
def test_chunk_scales(scale):
    n, m, H, d = [300, 40], [70, 40], 4, 64
    start, rows = [0, 70, 110], [0, 300, 340]
    kv, kr, q = rand(1, 340, H, 2 * d).to(BF), rand(2, 340, E).to(BF), rand(3, 110, H, d + E).to(BF)
    got, st = chunk(q.cuda(), kv.cuda(), kr.cuda(), start, rows, scale, F32)
    assert st == 0
    for s in range(2):
        r, t = slice(rows[s], rows[s + 1]), slice(start[s], start[s + 1])
        want, spread = ol.expanded_attention(f64(q[t]), f64(kv[r, :, :d]), f64(kv[r, :, d:]), f64(kr[r]), scale)
        near(got[t], want, spread, 2.0 ** -11, F32)


@pytest.mark.parametrize("start,refused", [([0, 0, 0], False), ([3, 3, 3], False), ([0, 2, 2], True)])
def test_chunk_of_padding_alone(start, refused):
    """No rows: nothing is written, and a sequence that has tokens all the same is refused on the device."""
    from paper_2609_34653_amd import omnitide as ot
    H, d = 4, 64
    none = torch.empty(0, H, 2 * d, dtype=BF, device="cuda")
    got, st = chunk(rand(1, 5, H, d + E).to(BF).cuda(), none, none[:, 0, :E], start, [0, 0, 0], 0.1, F32)
    assert st == (ot.E_CAPACITY if refused else 0) and torch.isnan(got).all()


def test_append_with_offsets_out_of_order():
    """Tokens that lie in the offsets of a sequence go to their rows there, each once; no other row changes."""
    from paper_2609_34653_amd import latent as la, paged as pg
    ctx, P, R, start = [40, 33, 20], 16, 256, [0, 5, 3, 12]
    kv = rand(1, 12, R + E).to(BF).cuda()
    table, n_pages = layout(ctx, P, 3)
    pool = torch.full((n_pages, P, R + E), 9.0, dtype=BF, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    la.omnitide_latent_append(kv[:, :R], kv[:, R:], pool, i32(table), i32(start), i32(ctx), d_status=st)
    assert int(st.item()) == pg.E_PAGES
    want = torch.full_like(pool, 9.0)
    for t in range(12):
        s = 0 if t < 5 else 2                                # the first sequence whose offsets hold the token
        r = ctx[s] - (start[s + 1] - t)
        want[int(table[s, r // P]), r % P] = kv[t]
    assert torch.equal(pool, want)
