"""Chunk and decode attention over the pages against float64.

Tolerances, per element, with S = sum_j p_j |v_j| + |out| (what an error of the probabilities acts
on: out' - out = sum_j dp_j (v_j - out)):
  chunk   2^-8 S (each probability rounded to bf16 once, half a step; the sum uses the rounded ones)
  decode  2^-16 S (bf16 plus bf16 remainder)
  both    + 2^-12 S for the scores: products of bf16 are exact in float, the sum of d <= 128 of them is off
          by at most 128 x 2^-24 sum|q k|; sum|q k| scale <= 20 on these inputs, so a probability by 2^-12.6;
          the exponential and the sums add 2^-18
          + the rounding of a bf16 output, 2^-8 |out| (half a step)."""
import numpy as np
import pytest
import torch

import oracle
from oracle import paged as op
from tests.test_gpu_norm_rope import BF, F32, f64, i32, layout

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_34653_amd import paged
    paged.lib()
    yield


def pools(ctx, table, n_pages, P, hkv, d, seed):
    """Pools whose rows in use are normal and whose other rows are NaN and infinities."""
    g = torch.Generator().manual_seed(seed)
    kp = torch.full((n_pages, P, hkv, d), float("nan"))
    vp = torch.full((n_pages, P, hkv, d), float("inf"))
    vp[:, ::2] = float("nan")
    for s, n in enumerate(ctx):
        r = np.arange(n)
        page, line = table[s, r // P] if n else r, r % P
        kp[page, line] = torch.randn(n, hkv, d, generator=g)
        vp[page, line] = torch.randn(n, hkv, d, generator=g)
    return kp.to(BF), vp.to(BF)


def run(decode, q, kp, vp, table, start, ctx, scale, out_dtype, ws_fill=0xff):
    from paper_2609_34653_amd import paged as pg
    hkv, d, P = kp.shape[2], kp.shape[3], kp.shape[1]
    out = torch.full(q.shape, float("nan"), dtype=out_dtype, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    cap = table.shape[1] * P
    if decode:
        nb = pg.omnitide_paged_decode_workspace_bytes(q.shape[0], q.shape[1], cap, q.shape[2], hkv, d)
    else:
        nb = pg.omnitide_paged_chunk_attn_workspace_bytes(q.shape[0], len(ctx), cap, q.shape[1], hkv, d)
    ws = torch.full((nb,), ws_fill, dtype=torch.uint8, device="cuda") if nb else None
    if decode:
        pg.omnitide_paged_decode_attn(q, kp, vp, i32(table), i32(ctx), scale, out, ws, st)
    else:
        pg.omnitide_paged_chunk_attn(q, kp, vp, i32(table), i32(start), i32(ctx), scale, out, ws, st)
    torch.cuda.synchronize()
    return out, int(st.item())


def assert_near(got, want, spread, p_step, dtype):
    tol = (p_step + 2.0 ** -12) * spread
    if dtype == BF:
        tol = tol + torch.finfo(BF).eps / 2 * (np.abs(want) + tol)
    err = np.abs(f64(got) - want)
    assert np.isfinite(f64(got)).all()
    assert (err <= tol).all(), (float(err.max()), float((err / np.maximum(tol, 1e-30)).max()))


CHUNKS = [
    # (ctx, new, page, hq, hkv, d, out)
    ([1], [1], 16, 4, 1, 64, F32),
    ([601], [89], 32, 4, 1, 64, BF),
    ([64, 65, 63, 128], [64, 65, 63, 1], 64, 8, 8, 64, F32),
    ([700], [129], 16, 28, 4, 128, F32),                     # 7 heads per KV head, ragged rows
    ([2100, 90, 1300], [130, 0, 7], 128, 32, 8, 128, BF),    # a sequence without tokens
    ([5000, 17], [3, 17], 256, 16, 2, 128, F32),             # few tokens over a long context
    ([33 * i + 1 for i in range(20)], [min(33 * i + 1, 5 * i + 1) for i in range(20)], 16, 14, 2, 64,
     F32),
    ([40 + i for i in range(70)], [1 + i % 3 for i in range(70)], 32, 4, 1, 128, BF),
    ([1030], [1030], 64, 16, 4, 128, F32),                   # a prompt: no context before it
    ([9 + i % 3 for i in range(300)], [i % 3 for i in range(300)], 16, 8, 4, 64, F32),
    ([900, 830], [600, 600], 64, 8, 8, 128, F32),            # row tiles alike, cut into even parts
    ([1400, 1390, 1410], [700, 710, 690], 32, 32, 8, 64, F32),   # more row tiles than workgroups
    ([2300], [2300], 64, 32, 8, 64, BF),                     # as many, of unequal work
    ([3000, 600, 40, 2000], [1500, 600, 40, 1], 16, 32, 16, 64, F32),   # and of unequal sequences
    ([4000, 2500], [300, 77], 256, 15, 3, 64, BF),           # 3 KV heads, 5 query heads on each
    ([700, 3], [90, 3], 16, 32, 32, 128, F32),               # a key head per query head
    ([1 + i % 23 for i in range(1024)], [(1 + i % 23) * (i % 5 > 0) // 2 for i in range(1024)], 16, 4,
     1, 64, F32),
    ([6000], [40], 16, 40, 1, 128, F32),                     # 40 query heads on one
]


@pytest.mark.parametrize("case", range(len(CHUNKS)))
def test_chunk(case):
    ctx, new, P, hq, hkv, d, out = CHUNKS[case]
    table, n_pages = layout(ctx, P, case)
    start = np.concatenate([[0], np.cumsum(new)]) + 1        # padding in front, two behind
    T = int(start[-1]) + 2
    kp, vp = pools(ctx, table, n_pages, P, hkv, d, case)
    q = torch.randn(T, hq, d, generator=torch.Generator().manual_seed(case)).to(BF)
    got, st = run(False, q.cuda(), kp.cuda(), vp.cuda(), table, start, ctx, d ** -0.5, out)
    assert st == 0
    want, spread = op.ragged_attention(f64(q), f64(kp), f64(vp), table, start, ctx, d ** -0.5)
    real = slice(int(start[0]), int(start[-1]))
    assert_near(got[real], want[real], spread[real], 2.0 ** -8, out)
    assert torch.isnan(got[0]).all() and torch.isnan(got[int(start[-1]):]).all()


SMALLER = len(CHUNKS)
CHUNKS += [
    # d = 128: a whole row tile per workgroup, 8 to 64 more cut into shares, past 64 pages on the way; two
    # whole ones and half as many more
    ([1400, 1390, 1410], [700, 710, 690], 16, 32, 8, 128, F32),
    ([1700, 400, 2200], [1200, 30, 1050], 16, 32, 16, 128, BF),
    ([2113], [1088], 32, 64, 16, 128, F32),
    ([640, 600], [600, 600], 64, 128, 32, 128, F32),
    ([4700, 2300], [33, 65], 16, 16, 2, 128, F32),           # parts of a few tiles, and past 64 pages
    ([9300], [7], 16, 8, 8, 128, BF),
]


@pytest.mark.parametrize("case", range(SMALLER, len(CHUNKS)))
def test_chunk_large_heads(case):
    """Rounds of whole row tiles, shares after them and many pages at d = 128."""
    test_chunk(case)


DECODES = [
    ([1], 1, 16, 4, 1, 64, F32),
    ([777], 1, 64, 32, 8, 128, F32),
    ([5000, 0, 63, 2048], 2, 128, 16, 8, 128, BF),           # an idle sequence
    ([129, 4, 40], 4, 16, 8, 4, 64, F32),                    # four tokens, causal among them
    ([3001, 64, 65], 1, 32, 16, 1, 64, F32),                 # 16 query heads on one KV head
    ([900, 16, 17, 1, 400], 1, 16, 28, 4, 128, F32),
    ([20 + 37 * i for i in range(70)], 1, 32, 16, 2, 128, BF),
    ([300, 2], 2, 256, 14, 2, 64, F32),
    ([30 + i % 50 for i in range(260)], 1, 16, 4, 2, 64, F32),
    ([12000], 1, 64, 32, 8, 128, BF),
    ([2900, 1, 700], 3, 32, 15, 3, 64, F32),                 # 3 KV heads; one row, three tokens
    ([50 + i % 41 for i in range(1024)], 1, 16, 3, 3, 64, BF),
    ([400, 90], 1, 16, 32, 32, 128, F32),
]


@pytest.mark.parametrize("case", range(len(DECODES)))
def test_decode(case):
    ctx, nq, P, hq, hkv, d, out = DECODES[case]
    table, n_pages = layout(ctx, P, case)
    kp, vp = pools(ctx, table, n_pages, P, hkv, d, case)
    S = len(ctx)
    q = torch.randn(S, nq, hq, d, generator=torch.Generator().manual_seed(case)).to(BF)
    got, st = run(True, q.cuda(), kp.cuda(), vp.cuda(), table, None, ctx, d ** -0.5, out)
    from paper_2609_34653_amd import omnitide as ot
    short = [0 < n < nq for n in ctx]                        # fewer rows than new tokens: refused
    assert st == (ot.E_CAPACITY if any(short) else 0)
    for s, n in enumerate(ctx):
        if short[s]:
            assert torch.isnan(got[s]).all()                 # not written
            continue
        if n == 0:
            assert (got[s] == 0).all()
            continue
        want, spread = op.ragged_attention(f64(q[s]), f64(kp), f64(vp), table[s:s + 1], [0, nq], [n],
                                           d ** -0.5)
        assert_near(got[s], want, spread, 2.0 ** -16, out)


LONG = [
    # (ctx, nq, page, KV heads, d, out): blocks of 16 keys of a share (two workgroups' per CU over the KV
    # heads), so a quarter of them of a wave
    ([18001, 9003, 8101], 2, 16, 64, 64, F32),      # 279: 70, 70, 70 and 69 blocks of a wave
    ([35400, 777], 1, 32, 64, 64, BF),              # 286: 72, 72, 71, 71
    ([30001, 5701, 17], 1, 16, 64, 64, F32),        # 284: 71 each
    ([40001, 33100], 1, 16, 32, 128, F32),          # 288: 72 each, two blocks in flight of each
    ([69703, 300, 17], 1, 64, 32, 128, BF),         # 276: 69 each
]


@pytest.mark.parametrize("bad", [False, True])
@pytest.mark.parametrize("case", range(len(LONG)))
def test_decode_long_shares(case, bad):
    """Waves with more blocks than the 64 page ids they hold, and many turns of their rings, which begin
    and end at every place of the ring; with a bad page among the second 64 ids."""
    from paper_2609_34653_amd import paged as pg
    ctx, nq, P, hkv, d, out = LONG[case]
    share = max(8, -(-sum(12 + -(-n // 16) for n in ctx) // (512 // hkv)))
    assert share - 12 > 4 * 64                              # so the first part has more than 64 of a wave
    table, n_pages = layout(ctx, P, case)
    g = torch.Generator(device="cuda").manual_seed(case)
    kp, vp = (torch.randn(n_pages, P, hkv, d, generator=g, device="cuda", dtype=BF) for _ in range(2))
    for s, n in enumerate(ctx):
        if n % P:
            kp[table[s, n // P], n % P:] = float("nan")
            vp[table[s, n // P], n % P:] = float("inf")
    q = torch.randn(len(ctx), nq, hkv, d, generator=g, device="cuda").to(BF)
    given = table.copy()
    if bad:
        given[0, (4 * 65 + 2) * 16 // P] = -1
    got, st = run(True, q, kp, vp, given, None, ctx, d ** -0.5, out)
    assert st == (pg.E_PAGES if bad else 0)
    heads = [0, 1, hkv // 2, hkv - 1]
    for s, n in enumerate(ctx):
        if bad and s == 0:
            assert torch.isnan(got[s]).all()
            continue
        pages = torch.from_numpy(table[s, :-(-n // P)]).long().cuda()
        k, v = (f64(p[pages][:, :, heads].flatten(0, 1)[:n]) for p in (kp, vp))
        qs = f64(q[s][:, heads])
        want = oracle.chunk_attention(qs, k, v, d ** -0.5)
        spread = oracle.chunk_attention(qs, k, np.abs(v), d ** -0.5) + np.abs(want)
        assert_near(got[s][:, heads], want, spread, 2.0 ** -16, out)
        assert torch.isfinite(got[s]).all()


@pytest.mark.parametrize("decode", [False, True])
def test_large_scores_and_equal_scores(decode):
    """Scores far from zero and a long rise (the running maximum moves), then all keys alike."""
    n, d = 1500, 64
    table, n_pages = layout([n], 32, 1)
    kp, vp = pools([n], table, n_pages, 32, 1, d, 3)
    q = torch.ones(1, 4, d, dtype=BF)
    r = np.arange(n)
    for rise in (True, False):
        ramp = torch.linspace(-3, 3, n) if rise else torch.zeros(n)
        kp[table[0, r // 32], r % 32] = ramp[:, None, None].expand(n, 1, d).to(BF)
        qq = q.view(1, 1, 4, d) if decode else q
        got, st = run(decode, qq.cuda(), kp.cuda(), vp.cuda(), table, [0, 1], [n], 1.0, F32)
        assert st == 0
        want, spread = op.ragged_attention(f64(q), f64(kp), f64(vp), table, [0, 1], [n], 1.0)
        # scores up to 192: the rounding of a float score, 2^-24 x 192 x (partial sums) < 2^-11
        err = np.abs(f64(got).reshape(want.shape) - want)
        assert (err <= (2.0 ** -8 + 2.0 ** -9) * spread).all()


def test_chunk_over_pages_in_order_is_chunk_attention():
    """A compacted pool is a paged one with its pages in order."""
    from paper_2609_34653_amd import omnitide as ot
    n, L, hq, hkv, d, P = 3000, 150, 32, 8, 128, 64
    cap = -(-n // P) * P
    g = torch.Generator().manual_seed(0)
    k, v = (torch.randn(1, cap, hkv, d, generator=g).to(BF).cuda() for _ in range(2))
    q = torch.randn(1, L, hq, d, generator=g).to(BF).cuda()
    ref = torch.zeros(1, L, hq, d, device="cuda")
    ws = torch.zeros(max(1, ot.omnitide_attn_workspace_bytes(1, cap, L, hq, hkv, d)),
                     dtype=torch.uint8, device="cuda")
    ot.omnitide_chunk_attn(q, k, v, i32([n]), d ** -0.5, ref, ws)
    got, st = run(False, q[0], k.view(-1, P, hkv, d), v.view(-1, P, hkv, d),
                  np.arange(cap // P)[None], [0, L], [n], d ** -0.5, F32)
    want, spread = op.ragged_attention(f64(q[0]), f64(k).reshape(-1, P, hkv, d),
                                       f64(v).reshape(-1, P, hkv, d), np.arange(cap // P)[None],
                                       [0, L], [n], d ** -0.5)
    assert st == 0
    assert_near(got, want, spread, 2.0 ** -8, F32)
    assert_near(ref[0], want, spread, 2.0 ** -8, F32)


@pytest.mark.parametrize("decode", [False, True])
@pytest.mark.parametrize("what", ["page", "negative", "low", "long", "order"])
def test_device_refusals(decode, what):
    """Reported on the device; the sequences that are right come out right."""
    from paper_2609_34653_amd import omnitide as ot, paged as pg
    if decode and what == "order":
        return
    ctx, P, hq, hkv, d, new = [300, 200], 32, 4, 1, 64, 2
    table, n_pages = layout(ctx, P, 2)
    kp, vp = pools(ctx, table, n_pages, P, hkv, d, 2)
    q = torch.randn(4, hq, d).to(BF)
    want, spread = op.ragged_attention(f64(q), f64(kp), f64(vp), table, [0, 2, 4], ctx, 0.125)
    bad, start, code = list(ctx), [0, 2, 4], pg.E_PAGES
    if what == "page":
        table[1, 3] = n_pages
    elif what == "negative":
        table[1, 0] = -1
    elif what == "low":
        bad[1], code = 1, ot.E_CAPACITY
    elif what == "long":
        bad[1], code = table.shape[1] * P + 1, ot.E_CAPACITY
    else:
        start = [0, 2, 1]
    qq = q.view(2, 2, hq, d) if decode else q
    got, st = run(decode, qq.cuda(), torch.nan_to_num(kp).cuda(), torch.nan_to_num(vp).cuda(), table,
                  start, bad, 0.125, F32)
    assert st == code
    got = got.view(4, hq, d)
    assert_near(got[:2], want[:2], spread[:2], 2.0 ** -8, F32)
    if what in ("low", "long", "order"):
        assert torch.isnan(got[2:]).all()                    # not written


@pytest.mark.parametrize("start", [[0, 7, 3, 9], [0, 5, 0, 5, 0, 5], [2, 1 << 30, 3, 4], [-3, 4, 8],
                                   [0] + 99 * [6] + [2] + 39 * [8]], ids=len)
def test_overlapping_offsets(start):
    """A sequence that starts in front of an earlier offset has no tokens: no output is written by two,
    and the work is bounded by the tokens."""
    from paper_2609_34653_amd import paged as pg
    n_seq, T, hq, hkv, d, P = len(start) - 1, 9, 4, 2, 64, 16
    ctx = [40 + 3 * (i % 7) for i in range(n_seq)]
    table, n_pages = layout(ctx, P, n_seq)
    kp, vp = pools(ctx, table, n_pages, P, hkv, d, n_seq)
    q = torch.randn(T, hq, d, generator=torch.Generator().manual_seed(n_seq)).to(BF)
    got, st = run(False, q.cuda(), kp.cuda(), vp.cuda(), table, start, ctx, 0.125, F32)
    assert st == pg.E_PAGES
    written, top = np.zeros(T, bool), 0
    for s in range(n_seq):
        a, b = start[s:s + 2]
        if top <= a < b <= T:
            want, spread = op.ragged_attention(f64(q[a:b]), f64(kp), f64(vp), table[s:s + 1],
                                               [0, b - a], [ctx[s]], 0.125)
            assert_near(got[a:b], want, spread, 2.0 ** -8, F32)
            written[a:b] = True
        top = max(top, a)
    assert torch.isnan(got[torch.from_numpy(~written).cuda()]).all()


BAD_PAGES = [
    # (decode, ctx, new, page, hq, hkv, d, (sequence, page of it, id) ...)
    (True, [300, 498], [4, 4], 16, 4, 1, 64, (1, 31, -1)),            # seen by the last two tokens
    (True, [90, 2000, 40], [1, 1, 1], 16, 16, 2, 128, (1, 0, 1 << 30), (2, 2, -(1 << 31))),
    (True, [12000, 700], [2, 2], 64, 32, 8, 128, (0, 100, -5)),       # in one of many shares
    (True, [3000, 64], [8, 8], 256, 8, 8, 64, (0, 10, 1 << 20), (0, 11, 1 << 20)),
    (False, [1500, 200], [700, 30], 16, 8, 8, 64, (0, 70, -1)),       # among the second 64 pages
    (False, [1500, 200], [700, 30], 16, 8, 8, 128, (0, 64, 1 << 30)),         # the first of them
    (False, [1500, 200], [700, 30], 16, 8, 8, 64, (0, 63, -1), (0, 64, -1), (1, 0, -7)),
    (False, [6000, 77], [40, 5], 16, 4, 1, 64, (0, 373, -1)),         # short parts
    (False, [6000, 77], [40, 5], 16, 4, 1, 128, (0, 200, -1)),        # all tokens, in one part
    (False, [1000, 900], [600, 1], 256, 8, 2, 128, (0, 2, 1 << 30)),
    (False, [1400, 1390], [700, 710], 16, 32, 16, 128, (1, 80, -1)),  # whole row tiles
    (False, [130, 129, 64], [130, 129, 64], 64, 4, 2, 64, (0, 1, -1), (1, 2, -1)),
]


@pytest.mark.parametrize("case", range(len(BAD_PAGES)))
def test_rows_of_a_bad_page(case):
    """Tokens that see a row of a page that is not there come out as NaN; every other one, of the same
    sequence too, comes out right: no other page's rows are attended to in its place."""
    from paper_2609_34653_amd import paged as pg
    decode, ctx, new, P, hq, hkv, d, *bad = BAD_PAGES[case]
    table, n_pages = layout(ctx, P, case)
    kp, vp = pools(ctx, table, n_pages, P, hkv, d, case)
    start = np.concatenate([[0], np.cumsum(new)])
    q = torch.randn(int(start[-1]), hq, d, generator=torch.Generator().manual_seed(case)).to(BF)
    want, spread = op.ragged_attention(f64(q), f64(kp), f64(vp), table, start, ctx, d ** -0.5)
    spoilt = np.zeros(len(q), bool)
    for s, page, no in bad:
        table[s, page] = no
        row = ctx[s] - new[s] + np.arange(new[s])
        spoilt[start[s]:start[s + 1]] |= row >= page * P
    assert spoilt.any() and not spoilt.all()
    for dtype in (F32, BF):
        got, st = run(decode, (q.view(len(ctx), -1, hq, d) if decode else q).cuda(), kp.cuda(),
                      vp.cuda(), table, start, ctx, d ** -0.5, dtype)
        assert st == pg.E_PAGES
        got = got.view(want.shape)
        assert torch.isnan(got[torch.from_numpy(spoilt).cuda()]).all()
        keep = torch.from_numpy(~spoilt).cuda()
        assert_near(got[keep], want[~spoilt], spread[~spoilt], 2.0 ** -8, dtype)


@pytest.mark.parametrize("decode", [False, True])
def test_past_four_gigabytes(decode):
    """Pages whose byte offset passes 32 bits, and their order reversed."""
    P, hkv, d, hq = 128, 16, 128, 32
    n_pages = (9 << 29) // (P * hkv * d * 2)
    n = 5 * P + 37
    table = (n_pages - 1 - np.arange(6))[None].astype(np.int32)
    g = torch.Generator(device="cuda").manual_seed(1)
    kp = torch.zeros(n_pages, P, hkv, d, dtype=BF, device="cuda")
    vp = torch.zeros_like(kp)
    kp[-6:] = torch.randn(6, P, hkv, d, generator=g, device="cuda").to(BF)
    vp[-6:] = torch.randn(6, P, hkv, d, generator=g, device="cuda").to(BF)
    q = torch.randn(2, hq, d, generator=g, device="cuda").to(BF)
    got, st = run(decode, q.view(1, 2, hq, d) if decode else q, kp, vp, table, [0, 2], [n], 0.1, F32)
    want, spread = op.ragged_attention(f64(q), f64(kp[-6:]), f64(vp[-6:]), [[5, 4, 3, 2, 1, 0]],
                                       [0, 2], [n], 0.1)
    assert st == 0
    assert_near(got.view(2, hq, d), want, spread, 2.0 ** -8, F32)


class Streams:
    """Three streams served together over one pool: chunks appended and attended to in turn, then
    single tokens, with norms and rotation; everything also kept in float64 for the oracle."""

    def __init__(self, hq=8, hkv=2, d=64, P=16, seed=0):
        from paper_2609_34653_amd import paged as pg
        self.hq, self.hkv, self.d, self.P = hq, hkv, d, P
        self.max_pages = 20
        n_pages = 3 * self.max_pages
        self.order = np.random.default_rng(seed).permutation(n_pages).reshape(3, -1).astype(np.int32)
        self.table = i32(self.order)
        self.kp, self.vp = torch.full((2, n_pages, P, hkv, d), float("nan"), dtype=BF, device="cuda")
        self.theta = pg.omnitide_rope_thetas(1.0e4, d, pg.ROPE_RAMP, 4.0, 100.0, 1.0, 8.0)
        g = torch.Generator().manual_seed(seed)
        self.wq, self.wk = ((1 + 0.2 * torch.randn(d, generator=g)).to(BF).cuda() for _ in range(2))
        self.g = g
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def inputs(self, T):
        x = torch.randn(T, self.hq + 2 * self.hkv, self.d, generator=self.g).to(BF).cuda()
        return x[:, :self.hq], x[:, self.hq:self.hq + self.hkv], x[:, self.hq + self.hkv:]

    def step(self, q, k, v, start, ctx, q_out, out, ws, decode):
        from paper_2609_34653_amd import paged as pg
        pg.omnitide_paged_append(k, v, self.kp, self.vp, self.table, start, ctx, theta=self.theta,
                                 magnitude=1.1, k_weight=self.wk, q=q, q_out=q_out,
                                 q_weight=self.wq, d_status=self.status)
        scale = self.d ** -0.5
        if decode:
            pg.omnitide_paged_decode_attn(q_out.view(3, 1, self.hq, self.d), self.kp, self.vp,
                                          self.table, ctx, scale, out.view(3, 1, self.hq, self.d),
                                          ws, self.status)
        else:
            pg.omnitide_paged_chunk_attn(q_out, self.kp, self.vp, self.table, start, ctx, scale, out,
                                         ws, self.status)

    def workspace(self, T, decode):
        from paper_2609_34653_amd import paged as pg
        cap = self.max_pages * self.P
        n = (pg.omnitide_paged_decode_workspace_bytes(3, 1, cap, self.hq, self.hkv, self.d) if decode
             else pg.omnitide_paged_chunk_attn_workspace_bytes(T, 3, cap, self.hq, self.hkv, self.d))
        return torch.empty(max(1, n), dtype=torch.uint8, device="cuda")

    def check(self, q, start, ctx, q_out, out):
        """The rotated queries and the attention over what the pages hold."""
        row = np.concatenate([np.arange(n - (start[s + 1] - start[s]), n)
                              for s, n in enumerate(ctx)])
        qw = op.norm_rope(f64(q), f64(self.wq), 1e-6, self.theta, row, "half", 1.1)
        assert np.abs(f64(q_out) - qw).max() <= 2.0 ** -8 * np.abs(qw).max() + 1e-4
        want, spread = op.ragged_attention(f64(q_out), f64(self.kp), f64(self.vp), self.order, start,
                                           ctx, self.d ** -0.5)
        assert_near(out, want, spread, 2.0 ** -8, BF)
        assert int(self.status.item()) == 0


def test_streams_served_together():
    st = Streams()
    ctx = np.zeros(3, int)
    hist = [[], [], []]
    for new in ([40, 3, 17], [1, 90, 0], [5, 5, 33], [1, 1, 1], [1, 1, 1]):
        ctx = ctx + new
        start = np.concatenate([[0], np.cumsum(new)])
        T, decode = int(start[-1]), new == [1, 1, 1]
        q, k, v = st.inputs(T)
        q_out = torch.empty(T, st.hq, st.d, dtype=BF, device="cuda")
        out = torch.empty_like(q_out)
        st.step(q, k, v, i32(start), i32(ctx), q_out, out, st.workspace(T, decode), decode)
        torch.cuda.synchronize()
        for s in range(3):
            hist[s].append((f64(k[start[s]:start[s + 1]]), f64(v[start[s]:start[s + 1]])))
        st.check(q, start, ctx, q_out, out)
    for s in range(3):                                       # what the pages hold of each stream
        k = np.concatenate([h[0] for h in hist[s]])
        v = np.concatenate([h[1] for h in hist[s]])
        want = op.norm_rope(k, f64(st.wk), 1e-6, st.theta, np.arange(ctx[s]), "half", 1.1)
        held = op.gather_rows(f64(st.kp), st.order[s], int(ctx[s]))
        assert np.abs(held - want).max() <= 2.0 ** -8 * np.abs(want).max() + 1e-4
        assert np.array_equal(op.gather_rows(f64(st.vp), st.order[s], int(ctx[s])), v)


@pytest.mark.parametrize("decode", [False, True])
def test_captured_step_replays_as_eager(decode):
    """Append and attention captured once on another stream; the lengths and inputs change between
    replays, with eager work and synchronisation in between."""
    st = Streams(seed=3)
    new = [1, 1, 1] if decode else [30, 2, 11]
    start = np.concatenate([[0], np.cumsum(new)])
    T = int(start[-1])
    ctx, ds = i32([0, 0, 0]), i32(start)
    q0, k0, v0 = (x.clone() for x in st.inputs(T))
    q_out = torch.zeros(T, st.hq, st.d, dtype=BF, device="cuda")
    out = torch.zeros_like(q_out)
    ws = st.workspace(T, decode)
    ctx.copy_(i32(new))
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        st.step(q0, k0, v0, ds, ctx, q_out, out, ws, decode)
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        st.step(q0, k0, v0, ds, ctx, q_out, out, ws, decode)
    have = np.array(new)
    for rep in range(4):
        q, k, v = st.inputs(T)
        for a, b in ((q0, q), (k0, k), (v0, v)):
            a.copy_(b)
        have = have + new if rep else have
        ctx.copy_(i32(have))
        out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        st.check(q, start, have, q_out, out)
        eager, kept = torch.zeros_like(out), q_out.clone()
        st.step(q, k, v, ds, ctx, q_out, eager, st.workspace(T, decode), decode)
        torch.cuda.synchronize()
        assert torch.equal(eager, out) and torch.equal(q_out, kept)


def both(decode, ctx, P, hq, hkv, d, seed, new=2):
    """Inputs of one call: (q, kp, vp, table, start, ctx)."""
    table, n_pages = layout(ctx, P, seed)
    kp, vp = pools(ctx, table, n_pages, P, hkv, d, seed)
    q = torch.randn(len(ctx) * new, hq, d, generator=torch.Generator().manual_seed(seed)).to(BF)
    q = q.view(len(ctx), new, hq, d) if decode else q
    return q.cuda(), kp.cuda(), vp.cuda(), table, new * np.arange(len(ctx) + 1), ctx


@pytest.mark.parametrize("decode", [False, True])
@pytest.mark.parametrize("scale", [0.0, -0.2])
def test_scales_that_are_not_positive(decode, scale):
    """All keys alike, and the least score the likeliest; masked keys stay out."""
    q, kp, vp, table, start, ctx = both(decode, [300, 65, 2], 16, 6, 2, 64, 9)
    got, st = run(decode, q, kp, vp, table, start, ctx, scale, F32)
    want, spread = op.ragged_attention(f64(q).reshape(6, 6, 64), f64(kp), f64(vp), table, start, ctx,
                                       scale)
    assert st == 0
    # |scale| sum|q k| <= 0.2 x 100 on these inputs, as the docstring above has it
    assert_near(got.view(6, 6, 64), want, spread, 2.0 ** -8, F32)


@pytest.mark.parametrize("decode", [False, True])
def test_sequences_share_pages(decode):
    """Three sequences with the same first pages, each with its own tail."""
    ctx, P, hq, hkv, d = [700, 650, 641], 64, 8, 2, 64
    table, n_pages = layout(ctx, P, 4)
    table[1:, :10] = table[0, :10]
    kp, vp = (torch.randn(n_pages, P, hkv, d).to(BF) for _ in range(2))
    q = torch.randn(6, hq, d).to(BF)
    got, st = run(decode, (q.view(3, 2, hq, d) if decode else q).cuda(), kp.cuda(), vp.cuda(), table,
                  [0, 2, 4, 6], ctx, 0.125, F32)
    want, spread = op.ragged_attention(f64(q), f64(kp), f64(vp), table, [0, 2, 4, 6], ctx, 0.125)
    assert st == 0
    assert_near(got.view(6, hq, d), want, spread, 2.0 ** -8, F32)


@pytest.mark.parametrize("decode", [False, True])
def test_a_sequence_of_nans_stays_alone(decode):
    """Rows in use that are NaN and infinite spoil their own sequence, no other one, to the bit."""
    ctx = [900, 333, 70, 500]
    q, kp, vp, table, start, _ = both(decode, ctx, 32, 8, 2, 128, 6)
    clean, _ = run(decode, q, kp, vp, table, start, ctx, 0.1, F32)
    kp[table[1, :11]] = float("nan")
    vp[table[1, :11]] = float("inf")
    got, st = run(decode, q, kp, vp, table, start, ctx, 0.1, F32)
    assert st == 0
    rows = [0, 2, 3] if decode else [0, 1, 4, 5, 6, 7]
    assert torch.equal(got[rows], clean[rows]) and torch.isfinite(clean).all()


@pytest.mark.parametrize("decode", [False, True])
@pytest.mark.parametrize("rows", [slice(0, 1), slice(640, 700), slice(0, None)])
def test_keys_that_are_no_numbers_are_not_lost(decode, rows):
    """A token that sees such keys comes out as NaN, be they one, a share's or all of them; never as
    zeros."""
    ctx = [2500, 90, 700]
    q, kp, vp, table, start, _ = both(decode, ctx, 16, 8, 2, 64, 12)
    clean, _ = run(decode, q, kp, vp, table, start, ctx, 0.1, F32)
    for s in (0, 2):
        r = np.arange(ctx[s])[rows]
        kp[table[s, r // 16], r % 16] = float("nan")
    got, st = run(decode, q, kp, vp, table, start, ctx, 0.1, F32)
    assert st == 0
    got, clean = got.view(3, 2, 8, 64), clean.view(3, 2, 8, 64)
    for s in (0, 2):
        assert torch.isnan(got[s, 1]).all()
        assert torch.isnan(got[s, 0]).all() or ctx[s] - 1 <= rows.start
    assert torch.equal(got[1], clean[1])


@pytest.mark.parametrize("decode", [False, True])
def test_two_streams_at_once(decode):
    """Two calls in flight with a workspace each, on streams given by name, against each alone."""
    from paper_2609_34653_amd import paged as pg
    calls, alone = [], []
    for seed, ctx in ((7, [5000, 300, 2000]), (8, [100, 6000, 900])):
        q, kp, vp, table, start, _ = both(decode, ctx, 64, 16, 4, 128, seed)
        out, st = run(decode, q, kp, vp, table, start, ctx, 0.1, BF)
        assert st == 0
        alone.append(out)
        cap = table.shape[1] * 64
        nb = (pg.omnitide_paged_decode_workspace_bytes(3, 2, cap, 16, 4, 128) if decode else
              pg.omnitide_paged_chunk_attn_workspace_bytes(6, 3, cap, 16, 4, 128))
        calls.append((q, kp, vp, i32(table), i32(start), i32(ctx), torch.empty_like(out),
                      torch.empty(nb, dtype=torch.uint8, device="cuda"), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for rep in range(8):
        for q, kp, vp, table, start, ctx, out, ws, stream in calls:
            with torch.cuda.stream(stream):
                out.zero_()
            if decode:
                pg.omnitide_paged_decode_attn(q, kp, vp, table, ctx, 0.1, out, ws, stream=stream)
            else:
                pg.omnitide_paged_chunk_attn(q, kp, vp, table, start, ctx, 0.1, out, ws,
                                             stream=stream)
    torch.cuda.synchronize()
    for c, want in zip(calls, alone):
        assert torch.equal(c[6], want)


def test_zero_tokens():
    from paper_2609_34653_amd import paged as pg
    e = torch.empty(0, 4, 64, dtype=BF, device="cuda")
    kp = torch.zeros(2, 16, 1, 64, dtype=BF, device="cuda")
    pg.omnitide_paged_chunk_attn(e, kp, kp, i32([[0, 1]]), i32([0, 0]), i32([5]), 1.0, e.clone())
