"""Eviction by attention weight against float64 and exact plans.

Tolerance of a weight, relative: 2 e + 2^-15, with e the error of a score, d 2^-24 sum|q k| scale <= d 20 / 2^24 on
these inputs (it moves a probability's numerator and its sum), and 2^-15 for the exponentials (2^-22 and 20 x
2^-23 for their arguments) and the sums (at most 250 roundings deep: 32 rows of a lane at a time over 1,024, the
lanes, heads and chunks).  Moved keys: half a step plus 2^-19 of their pair's length."""
import numpy as np
import pytest
import torch

from oracle import evict as oe
from oracle import paged as op
from tests.test_gpu_norm_rope import BF, F32, STYLE, assert_close, f64, i32, layout

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_34653_amd import evict
    evict.lib()
    yield


def rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def key_pool(ctx, table, n_pages, P, hkv, d, seed):
    """Keys in use normal, other rows NaN and infinities."""
    pool = torch.full((n_pages, P, hkv, d), float("nan"))
    pool[:, ::2] = float("inf")
    for s, n in enumerate(ctx):
        r = np.arange(n)
        if n:
            pool[table[s, r // P], r % P] = rand(seed + s, n, hkv, d)
    return pool.to(BF)


def weights(q, pool, table, start, ctx, max_q, scale, w_in=None, seen=None, decay=1.0, out=None):
    from paper_2609_34653_amd import evict as ev
    S, cap = table.shape[0], table.shape[1] * pool.shape[1]
    hkv = pool.shape[2] if pool.dim() == 4 else 1
    if out is None:
        out = torch.full((S, cap + 3), 77.0, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    nb = ev.omnitide_paged_attn_weights_workspace_bytes(q.shape[0], S, cap, max_q, q.shape[1], hkv,
                                                        q.shape[2])
    ws = torch.full((nb,), 0xff, dtype=torch.uint8, device="cuda")
    ev.omnitide_paged_attn_weights(q, pool, i32(table), i32(start), i32(ctx), max_q, scale, out,
                                   weight_in=w_in, seen_len=None if seen is None else i32(seen), decay=decay,
                                   workspace=ws, d_status=st)
    torch.cuda.synchronize()
    return out, int(st.item())


def tolerance(d):
    return 2 * d * 20 * 2.0 ** -24 + 2.0 ** -15


def spread_of(d):
    return (192 / d) ** 0.5 if d > 128 else 1.0


def scale_of(d):
    return 192 ** -0.5 if d > 128 else d ** -0.5


WEIGHTS = [
    # ctx, new, page, hq, hkv, d
    ([1], [1], 16, 4, 1, 64),
    ([601], [89], 32, 4, 1, 64),
    ([64, 65, 63, 128], [64, 65, 63, 1], 64, 8, 8, 64),
    ([700], [129], 16, 28, 4, 128),
    ([2100, 90, 1300], [130, 0, 7], 128, 32, 8, 128),        # a sequence without tokens
    ([5000, 17], [3, 17], 256, 16, 2, 128),
    ([777, 300, 20, 1], [1, 1, 1, 1], 64, 32, 8, 128),       # single tokens
    ([900, 130, 64], [2, 1, 2], 16, 14, 2, 64),
    ([33 * i + 1 for i in range(20)], [min(33 * i + 1, 5 * i + 1) for i in range(20)], 16, 14, 2, 64),
    ([1030], [1030], 64, 16, 4, 128),                        # a prompt
    ([9 + i % 3 for i in range(300)], [i % 3 for i in range(300)], 16, 8, 4, 64),
    ([1400, 1390, 1410], [700, 710, 690], 32, 32, 8, 64),    # more row tiles than workgroups
    ([700, 33], [5, 33], 16, 16, 1, 576),                    # latents
    ([300, 1200], [300, 1], 32, 20, 1, 320),
    ([400, 80], [1, 1], 16, 128, 1, 576),
    ([6000], [40], 16, 40, 1, 128),
    ([20 + 3 * i for i in range(1024)], [i % 2 for i in range(1024)], 16, 3, 3, 64),
    ([30000], [1], 64, 8, 2, 128),
    ([30000], [4], 16, 8, 1, 64),
    ([700, 33, 5000], [2, 1, 2], 16, 16, 1, 576),            # 32 vectors of a KV head, 16 in between
    ([900, 64, 20], [1, 1, 1], 32, 32, 1, 320),
    ([3000, 100], [3, 2], 64, 28, 4, 128),                   # 21 and 14
    ([40 + i for i in range(70)], [1 + i % 4 for i in range(70)], 16, 14, 2, 64),
    ([20000], [4], 16, 32, 4, 128),
    ([300 + i for i in range(80)], [1 + i % 2 for i in range(80)], 16, 16, 1, 576),
    ([2500, 900, 64], [3, 2, 1], 32, 16, 1, 576),            # 48, 32 and 16 of 64 vectors
    ([900, 31], [1, 1], 16, 64, 1, 320),
    ([100 + 5 * i for i in range(90)], [1 + i % 4 for i in range(90)], 16, 16, 1, 576),
    ([700, 90], [1, 1], 16, 65, 1, 576),
]


@pytest.mark.parametrize("case", range(len(WEIGHTS)))
def test_weights(case):
    ctx, new, P, hq, hkv, d = WEIGHTS[case]
    table, n_pages = layout(ctx, P, case)
    start = np.concatenate([[0], np.cumsum(new)]) + 1        # padding in front, two behind
    T = int(start[-1]) + 2
    pool = key_pool(ctx, table, n_pages, P, hkv, d, case)
    q = (rand(case, T, hq, d) * spread_of(d)).to(BF)
    q[0] = q[-2:] = float("nan")
    w_in = rand(case + 5, len(ctx), table.shape[1] * P + 3).exp().cuda()
    gpool = pool.cuda() if hkv > 1 or d <= 128 else pool.cuda().view(n_pages, P, d)
    got, st = weights(q.cuda(), gpool, table, start, ctx, max(new), scale_of(d), w_in, None, 0.75)
    assert st == 0
    again, _ = weights(q.cuda(), gpool, table, start, ctx, max(new), scale_of(d), w_in, None, 0.75)
    assert torch.equal(got, again)                           # the same bits
    # a larger bound max_q may take another way
    other, st = weights(q.cuda(), gpool, table, start, ctx, max(new) + 3000, scale_of(d), w_in, None, 0.75)
    assert st == 0 and torch.allclose(got, other, rtol=2 * tolerance(d), atol=0)
    old = f64(w_in)
    for s, (n, m) in enumerate(zip(ctx, new)):
        g = f64(got[s])
        if m == 0:
            assert (g == 77.0).all()
            continue
        k = pool[table[s, np.arange(n) // P], np.arange(n) % P].double().numpy()
        want = oe.row_weights(f64(q[start[s]:start[s + 1]]), k, scale_of(d))
        want[:n - m] += 0.75 * old[s, :n - m]
        assert (np.abs(g[:n] - want) <= tolerance(d) * want).all(), \
            float((np.abs(g[:n] - want) / want).max())
        assert (g[n:] == 77.0).all()


def test_weights_accumulate():
    """In place from call to call, with a window of its own, as the same in one call."""
    n, P, hq, hkv, d = 300, 16, 8, 2, 64
    table, n_pages = layout([n], P, 1)
    pool = key_pool([n], table, n_pages, P, hkv, d, 1)
    q = rand(2, 50, hq, d).to(BF).cuda()
    one, st = weights(q, pool.cuda(), table, [0, 50], [n], 50, 0.125)
    assert st == 0
    acc = torch.full((1, table.shape[1] * P), float("nan"), device="cuda")
    weights(q[:20], pool.cuda(), table, [0, 20], [270], 20, 0.125, out=acc)
    weights(q[20:], pool.cuda(), table, [0, 30], [n], 30, 0.125, w_in=acc, out=acc)   # 270 rows seen
    assert torch.allclose(one[0, :n], acc[0, :n], rtol=2 * tolerance(d), atol=0)
    assert torch.isnan(acc[0, n:]).all()
    # seen_len: out of range counts as the nearer end; weight_in of rows beyond is not read
    base = torch.ones(1, table.shape[1] * P, device="cuda")
    base[0, 40:] = float("nan")
    for seen, upto in ((40, 40), (-7, 0), (0, 0)):
        got, _ = weights(q, pool.cuda(), table, [0, 50], [n], 50, 0.125, base, [seen], 2.0,
                         out=torch.zeros_like(base))
        want = f64(one[0, :n])
        want[:upto] += 2.0
        assert np.allclose(f64(got[0, :n]), want, rtol=1e-6)
    full, _ = weights(q, pool.cuda(), table, [0, 50], [n], 50, 0.125, torch.ones_like(base), [1 << 30], 2.0,
                      out=torch.zeros_like(base))
    assert np.allclose(f64(full[0, :n]), f64(one[0, :n]) + 2.0, rtol=1e-6) and (full[0, n:] == 0).all()


@pytest.mark.parametrize("m", [1, 60])
@pytest.mark.parametrize("rise", [True, False])
def test_weights_large_and_equal_scores(m, rise):
    n, P, d = 1500, 32, 64
    table, n_pages = layout([n], P, 1)
    pool = key_pool([n], table, n_pages, P, 1, d, 3)
    ramp = torch.linspace(-3, 3, n) if rise else torch.zeros(n)
    r = np.arange(n)
    pool[table[0, r // P], r % P] = ramp[:, None, None].expand(n, 1, d).to(BF)
    q = torch.ones(m, 4, d, dtype=BF)
    got, st = weights(q.cuda(), pool.cuda(), table, [0, m], [n], m, 1.0)
    want = oe.row_weights(f64(q), pool[table[0, r // P], r % P].double().numpy(), 1.0)
    # scores up to 192, exact sums of up to 64 x 192 x 2^-24: 2^-10.4; small weights may leave float's range
    assert st == 0 and (np.abs(f64(got[0, :n]) - want) <= 2.0 ** -9 * want + 1e-37).all()


@pytest.mark.parametrize("what", ["page", "low", "long", "order", "many", "late"])
@pytest.mark.parametrize("m", [2, 40])
def test_weights_refused_on_the_device(what, m):
    from paper_2609_34653_amd import omnitide as ot, paged as pg
    ctx, P, hq, hkv, d = [300, 200, 150], 16, 4, 2, 64
    table, n_pages = layout(ctx, P, 2)
    pool = torch.nan_to_num(key_pool(ctx, table, n_pages, P, hkv, d, 2), posinf=1.0)
    q = rand(4, 3 * m, hq, d).to(BF)
    given, n, start, max_q, code = table.copy(), list(ctx), [0, m, 2 * m, 3 * m], m, pg.E_PAGES
    if what == "page":
        given[1, 3] = n_pages
    elif what == "late":
        given[1, 12] = -1                                    # rows 192.. : the last eight
    elif what == "low":
        n[1], code = m - 1, ot.E_CAPACITY
    elif what == "long":
        n[1], code = given.shape[1] * P + 1, ot.E_CAPACITY
    elif what == "order":
        start = [0, m, m - 1, 3 * m - 1]
        q = torch.cat([q[:m], q[m:2 * m], q[2 * m:]])
    else:
        max_q, code = m - 1, ot.E_CAPACITY
    got, st = weights(q.cuda(), pool.cuda(), given, start, n, max_q, 0.125)
    assert st == code
    if what == "many":
        assert (got == 77.0).all()
        return

    def want(s, upto=None):
        k = pool[table[s, np.arange(ctx[s]) // P], np.arange(ctx[s]) % P].double().numpy()
        return oe.row_weights(f64(q[s * m:(s + 1) * m]), k, 0.125)
    good = [0] if what == "order" else [0, 2]
    for s in good:
        w = want(s)
        assert (np.abs(f64(got[s, :ctx[s]]) - w) <= tolerance(d) * w).all()
    if what == "page":
        assert torch.isnan(got[1, :200]).all() and (got[1, 200:] == 77.0).all()
    elif what == "late":
        assert torch.isnan(got[1, :200]).all()               # the last token sees all rows
    else:
        assert (got[1] == 77.0).all()


@pytest.mark.parametrize("start", [[0, 7, 3, 9], [0, 5, 0, 5, 0, 5], [2, 1 << 30, 3, 4], [-3, 4, 8]], ids=len)
def test_weights_overlapping_offsets(start):
    """A sequence that starts in front of an earlier offset has no tokens, and is left alone."""
    from paper_2609_34653_amd import paged as pg
    S, T, hq, hkv, d, P = len(start) - 1, 9, 4, 2, 64, 16
    ctx = [40 + 3 * i for i in range(S)]
    table, n_pages = layout(ctx, P, S)
    pool = key_pool(ctx, table, n_pages, P, hkv, d, 1)
    q = rand(3, T, hq, d).to(BF)
    got, st = weights(q.cuda(), pool.cuda(), table, start, ctx, T, 0.125)
    assert st == pg.E_PAGES
    top = 0
    for s in range(S):
        a, b = start[s:s + 2]
        n = ctx[s]
        if a >= max(top, 0) and a < b <= T:
            k = pool[table[s, np.arange(n) // P], np.arange(n) % P].double().numpy()
            w = oe.row_weights(f64(q[a:b]), k, 0.125)
            assert (np.abs(f64(got[s, :n]) - w) <= tolerance(d) * w).all()
        else:
            assert (got[s] == 77.0).all()
        top = max(top, a)


# ------------------------------------------------------------------------------------- plan

def run_plan(w, ctx, high, budget, sink, recent, with_weights=True):
    from paper_2609_34653_amd import evict as ev
    S, cap = w.shape
    src = torch.full((S, high + 5), -9, dtype=torch.int32, device="cuda")
    new = torch.full((S,), -9, dtype=torch.int32, device="cuda")
    wo = torch.full((S, high + 2), -9.0, device="cuda") if with_weights else None
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    nb = ev.omnitide_evict_plan_workspace_bytes(S, cap)
    ws = torch.full((nb,), 0xff, dtype=torch.uint8, device="cuda") if nb else None
    ev.omnitide_evict_plan(w, i32(ctx), high, budget, sink, recent, src, new, wo, ws, st)
    torch.cuda.synchronize()
    return src.cpu().numpy(), new.cpu().numpy(), None if wo is None else wo.cpu().numpy(), int(st.item())


def some_weights(kind, S, n, seed):
    w = rand(seed, S, n)
    if kind == "exp":
        return (3 * w).exp()
    if kind == "few":                                        # many ties
        return torch.randint(0, 3, (S, n), generator=torch.Generator().manual_seed(seed)).float()
    if kind == "equal":
        return torch.full((S, n), 0.25)
    if kind == "signs":                                      # every kind of number
        pick = torch.tensor([float("nan"), float("inf"), -float("inf"), 0.0, -0.0, 1e-45, -1e-45, 3.0])
        at = torch.randint(0, 16, (S, n), generator=torch.Generator().manual_seed(seed))
        return torch.where(at < 8, pick[at % 8], w)
    if kind == "near":                                       # alike but for the last bits
        return 1.0 + torch.randint(0, 9, (S, n), generator=torch.Generator().manual_seed(seed)) * 2.0 ** -23
    return torch.arange(n).float().flip(0).expand(S, n).clone()


PLANS = [
    # ctx, high, budget, sink, recent
    ([1], 1, 1, 0, 0),
    ([2], 1, 1, 0, 1),
    ([5, 6, 0, 4], 5, 4, 1, 2),
    ([100, 90, 130, 64], 64, 64, 4, 16),
    ([1000, 1001, 3], 500, 77, 0, 0),
    ([1000, 1001, 3], 500, 77, 40, 37),                      # nothing between
    ([5000, 4097, 4096, 4095], 4000, 3999, 1, 2),
    ([40000], 16384, 16384, 64, 665),
    ([70000, 20000], 1000, 999, 10, 100),
    ([150001], 100000, 99999, 0, 1),
    ([300 + i for i in range(70)], 310, 200, 7, 9),
]


@pytest.mark.parametrize("kind", ["exp", "few", "equal", "signs", "near", "falling"])
@pytest.mark.parametrize("case", range(len(PLANS)))
def test_plan(case, kind):
    ctx, high, budget, sink, recent = PLANS[case]
    cap = max(ctx) + 7
    w = some_weights(kind, len(ctx), cap, case)
    wide = torch.full((len(ctx), cap + 9), float("nan"))
    wide[:, :cap] = w
    wide = wide.cuda()
    src, new, wo, st = run_plan(wide[:, :cap], ctx, high, budget, sink, recent)
    assert st == 0
    host = w.numpy()
    for s, n in enumerate(ctx):
        keep = oe.plan(host[s, :n].tolist(), high, budget, sink, recent)
        assert new[s] == len(keep)
        assert np.array_equal(src[s, :len(keep)], keep)
        assert (src[s, len(keep):] == -9).all()
        assert np.array_equal(wo[s, :len(keep)].view(np.int32), host[s, keep].view(np.int32))
        assert (wo[s, len(keep):] == -9.0).all()


@pytest.mark.parametrize("kind", ["exp", "equal", "near"])
@pytest.mark.parametrize("cap", [4096, 4097, 8192, 8193, 16384, 16385, 131072, 131073, 262145, 700000])
def test_plan_at_the_ends_of_slices(cap, kind):
    """Lengths around those that change how a sequence is cut: to the last row, one less, and a short one."""
    ctx, budget = [cap, cap - 1, 100], cap // 3
    w = some_weights(kind, len(ctx), cap, cap)
    src, new, wo, st = run_plan(w.cuda(), ctx, budget + 9, budget, 5, 70)
    assert st == 0 and list(new) == [budget, budget, 100]
    host = w.numpy()
    for s, n in enumerate(ctx):
        keep = oe.plan(host[s, :n].tolist(), budget + 9, budget, 5, 70)
        assert np.array_equal(src[s, :len(keep)], keep)
        assert np.array_equal(wo[s, :len(keep)].view(np.int32), host[s, keep].view(np.int32))
        assert (src[s, len(keep):] == -9).all() and (wo[s, len(keep):] == -9.0).all()


def test_plan_lengths_refused_on_the_device():
    from paper_2609_34653_amd import omnitide as ot
    w = rand(1, 4, 100).exp().cuda()
    src, new, _, st = run_plan(w, [100, 101, -1, 60], 50, 40, 1, 1, with_weights=False)
    assert st == ot.E_CAPACITY and list(new) == [40, 0, 0, 40]
    assert (src[1:3] == -9).all()
    for s, n in ((0, 100), (3, 60)):
        assert np.array_equal(src[s, :40], oe.plan(w[s, :n].tolist(), 50, 40, 1, 1))


# ------------------------------------------------------------------------------------- move

def tables(ctx, kept, P, seed):
    """Pages of the rows as they are and as they will be, apart from each other."""
    both, n_pages = layout(list(ctx) + list(kept), P, seed)
    S = len(ctx)
    return both[:S].copy(), both[S:].copy(), n_pages


MOVES = [
    # ctx, kept, page, heads, d, dims, offset, style, values
    ([1], [1], 16, 1, 576, 64, 512, "half", False),
    ([100, 90, 0, 64], [40, 90, 0, 1], 16, 8, 128, 128, 0, "half", True),
    ([300, 33], [200, 33], 32, 2, 64, 32, 0, "interleaved", True),
    ([500, 700], [123, 699], 128, 1, 576, 64, 512, "interleaved", False),
    ([300], [100], 64, 1, 320, 64, 256, "half", False),
    ([257, 100], [256, 50], 256, 3, 128, 24, 8, "half", True),
    ([257, 100], [256, 50], 16, 4, 128, 0, 0, "half", True),
    ([70 + i % 5 for i in range(70)], [20 + i % 30 for i in range(70)], 16, 1, 64, 64, 0, "half", True),
    ([3000], [1700], 64, 32, 128, 128, 0, "interleaved", True),
    ([90], [60], 16, 5, 24, 0, 0, "half", False),            # rows of 120 values
    ([90], [60], 16, 2, 40, 16, 16, "half", True),
]


@pytest.mark.parametrize("case", range(len(MOVES)))
def test_compact(case):
    from paper_2609_34653_amd import evict as ev, paged as pg
    ctx, kept, P, H, d, R, offset, style, values = MOVES[case]
    src_t, dst_t, n_pages = tables(ctx, kept, P, case)
    rng = np.random.default_rng(case)
    S, width = len(ctx), max(kept) + 4
    src = np.full((S, width), 1 << 29, np.int32)
    for s, (n, m) in enumerate(zip(ctx, kept)):
        src[s, :m] = np.sort(rng.choice(n, m, replace=False)) if m else []
    k = rand(case, n_pages, P, H, d).to(BF)
    v = rand(case + 1, n_pages, P, H, d).to(BF) if values else None
    th = pg.omnitide_rope_thetas(1.0e5, R) if R else None
    gk, gv = k.cuda(), None if v is None else v.cuda()
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ev.omnitide_paged_compact(gk, gv, i32(src_t), i32(ctx), i32(dst_t), i32(src), i32(kept), theta=th,
                              rope_style=STYLE[style], rope_offset=offset, d_status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    want_v = None if v is None else v.clone()
    touched = np.zeros((n_pages, P), bool)
    for s, m in enumerate(kept):
        if not m:
            continue
        i, j = np.arange(m), src[s, :m]
        fp, fl, tp, tl = src_t[s, j // P], j % P, dst_t[s, i // P], i % P
        if v is not None:
            want_v[tp, tl] = v[fp, fl]
        touched[tp, tl] = True
        x, got = k[fp, fl], gk.cpu()[tp, tl]
        plain = np.setdiff1d(np.arange(d), np.arange(offset, offset + R))
        assert torch.equal(got[..., plain], x[..., plain])
        stays = j == i
        assert torch.equal(got[stays], x[stays])
        if R:
            part = slice(offset, offset + R)
            want = op.norm_rope(f64(x[..., part]), None, 0.0, th, i - j, style)
            assert_close(got[..., part], want, f64(x[..., part]), R, style, BF)
    keep = torch.from_numpy(~touched)
    assert torch.equal(gk.cpu()[keep], k[keep])
    if v is not None:
        assert torch.equal(gv.cpu(), want_v)


def test_compact_pages_that_stay():
    """A destination page that is the source's where all of its rows stay."""
    from paper_2609_34653_amd import evict as ev, paged as pg
    n, P, H, d = 100, 16, 2, 64
    src_t, dst_t, n_pages = tables([n, n], [60, n], P, 1)
    keep = np.concatenate([np.arange(35), np.arange(40, 65)])                     # pages 0 and 1 stay
    src = np.stack([np.concatenate([keep, np.zeros(40, int)]), np.arange(100)])
    dst_t[0, :2] = src_t[0, :2]
    dst_t[1] = src_t[1, :dst_t.shape[1]]                                          # nothing evicted
    k, v = rand(1, n_pages, P, H, d).to(BF), rand(2, n_pages, P, H, d).to(BF)
    gk, gv = k.cuda(), v.cuda()
    th = pg.omnitide_rope_thetas(1.0e4, d)
    ev.omnitide_paged_compact(gk, gv, i32(src_t), i32([n, n]), i32(dst_t), i32(src), i32([60, n]), theta=th)
    torch.cuda.synchronize()
    want = v.clone()
    i = np.arange(60)
    want[dst_t[0, i // P], i % P] = v[src_t[0, keep // P], keep % P]
    assert torch.equal(gv.cpu(), want)
    r = np.arange(n)
    assert torch.equal(gk.cpu()[src_t[1, r // P], r % P], k[src_t[1, r // P], r % P])
    assert torch.equal(gk.cpu()[src_t[0, :2]], k[src_t[0, :2]])


def test_compact_pages_turned_in_place():
    """Whole pages go: the rows behind them keep their slots, their keys turn where they are."""
    from paper_2609_34653_amd import evict as ev, paged as pg
    n, P, H, d = 107, 16, 2, 64
    src_t, _, n_pages = tables([n], [1], P, 1)
    keep = np.concatenate([np.arange(32), np.arange(64, n)])
    dst_t = src_t[:, [0, 1, 4, 5, 6]]
    k, v = rand(1, n_pages, P, H, d).to(BF), rand(2, n_pages, P, H, d).to(BF)
    gk, gv = k.cuda(), v.cuda()
    th = pg.omnitide_rope_thetas(1.0e4, d)
    ev.omnitide_paged_compact(gk, gv, i32(src_t), i32([n]), i32(dst_t), i32(keep[None]), i32([len(keep)]),
                              theta=th)
    torch.cuda.synchronize()
    assert torch.equal(gv.cpu(), v)
    i = np.arange(32, len(keep))
    at = src_t[0, (i + 32) // P], i % P
    want = op.norm_rope(f64(k[at]), None, 0.0, th, np.full(len(i), -32), "half")
    assert_close(gk.cpu()[at], want, f64(k[at]), d, "half", BF)
    same = k.clone()
    same[at] = gk.cpu()[at]
    assert torch.equal(gk.cpu(), same)


def test_compact_long_src_row():
    """Room for 2^28 rows of 4096 values, a workgroup each: more threads than one launch's first dimension holds."""
    from paper_2609_34653_amd import evict as ev
    P, n = 256, 20
    k = rand(1, 4, P, 4096).to(BF).view(4, P, 1, 4096)
    gk = k.cuda()
    src = torch.zeros(1, 1 << 28, dtype=torch.int32, device="cuda")
    src[0, :n] = torch.arange(3, 3 + n)
    dst = torch.zeros(1, 1 << 20, dtype=torch.int32, device="cuda")
    dst[0, 0] = 2
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ev.omnitide_paged_compact(gk, None, i32([[1]]), i32([40]), dst, src, i32([n]), d_status=st)
    torch.cuda.synchronize()
    want = k.clone()
    want[2, :n] = k[1, 3:3 + n]
    assert int(st.item()) == 0
    assert torch.equal(gk.cpu(), want)


@pytest.mark.parametrize("what", ["src", "row", "dst", "kept", "long"])
def test_compact_refused_on_the_device(what):
    from paper_2609_34653_amd import evict as ev, omnitide as ot, paged as pg
    ctx, kept, P, H, d = [100, 90], [40, 50], 16, 2, 64
    src_t, dst_t, n_pages = tables(ctx, kept, P, 3)
    src = np.stack([np.arange(50) * 2 % 100, np.arange(50) + 30])
    good_s, good_d, n, m, code = src_t.copy(), dst_t.copy(), list(ctx), list(kept), pg.E_PAGES
    lost = None
    if what == "src":
        src_t[1, 3] = n_pages                                # rows 48..63
        lost = np.arange(18, 34)
    elif what == "dst":
        dst_t[1, 1] = -1
        lost = np.arange(16, 32)
    elif what == "row":
        src[1, 7], code = 90, ot.E_RANGE
        lost = np.array([7])
    elif what == "kept":
        m[1], code = dst_t.shape[1] * P + 1, ot.E_CAPACITY
    else:
        n[1], code = src_t.shape[1] * P + 1, ot.E_CAPACITY
    k = rand(1, n_pages, P, H, d).to(BF)
    gk = k.cuda()
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ev.omnitide_paged_compact(gk, None, i32(src_t), i32(n), i32(dst_t), i32(src), i32(m), d_status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == code
    want = k.clone()
    for s in (0, 1):
        rows = np.arange(kept[s])
        if s == 1:
            rows = np.setdiff1d(rows, lost) if lost is not None else rows[:0]
        j = src[s, rows]
        want[good_d[s, rows // P], rows % P] = k[good_s[s, j // P], j % P]
    assert torch.equal(gk.cpu(), want)


@pytest.mark.parametrize("m", [2, 60])
def test_pages_beyond_four_gib(m):
    """Weights and move on the last pages of a large pool: the bits of a small one."""
    from paper_2609_34653_amd import evict as ev, paged as pg
    ctx, kept, P, H, d = [200, 90], [150, 90], 32, 4, 128
    src_t, dst_t, n_pages = tables(ctx, kept, P, 3)
    small = torch.nan_to_num(key_pool(ctx, src_t, n_pages, P, H, d, 1), posinf=1.0).cuda()
    n = (7 << 30) // (P * H * d * 2)
    large = torch.zeros(n, P, H, d, dtype=BF, device="cuda")
    large[n - n_pages:] = small
    q = rand(2, 2 * m, 8, d).to(BF).cuda()
    src = np.stack([np.arange(150) + 50 * (np.arange(150) > 80), np.arange(150)])
    th = pg.omnitide_rope_thetas(1.0e4, d)
    got = []
    for pool, up in ((small, 0), (large, n - n_pages)):
        w, st = weights(q, pool, src_t + up, [0, m, 2 * m], ctx, m, 0.09)
        assert st == 0
        ev.omnitide_paged_compact(pool, pool.clone(), i32(src_t + up), i32(ctx), i32(dst_t + up), i32(src),
                                  i32(kept), theta=th)
        torch.cuda.synchronize()
        got.append((w, pool[up:].clone()))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


# --------------------------------------------------------------------------------- together

def evict_step(pool, v_pool, table, dst, ctx, w, high, budget, sink, recent, th, offset, style=0):
    from paper_2609_34653_amd import evict as ev
    S = table.shape[0]
    src = torch.zeros(S, high, dtype=torch.int32, device="cuda")
    new = torch.zeros(S, dtype=torch.int32, device="cuda")
    kept = torch.zeros(S, w.shape[1], device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    nb = ev.omnitide_evict_plan_workspace_bytes(*w.shape)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda") if nb else None
    ev.omnitide_evict_plan(w, ctx, high, budget, sink, recent, src, new, kept, ws, st)
    ev.omnitide_paged_compact(pool, v_pool, table, ctx, dst, src, new, th, style, offset, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    return src, new, kept


def test_streams_evict_and_go_on():
    """Two streams: a chunk appended and attended to, its weights, rows evicted to new pages, a token appended
    there and decoded: it attends to exactly the kept rows."""
    from paper_2609_34653_amd import paged as pg
    P, hq, hkv, d, mp = 16, 8, 2, 64, 16
    ctx, new = [200, 90], [60, 90]
    src_t, dst_t, n_pages = tables([mp * P] * 2, [130] * 2, P, 5)
    table, dst = i32(src_t[:, :mp]), i32(dst_t[:, :9])
    kp, vp = (torch.full((n_pages, P, hkv, d), float("nan"), dtype=BF, device="cuda") for _ in range(2))
    th = pg.omnitide_rope_thetas(1.0e4, d)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    w = torch.zeros(2, mp * P, device="cuda")
    first = [a - b for a, b in zip(ctx, new)]
    for lens, n, seed in ((first, first, 1), (new, ctx, 2)):
        T = sum(lens)
        x = rand(seed, T, hq + 2 * hkv, d).to(BF).cuda()
        q = torch.empty(T, hq, d, dtype=BF, device="cuda")
        start = np.concatenate([[0], np.cumsum(lens)])
        pg.omnitide_paged_append(x[:, hq:hq + hkv], x[:, hq + hkv:], kp, vp, table, i32(start), i32(n),
                                 theta=th, q=x[:, :hq], q_out=q, d_status=st)
        weights(q, kp, src_t[:, :mp], start, n, max(lens), 0.125, w_in=w, decay=0.5, out=w)
    assert int(st.item()) == 0
    k0, v0 = f64(kp), f64(vp)
    w0 = f64(w)
    src, kept, w2 = evict_step(kp, vp, table, dst, i32(ctx), w, 128, 100, 4, 20, th, 0)
    assert kept.tolist() == [100, 90]
    rows = [oe.plan(w0[s, :n].astype(np.float32).tolist(), 128, 100, 4, 20) for s, n in enumerate(ctx)]
    for s in range(2):
        m = len(rows[s])
        assert src[s, :m].tolist() == rows[s]
        assert np.array_equal(f64(w2[s, :m]), w0[s, rows[s]])
    # a token of each stream on the kept rows
    now = kept + 1
    x = rand(9, 2, hq + 2 * hkv, d).to(BF).cuda()
    q = torch.empty(2, hq, d, dtype=BF, device="cuda")
    pg.omnitide_paged_append(x[:, hq:hq + hkv], x[:, hq + hkv:], kp, vp, dst, i32([0, 1, 2]), now, theta=th,
                             q=x[:, :hq], q_out=q, d_status=st)
    out = torch.zeros(2, 1, hq, d, device="cuda")
    ws = torch.empty(pg.omnitide_paged_decode_workspace_bytes(2, 1, 9 * P, hq, hkv, d), dtype=torch.uint8,
                     device="cuda")
    pg.omnitide_paged_decode_attn(q.view(2, 1, hq, d), kp, vp, dst, now, 0.125, out, ws, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    import oracle
    for s in range(2):
        m = len(rows[s])
        j = np.array(rows[s])
        k = op.norm_rope(k0[src_t[s, j // P], j % P], None, 0.0, th, np.arange(m) - j, "half")
        v = v0[src_t[s, j // P], j % P]
        kn = op.norm_rope(f64(x[s:s + 1, hq:hq + hkv]), None, 0.0, th, [m], "half")
        qn = op.norm_rope(f64(x[s:s + 1, :hq]), None, 0.0, th, [m], "half")
        want = oracle.chunk_attention(qn, np.concatenate([k, kn]),
                                      np.concatenate([v, f64(x[s:s + 1, hq + hkv:])]), 0.125)
        # keys and queries rounded to bf16 twice: scores off by 2^-7 of about one each
        assert np.abs(f64(out[s]) - want).max() < 2.0 ** -5


def test_latents_evict_and_go_on():
    """The same of a latent cache: absorbed queries' weights, rows moved with their key part turned."""
    from paper_2609_34653_amd import latent as la, paged as pg
    from oracle import latent as ol
    R, E, H, P, mp = 256, 64, 16, 16, 16
    ctx = [200, 150]
    src_t, dst_t, n_pages = tables([mp * P] * 2, [100] * 2, P, 5)
    table, dst = i32(src_t[:, :mp]), i32(dst_t[:, :7])
    pool = torch.full((n_pages, P, R + E), float("nan"), dtype=BF, device="cuda")
    th = pg.omnitide_rope_thetas(1.0e4, E)
    kv = rand(1, sum(ctx), R + E).to(BF).cuda()
    la.omnitide_latent_append(kv[:, :R], kv[:, R:], pool, table, i32([0, 200, 350]), i32(ctx), theta=th,
                              rope_style=1)
    q = (rand(2, 2, H, R + E) * 0.8).to(BF).cuda()
    w, st = weights(q, pool, src_t[:, :mp], [0, 1, 2], ctx, 1, 0.07, out=torch.zeros(2, mp * P, device="cuda"))
    assert st == 0
    p0, w0 = f64(pool), f64(w)
    src, kept, _ = evict_step(pool, None, table, dst, i32(ctx), w, 90, 80, 2, 10, th, R, 1)
    out = torch.zeros(2, 1, H, R, device="cuda")
    ws = torch.empty(la.omnitide_latent_decode_workspace_bytes(2, 1, 7 * P, H, R), dtype=torch.uint8,
                     device="cuda")
    la.omnitide_latent_decode_attn(q.view(2, 1, H, R + E), pool, dst, kept, 0.07, out, ws)
    torch.cuda.synchronize()
    for s in range(2):
        j = np.array(oe.plan(w0[s, :ctx[s]].tolist(), 90, 80, 2, 10))
        assert src[s, :80].tolist() == j.tolist()
        rows = p0[src_t[s, j // P], j % P]
        rows[:, R:] = op.norm_rope(rows[:, None, R:], None, 0.0, th, np.arange(80) - j, "interleaved")[:, 0]
        want, _ = ol.absorbed_attention(f64(q[s:s + 1]), rows, R, 0.07)
        assert np.abs(f64(out[s]) - want).max() < 2.0 ** -5


def test_captured_step():
    """Weights, plan and move in a graph, replayed with other lengths between eager work: as the eager calls."""
    from paper_2609_34653_amd import evict as ev, paged as pg
    P, hq, hkv, d, mp, S = 16, 8, 2, 64, 12, 3
    src_t, dst_t, n_pages = tables([mp * P] * S, [100] * S, P, 5)
    table, dst = i32(src_t[:, :mp]), i32(dst_t[:, :7])
    lens = [[150, 90, 192], [101, 20, 130], [192, 192, 99]]
    pool0, v0 = rand(1, n_pages, P, hkv, d).to(BF).cuda(), rand(2, n_pages, P, hkv, d).to(BF).cuda()
    pool, vp = pool0.clone(), v0.clone()
    q = rand(3, 30, hq, d).to(BF).cuda()
    ctx, start = i32(lens[0]), i32([0, 1, 18, 30])
    w = torch.zeros(S, mp * P, device="cuda")
    src = torch.zeros(S, 100, dtype=torch.int32, device="cuda")
    new = torch.zeros(S, dtype=torch.int32, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    th = pg.omnitide_rope_thetas(1.0e4, d)
    nb = ev.omnitide_paged_attn_weights_workspace_bytes(30, S, mp * P, 17, hq, hkv, d)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    nb = ev.omnitide_evict_plan_workspace_bytes(S, mp * P)
    wp = torch.empty(nb, dtype=torch.uint8, device="cuda") if nb else None

    def calls():
        ev.omnitide_paged_attn_weights(q, pool, table, start, ctx, 17, 0.125, w, w, decay=0.5, workspace=ws,
                                       d_status=st)
        ev.omnitide_evict_plan(w, ctx, 100, 90, 3, 20, src, new, None, wp, st)
        ev.omnitide_paged_compact(pool, vp, table, ctx, dst, src, new, th, d_status=st)

    def load(i):
        ctx.copy_(i32(lens[i]))
        pool.copy_(pool0), vp.copy_(v0), w.fill_(0.5), src.zero_(), new.zero_()

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
        got = [x.clone() for x in (w, src, new, pool, vp)]
        load(i)
        calls()
        torch.cuda.synchronize()
        for x, y in zip(got, (w, src, new, pool, vp)):
            assert torch.equal(x, y)
    assert int(st.item()) == 0


# ------------------------------------------------------------------------------- mixed batches

@pytest.mark.parametrize("hq,hkv,d,cap", [(16, 4, 64, 1 << 14), (16, 1, 320, 4096)])
def test_weights_of_chunks_beside_single_tokens(hq, hkv, d, cap):
    """Several row chunks of some sequences, one of most, none of a few; more sequences than are counted at once."""
    new = [1] * 150
    new[3], new[70], new[149] = 700, 300, 431
    new[0], new[64], new[100] = 0, 0, 0
    ctx = [max(m, 30 + 7 * i % 400) for i, m in enumerate(new)]
    P = 16
    table, n_pages = layout(ctx, P, 1)
    wide = np.full((len(ctx), cap // P), -1)
    wide[:, :table.shape[1]] = table
    start = np.concatenate([[0], np.cumsum(new)])
    pool = key_pool(ctx, table, n_pages, P, hkv, d, 1)
    q = (rand(2, int(start[-1]), hq, d) * spread_of(d)).to(BF)
    gpool = pool.cuda() if d <= 128 else pool.cuda().view(n_pages, P, d)
    got, st = weights(q.cuda(), gpool, wide, start, ctx, 700, scale_of(d))
    assert st == 0
    for s, (n, m) in enumerate(zip(ctx, new)):
        if m == 0:
            assert (got[s] == 77.0).all()
        elif m > 1 or s % 11 == 0:
            k = pool[table[s, np.arange(n) // P], np.arange(n) % P].double().numpy()
            w = oe.row_weights(f64(q[start[s]:start[s + 1]]), k, scale_of(d))
            assert (np.abs(f64(got[s, :n]) - w) <= tolerance(d) * w).all()
        else:
            assert torch.isclose(got[s, :n].sum(), torch.tensor(float(hq)), rtol=1e-3)
        assert (got[s, n:] == 77.0).all()


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (16, 1, 576), (70, 2, 64)])
def test_weights_of_padded_batches(hq, hkv, d):
    """Far more tokens than sequences may have, one refused in the middle: both ways stay within the workspace of the
    call's own lengths, and one of the largest serves it with the same bits."""
    from paper_2609_34653_amd import evict as ev, omnitide as ot
    ctx, start, T, P, cap = [300, 200, 150, 90], [70, 72, 92, 93, 95], 300, 16, 512
    table, n_pages = layout(ctx, P, 1, max_pages=cap // P)
    pool = key_pool(ctx, table, n_pages, P, hkv, d, 1)
    q = (rand(2, T, hq, d) * spread_of(d)).to(BF)
    gpool = pool.cuda() if d <= 128 else pool.cuda().view(n_pages, P, d)
    got = []
    for size in ((T, 4, cap, 2), (T + 700, 9, 2 * cap, 400)):
        nb = ev.omnitide_paged_attn_weights_workspace_bytes(*size, hq, hkv, d)
        ws = torch.full((nb + 4096,), 0xff, dtype=torch.uint8, device="cuda")
        out, st = torch.full((4, cap), 77.0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        ev.omnitide_paged_attn_weights(q.cuda(), gpool, i32(table), i32(start), i32(ctx), 2, scale_of(d), out,
                                       workspace=ws[:nb], d_status=st)
        assert int(st.item()) == ot.E_CAPACITY and (ws[nb:] == 0xff).all()
        got.append(out)
    assert torch.equal(got[0], got[1])
    for s, n in enumerate(ctx):
        if s == 1:
            assert (got[0][s] == 77.0).all()
            continue
        k = pool[table[s, np.arange(n) // P], np.arange(n) % P].double().numpy()
        w = oe.row_weights(f64(q[start[s]:start[s + 1]]), k, scale_of(d))
        assert (np.abs(f64(got[0][s, :n]) - w) <= tolerance(d) * w).all()
        assert (got[0][s, n:] == 77.0).all()


# ----------------------------------------------------------------------- promises of the headers

@pytest.mark.parametrize("m", [2, 40])
@pytest.mark.parametrize("scale", [-0.05, 0.0])
def test_weights_scales(m, scale):
    ctx, P, hq, hkv, d = [300, 77], 16, 8, 2, 64
    table, n_pages = layout(ctx, P, 1)
    pool = key_pool(ctx, table, n_pages, P, hkv, d, 3)
    q = rand(4, 2 * m, hq, d).to(BF)
    got, st = weights(q.cuda(), pool.cuda(), table, [0, m, 2 * m], ctx, m, scale)
    assert st == 0
    for s, n in enumerate(ctx):
        k = pool[table[s, np.arange(n) // P], np.arange(n) % P].double().numpy()
        w = oe.row_weights(f64(q[s * m:(s + 1) * m]), k, scale)
        assert (np.abs(f64(got[s, :n]) - w) <= tolerance(d) * w).all()


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (16, 1, 576)])
@pytest.mark.parametrize("m", [2, 70])
@pytest.mark.parametrize("row", [3, 120, 231])
def test_weights_beside_a_key_that_is_no_number(m, row, hq, hkv, d):
    """Every row that a token sees beside it is NaN; what no such token sees, and the other sequences, are right."""
    ctx, P = [232, 150, 90], 16
    table, n_pages = layout(ctx, P, 1)
    pool = key_pool(ctx, table, n_pages, P, hkv, d, 3)
    pool[table[0, row // P], row % P, hkv - 1, 5] = float("nan")
    q = (rand(4, 3 * m, hq, d) * spread_of(d)).to(BF)
    gpool = pool.cuda() if d <= 128 else pool.cuda().view(n_pages, P, d)
    got, st = weights(q.cuda(), gpool, table, [0, m, 2 * m, 3 * m], ctx, m, scale_of(d))
    assert st == 0
    assert torch.isnan(got[0, :232]).all() and (got[0, 232:] == 77.0).all()      # (the last token sees all)
    for s in (1, 2):
        n = ctx[s]
        k = pool[table[s, np.arange(n) // P], np.arange(n) % P].double().numpy()
        w = oe.row_weights(f64(q[s * m:(s + 1) * m]), k, scale_of(d))
        assert (np.abs(f64(got[s, :n]) - w) <= tolerance(d) * w).all()
