"""Two additions to the paged cache, as measurable cases.

Latent attention: a cache with one shared latent vector and one rotated key part per token, its append,
the rows of streams in one piece (what a projection expands to keys and values), attention of single
tokens over the latents themselves (the absorbed form) and of chunks over expanded keys and values.

Eviction by attention weight: the weight that tokens give to each cached row, summed over heads and
accumulated from call to call, and the move of the rows that a budget keeps to pages of their own.

A case's structure (lengths) follows from the case alone; values and the order of the pages are drawn
on the GPU from the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

HALF, INTERLEAVED = 0, 1
EPS = 1.0e-6
E = 64                                   # rotated dimensions of a latent row and of a latent query


# ------------------------------------------------------------------------------------- cases

def listed():
    return [
        # One generated token for each of 24 streams: the token's latent, its rotated key part and the
        # 16 heads' rotated query parts.
        dict(name="latent_append_24x1tok", kind="append", seqs=24, q_lo=1, q_hi=1, ctx_lo=600,
             ctx_hi=9173, page=64, heads=16, latent=512, f32=False, style=INTERLEAVED, norm=True),
        # A float32 model's long prompts.
        dict(name="latent_append_f32_prompts", kind="append", seqs=3, q_lo=9000, q_hi=12011,
             ctx_lo=12288, ctx_hi=14000, page=16, heads=32, latent=512, f32=True, style=HALF,
             norm=True),
        # The 17K retained latents of one stream in one piece, for the projection that expands them.
        dict(name="rows_latent_1x17k", kind="rows", seqs=1, ctx_lo=17048, ctx_hi=17048, page=64,
             width=576),
        # The keys of eight streams (8 heads of 128) in one piece.
        dict(name="rows_keys_8_ragged", kind="rows", seqs=8, ctx_lo=1840, ctx_hi=18001, page=16,
             width=1024),
        # One generated token over one layer's 17K retained latents.
        dict(name="latent_decode_1x17k", kind="decode", seqs=1, nq=1, ctx_lo=16948, ctx_hi=16948,
             page=64, heads=16, latent=512),
        # 24 streams of unequal length, 128 heads on each latent.
        dict(name="latent_decode_24_ragged", kind="decode", seqs=24, nq=1, ctx_lo=600,
             ctx_hi=20000, page=128, heads=128, latent=512),
        # The smallest stream of the tests: an 89-token chunk over 512 kept tokens.
        dict(name="latent_chunk_89_tiny", kind="chunk", seqs=1, q_lo=89, q_hi=89, ctx_lo=601,
             ctx_hi=601, heads=4, d=64),
        # The benchmark's chunk over one layer's 17K retained tokens.
        dict(name="latent_chunk_665_17k", kind="chunk", seqs=1, q_lo=665, q_hi=665, ctx_lo=17048,
             ctx_hi=17048, heads=16, d=128),
        # Weights of one generated token for each of 24 streams of unequal length.
        dict(name="weights_24x1tok", kind="weights", seqs=24, q_lo=1, q_hi=1, ctx_lo=600,
             ctx_hi=20000, page=64, hq=32, hkv=8, d=128),
        # Weights of the benchmark's chunk over 17K retained tokens.
        dict(name="weights_665_17k", kind="weights", seqs=1, q_lo=665, q_hi=665, ctx_lo=17048,
             ctx_hi=17048, page=64, hq=32, hkv=8, d=128),
        # The 80K-token history cut to its budget, its keys turned to their new positions.
        dict(name="evict_1x80k", kind="evict", seqs=1, ctx_lo=81920, ctx_hi=81920, page=64, hkv=8,
             d=128, latent=0, high=16384, budget=16384, sink=64, recent=665, style=HALF),
        # 24 streams of latents, some below the mark from which rows go.
        dict(name="evict_24_latent", kind="evict", seqs=24, ctx_lo=1200, ctx_hi=9173, page=32,
             hkv=1, d=576, latent=512, high=4096, budget=2048, sink=16, recent=256,
             style=INTERLEAVED),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(4, 1, 64), (14, 2, 64), (16, 4, 128), (16, 2, 128), (28, 4, 128), (32, 8, 128),
          (32, 8, 128), (8, 8, 64), (16, 1, 576), (32, 1, 320)]


def draw(rng):
    kind = rng.choice(["append", "rows", "decode", "decode", "chunk", "chunk", "weights", "weights",
                       "evict", "evict"])
    c = dict(kind=kind, page=rng.choice([16, 32, 64, 64, 128, 256]))
    if kind == "append":
        seqs = _log(rng, 1, 64)
        hi = _log(rng, 1, 20000 // seqs)
        c.update(seqs=seqs, q_lo=max(1, hi // rng.choice([1, 4, 20])), q_hi=hi, ctx_lo=hi,
                 ctx_hi=hi + _log(rng, 1, 20000 // seqs), heads=rng.choice([4, 8, 16, 20, 32]),
                 latent=rng.choice([256, 512, 512]), f32=rng.random() < 0.3,
                 style=rng.choice([HALF, INTERLEAVED]), norm=rng.random() < 0.7)
    elif kind == "rows":
        seqs = _log(rng, 1, 64)
        hi = _log(rng, 60, 40000 // seqs + 60)
        c.update(seqs=seqs, ctx_lo=max(1, hi // rng.choice([1, 3, 50])), ctx_hi=hi,
                 width=rng.choice([64, 320, 576, 576, 1024]))
    elif kind == "decode":
        seqs = _log(rng, 1, 96)
        heads = rng.choice([4, 8, 16, 16, 20, 32, 64, 128])
        nq = rng.randint(1, max(1, min(4, 128 // heads)))
        hi = _log(rng, 300, max(600, min(60000, 20000000 // (seqs * max(64, heads * nq)))))
        c.update(seqs=seqs, nq=nq, ctx_lo=max(8, hi // rng.choice([1, 3, 50])), ctx_hi=hi,
                 heads=heads, latent=rng.choice([256, 512, 512]))
    elif kind == "chunk":
        seqs, hi, q_hi = _log(rng, 1, 12), _log(rng, 300, 18000), _log(rng, 2, 2400)
        heads = rng.choice([4, 8, 16, 16, 20])
        d = rng.choice([64, 128, 128])
        hi = min(hi, 110000000 // (seqs * heads * d))
        q_hi = max(1, min(q_hi, hi, 180000000 // (seqs * heads * hi)))
        c.update(seqs=seqs, q_lo=max(1, q_hi // rng.choice([1, 3, 100])), q_hi=q_hi,
                 ctx_lo=max(q_hi, hi // rng.choice([1, 2, 10])), ctx_hi=hi, heads=heads, d=d)
        del c["page"]
    elif kind == "weights":
        hq, hkv, d = rng.choice(_HEADS)
        if rng.random() < 0.5:
            seqs = _log(rng, 1, 64)
            hi = _log(rng, 300, min(40000, 100000000 // (seqs * hkv * d)))
            q_hi = rng.randint(1, 3)
        else:
            seqs, hi, q_hi = _log(rng, 1, 8), _log(rng, 300, 18000), _log(rng, 2, 2400)
            q_hi = max(1, min(q_hi, hi, 46000000000 // (seqs * hq * hi * d)))
        c.update(seqs=seqs, q_lo=max(1, q_hi // rng.choice([1, 3, 100])), q_hi=q_hi,
                 ctx_lo=max(q_hi, hi // rng.choice([1, 2, 10])), ctx_hi=hi, hq=hq, hkv=hkv, d=d)
    else:
        seqs = _log(rng, 1, 48)
        hkv, d, latent = rng.choice([(8, 128, 0), (2, 64, 0), (4, 128, 0), (1, 576, 512),
                                     (1, 320, 256)])
        hi = _log(rng, 600, 81920 if seqs == 1 else max(1200, 50000 // seqs))
        budget = _log(rng, 100, min(hi, 16384))
        c.update(seqs=seqs, ctx_lo=max(50, hi // rng.choice([1, 2, 8])), ctx_hi=hi, hkv=hkv, d=d,
                 latent=latent, high=budget + rng.choice([0, 0, budget // 3]), budget=budget,
                 sink=rng.randint(0, budget // 4), recent=rng.randint(0, budget // 2),
                 style=rng.choice([HALF, INTERLEAVED]))
    return c


# --------------------------------------------------------------------------------- structure

def _lens(c):
    """(rows with the new tokens, new tokens) of each sequence."""
    rng = random.Random("%d %d %d" % (c["seqs"], c["ctx_lo"], c["ctx_hi"]))
    ctx = [_log(rng, c["ctx_lo"], c["ctx_hi"]) for _ in range(c["seqs"])]
    if "q_lo" not in c:
        return ctx, [c.get("nq", 0)] * c["seqs"]
    return ctx, [min(n, _log(rng, c["q_lo"], c["q_hi"])) for n in ctx]


def _kept(c):
    """Rows of each sequence after an eviction."""
    return [n if n <= c["high"] else c["budget"] for n in _lens(c)[0]]


def _theta(dims):
    return 1.0e6 ** (-torch.arange(0, dims, 2, dtype=torch.float64) / dims)


def _scale(c):
    # a latent query stands for one of 128 plain dimensions and the rotated ones
    if c["kind"] == "chunk":
        return 1.0 / math.sqrt(c["d"] + E)
    return 1.0 / math.sqrt(c["d"]) if c.get("d", 576) <= 128 else 1.0 / math.sqrt(128 + E)


# ------------------------------------------------------------------------------------ inputs

def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _starts(n):
    return [sum(n[:i]) for i in range(len(n) + 1)]


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    kind = c["kind"]
    ctx, new = _lens(c)
    S, T = c["seqs"], sum(new)
    s = dict(c=c, ctx=_i32(ctx), ctx_host=ctx, new=new, status=_i32([0]))

    def normal(*shape, dtype=torch.bfloat16, std=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    if kind != "chunk":
        P = c["page"]
        pages = [-(-n // P) for n in ctx]
        more = [-(-n // P) for n in _kept(c)] if kind == "evict" else []
        n_pages = sum(pages) + sum(more) + 3
        order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
        at = 0

        def table(pages):
            nonlocal at
            t = torch.full((S, max(pages)), -1, dtype=torch.int32, device="cuda")
            for i, n in enumerate(pages):
                t[i, :n] = order[at:at + n]
                at += n
            return t

        s["table"] = table(pages)
        cap = s["table"].shape[1] * P
    if "q_lo" in c:
        s["start"] = _i32(_starts(new))
    if kind == "append":
        R, H, dt = c["latent"], c["heads"], torch.float32 if c["f32"] else torch.bfloat16
        kv = normal(T, R + E, dtype=dt)                  # the down projection's output
        q = normal(T, H, 128 + E, dtype=dt)              # the queries' projection
        s.update(latent=kv[:, :R], k_rope=kv[:, R:], q_rope=q[..., 128:],
                 q_out=torch.zeros(T, H, R + E, dtype=torch.bfloat16, device="cuda")[..., R:],
                 pool=normal(n_pages, P, R + E), theta=_theta(E), theta_dev=_theta(E).cuda())
        s["weight"] = (1.0 + 0.1 * normal(R, dtype=torch.float32)).to(dt) if c["norm"] else None
    elif kind == "rows":
        s.update(pool=normal(n_pages, P, c["width"]), row_start=_i32(_starts(ctx)),
                 out=torch.zeros(sum(ctx), c["width"], dtype=torch.bfloat16, device="cuda"))
    elif kind == "decode":
        R, H = c["latent"], c["heads"]
        # queries in the latents' space: scores as spread as those of unit normal heads
        s.update(pool=normal(n_pages, P, R + E),
                 q=normal(S, c["nq"], H, R + E, std=math.sqrt((128 + E) / (R + E))),
                 out=torch.zeros(S, c["nq"], H, R, dtype=torch.bfloat16, device="cuda"))
    elif kind == "chunk":
        H, d = c["heads"], c["d"]
        n = sum(ctx)
        kv = normal(n, H, 2 * d)                         # the up projection's output
        s.update(k=kv[..., :d], v=kv[..., d:], k_rope=normal(n, 512 + E)[:, 512:],
                 q=normal(T, H, d + E), kv_start=_i32(_starts(ctx)),
                 out=torch.zeros(T, H, d, dtype=torch.bfloat16, device="cuda"))
    elif kind == "weights":
        hq, hkv, d = c["hq"], c["hkv"], c["d"]
        std = math.sqrt((128 + E) / d) if d > 128 else 1.0
        s.update(q=normal(T, hq, d, std=std), k_pool=normal(n_pages, P, hkv, d),
                 weight=normal(S, cap, dtype=torch.float32).exp(),
                 weight_out=torch.zeros(S, cap, device="cuda"),
                 seen=_i32([n - m for n, m in zip(ctx, new)]))
    else:
        hkv, d = c["hkv"], c["d"]
        s["dst"] = table(more)
        s["k_pool"] = normal(n_pages, P, hkv, d)
        s["v_pool"] = None if c["latent"] else normal(n_pages, P, hkv, d)
        # weights as tokens leave them: a few rows with much, most with little, some with none
        w = normal(S, cap, dtype=torch.float32, std=2.0).exp()
        s["weight"] = w.masked_fill_(torch.rand(S, cap, generator=g, device="cuda") < 0.02, 0.0)
        m = c["high"]
        s.update(src_row=torch.zeros(S, m, dtype=torch.int32, device="cuda"),
                 new_len=_i32([0] * S), weight_out=torch.zeros(S, m, device="cuda"))
        s["theta"] = _theta(E if c["latent"] else d)
        s["theta_dev"] = s["theta"].cuda()
    if own:
        # the scratch that a program keeps for its calls
        from paper_2609_34653_amd import evict as ev, latent as la
        n = 0
        if kind == "decode":
            n = la.omnitide_latent_decode_workspace_bytes(S, c["nq"], cap, c["heads"], c["latent"])
        elif kind == "chunk":
            n = la.omnitide_latent_chunk_attn_workspace_bytes(T, S, sum(ctx), c["heads"], c["d"])
        elif kind == "weights":
            n = ev.omnitide_paged_attn_weights_workspace_bytes(T, S, cap, max(new), c["hq"],
                                                               c["hkv"], c["d"])
        elif kind == "evict":
            n = ev.omnitide_evict_plan_workspace_bytes(S, cap)
        s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    return s


# ---------------------------------------------------------------------------------- plain forms

def _plain_turn(x, theta, angle_at, style):
    """x [T, H, E] in float32 turned to angle_at [T] (whole numbers)."""
    phi = angle_at.double()[:, None] * theta
    cos, sin = (f(phi).float()[:, None, :] for f in (torch.cos, torch.sin))
    x = x.float()
    if style == HALF:
        n = x.shape[-1] // 2
        a, b = x[..., :n], x[..., n:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)


def _plain_rows(s):
    """(sequence, row) of each new token."""
    start = s["start"].long()
    t = torch.arange(sum(s["new"]), device=start.device)
    seq = (t[:, None] >= start[None, 1:]).sum(1)
    return seq, s["ctx"].long()[seq] - start[seq + 1] + t


def _plain_append(s):
    c = s["c"]
    R, P = c["latent"], c["page"]
    seq, row = _plain_rows(s)
    slot = s["table"].long()[seq, row // P] * P + row % P
    x = s["latent"].float()
    if s["weight"] is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s["weight"].float()
    k = _plain_turn(s["k_rope"][:, None], s["theta_dev"], row, c["style"])[:, 0]
    s["pool"].view(-1, R + E)[slot] = torch.cat([x, k], -1).to(torch.bfloat16)
    s["q_out"].copy_(_plain_turn(s["q_rope"], s["theta_dev"], row, c["style"]))
    return s["pool"], s["q_out"]


def _plain_gather(s, pool, i):
    """Rows in use of sequence i."""
    n, P = s["ctx_host"][i], s["c"]["page"]
    return pool[s["table"][i, :-(-n // P)].long()].flatten(0, 1)[:n]


def _plain_attn(x, v, hide):
    """Attention of scores x [..., rows, n] (hidden where `hide`) over v [..., n, d]."""
    x = x.masked_fill_(hide, -math.inf)
    x = torch.exp(x - x.amax(-1, keepdim=True))
    return torch.matmul(x, v) / x.sum(-1, keepdim=True)


def _hidden(m, n):
    """Keys [m, n] that the last m of n tokens do not see."""
    at = torch.arange(n, device="cuda")
    return at[None] > at[n - m:, None]


def _plain_decode(s):
    c = s["c"]
    R, nq, H = c["latent"], c["nq"], c["heads"]
    for i, n in enumerate(s["ctx_host"]):
        kv = _plain_gather(s, s["pool"], i).float()
        x = torch.matmul(s["q"][i].float().flatten(0, 1), kv.t()) * _scale(c)
        o = _plain_attn(x.view(nq, H, n), kv[:, :R], _hidden(nq, n)[:, None])
        s["out"][i] = o.to(torch.bfloat16)
    return s["out"]


def _plain_chunk(s):
    c = s["c"]
    d, t, r = c["d"], 0, 0
    for n, m in zip(s["ctx_host"], s["new"]):
        q = s["q"][t:t + m].float().transpose(0, 1)                    # [H, m, d + E]
        k, v = (s[x][r:r + n].float().transpose(0, 1) for x in "kv")
        x = torch.matmul(q[..., :d], k.transpose(1, 2).contiguous())
        x += torch.matmul(q[..., d:], s["k_rope"][r:r + n].float().t())
        s["out"][t:t + m] = _plain_attn(x.mul_(_scale(c)), v, _hidden(m, n)).transpose(0, 1)
        t, r = t + m, r + n
    return s["out"]


def _plain_weights(s):
    c, t = s["c"], 0
    G = c["hq"] // c["hkv"]
    out = s["weight_out"]
    for i, (n, m) in enumerate(zip(s["ctx_host"], s["new"])):
        k = _plain_gather(s, s["k_pool"], i).float()
        total = torch.zeros(n, device="cuda")
        for g in range(c["hkv"]):
            q = s["q"][t:t + m, g * G:(g + 1) * G].float()
            x = (torch.matmul(q, k[:, g].t()) * _scale(c)).masked_fill_(_hidden(m, n)[:, None],
                                                                        -math.inf)
            x = torch.exp(x - x.amax(-1, keepdim=True))
            total += (x / x.sum(-1, keepdim=True)).sum((0, 1))
        total[:n - m] += DECAY * s["weight"][i, :n - m]
        out[i, :n] = total
        t += m
    return out


DECAY = 0.96875


def _plain_evict(s):
    c, P = s["c"], s["c"]["page"]
    flat = (-1, c["hkv"], c["d"])
    for i, n in enumerate(s["ctx_host"]):
        w = s["weight"][i, :n]
        src = torch.arange(n, device="cuda")
        if n > c["high"]:
            # those in the middle by weight, ties to the lower row
            lo, hi = c["sink"], n - c["recent"]
            order = torch.sort(w[lo:hi], descending=True, stable=True).indices
            best = lo + order[:c["budget"] - c["sink"] - c["recent"]]
            src = torch.cat([src[:lo], best.sort().values, src[hi:]])
        m = src.numel()
        s["src_row"][i, :m] = src
        s["new_len"][i] = m
        s["weight_out"][i, :m] = w[src]
        dst = torch.arange(m, device="cuda")
        at = s["table"][i].long()[src // P] * P + src % P
        to = s["dst"][i].long()[dst // P] * P + dst % P
        k = s["k_pool"].view(flat)[at]
        a = c["latent"]
        turned = _plain_turn(k[..., a:], s["theta_dev"], dst - src, c["style"]).to(torch.bfloat16)
        s["k_pool"].view(flat)[to] = torch.cat([k[..., :a], turned], -1)
        if s["v_pool"] is not None:
            s["v_pool"].view(flat)[to] = s["v_pool"].view(flat)[at]
    return _evicted(s)


def _evicted(s):
    out = (s["src_row"], s["new_len"], s["weight_out"], s["k_pool"])
    return out if s["v_pool"] is None else out + (s["v_pool"],)


# ------------------------------------------------------------------------------------------ run

def run(s):
    c, kind = s["c"], s["c"]["kind"]
    if not own:
        if kind == "rows":
            parts = [_plain_gather(s, s["pool"], i) for i in range(c["seqs"])]
            return torch.cat(parts, out=s["out"])
        return dict(append=_plain_append, decode=_plain_decode, chunk=_plain_chunk,
                    weights=_plain_weights, evict=_plain_evict)[kind](s)
    from paper_2609_34653_amd import evict as ev, latent as la
    if kind == "append":
        la.omnitide_latent_append(s["latent"], s["k_rope"], s["pool"], s["table"], s["start"],
                                  s["ctx"], theta=s["theta"], rope_style=c["style"],
                                  latent_weight=s["weight"], eps=EPS, q_rope=s["q_rope"],
                                  q_out=s["q_out"], d_status=s["status"])
        return s["pool"], s["q_out"]
    if kind == "rows":
        la.omnitide_paged_rows(s["pool"], s["table"], s["row_start"], s["ctx"], s["out"],
                               s["status"])
    elif kind == "decode":
        la.omnitide_latent_decode_attn(s["q"], s["pool"], s["table"], s["ctx"], _scale(c), s["out"],
                                       s["ws"], s["status"])
    elif kind == "chunk":
        la.omnitide_latent_chunk_attn(s["q"], s["k"], s["v"], s["k_rope"], s["start"],
                                      s["kv_start"], _scale(c), s["out"], s["ws"], s["status"])
    elif kind == "weights":
        ev.omnitide_paged_attn_weights(s["q"], s["k_pool"], s["table"], s["start"], s["ctx"],
                                       max(s["new"]), _scale(c), s["weight_out"],
                                       weight_in=s["weight"], seen_len=s["seen"], decay=DECAY,
                                       workspace=s["ws"], d_status=s["status"])
        return s["weight_out"]
    else:
        ev.omnitide_evict_plan(s["weight"], s["ctx"], c["high"], c["budget"], c["sink"], c["recent"],
                               s["src_row"], s["new_len"], weight_out=s["weight_out"],
                               workspace=s["ws"], d_status=s["status"])
        ev.omnitide_paged_compact(s["k_pool"], s["v_pool"], s["table"], s["ctx"], s["dst"],
                                  s["src_row"], s["new_len"], theta=s["theta"],
                                  rope_style=c["style"], rope_offset=c["latent"],
                                  d_status=s["status"])
        return _evicted(s)
    return s["out"]


def work(c):
    kind = c["kind"]
    ctx, new = _lens(c)
    n, T = sum(ctx), sum(new)
    pairs = sum(m * k - m * (m - 1) // 2 for k, m in zip(ctx, new))
    table = 8 * c["seqs"] + 4 * n // c.get("page", n)
    if kind == "append":
        e = 4 if c["f32"] else 2
        vals = T * (c["latent"] + E + c["heads"] * E)
        return dict(bytes=vals * (e + 2) + table, flops=6 * vals)
    if kind == "rows":
        return dict(bytes=4 * n * c["width"] + table, flops=0)
    if kind == "decode":
        R, H = c["latent"], c["heads"]
        return dict(bytes=2 * n * (R + E) + 2 * T * H * (2 * R + E) + table,
                    flops=2 * pairs * H * (2 * R + E))
    if kind == "chunk":
        H, d = c["heads"], c["d"]
        return dict(bytes=2 * n * (2 * H * d + E) + 2 * T * H * (2 * d + E),
                    flops=2 * pairs * H * (2 * d + E))
    if kind == "weights":
        return dict(bytes=2 * n * c["hkv"] * c["d"] + 8 * n + 2 * T * c["hq"] * c["d"] + table,
                    flops=2 * pairs * c["hq"] * c["d"])
    m = sum(_kept(c))
    row = 2 * c["hkv"] * c["d"] * (1 if c["latent"] else 2)
    return dict(bytes=4 * n + 2 * m * row + 12 * m + table,
                flops=3 * m * c["hkv"] * (E if c["latent"] else c["d"]))


# ------------------------------------------------------------------------------------- exact

def _exact_turn(x, theta, at, interleaved):
    """x [T, H, dims] in float64, each pair as a complex number times its turn."""
    x = x.double()
    k = theta.numel()
    turn = torch.polar(torch.ones(at.numel(), k, dtype=torch.float64, device=x.device),
                       at.double()[:, None] * theta)
    first = torch.arange(k, device=x.device) * (2 if interleaved else 1)
    second = first + (1 if interleaved else k)
    z = torch.complex(x[..., first], x[..., second]) * turn[:, None]
    y = torch.empty_like(x)
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_keep(w, c):
    """Rows kept of one sequence's weights (a host list)."""
    n = len(w)
    if n <= c["high"]:
        return list(range(n))
    middle = sorted(range(c["sink"], n - c["recent"]), key=lambda r: (-w[r], r))
    return (list(range(c["sink"])) +
            sorted(middle[:c["budget"] - c["sink"] - c["recent"]]) +
            list(range(n - c["recent"], n)))


def exact(c, seed):
    s = prepare(c, seed)
    kind = c["kind"]
    ctx, new = _lens(c)
    P = c.get("page", 1)

    def rows(pool, i, n):
        r = torch.arange(n, device="cuda")
        return pool[s["table"][i][r // P].long(), r % P].double()

    if kind == "rows":
        return torch.cat([rows(s["pool"], i, n) for i, n in enumerate(ctx)])
    if kind == "append":
        R, pool, t, qs = c["latent"], s["pool"].double(), 0, []
        for i, (n, m) in enumerate(zip(ctx, new)):
            r = torch.arange(n - m, n, device="cuda")
            x = s["latent"][t:t + m].double()
            if c["norm"]:
                x = x / (x.square().sum(-1, keepdim=True) / R + EPS).sqrt() * s["weight"].double()
            turned = lambda y: _exact_turn(y, s["theta_dev"], r, c["style"] == INTERLEAVED)  # noqa: E731
            k = turned(s["k_rope"][t:t + m, None])[:, 0]
            pool[s["table"][i][r // P].long(), r % P] = torch.cat([x, k], 1)
            qs.append(turned(s["q_rope"][t:t + m]))
            t += m
        return pool, torch.cat(qs)
    if kind == "decode":
        out, R = [], c["latent"]
        for i, n in enumerate(ctx):
            kv = rows(s["pool"], i, n)
            for j in range(c["nq"]):
                seen = kv[:n - c["nq"] + 1 + j]
                w = torch.softmax(s["q"][i, j].double() @ seen.t() * _scale(c), -1)
                out.append(w @ seen[:, :R])
        return torch.stack(out).view(s["out"].shape)
    if kind == "chunk":
        out, d, t, r = [], c["d"], 0, 0
        for n, m in zip(ctx, new):
            seen = torch.ones(m, n, dtype=torch.bool, device="cuda").tril(n - m)
            kr, heads = s["k_rope"][r:r + n].double(), []
            for h in range(c["heads"]):
                k = torch.cat([s["k"][r:r + n, h].double(), kr], 1)
                w = (s["q"][t:t + m, h].double() @ k.t()) * _scale(c)
                w = torch.softmax(w.masked_fill(~seen, -math.inf), -1)
                heads.append(w @ s["v"][r:r + n, h].double())
            out.append(torch.stack(heads, 1))
            t, r = t + m, r + n
        return torch.cat(out)
    if kind == "weights":
        out, t = s["weight_out"].double(), 0
        for i, (n, m) in enumerate(zip(ctx, new)):
            k = rows(s["k_pool"], i, n)
            seen = torch.ones(m, n, dtype=torch.bool, device="cuda").tril(n - m)
            out[i, :n - m] = DECAY * s["weight"][i, :n - m].double()
            for h in range(c["hq"]):
                w = s["q"][t:t + m, h].double() @ k[:, h // (c["hq"] // c["hkv"])].t() * _scale(c)
                out[i, :n] += torch.softmax(w.masked_fill(~seen, -math.inf), -1).sum(0)
            t += m
        return out
    k, v, a = s["k_pool"].double(), s["v_pool"], c["latent"]
    v = None if v is None else v.double()
    weight = s["weight"].tolist()
    for i, n in enumerate(ctx):
        keep = _exact_keep(weight[i][:n], c)
        m = len(keep)
        src, to = torch.tensor(keep, device="cuda"), torch.arange(m, device="cuda")
        s["src_row"][i, :m], s["new_len"][i] = src.int(), m
        s["weight_out"][i, :m] = s["weight"][i][src]
        x = k[s["table"][i][src // P].long(), src % P]
        x[..., a:] = _exact_turn(x[..., a:], s["theta_dev"], to - src, c["style"] == INTERLEAVED)
        page, line = s["dst"][i][to // P].long(), to % P
        k[page, line] = x
        if v is not None:
            v[page, line] = v[s["table"][i][src // P].long(), src % P]
    out = (s["src_row"], s["new_len"], s["weight_out"], k)
    return out if v is None else out + (v,)
