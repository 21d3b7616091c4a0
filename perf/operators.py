"""The operators around a paged KV cache, as measurable cases: norm and rotation of queries and
keys, the append of new keys and values to the pages, chunk attention over the pages and its
single-token form, from one token of one stream to ragged batches over long contexts.

A case's structure (context and chunk lengths) follows from the case alone; values and the order
of the pages are drawn on the GPU from the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

HALF, INTERLEAVED = 0, 1
EPS = 1.0e-6


# ------------------------------------------------------------------------------------- cases

def listed():
    return [
        # The 665-token chunk (a frame and a second of audio) of the benchmark's layer: views of
        # one fused projection.
        dict(name="norm_rope_chunk_665", kind="norm_rope", tokens=665, hq=32, hkv=8, d=128,
             f32=False, rope=128, style=HALF, norm=True, scaled=False),
        # A long prompt of a small float32 model: interleaved pairs, half of the head rotated,
        # frequencies scaled for a longer context, no norms.
        dict(name="rope_f32_partial_23k", kind="norm_rope", tokens=23041, hq=14, hkv=2, d=64,
             f32=True, rope=32, style=INTERLEAVED, norm=False, scaled=True),
        # One generated token for each of 24 streams: q, k and v of the step in one call.
        dict(name="append_24x1tok", kind="append", seqs=24, q_lo=1, q_hi=1, ctx_lo=600,
             ctx_hi=9173, page=64, hq=32, hkv=8, d=128, f32=False, rope=128, style=HALF,
             norm=True, scaled=False, with_q=True),
        # Chunks of different lengths of six streams at once, keys and values alone.
        dict(name="append_6_chunks", kind="append", seqs=6, q_lo=89, q_hi=2329, ctx_lo=2400,
             ctx_hi=16384, page=128, hq=32, hkv=8, d=128, f32=False, rope=128, style=HALF,
             norm=False, scaled=True, with_q=False),
        # A float32 model's long prompts into small bf16 pages, part of the head rotated.
        dict(name="append_f32_prompts", kind="append", seqs=3, q_lo=9000, q_hi=12011,
             ctx_lo=12288, ctx_hi=14000, page=16, hq=16, hkv=4, d=128, f32=True, rope=64,
             style=INTERLEAVED, norm=True, scaled=False, with_q=True),
        # The smallest stream of the tests: an 89-token chunk over 512 kept tokens.
        dict(name="chunk_attn_89_tiny", kind="chunk", seqs=1, q_lo=89, q_hi=89, ctx_lo=601,
             ctx_hi=601, page=32, hq=4, hkv=1, d=64),
        # The benchmark's chunk over one layer's 17K retained tokens, in 64-token pages.
        dict(name="chunk_attn_665_17k", kind="chunk", seqs=1, q_lo=665, q_hi=665, ctx_lo=17048,
             ctx_hi=17048, page=64, hq=32, hkv=8, d=128),
        # Streams at different points of their turn in one call: a few tokens beside whole
        # chunks, short contexts beside long ones, small pages.
        dict(name="chunk_attn_8_ragged", kind="chunk", seqs=8, q_lo=1, q_hi=1500, ctx_lo=1840,
             ctx_hi=18001, page=16, hq=28, hkv=4, d=128),
        # High-resolution frames (2,304 tokens and a second of audio) of four streams at once.
        dict(name="chunk_attn_4_hires", kind="chunk", seqs=4, q_lo=2329, q_hi=2329, ctx_lo=10521,
             ctx_hi=10521, page=128, hq=32, hkv=8, d=128),
        # One generated token over one layer's 17K retained tokens.
        dict(name="decode_1x17k", kind="decode", seqs=1, nq=1, ctx_lo=16948, ctx_hi=16948,
             page=64, hq=32, hkv=8, d=128),
        # Two tokens (a drafted one beside the last) of 24 streams of unequal length.
        dict(name="decode_24_ragged_2tok", kind="decode", seqs=24, nq=2, ctx_lo=600,
             ctx_hi=20000, page=128, hq=32, hkv=8, d=128),
        # Many short and a few very long streams, eight query heads per KV head, small pages.
        dict(name="decode_96_ragged", kind="decode", seqs=96, nq=1, ctx_lo=200, ctx_hi=60000,
             page=16, hq=16, hkv=2, d=128),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(4, 1, 64), (14, 2, 64), (16, 4, 128), (16, 2, 128), (28, 4, 128), (32, 8, 128),
          (32, 8, 128), (8, 8, 64)]


def draw(rng):
    kind = rng.choice(["norm_rope", "append", "chunk", "chunk", "decode", "decode"])
    hq, hkv, d = rng.choice(_HEADS)
    c = dict(kind=kind, hq=hq, hkv=hkv, d=d)
    if kind in ("norm_rope", "append"):
        c.update(f32=rng.random() < 0.3, rope=rng.choice([32, d // 2, d, d]),
                 style=rng.choice([HALF, HALF, INTERLEAVED]), norm=rng.random() < 0.5,
                 scaled=rng.random() < 0.3)
    if kind == "norm_rope":
        c.update(tokens=_log(rng, 1, 25000000 // ((hq + hkv) * d)))
        return c
    c.update(page=rng.choice([16, 32, 64, 64, 128, 256]))
    if kind == "append":
        seqs = _log(rng, 1, 64)
        hi = _log(rng, 1, 20000 // seqs)
        c.update(seqs=seqs, q_lo=max(1, hi // rng.choice([1, 4, 20])), q_hi=hi, ctx_lo=hi,
                 ctx_hi=hi + _log(rng, 1, 20000 // seqs), with_q=rng.random() < 0.6)
    elif kind == "chunk":
        seqs, hi, q_hi = _log(rng, 1, 12), _log(rng, 300, 20000), _log(rng, 2, 2400)
        q_hi = max(1, min(q_hi, hi, 2000000000 // (seqs * hq * hi)))
        c.update(seqs=seqs, q_lo=max(1, q_hi // rng.choice([1, 3, 100])), q_hi=q_hi,
                 ctx_lo=max(q_hi, hi // rng.choice([1, 2, 10])), ctx_hi=hi)
    else:
        seqs = _log(rng, 1, 96)
        hi = _log(rng, 400, max(800, min(60000, 250000000 // (seqs * hkv * d))))
        c.update(seqs=seqs, nq=rng.randint(1, max(1, 8 // (hq // hkv))),
                 ctx_lo=max(8, hi // rng.choice([1, 3, 50])), ctx_hi=hi)
    return c


# --------------------------------------------------------------------------------- structure

def _lens(c):
    """(context length with the new tokens, new tokens) of each sequence."""
    rng = random.Random("%d %d %d %d" % (c["seqs"], c["ctx_lo"], c["ctx_hi"], c["page"]))
    ctx = [_log(rng, c["ctx_lo"], c["ctx_hi"]) for _ in range(c["seqs"])]
    if c["kind"] == "decode":
        return ctx, [c["nq"]] * c["seqs"]
    return ctx, [min(n, _log(rng, c["q_lo"], c["q_hi"])) for n in ctx]


def _theta(c):
    """Frequencies of the rotated pairs; scaled: those that turn slowly over 32,768 positions
    are lowered to an eighth, the fastest keep their value, a ramp between."""
    R = c["rope"]
    t = 1.0e6 ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)
    if c["scaled"]:
        w = ((32768.0 * t / (2.0 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
        t = t * (w + (1.0 - w) / 8.0)
    return t


def _magnitude(c):
    return 0.1 * math.log(8.0) + 1.0 if c["scaled"] else 1.0


# ------------------------------------------------------------------------------------ inputs

def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    hq, hkv, d, kind = c["hq"], c["hkv"], c["d"], c["kind"]
    s = dict(c=c)

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(*shape, generator=g, device="cuda").to(dtype)

    if kind != "norm_rope":
        ctx, new = _lens(c)
        S, P, T = c["seqs"], c["page"], sum(new)
        pages = [-(-n // P) for n in ctx]
        n_pages = sum(pages) + 3
        order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
        table = torch.full((S, max(pages)), -1, dtype=torch.int32, device="cuda")
        at = 0
        for i, n in enumerate(pages):
            table[i, :n] = order[at:at + n]
            at += n
        s.update(table=table, ctx=_i32(ctx),
                 start=_i32([sum(new[:i]) for i in range(S + 1)]), max_new=max(new))
        s["k_pool"], s["v_pool"] = normal(n_pages, P, hkv, d), normal(n_pages, P, hkv, d)
    if kind in ("norm_rope", "append"):
        dt = torch.float32 if c["f32"] else torch.bfloat16
        if kind == "norm_rope":
            T = c["tokens"]
            # positions of a stream whose history was cut: increasing, far from zero
            s["pos"] = (torch.arange(T, device="cuda") + 70000).to(torch.int32)
        qkv = normal(T, hq + 2 * hkv, d, dtype=dt)       # one fused projection's output
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        s["theta"] = _theta(c)                           # host and device copies
        s["theta_dev"] = s["theta"].cuda()
        wq, wk = (1.0 + 0.1 * torch.randn(d, generator=g, device="cuda") for _ in range(2))
        s["wq"], s["wk"] = (wq.to(dt), wk.to(dt)) if c["norm"] else (None, None)
        out = dt if kind == "norm_rope" else torch.bfloat16
        s["q_out"] = torch.zeros(T, hq, d, dtype=out, device="cuda")
        s["k_out"] = torch.zeros(T, hkv, d, dtype=out, device="cuda")
        if kind == "append" and not c["with_q"]:
            s["q"] = s["q_out"] = s["wq"] = None
    else:
        s["q"] = normal(T, hq, d) if kind == "chunk" else normal(S, c["nq"], hq, d)
        s["out"] = torch.zeros_like(s["q"])
        s["scale"] = 1.0 / math.sqrt(d)
    s["status"] = _i32([0])
    if own and kind in ("chunk", "decode"):
        # the scratch that a program keeps for its calls
        from paper_2609_34653_amd import paged as pg
        cap = s["table"].shape[1] * P
        n = (pg.omnitide_paged_chunk_attn_workspace_bytes(T, S, cap, hq, hkv, d)
             if kind == "chunk" else
             pg.omnitide_paged_decode_workspace_bytes(S, c["nq"], cap, hq, hkv, d))
        s["ws"] = torch.empty(max(1, n), dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------------- plain forms

def _plain_norm_rope(c, x, w, theta, pos):
    """x [T, H, d] normed per head (w given) and rotated, in float32."""
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    phi = pos.double()[:, None] * theta
    cos, sin = ((_magnitude(c) * f(phi)).float()[:, None, :] for f in (torch.cos, torch.sin))
    R = c["rope"]
    if c["style"] == HALF:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        return torch.cat([a * cos - b * sin, a * sin + b * cos, x[..., R:]], -1)
    a, b = x[..., 0:R:2], x[..., 1:R:2]
    r = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([r, x[..., R:]], -1)


def _plain_rows(s, T):
    """(sequence, cache row) of each of the T new tokens."""
    start = s["start"].long()
    t = torch.arange(T, device=start.device)
    seq = (t[:, None] >= start[None, 1:]).sum(1)
    row = s["ctx"].long()[seq] - start[seq + 1] + t
    return seq, row


def _plain_append(s):
    c = s["c"]
    T, P = s["k"].shape[0], c["page"]
    seq, row = _plain_rows(s, T)
    slot = s["table"].long()[seq, row // P] * P + row % P
    flat = (-1, c["hkv"], c["d"])
    k = _plain_norm_rope(c, s["k"], s["wk"], s["theta_dev"], row)
    s["k_pool"].view(flat)[slot] = k.to(torch.bfloat16)
    s["v_pool"].view(flat)[slot] = s["v"].to(torch.bfloat16)
    if s["q"] is None:
        return s["k_pool"], s["v_pool"]
    s["q_out"].copy_(_plain_norm_rope(c, s["q"], s["wq"], s["theta_dev"], row))
    return s["k_pool"], s["v_pool"], s["q_out"]


def _plain_attn(s, q, row, max_new):
    """q [S, max_new, hq, d] (float32) at cache rows `row` [S, max_new] over the pages."""
    c = s["c"]
    S, hq, hkv, d = c["seqs"], c["hq"], c["hkv"], c["d"]
    table = s["table"].clamp(min=0).long()
    k, v = (p[table].flatten(1, 2).permute(0, 2, 1, 3).float() for p in (s["k_pool"],
                                                                         s["v_pool"]))
    n = k.shape[2]                                      # [S, hkv, n, d]
    hide = torch.arange(n, device=q.device) > row[..., None]            # [S, max_new, n]
    v = v.masked_fill((torch.arange(n, device=q.device) >= s["ctx"][:, None])[:, None, :, None],
                      0.0)
    q = q.view(S, max_new, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).flatten(2, 3)
    x = torch.matmul(q, k.transpose(2, 3)) * s["scale"]               # [S, hkv, G max_new, n]
    x = x.view(S, hkv, hq // hkv, max_new, n).masked_fill_(hide[:, None, None], -math.inf)
    x = torch.exp(x - x.amax(-1, keepdim=True))
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(S, hkv, -1, n), v).view(S, hkv, hq // hkv, max_new, d) / total
    return o.permute(0, 3, 1, 2, 4).reshape(S, max_new, hq, d).to(torch.bfloat16)


def _plain(s):
    c, kind = s["c"], s["c"]["kind"]
    if kind == "norm_rope":
        s["q_out"].copy_(_plain_norm_rope(c, s["q"], s["wq"], s["theta_dev"], s["pos"]))
        s["k_out"].copy_(_plain_norm_rope(c, s["k"], s["wk"], s["theta_dev"], s["pos"]))
        return s["q_out"], s["k_out"]
    if kind == "append":
        return _plain_append(s)
    ctx = s["ctx"].long()
    if kind == "decode":
        row = ctx[:, None] - c["nq"] + torch.arange(c["nq"], device="cuda")
        return _plain_attn(s, s["q"].float(), row, c["nq"])
    # the ragged chunks as one padded batch, aligned at their ends
    m = s["max_new"]
    i = torch.arange(m, device="cuda")
    at = s["start"][1:, None].long() - m + i            # token of each padded place
    real = at >= s["start"][:-1, None]
    q = s["q"][at.clamp(min=0)].float().masked_fill_(~real[..., None, None], 0.0)
    out = _plain_attn(s, q, (ctx[:, None] - m + i).clamp(min=0), m)
    seq, _ = _plain_rows(s, s["q"].shape[0])
    t = torch.arange(s["q"].shape[0], device="cuda")
    return out[seq, m - (s["start"][1:].long()[seq] - t)]


# ------------------------------------------------------------------------------------------ run

def run(s):
    if not own:
        return _plain(s)
    from paper_2609_34653_amd import paged as pg
    c, kind = s["c"], s["c"]["kind"]
    if kind == "norm_rope":
        pg.omnitide_qk_norm_rope(s["q"], s["k"], s["pos"], s["q_out"], s["k_out"], s["theta"],
                                 rope_style=c["style"], magnitude=_magnitude(c),
                                 q_weight=s["wq"], k_weight=s["wk"], eps=EPS)
        return s["q_out"], s["k_out"]
    if kind == "append":
        pg.omnitide_paged_append(s["k"], s["v"], s["k_pool"], s["v_pool"], s["table"],
                                 s["start"], s["ctx"], theta=s["theta"], rope_style=c["style"],
                                 magnitude=_magnitude(c), k_weight=s["wk"], eps=EPS, q=s["q"],
                                 q_out=s["q_out"], q_weight=s["wq"], d_status=s["status"])
        if s["q"] is None:
            return s["k_pool"], s["v_pool"]
        return s["k_pool"], s["v_pool"], s["q_out"]
    if kind == "chunk":
        pg.omnitide_paged_chunk_attn(s["q"], s["k_pool"], s["v_pool"], s["table"], s["start"],
                                     s["ctx"], s["scale"], s["out"], s["ws"], s["status"])
    else:
        pg.omnitide_paged_decode_attn(s["q"], s["k_pool"], s["v_pool"], s["table"], s["ctx"],
                                      s["scale"], s["out"], s["ws"], s["status"])
    return s["out"]


def work(c):
    hq, hkv, d, kind = c["hq"], c["hkv"], c["d"], c["kind"]
    e = 4 if c.get("f32") else 2
    if kind == "norm_rope":
        n = c["tokens"] * (hq + hkv) * d
        return dict(bytes=2 * n * e + 4 * c["tokens"], flops=n * (10 if c["norm"] else 6))
    ctx, new = _lens(c)
    tables = 4 * (2 * c["seqs"] + 1) + 4 * sum(-(-n // c["page"]) for n in ctx)
    if kind == "append":
        T = sum(new)
        n = T * (hkv + (hq if c["with_q"] else 0)) * d
        return dict(bytes=(n + T * hkv * d) * (e + 2) + 8 * c["seqs"] + 4 * T // c["page"],
                    flops=n * (10 if c["norm"] else 6))
    pairs = sum(m * n - m * (m - 1) // 2 for n, m in zip(ctx, new))
    return dict(bytes=sum(ctx) * hkv * d * 4 + 2 * sum(new) * hq * d * 2 + tables,
                flops=4 * pairs * hq * d)


# ------------------------------------------------------------------------------------- exact

def _exact_rotate(x, weight, eps, theta, mag, pos, interleaved):
    """x [T, H, d] in float64: head norm, then each pair as a complex number times its turn."""
    x = x.double()
    if weight is not None:
        x = x / (x.square().sum(-1, keepdim=True) / x.shape[-1] + eps).sqrt() * weight.double()
    n = theta.numel()
    turn = torch.polar(torch.full((pos.numel(), n), float(mag), dtype=torch.float64,
                                  device=x.device), pos.double()[:, None] * theta)
    first = torch.arange(n, device=x.device) * (2 if interleaved else 1)
    second = first + (1 if interleaved else n)
    z = torch.complex(x[..., first], x[..., second]) * turn[:, None]
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(c, seed):
    s = prepare(c, seed)
    kind = c["kind"]
    if kind in ("norm_rope", "append"):
        turned = lambda x, w, p: _exact_rotate(x, w, EPS, s["theta_dev"], _magnitude(c), p,  # noqa: E731
                                               c["style"] == INTERLEAVED)
        if kind == "norm_rope":
            return turned(s["q"], s["wq"], s["pos"]), turned(s["k"], s["wk"], s["pos"])
    ctx, new = _lens(c)
    if kind == "append":
        kp, vp = s["k_pool"].double(), s["v_pool"].double()
        q, at = [], 0
        for i, (n, m) in enumerate(zip(ctx, new)):
            r = torch.arange(n - m, n, device="cuda")
            page, line = s["table"][i][r // c["page"]].long(), r % c["page"]
            kp[page, line] = turned(s["k"][at:at + m], s["wk"], r)
            vp[page, line] = s["v"][at:at + m].double()
            if c["with_q"]:
                q.append(turned(s["q"][at:at + m], s["wq"], r))
            at += m
        return (kp, vp, torch.cat(q)) if c["with_q"] else (kp, vp)
    group, out, at = c["hq"] // c["hkv"], [], 0
    q = s["q"].view(-1, c["hq"], c["d"])
    for i, (n, m) in enumerate(zip(ctx, new)):
        pages = s["table"][i, :-(-n // c["page"])].long()
        k, v = (p[pages].flatten(0, 1)[:n].double() for p in (s["k_pool"], s["v_pool"]))
        seen = torch.ones(m, n, dtype=torch.bool, device="cuda").tril(n - m)
        heads = []
        for h in range(c["hq"]):
            w = (q[at:at + m, h].double() @ k[:, h // group].t()) / math.sqrt(c["d"])
            w = torch.softmax(w.masked_fill(~seen, -math.inf), -1)
            heads.append(w @ v[:, h // group])
        out.append(torch.stack(heads, 1))
        at += m
    return torch.cat(out).view(s["q"].shape)
