"""Performance cases of the KV-cache operators (``paper_2607_12659_gb300/kv.py``, ``include/jpi_kv.h``).

A program that serves a model keeps a KV cache and, per step, codes the positions of the new tokens and
writes their keys and values into it (``append``), attends over it where many requests share one long
prefix (``attend``), accumulates the attention weight that each cached key received (``weigh``) and, when the
cache is full, keeps the keys with the most of it (``evict``). A case is one call of one of them on
inputs made from a seed; the handle, the caches and the output buffers are the program's own, made with
the inputs.

Caches are [caches][rows][KV heads][head dim] (``head_major``: stored [caches][KV heads][rows][head dim]).
Keys, values and new tokens are N(0, 1), queries N(0, 2^2): attention scores of std 2, as trained weights
have them. Attention weights to evict by are squared normals: a few large, many small, as accumulated
softmax weights are.
"""

from __future__ import annotations

import math
from types import SimpleNamespace

import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
# (heads, KV heads, head dim): the shapes of the expert and the LLM, of the small fp32 expert, of the correction
# module's heads, and generic ones with shared, unshared and odd head counts.
_SHAPES = [(8, 1, 256), (8, 1, 256), (4, 1, 64), (8, 8, 128), (32, 8, 128), (16, 16, 64), (6, 2, 80), (14, 2, 128),
           (12, 3, 96)]


def listed():
    return [
        # One generated token of one request: the shortest call there is, all latency.
        {"name": "append_b1", "kind": "append", "dtype": "bf16", "heads": 8, "kv_heads": 1, "head_dim": 256,
         "batch": 1, "tokens": 1,
         "rows": 867, "layout": "half", "dim": 256, "scaling": "none", "max_pos": 866, "head_major": False},
        # A token for each of 64 requests far into a long context: interleaved pairs, half of the head
        # coded, frequencies scaled by parts, a head-major cache.
        {"name": "append_b64_far", "kind": "append", "dtype": "bf16", "heads": 32, "kv_heads": 8, "head_dim": 128,
         "batch": 64,
         "tokens": 1, "rows": 512, "layout": "interleaved", "dim": 64, "scaling": "by_parts", "max_pos": 131071,
         "head_major": True},
        # Four prompts of up to 2048 tokens at the LLM's shapes, padded to the longest.
        {"name": "append_prompts", "kind": "append", "dtype": "bf16", "heads": 8, "kv_heads": 1, "head_dim": 256,
         "batch": 4,
         "tokens": 2048, "rows": 2100, "layout": "half", "dim": 256, "scaling": "linear", "max_pos": 2047,
         "head_major": False},
        # One token over one observation's prefix: latency.
        {"name": "attend_b1", "kind": "attend", "dtype": "bf16", "heads": 8, "kv_heads": 1, "head_dim": 256,
         "batch": 1, "tokens": 1,
         "groups": 1, "prefix": 816, "own": 40, "mask": "causal"},
        # The expert's layer: 16 action chunks of 51 suffix tokens, 8 drawn from each of two observations.
        {"name": "attend_b16_chunks", "kind": "attend", "dtype": "bf16", "heads": 8, "kv_heads": 1, "head_dim": 256,
         "batch": 16,
         "tokens": 51, "groups": 2, "prefix": 816, "own": 51, "mask": "context"},
        # 64 continuations of one long prompt, one token each, one KV head.
        {"name": "attend_b64_long", "kind": "attend", "dtype": "bf16", "heads": 8, "kv_heads": 1, "head_dim": 256,
         "batch": 64,
         "tokens": 1, "groups": 1, "prefix": 16384, "own": 512, "mask": "causal"},
        # 48 continuations of a longer one, eight KV heads, an odd length.
        {"name": "attend_b48_gqa", "kind": "attend", "dtype": "bf16", "heads": 32, "kv_heads": 8, "head_dim": 128,
         "batch": 48,
         "tokens": 1, "groups": 1, "prefix": 30011, "own": 1000, "mask": "causal"},
        # The fp32 verification mode at the small expert's shapes.
        {"name": "attend_fp32", "kind": "attend", "dtype": "fp32", "heads": 4, "kv_heads": 1, "head_dim": 64,
         "batch": 4, "tokens": 9,
         "groups": 1, "prefix": 333, "own": 9, "mask": "context"},
        # The weight that a prompt's last 32 tokens give to its keys, before the cache is cut.
        {"name": "weigh_window", "kind": "weigh", "dtype": "bf16", "heads": 8, "kv_heads": 1, "head_dim": 256,
         "batch": 1, "tokens": 32,
         "groups": 1, "prefix": 2048, "own": 32, "mask": "causal"},
        # The weight that 64 continuations give to their shared prompt in one step.
        {"name": "weigh_b64_long", "kind": "weigh", "dtype": "bf16", "heads": 8, "kv_heads": 1, "head_dim": 256,
         "batch": 64,
         "tokens": 1, "groups": 1, "prefix": 16384, "own": 512, "mask": "causal"},
        # The expert's store: half of an observation's 816 keys, every layer by its own weights.
        {"name": "evict_b1", "kind": "evict", "dtype": "bf16", "heads": 8, "kv_heads": 1, "head_dim": 256,
         "layers": 18, "caches": 1,
         "rows": 816, "keep": 408, "sink": 4, "recent": 48},
        # Four long caches of eight KV heads cut to a quarter.
        {"name": "evict_long", "kind": "evict", "dtype": "bf16", "heads": 32, "kv_heads": 8, "head_dim": 128,
         "layers": 4, "caches": 4,
         "rows": 16384, "keep": 4096, "sink": 4, "recent": 256},
    ]


def _heads(case):
    return case["heads"], case["kv_heads"], case["head_dim"]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "weigh", "weigh", "evict"])
    H, K, D = rng.choice(_SHAPES)
    dtype = "fp32" if rng.random() < 0.15 else "bf16"
    c = {"kind": kind, "dtype": dtype, "heads": H, "kv_heads": K, "head_dim": D}
    if kind == "append":
        batch = _log(rng, 1, 64)
        tokens = 1 if rng.random() < 0.4 else _log(rng, 2, 2048)
        while batch * tokens * (H + 2 * K) * D > 8192 * 10 * 256 // (2 if dtype == "fp32" else 1):
            batch, tokens = max(1, batch // 2), max(1, (2 * tokens) // 3)
        c.update(batch=batch, tokens=tokens, rows=tokens + rng.randint(0, 100),
                 layout=rng.choice(["half", "interleaved"]), dim=rng.choice([D, D, D // 2, 16]),
                 scaling=rng.choice(["none", "linear", "ntk", "by_parts"]),
                 max_pos=tokens - 1 + _log(rng, 1, 1 << 20), head_major=rng.random() < 0.3)
        return c
    if kind == "evict":
        layers, caches, rows = _log(rng, 1, 18), _log(rng, 1, 8), _log(rng, 16, 16384)
        keep = rng.randint(max(1, rows // 8), rows)
        while layers * caches * keep * K * D > 16 * 4096 * 8 * 128 // (2 if dtype == "fp32" else 1):
            layers, caches, rows, keep = max(1, layers // 2), max(1, caches // 2), rows // 2 + 1, keep // 2
        sink = min(rng.choice([0, 1, 4]), keep)
        c.update(layers=layers, caches=caches, rows=rows, keep=keep, sink=sink,
                 recent=rng.randint(0, (keep - sink) // 2))
        return c
    groups = rng.choice([1, 1, 1, 2, 3])
    batch = groups * _log(rng, 1, 64 // groups)
    tokens = 1 if rng.random() < 0.6 else _log(rng, 2, 64)
    prefix, tail = _log(rng, 1, 32768), tokens + _log(rng, 1, 1024)
    # Neither more arithmetic nor more cache than the largest listed case has.
    ops, cells = (64 * 8 * 16384 * 256, 30011 * 8 * 128) if kind == "attend" else (64 * 8 * 16384 * 256, 16384 * 256)
    if dtype == "fp32":
        ops, cells = ops // 64, cells // 4
    while (batch * tokens * H * (prefix + tail) * D > ops or groups * prefix * K * D > cells
           or batch * tail * K * D > cells // 2):
        prefix = max(1, prefix // 2)
        if batch * tail * K * D > cells // 2 or batch * tokens * H * tail * D > ops // 2:
            batch, tail = groups * max(1, batch // groups // 2), tokens + max(1, (tail - tokens) // 2)
    c.update(batch=batch, tokens=tokens, groups=groups, prefix=prefix, own=tail,
             mask=rng.choice(["causal", "causal", "context"]))
    return c


def _rope_args(case):
    """The rotary coding of a case, as keywords of kv.Rope."""
    a = dict(dim=case["dim"], layout=case["layout"], base=10000.0, scaling=case["scaling"])
    if case["scaling"] in ("linear", "ntk"):
        a.update(factor=4.0)
    elif case["scaling"] == "by_parts":
        a.update(factor=16.0, low=1.0, high=32.0, original=8192, mscale=0.1 * math.log(16.0) + 1.0)
    return a


def _inputs(case, seed):
    """Every input of a case, on the GPU, from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = _DT[case["dtype"]]
    H, K, D = _heads(case)

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * std).to(dt)

    def ints(lo, hi, *shape):
        return torch.randint(lo, hi + 1, shape, generator=gen, device="cuda", dtype=torch.int32)

    s = SimpleNamespace(case=case)
    if case["kind"] == "append":
        B, T, R = case["batch"], case["tokens"], case["rows"]
        # The projections of a layer come as one row a token: queries, then keys, then values.
        s.qkv = normal(B, T, H + 2 * K, D)
        if case["head_major"]:
            s.K, s.V = (normal(B, K, R, D).transpose(1, 2) for _ in range(2))
        else:
            s.K, s.V = (normal(B, R, K, D) for _ in range(2))
        t = torch.arange(T, device="cuda", dtype=torch.int32)[None]
        start = ints(0, case["max_pos"] - (T - 1), B, 1)
        first = ints(0, R - T, B, 1)
        valid = ints(max(1, T // 2), T, B, 1)
        s.positions = (start + t).contiguous()
        s.rows = torch.where(t < valid, first + t, torch.full_like(first + t, -1))
        s.q_out = torch.zeros((B, T, H, D), dtype=dt, device="cuda")
    elif case["kind"] == "evict":
        L, N, R = case["layers"], case["caches"], case["rows"]
        s.K, s.V = (normal(L, N, R, K, D) for _ in range(2))
        s.w = torch.randn((L, N, K, R), generator=gen, device="cuda").square()
        s.length = ints(R - R // 16, R, N)
        s.outK, s.outV = (torch.zeros((L, N, case["keep"], K, D), dtype=dt, device="cuda") for _ in range(2))
        s.outw = torch.zeros((L, N, K, case["keep"]), device="cuda")
        s.outlen = torch.zeros((N,), dtype=torch.int32, device="cuda")
    else:
        B, T, G, P, R = case["batch"], case["tokens"], case["groups"], case["prefix"], case["own"]
        s.q = normal(B, T, H, D, std=2.0)
        s.pK, s.pV = (normal(G, P, K, D) for _ in range(2))
        s.oK, s.oV = (normal(B, R, K, D) for _ in range(2))
        s.prefix_len = ints(P - P // 16, P, G)
        t = torch.arange(T, device="cuda", dtype=torch.int32)[None]
        length = ints(T, R, B, 1)
        if case["mask"] == "causal":      # the T newest rows of each request see what came before them
            s.seen = (length - T + 1 + t).contiguous()
        else:                             # the first token sees itself only, the others every row
            s.seen = torch.where(t == 0, torch.ones_like(length), length).contiguous()
        if case["kind"] == "attend":
            s.out = torch.zeros((B, T, H, D), dtype=dt, device="cuda")
            s.lse = torch.zeros((B, T, H), device="cuda")
        else:
            s.lse = _row_lse(s, torch.float64).float()
            s.w_prefix = torch.randn((G, K, P), generator=gen, device="cuda").square()
            s.w_own = torch.randn((B, K, R), generator=gen, device="cuda").square()
            s.out_prefix, s.out_own = torch.zeros_like(s.w_prefix), torch.zeros_like(s.w_own)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2607_12659_gb300 import kv

        H, K, D = _heads(case)
        s.h = kv.KV(H, K, D, max_batch=case.get("batch", 1), max_tokens=case.get("tokens", 1), precision=case["dtype"],
                    rope=kv.Rope(**_rope_args(case)) if case["kind"] == "append" else None)
    return s


# ------------------------------------------------------------------ plain forms

def _theta(a):
    """Angle per position of each rotary pair, 64 bits."""
    i = torch.arange(a["dim"] // 2, device="cuda", dtype=torch.float64)
    base = a["base"]
    if a["scaling"] == "ntk":
        base = base * a["factor"] ** (a["dim"] / (a["dim"] - 2))
    th = base ** (-2.0 * i / a["dim"])
    if a["scaling"] == "linear":
        return th / a["factor"]
    if a["scaling"] == "by_parts":
        turns = a["original"] * th / (2.0 * math.pi)
        g = ((turns - a["low"]) / (a["high"] - a["low"])).clamp(0.0, 1.0)
        return (1.0 - g) * th / a["factor"] + g * th
    return th


def _plain_append(s):
    a = _rope_args(s.case)
    H, K, D = _heads(s.case)
    ang = s.positions.double()[..., None] * _theta(a)                       # [B][T][dim / 2], 64 bits
    m = a.get("mscale", 1.0)
    c, si = (ang.cos() * m).float()[:, :, None], (ang.sin() * m).float()[:, :, None]
    x = s.qkv[:, :, :H + K].float()
    n = a["dim"]
    y = x.clone()
    if a["layout"] == "half":
        x1, x2 = x[..., :n // 2], x[..., n // 2:n]
        y[..., :n // 2], y[..., n // 2:n] = x1 * c - x2 * si, x2 * c + x1 * si
    else:
        x1, x2 = x[..., 0:n:2], x[..., 1:n:2]
        y[..., 0:n:2], y[..., 1:n:2] = x1 * c - x2 * si, x2 * c + x1 * si
    y = y.to(s.qkv.dtype)
    b, t = (s.rows >= 0).nonzero(as_tuple=True)                             # padding: nothing is written
    r = s.rows[b, t].long()
    s.q_out[b, t] = y[b, t, :H]
    s.K[b, r] = y[b, t, H:]
    s.V[b, r] = s.qkv[b, t, H + K:]
    return s.q_out, s.K, s.V


def _scores(s, dt):
    """Scaled scores [B][T][KV heads][heads per KV head][keys] over the shared prefix and the own rows, -inf where
    a key is not seen."""
    c = s.case
    H, K, D = _heads(c)
    B, T, G, P, R = c["batch"], c["tokens"], c["groups"], c["prefix"], c["own"]
    q = s.q.to(dt).reshape(G, (B // G) * T, K, H // K, D).permute(0, 2, 1, 3, 4)          # G K nT gq D
    sp = q.reshape(G, K, -1, D) @ s.pK.to(dt).permute(0, 2, 3, 1)                         # G K (nT gq) P
    sp = sp.reshape(G, K, B // G, T, H // K, P).permute(0, 2, 3, 1, 4, 5).reshape(B, T, K, H // K, P)
    qo = s.q.to(dt).reshape(B, T, K, H // K, D).permute(0, 2, 1, 3, 4).reshape(B, K, -1, D)
    so = (qo @ s.oK.to(dt).permute(0, 2, 3, 1)).reshape(B, K, T, H // K, R).permute(0, 2, 1, 3, 4)
    scale = 1.0 / math.sqrt(D)
    hid_p = torch.arange(P, device="cuda")[None] >= s.prefix_len[:, None]                 # G P
    hid_p = hid_p.repeat_interleave(B // G, 0)[:, None, None, None]
    hid_o = (torch.arange(R, device="cuda") >= s.seen[..., None])[:, :, None, None]       # B T 1 1 R
    return (sp * scale).masked_fill(hid_p, -math.inf), (so * scale).masked_fill(hid_o, -math.inf)


def _row_lse(s, dt):
    """log of the sum of exp(score) of every query row, [B][T][H]."""
    sp, so = _scores(s, dt)
    m = torch.maximum(sp.amax(-1), so.amax(-1))
    safe = torch.where(m == -math.inf, torch.zeros_like(m), m)[..., None]
    tot = (sp - safe).exp().sum(-1) + (so - safe).exp().sum(-1)
    return (safe[..., 0] + tot.log()).reshape(s.q.shape[:3])


def _plain_attend(s):
    c = s.case
    H, K, D = _heads(c)
    B, T, G = c["batch"], c["tokens"], c["groups"]
    sp, so = _scores(s, torch.float32)
    m = torch.maximum(sp.amax(-1), so.amax(-1))
    safe = torch.where(m == -math.inf, torch.zeros_like(m), m)[..., None]
    pp, po = (sp - safe).exp(), (so - safe).exp()
    tot = pp.sum(-1) + po.sum(-1)
    pg = pp.reshape(G, B // G, T, K, H // K, -1).permute(0, 3, 1, 2, 4, 5).reshape(G, K, -1, pp.shape[-1])
    o = (pg @ s.pV.float().permute(0, 2, 1, 3)).reshape(G, K, B // G, T, H // K, D)
    o = o.permute(0, 2, 3, 1, 4, 5).reshape(B, T, K, H // K, D)
    og = po.permute(0, 2, 1, 3, 4).reshape(B, K, T * (H // K), -1) @ s.oV.float().permute(0, 2, 1, 3)
    o = o + og.reshape(B, K, T, H // K, D).permute(0, 2, 1, 3, 4)
    some = tot[..., None] > 0
    o = torch.where(some, o / torch.where(some, tot[..., None], torch.ones_like(o)), torch.zeros_like(o))
    return o.reshape(B, T, H, D).to(s.q.dtype), (safe[..., 0] + tot.log()).reshape(B, T, H)


def _plain_weigh(s):
    c = s.case
    H, K, D = _heads(c)
    B, T, G = c["batch"], c["tokens"], c["groups"]
    sp, so = _scores(s, torch.float32)
    lse = s.lse.reshape(B, T, K, H // K, 1)
    some = lse > -math.inf
    lse = torch.where(some, lse, torch.zeros_like(lse))
    pp = torch.where(some, (sp - lse).exp(), torch.zeros_like(sp)).sum((1, 3))                 # B K P
    po = torch.where(some, (so - lse).exp(), torch.zeros_like(so)).sum((1, 3))                 # B K R
    pp = pp.reshape(G, B // G, K, -1).sum(1)
    live_p = (torch.arange(pp.shape[-1], device="cuda") < s.prefix_len[:, None])[:, None]
    live_o = (torch.arange(po.shape[-1], device="cuda") < s.seen.amax(1)[:, None])[:, None]
    # Entries of rows that hold no key are left as they were.
    s.out_prefix.copy_(torch.where(live_p, 0.9 * s.w_prefix + pp, s.out_prefix))
    s.out_own.copy_(torch.where(live_o, 0.9 * s.w_own + po, s.out_own))
    return s.out_prefix, s.out_own


def _plain_evict(s):
    c = s.case
    L, N, R, keep = c["layers"], c["caches"], c["rows"], c["keep"]
    K = c["kv_heads"]
    j = torch.arange(R, device="cuda")[None]
    n = s.length[:, None]
    # First rows and newest rows first of all, rows past the end last of all, then by weight; ties to the lowest row.
    rank = torch.where((j < c["sink"]) | (j >= n - c["recent"]), math.inf, 0.0)
    rank = torch.where(j >= n, -math.inf, rank)[None, :, None]                                 # 1 N 1 R
    order = torch.sort(torch.where(rank == 0, s.w, rank.expand_as(s.w)), dim=-1, descending=True, stable=True)[1]
    kept = torch.sort(order[..., :keep], dim=-1)[0]                                            # L N K keep
    new = s.length.clamp(max=keep)
    live = (torch.arange(keep, device="cuda")[None] < new[:, None])[None, :, None]             # 1 N 1 keep
    kept = torch.where(live, kept, torch.full_like(kept, -1))
    at = kept.clamp(min=0)
    rows = at.permute(0, 1, 3, 2)[..., None].expand(L, N, keep, K, c["head_dim"])
    livek = live.permute(0, 1, 3, 2)[..., None]
    s.outK.copy_(torch.where(livek, s.K.gather(2, rows), s.outK))
    s.outV.copy_(torch.where(livek, s.V.gather(2, rows), s.outV))
    s.outw.copy_(torch.where(live, s.w.gather(3, at), s.outw))
    s.outlen.copy_(new)
    return kept.int(), s.outK, s.outV, s.outw, s.outlen


def run(s):
    kind = s.case["kind"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "weigh": _plain_weigh, "evict": _plain_evict}[kind](s)
    c = s.case
    H, K, D = _heads(c)
    if kind == "append":
        s.h.append(s.qkv[:, :, :H], s.qkv[:, :, H:H + K], s.qkv[:, :, H + K:], s.positions, s.rows, s.K, s.V,
                   q_out=s.q_out)
        return s.q_out, s.K, s.V
    if kind == "attend":
        return s.h.attend(s.q, prefix=(s.pK, s.pV), prefix_len=s.prefix_len, own=(s.oK, s.oV), seen=s.seen, out=s.out,
                          lse=s.lse)
    if kind == "weigh":
        return s.h.weigh(s.q, s.lse, prefix=s.pK, prefix_len=s.prefix_len, own=s.oK, seen=s.seen, w_prefix=s.w_prefix,
                         w_own=s.w_own, decay=0.9, out_prefix=s.out_prefix, out_own=s.out_own)
    kept = s.h.evict(s.K, s.V, s.w, s.length, c["keep"], sink=c["sink"], recent=c["recent"], out_k=s.outK, out_v=s.outV,
                     out_w=s.outw, out_length=s.outlen)
    return kept, s.outK, s.outV, s.outw, s.outlen


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    H, K, D = _heads(case)
    if case["kind"] == "append":
        n = case["batch"] * case["tokens"]
        return {"bytes": n * (2 * (H + 2 * K) * D * e + 8), "flops": n * 3 * (H + K) * case["dim"]}
    if case["kind"] == "evict":
        c = case["layers"] * case["caches"] * K
        return {"bytes": c * (case["rows"] * 4 + case["keep"] * (4 * D * e + 8)), "flops": c * case["rows"]}
    B, T, G, P, R = case["batch"], case["tokens"], case["groups"], case["prefix"], case["own"]
    pairs = B * T * H * (P + (R + T) / 2)      # own rows: T .. R of them, evenly drawn
    if case["kind"] == "attend":
        return {"bytes": int((G * P + B * (R + T) / 2) * K * D * 2 * e + B * T * H * (2 * D * e + 4)),
                "flops": int(4 * D * pairs)}
    keys = G * P + B * (R + T) / 2
    return {"bytes": int(keys * K * (D * e + 8) + B * T * H * (D * e + 4)), "flops": int(2 * D * pairs)}


# ------------------------------------------------------------------ definitions in 64 bits

def _exact_append(s, case):
    a = _rope_args(case)
    H, K, D = _heads(case)
    n = a["dim"] // 2
    base = a["base"] * (a["factor"] ** (a["dim"] / (a["dim"] - 2.0)) if a["scaling"] == "ntk" else 1.0)
    freq = []
    for i in range(n):
        f = math.exp(-2.0 * i / a["dim"] * math.log(base))
        if a["scaling"] == "linear":
            f /= a["factor"]
        elif a["scaling"] == "by_parts":
            g = min(1.0, max(0.0, (a["original"] * f / (2 * math.pi) - a["low"]) / (a["high"] - a["low"])))
            f = f / a["factor"] * (1.0 - g) + f * g
        freq.append(f)
    rot = torch.polar(torch.full_like(s.positions, a.get("mscale", 1.0), dtype=torch.float64)[..., None],
                      s.positions[..., None].double() * torch.tensor(freq, dtype=torch.float64, device="cuda"))
    x = s.qkv.double()
    i = torch.arange(n, device="cuda")
    lo, hi = (i, i + n) if a["layout"] == "half" else (2 * i, 2 * i + 1)
    z = torch.complex(x[:, :, :H + K][..., lo], x[:, :, :H + K][..., hi]) * rot[:, :, None]
    y = x[:, :, :H + K].clone()
    y[..., lo], y[..., hi] = z.real, z.imag
    q_out, kc, vc = s.q_out.double(), s.K.double().clone(), s.V.double().clone()
    for b in range(case["batch"]):
        ok = s.rows[b] >= 0
        r = s.rows[b][ok].long()
        q_out[b, ok] = y[b, ok, :H]
        kc[b, r] = y[b, ok, H:]
        vc[b, r] = x[b, ok, H + K:]
    return q_out, kc, vc


def _exact_rows(s, case):
    """Per request: (its keys, its values, which of them each of its tokens sees)."""
    n = case["batch"] // case["groups"]
    lens, seen = s.prefix_len.tolist(), s.seen.tolist()
    for b in range(case["batch"]):
        P, top = lens[b // n], max(seen[b])
        k = torch.cat([s.pK[b // n, :P], s.oK[b, :top]]).double()
        v = torch.cat([s.pV[b // n, :P], s.oV[b, :top]]).double()
        vis = torch.ones((case["tokens"], P + top), dtype=torch.bool, device="cuda")
        vis[:, P:] = torch.arange(top, device="cuda")[None] < s.seen[b][:, None]
        yield b, P, top, k, v, vis


def _exact_logits(s, case, b, k, vis):
    H, K, D = _heads(case)
    q = s.q[b].double().reshape(case["tokens"], K, H // K, D)
    lg = torch.einsum("tkgd,jkd->tkgj", q, k) * D ** -0.5
    return lg.masked_fill(~vis[:, None, None], -math.inf)


def _exact_attend(s, case):
    H, K, D = _heads(case)
    out = torch.zeros(s.out.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s.lse.shape, -math.inf, dtype=torch.float64, device="cuda")
    for b, P, top, k, v, vis in _exact_rows(s, case):
        if P + top == 0:
            continue
        lg = _exact_logits(s, case, b, k, vis)
        z = torch.logsumexp(lg, -1, keepdim=True)
        p = torch.where(z > -math.inf, (lg - z).exp(), torch.zeros_like(lg))
        out[b] = torch.einsum("tkgj,jkd->tkgd", p, v).reshape(case["tokens"], H, D)
        lse[b] = z.reshape(case["tokens"], H)
    return out, lse


def _exact_weigh(s, case):
    K = case["kv_heads"]
    wp, wo = s.out_prefix.double(), s.out_own.double()
    n = case["batch"] // case["groups"]
    for g, P in enumerate(s.prefix_len.tolist()):
        wp[g, :, :P] = 0.9 * s.w_prefix[g, :, :P].double()
    for b, P, top, k, v, vis in _exact_rows(s, case):
        lse = s.lse[b].double().reshape(case["tokens"], K, -1, 1)
        lg = _exact_logits(s, case, b, k, vis)
        p = torch.where(lse > -math.inf, (lg - lse).exp(), torch.zeros_like(lg)).sum((0, 2))   # K keys
        wp[b // n, :, :P] += p[:, :P]
        wo[b, :, :top] = 0.9 * s.w_own[b, :, :top].double() + p[:, P:]
    return wp, wo


def _exact_evict(s, case):
    """The kept rows by counting, per cache, layer and head: copies and whole numbers, with no rounding."""
    kept = torch.full((*s.w.shape[:3], case["keep"]), -1, dtype=torch.int32, device="cuda")
    K, V, w = s.outK.double(), s.outV.double(), s.outw.double()
    for n, m in enumerate(s.length.tolist()):
        k = min(m, case["keep"])
        for l in range(case["layers"]):
            for h in range(case["kv_heads"]):
                free = s.w[l, n, h, :m].double().clone()
                free[:case["sink"]] = math.inf
                if case["recent"]:
                    free[max(0, m - case["recent"]):] = math.inf
                at = torch.argsort(-free, stable=True)[:k].sort()[0]
                kept[l, n, h, :k] = at.int()
                K[l, n, :k, h], V[l, n, :k, h] = s.K[l, n, at, h].double(), s.V[l, n, at, h].double()
                w[l, n, h, :k] = s.w[l, n, h, at].double()
    return kept, K, V, w, s.length.clamp(max=case["keep"])


_EXACT = {"append": _exact_append, "attend": _exact_attend, "weigh": _exact_weigh, "evict": _exact_evict}


def exact(case, seed):
    s = _inputs(case, seed)
    return _EXACT[case["kind"]](s, case)
