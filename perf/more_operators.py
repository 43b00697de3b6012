"""Performance cases of further KV-cache operators (``paper_2607_12659_gb300/kv.py``, ``include/jpi_kv.h``).

Around a KV cache a program that serves a model also normalises each head's queries and keys before their
rotary coding, in the pass that writes the cache (``append`` with a ``norm``); keeps a cache in 8 bits with a scale for
each block of tokens and head (``append8``) and attends over it (``attend8``); and lets a token see a window of the
newest rows and a few first ones only (``attend_window``, and the same of an 8-bit cache). A case is one call of
one of them on inputs made from a seed; the handle, the caches and the output buffers are the program's own,
made with the inputs.

Caches are [caches][rows][KV heads][head dim] (``head_major``: stored [caches][KV heads][rows][head dim]). An 8-bit cache
holds e4m3 codes and, per cache, KV head and block of rows, a power of two that they are multiplied by (e8m0); both come back
in those types, whose values they are. New tokens' keys and values are N(0, 1) times a gain of each request's own, as layers
and prompts differ, so that some blocks' scales grow as a token comes; keys have a few large channels. Queries are N(0, 1.5^2).
"""

from __future__ import annotations

import math
from types import SimpleNamespace

import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
_EPS = 1e-6
# (heads, KV heads, head dim): the shapes of the expert and the LLM, of the small fp32 expert, of the correction
# module's heads, and generic ones with shared, unshared and odd head counts.
_SHAPES = [(8, 1, 256), (8, 1, 256), (4, 1, 64), (8, 8, 128), (32, 8, 128), (16, 16, 64), (6, 2, 80), (14, 2, 128),
           (12, 3, 96)]


def listed():
    return [
        # One generated token of one request, its heads normalised, coded and written: all latency.
        {"name": "norm_b1", "kind": "norm", "dtype": "bf16", "heads": 8, "kv_heads": 1, "head_dim": 256, "batch": 1,
         "tokens": 1, "rows": 867, "layout": "half", "dim": 256, "scaling": "none", "max_pos": 866, "head_major": False},
        # Four prompts of up to 2048 tokens at the LLM's shapes, padded to the longest.
        {"name": "norm_prompts", "kind": "norm", "dtype": "bf16", "heads": 8, "kv_heads": 1, "head_dim": 256, "batch": 4,
         "tokens": 2048, "rows": 2100, "layout": "half", "dim": 256, "scaling": "linear", "max_pos": 2047,
         "head_major": False},
        # A token for each of 64 requests into 8-bit caches of eight KV heads, far into a context, interleaved pairs.
        {"name": "append8_b64", "kind": "append8", "dtype": "bf16", "heads": 32, "kv_heads": 8, "head_dim": 128,
         "batch": 64, "tokens": 1, "rows": 2048, "block": 32, "layout": "interleaved", "dim": 64, "scaling": "by_parts",
         "max_pos": 131071, "norm": False},
        # Four prompts into 8-bit caches, normalised, from rows inside a block on.
        {"name": "append8_prompts", "kind": "append8", "dtype": "bf16", "heads": 8, "kv_heads": 1, "head_dim": 256,
         "batch": 4, "tokens": 2048, "rows": 2100, "block": 64, "layout": "half", "dim": 256, "scaling": "none",
         "max_pos": 2047, "norm": True},
        # One token that sees the newest 1024 rows of a long cache and its first 4: latency.
        {"name": "window_b1", "kind": "window", "dtype": "bf16", "heads": 8, "kv_heads": 1, "head_dim": 256, "batch": 1,
         "tokens": 1, "rows": 16384, "window": 1024, "sink": 4},
        # A token for each of 64 requests, eight KV heads, a window of 4096.
        {"name": "window_b64_gqa", "kind": "window", "dtype": "bf16", "heads": 32, "kv_heads": 8, "head_dim": 128,
         "batch": 64, "tokens": 1, "rows": 6001, "window": 4096, "sink": 4},
        # Two prompts of up to 4096 tokens, each token with its own window.
        {"name": "window_prompts", "kind": "window", "dtype": "bf16", "heads": 8, "kv_heads": 1, "head_dim": 256,
         "batch": 2, "tokens": 4096, "rows": 4096, "window": 1024, "sink": 4},
        # The fp32 verification mode at the small expert's shapes.
        {"name": "window_fp32", "kind": "window", "dtype": "fp32", "heads": 4, "kv_heads": 1, "head_dim": 64, "batch": 4,
         "tokens": 9, "rows": 1333, "window": 300, "sink": 3},
        # One token over one observation's cache in 8 bits: latency.
        {"name": "attend8_b1", "kind": "attend8", "dtype": "bf16", "heads": 8, "kv_heads": 1, "head_dim": 256, "batch": 1,
         "tokens": 1, "rows": 867, "block": 32, "window": 0, "sink": 0},
        # A token for each of 64 requests over long contexts of one KV head.
        {"name": "attend8_b64_long", "kind": "attend8", "dtype": "bf16", "heads": 8, "kv_heads": 1, "head_dim": 256,
         "batch": 64, "tokens": 1, "rows": 16384, "block": 64, "window": 0, "sink": 0},
        # 48 requests of eight KV heads, an odd length, small blocks.
        {"name": "attend8_b48_gqa", "kind": "attend8", "dtype": "bf16", "heads": 32, "kv_heads": 8, "head_dim": 128,
         "batch": 48, "tokens": 1, "rows": 5003, "block": 16, "window": 0, "sink": 0},
        # The expert's layer over observations kept in 8 bits: 16 chunks of 51 suffix tokens.
        {"name": "attend8_chunks", "kind": "attend8", "dtype": "bf16", "heads": 8, "kv_heads": 1, "head_dim": 256,
         "batch": 16, "tokens": 51, "rows": 867, "block": 32, "window": 0, "sink": 0},
    ]


def _heads(case):
    return case["heads"], case["kv_heads"], case["head_dim"]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "append8", "window", "window", "attend8", "attend8"])
    H, K, D = rng.choice(_SHAPES)
    dtype = "fp32" if rng.random() < 0.15 else "bf16"
    c = {"kind": kind, "dtype": dtype, "heads": H, "kv_heads": K, "head_dim": D}
    if kind in ("norm", "append8"):
        batch = _log(rng, 1, 64)
        tokens = 1 if rng.random() < 0.4 else _log(rng, 2, 2048)
        while batch * tokens * (H + 2 * K) * D > 8192 * 10 * 256 // (2 if dtype == "fp32" else 1):
            batch, tokens = max(1, batch // 2), max(1, (2 * tokens) // 3)
        c.update(batch=batch, tokens=tokens, rows=tokens + _log(rng, 1, 1000), layout=rng.choice(["half", "interleaved"]),
                 dim=rng.choice([D, D, D // 2, 16]), scaling=rng.choice(["none", "linear", "ntk", "by_parts"]),
                 max_pos=tokens - 1 + _log(rng, 1, 1 << 20))
        if kind == "norm":
            c.update(head_major=rng.random() < 0.3)
        else:
            c.update(block=rng.choice([16, 32, 64]), norm=rng.random() < 0.5)
        return c
    batch = _log(rng, 1, 64)
    tokens = 1 if rng.random() < 0.6 else _log(rng, 2, 2048 if kind == "window" else 256)
    rows = tokens + _log(rng, 1, 16384)
    # Neither more arithmetic nor more cache than the largest listed case of the kind has.
    ops, cells = (2 * 4096 * 8 * 4096 * 256, 64 * 6001 * 8 * 128) if kind == "window" else (64 * 8 * 16384 * 256, 64 * 16384 * 256)
    if dtype == "fp32":
        ops, cells = ops // 64, cells // 4
    while batch * tokens * H * rows * D > ops or batch * rows * K * D > cells:
        if batch > 1 and rng.random() < 0.5:
            batch = batch // 2
        else:
            tokens = max(1, tokens // 2)
            rows = tokens + max(1, (rows - tokens) // 2)
    c.update(batch=batch, tokens=tokens, rows=rows)
    windowed = kind == "window" or rng.random() < 0.3
    c.update(window=_log(rng, 1, rows) if windowed else 0, sink=rng.choice([0, 1, 4, 4, 17]) if windowed else 0)
    if kind == "attend8":
        c.update(block=rng.choice([16, 32, 64]))
    return c


def _rope_args(case):
    """The rotary coding of a case, as keywords of kv.Rope."""
    a = dict(dim=case["dim"], layout=case["layout"], base=10000.0, scaling=case["scaling"])
    if case["scaling"] in ("linear", "ntk"):
        a.update(factor=4.0)
    elif case["scaling"] == "by_parts":
        a.update(factor=16.0, low=1.0, high=32.0, original=8192, mscale=0.1 * math.log(16.0) + 1.0)
    return a


def _pow2(e):
    """2^(e - 127) as fp32 for integers 1 .. 254."""
    return (e.int() << 23).view(torch.float32)


def _exponent(amax):
    """The scale's byte: the least e in 1 .. 254 with amax <= 448 2^(e - 127)."""
    m, x = torch.frexp(amax)                      # amax = m 2^x, 1/2 <= m < 1; 448 = 7/8 2^9
    e = torch.where(amax > 0, x - 9 + (m > 0.875).int() + 127, torch.ones_like(x))
    return e.clamp(1, 254)


def _inputs(case, seed):
    """Every input of a case, on the GPU, from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = _DT[case["dtype"]]
    kind = case["kind"]
    H, K, D = _heads(case)
    B, T, R = case["batch"], case["tokens"], case["rows"]

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * std).to(dt)

    def ints(lo, hi, *shape):
        return torch.randint(lo, hi + 1, shape, generator=gen, device="cuda", dtype=torch.int32)

    large = torch.where(torch.arange(D, device="cuda") % 29 == 11, 4.0, 1.0)     # a few large channels of the keys

    def held8():
        """A cache in 8 bits: codes and the scales of its blocks."""
        n = -(-R // case["block"])
        codes, scales = [], []
        for wide in (large, torch.ones_like(large)):
            x = torch.randn((B, n, case["block"], K, D), generator=gen, device="cuda") * wide
            x *= torch.exp(0.5 * torch.randn((B, n, 1, K, 1), generator=gen, device="cuda"))
            e = _exponent(x.abs().amax((2, 4)))                                  # B n K
            x *= _pow2(254 - e)[:, :, None, :, None]
            codes.append(x.to(torch.float8_e4m3fn).reshape(B, -1, K, D)[:, :R].contiguous())
            scales.append(e.to(torch.uint8).transpose(1, 2).contiguous().view(torch.float8_e8m0fnu))
        return codes, scales

    s = SimpleNamespace(case=case)
    if kind in ("norm", "append8"):
        # The projections of a layer come as one row a token: queries, then keys, then values.
        gain = torch.exp(0.7 * torch.randn((B, 1, 1, 1), generator=gen, device="cuda")).to(dt)
        s.qkv = normal(B, T, H + 2 * K, D) * gain
        s.qkv[:, :, H:H + K] *= large.to(dt)
        s.q_weight, s.k_weight = (1.0 + 0.2 * torch.randn((D,), generator=gen, device="cuda") for _ in range(2))
        t = torch.arange(T, device="cuda", dtype=torch.int32)[None]
        start = ints(0, case["max_pos"] - (T - 1), B, 1)
        first = ints(0, R - T, B, 1)
        valid = ints(max(1, T // 2), T, B, 1)
        s.positions = (start + t).contiguous()
        s.q_out = torch.zeros((B, T, H, D), dtype=dt, device="cuda")
        if kind == "norm":
            if case["head_major"]:
                s.K, s.V = (normal(B, K, R, D).transpose(1, 2) for _ in range(2))
            else:
                s.K, s.V = (normal(B, R, K, D) for _ in range(2))
            s.rows = torch.where(t < valid, first + t, torch.full_like(first + t, -1))
        else:
            (s.K, s.V), (s.k_scale, s.v_scale) = held8()
            s.start, s.count = first[:, 0].contiguous(), valid[:, 0].contiguous()
        return s
    s.q = normal(B, T, H, D, std=1.5)
    if kind == "window":
        s.K, s.V = ((torch.randn((B, R, K, D), generator=gen, device="cuda") * w).to(dt) for w in (large, torch.ones_like(large)))
    else:
        (s.K, s.V), (s.k_scale, s.v_scale) = held8()
    # The newest rows of each cache are its tokens' own; a shorter request's last tokens are padding that sees nothing.
    t = torch.arange(T, device="cuda", dtype=torch.int32)[None]
    length = ints(max(T, R - R // 8), R, B, 1)
    valid = ints(T - T // 8, T, B, 1)
    s.seen = torch.where(t < valid, length - T + 1 + t, torch.zeros_like(length)).contiguous()
    s.out = torch.zeros((B, T, H, D), dtype=dt, device="cuda")
    s.lse = torch.zeros((B, T, H), device="cuda")
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2607_12659_gb300 import kv

        H, K, D = _heads(case)
        s.h = kv.KV(H, K, D, max_batch=case["batch"], max_tokens=case["tokens"], precision=case["dtype"],
                    rope=kv.Rope(**_rope_args(case)) if "dim" in case else None)
        if "block" in case:
            s.cache = kv.Cache8(s.K, s.V, s.k_scale, s.v_scale, case["block"])
        if case["kind"] == "norm" or case.get("norm"):
            s.norm = kv.Norm(s.q_weight, s.k_weight, _EPS)
        else:
            s.norm = None
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


def _plain_coded(s, norm):
    """Queries and keys, normalised and coded, fp32 [B][T][H + K][D]."""
    a = _rope_args(s.case)
    H, K, D = _heads(s.case)
    ang = s.positions.double()[..., None] * _theta(a)                       # [B][T][dim / 2], 64 bits
    m = a.get("mscale", 1.0)
    c, si = (ang.cos() * m).float()[:, :, None], (ang.sin() * m).float()[:, :, None]
    x = s.qkv[:, :, :H + K].float()
    if norm:
        w = torch.cat([s.q_weight.expand(H, D), s.k_weight.expand(K, D)])
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPS) * w
    n = a["dim"]
    y = x.clone()
    if a["layout"] == "half":
        x1, x2 = x[..., :n // 2], x[..., n // 2:n]
        y[..., :n // 2], y[..., n // 2:n] = x1 * c - x2 * si, x2 * c + x1 * si
    else:
        x1, x2 = x[..., 0:n:2], x[..., 1:n:2]
        y[..., 0:n:2], y[..., 1:n:2] = x1 * c - x2 * si, x2 * c + x1 * si
    return y


def _plain_norm(s):
    H, K, D = _heads(s.case)
    y = _plain_coded(s, True).to(s.qkv.dtype)
    b, t = (s.rows >= 0).nonzero(as_tuple=True)                             # padding: nothing is written
    r = s.rows[b, t].long()
    s.q_out[b, t] = y[b, t, :H]
    s.K[b, r] = y[b, t, H:]
    s.V[b, r] = s.qkv[b, t, H + K:]
    return s.q_out, s.K, s.V


def _plain_store8(s, x, cache, scale):
    """Writes x [B][T][K][D] (fp32) into the rows start .. start + count - 1 of 8-bit caches: a block that holds rows before
    `start` keeps its scale or has it raised, its codes with it; the others get the scale that their new rows need."""
    c = s.case
    B, T, R, n = c["batch"], c["tokens"], c["rows"], c["block"]
    nb = (T + 2 * n - 2) // n                                               # blocks that T rows can touch
    start = s.start.long()[:, None]
    b = torch.arange(B, device="cuda")[:, None]
    f = start // n * n + torch.arange(nb * n, device="cuda")                # B F: the rows of those blocks
    t = f - start
    new = (t >= 0) & (t < s.count[:, None]) & (f < R)
    kept = t < 0
    at, blocks = f.clamp(max=R - 1), (f[:, ::n] // n).clamp(max=scale.shape[2] - 1)
    x = torch.where(new[..., None, None], x[b, t.clamp(0, T - 1)], 0.0)      # B F K D
    bits = scale.view(torch.uint8)
    e_old = bits[b, :, blocks].int()                                        # B nb K
    fine = torch.where(x.abs() < math.inf, x.abs(), 0.0)                    # (neither infinities nor NaN set a scale)
    e = _exponent(fine.reshape(B, nb, n, *x.shape[2:]).amax((2, 4)))
    kept_any, new_any = kept[:, ::n, None], new.reshape(B, nb, n).any(-1)
    e = torch.where(kept_any, torch.maximum(e, e_old), e)
    by = lambda v: v.repeat_interleave(n, 1)[..., None]                     # noqa: E731
    code = x * by(_pow2(254 - e))
    old = cache.view(torch.uint8)[b, at].view(torch.float8_e4m3fn).float() * by(_pow2((e_old - e + 127).clamp(1, 254)))
    code = torch.where(new[..., None, None], code, old).to(torch.float8_e4m3fn).view(torch.uint8)
    bi, fi = (new | (kept & new_any.repeat_interleave(n, 1))).nonzero(as_tuple=True)
    cache.view(torch.uint8)[bi, f[bi, fi]] = code[bi, fi]
    bi, ni = new_any.nonzero(as_tuple=True)
    bits[bi, :, blocks[bi, ni]] = e[bi, ni].to(torch.uint8)


def _plain_append8(s):
    H, K, D = _heads(s.case)
    y = _plain_coded(s, s.case["norm"])
    t = torch.arange(s.case["tokens"], device="cuda")[None]
    b, t = ((t < s.count[:, None]) & (s.start[:, None] + t < s.case["rows"])).nonzero(as_tuple=True)
    s.q_out[b, t] = y[b, t, :H].to(s.qkv.dtype)
    _plain_store8(s, y[:, :, H:], s.K, s.k_scale)
    _plain_store8(s, s.qkv[:, :, H + K:].float(), s.V, s.v_scale)
    return s.q_out, s.K, s.V, s.k_scale, s.v_scale


def _plain_values8(s, cache, scale):
    n = s.case["block"]
    by = scale.float().transpose(1, 2).repeat_interleave(n, 1)[:, :cache.shape[1], :, None]
    return cache.float() * by


def _plain_attend(s):
    c = s.case
    H, K, D = _heads(c)
    B, T, R = c["batch"], c["tokens"], c["rows"]
    if c["kind"] == "attend8":
        k, v = _plain_values8(s, s.K, s.k_scale), _plain_values8(s, s.V, s.v_scale)
    else:
        k, v = s.K.float(), s.V.float()
    q = s.q.float().reshape(B, T, K, H // K, D).transpose(1, 2).reshape(B, K, T * (H // K), D)
    sc = ((q @ k.permute(0, 2, 3, 1)) * (1.0 / math.sqrt(D))).reshape(B, K, T, H // K, R)
    j = torch.arange(R, device="cuda")
    hidden = j >= s.seen[..., None]                                          # B T R
    if c["window"]:
        hidden |= (j >= c["sink"]) & (j < s.seen[..., None] - c["window"])
    sc = sc.masked_fill(hidden[:, None, :, None], -math.inf)
    m = sc.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = (sc - m).exp()
    tot = p.sum(-1, keepdim=True)
    o = (p.reshape(B, K, T * (H // K), R) @ v.transpose(1, 2)).reshape(B, K, T, H // K, D)
    o = torch.where(tot > 0, o / torch.where(tot > 0, tot, torch.ones_like(tot)), torch.zeros_like(o))
    return (o.transpose(1, 2).reshape(B, T, H, D).to(s.q.dtype),
            (m + tot.log())[..., 0].transpose(1, 2).reshape(B, T, H))


_PLAIN = {"norm": _plain_norm, "append8": _plain_append8, "window": _plain_attend, "attend8": _plain_attend}


def run(s):
    c = s.case
    kind = c["kind"]
    if not own:
        return _PLAIN[kind](s)
    H, K, D = _heads(c)
    if kind in ("norm", "append8"):
        q, k, v = s.qkv[:, :, :H], s.qkv[:, :, H:H + K], s.qkv[:, :, H + K:]
        if kind == "norm":
            s.h.append(q, k, v, s.positions, s.rows, s.K, s.V, q_out=s.q_out, norm=s.norm)
            return s.q_out, s.K, s.V
        s.h.append8(q, k, v, s.positions, s.start, s.cache, count=s.count, norm=s.norm, q_out=s.q_out)
        return s.q_out, s.K, s.V, s.k_scale, s.v_scale
    if kind == "window":
        return s.h.attend_window(s.q, (s.K, s.V), s.seen, c["window"], sink=c["sink"], out=s.out, lse=s.lse)
    return s.h.attend8(s.q, s.cache, s.seen, window=c["window"], sink=c["sink"], out=s.out, lse=s.lse)


def _spans(case):
    """(rows of its cache that a request reads, rows that its tokens see in all), on the average of the lengths."""
    T, R = case["tokens"], case["rows"]
    n = (max(T, R - R // 8) + R) / 2                                         # rows of the last token
    live = T - T // 16                                                       # tokens that are no padding
    if not case["window"]:
        return n - T + live, sum(n - T + 1 + t for t in range(live))
    w, sink = case["window"], case["sink"]
    first = max(0.0, n - T + 1 - w)                                          # the first token's window begins here
    pairs = sum(min(n - T + 1 + t, w + min(sink, max(0.0, n - T + 1 + t - w))) for t in range(live))
    return n - T + live - first + min(sink, first), pairs


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    H, K, D = _heads(case)
    B, T = case["batch"], case["tokens"]
    if case["kind"] in ("norm", "append8"):
        n = B * (max(1, T // 2) + T) / 2                                     # tokens that are no padding
        normed = 4 * D * (H + K) if case["kind"] == "norm" or case["norm"] else 0
        held = 2 * K * D * e if case["kind"] == "norm" else 2 * K * (D + 1 / case["block"])
        return {"bytes": int(n * ((H + 2 * K) * D * e + H * D * e + held + 4)),
                "flops": int(n * (3 * (H + K) * case["dim"] + normed + (4 * K * D if case["kind"] == "append8" else 0)))}
    rows, pairs = _spans(case)
    held = D * e if case["kind"] == "window" else D + 1 / case["block"]
    return {"bytes": int(B * rows * K * 2 * held + B * T * (H * (2 * D * e + 4) + 4)), "flops": int(4 * D * B * H * pairs)}


# ------------------------------------------------------------------ definitions in 64 bits

def _exact_coded(s, case, norm):
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
    x = s.qkv[:, :, :H + K].double().clone()
    if norm:
        for lo, hi, w in ((0, H, s.q_weight), (H, H + K, s.k_weight)):
            h = x[:, :, lo:hi]
            x[:, :, lo:hi] = h / ((h * h).sum(-1, keepdim=True) / D + _EPS).sqrt() * w.double()
    i = torch.arange(n, device="cuda")
    lo, hi = (i, i + n) if a["layout"] == "half" else (2 * i, 2 * i + 1)
    z = torch.complex(x[..., lo], x[..., hi]) * rot[:, :, None]
    x[..., lo], x[..., hi] = z.real, z.imag
    return x


def _exact_norm(s, case):
    H, K, D = _heads(case)
    y = _exact_coded(s, case, True)
    q_out, kc, vc = s.q_out.double(), s.K.double().clone(), s.V.double().clone()
    for b in range(case["batch"]):
        ok = s.rows[b] >= 0
        r = s.rows[b][ok].long()
        q_out[b, ok] = y[b, ok, :H]
        kc[b, r] = y[b, ok, H:]
        vc[b, r] = s.qkv[b, ok, H + K:].double()
    return q_out, kc, vc


def _two_to(p):
    """2^p as a 64-bit number (exact, which exp2 and ldexp on the GPU are not)."""
    return ((p.long() + 1023) << 52).view(torch.float64)


def _exact_code(x):
    """The e4m3 value nearest to x (|x| <= 448), ties to the even code."""
    _, p = torch.frexp(x.abs().clamp(min=2.0 ** -6))          # 2^(p - 1) <= |x| < 2^p
    step = _two_to(p - 4)
    return torch.round(x / step) * step


def _exact_scale(amax):
    """The least power of two with amax <= 448 of it."""
    m, p = torch.frexp(amax / 448.0)
    return _two_to(torch.where(m > 0.5, p, p - 1))


def _exact_append8(s, case):
    H, K, D = _heads(case)
    n, R = case["block"], case["rows"]
    y = torch.cat([_exact_coded(s, case, case["norm"]), s.qkv[:, :, H + K:].double()], 2)
    q_out = s.q_out.double()
    codes = [s.K.double(), s.V.double()]
    scales = [s.k_scale.double(), s.v_scale.double()]
    for b, (first, count) in enumerate(zip(s.start.tolist(), s.count.tolist())):
        count = min(count, R - first)
        q_out[b, :count] = y[b, :count, :H]
        for x, code, scale in zip((y[b, :count, H:H + K], y[b, :count, H + K:]), codes, scales):
            for i in range(first // n, (first + count - 1) // n + 1):
                lo, hi = max(first, i * n), min(first + count, (i + 1) * n)
                part = x[lo - first:hi - first]
                sc = _exact_scale(part.abs().amax((0, 2)))      # K
                if i * n < first:
                    new = torch.maximum(sc, scale[b, :, i])
                    code[b, i * n:first] = _exact_code(code[b, i * n:first] * (scale[b, :, i] / new)[None, :, None])
                    sc = new
                code[b, lo:hi] = _exact_code(part / sc[None, :, None])
                scale[b, :, i] = sc
    return q_out, codes[0], codes[1], scales[0], scales[1]


def _exact_attend(s, case):
    H, K, D = _heads(case)
    T, R = case["tokens"], case["rows"]
    out = torch.zeros(s.out.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s.lse.shape, -math.inf, dtype=torch.float64, device="cuda")
    j = torch.arange(R, device="cuda")
    for b in range(case["batch"]):
        k, v = s.K[b].double(), s.V[b].double()
        if case["kind"] == "attend8":
            k = k * s.k_scale[b].double()[:, j // case["block"]].T[..., None]
            v = v * s.v_scale[b].double()[:, j // case["block"]].T[..., None]
        seen = s.seen[b][:, None]
        vis = j < seen
        if case["window"]:
            vis = vis & ((j < case["sink"]) | (j >= seen - case["window"]))
        for h in range(K):
            q = s.q[b].double().reshape(T, K, H // K, D)[:, h]
            lg = (torch.einsum("tgd,jd->tgj", q, k[:, h]) * D ** -0.5).masked_fill(~vis[:, None], -math.inf)
            z = torch.logsumexp(lg, -1, keepdim=True)
            p = torch.where(z > -math.inf, (lg - z).exp(), torch.zeros_like(lg))
            out[b].reshape(T, K, H // K, D)[:, h] = torch.einsum("tgj,jd->tgd", p, v[:, h])
            lse[b].reshape(T, K, H // K)[:, h] = z[..., 0]
    return out, lse


_EXACT = {"norm": _exact_norm, "append8": _exact_append8, "window": _exact_attend, "attend8": _exact_attend}


def exact(case, seed):
    s = _inputs(case, seed)
    return _EXACT[case["kind"]](s, case)
