"""Attention over windows and over 8-bit caches on the GPU against their fp64 oracle.

Tolerances are those of the other attention tests (test_gpu_kv.py): worst-case bounds from the formats and the lengths of the sums.
Over an 8-bit cache a query may enter the first product as fp16 at a power of two of its own (an element off by at most 2^-25 of
its head's largest), and a probability the second as fp16: off by half of fp16's least step 2^-24, in units of 2^-4 of a
probability times the largest scale seen, under which a value is at most 448 and the largest at least half of that: 2^-28 of the largest.
"""

import math

import numpy as np
import pytest

from oracle import kv as okv
from test_gpu_kv import DT, HALF_EPS, SHAPES, head_major, i32, kv, np64, padded, rand, tiles, within  # noqa: F401
from test_gpu_kv_heads import fill8, head_major8, padded8

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BAD = (float("nan"), float("inf"), -float("inf"))


def counts(rng, mask, B, T, R):
    if mask == "causal":
        top = rng.integers(0, R + 1, B)
        return np.clip(top[:, None] - T + 1 + np.arange(T), 0, None)
    if mask == "full":
        return np.clip(R - T + 1 + np.arange(T), 0, None)[None].repeat(B, 0)
    return rng.integers(-1, R + 2, (B, T))


def hidden(seen, R, window, sink):
    """[B][R]: rows that no token of a request sees."""
    h = np.ones((seen.shape[0], R), bool)
    for b in range(seen.shape[0]):
        for n in set(seen[b].tolist()):
            h[b, okv.visible(n, R, window, sink)] = False
    return h


def tols(q, k, v, n, dtype, ref, dot, mass, lse, scale):
    D = q.shape[-1]
    rel = (D + 2) * 2.0 ** -22 * dot + 2.0 ** -20 + n * 2.0 ** -23 + 2.0 ** -22 * np.where(np.isinf(lse), 0, np.abs(lse))
    rel = rel + scale * 2.0 ** -24 * np.abs(q).max(-1) * np.nanmax(np.abs(np.where(np.isfinite(k), k, 0)).sum(-1))
    big = np.abs(np.where(np.isfinite(v), v, 0)).max()
    out = HALF_EPS[dtype] * np.abs(ref) + (2 * rel[..., None] + (2.0 ** -8 if dtype == "bf16" else 0)) * mass + n * 2.0 ** -28 * big + 1e-37
    return out, rel + 1e-6


def finish(out, lse, again, ref, tol):
    ro, rl, _, _ = ref
    within(out, ro, tol[0], "out")
    within(lse, rl, tol[1], "lse")
    empty = np.isinf(rl)
    assert np.all(np64(out)[empty] == 0) and np.all(np64(lse)[empty] == -np.inf)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1]), "two runs differ"


def check_window(kv, dtype, H, K, D, B, T, R, window, sink, seed=0, mask="causal", store=lambda t: t, scale=0.0):
    rng = np.random.default_rng(seed)
    q, k, v = rand(seed, B, T, H, D, dtype=dtype, std=2.0), rand(seed + 1, B, R, K, D, dtype=dtype), rand(seed + 2, B, R, K, D, dtype=dtype)
    seen = counts(rng, mask, B, T, R)
    # Rows that no token sees hold NaN and infinities.
    h = torch.tensor(hidden(seen, R, window, sink), device="cuda")
    for t, off in ((k, 0), (v, 1)):
        for b in range(B):
            t[b, h[b]] = BAD[(b + off) % 3]
    hd = kv.KV(H, K, D, max_batch=B, max_tokens=T, precision=dtype, scale=scale)
    cache = (store(k), store(v))
    out, lse = hd.attend_window(q, cache, i32(seen), window, sink=sink)
    again = hd.attend_window(q, cache, i32(seen), window, sink=sink)
    hd.device_status()
    sc = scale or 1 / math.sqrt(D)
    ref = okv.attend_window(np64(q), np64(k), np64(v), seen, window, sink, sc)
    finish(out, lse, again, ref, tols(np64(q), np64(k), np64(v), R, dtype, *ref[:1], ref[2], ref[3], ref[1], sc))
    return hd, (q, cache, i32(seen), window, sink), out, lse


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H,K,D", SHAPES)
def test_window_head_shapes(kv, dtype, H, K, D):
    check_window(kv, dtype, H, K, D, 3, 1, 97, 20, 4, seed=H)
    check_window(kv, dtype, H, K, D, 2, 5, 133, 31, 3, seed=H + 1, mask="any")


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("R,window,sink", [(1, 1, 0), (1, 5, 3), (2, 1, 1), (64, 64, 0), (65, 64, 0), (129, 64, 1), (129, 65, 64), (200, 1, 0), (200, 1, 200),
                                           (300, 63, 65), (300, 17, 130), (500, 128, 16), (777, 300, 4), (777, 2147483647, 2147483647), (513, 5, 511)])
def test_window_lengths(kv, dtype, R, window, sink):
    check_window(kv, dtype, 8, 1, 128, 2, 1, R, window, sink, seed=R + sink, mask="full")
    check_window(kv, dtype, 8, 2, 64, 2, 3, R, window, sink, seed=R + window % 100)


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("mask", ["causal", "any", "full"])
@pytest.mark.parametrize("H,K,D,B,T,R,window,sink", [
    (8, 1, 256, 1, 100, 260, 70, 4), (16, 2, 128, 2, 64, 500, 100, 3), (4, 1, 64, 2, 130, 400, 33, 1), (8, 8, 128, 1, 150, 300, 64, 0),
    (8, 1, 256, 2, 51, 867, 500, 17), (2, 2, 64, 1, 300, 300, 128, 70), (8, 1, 64, 33, 4, 90, 30, 2), (16, 1, 256, 1, 40, 700, 1, 1),
    (14, 2, 128, 3, 33, 211, 50, 5), (12, 3, 96, 2, 47, 300, 111, 0)])
def test_window_many_rows(kv, mask, H, K, D, B, T, R, window, sink):
    check_window(kv, "bf16", H, K, D, B, T, R, window, sink, seed=T, mask=mask)


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("store", [head_major, padded])
def test_window_cache_layouts(kv, dtype, store):
    check_window(kv, dtype, 8, 4, 128, 4, 3, 190, 40, 3, seed=3, store=store)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B,T,R,window,sink", [(64, 1, 1500, 1000, 4), (1, 1, 9000, 4096, 4), (5, 2, 4000, 3000, 100)])
def test_window_splits(kv, dtype, B, T, R, window, sink):
    check_window(kv, dtype, 8, 1, 64, B, T, R, window, sink, seed=B)


def test_window_over_everything_is_attend(kv):
    """The same numbers to rounding, on caches that attend reads too."""
    q, k, v = rand(1, 4, 9, 8, 128), rand(2, 4, 300, 2, 128), rand(3, 4, 300, 2, 128)
    seen = i32(np.random.default_rng(0).integers(0, 301, (4, 9)))
    h = kv.KV(8, 2, 128, max_batch=4, max_tokens=9)
    a, la = h.attend(q, own=(k, v), seen=seen)
    b, lb = h.attend_window(q, (k, v), seen, 300)
    assert (la - lb).nan_to_num().abs().max() < 1e-5 and (a.float() - b.float()).abs().max() < 2e-2


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("T", [1, 3, 40])
def test_window_nan_and_infinities_reach_those_that_see_them(kv, T):
    """A NaN key makes the rows that see it NaN, an infinite value the element infinite; others are as without."""
    H, K, D, R, window, sink = 8, 1, 128, 200, 50, 2
    q, k, v = rand(1, 1, T, H, D), rand(2, 1, R, K, D), rand(3, 1, R, K, D)
    seen = np.linspace(60, R, T).astype(int)[None]
    h = kv.KV(H, K, D, max_tokens=T)
    clean, clse = h.attend_window(q, (k, v), i32(seen), window, sink=sink)
    row = int(seen[0, T // 2]) - 20
    sees = np.array([row in okv.visible(n, R, window, sink) for n in seen[0]])
    assert sees[T // 2]
    bad = k.clone()
    bad[0, row, 0, 7] = float("nan")
    out, lse = h.attend_window(q, (bad, v), i32(seen), window, sink=sink)
    assert torch.isnan(out[0, sees]).all() and torch.isnan(lse[0, sees]).all()
    assert np.allclose(np64(out)[0, ~sees], np64(clean)[0, ~sees], atol=2e-2) and not torch.isnan(lse[0, ~sees]).any()
    bad = v.clone()
    bad[0, row, 0, 9] = -float("inf")
    out, lse = h.attend_window(q, (k, bad), i32(seen), window, sink=sink)
    got = np64(out)
    assert np.all(got[0, sees][:, :, 9] == -np.inf) and np.all(np.isfinite(np.delete(got[0, sees], 9, -1)))
    assert np.all(np.isfinite(got[0, ~sees])) and np.allclose(np64(lse), np64(clse), atol=1e-5)
    h.device_status()


# ------------------------------------------------------------------ 8 bits

def check_attend8(kv, dtype, H, K, D, B, T, R, block, window=0, sink=0, seed=0, mask="causal", spread=0.7, store=lambda t: t, std=2.0):
    rng = np.random.default_rng(seed)
    hd = kv.KV(H, K, D, max_batch=B, max_tokens=T, precision=dtype)
    c = fill8(kv, hd, B, R, block, seed, spread=spread, store=store)
    # Scales of each block by themselves.
    for s in (c.v_scale, c.k_scale):
        b = s.view(torch.uint8)
        if s is c.v_scale:
            b += torch.tensor(rng.integers(-3, 4, b.shape), dtype=torch.uint8, device="cuda")
    seen = counts(rng, mask, B, T, R)
    none = hidden(seen, R, window, sink)
    nb = -(-R // block)
    for b in range(B):
        c.k.view(torch.uint8)[b, torch.tensor(none[b], device="cuda")] = 0x7f
        c.v.view(torch.uint8)[b, torch.tensor(none[b], device="cuda")] = 0xff
        for i in range(nb):
            if none[b, i * block:(i + 1) * block].all():
                for s in (c.k_scale, c.v_scale):
                    s.view(torch.uint8)[b, :, i] = (255, 254, 0)[i % 3]
    q = rand(seed, B, T, H, D, dtype=dtype, std=std)
    k, v = (okv.values8(np64(x), s.view(torch.uint8).cpu().numpy().astype(np.int64), block) for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
    k[none], v[none] = 0, 0
    out, lse = hd.attend8(q, c, i32(seen), window=window, sink=sink)
    again = hd.attend8(q, c, i32(seen), window=window, sink=sink)
    hd.device_status()
    sc = 1 / math.sqrt(D)
    ref = okv.attend_window(np64(q), k, v, seen, window, sink, sc)
    finish(out, lse, again, ref, tols(np64(q), k, v, R, dtype, *ref[:1], ref[2], ref[3], ref[1], sc))
    return hd, q, c, seen


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H,K,D", [s for s in SHAPES if s[2] % 16 == 0] + [(1, 1, 16), (4, 2, 48), (2, 1, 240), (24, 1, 128), (20, 1, 256)])
def test_attend8_head_shapes(kv, dtype, H, K, D):
    check_attend8(kv, dtype, H, K, D, 3, 1, 97, 32, seed=H)
    check_attend8(kv, dtype, H, K, D, 2, 5, 133, 16, 31, 3, seed=H + 1, mask="any")


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("block", [16, 32, 64])
@pytest.mark.parametrize("R", [1, 15, 16, 17, 63, 64, 65, 129, 300, 867])
def test_attend8_lengths(kv, dtype, block, R):
    check_attend8(kv, dtype, 8, 1, 128, 2, 1, R, block, seed=R, mask="full")
    check_attend8(kv, dtype, 8, 2, 64, 3, 2, R, block, max(1, R // 3), R // 50, seed=R + 1)


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("mask", ["causal", "any", "full"])
@pytest.mark.parametrize("H,K,D,B,T,R,block,window,sink", [
    (8, 1, 256, 2, 51, 300, 32, 0, 0), (8, 1, 256, 1, 100, 260, 64, 70, 4), (16, 2, 128, 2, 64, 500, 16, 100, 3), (4, 1, 64, 2, 130, 400, 32, 0, 0),
    (8, 8, 128, 1, 150, 300, 64, 0, 0), (2, 2, 64, 1, 300, 300, 16, 128, 70), (8, 1, 64, 33, 4, 90, 32, 0, 0), (14, 2, 128, 3, 33, 211, 32, 50, 5),
    (12, 3, 96, 2, 47, 300, 16, 0, 0), (16, 1, 80, 1, 40, 130, 64, 0, 0)])
def test_attend8_many_rows(kv, mask, H, K, D, B, T, R, block, window, sink):
    check_attend8(kv, "bf16", H, K, D, B, T, R, block, window, sink, seed=T, mask=mask)


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("store", [head_major8, padded8])
def test_attend8_cache_layouts(kv, dtype, store):
    check_attend8(kv, dtype, 8, 4, 128, 4, 3, 90, 32, seed=3, store=store)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B,T,R", [(64, 1, 1500), (1, 1, 9000), (5, 2, 4000)])
def test_attend8_splits(kv, dtype, B, T, R):
    check_attend8(kv, dtype, 8, 1, 64, B, T, R, 32, seed=B)


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("std", [2.0 ** -20, 30.0])
def test_attend8_scales_far_apart(kv, std):
    """Blocks of a cache many powers of two apart, queries far from one."""
    H, K, D, R, block = 8, 1, 64, 160, 16
    for T in (1, 20):
        hd = kv.KV(H, K, D, max_tokens=T)
        c = fill8(kv, hd, 1, R, block, 1)
        c.v_scale.view(torch.uint8)[0, 0] = torch.tensor([120, 100, 119, 140, 90, 121, 118, 1, 60, 122], dtype=torch.uint8, device="cuda")
        c.k_scale.view(torch.uint8)[0, 0] = torch.tensor([120, 110, 119, 115, 90, 121, 118, 1, 60, 119], dtype=torch.uint8, device="cuda")
        q = rand(2, 1, T, H, D, std=std)
        seen = np.linspace(1, R, T).astype(int)[None] if T > 1 else np.array([[R]])
        k, v = (okv.values8(np64(x), s.view(torch.uint8).cpu().numpy().astype(np.int64), block) for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
        out, lse = hd.attend8(q, c, i32(seen))
        ref = okv.attend_window(np64(q), k, v, seen, 0, 0, 1 / 8)
        finish(out, lse, (out, lse), ref, tols(np64(q), k, v, R, "bf16", *ref[:1], ref[2], ref[3], ref[1], 1 / 8))


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [1, 3, 40])
def test_attend8_nan_reaches_those_that_see_it(kv, dtype, T):
    H, K, D, R, block, window, sink = 8, 1, 128, 200, 16, 60, 2
    hd = kv.KV(H, K, D, max_tokens=T, precision=dtype)
    c = fill8(kv, hd, 1, R, block, 1)
    q = rand(1, 1, T, H, D, dtype=dtype)
    seen = np.linspace(70, R, T).astype(int)[None]
    clean, clse = hd.attend8(q, c, i32(seen), window=window, sink=sink)
    row = int(seen[0, T // 2]) - 20
    at = [okv.visible(n, R, window, sink) for n in seen[0]]
    for what in ("key", "value", "key scale", "value scale"):
        sees = np.array([row in a if "scale" not in what else bool(np.any(a // block == row // block)) for a in at])
        t = {"key": c.k, "value": c.v, "key scale": c.k_scale, "value scale": c.v_scale}[what].view(torch.uint8)
        kept = t.clone()
        if "scale" in what:
            t[0, 0, row // block] = 255
        else:
            t[0, row, 0, 9] = 0x7f
        out, lse = hd.attend8(q, c, i32(seen), window=window, sink=sink)
        t.copy_(kept)
        o, l = np64(out)[0], np64(lse)[0]
        if what == "value":
            assert np.all(np.isnan(o[sees][:, :, 9])) and np.all(np.isfinite(np.delete(o[sees], 9, -1)))
        else:
            assert np.all(np.isnan(o[sees]))
        assert np.all(np.isnan(l[sees])) if "key" in what else np.allclose(l, np64(clse)[0], atol=1e-5)
        assert np.allclose(o[~sees], np64(clean)[0, ~sees], atol=2e-2) and np.all(np.isfinite(l[~sees]))
    hd.device_status()


def test_attend8_reads_what_append8_wrote(kv):
    """A generation: a prompt, then tokens, normed and coded into 8-bit caches and attended over with a window, against the
    definition on what the caches hold."""
    H, K, D, B, T, R, block, window, sink = 8, 2, 64, 3, 45, 80, 16, 40, 3
    g = torch.Generator(device="cuda").manual_seed(3)
    nm = kv.Norm(*(1 + 0.2 * torch.randn(D, generator=g, device="cuda") for _ in range(2)))
    h = kv.KV(H, K, D, max_batch=B, max_tokens=T, rope=kv.Rope(dim=D))
    c = h.cache8(B, R, block)
    length = np.array([45, 30, 1])
    pos = np.arange(T)[None].repeat(B, 0)
    for step in range(12):
        n = T if step == 0 else 1
        x = rand(10 + step, B, n, H + 2 * K, D, std=1 + 0.2 * step)
        start = np.zeros(B, int) if step == 0 else length.copy()
        count = length if step == 0 else np.ones(B, int)
        p = pos if step == 0 else length[:, None]
        q = h.append8(x[:, :, :H], x[:, :, H:H + K], x[:, :, H + K:], i32(p), i32(start), c, count=i32(count), norm=nm)
        if step:
            length = length + 1
        seen = np.where(np.arange(n)[None] < count[:, None], start[:, None] + 1 + np.arange(n), 0)
        out, lse = h.attend8(q, c, i32(seen), window=window, sink=sink)
        k, v = (np64(t) for t in c.values())
        ref = okv.attend_window(np64(q), k, v, seen, window, sink, 1 / 8)
        finish(out, lse, (out, lse), ref, tols(np64(q), k, v, R, "bf16", *ref[:1], ref[2], ref[3], ref[1], 1 / 8))
        # The cache holds its tokens to e4m3's precision.
        want = np64(x[:, :, H + K:])
        for b in range(B):
            rows = slice(int(start[b]), int(start[b]) + int(count[b]))
            assert np.abs(v[b, rows] - want[b, :int(count[b])]).max() <= 2.0 ** -4 * np.abs(want).max()
    h.device_status()


def test_spans_on_another_stream_and_in_a_graph(kv):
    H, K, D, B, R = 8, 1, 128, 12, 64
    h = kv.KV(H, K, D, max_batch=B, rope=kv.Rope(dim=D))
    x, nm = rand(1, B, 1, H + 2 * K, D), kv.Norm(torch.full((D,), 1.5, device="cuda"))
    base = fill8(kv, h, B, R, 16, 2)

    def state(n=9):
        c8 = kv.Cache8(*(t.view(torch.uint8).clone().view(t.dtype) for t in (base.k, base.v, base.k_scale, base.v_scale)), 16)
        return rand(4, B, R, K, D), rand(5, B, R, K, D), i32([[n]] * B), i32([n] * B), i32([[n + 1]] * B), c8

    def step(s, stream=None):
        k, v, pos, start, seen, c8 = s
        q = h.append(x[:, :, :H], x[:, :, H:H + K], x[:, :, H + K:], pos, pos, k, v, norm=nm, stream=stream)
        a = h.attend_window(q, (k, v), seen, 5, sink=2, stream=stream)
        q8 = h.append8(x[:, :, :H], x[:, :, H:H + K], x[:, :, H + K:], pos, start, c8, norm=nm, stream=stream)
        b = h.attend8(q8, c8, seen, window=6, sink=1, stream=stream)
        return [q, *a, q8, *b, k, v, *(t.view(torch.uint8) for t in (c8.k, c8.v, c8.k_scale, c8.v_scale))]

    want = step(state())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    s = state()
    torch.cuda.synchronize()
    got = step(s, side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    s = state()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step(s)

    def reset(n):
        for t, src in zip(s[:5], state(n)[:5]):
            t.copy_(src)
        for t, src in zip((s[5].k, s[5].v, s[5].k_scale, s[5].v_scale), (base.k, base.v, base.k_scale, base.v_scale)):
            t.view(torch.uint8).copy_(src.view(torch.uint8))

    for n in (9, 40):      # lengths are read on the device
        want = [t.clone() for t in step(state(n))]
        reset(n)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    h.device_status()


def test_span_refusals(kv):
    h = kv.KV(4, 2, 64, max_batch=2, max_tokens=3)
    q, k, s = rand(1, 2, 3, 4, 64), rand(2, 2, 9, 2, 64), i32([[1, 2, 3]] * 2)
    c = h.cache8(2, 9, 16)
    h.attend_window(q, (k, k), s, 1)
    h.attend8(q, c, s)
    for window, sink in ((0, 0), (-1, 0), (1, -1)):
        with pytest.raises(Exception, match="window"):
            h.attend_window(q, (k, k), s, window, sink=sink)
    for window, sink in ((-1, 0), (1, -1), (0, -1)):
        with pytest.raises(Exception, match="window"):
            h.attend8(q, c, s, window=window, sink=sink)
    for bad in (None, k, (k,), (k, k[:, :8]), (k[:1], k[:1]), (k.float(), k.float()), (k.cpu(), k.cpu())):
        with pytest.raises((ValueError, TypeError)):
            h.attend_window(q, bad, s, 4)
    for args in ((q[:, :, :3], c, s), (q, c, s[:1]), (q, c, s.long()), (q.float(), c, s)):
        with pytest.raises(ValueError):
            h.attend8(*args)
    with pytest.raises((ValueError, TypeError, AttributeError)):
        h.attend8(q, None, s)
    with pytest.raises((ValueError, TypeError)):
        h.attend_window(q, (k, k), s, 2 ** 40)
    with pytest.raises(ValueError):
        h.attend8(q, c, s, out=torch.zeros((2, 3, 4, 64), device="cuda"))
    with pytest.raises(Exception, match="exceed"):
        h.attend8(rand(1, 3, 1, 4, 64), h.cache8(3, 9, 16), i32([[1]] * 3))
    odd = kv.KV(2, 1, 24)
    with pytest.raises(Exception, match="multiple of 16"):
        odd.attend8(rand(1, 1, 1, 2, 24), odd.cache8(1, 16, 16), i32([[1]]))
