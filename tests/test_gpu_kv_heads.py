"""Norms of heads with their rotary coding, and appends to 8-bit caches, on the GPU against their fp64 oracle.

Tolerances are worst-case bounds. The norm: a sum of D squares in fp32 is off by at most (D + 1) 2^-24 of itself, its root by half
of that, with 2^-22 for the reciprocal root and three roundings. The coding: sines and cosines to 2^-22, two products and a sum in
fp32. A code of e4m3 is off by at most 2^-4 of its value, or 2^-10 of its scale.
"""

import numpy as np
import pytest

from oracle import kv as okv
from test_gpu_kv import DT, HALF_EPS, ROPES, head_major, i32, kv, np64, padded, rand, within  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def weights(seed, D):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return tuple(1.0 + 0.3 * torch.randn((D,), generator=g, device="cuda") for _ in range(2))


def norm_tol(y, D):
    """What a normed element's fp32 value may be off by, over its value."""
    return (D / 2 + 10) * 2.0 ** -24


def coded_tol(coded, x, r, D):
    """Of a coded element: both of the pair's elements x (normed already) at most, as their largest of the head."""
    big = np.abs(x).max(-1, keepdims=True) * (1.0 if r is None else 2 * r.mscale)
    return big * (norm_tol(x, D) + 2.0 ** -21)


def check_normed(kv, dtype, H, K, D, B, T, R, rope, seed, eps=1e-6, max_pos=5000, store=lambda t: t, given=(True, True)):
    r = None if rope is None else kv.Rope(**rope)
    h = kv.KV(H, K, D, max_batch=B, max_tokens=T, precision=dtype, rope=r)
    rng = np.random.default_rng(seed)
    qkv = rand(seed, B, T, H + 2 * K, D, dtype=dtype) * torch.tensor(10.0 ** rng.uniform(-3, 2, (B, T, H + 2 * K, 1)), device="cuda").to(DT[dtype])
    ck, cv = store(rand(seed + 1, B, R, K, D, dtype=dtype)), store(rand(seed + 2, B, R, K, D, dtype=dtype))
    pos = rng.integers(-max_pos, max_pos + 1, (B, T))
    rows = np.stack([rng.permutation(R)[:T] for _ in range(B)])
    rows[rng.random((B, T)) < 0.2] = -1
    rows[0, 0] = R if T > 1 else rows[0, 0]     # past the end: padding too
    q, k, v = qkv[:, :, :H], qkv[:, :, H:H + K], qkv[:, :, H + K:]
    qw, kw = (w if g else None for w, g in zip(weights(seed, D), given))
    xq, xk = okv.norm(np64(q), np64(qw), eps), okv.norm(np64(k), np64(kw), eps)
    want_q, want_k, want_v = okv.append(xq, xk, np64(v), pos, rows, np64(ck), np64(cv), r)
    got = torch.full((B, T, H, D), 3.5, dtype=DT[dtype], device="cuda")
    h.append(q, k, v, i32(pos), i32(rows), ck, cv, q_out=got, norm=kv.Norm(qw, kw, eps))
    torch.cuda.synchronize()
    live = (rows >= 0) & (rows < R)
    assert np.all(np64(got)[~live] == 3.5)
    tol = HALF_EPS[dtype] * np.abs(want_q) + coded_tol(want_q, xq, r, D) + 1e-30
    within(got[torch.tensor(live)], want_q[live], tol[live], "q")
    ktol = np.zeros(want_k.shape)
    for b, t in np.argwhere(live):
        ktol[b, rows[b, t]] = HALF_EPS[dtype] * np.abs(want_k[b, rows[b, t]]) + coded_tol(None, xk[b, t], r, D) + 1e-30
    within(ck, want_k, ktol, "k")
    assert np.array_equal(np64(cv), want_v)
    return h


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", range(len(ROPES)))
def test_normed_codings(kv, dtype, n):
    check_normed(kv, dtype, 6, 2, 256, 3, 5, 11, ROPES[n], 10 * n)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H,K,D,dim", [(8, 1, 256, 256), (4, 1, 64, 32), (32, 8, 128, 128), (6, 2, 80, 80), (14, 2, 128, 16), (12, 3, 96, 48),
                                       (1, 1, 8, 8), (5, 5, 40, 10), (16, 1, 24, 24), (3, 1, 160, 36), (2, 2, 248, 240)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_normed_head_shapes(kv, dtype, H, K, D, dim, layout):
    check_normed(kv, dtype, H, K, D, 2, 7, 9, dict(dim=dim, layout=layout), H + D)
    check_normed(kv, dtype, H, K, D, 1, 1, 1, dict(dim=dim, layout=layout), H + D + 1, given=(False, True))


@pytest.mark.parametrize("B,T", [(1, 1), (64, 1), (3, 700), (16, 51), (1, 2049)])
def test_normed_sizes(kv, B, T):
    check_normed(kv, "bf16", 8, 1, 64, B, T, T + 3, dict(dim=64), B)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("store", [head_major, padded])
def test_normed_cache_layouts(kv, dtype, store):
    check_normed(kv, dtype, 4, 4, 128, 2, 9, 12, dict(dim=64), 5, store=store)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_normed_extremes(kv, dtype):
    """Heads of zeros, of values whose squares pass fp32's range either way, and of infinities and NaN."""
    D = 64
    h = kv.KV(2, 1, D, max_tokens=6, precision=dtype)
    x = torch.ones((1, 6, 2, D), dtype=DT[dtype], device="cuda")
    x *= torch.tensor([0.0, 2.0 ** 100, 2.0 ** 126, 2.0 ** -100, 1.0, 1.0], device="cuda").to(DT[dtype])[None, :, None, None]
    x[0, 4, 0, 3], x[0, 5, 1, 7] = float("inf"), float("nan")
    out = np64(h.append(x, None, None, i32([[0] * 6]), i32([[0] * 6]), norm=kv.Norm(eps=1e-6)))
    with np.errstate(invalid="ignore", over="ignore"):
        want = okv.norm(np64(x), None, 1e-6)
    assert np.all(out[0, 0] == 0) and np.all(np.abs(out[0, 1:3] - 1) < 1e-2) and np.all(np.abs(out[0, 3] - want[0, 3]) <= 1e-2 * np.abs(want[0, 3]))
    assert np.isnan(out[0, 4, 0, 3]) and np.all(np.delete(out[0, 4, 0], 3) == 0) and np.all(np.abs(out[0, 4, 1] - 1) < 1e-2)
    assert np.all(np.isnan(out[0, 5, 1])) and np.all(np.abs(out[0, 5, 0] - 1) < 1e-2)


def test_normed_in_place_and_halves(kv):
    """Queries alone over themselves, and keys in a cache normed and coded in place, give what a call of both gives; the
    tokens' rows in place are read before they are written, for pairs of chunks and of single elements."""
    for dim in (128, 20):
        H, K, D, B, T = 4, 2, 128, 2, 33
        h = kv.KV(H, K, D, max_batch=B, max_tokens=T, rope=kv.Rope(dim=dim))
        q, k, v = rand(1, B, T, H, D), rand(2, B, T, K, D), rand(3, B, T, K, D)
        pos, rows = i32([list(range(T))] * B), i32([list(range(T))] * B)
        nm = kv.Norm(*weights(4, D))
        ck, cv = torch.zeros((B, T, K, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((B, T, K, D), dtype=torch.bfloat16, device="cuda")
        want = h.append(q, k, v, pos, rows, ck, cv, norm=nm)
        assert torch.equal(cv, v)
        q2, k2 = q.clone(), k.clone()
        assert torch.equal(h.append(q2, None, None, pos, rows, q_out=q2, norm=nm), want)
        h.append(None, k2, None, pos, rows, k2, norm=nm)
        assert torch.equal(k2, ck)


def test_normed_refusals(kv):
    h = kv.KV(4, 2, 64, max_batch=2, max_tokens=3, rope=kv.Rope(dim=64))
    q, k = rand(1, 2, 3, 4, 64), rand(2, 2, 3, 2, 64)
    c, i = rand(3, 2, 5, 2, 64), i32([[0, 1, 2]] * 2)
    call = lambda **n: h.append(q, k, k, i, i, c, c.clone(), norm=kv.Norm(**n))
    call()
    for eps in (0.0, -1.0, float("nan"), float("inf"), 1e-40):
        with pytest.raises(Exception, match="eps"):
            call(eps=eps)
    w = torch.ones(64, device="cuda")
    for bad in (w[:63], w.double(), w.bfloat16(), torch.ones(128, device="cuda")[::2], w.cpu()):
        with pytest.raises(ValueError):
            call(q_weight=bad)
        with pytest.raises(ValueError):
            call(k_weight=bad)
    call(q_weight=torch.ones(65, device="cuda")[1:], k_weight=w)      # (no alignment beyond the type's)


# ------------------------------------------------------------------ 8 bits

def bits(t):
    return t.view(torch.uint8).cpu().numpy().astype(np.int64)


def fill8(kv, h, B, R, block, seed, spread=1.0, store=lambda t: t):
    """A cache whose rows all hold something, under scales that fit them."""
    rng = np.random.default_rng(seed)
    c = h.cache8(B, R, block)
    nb = -(-R // block)
    codes, scales = [], []
    for i in range(2):
        x = rng.normal(size=(B, R, h.kv_heads, h.head_dim)) * np.exp(spread * rng.normal(size=(B, 1, h.kv_heads, 1)))
        e = np.zeros((B, h.kv_heads, nb), np.int64)
        z = np.zeros(x.shape)
        z, e = okv.append8(x, [0] * B, [R] * B, z, e, block)
        codes.append(store(torch.tensor(z, device="cuda").to(torch.float8_e4m3fn).view(torch.uint8)).view(torch.float8_e4m3fn))
        scales.append(torch.tensor(e, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu))
    return kv.Cache8(*codes, *scales, block)


def head_major8(t):
    return t.transpose(1, 2).contiguous().transpose(1, 2)


def padded8(t):
    big = torch.full((t.shape[0], t.shape[1] + 2, t.shape[2] + 3, t.shape[3]), 0x7f, dtype=torch.uint8, device="cuda")
    big[:, :t.shape[1], :t.shape[2]] = t
    return big[:, :t.shape[1], :t.shape[2]]


def check_append8(kv, dtype, H, K, D, B, T, R, block, rope, seed, norm=False, store=lambda t: t, start=None, count=None, gain=1.0,
                  max_pos=5000):
    r = None if rope is None else kv.Rope(**rope)
    h = kv.KV(H, K, D, max_batch=B, max_tokens=T, precision=dtype, rope=r)
    rng = np.random.default_rng(seed)
    c = fill8(kv, h, B, R, block, seed, store=store)
    grow = torch.tensor(np.exp(gain * rng.normal(size=(B, T, H + 2 * K, 1))), device="cuda").to(DT[dtype])
    qkv = rand(seed, B, T, H + 2 * K, D, dtype=dtype) * grow
    q, k, v = qkv[:, :, :H], qkv[:, :, H:H + K], qkv[:, :, H + K:]
    pos = rng.integers(-max_pos, max_pos + 1, (B, T))
    start = rng.integers(0, max(1, R - T + 1), B) if start is None else np.asarray(start)
    counts = rng.integers(0, T + 1, B) if count is None else np.asarray(count)
    qw, kw = weights(seed, D)
    eps = 1e-5
    xq, xk = (okv.norm(np64(q), np64(qw), eps), okv.norm(np64(k), np64(kw), eps)) if norm else (np64(q), np64(k))
    coded_q, coded_k = (np.stack([[[okv.rope(x[b, t, i], int(pos[b, t]), r) for i in range(x.shape[2])] for t in range(T)] for b in range(B)])
                        for x in (xq, xk))
    before = [np64(c.k), np64(c.v)], [bits(c.k_scale), bits(c.v_scale)]
    raw = [bits(c.k), bits(c.v)]
    want = [okv.append8(x, start, counts, before[0][i], before[1][i], block) for i, x in enumerate((coded_k, np64(v)))]
    got = torch.full((B, T, H, D), 3.5, dtype=DT[dtype], device="cuda")
    h.append8(q, k, v, i32(pos), i32(start), c, count=i32(counts), norm=kv.Norm(qw, kw, eps) if norm else None, q_out=got)
    torch.cuda.synchronize()
    # Values are not computed with: codes and scales are the oracle's.
    assert np.array_equal(bits(c.v_scale), want[1][1])
    within(c.v, want[1][0], 0, "v codes")
    live = np.zeros((B, T), bool)
    written = np.zeros((B, R), bool)
    for b in range(B):
        n = min(max(int(counts[b]), 0), T, R - int(start[b])) if 0 <= start[b] < R else 0
        live[b, :n] = True
        written[b, int(start[b]):int(start[b]) + n] = True
    # Queries, as the other appends'.
    slack = coded_tol(None, xq, r, D)
    assert np.all(np64(got)[~live] == 3.5)
    within(got[torch.tensor(live)], coded_q[live], (HALF_EPS[dtype] * np.abs(coded_q) + slack + 1e-30)[live], "q")
    # Keys: a scale may be the other one where the largest element is at the border within fp32's error; here none is.
    assert np.array_equal(bits(c.k_scale), want[0][1])
    s = np.repeat(2.0 ** (want[0][1] - 127.0), block, 2)[:, :, :R].transpose(0, 2, 1)[..., None]
    hold = np64(c.k) * s
    ref = want[0][0] * s
    exact = ref.copy()
    tol = np.zeros(ref.shape)
    for b in range(B):
        n = int(live[b].sum())
        at = slice(int(start[b]), int(start[b]) + n)
        if n:
            exact[b, at] = coded_k[b, :n]
            err = np.broadcast_to(coded_tol(None, xk[b, :n], r, D), coded_k[b, :n].shape)
            tol[b, at] = 2.0 ** -4 * (np.abs(coded_k[b, :n]) + err) + 2.0 ** -10 * s[b, at] + err
    bad = ~(np.abs(hold - exact) <= np.maximum(tol, 0)) & written[..., None, None]
    assert not bad.any(), f"k: {bad.sum()} new elements off"
    # What was there: the codes of the oracle, bit for bit where nothing was written.
    rest = ~written
    assert np.array_equal(np64(c.k)[rest], want[0][0][rest])
    assert np.array_equal(bits(c.k)[rest][want[0][0][rest] == before[0][0][rest]], raw[0][rest][want[0][0][rest] == before[0][0][rest]])
    return h, c


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("block", [16, 32, 64])
@pytest.mark.parametrize("norm", [False, True])
def test_append8_blocks(kv, dtype, block, norm):
    check_append8(kv, dtype, 4, 2, 128, 5, 70, 200, block, dict(dim=128), block + norm, norm=norm)
    check_append8(kv, dtype, 4, 2, 128, 9, 1, 77, block, dict(dim=64, layout="interleaved"), block + norm + 1, norm=norm, count=[1] * 9)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H,K,D,dim", [(8, 1, 256, 256), (4, 1, 64, 32), (8, 8, 128, 128), (6, 2, 80, 80), (12, 3, 96, 36), (1, 1, 16, 16),
                                       (2, 1, 48, 10), (3, 1, 160, 36), (2, 2, 240, 240)])
def test_append8_head_shapes(kv, dtype, H, K, D, dim):
    check_append8(kv, dtype, H, K, D, 3, 21, 50, 32, dict(dim=dim), H + D)
    check_append8(kv, dtype, H, K, D, 3, 21, 50, 64, dict(dim=dim, layout="interleaved"), H + D + 1, norm=True)
    check_append8(kv, dtype, H, K, D, 2, 3, 9, 16, None, H + D + 2)


@pytest.mark.parametrize("start,count", [([0, 31, 32, 63], [5, 1, 40, 40]), ([-1, 100, 99, 0], [40, 40, 40, 40]),
                                         ([5, 5, 5, 90], [0, -3, 400, 40]), ([99, 96, 64, 2147483647], [1, 4, 40, 2])])
def test_append8_starts_and_counts(kv, start, count):
    check_append8(kv, "bf16", 2, 2, 64, 4, 40, 100, 32, dict(dim=64), 3, start=start, count=count)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("store", [head_major8, padded8])
def test_append8_cache_layouts(kv, dtype, store):
    check_append8(kv, dtype, 4, 4, 64, 3, 30, 70, 16, dict(dim=64), 8, store=store)


@pytest.mark.parametrize("gain", [0.0, 4.0, 20.0])
def test_append8_scales_far_apart(kv, gain):
    """Scales that grow by many powers of two, to where the old rows round to zero."""
    check_append8(kv, "fp32", 2, 2, 64, 8, 3, 64, 64, None, 5, gain=gain)
    check_append8(kv, "bf16", 2, 2, 64, 8, 40, 64, 16, None, 6, gain=gain)


def test_append8_token_by_token_holds_what_one_call_holds(kv):
    """Blocks filled a token at a time end with the scales of one call, and its codes but for elements that were below
    2^-6 of their scale when it grew."""
    H, K, D, R, block = 2, 2, 64, 50, 16
    h = kv.KV(H, K, D, max_tokens=R, rope=kv.Rope(dim=D))
    k, v = rand(1, 1, R, K, D) * torch.linspace(0.1, 3, R, device="cuda").bfloat16()[None, :, None, None], rand(2, 1, R, K, D)
    pos = i32([list(range(R))])
    one, many = h.cache8(1, R, block), h.cache8(1, R, block)
    h.append8(None, k, v, pos, i32([0]), one)
    for t in range(R):
        h.append8(None, k[:, t:t + 1], v[:, t:t + 1], pos[:, t:t + 1].contiguous(), i32([t]), many)
    assert np.array_equal(bits(one.k_scale), bits(many.k_scale)) and np.array_equal(bits(one.v_scale), bits(many.v_scale))
    for a, b, s in ((one.k, many.k, one.k_scale), (one.v, many.v, one.v_scale)):
        a, b = np64(a), np64(b)
        big = np.abs(a) >= 2.0 ** -6
        assert np.array_equal(a[big], b[big]) and np.abs(a - b).max() <= 2.0 ** -9


def test_append8_infinities_and_nan(kv):
    """They are held as NaN, and set no scale; a scale of NaN under rows that stay is kept."""
    h = kv.KV(2, 1, 32, max_tokens=4, precision="bf16")
    c = h.cache8(1, 32, 16)
    x = rand(1, 1, 4, 1, 32)
    x[0, 1, 0, 5], x[0, 2, 0, 6], x[0, 3, 0, 0] = float("inf"), float("nan"), -float("inf")
    h.append8(None, x, x, i32([[0] * 4]), i32([0]), c)
    want, scale = okv.append8(np64(x), [0], [4], np.zeros((1, 32, 1, 32)), np.full((1, 1, 2), 127), 16)
    assert np.array_equal(np64(c.k), want, equal_nan=True) and np.array_equal(bits(c.k_scale), scale) and np.isnan(want).sum() == 3
    c.v_scale.view(torch.uint8)[0, 0, 0] = 255
    h.append8(None, x, x, i32([[0] * 4]), i32([4]), c)
    assert bits(c.v_scale)[0, 0].tolist() == [255, 127] and bits(c.k_scale)[0, 0, 0] == scale[0, 0, 0]
    h.append8(None, x, x, i32([[0] * 4]), i32([0]), c)     # nothing stays: a new scale
    assert bits(c.v_scale)[0, 0, 0] == scale[0, 0, 0]


def test_append8_refusals(kv):
    h = kv.KV(4, 2, 64, max_batch=2, max_tokens=3, rope=kv.Rope(dim=64))
    q, k, i, s = rand(1, 2, 3, 4, 64), rand(2, 2, 3, 2, 64), i32([[0, 1, 2]] * 2), i32([0, 1])
    c = h.cache8(2, 40, 32)
    h.append8(q, k, k, i, s, c)
    h.append8(q, None, None, i, s, c)
    before = bits(c.k)
    B = lambda **kw: kv.Cache8(**{**dict(k=c.k, v=c.v, k_scale=c.k_scale, v_scale=c.v_scale, block=32), **kw})
    for bad in (B(block=8), B(block=0), B(block=64), B(k=c.k.view(torch.uint8)), B(k=c.k[:1], v=c.v[:1]), B(v=c.v[:, :39]), B(k_scale=c.k_scale.view(torch.uint8)),
                B(v_scale=c.v_scale[:, :, :1]), B(k=c.k[..., :32], v=c.v[..., :32]), B(k=c.k.cpu(), v=c.v.cpu())):
        with pytest.raises(Exception):
            h.append8(q, k, k, i, s, bad)
    for args in ((q, k, None, i, s, c), (None, None, None, i, s, c), (q, k, k, i[:1], s, c), (q, k, k, i, s[:1], c), (q, k[:, :2], k, i, s, c),
                 (q, k, k, i.long(), s, c), (q, k, k, i, s.long(), c)):
        with pytest.raises(ValueError):
            h.append8(*args)
    with pytest.raises(ValueError):
        h.append8(q, k, k, i, s, c, count=s[:1])
    with pytest.raises(Exception, match="eps"):
        h.append8(q, k, k, i, s, c, norm=kv.Norm(eps=0.0))
    with pytest.raises(Exception, match="exceed"):
        h.append8(rand(1, 2, 4, 4, 64), None, None, i32([[0] * 4] * 2), s, c)
    assert np.array_equal(bits(c.k), before)
    odd = kv.KV(2, 1, 24, max_tokens=3)
    with pytest.raises(Exception, match="multiple of 16"):
        odd.append8(None, rand(1, 1, 3, 1, 24), rand(1, 1, 3, 1, 24), i32([[0] * 3]), i32([0]), odd.cache8(1, 16, 16))
