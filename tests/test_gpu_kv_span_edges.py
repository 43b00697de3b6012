"""Norms, windows and 8-bit caches at the ends of what their contract allows, on the GPU against the fp64 oracle."""

import numpy as np
import pytest

from oracle import kv as okv
from test_gpu_kv import DT, HALF_EPS, i32, kv, np64, rand, within  # noqa: F401
from test_gpu_kv_heads import bits, fill8, norm_tol
from test_gpu_kv_spans import finish, hidden, tols
from test_kv_span_rounding_host import bound, crafted

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("byte", [246, 252, 253, 254])
def test_append8_under_the_largest_scales(kv, dtype, byte):
    """A block begun under a scale near 2^127: new elements are rounded to it, codes before them stay. Values are not computed
    with, so that codes and scales are the oracle's."""
    R, block, D = 32, 16, 64
    h = kv.KV(2, 1, D, max_tokens=3, precision=dtype)
    c = h.cache8(1, R, block)
    for s in (c.k_scale, c.v_scale):
        s.view(torch.uint8)[0, 0, 0] = byte
    c.k.view(torch.uint8)[0, :4], c.v.view(torch.uint8)[0, :4] = 0x31, 0xb5
    x = rand(byte, 1, 3, 1, D, dtype=dtype) * torch.tensor([2.0 ** 126, 2.0 ** 121, 2.0 ** 112], device="cuda").to(DT[dtype])[None, :, None, None]
    x = x.clamp(-3e38, 3e38)
    want = [okv.append8(np64(x), [4], [3], np64(t), bits(s), block) for t, s in ((c.k, c.k_scale), (c.v, c.v_scale))]
    h.append8(None, x, x, i32([[0] * 3]), i32([4]), c)
    for (codes, scales), t, s in zip(want, (c.k, c.v), (c.k_scale, c.v_scale)):
        assert np.array_equal(bits(s), scales) and scales[0, 0, 0] == max(byte, okv.scale8(np64(x)))
        assert np.array_equal(np64(t), codes) and np.any(codes[0, 4])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [8, 64, 248])
@pytest.mark.parametrize("eps", [1e-6, 1e30, 3e37, 1e38, 3.4e38])
def test_norms_of_large_heads_under_any_eps(kv, dtype, D, eps):
    """Mean squares and eps on both sides of where their sum passes fp32's range."""
    size = np.array([1e-3, 1.0, 3e17, 1e18, 2e18, 5e18, 1.3e19, 2.0 ** 64, 2.0 ** 100, 2.0 ** 126])
    T = len(size)
    x = rand(D, 1, T, 2, D, dtype=dtype).clamp(-1.9, 1.9) * torch.tensor(size, device="cuda").to(DT[dtype])[None, :, None, None]
    i = i32([[0] * T])
    got = kv.KV(2, 1, D, max_tokens=T, precision=dtype).append(x, None, None, i, i, norm=kv.Norm(eps=eps))
    want = okv.norm(np64(x), None, eps)
    within(got, want, HALF_EPS[dtype] * np.abs(want) + norm_tol(want, D) * np.abs(want) + 2.0 ** -125, "norm")


def wide_cache(kv, h, B, R, block, seed, k_byte):
    """An 8-bit cache with its keys under one scale, and the numbers that it holds."""
    c = fill8(kv, h, B, R, block, seed)
    c.k_scale.view(torch.uint8).fill_(k_byte)
    return c, [okv.values8(np64(x), bits(s), block) for x, s in ((c.k, c.k_scale), (c.v, c.v_scale))]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tiles", ["0", "1"])
@pytest.mark.parametrize("k_byte,q_log2", [(245, -121), (228, -104), (10, 120), (30, 100)])
@pytest.mark.parametrize("B,T", [(1, 1), (3, 20), (200, 1)])
def test_attend8_where_scores_are_in_range_and_their_factors_far_from_it(kv, monkeypatch, dtype, tiles, k_byte, q_log2, B, T):
    """Keys of 2^118 under queries of 2^-121 and the other way round."""
    monkeypatch.setenv("JPI_KV_TILES", tiles)
    H, K, D, R, block = 8, 1, 64, 150, 16
    h = kv.KV(H, K, D, max_batch=B, max_tokens=T, precision=dtype)
    c, (k, v) = wide_cache(kv, h, B, R, block, 3, k_byte)
    q = rand(5, B, T, H, D, dtype=dtype) * 2.0 ** q_log2
    assert torch.isfinite(q).all() and np.abs(k).max() < 3e38
    seen = np.clip(R - 10 * np.arange(T), 0, None)[None].repeat(B, 0)
    out, lse = h.attend8(q, c, i32(seen))
    again = h.attend8(q, c, i32(seen))
    h.device_status()
    ref = okv.attend_window(np64(q), k, v, seen, 0, 0, 1 / 8)
    finish(out, lse, again, ref, tols(np64(q), k, v, R, dtype, *ref[:1], ref[2], ref[3], ref[1], 1 / 8))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tiles", ["0", "1"])
def test_attend8_of_queries_far_from_each_other(kv, monkeypatch, dtype, tiles):
    """Tokens of one tile whose queries are 0, below fp32's normal numbers, or up to 2^100: each as by itself."""
    monkeypatch.setenv("JPI_KV_TILES", tiles)
    H, K, D, R, block = 8, 1, 64, 150, 16
    size = [0.0, 2.0 ** -130, 2.0 ** -60, 2.0 ** -8, 1.0, 2.0 ** 20, 2.0 ** 60, 2.0 ** 100]
    T = len(size)
    h = kv.KV(H, K, D, max_tokens=T, precision=dtype)
    c = fill8(kv, h, 1, R, block, 3)
    k, v = (okv.values8(np64(x), bits(s), block) for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
    q = rand(5, 1, T, H, D, dtype="fp32") * torch.tensor(size, device="cuda")[None, :, None, None]
    q = q.to(DT[dtype])
    seen = np.full((1, T), R)
    out, lse = h.attend8(q, c, i32(seen))
    h.device_status()
    ref, rlse, dot, mass = okv.attend_window(np64(q), k, v, seen, 0, 0, 1 / 8)
    small = slice(0, 5)
    bound = tols(np64(q[:, small]), k, v, R, dtype, ref[:, small], dot[:, small], mass[:, small], rlse[:, small], 1 / 8)
    within(out[:, small], ref[:, small], bound[0], "out")
    within(lse[:, small], rlse[:, small], bound[1], "lse")
    # The large ones see one key, where the next is far enough below the first.
    score = np.einsum("thd,jd->thj", np64(q)[0], k[0, :, 0]) / 8
    top = np.sort(score, -1)
    clear = (top[..., -1] - top[..., -2] > 2.0 ** -12 * dot[0] + 50) & (np.arange(T)[:, None] >= 5)
    assert clear.sum() > 2 * H
    got = np64(out)[0]
    best = v[0, score.argmax(-1), 0]
    assert np.all(np.abs(got - best)[clear] <= HALF_EPS[dtype] * np.abs(best[clear]) + 2.0 ** -10 * np.abs(v).max())
    assert np.all(np.abs(np64(lse)[0] - top[..., -1])[clear] <= 2.0 ** -14 * dot[0][clear])


# ------------------------------------------------------------------ what the probabilities are rounded to

def crafted_call(seed, B, K, R, D, dtype, held8):
    """Queries whose first element is 1 and nothing else, keys and values of `crafted`."""
    rng = np.random.default_rng(seed)
    scale = D ** -0.5
    k, v = np.zeros((B, R, K, D)), np.zeros((B, R, K, D))
    for b in range(B):
        for h in range(K):
            x, s = crafted(rng, R, scale, held8)
            k[b, :, h, 0], v[b, :, h] = x, s[:, None] * np.where(np.arange(D) % 3 == 0, -1, 1)
    k[..., 1:] = rng.integers(-3, 4, k[..., 1:].shape)      # (under queries of 0)
    return [torch.tensor(t, device="cuda").to(DT[dtype]) for t in (k, v)]


ROUNDED = [(8, 8, 64, 1, 1, 512), (8, 1, 64, 1, 3, 512), (32, 8, 128, 64, 1, 256), (8, 1, 256, 1, 1, 512), (8, 8, 64, 64, 1, 256),
           (8, 1, 64, 2, 40, 512), (16, 2, 128, 2, 30, 512), (8, 1, 256, 3, 51, 256), (8, 1, 256, 40, 51, 256)]


@pytest.mark.parametrize("tiles", ["0", "by size", "1"])
@pytest.mark.parametrize("H,K,D,B,T,R", ROUNDED)
@pytest.mark.parametrize("held8", [False, True])
def test_rounding_of_the_probabilities(kv, monkeypatch, tiles, held8, H, K, D, B, T, R):
    """Over bf16 caches two bf16 terms (2^-16) outside the tiles, one (2^-8) on them; over 8-bit caches one of fp16 (2^-11)."""
    if tiles != "by size":
        monkeypatch.setenv("JPI_KV_TILES", tiles)
    h = kv.KV(H, K, D, max_batch=B, max_tokens=T)
    k, v = crafted_call(D + T, B, K, R, D, "bf16", held8)
    q = torch.zeros((B, T, H, D), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1
    seen = i32(np.full((B, T), R))
    if held8:
        c = h.cache8(B, R, 32)
        c.k.copy_(k.to(torch.float8_e4m3fn)), c.v.copy_(v.to(torch.float8_e4m3fn))
        assert torch.equal(c.k.float(), k.float()) and torch.equal(c.v.float(), v.float())
        out, lse = h.attend8(q, c, seen)
    else:
        out, lse = h.attend_window(q, (k, v), seen, R)
    h.device_status()
    ref, rlse, _, mass = okv.attend_window(np64(q), np64(k), np64(v), np.full((B, T), R), R, 0, D ** -0.5)
    prob = 2.0 ** -11 if held8 else 2.0 ** -16 if tiles == "0" or T == 1 and tiles != "1" else 2.0 ** -8
    within(out, ref, bound(ref, mass, R, prob, 2.0 ** -8), "out")
    within(lse, rlse, 2.0 ** -18 + (R / 8 + 16) * 2.0 ** -23, "lse")


# ------------------------------------------------------------------ values of 8 bits far apart

@pytest.mark.parametrize("tiles", ["0", "1"])
@pytest.mark.parametrize("std", [2.0 ** -20, 30.0])
@pytest.mark.parametrize("T", [1, 20])
def test_values_far_apart_by_what_each_row_sees(kv, monkeypatch, tiles, std, T):
    """A probability is an fp16 number in units of 2^-7 of a probability (the tiles: 2^-4) times the largest scale that its row
    sees: off by half of fp16's least step, 2^-25, for a value of at most 448 of its scale."""
    monkeypatch.setenv("JPI_KV_TILES", tiles)
    H, K, D, R, block = 8, 1, 64, 160, 16
    hd = kv.KV(H, K, D, max_tokens=T)
    c = fill8(kv, hd, 1, R, block, 1)
    vs, ks = [120, 100, 119, 140, 90, 121, 118, 1, 60, 122], [120, 110, 119, 115, 90, 121, 118, 1, 60, 119]
    c.v_scale.view(torch.uint8)[0, 0] = torch.tensor(vs, dtype=torch.uint8, device="cuda")
    c.k_scale.view(torch.uint8)[0, 0] = torch.tensor(ks, dtype=torch.uint8, device="cuda")
    q = rand(2, 1, T, H, D, std=std)
    seen = np.linspace(1, R, T).astype(int)[None] if T > 1 else np.array([[48]])
    k, v = (okv.values8(np64(x), bits(s), block) for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
    out, lse = hd.attend8(q, c, i32(seen))
    again = hd.attend8(q, c, i32(seen))
    ref, rlse, dot, mass = okv.attend_window(np64(q), k, v, seen, 0, 0, 1 / 8)
    rel = (D + 2) * 2.0 ** -22 * dot + 2.0 ** -20 + R * 2.0 ** -23 + 2.0 ** -22 * np.abs(rlse)
    far = np.zeros((1, T, H, 1))
    for t, n in enumerate(seen[0]):
        rel[0, t] += 2.0 ** -24 / 8 * np.abs(np64(q)[0, t]).max(-1) * np.abs(k[0, :n]).sum(-1).max()
        far[0, t] = n * 448 * 2.0 ** (max(vs[:-(-n // block)]) - 127) * 2.0 ** (-29 if tiles == "1" else -32)
    # Rows that do not see the largest block would show it if they took its scale for theirs.
    assert np.all(far[0, seen[0] <= 48] < 2.0 ** -4 * np.abs(ref[0, seen[0] <= 48]).max(-1, keepdims=True))
    finish(out, lse, again, (ref, rlse, None, None), (2.0 ** -8 * np.abs(ref) + (2 * rel[..., None] + 2.0 ** -11) * mass + far, rel + 1e-6))


# ------------------------------------------------------------------ counts far apart

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tiles", ["0", "1"])
@pytest.mark.parametrize("held8", [False, True])
def test_counts_far_apart_in_one_request(kv, monkeypatch, dtype, tiles, held8):
    """Tokens whose windows are thousands of rows from each other: each has its own, whatever lies between."""
    monkeypatch.setenv("JPI_KV_TILES", tiles)
    H, K, D, B, T, R, window, sink = 8, 1, 64, 2, 6, 5000, 33, 2
    seen = np.array([[100, 4990, 0, 2500, 101, 5000], [5000, 40, 41, 3000, 3100, 1]])
    h = kv.KV(H, K, D, max_batch=B, max_tokens=T, precision=dtype)
    none = torch.tensor(hidden(seen, R, window, sink), device="cuda")
    q = rand(1, B, T, H, D, dtype=dtype)
    if held8:
        c = fill8(kv, h, B, R, 32, 3)
        k, v = (okv.values8(np64(x), bits(s), 32) for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
        c.k.view(torch.uint8)[none], c.v.view(torch.uint8)[none] = 0x7f, 0xff
        call = lambda: h.attend8(q, c, i32(seen), window=window, sink=sink)
    else:
        kc, vc = rand(2, B, R, K, D, dtype=dtype), rand(3, B, R, K, D, dtype=dtype)
        k, v = np64(kc), np64(vc)
        kc[none], vc[none] = float("nan"), float("inf")
        call = lambda: h.attend_window(q, (kc, vc), i32(seen), window, sink=sink)
    (out, lse), again = call(), call()
    h.device_status()
    ref = okv.attend_window(np64(q), k, v, seen, window, sink, 1 / 8)
    finish(out, lse, again, ref, tols(np64(q), k, v, window + sink, dtype, *ref[:1], ref[2], ref[3], ref[1], 1 / 8))


def test_a_window_over_everything_has_the_sums_of_attend(kv):
    """The sums' logarithms agree, and both are -infinity where nothing is seen, and nowhere else."""
    q, k, v = rand(1, 4, 9, 8, 128), rand(2, 4, 300, 2, 128), rand(3, 4, 300, 2, 128)
    seen = np.random.default_rng(0).integers(0, 301, (4, 9))
    seen[1, 3] = seen[2, 0] = 0
    h = kv.KV(8, 2, 128, max_batch=4, max_tokens=9)
    la, lb = h.attend(q, own=(k, v), seen=i32(seen))[1], h.attend_window(q, (k, v), i32(seen), 300)[1]
    la, lb = np64(la), np64(lb)
    assert np.array_equal(la == -np.inf, np.broadcast_to((seen == 0)[..., None], la.shape)) and np.array_equal(la == -np.inf, lb == -np.inf)
    some = seen > 0
    assert np.all(np.isfinite(lb[some])) and np.abs(la[some] - lb[some]).max() < 1e-5


# ------------------------------------------------------------------ the first call of a handle

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("held8", [False, True])
@pytest.mark.parametrize("T", [1, 40])
def test_the_first_attention_of_a_handle_may_be_captured(kv, dtype, held8, T):
    H, K, D, R = 8, 1, 128, 200
    q, k, v, s = rand(1, 1, T, H, D, dtype=dtype), rand(2, 1, R, K, D, dtype=dtype), rand(3, 1, R, K, D, dtype=dtype), i32([list(range(R - T + 1, R + 1))])
    h, h2 = (kv.KV(H, K, D, max_tokens=T, precision=dtype) for _ in range(2))
    c = fill8(kv, h, 1, R, 32, 5)
    call = lambda x: x.attend8(q, c, s, window=77) if held8 else x.attend_window(q, (k, v), s, 77)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = call(h)
    g.replay()
    want = call(h2)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(call(h)[0], want[0])
    h.device_status()
