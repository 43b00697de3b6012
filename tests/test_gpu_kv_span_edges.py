"""Norms, windows and 8-bit caches at the ends of what their contract allows, on the GPU against the fp64 oracle."""

import numpy as np
import pytest

from oracle import kv as okv
from test_gpu_kv import DT, HALF_EPS, i32, kv, np64, rand, within  # noqa: F401
from test_gpu_kv_heads import bits, fill8, norm_tol
from test_gpu_kv_spans import finish, tols
from test_kv_span_rounding_host import bound

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
