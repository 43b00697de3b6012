"""Norms, windows and 8-bit caches at the ends of what their contract allows, on the GPU against the fp64 oracle."""

import numpy as np
import pytest

from oracle import kv as okv
from test_gpu_kv import DT, HALF_EPS, i32, kv, np64, rand, within  # noqa: F401
from test_gpu_kv_heads import bits, norm_tol

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
