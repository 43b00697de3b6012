"""Rows of a long cache whose offsets pass 32 bits, in the appends with norms and to 8 bits and in attention over windows and over 8-bit
caches: the caches are allocated whole, and only their last rows are written and read."""

import math

import numpy as np
import pytest

from oracle import kv as okv
from test_gpu_kv import i32, kv, np64, rand  # noqa: F401
from test_gpu_kv_spans import finish, tols

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

H, K, D = 16, 8, 128
LAST = 640          # rows that hold something


def far(dtype, rows):
    """A cache of `rows` rows and its last ones."""
    if torch.cuda.mem_get_info()[0] < 4 * rows * K * D * dtype.itemsize:
        pytest.skip("not enough memory")
    t = torch.empty((1, rows, K, D), dtype=dtype, device="cuda")
    return t, t[:, rows - LAST:]


@pytest.mark.parametrize("T", [1, 40, 160])
def test_windows_and_appends_with_norms(kv, T):
    R = 2 ** 31 // (K * D) + 1000            # elements pass 2^31, bytes 2^32
    (k, k_end), (v, v_end) = far(torch.bfloat16, R), far(torch.bfloat16, R)
    k_end.copy_(rand(1, 1, LAST, K, D)), v_end.copy_(rand(2, 1, LAST, K, D))
    h = kv.KV(H, K, D, max_tokens=T)
    x = rand(3, 1, T, H + 2 * K, D)
    pos, rows = i32([list(range(T))]), i32([list(range(R - T, R))])
    q = h.append(x[:, :, :H], x[:, :, H:H + K], x[:, :, H + K:], pos, rows, k, v, norm=kv.Norm())
    # The same into a small cache.
    k2, v2 = k_end.clone(), v_end.clone()
    k2[:, LAST - T:], v2[:, LAST - T:] = 0, 0
    q2 = h.append(x[:, :, :H], x[:, :, H:H + K], x[:, :, H + K:], pos, rows - (R - LAST), k2, v2, norm=kv.Norm())
    assert torch.equal(q, q2) and torch.equal(k_end, k2) and torch.equal(v_end, v2)
    seen = np.arange(R - T + 1, R + 1)[None]
    out, lse = h.attend_window(q, (k, v), i32(seen), 300)
    again = h.attend_window(q, (k, v), i32(seen), 300)
    h.device_status()
    ref = okv.attend_window(np64(q), np64(k2), np64(v2), seen - (R - LAST), 300, 0, 1 / math.sqrt(D))
    finish(out, lse, again, ref, tols(np64(q), np64(k2), np64(v2), LAST, "bf16", *ref[:1], ref[2], ref[3], ref[1], 1 / math.sqrt(D)))


@pytest.mark.parametrize("T", [1, 40, 160])
def test_8_bit_caches(kv, T):
    R = (2 ** 32 // (K * D) + 1000) // 32 * 32   # bytes pass 2^32
    e4 = torch.float8_e4m3fn
    (k, k_end), (v, v_end) = far(e4, R), far(e4, R)
    for t in (k_end, v_end):
        t.view(torch.uint8).zero_()
    scales = [torch.full((1, K, R // 32), 127, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu) for _ in range(2)]
    c = kv.Cache8(k, v, *scales, 32)
    h = kv.KV(H, K, D, max_tokens=LAST)
    small = h.cache8(1, LAST, 32)
    x = rand(3, 1, LAST, H + 2 * K, D)
    args = (x[:, :, :H], x[:, :, H:H + K], x[:, :, H + K:], i32([list(range(LAST))]))
    q = h.append8(*args, i32([R - LAST]), c)
    q2 = h.append8(*args, i32([0]), small)
    assert torch.equal(q, q2) and torch.equal(k_end.view(torch.uint8), small.k.view(torch.uint8))
    assert torch.equal(v_end.view(torch.uint8), small.v.view(torch.uint8))
    q = q[:, LAST - T:].contiguous()
    seen = np.arange(R - T + 1, R + 1)[None]
    out, lse = h.attend8(q, c, i32(seen), window=300)
    again = h.attend8(q, c, i32(seen), window=300)
    h.device_status()
    k2, v2 = (np64(t) for t in small.values())
    ref = okv.attend_window(np64(q), k2, v2, seen - (R - LAST), 300, 0, 1 / math.sqrt(D))
    finish(out, lse, again, ref, tols(np64(q), k2, v2, LAST, "bf16", *ref[:1], ref[2], ref[3], ref[1], 1 / math.sqrt(D)))
