"""Attention over windows and over 8-bit caches in one launch: tiles of query rows dealt to clusters of one to eight blocks, whose
parts are joined through shared memory (few tiles, few keys), against the fp64 oracle with the tolerances of test_gpu_kv_spans.py."""

import math

import numpy as np
import pytest

from oracle import kv as okv
from test_gpu_kv import i32, kv, np64, rand  # noqa: F401
from test_gpu_kv_heads import fill8
from test_gpu_kv_spans import check_attend8, check_window, finish, tols

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# Tiles of 8 query rows: from one (clusters of eight blocks) to some hundred (one block each).
CALLS = [(8, 1, 256, 1, 1), (6, 3, 80, 4, 1), (32, 8, 128, 3, 1), (8, 8, 64, 8, 1), (12, 2, 128, 2, 9), (16, 16, 64, 9, 1), (8, 1, 256, 4, 33), (4, 4, 128, 38, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("R,window,sink", [(1, 1, 0), (40, 33, 1), (333, 300, 5), (1000, 600, 70)])
@pytest.mark.parametrize("H,K,D,B,T", CALLS)
def test_windows_of_few_tiles(kv, dtype, H, K, D, B, T, R, window, sink):
    check_window(kv, dtype, H, K, D, B, T, R, window, sink, seed=R, mask="any" if T > 1 else "causal")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("R,block,window,sink", [(1, 16, 0, 0), (100, 16, 0, 0), (700, 32, 0, 0), (1001, 64, 500, 20)])
@pytest.mark.parametrize("H,K,D,B,T", CALLS)
def test_8_bit_caches_under_few_tiles(kv, dtype, H, K, D, B, T, R, block, window, sink):
    check_attend8(kv, dtype, H, K, D, B, T, R, block, window, sink, seed=R, mask="any" if T > 1 else "causal")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [1, 5])
def test_what_only_one_part_sees_reaches_its_rows_alone(kv, dtype, T):
    """NaN keys, NaN and infinite values in single rows of the cache, each in another part of the cluster."""
    H, K, D, B, R = 4, 1, 64, 3, 900
    q, k, v = rand(1, B, T, H, D, dtype=dtype), rand(2, B, R, K, D, dtype=dtype), rand(3, B, R, K, D, dtype=dtype)
    k[0, 700, 0, 5] = float("nan")
    v[1, 30, 0, 7] = float("nan")
    v[2, 890, 0, 9] = float("inf")
    seen = np.array([[R - 250 + 100 * t for t in range(T)], [R] * T, [R - 20 + 5 * t for t in range(T)]])
    seen = np.minimum(seen, R)
    h = kv.KV(H, K, D, max_batch=B, max_tokens=T, precision=dtype)
    out, lse = h.attend_window(q, (k, v), i32(seen), R)
    out, lse = np64(out), np64(lse)
    h.device_status()
    nan_key = seen[0] > 700
    assert np.isnan(out[0][nan_key]).all() and np.isnan(lse[0][nan_key]).all()
    assert np.isfinite(out[0][~nan_key]).all() and np.isfinite(lse[0][~nan_key]).all()
    bad = np.zeros(D, bool)
    bad[7] = True
    assert np.isnan(out[1][..., bad]).all() and np.isfinite(out[1][..., ~bad]).all() and np.isfinite(lse[1]).all()
    bad[:] = False
    bad[9] = True
    inf = seen[2] > 890
    assert np.isposinf(out[2][inf][..., bad]).all() and np.isfinite(out[2][~inf]).all() and np.isfinite(out[2][..., ~bad]).all()


def test_one_launch_in_a_graph_beside_another_stream(kv):
    """A captured call of clusters replayed while another handle's runs on another stream: neither has a workspace of the other's."""
    H, K, D, B, R = 8, 1, 256, 2, 867
    handles = [kv.KV(H, K, D, max_batch=B) for _ in range(2)]
    q, s = rand(1, B, 1, H, D), i32([[R], [R - 100]])
    c8 = fill8(kv, handles[0], B, R, 32, 5)
    k, v = rand(2, B, R, K, D), rand(3, B, R, K, D)
    want = [t.clone() for t in (*handles[0].attend8(q, c8, s), *handles[1].attend_window(q, (k, v), s, 500, sink=4))]
    ref = okv.attend_window(np64(q), np64(k), np64(v), np64(s).astype(int), 500, 4, 1 / math.sqrt(D))
    finish(want[2], want[3], want[2:], ref, tols(np64(q), np64(k), np64(v), R, "bf16", *ref[:1], ref[2], ref[3], ref[1], 1 / math.sqrt(D)))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = handles[0].attend8(q, c8, s)
    side = torch.cuda.Stream()
    outs = []
    for _ in range(20):
        g.replay()
        outs.append(handles[1].attend_window(q, (k, v), s, 500, sink=4, stream=side))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want[:2], got))
    for o in outs:
        assert all(torch.equal(a, b) for a, b in zip(want[2:], o))
    for h in handles:
        h.device_status()
