"""Host-side checks of the norms, windows and 8-bit caches of the KV-cache operators that need no GPU: struct layouts, refusals
that come before any device call, and pins of their CPU oracle."""

import ctypes
import math
import os
import subprocess

import numpy as np
import pytest

from oracle import kv as okv
from paper_2607_12659_gb300 import build, jpi, kv


@pytest.fixture(scope="module")
def lib():
    build.build()
    return jpi.load()


@pytest.mark.parametrize("name", ["jpi_kv_norm", "jpi_kv8_cache"])
def test_binding_structs_match_the_c_layout(name, tmp_path):
    st = getattr(kv, name)
    fields = [f[0] for f in st._fields_]
    src = tmp_path / "probe.c"
    src.write_text("\n".join(['#include <stdio.h>', '#include <stddef.h>', '#include "jpi_kv.h"', "int main(void) {",
                              f'  printf("%zu\\n", sizeof({name}));'] +
                             [f'  printf("%zu\\n", offsetof({name}, {f}));' for f in fields] + ["  return 0;", "}"]))
    exe = tmp_path / "probe"
    subprocess.run(["gcc", "-I", os.path.join(build.ROOT, "include"), str(src), "-o", str(exe)], check=True, capture_output=True)
    out = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert [ctypes.sizeof(st)] + [getattr(st, f).offset for f in fields] == out


def test_null_handles_and_caches_are_refused(lib):
    assert lib.jpi_kv_append_normed(None, *[None, 0] * 3, None, None, None, 1, 1, None, None, None) == -1
    assert lib.jpi_kv_attend_window(None, None, 0, 1, 1, None, None, 1, 0, None, None, None) == -1
    assert lib.jpi_kv8_append(None, *[None, 0] * 3, None, None, None, None, 1, 1, None, None, None) == -1
    assert lib.jpi_kv8_attend(None, None, 0, 1, 1, None, None, 0, 0, None, None, None) == -1
    assert lib.jpi_last_error()


def test_the_module_of_checks_refuses_before_any_call(lib):
    torch = pytest.importorskip("torch")
    from paper_2607_12659_gb300 import _kv
    c = _kv.calls(8, 2, 64, True, 0, *[0] * 8)
    q, k = torch.zeros((2, 3, 8, 64), dtype=torch.bfloat16), torch.zeros((2, 5, 2, 64), dtype=torch.bfloat16)
    i, f = torch.zeros((2, 3), dtype=torch.int32), torch.zeros((2, 3, 8))
    k8, s8 = k.to(torch.float8_e4m3fn), torch.zeros((2, 2, 1), dtype=torch.uint8).view(torch.float8_e8m0fnu)
    with pytest.raises(ValueError, match="cpu"):
        _kv.append_normed(c, 1, 0, q, k, k, i, i, k, k, q, None, None, 1e-6)
    with pytest.raises(TypeError, match="eps"):
        _kv.append_normed(c, 1, 0, q, k, k, i, i, k, k, q, None, None, "small")
    with pytest.raises(ValueError, match="cpu"):
        _kv.append_normed(c, 1, 0, q, k, k, i, i, k, k, q, torch.zeros(64), None, 1e-6)
    with pytest.raises(ValueError, match="cpu"):
        _kv.attend_window(c, 1, 0, q, (k, k), i, 4, 0, q, f)
    with pytest.raises(ValueError, match="cpu"):
        _kv.append8(c, 1, 0, q, k, k, i, i[:, 0], None, k8, k8, s8, s8, 32, q, None, None, None, None)
    with pytest.raises(ValueError, match="neither"):
        _kv.append8(c, 1, 0, None, None, k, i, i[:, 0], None, k8, k8, s8, s8, 32, q, None, None, None, None)
    with pytest.raises(ValueError, match="cpu"):
        _kv.attend8(c, 1, 0, q, k8, k8, s8, s8, 32, i, 0, 0, q, f)
    for call, n in ((_kv.append_normed, 14), (_kv.attend_window, 10), (_kv.append8, 19), (_kv.attend8, 14)):
        with pytest.raises(TypeError, match=f"{n} arguments"):
            call(c, 1, 0, q)


# ------------------------------------------------------------------ the oracle

def test_a_normed_head_has_its_weights_for_a_root_mean_square():
    rng = np.random.default_rng(0)
    x, w = rng.normal(size=(3, 4, 16)) * 7, rng.normal(size=16)
    y = okv.norm(x, None, 1e-12)
    assert np.allclose((y ** 2).mean(-1), 1) and np.allclose(y * np.sqrt((x ** 2).mean(-1, keepdims=True)), x)
    assert np.allclose(okv.norm(x, w, 1e-12), y * w)
    assert np.allclose(okv.norm(np.full((1, 4), 2.0), None, 5.0), 2 / 3)
    assert np.all(okv.norm(np.zeros((1, 4)), None, 1e-6) == 0)


def test_what_a_window_shows():
    assert okv.visible(10, 20, 3, 0).tolist() == [7, 8, 9]
    assert okv.visible(10, 20, 3, 2).tolist() == [0, 1, 7, 8, 9]
    assert okv.visible(10, 20, 3, 8).tolist() == list(range(10))
    assert okv.visible(2, 20, 3, 8).tolist() == [0, 1] and okv.visible(0, 20, 3, 8).tolist() == []
    assert okv.visible(-4, 20, 3, 0).tolist() == [] and okv.visible(99, 4, 2, 1).tolist() == [0, 2, 3]
    assert okv.visible(5, 9, 0, 0).tolist() == list(range(5))


def test_a_window_over_everything_is_plain_attention():
    rng = np.random.default_rng(1)
    q, k, v = rng.normal(size=(2, 3, 4, 8)), rng.normal(size=(2, 9, 2, 8)), rng.normal(size=(2, 9, 2, 8))
    seen = np.array([[0, 4, 9], [1, 2, 3]])
    for a, b in zip(okv.attend_window(q, k, v, seen, 9, 0, 0.3), okv.attend(q, None, None, (k, v), seen, 0.3)):
        assert np.allclose(a, b)
    out, lse, _, _ = okv.attend_window(q, k, v, seen, 1, 0, 0.3)
    assert np.allclose(out[0, 2].reshape(2, 2, 8), v[0, 8][:, None]) and np.all(lse[0, 0] == -np.inf) and np.all(out[0, 0] == 0)


def test_e4m3_numbers():
    torch = pytest.importorskip("torch")
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    fine = codes[np.isfinite(codes)]
    assert np.array_equal(okv.e4m3(fine), fine) and fine.max() == 448
    rng = np.random.default_rng(2)
    x = rng.uniform(-448, 448, 2000) * 2.0 ** rng.integers(-18, 1, 2000)
    near = fine[np.abs(x[:, None] - fine).argmin(1)]
    assert np.all(np.abs(okv.e4m3(x) - x) <= np.abs(near - x))
    assert np.all(np.abs(okv.e4m3(x) - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10))
    assert okv.e4m3(17.0) == 16 and okv.e4m3(19.0) == 20 and np.all(np.isnan(okv.e4m3([np.inf, np.nan])))


def test_scales_are_the_least_that_hold_a_block():
    for top in (448.0, 449.0, 1.0, 1.75, 1.7500001, 3e-3, 1e30, 2.0 ** -140, 5e37):
        e = okv.scale8([0.0, -top])
        assert top <= 448 * 2.0 ** (e - 127) and (e == 1 or top > 448 * 2.0 ** (e - 128))
    assert okv.scale8([0.0]) == 1 and okv.scale8([math.nan, math.inf, 448.0]) == 127


def test_blocks_that_are_begun_keep_or_raise_their_scale():
    block, R = 4, 10
    codes, scales = np.full((1, R, 1, 2), 8.0), np.full((1, 1, 3), 127)
    x = np.array([100.0, 1000.0, 3.0, 3.0, 3.0])[None, :, None, None] * np.ones(2)
    c, s = okv.append8(x, [2], [5], codes, scales, block)
    # Block 0 holds rows 0 and 1 already: raised to 4 by the 1000. Block 1 is new: its own scale. Block 2 is not touched.
    assert s.tolist() == [[[129, 127 - 7, 127]]]
    v = okv.values8(c, s, block)[0, :, 0, 0]
    assert v.tolist() == [8, 8, 96, 1024, 3, 3, 3, 8 / 128, 8, 8]   # (row 7: left as it was, under its block's new scale)
    c, s = okv.append8(x, [2], [1], codes, scales, block)
    assert s.tolist() == [[[127, 127, 127]]] and c[0, :4, 0, 0].tolist() == [8, 8, 96, 8]
    for start, count in ((-1, 3), (10, 3), (2, 0), (2, -1)):
        c, s = okv.append8(x, [start], [count], codes, scales, block)
        assert np.array_equal(c, codes) and np.array_equal(s, scales)
    c, s = okv.append8(x, [8], [5], codes, scales, block)
    assert c.shape == codes.shape and s[0, 0, 2] == 127 + 2 and s[0, 0, :2].tolist() == [127, 127]
