"""Host-side checks of the KV-cache operators that need no GPU: struct layouts, refusals that come
before any device call, and pins of their CPU oracle."""

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


@pytest.mark.parametrize("name", ["jpi_kv_config", "jpi_kv_rope", "jpi_kv_cache"])
def test_binding_structs_match_the_c_layout(name, tmp_path):
    inc = os.path.join(build.ROOT, "include")
    st = getattr(kv, name)
    fields = [f[0] for f in st._fields_]
    src = tmp_path / "probe.c"
    src.write_text("\n".join(['#include <stdio.h>', '#include <stddef.h>', '#include "jpi_kv.h"', "int main(void) {",
                              f'  printf("%zu\\n", sizeof({name}));'] +
                             [f'  printf("%zu\\n", offsetof({name}, {f}));' for f in fields] + ["  return 0;", "}"]))
    exe = tmp_path / "probe"
    subprocess.run(["gcc", "-I", inc, str(src), "-o", str(exe)], check=True, capture_output=True)
    out = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert [ctypes.sizeof(st)] + [getattr(st, f).offset for f in fields] == out


GOOD = dict(n_heads=8, n_kv_heads=1, head_dim=256, max_batch=4, max_tokens=4, scale=0.0, precision=0)


@pytest.mark.parametrize("bad", [dict(n_heads=0), dict(n_kv_heads=0), dict(n_heads=8, n_kv_heads=3), dict(head_dim=0),
                                 dict(head_dim=260), dict(head_dim=264), dict(head_dim=12), dict(head_dim=6, precision=1),
                                 dict(max_batch=0), dict(max_tokens=0), dict(max_batch=70000), dict(precision=2),
                                 dict(max_batch=60000, max_tokens=60000), dict(scale=-1.0), dict(scale=math.inf),
                                 dict(scale=math.nan), dict(n_heads=2048)])
def test_bad_configs_are_refused_before_any_device_call(lib, bad):
    h = ctypes.c_void_p()
    cfg = kv.jpi_kv_config(**{**GOOD, **bad})
    assert lib.jpi_kv_create(ctypes.byref(cfg), None, ctypes.byref(h)) in (-1, -2, -7)
    assert h.value is None and lib.jpi_last_error()


ROPE = dict(dim=64, layout="half", base=1e4, scaling="none", factor=1.0, low=1.0, high=32.0, original=1, mscale=1.0)


@pytest.mark.parametrize("bad", [dict(dim=0), dict(dim=63), dict(dim=258), dict(base=0.5), dict(base=math.inf),
                                 dict(base=math.nan), dict(mscale=0.0), dict(mscale=math.nan),
                                 dict(scaling="linear", factor=0.5), dict(scaling="ntk", factor=2.0, dim=2),
                                 dict(scaling="ntk", factor=math.inf), dict(scaling="by_parts", low=2.0, high=2.0),
                                 dict(scaling="by_parts", original=0), dict(scaling="by_parts", high=math.inf)])
def test_bad_rotary_codings_are_refused_before_any_device_call(lib, bad):
    h = ctypes.c_void_p()
    cfg, r = kv.jpi_kv_config(**GOOD), kv.Rope(**{**ROPE, **bad}).c()
    assert lib.jpi_kv_create(ctypes.byref(cfg), ctypes.byref(r), ctypes.byref(h)) == -1
    assert h.value is None and b"rope" in lib.jpi_last_error().lower()


def test_unknown_rotary_enums_are_refused(lib):
    h = ctypes.c_void_p()
    cfg = kv.jpi_kv_config(**GOOD)
    for field in ("layout", "scaling"):
        r = kv.Rope(**ROPE).c()
        setattr(r, field, 9)
        assert lib.jpi_kv_create(ctypes.byref(cfg), ctypes.byref(r), ctypes.byref(h)) == -1


def test_null_handles_are_refused(lib):
    c = kv.jpi_kv_cache()
    b, h = ctypes.c_longlong(), ctypes.c_void_p()
    assert lib.jpi_kv_create(None, None, ctypes.byref(h)) == -1
    assert lib.jpi_kv_create(None, None, None) == -1
    assert lib.jpi_kv_destroy(None) == 0
    assert lib.jpi_kv_append(None, None, 0, None, 0, None, 0, None, None, 1, 1, None, None, None) == -1
    assert lib.jpi_kv_attend(None, None, 0, 1, 1, None, 1, None, None, None, None, None, None) == -1
    assert lib.jpi_kv_weigh(None, None, 0, None, 1, 1, None, 1, None, None, None, 1.0, None, None, None, None, None) == -1
    assert lib.jpi_kv_evict(None, ctypes.byref(c), None, None, 1, 1, 1, 0, 0, ctypes.byref(c), None, None, None, None) == -1
    assert lib.jpi_kv_device_status(None) == -1
    assert lib.jpi_kv_memory_usage(None, ctypes.byref(b)) == -1


def test_null_experts_are_refused_by_the_calls_on_a_stored_prefix(lib):
    assert lib.jpi_share_prefix(None, 2) == -1
    assert lib.jpi_weigh_prefix(None, None, None, 0.0, 1, 1, 1.0, None, None) == -1
    assert lib.jpi_evict_prefix(None, None, 1, 0, 0, None, None) == -1
    assert lib.jpi_append_prefix(None, None, None, 1, None) == -1
    assert lib.jpi_commit_prefix_at(None, 1, 1, 1) == -1


# ------------------------------------------------------------------ pins of the oracle

@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_is_a_rotation_that_knows_differences_only(layout):
    rng = np.random.default_rng(0)
    r = kv.Rope(dim=12, layout=layout)
    q, k = rng.normal(size=16), rng.normal(size=16)
    assert np.allclose(okv.rope(q, 0, r), q)
    a = okv.rope(q, 9, r)
    assert np.allclose(np.linalg.norm(a), np.linalg.norm(q)) and np.allclose(a[12:], q[12:])
    assert np.allclose(okv.rope(q, 9, r) @ okv.rope(k, 4, r), okv.rope(q, 105, r) @ okv.rope(k, 100, r))
    assert np.allclose(okv.rope(okv.rope(q, 7, r), -7, r), q)


def test_rope_layouts_are_permutations_of_each_other():
    x = np.arange(8.0)
    perm = [0, 4, 1, 5, 2, 6, 3, 7]   # interleaved element p holds half-layout element perm[p]
    half = okv.rope(x, 3, kv.Rope(dim=8))
    assert np.allclose(okv.rope(x[perm], 3, kv.Rope(dim=8, layout="interleaved")), half[perm])


def test_rope_scalings():
    th = okv.rope_theta(kv.Rope(dim=64))
    assert th[0] == 1.0 and np.allclose(th[1:] / th[:-1], 1e4 ** (-2 / 64))
    assert np.allclose(okv.rope_theta(kv.Rope(dim=64, scaling="linear", factor=4.0)), th / 4)
    ntk = okv.rope_theta(kv.Rope(dim=64, scaling="ntk", factor=4.0))
    assert ntk[0] == 1.0 and np.isclose(ntk[-1], th[-1] / 4)      # the fastest pair stays, the slowest is interpolated
    parts = okv.rope_theta(kv.Rope(dim=64, scaling="by_parts", factor=4.0, original=4096, low=1.0, high=32.0))
    turns = 4096 * th / (2 * math.pi)
    assert np.allclose(parts[turns > 32], th[turns > 32]) and np.allclose(parts[turns < 1], th[turns < 1] / 4)
    assert np.all(parts <= th) and np.all(parts >= th / 4)


def test_attention_over_a_shared_prefix_is_attention_over_both_parts():
    rng = np.random.default_rng(1)
    q = rng.normal(size=(4, 2, 4, 8))
    pk, pv = rng.normal(size=(2, 5, 2, 8)), rng.normal(size=(2, 5, 2, 8))
    k, v = rng.normal(size=(4, 3, 2, 8)), rng.normal(size=(4, 3, 2, 8))
    plen, seen = np.array([5, 2]), np.array([[2, 3]] * 4)
    out, lse, _, _ = okv.attend(q, (pk, pv), plen, (k, v), seen, 0.5)
    for b in range(4):
        kk = np.concatenate([pk[b // 2, :plen[b // 2]], k[b, :2]])[:, 1]
        vv = np.concatenate([pv[b // 2, :plen[b // 2]], v[b, :2]])[:, 1]
        e = np.exp(0.5 * kk @ q[b, 0, 3])
        assert np.allclose(out[b, 0, 3], e @ vv / e.sum()) and np.isclose(lse[b, 0, 3], np.log(e.sum()))


def test_weights_of_a_query_sum_to_one_and_the_empty_query_gives_none():
    rng = np.random.default_rng(2)
    q, k = rng.normal(size=(1, 3, 2, 8)), rng.normal(size=(1, 6, 1, 8))
    seen = np.array([[0, 3, 6]])
    _, lse, _, _ = okv.attend(q, None, None, (k, k), seen, 1.0)
    assert np.all(lse[0, 0] == -np.inf)
    _, (w, _) = okv.weigh(q, lse, None, None, k, seen, 1.0, 0.0, None, None, None, np.full((1, 1, 6), 7.0))
    assert np.isclose(w.sum(), 2 * 2)   # two tokens that see something, two heads each


def test_evict_keeps_the_protected_rows_and_the_heaviest():
    w = [0.0, 9.0, 1.0, 5.0, 5.0, math.nan, 5.0, 2.0]
    assert okv.evict(w, 8, 5, 1, 1) == [0, 1, 3, 4, 7]          # ties to the lowest row
    assert okv.evict(w, 8, 2, 1, 1) == [0, 7]
    assert okv.evict(w, 8, 8, 1, 1) == list(range(8)) and okv.evict(w, 3, 5, 1, 1) == [0, 1, 2]
    assert okv.evict([math.nan, math.nan, -math.inf], 3, 2, 0, 0) == [0, 2]


def test_the_module_of_checks_refuses_before_any_call(lib):
    """The checked calls' own refusals: nothing here reaches the entry points (their addresses are zero)."""
    torch = pytest.importorskip("torch")
    from paper_2607_12659_gb300 import _kv
    c = _kv.calls(8, 2, 64, True, 0, 0, 0, 0, 0)
    q, k = torch.zeros((2, 3, 8, 64), dtype=torch.bfloat16), torch.zeros((2, 5, 2, 64), dtype=torch.bfloat16)
    i, f = torch.zeros((2, 3), dtype=torch.int32), torch.zeros((2, 3, 8))
    with pytest.raises(ValueError, match="q is a Strided tensor on cpu, the handle on cuda:0"):
        _kv.attend(c, 1, 0, q, (k, k), i, None, None, q, f)
    with pytest.raises(ValueError, match="cpu"):
        _kv.weigh(c, 1, 0, q, f, k, i, None, None, 1.0, None, None, None, None)
    with pytest.raises(ValueError, match="cpu"):
        _kv.append(c, 1, 0, q, k, k, i, i, k, k, q)
    with pytest.raises(ValueError, match="cpu"):
        _kv.evict(c, 1, 0, k[None], k[None], f, i, 1, 0, 0, k[None], k[None], f, i)
    with pytest.raises(ValueError, match="neither q nor k"):
        _kv.append(c, 1, 0, None, None, k, i, i, k, k, q)
    with pytest.raises(ValueError, match="layers"):
        _kv.evict(c, 1, 0, k, k, f, i, 1, 0, 0, k, k, f, i)
    for bad in (None, 3, [1.0]):
        with pytest.raises(TypeError, match="q must be a tensor"):
            _kv.attend(c, 1, 0, bad, (k, k), i, None, None, q, f)
    with pytest.raises(TypeError, match="10 arguments"):
        _kv.attend(c, 1, 0, q)
    with pytest.raises(TypeError):
        _kv.calls(8, 2, 64)
    for capsule, handle in ((None, 1), (c, "x")):
        with pytest.raises((TypeError, ValueError)):
            _kv.attend(capsule, handle, 0, q, (k, k), i, None, None, q, f)
    sparse = torch.sparse_coo_tensor(torch.zeros((4, 1), dtype=torch.int64), torch.ones(1, dtype=torch.bfloat16), (2, 3, 8, 64))
    for odd in (sparse, torch.empty((2, 3, 8, 64), dtype=torch.bfloat16, device="meta")):
        with pytest.raises(ValueError):
            _kv.attend(c, 1, 0, odd, (k, k), i, None, None, q, f)


def test_a_missing_module_of_checks_is_an_error(lib, monkeypatch):
    import sys
    monkeypatch.setitem(sys.modules, "paper_2607_12659_gb300._kv", None)
    monkeypatch.delattr("paper_2607_12659_gb300._kv", raising=False)
    with pytest.raises(RuntimeError, match="not built"):
        kv._checked_calls(8, 2, 64, True, 0)


def test_a_module_that_does_not_build_leaves_no_older_one(tmp_path, monkeypatch):
    """One built for another torch or Python would be imported in its place."""
    for name, file in (("BUILD", "."), ("KV_CALLS_LIB", "_kv.so")):
        monkeypatch.setattr(build, name, str(tmp_path / file))
    (tmp_path / "_kv.so").write_bytes(b"older")
    (tmp_path / "kv_calls.txt").write_text("older")
    for compiler in ("false", "no-such-compiler"):
        monkeypatch.setenv("CXX", compiler)
        with pytest.raises((RuntimeError, OSError)):
            build.build_kv_calls()
        assert not (tmp_path / "_kv.so").exists()
