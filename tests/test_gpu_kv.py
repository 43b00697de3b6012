"""KV-cache operators on the GPU against their fp64 oracle.

Tolerances are worst-case bounds from the formats and the lengths of the sums. A rounding to a type is off
by at most eps / 2 of the value. Products of two bf16 values are exact in fp32; a score is a sum of D of
them in fp32 (D + 2 steps of 2^-23 of the sum of |q_d k_d|, doubled for sums that round towards zero);
2^x comes within 2^-21; a probability in bf16 is off by 2^-8 of itself, as two bf16 terms by 2^-16.
"""

import math
from decimal import Decimal, localcontext

import numpy as np
import pytest

from gpu_util import lib
from oracle import kv as okv

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def kv():
    lib()
    from paper_2607_12659_gb300 import kv
    return kv


@pytest.fixture(params=["by size", "1"])
def tiles(request, monkeypatch):
    """Kernels chosen by size, and the tensor-core tiles also where a call is too small for them."""
    if request.param == "1":
        monkeypatch.setenv("JPI_KV_TILES", "1")


DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF_EPS = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


def rand(seed, *shape, dtype="bf16", std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(DT[dtype])


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def np64(t):
    return None if t is None else t.double().cpu().numpy()


def within(got, ref, tol, what=""):
    got, ref = np64(got), np.asarray(ref)
    assert got.shape == ref.shape
    with np.errstate(invalid="ignore"):
        bad = ~(np.abs(got - ref) <= tol) & ~((got == ref) & np.isinf(ref))
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        pytest.fail(f"{what}: {bad.sum()} of {bad.size} off, first at {i}: {got[i]} for {ref[i]}, tolerance "
                    f"{np.broadcast_to(tol, ref.shape)[i]:.3g}")


def head_major(t):
    """The same cache stored [caches][KV heads][rows][D]."""
    return t.transpose(1, 2).contiguous().transpose(1, 2)


def padded(t, extra=3):
    """The same cache inside a longer one with another row stride."""
    big = torch.full((t.shape[0], t.shape[1], t.shape[2] + extra, t.shape[3]), float("nan"), dtype=t.dtype, device="cuda")
    big[:, :, :t.shape[2]] = t
    return big[:, :, :t.shape[2]]


# ------------------------------------------------------------------ append

ROPES = [None, dict(dim=256), dict(dim=64, layout="interleaved"), dict(dim=32, scaling="linear", factor=4.0),
         dict(dim=128, scaling="ntk", factor=8.0), dict(dim=96, layout="interleaved", scaling="ntk", factor=3.0),
         dict(dim=64, scaling="by_parts", factor=16.0, original=4096, mscale=1.25), dict(dim=10),
         dict(dim=2, layout="interleaved", base=500000.0), dict(dim=20, mscale=0.5)]


def check_append(kv, dtype, H, K, D, B, T, R, rope, seed, max_pos=5000, store=lambda t: t, padding=0.2):
    r = None if rope is None else kv.Rope(**rope)
    h = kv.KV(H, K, D, max_batch=B, max_tokens=T, precision=dtype, rope=r)
    rng = np.random.default_rng(seed)
    qkv = rand(seed, B, T, H + 2 * K, D, dtype=dtype)
    ck, cv = store(rand(seed + 1, B, R, K, D, dtype=dtype)), store(rand(seed + 2, B, R, K, D, dtype=dtype))
    pos = rng.integers(-max_pos, max_pos + 1, (B, T))
    rows = np.stack([rng.permutation(R)[:T] for _ in range(B)])
    rows[rng.random((B, T)) < padding] = -1
    rows[0][rows[0] == 0] = -1      # row 0 once: of two tokens with one row either may stay
    rows[0, 0] = 0
    if T > 1:
        rows[0, 1] = R   # past the end: padding too
    q, k, v = qkv[:, :, :H], qkv[:, :, H:H + K], qkv[:, :, H + K:]
    want_q, want_k, want_v = okv.append(np64(q), np64(k), np64(v), pos, rows, np64(ck), np64(cv), r)
    mark = torch.full((B, T, H, D), 3.5, dtype=DT[dtype], device="cuda")
    got = h.append(q, k, v, i32(pos), i32(rows), ck, cv, q_out=mark)
    torch.cuda.synchronize()
    live = (rows >= 0) & (rows < R)
    # sin and cos to 2^-22, two products and a sum in fp32
    size = (1.0 if r is None else r.mscale) * 2 * max(np.abs(np64(qkv)).max(), 1.0)
    abs_tol = size * 2.0 ** -21
    half = HALF_EPS[dtype]
    assert np.all(np64(got)[~live] == 3.5)
    within(got[torch.tensor(live)], want_q[live], half * np.abs(want_q[live]) + abs_tol, "q")
    within(ck, want_k, half * np.abs(want_k) + abs_tol, "k")
    assert np.array_equal(np64(cv), want_v)
    # untouched rows are the same bit for bit: the oracle holds them unrounded
    return h


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", range(len(ROPES)))
def test_append_codings(kv, dtype, n):
    check_append(kv, dtype, 6, 2, 256, 3, 5, 11, ROPES[n], 10 * n)


@pytest.mark.parametrize("dtype,H,K,D,B,T,R", [
    ("bf16", 1, 1, 8, 1, 1, 1), ("bf16", 8, 1, 256, 1, 1, 867), ("bf16", 32, 8, 128, 7, 1, 40), ("bf16", 12, 3, 96, 2, 33, 40),
    ("fp32", 4, 1, 64, 2, 17, 17), ("fp32", 3, 3, 20, 5, 2, 9), ("bf16", 64, 64, 80, 2, 3, 4)])
def test_append_shapes_and_layouts(kv, dtype, H, K, D, B, T, R):
    for i, store in enumerate((lambda t: t, head_major, padded)):
        check_append(kv, dtype, H, K, D, B, T, R, dict(dim=D // 2 // 2 * 2 or 2), 100 + i, store=store)


def test_append_far_positions_are_exact(kv):
    # Angles of positions near 2^31, where 32-bit angles would be off by whole turns.
    check_append(kv, "fp32", 2, 1, 64, 2, 9, 20, dict(dim=64), 5, max_pos=2 ** 31 - 1)


def test_append_parts(kv):
    """Queries alone, keys alone, and keys coded where they lie, forth and back."""
    r = kv.Rope(dim=64)
    h = kv.KV(4, 2, 64, max_batch=2, max_tokens=6, precision="fp32", rope=r)
    q, k = rand(1, 2, 6, 4, 64, dtype="fp32"), rand(2, 2, 6, 2, 64, dtype="fp32")
    pos, rows = i32([[5, 6, 7, 8, 9, 10]] * 2), i32([[0, 1, 2, 3, 4, 5]] * 2)
    out = h.append(q, None, None, pos, rows)
    ref = np.stack([[[okv.rope(np64(q)[b, t, n], int(pos[b, t]), r) for n in range(4)] for t in range(6)] for b in range(2)])
    within(out, ref, 2.0 ** -24 * np.abs(ref) + 2.0 ** -18)
    cache = k.clone()
    h.append(None, cache, None, pos, rows, cache)
    assert not torch.equal(cache, k)
    h.append(None, cache, None, -pos, rows, cache)
    within(cache, np64(k), np.full(k.shape, 2.0 ** -18))


def test_append_passes_32_bit_offsets(kv):
    """A row more than 2^31 elements into a cache."""
    K, D, R = 1, 256, (1 << 23) + 10
    cache = torch.zeros((1, R, K, D), dtype=torch.bfloat16, device="cuda")
    h = kv.KV(1, 1, D, rope=kv.Rope(dim=D))
    x = rand(3, 1, 1, 1, D)
    h.append(None, x, x, i32([[0]]), i32([[R - 1]]), cache, cache.clone())
    assert torch.equal(cache[0, R - 1], x[0, 0]) and not cache[0, :100].any()
    out, _ = kv.KV(1, 1, D).attend(x, prefix=(cache[:, R - 20:], cache[:, R - 20:]), prefix_len=i32([20]))
    assert out.isfinite().all()
    got, _ = kv.KV(1, 1, D).attend(x, prefix=(cache, cache), prefix_len=i32([R]))
    assert got.float().abs().max() > 1e-2      # the last row's weight: e^(|x|^2 / 16) of 2^23 zeros'
    del cache


def turns_exact(dim, i, base):
    """Turns per position of pair i of a plain coding, in 60 digits."""
    with localcontext() as ctx:
        ctx.prec = 60
        two_pi = Decimal("6.28318530717958647692528676655900576839433879875021164194989")
        return (-(Decimal(base).ln() * 2 * i / dim)).exp() / two_pi


def test_append_angles_at_any_position(kv):
    """Angles within 2^-26 + |position| 2^-53 turns, against 60 digits: pairs (1, 0) become (cos, sin)."""
    dim, base = 64, 10000.0
    pos = [0, 1, 7, 816, 4095, 131071, 10 ** 6, 2 ** 24 + 1, 2 ** 28 - 3, 2 ** 30 + 12345, 2 ** 31 - 1, -1, -131071, -(2 ** 31)]
    T = len(pos)
    h = kv.KV(1, 1, dim, max_tokens=T, precision="fp32", rope=kv.Rope(dim=dim, base=base))
    x = torch.zeros((1, T, 1, dim), device="cuda")
    x[..., :dim // 2] = 1.0
    got = np64(h.append(x, None, None, i32([pos]), i32([list(range(T))])))[0, :, 0]
    turns = [turns_exact(dim, i, base) for i in range(dim // 2)]
    for t, p in enumerate(pos):
        frac = np.array([float((p * x) % 1) for x in turns])
        # sines and cosines to 2^-22 beside the angle's bound
        tol = 2 * math.pi * (2.0 ** -26 + abs(p) * 2.0 ** -53) + 2.0 ** -22
        for part, want in ((got[t, :dim // 2], np.cos(2 * math.pi * frac)), (got[t, dim // 2:], np.sin(2 * math.pi * frac))):
            assert np.abs(part - want).max() <= tol, (p, np.abs(part - want).max(), tol)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_append_two_tokens_of_one_row(kv, dtype):
    """What the row holds then is either token's, element by element; every other row is as without them."""
    H, K, D, B, T, R = 4, 2, 64, 2, 40, 50
    h = kv.KV(H, K, D, max_batch=B, max_tokens=T, precision=dtype, rope=kv.Rope(dim=D))
    q, k, v = rand(1, B, T, H, D, dtype=dtype), rand(2, B, T, K, D, dtype=dtype), rand(3, B, T, K, D, dtype=dtype)
    pos = i32([list(range(T))] * B)
    rows = np.stack([np.random.default_rng(b).permutation(R)[:T] for b in range(B)])
    alone = [torch.zeros((B, R, K, D), dtype=DT[dtype], device="cuda") for _ in range(2)]
    want_q = h.append(q, k, v, pos, i32(rows), *alone)
    twice = rows.copy()
    twice[:, 7] = rows[:, 30]
    got = [torch.zeros((B, R, K, D), dtype=DT[dtype], device="cuda") for _ in range(2)]
    assert torch.equal(h.append(q, k, v, pos, i32(twice), *got), want_q)
    for a, b in zip(got, alone):
        for n in range(B):
            one, other = b[n, rows[n, 7]], b[n, rows[n, 30]]
            assert ((a[n, rows[n, 30]] == one) | (a[n, rows[n, 30]] == other)).all()
            want = b[n].clone()
            want[rows[n, 7]], want[rows[n, 30]] = 0, a[n, rows[n, 30]]
            assert torch.equal(a[n], want)


# ------------------------------------------------------------------ attend

def make_call(seed, dtype, H, K, D, B, T, G, P, R, mask="causal", store=lambda t: t, std=2.0):
    """Inputs of a call; rows that no query sees hold NaN and infinities."""
    rng = np.random.default_rng(seed)
    c = dict(q=rand(seed, B, T, H, D, dtype=dtype, std=std), prefix=None, prefix_len=None, own=None, seen=None)
    bad = torch.tensor([float("nan"), float("inf"), -float("inf")], device="cuda", dtype=DT[dtype])
    if P:
        pk, pv = rand(seed + 1, G, P, K, D, dtype=dtype), rand(seed + 2, G, P, K, D, dtype=dtype)
        n = rng.integers(max(0, P - 20), P + 1, G)
        if G > 1:
            n[rng.integers(G)] = 0
        for g in range(G):
            pk[g, n[g]:] = bad[g % 3]
            pv[g, n[g]:] = bad[(g + 1) % 3]
        c.update(prefix=(store(pk), store(pv)), prefix_len=i32(n))
    if R:
        ok, ov = rand(seed + 3, B, R, K, D, dtype=dtype), rand(seed + 4, B, R, K, D, dtype=dtype)
        top = rng.integers(0, R + 1, B)
        if mask == "causal":
            seen = np.clip(top[:, None] - T + 1 + np.arange(T), 0, None)
        elif mask == "context":
            seen = np.where(np.arange(T) < max(1, T // 3), np.minimum(1, top)[:, None], top[:, None])
        else:
            seen = rng.integers(0, R + 1, (B, T))
        for b in range(B):
            ok[b, seen[b].max():] = bad[b % 3]
            ov[b, seen[b].max():] = bad[(b + 2) % 3]
        c.update(own=(store(ok), store(ov)), seen=i32(seen))
    return c


def attend_ref(c, scale):
    f = lambda p: None if p is None else tuple(np64(t) for t in p)
    seen = None if c["seen"] is None else c["seen"].cpu().numpy()
    plen = None if c["prefix_len"] is None else c["prefix_len"].cpu().numpy()
    return okv.attend(np64(c["q"]), f(c["prefix"]), plen, f(c["own"]), seen, scale)


def attend_tols(c, dtype, ref, dot, mass, lse):
    B, T, H, D = c["q"].shape
    n = sum(p[0].shape[1] for p in (c["prefix"], c["own"]) if p is not None)
    rel = (D + 2) * 2.0 ** -22 * dot + 2.0 ** -20 + n * 2.0 ** -23 + 2.0 ** -22 * np.where(np.isinf(lse), 0, np.abs(lse))
    out = HALF_EPS[dtype] * np.abs(ref) + (2 * rel[..., None] + (2.0 ** -8 if dtype == "bf16" else 0)) * mass + 1e-37
    return out, rel + 1e-6


def check_attend(kv, dtype, H, K, D, B, T, G, P, R, seed=0, scale=0.0, **kw):
    c = make_call(seed, dtype, H, K, D, B, T, G, P, R, **kw)
    h = kv.KV(H, K, D, max_batch=B, max_tokens=T, precision=dtype, scale=scale)
    out, lse = h.attend(**c)
    again, lse2 = h.attend(**c)
    h.device_status()
    ref, rlse, dot, mass = attend_ref(c, scale or 1 / math.sqrt(D))
    tol, ltol = attend_tols(c, dtype, ref, dot, mass, rlse)
    within(out, ref, tol, "out")
    within(lse, rlse, ltol, "lse")
    empty = np.isinf(rlse)
    assert np.all(np64(out)[empty] == 0) and np.all(np64(lse)[empty] == -np.inf)
    assert torch.equal(out, again) and torch.equal(lse, lse2), "two runs differ"
    return c, out, lse


SHAPES = [(8, 1, 256), (4, 1, 64), (8, 8, 128), (32, 8, 128), (6, 2, 80), (14, 2, 128), (12, 3, 96), (1, 1, 8), (5, 5, 40),
          (16, 1, 256), (3, 1, 160)]


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H,K,D", SHAPES)
def test_attend_head_shapes(kv, dtype, H, K, D):
    check_attend(kv, dtype, H, K, D, 3, 1, 1, 77, 20, seed=H)
    check_attend(kv, dtype, H, K, D, 4, 5, 2, 33, 18, seed=H + 1, mask="any")


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("P,R", [(1, 0), (0, 1), (1, 1), (15, 17), (16, 16), (63, 0), (64, 3), (65, 1), (129, 0), (816, 51),
                                 (1000, 0), (0, 300), (2049, 5)])
def test_attend_lengths(kv, dtype, P, R):
    check_attend(kv, dtype, 8, 1, 128, 2, 3, 1, P, R, seed=P + R)


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("mask", ["causal", "context", "any"])
@pytest.mark.parametrize("B,T,G", [(1, 1, 1), (2, 51, 1), (6, 7, 3), (8, 16, 4), (5, 40, 5), (33, 2, 1), (64, 4, 2)])
def test_attend_batches_and_masks(kv, mask, B, T, G):
    check_attend(kv, "bf16", 8, 1, 64, B, T, G, 100, 60, seed=B + T, mask=mask)


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("H,K,D,B,T,G,P,R", [
    (8, 1, 256, 2, 100, 1, 130, 300), (16, 2, 128, 3, 64, 3, 70, 1000), (4, 1, 64, 2, 33, 1, 5, 129), (8, 1, 256, 1, 300, 1, 0, 700),
    (8, 1, 256, 16, 1, 1, 816, 40), (8, 1, 256, 40, 1, 1, 333, 9), (8, 1, 256, 4, 51, 2, 200, 51), (8, 1, 128, 32, 1, 1, 700, 5),
    (32, 8, 128, 48, 1, 1, 450, 33), (16, 16, 64, 64, 2, 1, 260, 12), (8, 1, 256, 18, 8, 1, 64, 0), (8, 1, 64, 16, 3, 1, 1, 1)])
def test_attend_many_rows_on_one_prefix(kv, H, K, D, B, T, G, P, R):
    check_attend(kv, "bf16", H, K, D, B, T, G, P, R, seed=B)


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("H,K,D,B,T,P,R", [(8, 1, 256, 64, 1, 4096, 300), (8, 1, 256, 64, 1, 16384, 512), (32, 8, 128, 48, 1, 4000, 100),
                                            (8, 1, 64, 64, 2, 8000, 0), (8, 2, 256, 9, 16, 2100, 700)])
def test_attend_long_prefix_many_rows(kv, H, K, D, B, T, P, R):
    """Blocks of many keys: the last products are waited for, however far behind the scores they are."""
    c, out, lse = check_attend(kv, "bf16", H, K, D, B, T, 1, P, R, seed=P)
    h = kv.KV(H, K, D, max_batch=B, max_tokens=T)
    for _ in range(10):
        again, lse2 = h.attend(**c)
        assert torch.equal(out, again) and torch.equal(lse, lse2), "two runs differ"


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("store", [head_major, padded])
def test_attend_cache_layouts(kv, dtype, store):
    check_attend(kv, dtype, 8, 4, 128, 4, 3, 2, 90, 30, seed=3, store=store)
    check_attend(kv, dtype, 8, 2, 256, 40, 2, 1, 190, 30, seed=4, store=store)


@pytest.mark.usefixtures("tiles")
def test_attend_scale_and_large_scores(kv):
    check_attend(kv, "bf16", 8, 1, 64, 2, 2, 1, 120, 10, seed=1, scale=0.02)
    check_attend(kv, "bf16", 8, 1, 128, 20, 1, 1, 300, 10, seed=2, std=30.0)
    check_attend(kv, "fp32", 2, 1, 64, 2, 2, 1, 120, 10, seed=3, std=30.0)


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("dtype,H,K,D,T,R", [("fp32", 8, 1, 64, 6, 12), ("bf16", 2, 1, 64, 6, 12), ("bf16", 8, 1, 64, 6, 12),
                                             ("bf16", 8, 1, 256, 40, 150), ("bf16", 16, 2, 128, 70, 300), ("bf16", 8, 1, 96, 20, 70),
                                             ("bf16", 4, 4, 64, 50, 200)])
def test_attend_a_bad_value_reaches_only_the_queries_that_see_it(kv, dtype, H, K, D, T, R):
    """Infinities and NaN among the values, in the first, a middle and the last rows: the queries that see them get
    non-finite results in that element, the others what the oracle gives without them."""
    c = make_call(7, dtype, H, K, D, 2, T, 1, 20, R, mask="any")
    rng = np.random.default_rng(R)
    seen = np.sort(rng.integers(0, R + 1, (2, T)), axis=1)
    seen[0, 0], seen[0, -1] = 0, R
    seen[1] = rng.permutation(seen[1])
    c["seen"] = i32(seen)
    for t in c["own"]:
        t.copy_(rand(8, *t.shape, dtype=dtype))
    ref, rlse, dot, mass = attend_ref(c, 1 / math.sqrt(D))
    tol, ltol = attend_tols(c, dtype, ref, dot, mass, rlse)
    h = kv.KV(H, K, D, max_batch=2, max_tokens=T, precision=dtype)
    for bad in (float("nan"), float("inf")):
        for at in (0, R // 2, R - 1):
            dirty = dict(c, own=(c["own"][0], c["own"][1].clone()))
            dirty["own"][1][:, at, 0, 3] = bad
            got, lse = h.attend(**dirty)
            h.device_status()
            within(lse, rlse, ltol, "lse")
            sees = seen > at                                            # [2][T]
            hit = np.zeros(ref.shape, bool)
            hit[:, :, :H // K, 3] = sees[:, :, None]
            assert not np.isfinite(np64(got)[hit]).any()
            clean = torch.where(torch.tensor(hit, device="cuda"), torch.zeros_like(got), got)
            within(clean, np.where(hit, 0.0, ref), np.where(hit, 0.0, tol), f"value {bad} in row {at}")


@pytest.mark.usefixtures("tiles")
def test_attend_lowest_values_and_lengths_out_of_range(kv):
    # Scores of the type's lowest value are values; lengths outside a cache are taken as its ends.
    q = torch.full((1, 1, 1, 8), torch.finfo(torch.bfloat16).max, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros((1, 2, 1, 8), dtype=torch.bfloat16, device="cuda")
    k[0, 0, 0, 0] = -1.0
    v = rand(1, 1, 2, 1, 8)
    out, lse = kv.KV(1, 1, 8, scale=1.0).attend(q, own=(k, v), seen=i32([[99]]))
    assert torch.equal(out[0, 0, 0], v[0, 1, 0]) and lse.item() == 0.0
    out, lse = kv.KV(1, 1, 8, scale=1.0).attend(q, own=(k, v), seen=i32([[-5]]))
    assert not out.any() and lse.item() == -math.inf
    out, lse = kv.KV(1, 1, 8, scale=1.0).attend(q, own=(k, v), seen=i32([[1]]))
    assert torch.equal(out[0, 0, 0], v[0, 0, 0])     # the only key, however low its score


@pytest.mark.parametrize("tiles,prob", [("0", 2.0 ** -16), ("1", 2.0 ** -8)])
@pytest.mark.parametrize("H,K,D,B,T,G,P,R", [(8, 1, 256, 8, 20, 2, 300, 30), (16, 2, 128, 40, 1, 1, 700, 20), (8, 1, 64, 2, 64, 1, 40, 300)])
def test_attend_rounding_of_the_probabilities(kv, monkeypatch, tiles, prob, H, K, D, B, T, G, P, R):
    """Two bf16 terms in the row kernels (each half an eps of what it holds: 2^-8 of 2^-8), one on the tiles."""
    monkeypatch.setenv("JPI_KV_TILES", tiles)
    c = make_call(D, "bf16", H, K, D, B, T, G, P, R)
    out, lse = kv.KV(H, K, D, max_batch=B, max_tokens=T).attend(**c)
    ref, rlse, dot, mass = attend_ref(c, 1 / math.sqrt(D))
    tol, _ = attend_tols(c, "fp32", ref, dot, mass, rlse)      # scores, 2^x and sums
    within(out, ref, tol - HALF_EPS["fp32"] * np.abs(ref) + HALF_EPS["bf16"] * np.abs(ref) + prob * (1 + 2.0 ** -7) * mass, "out")


# ------------------------------------------------------------------ weigh

def check_weigh(kv, dtype, H, K, D, B, T, G, P, R, seed=0, decay=0.75, with_in=True, **kw):
    c = make_call(seed, dtype, H, K, D, B, T, G, P, R, **kw)
    scale = 1 / math.sqrt(D)
    _, lse, _, _ = attend_ref(c, scale)
    lse = torch.tensor(lse, dtype=torch.float32, device="cuda")
    h = kv.KV(H, K, D, max_batch=B, max_tokens=T, precision=dtype)
    shape = {"prefix": (G, K, P), "own": (B, K, R)}
    live = {k: c[k] is not None for k in shape}
    w = {k: rand(seed + 9, *s, dtype="fp32").square() if live[k] and with_in else None for k, s in shape.items()}
    out = {k: torch.full(s, 5.0, device="cuda") if live[k] else None for k, s in shape.items()}
    seen = None if c["seen"] is None else c["seen"].cpu().numpy()
    plen = None if c["prefix_len"] is None else c["prefix_len"].cpu().numpy()
    ref = okv.weigh(np64(c["q"]), np64(lse), *(np64(x) for x in ((c["prefix"] or [None])[0],)), plen,
                    np64((c["own"] or [None])[0]), seen, scale, decay, np64(w["prefix"]), np64(w["own"]),
                    np64(out["prefix"]), np64(out["own"]))
    args = dict(prefix=(c["prefix"] or [None])[0], prefix_len=c["prefix_len"], own=(c["own"] or [None])[0], seen=c["seen"],
                w_prefix=w["prefix"], w_own=w["own"], decay=decay)
    got = h.weigh(c["q"], lse, **args, out_prefix=out["prefix"], out_own=out["own"])
    got = [None if g is None else g.clone() for g in got]
    again = h.weigh(c["q"], lse, **args, out_prefix=out["prefix"], out_own=out["own"])
    h.device_status()
    for g, a, (y, e) in zip(got, again, ref):
        assert (g is None) == (y is None)
        if g is not None:
            within(g, y, 2 * e + 1e-30)      # rows that hold no key keep the 5 they had: their bound is zero
            assert torch.equal(g, a), "two runs differ"
    return h, c, lse, got


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H,K,D", SHAPES)
def test_weigh_head_shapes(kv, dtype, H, K, D):
    check_weigh(kv, dtype, H, K, D, 4, 3, 2, 45, 18, seed=H, mask="any")


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("P,R", [(1, 0), (0, 1), (15, 17), (64, 3), (127, 0), (129, 4), (816, 51), (0, 300)])
def test_weigh_lengths(kv, P, R):
    check_weigh(kv, "bf16", 8, 1, 128, 2, 3, 1, P, R, seed=P)


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("H,K,D,B,T,G,P,R", [(8, 1, 256, 40, 1, 1, 333, 9), (8, 1, 256, 1, 32, 1, 500, 32), (32, 8, 128, 48, 1, 1, 450, 33),
                                             (16, 16, 64, 64, 2, 1, 260, 12), (8, 1, 64, 33, 4, 3, 130, 7), (8, 1, 256, 24, 3, 2, 90, 0)])
def test_weigh_many_rows(kv, H, K, D, B, T, G, P, R):
    check_weigh(kv, "bf16", H, K, D, B, T, G, P, R, seed=B, decay=1.0)


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("H,K,D,B,T,G,P,R", [(8, 1, 256, 5, 36, 1, 8, 40), (8, 1, 256, 4, 80, 2, 700, 0), (16, 2, 128, 9, 31, 1, 130, 3),
                                             (8, 1, 64, 130, 1, 1, 129, 1), (4, 1, 80, 3, 100, 3, 1, 5), (8, 2, 256, 48, 17, 3, 300, 7)])
def test_weigh_few_keys_many_rows(kv, H, K, D, B, T, G, P, R):
    """Row tiles of one key tile dealt to several blocks, in equal and unequal numbers."""
    check_weigh(kv, "bf16", H, K, D, B, T, G, P, R, seed=P)



@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_weigh_leaves_out_rows_without_a_sum(kv, dtype):
    """An lse of -infinity marks a row that saw nothing: it weighs nothing, whatever its query holds."""
    B, T, H, D = 3, 50, 8, 64
    c = make_call(3, dtype, H, 1, D, B, T, 1, 200, 60, mask="any")
    out, lse = kv.KV(H, 1, D, max_batch=B, max_tokens=T, precision=dtype).attend(**c)
    h = kv.KV(H, 1, D, max_batch=B, max_tokens=T, precision=dtype)
    c["prefix"], c["own"] = c["prefix"][0], c["own"][0]
    gone = torch.rand((B, T, 1), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") < 0.4
    lse = torch.where(gone, torch.full_like(lse, -math.inf), lse)
    want = h.weigh(lse=lse, **dict(c, q=torch.where(gone[..., None], torch.zeros_like(c["q"]), c["q"])))
    for bad in (float("nan"), float("inf"), -float("inf")):
        got = h.weigh(lse=lse, **dict(c, q=torch.where(gone[..., None], torch.full_like(c["q"], bad), c["q"])))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert want[0].isfinite().all() and want[0].sum() > 0


@pytest.mark.usefixtures("tiles")
def test_weigh_in_place_no_input_and_decay_zero(kv):
    check_weigh(kv, "bf16", 8, 2, 64, 2, 3, 1, 40, 9, with_in=False)
    h, c, lse, got = check_weigh(kv, "bf16", 8, 2, 64, 2, 3, 1, 40, 9, decay=0.5)
    nan = torch.full((1, 2, 40), float("nan"), device="cuda")
    a, _ = h.weigh(c["q"], lse, prefix=c["prefix"][0], prefix_len=c["prefix_len"], w_prefix=nan, decay=0.0)
    b, _ = h.weigh(c["q"], lse, prefix=c["prefix"][0], prefix_len=c["prefix_len"])
    assert torch.equal(a, b)
    h.weigh(c["q"], lse, prefix=c["prefix"][0], prefix_len=c["prefix_len"], w_prefix=a, out_prefix=a)
    within(a, 2 * np64(b), np64(b) * 2.0 ** -22 + 1e-30)
    for layout in (head_major, padded):
        check_weigh(kv, "bf16", 8, 4, 128, 4, 3, 2, 90, 30, store=layout)


# ------------------------------------------------------------------ evict

def check_evict(kv, w, lengths, keep, sink, recent, K=1, D=64, dtype="bf16", in_place=False, store=lambda t: t, seed=0):
    """w [L][N][K][R]."""
    w = torch.as_tensor(w, dtype=torch.float32, device="cuda")
    L, N, _, R = w.shape
    h = kv.KV(K, K, D, precision=dtype)
    k, v = (torch.stack([store(x) for x in rand(seed + i, L, N, R, K, D, dtype=dtype)]) for i in (1, 2))
    k0, v0, w0 = k.clone(), v.clone(), w.clone()
    length = i32(lengths)
    if in_place:
        kept = h.evict(k, v, w, length, keep, sink, recent)
        ok, ov, ow, ol = k, v, w, length
    else:
        ok, ov, ow = (torch.full_like(t, 7.0) for t in (k, v, w))
        ol = torch.full_like(length, -1)
        kept = h.evict(k, v, w, length, keep, sink, recent, out_k=ok, out_v=ov, out_w=ow, out_length=ol)
        assert torch.equal(k, k0) and torch.equal(v, v0) and torch.equal(w.nan_to_num(9e9), w0.nan_to_num(9e9))
    h.device_status()
    same = lambda a, b: torch.equal(a.nan_to_num(9e9), b.nan_to_num(9e9))
    for n in range(N):
        m = min(max(int(lengths[n]), 0), R)
        assert ol[n].item() == min(m, keep)
        for l in range(L):
            for hd in range(K):
                want = okv.evict(w0[l, n, hd].tolist(), m, keep, sink, recent)
                got = kept[l, n, hd].tolist()
                assert got == want + [-1] * (keep - len(want)), (l, n, hd)
                c = len(want)
                idx = torch.tensor(want, dtype=torch.long, device="cuda")
                for new, old, axis in ((ok, k0, 0), (ov, v0, 0)):
                    assert same(new[l, n, :c, hd], old[l, n, idx, hd])
                    rest = old[l, n, c:, hd] if in_place else torch.full_like(old[l, n, c:, hd], 7.0)
                    assert same(new[l, n, c:, hd], rest), "rows behind the kept ones changed"
                assert same(ow[l, n, hd, :c], w0[l, n, hd, idx])
                assert same(ow[l, n, hd, c:], w0[l, n, hd, c:] if in_place else torch.full_like(w0[l, n, hd, c:], 7.0))


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("R,keep,sink,recent", [(1, 1, 0, 0), (2, 1, 0, 0), (2, 1, 1, 0), (2, 1, 0, 1), (17, 5, 2, 3), (17, 5, 2, 2), (17, 17, 1, 1),
                                                (100, 99, 0, 0), (816, 408, 4, 48), (1025, 3, 0, 0), (2500, 1300, 1, 100),
                                                (5000, 4999, 4, 9)])
def test_evict_sizes(kv, in_place, R, keep, sink, recent):
    w = np.random.default_rng(R).normal(size=(2, 2, 2, R)) ** 2
    check_evict(kv, w, [R, max(0, R - 3)], keep, sink, recent, K=2, in_place=in_place)


@pytest.mark.parametrize("in_place", [False, True])
def test_evict_ties_nan_infinities_and_signs(kv, in_place):
    rng = np.random.default_rng(3)
    pool = np.array([0.0, -0.0, 1.0, 1.0 + 2 ** -23, -1.0, np.inf, -np.inf, np.nan, 1e-45, -1e-45, 3e38, 1e-38], np.float32)
    w = rng.choice(pool, size=(3, 3, 1, 700))
    w[0, 0] = 2.0
    w[0, 1] = np.nan
    w[0, 2] = -np.inf
    check_evict(kv, w, [700, 700, 650], 300, 3, 20, in_place=in_place)


def test_evict_short_and_empty_caches(kv):
    w = np.random.default_rng(4).normal(size=(1, 6, 2, 50))
    for in_place in (False, True):
        check_evict(kv, w, [0, 1, 20, 21, 50, 999], 20, 4, 4, K=2, in_place=in_place)
    check_evict(kv, w, [-3, 1, 20, 21, 50, 999], 20, 10, 10, K=2)      # protected rows alone


@pytest.mark.parametrize("dtype,D", [("bf16", 8), ("bf16", 80), ("bf16", 256), ("fp32", 20), ("fp32", 256)])
def test_evict_types_and_layouts(kv, dtype, D):
    w = np.random.default_rng(5).normal(size=(2, 3, 4, 130))
    for in_place in (False, True):
        check_evict(kv, w, [130, 128, 90], 70, 1, 5, K=4, D=D, dtype=dtype, in_place=in_place)
        check_evict(kv, w, [130, 128, 90], 70, 1, 5, K=4, D=D, dtype=dtype, in_place=in_place, store=head_major)


@pytest.mark.parametrize("R", [900, 1024, 2048, 4096, 4100, 16384, 16388])
def test_evict_caches_far_from_full(kv, R):
    """Lengths that end anywhere in a cache, odd ones among them: threads of the choice past the end read nothing."""
    w = np.random.default_rng(R).normal(size=(1, 4, 1, R)).astype(np.float32) ** 2
    check_evict(kv, w, [R // 2 + 1, R // 3 + 2, 130, 101], 100, 2, 7, D=8)
    check_evict(kv, w, [R - 1, R // 3, 133, 99], 100, 2, 7, D=8, in_place=True)


def test_evict_long_cache(kv):
    w = np.random.default_rng(6).normal(size=(1, 1, 1, 70000)).astype(np.float32) ** 2
    check_evict(kv, w, [70000], 20001, 4, 500, in_place=True)
    check_evict(kv, w, [69999], 20001, 4, 500)


# ------------------------------------------------------------------ together

def test_a_decode_loop_with_eviction(kv):
    """append, attend and weigh token by token over a shared prefix, the requests' caches cut when they are full; every step
    against the oracle on the same (stored) keys and values."""
    H, K, D, B, P, R = 8, 2, 64, 4, 50, 24
    r = kv.Rope(dim=32, layout="interleaved", scaling="by_parts", factor=4.0, original=32)
    h = kv.KV(H, K, D, max_batch=B, rope=r)
    prefix = rand(1, 2, P, K, D), rand(2, 2, P, K, D)
    plen = i32([P, P - 7])
    k, v = (torch.zeros((B, R, K, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    w_prefix, w_own = torch.zeros((2, K, P), device="cuda"), torch.zeros((B, K, R), device="cuda")
    length = torch.zeros(B, dtype=torch.int32, device="cuda")
    for step in range(40):
        x = rand(100 + step, B, 1, H + 2 * K, D)
        pos = torch.full((B, 1), P + step, dtype=torch.int32, device="cuda")
        q = h.append(x[:, :, :H], x[:, :, H:H + K], x[:, :, H + K:], pos, length[:, None].contiguous(), k, v)
        length += 1
        seen = length[:, None].contiguous()
        c = dict(q=q, prefix=prefix, prefix_len=plen, own=(k, v), seen=seen)
        out, lse = h.attend(**c)
        ref, rlse, dot, mass = attend_ref(c, 1 / 8)
        tol, ltol = attend_tols(c, "bf16", ref, dot, mass, rlse)
        within(out, ref, tol, f"step {step}")
        h.weigh(q, lse, prefix=prefix[0], prefix_len=plen, own=k, seen=seen, w_prefix=w_prefix, w_own=w_own, decay=0.9,
                out_prefix=w_prefix, out_own=w_own)
        # Each KV head's weights of a step sum to its query heads, over the prefix and the own rows together.
        if step == 0:
            per_run = w_prefix.sum(-1) + torch.stack([w_own[b:b + 2, :, :1].sum((0, 2)) for b in (0, 2)])
            assert torch.allclose(per_run, torch.full_like(per_run, 2 * H / K), rtol=1e-4)
        if int(length[0]) == R:
            before = k[:, :, :].clone()
            kept = h.evict(k[None], v[None], w_own[None], length, 16, sink=2, recent=4)
            assert length.tolist() == [16] * B
            for b in range(B):
                for n in range(K):
                    assert torch.equal(k[b, :16, n], before[b, kept[0, b, n].long(), n])
    h.device_status()


@pytest.mark.usefixtures("tiles")
def test_calls_on_another_stream_and_in_a_graph(kv):
    H, K, D, B = 8, 1, 128, 12
    h = kv.KV(H, K, D, max_batch=B, rope=kv.Rope(dim=D))
    x = rand(1, B, 1, H + 2 * K, D)
    prefix = rand(2, 1, 400, K, D), rand(3, 1, 400, K, D)
    plen = i32([400])

    def state():
        return (rand(4, B, 40, K, D), rand(5, B, 40, K, D), i32([[9]] * B), i32([[9]] * B), i32([[10]] * B), torch.zeros((1, K, 400), device="cuda"),
                torch.zeros((B, K, 40), device="cuda"), i32([10] * B))

    def step(s, stream=None):
        k, v, pos, rows, seen, wp, wo, n = s
        q = h.append(x[:, :, :H], x[:, :, H:H + K], x[:, :, H + K:], pos, rows, k, v, stream=stream)
        out, lse = h.attend(q, prefix=prefix, prefix_len=plen, own=(k, v), seen=seen, stream=stream)
        h.weigh(q, lse, prefix=prefix[0], prefix_len=plen, own=k, seen=seen, w_prefix=wp, w_own=wo, out_prefix=wp, out_own=wo, stream=stream)
        kept = h.evict(k[None], v[None], wo[None], n, 6, sink=1, recent=2, stream=stream)
        return out, lse, kept, k, v, wp, wo, n

    want = step(state())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    s = state()
    torch.cuda.synchronize()
    got = step(s, side)
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    # Captured once, replayed over other lengths: lengths are read on the device.
    s = state()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step(s)
    for t, src in zip(s, state()):
        t.copy_(src)
    g.replay()
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    s2 = state()
    s2[4].fill_(8)
    s2[7].fill_(8)
    want2 = step(s2)
    want2 = [t.clone() for t in want2]
    for t, src in zip(s, state()):
        t.copy_(src)
    s[4].fill_(8)
    s[7].fill_(8)
    g.replay()
    torch.cuda.synchronize()
    for a, b in zip(want2, got):
        assert torch.equal(a, b)


def test_several_handles_at_once(kv):
    """Three handles on three streams share the SMs (tensor memory among them) and nothing else: what they give alone, bit for bit."""
    shapes = [(8, 1, 256, 48, 2, 1, 4000, 300), (32, 8, 128, 24, 1, 1, 9000, 200), (8, 1, 64, 40, 4, 2, 3000, 100)]
    runs = []
    for i, (H, K, D, B, T, G, P, R) in enumerate(shapes):
        c = clean_call(i, "bf16", H, K, D, B, T, G, P, R)
        h = kv.KV(H, K, D, max_batch=B, max_tokens=T)
        keys = dict(prefix=c["prefix"][0], prefix_len=c["prefix_len"], own=c["own"][0], seen=c["seen"])
        out, lse = h.attend(**c)
        runs.append((h, c, keys, out, lse, h.weigh(c["q"], lse, **keys), torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = []
    for _ in range(8):
        for h, c, keys, _, _, _, stream in runs:
            out, lse = h.attend(**c, stream=stream)
            got.append((out, lse, *h.weigh(c["q"], lse, **keys, stream=stream)))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        h, _, _, out, lse, w, _ = runs[i % len(runs)]
        h.device_status()
        for a, b in zip(g, (out, lse, *w)):
            assert torch.equal(a, b)


# ------------------------------------------------------------------ refusals

def test_refusals_of_the_entry_points(kv):
    import ctypes
    h = kv.KV(8, 2, 64, max_batch=4, max_tokens=4)
    L = kv.load()
    q, k = rand(1, 4, 4, 8, 64), rand(2, 4, 10, 2, 64)
    n, seen, w = i32([10] * 4), i32([[10] * 4] * 4), torch.zeros((4, 2, 10), device="cuda")
    lse, out = torch.zeros((4, 4, 8), device="cuda"), torch.empty_like(q)
    p = lambda t: t.data_ptr()
    good = dict(h=h.handle, q=p(q), qs=512, B=4, T=4, prefix=kv.cache_of(k, k), G=4, plen=p(n), own=kv.cache_of(k, k), seen=p(seen),
                out=p(out), lse=p(lse), st=None)
    bad_cache = lambda **kw: (lambda c: [setattr(c, a, b) for a, b in kw.items()] and c or c)(kv.cache_of(k, k))
    R = ctypes.byref

    def attend(**kw):
        a = {**good, **kw}
        return L.jpi_kv_attend(a["h"], a["q"], a["qs"], a["B"], a["T"], R(a["prefix"]) if a["prefix"] else None, a["G"], a["plen"],
                               R(a["own"]) if a["own"] else None, a["seen"], a["out"], a["lse"], None)

    assert attend() == 0
    common = [dict(q=None), dict(q=p(q) + 2), dict(qs=511), dict(qs=516), dict(B=0), dict(B=5), dict(T=0), dict(T=5), dict(G=3), dict(G=0),
              dict(plen=None), dict(seen=None), dict(prefix=None), dict(own=None), dict(prefix=None, plen=None, own=None, seen=None),
              dict(prefix=None, plen=None), dict(own=bad_cache(k=p(k) + 2)), dict(own=bad_cache(rows=0)), dict(own=bad_cache(row_stride=60)),
              dict(own=bad_cache(row_stride=132)), dict(own=bad_cache(cache_stride=0)), dict(own=bad_cache(head_stride=-64)),
              dict(prefix=bad_cache(k=None)), dict(prefix=bad_cache(row_stride=1 << 62))]
    for kw in common + [dict(out=None), dict(out=p(out) + 2), dict(own=bad_cache(v=None))]:
        assert attend(**kw) in (-1, -2), kw

    def weigh(**kw):
        a = {**good, "decay": 1.0, "pin": p(w), "pout": p(w), "oin": p(w), "oout": p(w), **kw}
        return L.jpi_kv_weigh(a["h"], a["q"], a["qs"], a["lse"], a["B"], a["T"], R(a["prefix"]) if a["prefix"] else None, a["G"], a["plen"],
                              R(a["own"]) if a["own"] else None, a["seen"], a["decay"], a["pin"], a["pout"], a["oin"], a["oout"], None)

    assert weigh() == 0
    for kw in common + [dict(lse=None), dict(pout=None), dict(oout=None), dict(decay=-1.0), dict(decay=math.nan), dict(decay=math.inf),
                        dict(prefix=None, plen=None, G=1)]:
        assert weigh(**kw) in (-1, -2), kw
    x, row = rand(3, 4, 4, 2, 64), i32([[0, 1, 2, 3]] * 4)
    ga = dict(q=p(q), qs=512, k=p(x), ks=128, v=p(x), vs=128, pos=p(row), row=p(row), B=4, T=4, out=p(out), cache=kv.cache_of(k, k))

    def append(**kw):
        a = {**ga, **kw}
        return L.jpi_kv_append(h.handle, a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["pos"], a["row"], a["B"], a["T"], a["out"],
                               R(a["cache"]) if a["cache"] else None, None)

    assert append() == 0
    for kw in [dict(q=None), dict(out=None), dict(k=None), dict(cache=None), dict(pos=None), dict(row=None), dict(B=5), dict(T=0), dict(qs=504),
               dict(ks=120), dict(vs=132), dict(k=p(x) + 4), dict(v=p(x) + 4), dict(out=p(out) + 8), dict(cache=bad_cache(v=None)),
               dict(q=None, out=None, k=None, v=None, cache=None), dict(k=None, cache=None)]:
        assert append(**kw) in (-1, -2), kw
    k2, w2, kept = torch.zeros_like(k), torch.zeros_like(w), torch.zeros((4, 2, 10), dtype=torch.int32, device="cuda")
    ge = dict(src=kv.cache_of(k, k2), w=p(w), n=p(n), layers=1, caches=4, keep=5, sink=1, recent=1, dst=kv.cache_of(k, k2), wo=p(w), no=p(n),
              kept=p(kept))

    def evict(**kw):
        a = {**ge, **kw}
        return L.jpi_kv_evict(h.handle, R(a["src"]), a["w"], a["n"], a["layers"], a["caches"], a["keep"], a["sink"], a["recent"], R(a["dst"]),
                              a["wo"], a["no"], a["kept"], None)

    assert evict() == 0
    half = kv.cache_of(k[:, :5], k2[:, :5])
    for kw in [dict(w=None), dict(n=None), dict(wo=None), dict(no=None), dict(kept=None), dict(keep=0), dict(keep=11), dict(sink=-1), dict(recent=-1),
               dict(sink=3, recent=3), dict(layers=0), dict(caches=0), dict(caches=70000), dict(dst=half), dict(wo=p(w2)),
               dict(dst=kv.cache_of(k2, k)), dict(dst=kv.cache_of(k[:, :4], k2[:, :4]), wo=p(w2))]:
        assert evict(**kw) in (-1, -2), kw
    torch.cuda.synchronize()


def test_the_binding_checks_what_the_c_abi_cannot_see(kv):
    h = kv.KV(8, 2, 64, max_batch=4, max_tokens=4)
    q, k = rand(1, 4, 4, 8, 64), rand(2, 4, 10, 2, 64)
    n, seen = i32([10]), i32([[10] * 4] * 4)
    for kw in [dict(q=q.float()), dict(q=q.cpu()), dict(q=q[:, :, :7]), dict(own=(k[:2], k[:2])), dict(own=(k, k.float())), dict(own=(k, head_major(k))),
               dict(seen=seen.long()), dict(seen=seen[:, :2]), dict(seen=None), dict(own=(k[..., :32], k[..., :32])),
               dict(out=torch.empty_like(q).transpose(0, 1)), dict(lse=torch.empty((4, 4, 7), device="cuda")), dict(own=(k[..., None, :], k))]:
        with pytest.raises(ValueError):
            h.attend(**{**dict(q=q, own=(k, k), seen=seen), **kw})
    with pytest.raises(ValueError):
        h.evict(k[None], k[None], torch.zeros((1, 4, 2, 9), device="cuda"), i32([10] * 4), 5)
    with pytest.raises(ValueError):
        h.evict(k[None], k[None], torch.zeros((1, 4, 2, 10), device="cuda"), i32([10] * 4), 5, out_k=k[None])
    from paper_2607_12659_gb300.jpi import JpiError
    with pytest.raises(JpiError):
        h.attend(rand(1, 5, 1, 8, 64), own=(rand(1, 5, 3, 2, 64),) * 2, seen=i32([[1]] * 5))


def test_the_binding_takes_rows_of_any_stride_and_refuses_what_is_no_cache(kv):
    h = kv.KV(8, 2, 64, max_batch=4, max_tokens=4)
    q, k = rand(1, 4, 4, 8, 64), rand(2, 4, 10, 2, 64)
    seen = i32([[10] * 4] * 4)
    want, lse = h.attend(q, own=(k, k), seen=seen)
    flat = rand(3, 4 * 4 * 8 * 64 + 1)
    off = flat[1:].view(4, 4, 8, 64)      # contiguous, two bytes past a 16-byte boundary
    off.copy_(q)
    rows = rand(4, 4, 4, 11, 64)[:, :, 2:10]
    rows.copy_(q)
    cols = rand(5, 4, 4, 8, 65)[..., :64]
    cols.copy_(q)
    for x in (off, rows, cols, q.transpose(0, 1).contiguous().transpose(0, 1), q.transpose(1, 2).contiguous().transpose(1, 2)):
        got, lse2 = h.attend(x, own=[k, k], seen=seen)      # a list is a pair too
        assert torch.equal(got, want) and torch.equal(lse2, lse)
    for kw in [dict(own=k), dict(own=(k,)), dict(own=(k, None)), dict(own=(k, 3)), dict(q=None, out=q, lse=lse), dict(seen=[[10] * 4] * 4)]:
        with pytest.raises((TypeError, ValueError)):
            h.attend(**{**dict(q=q, own=(k, k), seen=seen), **kw})
    w, n = torch.zeros((1, 4, 2, 10), device="cuda"), i32([10] * 4)
    for keep in (2 ** 40, 2 ** 31 - 1, -1, 11, 1.5):
        with pytest.raises((TypeError, ValueError)):
            h.evict(k[None], k[None], w, n, keep)
    with pytest.raises(ValueError):
        h.evict(k, k, w, n, 5)
    sparse = torch.sparse_coo_tensor(torch.zeros((4, 1), dtype=torch.int64, device="cuda"), torch.ones(1, device="cuda").bfloat16(), q.shape)
    with pytest.raises(ValueError):
        h.attend(sparse, own=(k, k), seen=seen)
    h.close()
    from paper_2607_12659_gb300.jpi import JpiError
    with pytest.raises(JpiError):
        h.attend(q, own=(k, k), seen=seen)


# ------------------------------------------------------------------ NaN and infinities that a query sees

def clean_call(seed, dtype, H, K, D, B, T, G, P, R, std=2.0):
    """Inputs of finite numbers; the last query of the first and of the last request sees every row, and rows that no query
    sees hold NaN."""
    c = make_call(seed, dtype, H, K, D, B, T, G, P, R, mask="any", std=std)
    if P:
        c["prefix_len"].fill_(P - 1)
        c["prefix"] = tuple(rand(seed + i, G, P, K, D, dtype=dtype) for i in (11, 12))
        for t in c["prefix"]:
            t[:, P - 1] = float("nan")
    if R:
        c["seen"][0, -1] = c["seen"][-1, -1] = R
        c["own"] = tuple(rand(seed + i, B, R, K, D, dtype=dtype) for i in (13, 14))
        for b in range(B):
            for t in c["own"]:
                t[b, int(c["seen"][b].max()):] = float("nan")
    return c


def check_attend_special(kv, dtype, c, what):
    """Attention over infinities and NaN: what the formula gives, NaN where it gives NaN."""
    B, T, H, D = c["q"].shape
    K = (c["prefix"] or c["own"])[0].shape[2]
    h = kv.KV(H, K, D, max_batch=B, max_tokens=T, precision=dtype)
    out, lse = h.attend(**c)
    h.device_status()
    with np.errstate(invalid="ignore"):
        ref, rlse, dot, mass = attend_ref(c, 1 / math.sqrt(D))
    assert not np.isfinite(ref).all(), "the case has nothing special"
    tol, ltol = attend_tols(c, dtype, *(np.where(np.isfinite(a), a, 0.0) for a in (ref, dot, mass)), rlse)
    for name, got, want, bound in (("out", out, ref, tol), ("lse", lse, rlse, ltol)):
        assert np.array_equal(np.isnan(np64(got)), np.isnan(want)), f"{what}: NaN of {name}"
        # (an infinite element has to be equal)
        within(got.nan_to_num(0.0, math.inf, -math.inf), np.where(np.isnan(want), 0.0, want), np.where(np.isfinite(want), bound, 0.0), f"{what}: {name}")
    return lse


# One part and several, few query rows and many, each side alone and both.
SPECIAL = [("fp32", 4, 2, 64, 3, 2, 1, 70, 20), ("fp32", 2, 1, 64, 1, 1, 1, 30, 0), ("fp32", 8, 1, 256, 2, 9, 1, 333, 40),
           ("fp32", 8, 2, 128, 2, 40, 1, 0, 64), ("bf16", 4, 2, 64, 3, 2, 1, 70, 20), ("bf16", 2, 1, 64, 1, 1, 1, 9, 0),
           ("bf16", 8, 1, 256, 2, 3, 1, 900, 40), ("bf16", 8, 2, 96, 2, 40, 1, 0, 150), ("bf16", 16, 2, 128, 8, 4, 2, 300, 130),
           ("bf16", 8, 1, 256, 4, 51, 2, 200, 51)]
NAN_KINDS = ["a query", "a key", "a key of the last rows", "the first keys", "all keys of a side"]


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("kind", NAN_KINDS)
@pytest.mark.parametrize("dtype,H,K,D,B,T,G,P,R", SPECIAL)
def test_attend_a_nan_query_or_key_gives_nan(kv, dtype, H, K, D, B, T, G, P, R, kind):
    """A NaN score is no missing key: the rows that have one are NaN and so is their lse, however the call is split, and the
    weights that come of them."""
    c = clean_call(H + D, dtype, H, K, D, B, T, G, P, R)
    k = (c["prefix"] or c["own"])[0]
    if kind == "a query":
        c["q"][-1, -1, -1, 3] = float("nan")
    elif kind == "a key":
        k[0, 1, 0, 2] = float("nan")
    elif kind == "a key of the last rows":
        (c["own"] or c["prefix"])[0][-1, (R or P - 1) - 1, -1, 5] = float("nan")
    elif kind == "the first keys":
        k[0, :35] = float("nan")
    else:
        k[:] = float("nan")
    lse = check_attend_special(kv, dtype, c, kind)
    keys = dict(prefix=(c["prefix"] or [None])[0], prefix_len=c["prefix_len"], own=(c["own"] or [None])[0], seen=c["seen"])
    got = kv.KV(H, K, D, max_batch=B, max_tokens=T, precision=dtype).weigh(c["q"], lse, **keys)
    host = [None if t is None else t.cpu().numpy() if t.dtype is torch.int32 else np64(t) for t in keys.values()]
    with np.errstate(invalid="ignore"):
        ref = okv.weigh(np64(c["q"]), np64(lse), *host, 1 / math.sqrt(D), 1.0, None, None, *(None if g is None else np.zeros(g.shape) for g in got))
    for g, (y, _) in zip(got, ref):
        assert g is None or np.array_equal(np.isnan(np64(g)), np.isnan(y)), "NaN of the weights"


@pytest.mark.usefixtures("tiles")
@pytest.mark.parametrize("dtype,H,K,D,B,T,G,P,R", SPECIAL)
def test_attend_an_infinite_value_that_a_query_sees_stays_infinite(kv, dtype, H, K, D, B, T, G, P, R):
    """An infinite value of positive weight makes its element that infinity, NaN only where both signs meet; queries that do
    not see it keep what they have."""
    n = R or P - 1
    for at in (0, n // 2, n - 1):
        c = clean_call(D + at, dtype, H, K, D, B, T, G, P, R, std=1.0)
        v = (c["own"] or c["prefix"])[1]
        v[0, at, 0, 3], v[0, at, 0, 4] = float("inf"), -float("inf")
        v[0, 0, 0, 6], v[0, n - 1, 0, 6] = float("inf"), -float("inf")
        if P and R:
            c["prefix"][1][0, 1, -1, 7], v[0, at, -1, 7] = float("inf"), -float("inf")
        check_attend_special(kv, dtype, c, f"row {at}")
