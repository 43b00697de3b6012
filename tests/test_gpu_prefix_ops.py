"""The expert's calls on a stored prefix (jpi_share_prefix, jpi_weigh_prefix, jpi_evict_prefix, jpi_append_prefix,
jpi_commit_prefix_at) against the fp64 oracle: several requests over one prefix, the weights its keys receive,
denoises over what eviction leaves and over appended tokens. Tolerances of the denoise are the expert's own."""

import contextlib

import numpy as np
import pytest

import oracle
import oracle.expert as oe
from synth import PI05, TINY, make_correction, make_requests, make_weights
from tests.gpu_util import SMALL_BF16, assert_close, gpu_denoise, lib, make_expert, oracle_denoise, to_dev_kv

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.fail("the gpu tests need a CUDA device")
    torch.cuda.set_device(0)
    lib()


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def shared(cfg, seed, groups, share, P, C):
    """Requests of which each run of `share` has the prefix of its first."""
    r = make_requests(cfg, seed, groups * share, P, C)
    first = np.repeat(np.arange(groups) * share, share)
    return {**r, "prefix_k": r["prefix_k"][:, first], "prefix_v": r["prefix_v"][:, first]}, np.arange(groups) * share


CASES = [(TINY, 1, 1, 3, 40, 6), (TINY, 2, 2, 2, 33, 8), (SMALL_BF16, 3, 1, 2, 50, 7), (SMALL_BF16, 4, 2, 3, 100, 20),
         (SMALL_BF16, 5, 1, 12, 65, 33)]


@pytest.mark.parametrize("cfg,seed,groups,share,P,C", CASES)
def test_several_chunks_from_one_prefix(cfg, seed, groups, share, P, C):
    w = make_weights(cfg, 0)
    B = groups * share
    r, slots = shared(cfg, seed, groups, share, P, C)
    corr = make_correction(cfg, seed, B, 3)
    ex = make_expert(cfg, w, max_batch=B, max_prefix=P + 7, max_chunk=C, max_steps=3)
    try:
        k, v = to_dev_kv(r, cfg)
        ex.share_prefix(share)
        ex.set_prefix_kv(k[:, slots], v[:, slots])
        state, noise = dev(r["state"]), dev(r["noise"])
        got = ex.denoise(state, noise, 3)
        ex.device_status()
        ref = oracle_denoise(cfg, w, r, 3)
        assert_close(got.cpu().numpy(), ref, cfg, f"shared prefix {groups} x {share}")
        assert torch.equal(got, ex.denoise(state, noise, 3)), "two replays differ"
        ex.set_correction(dev(corr))
        got = ex.denoise(state, noise, 2)
        ref = oracle.denoise_batch(r["noise"], r["state"], 2, r["prefix_k"], r["prefix_v"], w, cfg, corr=corr)
        assert_close(got.cpu().numpy(), ref, cfg, "shared prefix with items")
        ex.set_correction(None)
        # Back to one request a prefix: what ran before gives what it gave.
        ex.share_prefix(1)
        got = gpu_denoise(ex, cfg, r, 3)
        assert_close(got, oracle_denoise(cfg, w, r, 3), cfg, "unshared again")
    finally:
        ex.close()


def test_shared_prefix_at_pi05_sizes():
    w = make_weights(PI05, 0)
    r, slots = shared(PI05, 9, 2, 4, 816, 50)
    ex = make_expert(PI05, w, max_batch=8, max_prefix=816, max_chunk=50, max_steps=10)
    try:
        k, v = to_dev_kv(r, PI05)
        ex.share_prefix(4)
        ex.set_prefix_kv(k[:, slots], v[:, slots])
        got = ex.denoise(dev(r["state"]), dev(r["noise"]), 10)
        ex.device_status()
        some = [0, 5]
        assert_close(got.cpu().numpy()[some], oracle_denoise(PI05, w, r, 10, some), PI05, "pi0.5 shared 2 x 4")
    finally:
        ex.close()


def oracle_weights(r, w, cfg, t, groups, share, monkeypatch):
    """[L][groups][P] summed attention weights of one oracle evaluation."""
    P, L = r["prefix_k"].shape[2], cfg.n_layers
    out = np.zeros((L, groups, P))
    real = oe.attention
    calls = []

    def spy(q, K, V, visible):
        S, H, D = q.shape
        s = np.einsum("shd,jd->shj", q, K) / np.sqrt(D)
        s = np.where(visible[:, None], s, -np.inf)
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        n = len(calls)
        out[n % L, n // L // share] += p[:, :, :P].sum((0, 1))
        calls.append(0)
        return real(q, K, V, visible)

    monkeypatch.setattr(oe, "attention", spy)
    oracle.forward_batch(r["noise"], r["state"], t, r["prefix_k"], r["prefix_v"], w, cfg)
    monkeypatch.undo()
    return out


@pytest.mark.parametrize("cfg,seed,groups,share,P,C", [(TINY, 1, 2, 1, 40, 6), (TINY, 2, 1, 3, 64, 8), (SMALL_BF16, 3, 2, 2, 50, 9),
                                                       (SMALL_BF16, 4, 1, 9, 130, 30)])
def test_weights_of_the_prefix_and_a_denoise_over_what_they_leave(cfg, seed, groups, share, P, C, monkeypatch):
    w = make_weights(cfg, 0)
    B = groups * share
    r, slots = shared(cfg, seed, groups, share, P, C)
    ex = make_expert(cfg, w, max_batch=B, max_prefix=P, max_chunk=C, max_steps=2)
    try:
        k, v = to_dev_kv(r, cfg)
        ex.share_prefix(share)
        ex.set_prefix_kv(k[:, slots], v[:, slots])
        state, noise = dev(r["state"]), dev(r["noise"])
        weights = torch.full((cfg.n_layers, groups, P), float("nan"), device="cuda")
        ex.weigh_prefix(state, noise, 0.25, weights, decay=0.0)
        once = weights.clone()
        ex.weigh_prefix(state, noise, 0.25, weights, decay=0.5)
        ex.device_status()
        ref = oracle_weights(r, w, cfg, 0.25, groups, share, monkeypatch)
        rel = np.abs(once.cpu().numpy() - ref).max() / ref.max()
        # bf16: queries and keys rounded to 2^-8 of themselves move a score of magnitude s by about 2^-7 s
        assert rel < (2e-2 if cfg.precision == "bf16" else 1e-4), rel
        assert torch.allclose(weights, 1.5 * once, rtol=1e-6)
        # Half of the tokens stay, layer by layer; a denoise over them, positions as before.
        keep = P // 2
        order = weights.clone()
        kept = ex.evict_prefix(weights, keep, sink=2, recent=5)
        want = torch.empty_like(kept)
        for l in range(cfg.n_layers):
            for g in range(groups):
                best = torch.argsort(-order[l, g, 2:P - 5], stable=True)[:keep - 7] + 2
                want[l, g] = torch.cat([torch.arange(2, device="cuda"), best.sort()[0], torch.arange(P - 5, P, device="cuda")])
        assert torch.equal(kept, want)
        flat = weights.flatten(1)
        got = ex.denoise(state, noise, 2)
        ex.device_status()
        idx = kept.cpu().numpy().repeat(share, axis=1)
        cut = {**r, **{n: np.take_along_axis(r[n], idx[..., None], axis=2) for n in ("prefix_k", "prefix_v")}}
        real = oe.rope
        monkeypatch.setattr(oe, "rope", lambda x, pos, base: real(x, pos + (P - keep), base))
        assert_close(got.cpu().numpy(), oracle_denoise(cfg, w, cut, 2), cfg, "denoise over the kept tokens")
        monkeypatch.undo()
        # The next observation starts afresh.
        ex.set_prefix_kv(k[:, slots], v[:, slots])
        assert_close(ex.denoise(state, noise, 2).cpu().numpy(), oracle_denoise(cfg, w, r, 2), cfg, "a new prefix")
    finally:
        ex.close()


@pytest.mark.parametrize("cfg", [TINY, SMALL_BF16])
def test_appended_tokens_are_prefix_tokens(cfg):
    w = make_weights(cfg, 0)
    P, T, C, B = 40, 9, 6, 2
    r = make_requests(cfg, 6, B, P + T, C)
    ex = make_expert(cfg, w, max_batch=B, max_prefix=P + T, max_chunk=C, max_steps=2)
    try:
        k, v = to_dev_kv(r, cfg)
        ex.set_prefix_kv(k[:, :, :P], v[:, :, :P])
        # Keys without position code whose coding gives a prefix that the oracle can be given.
        raw = k[:, :, P:]
        ex.append_prefix(raw, v[:, :, P:])
        got = ex.denoise(dev(r["state"]), dev(r["noise"]), 2)
        ex.device_status()
        coded = oe.rope(raw.double().cpu().numpy().transpose(2, 0, 1, 3), np.arange(P, P + T), cfg.rope_base)
        full = {**r, "prefix_k": np.concatenate([r["prefix_k"][:, :, :P], coded.transpose(1, 2, 0, 3)], axis=2)}
        assert_close(got.cpu().numpy(), oracle_denoise(cfg, w, full, 2), cfg, "appended tokens")
    finally:
        ex.close()


def test_commit_at_a_position():
    cfg = TINY
    w = make_weights(cfg, 0)
    r = make_requests(cfg, 8, 1, 30, 5)
    ex = make_expert(cfg, w, max_batch=1, max_prefix=64, max_chunk=5, max_steps=2)
    from paper_2607_12659_gb300 import jpi
    try:
        k, v = to_dev_kv(r, cfg)
        ex.set_prefix_kv(k, v)
        jpi.jpi_commit_prefix_at(ex.handle, 1, 30, 41)
        got = ex.denoise(dev(r["state"]), dev(r["noise"]), 2).cpu().numpy()
        real = oe.rope
        try:
            oe.rope = lambda x, pos, base: real(x, pos + 11, base)
            ref = oracle_denoise(cfg, w, r, 2)
        finally:
            oe.rope = real
        assert_close(got, ref, cfg, "positions from 41")
        for bad in ((1, 30, 29), (1, 30, 65), (2, 30, 30)):
            with pytest.raises(jpi.JpiError):
                jpi.jpi_commit_prefix_at(ex.handle, *bad)
    finally:
        ex.close()


def test_refusals(monkeypatch):
    from paper_2607_12659_gb300 import jpi
    w = make_weights(TINY, 0)
    r = make_requests(TINY, 8, 2, 30, 5)
    ex = make_expert(TINY, w, max_batch=4, max_prefix=32, max_chunk=5, max_steps=2)
    weights = torch.zeros((TINY.n_layers, 2, 30), device="cuda")
    state, noise = dev(r["state"]), dev(r["noise"])
    k, v = to_dev_kv(r, TINY)
    try:
        with pytest.raises(jpi.JpiError):
            ex.evict_prefix(weights, 5)                    # no prefix yet
        with pytest.raises(jpi.JpiError):
            ex.append_prefix(k[:, :, :1], v[:, :, :1])
        ex.set_prefix_kv(k, v)
        for bad in (0, -1, 5):
            with pytest.raises(jpi.JpiError):
                ex.share_prefix(bad)
        for bad in (dict(keep=0), dict(keep=31), dict(keep=5, sink=3, recent=3), dict(keep=5, sink=-1)):
            with pytest.raises(jpi.JpiError):
                ex.evict_prefix(weights, **bad)
        with pytest.raises(jpi.JpiError):
            ex.append_prefix(k[:, :, :3], v[:, :, :3])     # 30 + 3 > 32
        with pytest.raises(jpi.JpiError):
            ex.weigh_prefix(state, noise, 0.0, weights, decay=-1.0)
        ex.share_prefix(2)
        with pytest.raises(jpi.JpiError):
            ex.denoise(state, noise, 1)                    # two prefixes, two requests each: four are wanted
        ex.share_prefix(1)
        assert ex.prefix_shape() == (2, 30, 30)
        for bad in (weights[:, :1], weights[..., :29].contiguous(), weights[:1], weights.double(), weights.cpu(), weights.transpose(0, 1)):
            with pytest.raises(ValueError):                # too small for the stored prefix, or no block of fp32
                ex.weigh_prefix(state, noise, 0.0, bad)
            with pytest.raises(ValueError):
                ex.evict_prefix(bad, 5)
        for bad in (k[:, :1, :1], k[:1, :, :1], k[:, :, :1, :-8], k[:, :, :1].double(), k[:, :, :1].cpu()):
            with pytest.raises(ValueError):
                ex.append_prefix(bad, bad)
        assert_close(gpu_denoise(ex, TINY, r, 2), oracle_denoise(TINY, w, r, 2), TINY, "after the refusals")
    finally:
        ex.close()
    monkeypatch.setenv("JPI_BATCH_INVARIANT", "1")
    ex = make_expert(TINY, w, max_batch=4, max_prefix=32, max_chunk=5, max_steps=2)
    try:
        ex.set_prefix_kv(k, v)
        with pytest.raises(jpi.JpiError):
            ex.share_prefix(2)
    finally:
        ex.close()


@pytest.mark.parametrize("cfg,share", [(TINY, 1), (TINY, 3), (SMALL_BF16, 1), (SMALL_BF16, 2)])
def test_tokens_appended_to_what_eviction_left(cfg, share, monkeypatch):
    """The rows that eviction frees take new tokens, at the positions that follow, past max_prefix too."""
    w = make_weights(cfg, 0)
    P, T, C, G = 40, 17, 6, 2
    B, L = G * share, cfg.n_layers
    r, slots = shared(cfg, 6, G, share, P, C)
    ex = make_expert(cfg, w, max_batch=B, max_prefix=P, max_chunk=C, max_steps=2)
    rng = np.random.default_rng(share)
    state, noise = dev(r["state"]), dev(r["noise"])
    real = oe.rope
    try:
        k, v = to_dev_kv(r, cfg)
        ex.share_prefix(share)
        ex.set_prefix_kv(k[:, slots], v[:, slots])
        keys, values = (a[:, slots].astype(np.float64) for a in (r["prefix_k"], r["prefix_v"]))
        end = P
        for turn in range(3):
            weights = dev(rng.random((L, G, keys.shape[2]), np.float32))
            before, keep = weights.clone(), 20 + (turn > 0)      # (the last turn: the same shapes at later positions)
            kept = ex.evict_prefix(weights, keep, sink=1, recent=3)
            assert ex.prefix_shape() == (G, keep, end)
            moved = torch.gather(before, 2, kept.long())
            assert torch.equal(weights[..., :keep], moved) and torch.equal(weights[..., keep:], before[..., keep:])
            idx = kept.cpu().numpy()[..., None]
            keys, values = (np.take_along_axis(a, idx, axis=2) for a in (keys, values))
            new_k, new_v = (dev(rng.standard_normal((L, G, T, cfg.head_dim)).astype(np.float32)).to(k.dtype) for _ in range(2))
            with pytest.raises(lib().JpiError):
                ex.append_prefix(*(torch.cat([t, t], dim=2) for t in (new_k, new_v)))      # more rows than are free
            ex.append_prefix(new_k, new_v)
            coded = real(new_k.double().cpu().numpy().transpose(2, 0, 1, 3), np.arange(end, end + T), cfg.rope_base).transpose(1, 2, 0, 3)
            if cfg.precision == "bf16":     # as the store holds them
                coded = torch.from_numpy(coded).bfloat16().double().numpy()
            keys, values = np.concatenate([keys, coded], axis=2), np.concatenate([values, new_v.double().cpu().numpy()], axis=2)
            end += T
            assert ex.prefix_shape() == (G, keep + T, end) and end > P
            run = np.repeat(np.arange(G), share)
            now = {**r, "prefix_k": keys[:, run], "prefix_v": values[:, run]}
            for steps in (2, 1):
                got = ex.denoise(state, noise, steps)
                ex.device_status()
                monkeypatch.setattr(oe, "rope", lambda x, pos, base: real(x, pos + (end - keep - T), base))
                ref = oracle_denoise(cfg, w, now, steps)
                monkeypatch.undo()
                assert_close(got.cpu().numpy(), ref, cfg, f"turn {turn}, {steps} steps")
        # The next observation starts afresh.
        ex.set_prefix_kv(k[:, slots], v[:, slots])
        assert ex.prefix_shape() == (G, P, P)
        assert_close(ex.denoise(state, noise, 2).cpu().numpy(), oracle_denoise(cfg, w, r, 2), cfg, "a new prefix")
    finally:
        ex.close()


def test_weights_go_on_after_an_eviction():
    """The moved weights are the first `keep` of each row: a contiguous copy of them is the cut prefix's."""
    cfg, P, B, C, keep = SMALL_BF16, 50, 2, 6, 30
    r = make_requests(cfg, 9, B, P, C)
    ex = make_expert(cfg, make_weights(cfg, 0), max_batch=B, max_prefix=P, max_chunk=C, max_steps=1)
    try:
        ex.set_prefix_kv(*to_dev_kv(r, cfg))
        state, noise = dev(r["state"]), dev(r["noise"])
        w = torch.zeros((cfg.n_layers, B, P), device="cuda")
        ex.weigh_prefix(state, noise, 0.5, w)
        ex.evict_prefix(w, keep, sink=1, recent=2)
        with pytest.raises(ValueError):
            ex.weigh_prefix(state, noise, 0.5, w)
        moved = w[..., :keep].contiguous()
        once = ex.weigh_prefix(state, noise, 0.5, torch.zeros_like(moved))
        both = ex.weigh_prefix(state, noise, 0.5, moved.clone())
        # one product and one sum, rounded once or twice: an eps of the sum
        assert ((both - (moved + once)).abs() <= 2.0 ** -23 * both).all() and once.sum() > 0
        kept = ex.evict_prefix(both, keep - 7)
        assert torch.equal(kept, torch.topk(moved + once, keep - 7).indices.sort(-1).values.int())
        ex.device_status()
    finally:
        ex.close()


def test_the_c_entry_points_on_the_stored_prefix():
    """The operators on the expert's own store, by its addresses (jpi_prefix_kv_ptr): what they give on copies of it."""
    from paper_2607_12659_gb300 import jpi, kv
    cfg, P, B, T, layer = SMALL_BF16, 40, 2, 5, 1
    H, D = cfg.n_heads, cfg.head_dim
    r = make_requests(cfg, 10, B, P, 4)
    ex = make_expert(cfg, make_weights(cfg, 0), max_batch=B, max_prefix=P, max_chunk=4, max_steps=1)
    h = kv.KV(H, 1, D, max_batch=B, max_tokens=T, rope=kv.Rope(dim=D))
    g = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    try:
        k, v = to_dev_kv(r, cfg)
        ex.set_prefix_kv(k, v)
        ck, cv = (t[layer][:, :, None].clone() for t in (k, v))      # [B][P][1][D]
        pk, pv, stride = jpi.jpi_prefix_kv_ptr(ex.handle, layer)
        store = kv.jpi_kv_cache(pk, pv, stride, D, D, 0, P)
        q, nk, nv = new(B, T, H, D), new(B, T, 1, D), new(B, T, 1, D)
        pos, rows = i32([[7 + t for t in range(T)]] * B), i32([[P - T + t for t in range(T)]] * B)
        coded = torch.empty_like(q)
        kv.jpi_kv_append(h.handle, q, H * D, nk, D, nv, D, pos, rows, B, T, coded, store)
        assert torch.equal(coded, h.append(q, nk, nv, pos, rows, ck, cv))
        length, seen = i32([P] * B), i32([[P - T + 1 + t for t in range(T)]] * B)
        for side in (dict(prefix=store, groups=B, prefix_len=length, own=None, seen=None), dict(prefix=None, groups=1, prefix_len=None, own=store, seen=seen)):
            out, lse = torch.empty_like(q), torch.empty((B, T, H), device="cuda")
            kv.jpi_kv_attend(h.handle, coded, H * D, B, T, out=out, lse=lse, **side)
            name = "prefix" if side["prefix"] else "own"
            lens = dict(prefix_len=length) if side["prefix"] else dict(seen=seen)
            want = h.attend(coded, **{name: (ck, cv)}, **lens)
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
            w = torch.zeros((B, 1, P), device="cuda")
            into = dict(prefix_in=None, prefix_out=None, own_in=None, own_out=None)
            into[name + "_out"] = w
            kv.jpi_kv_weigh(h.handle, coded, H * D, lse, B, T, decay=1.0, **side, **into)
            assert torch.equal(w, [x for x in h.weigh(coded, lse, **{name: ck}, **lens) if x is not None][0])
        kept, cut, n = torch.empty((1, B, 1, 25), dtype=torch.int32, device="cuda"), w.clone(), length.clone()
        kv.jpi_kv_evict(h.handle, store, cut, n, 1, B, 25, 2, 3, store, cut, n, kept)
        assert torch.equal(kept, h.evict(ck[None], cv[None], w[None], length, 25, 2, 3))
        assert torch.equal(cut, w) and torch.equal(n, length) and n.tolist() == [25] * B
        out, lse = torch.empty_like(q), torch.empty((B, T, H), device="cuda")
        kv.jpi_kv_attend(h.handle, coded, H * D, B, T, store, B, n, None, None, out, lse)
        assert torch.equal(out, h.attend(coded, prefix=(ck, cv), prefix_len=n)[0])
        h.device_status()
    finally:
        ex.close()


@pytest.mark.parametrize("cfg,groups,share,P,C", [(TINY, 1, 3, 40, 6), (SMALL_BF16, 2, 2, 50, 7), (SMALL_BF16, 1, 12, 300, 33)])
def test_a_broken_request_shows_and_stays_alone(cfg, groups, share, P, C):
    """NaN in one request's state: its actions are NaN (its own state token is a key that they see), the other requests of the
    prefix get what they get without it, and the weights of that prefix's keys are NaN."""
    B = groups * share
    r, slots = shared(cfg, 11, groups, share, P, C)
    ex = make_expert(cfg, make_weights(cfg, 0), max_batch=B, max_prefix=P, max_chunk=C, max_steps=2)
    try:
        k, v = to_dev_kv(r, cfg)
        ex.share_prefix(share)
        ex.set_prefix_kv(k[:, slots], v[:, slots])
        state, noise = dev(r["state"]), dev(r["noise"])
        want = ex.denoise(state, noise, 2).clone()
        broken = state.clone()
        broken[-1, 0] = float("nan")
        got = ex.denoise(broken, noise, 2)
        assert want.isfinite().all() and got[-1].isnan().all() and torch.equal(got[:-1], want[:-1])
        w = ex.weigh_prefix(broken, noise, 0.5, torch.zeros((cfg.n_layers, groups, P), device="cuda"))
        assert w[:, -1].isnan().all() and w[:, :-1].isfinite().all()
        # The bf16 projections exchange partial sums as fp16 and report that these did not fit (code 4; no wait gave up).
        with pytest.raises(lib().JpiError, match="code 4") if cfg.precision == "bf16" else contextlib.nullcontext():
            ex.device_status()
        assert torch.equal(ex.denoise(state, noise, 2), want)
        ex.device_status()
    finally:
        ex.close()
