"""CPU oracle of the KV-cache operators (fp64, numpy), request by request and head by head.

TEST INFRASTRUCTURE ONLY. Only the tests may import it; the library never does, and it shares no
code with the CUDA path. The operators are defined in include/jpi_kv.h; the paper has no
counterpart beyond the per-layer KV cache itself (App. A).
"""

from __future__ import annotations

import math

import numpy as np

F64 = np.float64


def rope_theta(r) -> np.ndarray:
    """Angle per position of every pair of a rotary coding with the attributes of kv.Rope."""
    out = []
    for i in range(r.dim // 2):
        base = r.base
        if r.scaling == "ntk":
            base = r.base * r.factor ** (r.dim / (r.dim - 2))
        th = base ** (-2.0 * i / r.dim)
        if r.scaling == "linear":
            th = th / r.factor
        if r.scaling == "by_parts":
            turns = r.original * th / (2 * math.pi)
            g = min(1.0, max(0.0, (turns - r.low) / (r.high - r.low)))
            th = (1 - g) * th / r.factor + g * th
        out.append(th)
    return np.array(out, F64)


def rope(x: np.ndarray, position: int, r) -> np.ndarray:
    """One head's elements x [D] at a position."""
    if r is None:
        return x.astype(F64)
    y = x.astype(F64).copy()
    for i, th in enumerate(rope_theta(r)):
        a, b = (i, i + r.dim // 2) if r.layout == "half" else (2 * i, 2 * i + 1)
        c, s = math.cos(position * th) * r.mscale, math.sin(position * th) * r.mscale
        y[a] = float(x[a]) * c - float(x[b]) * s
        y[b] = float(x[b]) * c + float(x[a]) * s
    return y


def append(q, k, v, positions, rows, cache_k, cache_v, r):
    """(q_out, K, V) after the call; q_out rows of padding are NaN (not written)."""
    B, T = positions.shape
    K, V = cache_k.astype(F64).copy(), cache_v.astype(F64).copy()
    q_out = np.full(q.shape, np.nan)
    for b in range(B):
        for t in range(T):
            if not 0 <= rows[b, t] < K.shape[1]:
                continue
            for h in range(q.shape[2]):
                q_out[b, t, h] = rope(q[b, t, h], int(positions[b, t]), r)
            for h in range(k.shape[2]):
                K[b, rows[b, t], h] = rope(k[b, t, h], int(positions[b, t]), r)
                V[b, rows[b, t], h] = v[b, t, h]
    return q_out, K, V


def _keys(b, t, prefix, prefix_len, own, seen, batch, which):
    """Rows (which: 0 keys, 1 values) that token t of request b sees, [n][K][D], fp64."""
    parts = []
    if prefix is not None:
        g = b // (batch // len(prefix_len))
        parts.append(prefix[which][g, :min(max(int(prefix_len[g]), 0), prefix[which].shape[1])])
    if own is not None:
        parts.append(own[which][b, :min(max(int(seen[b, t]), 0), own[which].shape[1])])
    return np.concatenate(parts).astype(F64)


def attend(q, prefix, prefix_len, own, seen, scale):
    """(out [B][T][H][D], lse [B][T][H], bound): `bound` holds per (b, t, h) the largest sum of |q_d k_d| over the
    keys, and per output element the sum of p |v|, for error bounds."""
    B, T, H, D = q.shape
    K = (prefix or own)[0].shape[2]
    out, lse = np.zeros(q.shape, F64), np.full((B, T, H), -np.inf)
    dot, mass = np.zeros((B, T, H)), np.zeros(q.shape, F64)
    for b in range(B):
        for t in range(T):
            k, v = (_keys(b, t, prefix, prefix_len, own, seen, B, w) for w in (0, 1))
            if len(k) == 0:
                continue
            for h in range(H):
                x, kk, vv = q[b, t, h].astype(F64), k[:, h // (H // K)], v[:, h // (H // K)]
                s = scale * (kk @ x)
                m = s.max()
                p = np.exp(s - m)
                lse[b, t, h] = m + math.log(p.sum())
                p /= p.sum()
                out[b, t, h] = p @ vv
                dot[b, t, h] = scale * (np.abs(kk) @ np.abs(x)).max()
                mass[b, t, h] = p @ np.abs(vv)
    return out, lse, dot, mass


def weigh(q, lse, prefix, prefix_len, own, seen, scale, decay, w_prefix, w_own, out_prefix, out_own):
    """(prefix weights, own weights, their error scales) after the call; prefix and own are keys."""
    B, T, H, D = q.shape
    K = (prefix if prefix is not None else own).shape[2]
    live_p = [min(max(int(n), 0), prefix.shape[1]) for n in prefix_len] if prefix is not None else []
    live_o = [min(max(int(seen[b].max()), 0), own.shape[1]) for b in range(B)] if own is not None else []
    res = []
    for w, out, live in ((w_prefix, out_prefix, live_p), (w_own, out_own, live_o)):
        if out is None:
            res.append((None, None))
            continue
        y = out.astype(F64).copy()
        e = np.zeros_like(y)
        for c, n in enumerate(live):
            y[c, :, :n] = 0.0 if w is None or decay == 0.0 else decay * w[c, :, :n].astype(F64)
            e[c, :, :n] = np.abs(y[c, :, :n]) * 2.0 ** -23
        res.append((y, e))
    for b in range(B):
        for t in range(T):
            for h in range(H):
                if lse[b, t, h] == -np.inf:
                    continue
                x = q[b, t, h].astype(F64)
                sides = []
                if prefix is not None:
                    g = b // (B // len(prefix_len))
                    sides.append((0, g, prefix[g, :live_p[g], h // (H // K)]))
                if own is not None:
                    n = min(max(int(seen[b, t]), 0), own.shape[1])
                    sides.append((1, b, own[b, :n, h // (H // K)]))
                for side, c, kk in sides:
                    kk = kk.astype(F64)
                    p = np.exp(scale * (kk @ x) - float(lse[b, t, h]))
                    res[side][0][c, h // (H // K), :len(p)] += p
                    # fp32 dot of D terms, the score and lse in log2 units, 2^x by approximation, the sums
                    rel = (D + 2) * 2.0 ** -23 * scale * (np.abs(kk) @ np.abs(x)) + 2.0 ** -22 * abs(float(lse[b, t, h])) \
                        + (4 + B * T * H) * 2.0 ** -23
                    res[side][1][c, h // (H // K), :len(p)] += p * rel
    return res


def evict(w, n, keep, sink, recent) -> list:
    """Rows that stay of one head's first n rows, ascending."""
    if n <= keep:
        return list(range(n))
    first = [i for i in range(n) if i < sink or i >= n - recent]
    rest = [i for i in range(n) if sink <= i < n - recent]
    # Python's sort is stable: ties keep the lowest row first; NaN below everything.
    rest.sort(key=lambda i: (1, 0.0) if math.isnan(w[i]) else (0, -float(w[i])))
    return sorted(first + rest[:keep - len(first)])


# ------------------------------------------------------------------ norms, windows, 8 bits

def norm(x, weight, eps) -> np.ndarray:
    """Heads x [..][D] divided by the root of their mean square, times the weight (None: ones)."""
    x = x.astype(F64)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + float(np.float32(eps)))
    return y if weight is None else y * weight.astype(F64)


def append_normed(q, k, v, positions, rows, cache_k, cache_v, r, q_weight, k_weight, eps):
    return append(norm(q, q_weight, eps), norm(k, k_weight, eps), v, positions, rows, cache_k, cache_v, r)


def visible(n, rows, window, sink) -> np.ndarray:
    """Rows that a token of count n sees of a cache of `rows` rows (window 0: all before n)."""
    n = min(max(int(n), 0), rows)
    r = np.arange(n)
    return r if window == 0 else r[(r < sink) | (r >= n - window)]


def attend_window(q, k, v, seen, window, sink, scale):
    """(out, lse, dot, mass) as attend's, over the rows that `visible` says."""
    B, T, H, D = q.shape
    K = k.shape[2]
    out, lse = np.zeros(q.shape, F64), np.full((B, T, H), -np.inf)
    dot, mass = np.zeros((B, T, H)), np.zeros(q.shape, F64)
    for b in range(B):
        for t in range(T):
            at = visible(seen[b, t], k.shape[1], window, sink)
            if len(at) == 0:
                continue
            x = q[b, t].astype(F64).reshape(K, H // K, D)
            kk, vv = k[b, at].astype(F64), v[b, at].astype(F64)
            s = scale * np.einsum("kgd,jkd->kgj", x, kk)
            m = s.max(-1, keepdims=True)
            p = np.exp(s - m)
            tot = p.sum(-1, keepdims=True)
            lse[b, t] = (m + np.log(tot)).reshape(H)
            p /= tot
            out[b, t] = np.einsum("kgj,jkd->kgd", p, vv).reshape(H, D)
            dot[b, t] = scale * np.einsum("kgd,jkd->kgj", np.abs(x), np.abs(kk)).max(-1).reshape(H)
            mass[b, t] = np.einsum("kgj,jkd->kgd", p, np.abs(vv)).reshape(H, D)
    return out, lse, dot, mass


def e4m3(x) -> np.ndarray:
    """The e4m3 number nearest to each x of magnitude up to 448 (ties to the even one); what is not finite becomes NaN."""
    x = np.asarray(x, F64)
    _, p = np.frexp(np.maximum(np.abs(np.where(np.isfinite(x), x, 0.0)), 2.0 ** -6))
    step = np.ldexp(1.0, p - 4)
    return np.where(np.isfinite(x), np.rint(np.where(np.isfinite(x), x, 0.0) / step) * step, np.nan)


def scale8(x) -> int:
    """The byte of the least power of two 2^(byte - 127), byte >= 1, at which the finite x are at most 448 of it."""
    x = np.abs(np.asarray(x, F64))
    top = float(x[np.isfinite(x)].max(initial=0.0))
    m, p = math.frexp(top / 448.0)
    return max(1, (p if m > 0.5 else p - 1) + 127) if top > 0 else 1


def append8(x, start, count, codes, scales, block):
    """(codes, scales) of 8-bit caches after rows x [B][T][K][D] (coded already, fp64) went to rows start .. : codes are e4m3
    numbers [B][R][K][D], scales bytes [B][K][blocks]."""
    codes, scales = codes.astype(F64).copy(), scales.astype(np.int64).copy()
    B, T, K, _ = x.shape
    R = codes.shape[1]
    for b in range(B):
        s = int(start[b])
        if not 0 <= s < R:
            continue
        end = min(R, s + min(max(int(count[b]), 0), T))
        for i in range(s // block, (end - 1) // block + 1 if end > s else 0):
            lo, hi = max(s, i * block), min(end, (i + 1) * block)
            for h in range(K):
                part = x[b, lo - s:hi - s, h]
                e = scale8(part)
                if i * block < s:
                    old = int(scales[b, h, i])
                    e = max(e, old)
                    if e > old:
                        codes[b, i * block:s, h] = e4m3(codes[b, i * block:s, h] * 2.0 ** (old - e))
                scales[b, h, i] = e
                codes[b, lo:hi, h] = e4m3(part * 2.0 ** (127 - e)) if e < 255 else np.nan
    return codes, scales


def values8(codes, scales, block) -> np.ndarray:
    """The numbers that 8-bit caches hold."""
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(F64) - 127))
    return codes.astype(F64) * np.repeat(s, block, axis=2)[:, :, :codes.shape[1]].transpose(0, 2, 1)[..., None]
