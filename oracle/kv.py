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
