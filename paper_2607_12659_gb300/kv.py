"""ctypes binding of the KV-cache operators (``include/jpi_kv.h``, ``libjpi.so``; argument
marshalling only).

``KV`` fixes an attention's geometry and rotary coding; its methods run on caches that the caller
keeps, torch tensors [caches][rows][KV heads][head dim] of any strides with contiguous heads (a
head-major cache is ``stored.transpose(1, 2)``):

``append``  codes the positions of new tokens' queries and keys and writes keys and values into rows
``attend``  attention of a batch over shared prefixes and each request's own rows
``weigh``   accumulates the attention weight each cached key received
``evict``   keeps the rows with the most of it
"""

from __future__ import annotations

import ctypes
from ctypes import byref, c_float, c_int, c_longlong, c_void_p
from dataclasses import dataclass

from . import jpi
from .jpi import JPI_BF16, JPI_FP32, OnStream, _check, _ptr, _stream, load


class jpi_kv_rope(ctypes.Structure):
    _fields_ = [(n, c_int) for n in ("dim", "layout", "scaling", "original")] + [
        (n, c_float) for n in ("base", "factor", "low", "high", "mscale")]


class jpi_kv_config(ctypes.Structure):
    _fields_ = [(n, c_int) for n in ("n_heads", "n_kv_heads", "head_dim", "max_batch", "max_tokens")] + [
        ("scale", c_float), ("precision", c_int)]


class jpi_kv_cache(ctypes.Structure):
    _fields_ = [("k", c_void_p), ("v", c_void_p)] + [
        (n, c_longlong) for n in ("cache_stride", "row_stride", "head_stride", "layer_stride")] + [("rows", c_int)]


LAYOUTS = {"half": 0, "interleaved": 1}
SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "by_parts": 3}


# ------------------------------------------------------------------ thin C-ABI mirrors

def jpi_kv_create(cfg: jpi_kv_config, rope: jpi_kv_rope | None = None) -> int:
    h = c_void_p()
    _check(load().jpi_kv_create(byref(cfg), byref(rope) if rope is not None else None, byref(h)), "jpi_kv_create")
    return h.value


def jpi_kv_destroy(h: int):
    _check(load().jpi_kv_destroy(h), "jpi_kv_destroy")


def jpi_kv_append(h, q, q_stride, k, k_stride, v, v_stride, position, row, batch, tokens, q_out, cache, stream=None):
    _check(load().jpi_kv_append(h, _ptr(q), q_stride, _ptr(k), k_stride, _ptr(v), v_stride, _ptr(position), _ptr(row),
                                batch, tokens, _ptr(q_out), byref(cache) if cache is not None else None,
                                _stream(stream)), "jpi_kv_append")


def jpi_kv_attend(h, q, q_stride, batch, tokens, prefix, groups, prefix_len, own, seen, out, lse, stream=None):
    _check(load().jpi_kv_attend(h, _ptr(q), q_stride, batch, tokens, byref(prefix) if prefix is not None else None,
                                groups, _ptr(prefix_len), byref(own) if own is not None else None, _ptr(seen),
                                _ptr(out), _ptr(lse), _stream(stream)), "jpi_kv_attend")


def jpi_kv_weigh(h, q, q_stride, lse, batch, tokens, prefix, groups, prefix_len, own, seen, decay, prefix_in,
                 prefix_out, own_in, own_out, stream=None):
    _check(load().jpi_kv_weigh(h, _ptr(q), q_stride, _ptr(lse), batch, tokens,
                               byref(prefix) if prefix is not None else None, groups, _ptr(prefix_len),
                               byref(own) if own is not None else None, _ptr(seen), float(decay), _ptr(prefix_in),
                               _ptr(prefix_out), _ptr(own_in), _ptr(own_out), _stream(stream)), "jpi_kv_weigh")


def jpi_kv_evict(h, src, w, length, layers, caches, keep, sink, recent, dst, w_out, length_out, kept, stream=None):
    _check(load().jpi_kv_evict(h, byref(src), _ptr(w), _ptr(length), layers, caches, keep, sink, recent, byref(dst),
                               _ptr(w_out), _ptr(length_out), _ptr(kept), _stream(stream)), "jpi_kv_evict")


def jpi_kv_device_status(h):
    _check(load().jpi_kv_device_status(h), "jpi_kv_device_status")


def jpi_kv_memory_usage(h) -> int:
    b = c_longlong()
    _check(load().jpi_kv_memory_usage(h, byref(b)), "jpi_kv_memory_usage")
    return b.value


# ------------------------------------------------------------------ convenience wrapper

@dataclass(frozen=True)
class Rope:
    """Rotary coding of the first ``dim`` elements of a head (jpi_kv_rope)."""
    dim: int
    layout: str = "half"        # half, interleaved
    base: float = 10000.0
    scaling: str = "none"       # none, linear, ntk, by_parts
    factor: float = 1.0
    low: float = 1.0
    high: float = 32.0
    original: int = 1
    mscale: float = 1.0

    def c(self) -> jpi_kv_rope:
        return jpi_kv_rope(dim=self.dim, layout=LAYOUTS[self.layout], scaling=SCALINGS[self.scaling],
                           original=self.original, base=self.base, factor=self.factor, low=self.low, high=self.high,
                           mscale=self.mscale)


def cache_of(k, v=None, layers=False) -> jpi_kv_cache:
    """The jpi_kv_cache of tensors [caches][rows][KV heads][head dim], or with `layers` another dimension before them."""
    n = 5 if layers else 4
    if k.dim() != n or (v is not None and (v.shape != k.shape or v.stride() != k.stride() or v.dtype != k.dtype)):
        raise ValueError(f"k and v must be {n}-dimensional caches of one shape, type and strides")
    if k.stride(-1) != 1 and k.shape[-1] > 1:
        raise ValueError("a head's elements must be contiguous")
    st = k.stride()[-4:]
    return jpi_kv_cache(k=k.data_ptr(), v=v.data_ptr() if v is not None else None, cache_stride=st[0], row_stride=st[1],
                        head_stride=st[2], layer_stride=k.stride(0) if layers else 0, rows=k.shape[-3])


class KV:
    """A created handle of the KV-cache operators (jpi_kv_handle)."""

    def __init__(self, n_heads: int, n_kv_heads: int, head_dim: int, max_batch: int = 1, max_tokens: int = 1,
                 precision: str = "bf16", scale: float = 0.0, rope: Rope | None = None):
        import torch
        self.handle = None
        self.cfg = jpi_kv_config(n_heads=n_heads, n_kv_heads=n_kv_heads, head_dim=head_dim, max_batch=max_batch,
                                 max_tokens=max_tokens, scale=scale,
                                 precision={"bf16": JPI_BF16, "fp32": JPI_FP32}[precision])
        self.dtype = torch.bfloat16 if precision == "bf16" else torch.float32
        self.handle = jpi_kv_create(self.cfg, rope.c() if rope is not None else None)
        self.device = torch.device("cuda", torch.cuda.current_device())

    def close(self):
        if self.handle:
            jpi_kv_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # The C-ABI sees addresses only: what they point to is checked here.
    def _data(self, name, t, shape=None, dtype=None):
        if t is None:
            return
        if t.device != self.device:
            raise ValueError(f"{name} is on {t.device}, the handle on {self.device}")
        if t.dtype != (dtype or self.dtype):
            raise ValueError(f"{name} is {t.dtype}, not {dtype or self.dtype}")
        if shape is not None and tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")

    def _whole(self, name, t, shape, dtype):
        """A tensor that is taken (and written) as one contiguous block."""
        self._data(name, t, shape, dtype)
        if t is not None and not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")

    def _cache(self, name, k, v, n, layers=None):
        K, D = self.cfg.n_kv_heads, self.cfg.head_dim
        lead = (n,) if layers is None else (layers, n)
        for part, t in (("k", k), ("v", v)):
            if t is not None:
                self._data(f"{name} {part}", t)
                if tuple(t.shape) != (*lead, t.shape[len(lead)], K, D):
                    raise ValueError(f"{name} {part} has shape {tuple(t.shape)}, not [{', '.join(map(str, lead))}][rows][{K}][{D}]")
        return cache_of(k, v, layers is not None)

    def _tokens(self, name, t, heads):
        """(tensor, token stride): new tokens [batch][tokens][heads][D], one row of `stride` elements each."""
        self._data(name, t, (*t.shape[:2], heads, self.cfg.head_dim))
        B, T, _, D = t.shape
        s = t.stride()
        whole = s[3] == 1 and (s[2] == D or heads == 1)
        stride = s[1] if T > 1 else s[0] if B > 1 else heads * D
        if not whole or (B > 1 and T > 1 and s[0] != T * s[1]) or stride < heads * D or (stride * t.element_size()) % 16 \
                or t.data_ptr() % 16:
            t = t.contiguous()
            stride = heads * D
        return t, stride

    def append(self, q, k, v, positions, rows, cache_k=None, cache_v=None, q_out=None, stream=None):
        """Codes q [B][T][H][D] and k [B][T][Hk][D] for `positions` (int32 [B][T]) and writes k and v into `rows`
        (int32 [B][T]; a row outside the cache marks padding) of the caches. Returns the coded queries. q, v, or k
        with v and the caches may be None."""
        import torch
        H, K, D = self.cfg.n_heads, self.cfg.n_kv_heads, self.cfg.head_dim
        if q is None and k is None:
            raise ValueError("neither q nor k is given")
        B, T = (q if q is not None else k).shape[:2]
        dev = self.device
        with OnStream(stream, dev) as on:
            args = []
            for name, t, heads in (("q", q, H), ("k", k, K), ("v", v, K)):
                if t is None:
                    args += [None, 0]
                    continue
                if tuple(t.shape[:2]) != (B, T):
                    raise ValueError(f"{name} has shape {tuple(t.shape)}, not [{B}][{T}]..")
                on.reads(t)
                args += self._tokens(name, t, heads)
            self._whole("positions", positions, (B, T), torch.int32)
            self._whole("rows", rows, (B, T), torch.int32)
            on.reads(positions, rows)
            cache = None
            if k is not None:
                if cache_k is None or (v is not None and cache_v is None):
                    raise ValueError("k and v need the caches they go to")
                cache = self._cache("cache", cache_k, cache_v if v is not None else None, B)
                on.reads(cache_k, *(() if v is None else (cache_v,)))
            if q is None:
                q_out = None
            elif q_out is None:
                q_out = torch.zeros((B, T, H, D), dtype=self.dtype, device=dev)
                on.returns(q_out)
            else:
                self._whole("q_out", q_out, (B, T, H, D), self.dtype)
                on.reads(q_out)
        jpi_kv_append(self.handle, *args, positions, rows, B, T, q_out, cache, stream)
        return q_out

    def _sides(self, on, q, prefix, prefix_len, own, seen):
        """(q, stride, B, T, prefix cache, groups, own cache) of attend and weigh; prefix and own are (k, v)."""
        import torch
        H = self.cfg.n_heads
        B, T = q.shape[:2]
        on.reads(q)
        q, stride = self._tokens("q", q, H)
        if (prefix is None) != (prefix_len is None) or (own is None) != (seen is None):
            raise ValueError("prefix goes with prefix_len, own with seen")
        p = o = None
        groups = 1
        if prefix is not None:
            groups = prefix[0].shape[0]
            p = self._cache("prefix", *prefix, groups)
            self._whole("prefix_len", prefix_len, (groups,), torch.int32)
            on.reads(prefix_len, *(t for t in prefix if t is not None))
        if own is not None:
            o = self._cache("own", *own, B)
            self._whole("seen", seen, (B, T), torch.int32)
            on.reads(seen, *(t for t in own if t is not None))
        return q, stride, B, T, p, groups, o

    def attend(self, q, prefix=None, prefix_len=None, own=None, seen=None, out=None, lse=None, stream=None):
        """Attention of q [B][T][H][D] over the first prefix_len[g] rows of prefix (k, v) [G][P][Hk][D], shared by each
        run of B / G requests, and the first seen[b][t] rows of own (k, v) [B][R][Hk][D]. Returns (out, lse)."""
        import torch
        H, D = self.cfg.n_heads, self.cfg.head_dim
        with OnStream(stream, self.device) as on:
            q, stride, B, T, p, groups, o = self._sides(on, q, prefix, prefix_len, own, seen)
            if out is None:
                out = torch.empty((B, T, H, D), dtype=self.dtype, device=self.device)
                on.returns(out)
            else:
                self._whole("out", out, (B, T, H, D), self.dtype)
                on.reads(out)
            if lse is None:
                lse = torch.empty((B, T, H), dtype=torch.float32, device=self.device)
                on.returns(lse)
            else:
                self._whole("lse", lse, (B, T, H), torch.float32)
                on.reads(lse)
        jpi_kv_attend(self.handle, q, stride, B, T, p, groups, prefix_len, o, seen, out, lse, stream)
        return out, lse

    def weigh(self, q, lse, prefix=None, prefix_len=None, own=None, seen=None, w_prefix=None, w_own=None, decay=1.0,
              out_prefix=None, out_own=None, stream=None):
        """Adds the attention weight that q's tokens and heads give to each key of `prefix` (keys [G][P][Hk][D]) and
        `own` (keys [B][R][Hk][D]) to decay times w_prefix [G][Hk][P] and w_own [B][Hk][R] (None: zeros). Returns
        the sums, in out_prefix and out_own (None: new ones, zero where a row holds no key)."""
        import torch
        H, K = self.cfg.n_heads, self.cfg.n_kv_heads
        with OnStream(stream, self.device) as on:
            q, stride, B, T, p, groups, o = self._sides(on, q, None if prefix is None else (prefix, None), prefix_len,
                                                        None if own is None else (own, None), seen)
            self._whole("lse", lse, (B, T, H), torch.float32)
            on.reads(lse)
            outs = []
            for name, cache, n, w, out in (("prefix", p, groups, w_prefix, out_prefix), ("own", o, B, w_own, out_own)):
                if cache is None:
                    if w is not None or out is not None:
                        raise ValueError(f"weights of {name} without {name}")
                    outs += [None, None]
                    continue
                shape = (n, K, cache.rows)
                if w is not None:
                    self._whole(f"w_{name}", w, shape, torch.float32)
                    on.reads(w)
                if out is None:
                    out = torch.zeros(shape, dtype=torch.float32, device=self.device)
                    on.returns(out)
                else:
                    self._whole(f"out_{name}", out, shape, torch.float32)
                    on.reads(out)
                outs += [w, out]
        jpi_kv_weigh(self.handle, q, stride, lse, B, T, p, groups, prefix_len, o, seen, decay, *outs, stream)
        return outs[1], outs[3]

    def evict(self, k, v, w, length, keep, sink=0, recent=0, out_k=None, out_v=None, out_w=None, out_length=None,
              stream=None):
        """Keeps `keep` of the first length[c] rows of every cache of k, v [L][N][R][Hk][D]: the first `sink`, the last
        `recent`, the best of the others by w [L][N][Hk][R]. In place, or into out_k, out_v and out_w of at least `keep`
        rows; the new lengths go to out_length (None: `length` itself). Returns the rows kept, int32 [L][N][Hk][keep],
        -1 behind them."""
        import torch
        K = self.cfg.n_kv_heads
        outs = (out_k, out_v, out_w)
        if any(t is None for t in outs) and any(t is not None for t in outs):
            raise ValueError("out_k, out_v and out_w go together")
        if out_k is None:
            out_k, out_v, out_w = k, v, w
        if out_length is None:
            out_length = length
        L, N, R = k.shape[:3]
        with OnStream(stream, self.device) as on:
            src = self._cache("k, v", k, v, N, L)
            dst = self._cache("out", out_k, out_v, N, L)
            self._whole("w", w, (L, N, K, R), torch.float32)
            self._whole("out_w", out_w, (L, N, K, out_k.shape[2]), torch.float32)
            self._whole("length", length, (N,), torch.int32)
            self._whole("out_length", out_length, (N,), torch.int32)
            on.reads(k, v, w, length, out_k, out_v, out_w, out_length)
            kept = torch.empty((L, N, K, max(keep, 0)), dtype=torch.int32, device=self.device)
            on.returns(kept)
        jpi_kv_evict(self.handle, src, w, length, L, N, keep, sink, recent, dst, out_w, out_length, kept, stream)
        return kept

    def device_status(self):
        jpi_kv_device_status(self.handle)

    def memory_usage(self) -> int:
        return jpi_kv_memory_usage(self.handle)


__all__ = ["KV", "Rope", "cache_of", "jpi_kv_create", "jpi_kv_destroy", "jpi_kv_append", "jpi_kv_attend", "jpi_kv_weigh",
           "jpi_kv_evict", "jpi_kv_device_status", "jpi_kv_memory_usage"]
