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

from .jpi import _HERE, JPI_BF16, JPI_FP32, OnStream, _check, _ptr, _stream, load


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
    s = k.stride()
    if v is not None and (v.stride() != s or v.shape != k.shape or v.dtype is not k.dtype):
        raise ValueError("k and v must be caches of one shape, type and strides")
    if len(s) != (5 if layers else 4):
        raise ValueError("a cache is [caches][rows][KV heads][head dim], with layers [layers] before that")
    if s[-1] != 1 and k.shape[-1] > 1:
        raise ValueError("a head's elements must be contiguous")
    return jpi_kv_cache(k.data_ptr(), None if v is None else v.data_ptr(), s[-4], s[-3], s[-2], s[0] if layers else 0,
                        k.shape[-3])


def _checked_calls(*geometry):
    """The module _kv and its view of a handle's geometry, with the entry points of the library that is loaded."""
    try:
        from . import _kv
    except ImportError as e:
        raise RuntimeError(f"the module _kv is not built ({e}): run `python -m paper_2607_12659_gb300.build`") from e
    lib = load()
    return _kv, _kv.calls(*geometry, *(ctypes.cast(getattr(lib, f"jpi_kv_{n}"), c_void_p).value for n in ("append", "attend", "weigh", "evict")))


class KV:
    """A created handle of the KV-cache operators (jpi_kv_handle)."""

    def __init__(self, n_heads: int, n_kv_heads: int, head_dim: int, max_batch: int = 1, max_tokens: int = 1,
                 precision: str = "bf16", scale: float = 0.0, rope: Rope | None = None):
        import torch
        self.handle = None
        self.cfg = jpi_kv_config(n_heads=n_heads, n_kv_heads=n_kv_heads, head_dim=head_dim, max_batch=max_batch,
                                 max_tokens=max_tokens, scale=scale,
                                 precision={"bf16": JPI_BF16, "fp32": JPI_FP32}[precision])
        self.heads, self.kv_heads, self.head_dim = n_heads, n_kv_heads, head_dim
        self.dtype = torch.bfloat16 if precision == "bf16" else torch.float32
        self.handle = jpi_kv_create(self.cfg, rope.c() if rope is not None else None)
        self.index = torch.cuda.current_device()
        self.device = torch.device("cuda", self.index)
        self._torch, self._float = torch, torch.float32
        self._kv, self._calls = _checked_calls(n_heads, n_kv_heads, head_dim, precision == "bf16", self.index)

    def close(self):
        if self.handle:
            jpi_kv_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # The C-ABI sees addresses only: what the tensors are is checked by the module _kv (csrc/kv/kv_calls.cpp), with
    # ValueError, before each call.
    def _on(self, stream):
        """Torch's side of a call on another stream than the current one (None: this one)."""
        return _HERE if stream is None else OnStream(stream, self.device)

    def _call(self, fn, on, stream, args, reads, returns):
        """The checked call, and its result if it makes one; on a stream of its own, what it reads and returns is kept."""
        raw = self._torch._C._cuda_getCurrentRawStream(self.index) if on is None else _stream(stream)
        result = getattr(self._kv, fn)(self._calls, self.handle, raw, *args)
        made = type(result) is not int      # else a status
        if not made and result:
            _check(result, "jpi_kv_" + fn)
        if on is not None:
            on.reads(*(t for t in reads if t is not None))
            on.returns(*returns, *((result,) if made else ()))
        return result

    def append(self, q, k, v, positions, rows, cache_k=None, cache_v=None, q_out=None, stream=None):
        """Codes q [B][T][H][D] and k [B][T][Hk][D] for `positions` (int32 [B][T]) and writes k and v into `rows`
        (int32 [B][T]; a row outside the cache marks padding, one that a request names twice holds a mixture) of the caches.
        Returns the coded queries. q, v, or k with v and the caches may be None."""
        with self._on(stream) as on:
            returns = ()
            if q is None:
                q_out = None
            elif q_out is None:
                q_out = self._torch.zeros((*q.shape[:2], self.heads, self.head_dim), dtype=self.dtype, device=self.device)
                returns = (q_out,)
            self._call("append", on, stream, (q, k, v, positions, rows, cache_k, cache_v, q_out),
                       (q, k, v, positions, rows, cache_k, cache_v, None if returns else q_out), returns)
        return q_out

    def attend(self, q, prefix=None, prefix_len=None, own=None, seen=None, out=None, lse=None, stream=None):
        """Attention of q [B][T][H][D] over the first prefix_len[g] rows of prefix (k, v) [G][P][Hk][D], shared by each
        run of B / G requests, and the first seen[b][t] rows of own (k, v) [B][R][Hk][D]. Returns (out, lse)."""
        with self._on(stream) as on:
            reads, returns = (out, lse), []
            if out is None:
                out = self._torch.empty((*q.shape[:2], self.heads, self.head_dim), dtype=self.dtype, device=self.device)
                returns.append(out)
            if lse is None:
                lse = self._torch.empty((*q.shape[:2], self.heads), dtype=self._float, device=self.device)
                returns.append(lse)
            if on is not None:
                reads += (q, prefix_len, seen, *(prefix or ()), *(own or ()))
            self._call("attend", on, stream, (q, prefix, prefix_len, own, seen, out, lse), reads, returns)
        return out, lse

    def weigh(self, q, lse, prefix=None, prefix_len=None, own=None, seen=None, w_prefix=None, w_own=None, decay=1.0,
              out_prefix=None, out_own=None, stream=None):
        """Adds the attention weight that q's tokens and heads give to each key of `prefix` (keys [G][P][Hk][D]) and
        `own` (keys [B][R][Hk][D]) to decay times w_prefix [G][Hk][P] and w_own [B][Hk][R] (None: zeros). Returns
        the sums, in out_prefix and out_own (None: new ones, zero where a row holds no key)."""
        with self._on(stream) as on:
            reads, returns = (q, lse, prefix, prefix_len, own, seen, w_prefix, w_own, out_prefix, out_own), []
            outs = [out_prefix, out_own]
            for i, keys in enumerate((prefix, own)):
                if keys is not None and outs[i] is None:
                    outs[i] = self._torch.zeros((keys.shape[0], self.kv_heads, keys.shape[1]), dtype=self._float, device=self.device)
                    returns.append(outs[i])
            self._call("weigh", on, stream, (q, lse, prefix, prefix_len, own, seen, decay, w_prefix, outs[0], w_own, outs[1]),
                       reads, returns)
        return outs[0], outs[1]

    def evict(self, k, v, w, length, keep, sink=0, recent=0, out_k=None, out_v=None, out_w=None, out_length=None,
              stream=None):
        """Keeps `keep` of the first length[c] rows of every cache of k, v [L][N][R][Hk][D]: the first `sink`, the last
        `recent`, the best of the others by w [L][N][Hk][R]. In place, or into out_k, out_v and out_w of at least `keep`
        rows; the new lengths go to out_length (None: `length` itself). Returns the rows kept, int32 [L][N][Hk][keep],
        -1 behind them."""
        outs = (out_k, out_v, out_w)
        if any(t is None for t in outs):
            if any(t is not None for t in outs):
                raise ValueError("out_k, out_v and out_w go together")
            out_k, out_v, out_w = k, v, w
        if out_length is None:
            out_length = length
        with self._on(stream) as on:
            return self._call("evict", on, stream, (k, v, w, length, keep, sink, recent, out_k, out_v, out_w, out_length),
                              (k, v, w, length, out_k, out_v, out_w, out_length), ())

    def device_status(self):
        jpi_kv_device_status(self.handle)

    def memory_usage(self) -> int:
        return jpi_kv_memory_usage(self.handle)


__all__ = ["KV", "Rope", "cache_of", "jpi_kv_create", "jpi_kv_destroy", "jpi_kv_append", "jpi_kv_attend", "jpi_kv_weigh",
           "jpi_kv_evict", "jpi_kv_device_status", "jpi_kv_memory_usage"]
