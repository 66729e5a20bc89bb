"""Binding of the calls for serving after the prefill: rotary positions, the
paged cache, one new token's attention and eviction (include/xattn.h).

Argument checks and marshalling only, as in binding.py; every tensor is on the
current device.

Tensor layouts:
  vectors  bf16 [batch, heads, tokens, 128] or [heads, tokens, 128], any strides
           that keep a vector's 128 values together and 16-byte aligned
  cache    bf16 or float8_e4m3fn [pages, hkv, page, 128] (KVCache)
  table    int32 [batch, table_pages]; -1 (any value outside 0 .. pages-1): no page
  weights  fp32 [batch, hkv, table_pages * page]
"""
from __future__ import annotations

import ctypes
import functools

import numpy as np
import torch

from .binding import (XATTN_ERR_ARG, Cache, RotaryPlan, XAttnError, _check, _check_shape,
                      _check_workspace, _need, _ptr, lib)

HEAD_DIM = 128
_PAGES = (16, 32, 64, 128, 256)
_I3 = ctypes.c_int64 * 3


def _fail(message):
    raise XAttnError(XATTN_ERR_ARG, message)


def rotary_freqs(pairs, base: float = 10000.0, restart: bool = False) -> np.ndarray:
    """The usual frequencies of Rotary: pair i of n rotates by base^(-i/n) a position, counted
    over all axes, or from 0 for each axis of `pairs` (restart)."""
    if restart:
        return np.concatenate([float(base) ** (-np.arange(n) / n) for n in pairs])
    n = int(sum(pairs))
    return float(base) ** (-np.arange(n) / n)


class _Fixed:
    """An object whose C struct holds what its attributes of _FIXED say: neither changes once it
    is made."""
    _FIXED = frozenset()

    def __setattr__(self, name, value):
        if name in self._FIXED and "_ref" in self.__dict__:  # the last that is set
            _fail(f"the {name} of a {type(self).__name__} is fixed: make another one")
        super().__setattr__(name, value)

    def __delattr__(self, name):
        if name in self._FIXED:
            _fail(f"the {name} of a {type(self).__name__} is fixed")
        super().__delattr__(name)


class Rotary(_Fixed):
    """Rotary positions of one model: pairs[a] of a head's 64 pairs turn with position axis a, by
    freq (float64, one a pair, radians per position); pair i is elements (2i, 2i+1) if interleaved,
    else (i, i+64). Pairs behind them are not rotated."""
    _FIXED = frozenset(("axes", "pairs", "interleaved", "_freq", "_plan", "_ref"))

    def __init__(self, pairs, freq, interleaved: bool = False):
        pairs = [int(n) for n in pairs]
        if not 1 <= len(pairs) <= 3 or min(pairs) < 1 or sum(pairs) > 64:
            _fail(f"pairs must be 1 to 3 positive numbers of sum <= 64, got {pairs}")
        self._freq = np.array(freq, dtype=np.float64)  # a copy: the plan points into it
        if self._freq.shape != (sum(pairs),) or not np.isfinite(self._freq).all():
            _fail(f"freq must be {sum(pairs)} finite numbers")
        self.pairs, self.interleaved = tuple(pairs), bool(interleaved)
        self._plan = RotaryPlan(len(pairs), (ctypes.c_int32 * 3)(*pairs), int(self.interleaved),
                                self._freq.ctypes.data)
        self.axes = len(pairs)
        self._ref = ctypes.byref(self._plan)


class KVCache(_Fixed):
    """A pool of pages: k, v [pages, hkv, page, 128], bf16, or float8_e4m3fn with the bytes of
    their power-of-two scales k_scale, v_scale uint8 [pages, hkv, page]. A larger pool is another
    KVCache."""
    _FIXED = frozenset(("k", "v", "k_scale", "v_scale", "pages", "hkv", "page", "e4m3", "device",
                        "_struct", "_ref"))

    def __init__(self, k, v, k_scale=None, v_scale=None):
        if k.dim() != 4 or k.shape[3] != HEAD_DIM or k.shape[2] not in _PAGES or 0 in k.shape:
            _fail(f"k must be [pages, hkv, page, {HEAD_DIM}] with pages of {_PAGES} tokens, got "
                  f"{tuple(k.shape)}")
        if k.dtype not in (torch.bfloat16, torch.float8_e4m3fn):
            _fail(f"k must be torch.bfloat16 or torch.float8_e4m3fn, got {k.dtype}")
        _check_shape(v, k.shape, k.dtype, "v")
        self.e4m3 = k.dtype != torch.bfloat16
        if self.e4m3:
            if k_scale is None or v_scale is None:
                _fail("an e4m3 cache needs k_scale and v_scale")
            for t, n in ((k_scale, "k_scale"), (v_scale, "v_scale")):
                _check_shape(t, k.shape[:3], torch.uint8, n)
        elif k_scale is not None or v_scale is not None:
            _fail("a bf16 cache has no scales")
        arrays = [t for t in (k, v, k_scale, v_scale) if t is not None]
        for t, n in zip(arrays, ("k", "v", "k_scale", "v_scale")):
            _need(t, t.dtype, n)
            if t.device != k.device:
                _fail(f"{n} must be on k's device {k.device}, got {t.device}")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.pages, self.hkv, self.page = (int(n) for n in k.shape[:3])
        self.device = k.device
        self._struct = Cache(self.pages, self.page, self.hkv, HEAD_DIM, int(self.e4m3), _ptr(k),
                             _ptr(v), _ptr(k_scale), _ptr(v_scale))
        self._ref = ctypes.byref(self._struct)

    @classmethod
    def empty(cls, pages, hkv, page=64, dtype=torch.bfloat16, device="cuda"):
        """A pool of zeros."""
        def zeros(*shape, dtype):
            return torch.zeros(shape, dtype=dtype, device=device)
        if dtype == torch.bfloat16:
            return cls(*[zeros(pages, hkv, page, HEAD_DIM, dtype=dtype) for _ in "kv"])
        if dtype != torch.float8_e4m3fn:
            _fail(f"dtype must be torch.bfloat16 or torch.float8_e4m3fn, got {dtype}")
        kv = [zeros(pages, hkv, page, HEAD_DIM, dtype=torch.uint8).view(dtype) for _ in "kv"]
        return cls(*kv, *[zeros(pages, hkv, page, dtype=torch.uint8).fill_(127) for _ in "kv"])


def _here(first, others, names, dense=()):
    """Every tensor on the current device, where the stream is, and those of `dense` contiguous;
    `names` are of (first, *others). Returns the device's index."""
    at = first.get_device()
    if at < 0:
        _fail(f"{names[0]} must be a device tensor")
    if at != torch._C._cuda_getDevice():
        _fail(f"{names[0]} must be on the current device, got {first.device}")
    for i, t in enumerate(others):
        if t is not None and t.get_device() != at:
            _fail(f"{names[i + 1]} must be a device tensor on {first.device}, got {t.device}")
    for t in dense:
        if t is not None and not t.is_contiguous():
            at = [x is t for x in (first, *others)].index(True)
            _fail(f"{names[at]} must be contiguous")
    return at


def _is(t, shape, dtype, name):
    """_check_shape of a tensor that must be given, at the cost of two comparisons where all is
    well."""
    if t is None:
        _fail(f"{name} must be given")
    if t.shape != shape or t.dtype is not dtype:
        _check_shape(t, shape, dtype, name)


def _may_be(t, shape, dtype, name):
    """The same of one that may be None."""
    if t is not None:
        _is(t, shape, dtype, name)


def _int32(value, name):
    """A number that goes to C as 32 bits, where a larger one would become another."""
    n = int(value)
    if not -2**31 <= n < 2**31:
        _fail(f"{name} must fit 32 bits, got {n}")
    return n


@functools.lru_cache(maxsize=1024)
def _strides(batch, head, token):
    return _I3(batch, head, token)  # only ever read


def _vectors(t, name, like=None):
    """(batch, heads, tokens, strides) of bf16 vectors, checked but for the device."""
    if t.dtype is not torch.bfloat16:
        _fail(f"{name} must be torch.bfloat16, got {t.dtype}")
    shape, strides = t.shape, t.stride()
    if len(shape) == 3:
        shape, strides = (1, *shape), (0, *strides)
    if len(shape) != 4 or shape[3] != HEAD_DIM or 0 in shape:
        _fail(f"{name} must be [batch, heads, tokens, {HEAD_DIM}] or [heads, tokens, {HEAD_DIM}], "
              f"got {tuple(t.shape)}")
    if like is not None and t.shape != like.shape:
        _fail(f"{name} must have shape {tuple(like.shape)}, got {tuple(t.shape)}")
    if strides[3] != 1:
        _fail(f"the {HEAD_DIM} values of a vector of {name} must be contiguous")
    return shape[0], shape[1], shape[2], _strides(*strides[:3])


def _positions(pos, rotary, batch, tokens, dims):
    if not isinstance(rotary, Rotary):
        _fail(f"rotary must be a Rotary, got {type(rotary).__name__}")
    _is(pos, (rotary.axes, batch, tokens) if dims == 4 else (rotary.axes, tokens), torch.int32,
        "pos")


def _is_cache(cache):
    if not isinstance(cache, KVCache):
        _fail(f"cache must be a KVCache, got {type(cache).__name__}")


def _table(table, batch, name="table"):
    """Columns of a page table of `batch` rows."""
    shape = table.shape
    if len(shape) != 2 or shape[0] != batch or shape[1] < 1:
        _fail(f"{name} must be [{batch}, pages], got {tuple(shape)}")
    if table.dtype is not torch.int32:
        _fail(f"{name} must be torch.int32, got {table.dtype}")
    return shape[1]


def _extent(t):
    """First and last byte of a strided tensor."""
    last = sum((n - 1) * s for n, s in zip(t.shape, t.stride()))
    return t.data_ptr(), t.data_ptr() + (last + 1) * t.element_size()


def _apart(a, b):
    """Whether two tensors of one shape lie apart, as far as the C call cannot tell: it can where
    they have the same strides."""
    if all(n == 1 or x == y for n, x, y in zip(a.shape, a.stride(), b.stride())):
        return True
    (a0, a1), (b0, b1) = _extent(a), _extent(b)
    return a1 <= b0 or b1 <= a0


def _made(stream, allocate):
    """What `allocate` makes, of the memory of the stream that the call runs on."""
    if stream is None:
        return allocate()
    with torch.cuda.stream(stream):
        return allocate()


def _handle(stream, at):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(at)
    if stream.device_index != at:
        _fail(f"stream must be one of the current device {at}, got {stream.device}")
    return stream.cuda_stream


def xattn_rotary(x, pos, rotary: Rotary, inverse=False, out=None, stream=None):
    """x rotated by its positions (back with inverse, which is also the gradient: nothing is
    recorded for it, and an x that requires one is refused while gradients are recorded). pos int32
    [axes, batch, tokens] ([axes, tokens] for 3-D x). out: contiguous if not given; may be x, or
    another slice of its buffer."""
    b, h, n, xs = _vectors(x, "x")
    if x.requires_grad and torch.is_grad_enabled():
        _fail("x requires a gradient, which the call does not record: call it under torch.no_grad() "
              "(in an autograd function the backward is the call with inverse)")
    _positions(pos, rotary, b, n, x.dim())
    if out is None:
        at = _here(x, (pos,), ("x", "pos"), (pos,))
        out = x.new_empty(x.shape) if stream is None else _made(
            stream, lambda: x.new_empty(x.shape))
        os = _strides(h * n * HEAD_DIM, n * HEAD_DIM, HEAD_DIM)
    else:
        _, _, _, os = _vectors(out, "out", x)
        at = _here(x, (out, pos), ("x", "out", "pos"), (pos,))
        if not _apart(out, x):
            _fail("out must be x itself or lie apart from it")
    _check(lib().xattn_rotary(x.data_ptr(), xs, b, h, n, HEAD_DIM, pos.data_ptr(), rotary._ref,
                              1 if inverse else 0, out.data_ptr(), os, _handle(stream, at)))
    return out


def xattn_cache_append(k, v, cache: KVCache, table, start, count=None, pos=None, rotary=None,
                       stream=None):
    """Writes k, v [batch, hkv, tokens, 128] as tokens start[b] .. of each sequence (count[b] of
    them, or all) into the cache's pages, the keys rotated by pos if rotary is given."""
    _is_cache(cache)
    b, h, n, ks = _vectors(k, "k")
    _, _, _, vs = _vectors(v, "v", k)
    if h != cache.hkv:
        _fail(f"k has {h} heads, the cache {cache.hkv}")
    width = _table(table, b)
    _is(start, (b,), torch.int32, "start")
    _may_be(count, (b,), torch.int32, "count")
    if (pos is None) != (rotary is None):
        _fail("pos and rotary go together")
    if rotary is not None:
        _positions(pos, rotary, b, n, k.dim())
    at = _here(k, (v, table, start, count, pos, cache.k),
               ("k", "v", "table", "start", "count", "pos", "cache"), (table, start, count, pos))
    _check(lib().xattn_cache_append(k.data_ptr(), ks, v.data_ptr(), vs, b, n, _ptr(count),
                                    start.data_ptr(), table.data_ptr(), width, _ptr(pos),
                                    None if rotary is None else rotary._ref, cache._ref,
                                    _handle(stream, at)))


@functools.lru_cache(maxsize=256)
def _decode_bytes(hkv, page, e4m3, batch, hq, table_pages, weights):
    """Workspace bytes of a shape; a function of the shape alone."""
    c = Cache(1, page, hkv, HEAD_DIM, int(e4m3), None, None, None, None)
    n = ctypes.c_size_t(0)
    _check(lib().xattn_decode_workspace_size(ctypes.byref(c), batch, hq, table_pages, weights,
                                             ctypes.byref(n)))
    return n.value


def decode_workspace_size(cache: KVCache, batch: int, hq: int, table_pages: int,
                          weights: bool = False) -> int:
    """Bytes of xattn_decode's workspace."""
    _is_cache(cache)
    return _decode_bytes(cache.hkv, cache.page, cache.e4m3, _int32(batch, "batch"),
                         _int32(hq, "hq"), _int32(table_pages, "table_pages"), int(bool(weights)))


def xattn_decode(q, cache: KVCache, table, lens, o=None, lse=None, weights=None, workspace=None,
                 want_lse=False, stream=None):
    """Attention of one new token per sequence, q bf16 [batch, hq, 128], over its lens[b] cached
    tokens: (o like q, and may be q; lse fp32 [batch, hq] or None). weights (fp32 [batch, hkv,
    table_pages * page]), if given, grow by each key's softmax weights, summed over its heads."""
    _is_cache(cache)
    shape = q.shape
    if len(shape) != 3 or shape[2] != HEAD_DIM or 0 in shape:
        _fail(f"q must be [batch, hq, {HEAD_DIM}], got {tuple(shape)}")
    if q.dtype is not torch.bfloat16:
        _fail(f"q must be torch.bfloat16, got {q.dtype}")
    b, hq, _ = shape
    width = _table(table, b)
    _is(lens, (b,), torch.int32, "lens")
    _may_be(o, shape, torch.bfloat16, "o")
    _may_be(lse, (b, hq), torch.float32, "lse")
    _may_be(weights, (b, cache.hkv, width * cache.page), torch.float32, "weights")
    _check_workspace(workspace)
    dense = (q, table, lens, o, lse, weights, workspace)
    at = _here(q, (table, lens, cache.k, o, lse, weights, workspace),
               ("q", "table", "lens", "cache", "o", "lse", "weights", "workspace"), dense)
    def allocate():
        need = 0 if workspace is not None else _decode_bytes(
            cache.hkv, cache.page, cache.e4m3, b, hq, width, int(weights is not None))
        return (q.new_empty(shape) if o is None else o,
                q.new_empty((b, hq), dtype=torch.float32) if lse is None and want_lse else lse,
                q.new_empty((need,), dtype=torch.uint8) if need else workspace)

    o, lse, workspace = _made(stream, allocate)
    _check(lib().xattn_decode(q.data_ptr(), cache._ref, b, hq, table.data_ptr(), width,
                              lens.data_ptr(), o.data_ptr(), _ptr(lse), _ptr(weights),
                              _ptr(workspace), 0 if workspace is None else workspace.numel(),
                              _handle(stream, at)))
    return o, lse


@functools.lru_cache(maxsize=256)
def _evict_bytes(hkv, page, batch, table_pages):
    """Workspace bytes of a shape; a function of the shape alone."""
    c = Cache(1, page, hkv, HEAD_DIM, 0, None, None, None, None)
    n = ctypes.c_size_t(0)
    _check(lib().xattn_evict_workspace_size(ctypes.byref(c), batch, table_pages, ctypes.byref(n)))
    return n.value


def evict_workspace_size(cache: KVCache, batch: int, table_pages: int) -> int:
    """Bytes of xattn_cache_evict's workspace."""
    _is_cache(cache)
    return _evict_bytes(cache.hkv, cache.page, _int32(batch, "batch"),
                        _int32(table_pages, "table_pages"))


def xattn_cache_evict(cache: KVCache, table, lens, weights, new_table, budget: int, recent: int,
                      kept=None, new_lens=None, new_weights=None, workspace=None, stream=None):
    """Moves the `budget` most valuable tokens of every sequence and key head (the last `recent`
    and the heaviest before them) to the pages of new_table, none of which is in table. Tokens that
    can be kept need a page: of others the new place is left as it was. Returns
    (kept int32 [batch, hkv, budget], new_lens int32 [batch], new_weights fp32 [batch, hkv,
    new_pages * page])."""
    _is_cache(cache)
    if table.dim() != 2:
        _fail(f"table must be [batch, pages], got {tuple(table.shape)}")
    b, h, budget, recent = table.shape[0], cache.hkv, int(budget), int(recent)
    width, new_width = _table(table, b), _table(new_table, b, "new_table")
    _is(lens, (b,), torch.int32, "lens")
    _is(weights, (b, h, width * cache.page), torch.float32, "weights")
    if not 1 <= budget <= new_width * cache.page:
        _fail(f"budget must be 1 to {new_width * cache.page} (the new table's tokens), got "
              f"{budget}")
    if not 0 <= recent <= budget:
        _fail(f"recent must be 0 to {budget} (the budget), got {recent}")
    _may_be(kept, (b, h, budget), torch.int32, "kept")
    _may_be(new_lens, (b,), torch.int32, "new_lens")
    _may_be(new_weights, (b, h, new_width * cache.page), torch.float32, "new_weights")
    _check_workspace(workspace)
    tensors = (lens, weights, new_table, kept, new_lens, new_weights, workspace)
    at = _here(table, (*tensors, cache.k), ("table", "lens", "weights", "new_table", "kept",
                                            "new_lens", "new_weights", "workspace", "cache"),
               (table, *tensors))
    def allocate():
        need = 0 if workspace is not None else _evict_bytes(h, cache.page, b, width)
        return (lens.new_empty((b, h, budget)) if kept is None else kept,
                lens.new_empty((b,)) if new_lens is None else new_lens,
                weights.new_empty((b, h, new_width * cache.page)) if new_weights is None
                else new_weights,
                lens.new_empty((need,), dtype=torch.uint8) if need else workspace)

    kept, new_lens, new_weights, workspace = _made(stream, allocate)
    _check(lib().xattn_cache_evict(cache._ref, b, _ptr(table), width, _ptr(lens), _ptr(weights),
                                   budget, recent, _ptr(new_table), new_width, _ptr(kept),
                                   _ptr(new_lens), _ptr(new_weights), _ptr(workspace),
                                   0 if workspace is None else workspace.numel(),
                                   _handle(stream, at)))
    return kept, new_lens, new_weights
