"""Binding of rotary positions and the paged cache in 32, 16 or 8 bits (``include/laq_cache.h``) -- argument marshalling only, as in ``binding``.

A cache is a pool of blocks (``PagedCache``) that requests own through a block table; the table, the requests' lengths and the slots of new rows
are int32 tensors on the GPU, kept by ``laq_block_map``.
"""
from __future__ import annotations

import ctypes
import math
from typing import NamedTuple, Optional, Sequence, Tuple

import torch

from . import binding
from .binding import LaqError, _aligned, _budget_array, _cache, _dev, _dtype_code, _empty, _Heads, _out, _PagedCache, _RopePlan, _shape, _stream, load_library
from .fp4 import _here, _int32, _ints, _tokens

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float8_e4m3fn: 2}
_LAYOUTS = ("half", "interleaved")


class PagedCache(NamedTuple):
    """K and V [n_blocks, Hkv, block_rows, d] (fp32, bf16 or float8_e4m3fn) on the GPU and, for float8_e4m3fn, the rows' scales [n_blocks, Hkv,
    block_rows] (uint8, dense; otherwise None).  K and V dense, or views of that shape whose last dimension is contiguous (token-major blocks:
    allocate [n_blocks, block_rows, Hkv, d] and hand over .transpose(1, 2)), both with the same strides."""
    k: torch.Tensor
    k_scale: Optional[torch.Tensor]
    v: torch.Tensor
    v_scale: Optional[torch.Tensor]


class Rope(NamedTuple):
    """Rotary positions: inv_freq, fp32 [rot / 2] on the GPU, the angle per position of each pair of the first rot numbers of a head (see
    laq_rope_frequencies); layout "half" (pairs i, i + rot / 2) or "interleaved" (2i, 2i + 1); mscale: factor of what is rotated."""
    inv_freq: torch.Tensor
    layout: str = "half"
    mscale: float = 1.0


def laq_rope_frequencies(rot: int, base: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0, trained: int = 0, slow: float = 1.0,
                         fast: float = 32.0, device="cuda:0") -> torch.Tensor:
    """inv_freq of Rope, base^(-2i / rot), scaled for contexts `factor` times as long as those that a model was trained with:
    "linear"  every frequency divided by factor (positions interpolated);
    "base"    the base raised so that the slowest pair's frequency is divided by factor and the fastest one's stays: base * factor^(rot / (rot - 2));
    "parts"   pairs that turn at most `slow` times within `trained` positions divided by factor, those that turn at least `fast` times as they are, those
              between in proportion to their number of turns;
    "ramp"    the same, those between in proportion to their index, from the (rounded) index that turns `fast` times to the one that turns `slow` times."""
    if rot < 2 or rot % 2 or not base > 1.0 or not factor >= 1.0:
        raise ValueError("rot is even, base above 1, factor at least 1")
    i = torch.arange(0, rot, 2, dtype=torch.float64)
    if scaling == "base":
        if rot < 4:
            raise ValueError("scaling the base takes two pairs at least")
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-i / rot)
    if scaling == "linear":
        f = f / factor
    elif scaling in ("parts", "ramp"):
        if trained < 1 or not 0 < slow < fast:
            raise ValueError("trained is the number of positions a model was trained with, slow and fast numbers of turns, slow below fast")
        if scaling == "parts":
            stay = ((f * trained / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
        else:
            at = [rot * math.log(trained / (turns * 2 * math.pi)) / (2 * math.log(base)) for turns in (fast, slow)]
            low, high = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
            stay = 1 - ((i / 2 - low) / max(high - low, 0.001)).clamp(0, 1)
        f = f / factor * (1 - stay) + f * stay
    elif scaling not in (None, "base"):
        raise ValueError("scaling is None, 'linear', 'base', 'parts' or 'ramp'")
    return f.float().to(device)


def laq_cache(n_blocks: int, Hkv: int, block_rows: int, d: int, dtype: torch.dtype = torch.bfloat16, device="cuda:0") -> PagedCache:
    """A cache of zeros."""
    if dtype not in _TYPES:
        raise TypeError("a cache is fp32, bf16 or float8_e4m3fn, not %s" % dtype)
    if d % 8 or not 8 <= d <= 256 or block_rows % 16 or min(n_blocks, Hkv, block_rows) < 1:
        raise ValueError("d is a multiple of 8 up to 256, block_rows a multiple of 16")
    planes = []
    for _ in range(2):
        if dtype == torch.float8_e4m3fn:
            planes += [torch.zeros(n_blocks, Hkv, block_rows, d, dtype=torch.uint8, device=device).view(dtype),
                       torch.zeros(n_blocks, Hkv, block_rows, dtype=torch.uint8, device=device)]
        else:
            planes += [torch.zeros(n_blocks, Hkv, block_rows, d, dtype=dtype, device=device), None]
    return PagedCache(*planes)


def _paged(cache: PagedCache) -> _PagedCache:
    k, k_scale, v, v_scale = cache
    if k.device.type != "cuda":
        raise ValueError("the cache must live on the GPU")
    _here(k)
    if k.dtype not in _TYPES:
        raise TypeError("a cache is fp32, bf16 or float8_e4m3fn, not %s" % k.dtype)
    if k.dim() != 4 or k.stride(3) != 1:
        raise ValueError("k must be [n_blocks, Hkv, block_rows, d] with contiguous rows")
    n_blocks, Hkv, block_rows, d = k.shape
    if v.dtype != k.dtype or v.device != k.device or v.shape != k.shape or v.stride() != k.stride():
        raise ValueError("v must be %s %s on %s with the strides of k" % (k.dtype, tuple(k.shape), k.device))
    scales = [0, 0]
    if k.dtype == torch.float8_e4m3fn:
        for i, (t, name) in enumerate(((k_scale, "k_scale"), (v_scale, "v_scale"))):
            if t is None or t.dtype != torch.uint8 or t.device != k.device or t.shape != k.shape[:3] or not t.is_contiguous():
                raise ValueError("%s must be dense uint8 %s on %s" % (name, tuple(k.shape[:3]), k.device))
            scales[i] = t.data_ptr()
    elif k_scale is not None or v_scale is not None:
        raise ValueError("only a cache of float8_e4m3fn has scales")
    strides = (0, 0, 0) if k.is_contiguous() else k.stride()[:3]
    return _PagedCache(k.data_ptr(), v.data_ptr(), scales[0], scales[1], n_blocks, Hkv, block_rows, d, _TYPES[k.dtype], *strides)


def _heads(t: Optional[torch.Tensor], name: str, heads: Optional[int], d: int, like: torch.Tensor, n_tokens: int) -> Optional[_Heads]:
    """A tensor [n_tokens, heads, d] as the library takes it; None: none."""
    if t is None:
        return None
    strides = _tokens(t, name, heads, d)
    if t.dtype != like.dtype or t.device != like.device or t.shape[0] != n_tokens:
        raise ValueError("%s must be %s [%d, heads, %d] on %s" % (name, like.dtype, n_tokens, d, like.device))
    return _Heads(t.data_ptr(), t.shape[1], *strides)


def _ref(x):
    return ctypes.byref(x) if x is not None else None


def _plan(rope: Rope, like: torch.Tensor) -> _RopePlan:
    f = rope.inv_freq
    if f.device != like.device or f.dtype != torch.float32 or f.dim() != 1 or not f.is_contiguous():
        raise ValueError("inv_freq must be a dense fp32 [rot / 2] tensor on %s" % like.device)
    if rope.layout not in _LAYOUTS:
        raise ValueError("layout is 'half' or 'interleaved'")
    return _RopePlan(f.data_ptr(), 2 * f.numel(), _LAYOUTS.index(rope.layout), float(rope.mscale))


def laq_rope(q: Optional[torch.Tensor], k: Optional[torch.Tensor], positions: torch.Tensor, rope: Rope, q_out: Optional[torch.Tensor] = None,
             k_out: Optional[torch.Tensor] = None, stream=None) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """q [tokens, Hq, d] and k [tokens, Hkv, d] (one of them may be None; views with contiguous rows, e.g. of a fused projection, are fine)
    rotated to positions [tokens] (int32).  Returns (q_out, k_out), made dense if not given; an input may be its own output."""
    lib = binding._lib or load_library()
    if stream is None and binding._native is not None:
        got = binding._native.rope(q, k, positions, rope, q_out, k_out)
        if got is not None:
            if type(got) is int:
                raise LaqError(got, "laq_rope")
            return got
    like = q if q is not None else k
    if like is None:
        raise ValueError("q or k is needed")
    if like.dim() != 3:
        raise ValueError("q and k are [tokens, heads, d]")
    T, _, d = like.shape
    code = _dtype_code(like)
    plan = _plan(rope, like)
    found = []
    for x, out, name in ((q, q_out, "q"), (k, k_out, "k")):
        a = _heads(x, name, None, d, like, T)
        if x is None and out is not None:
            raise ValueError("%s_out without %s" % (name, name))
        if x is not None and out is None:
            out = _empty(stream, *x.shape, dtype=x.dtype, device=x.device)
        found.append((out, a, _heads(out, name + "_out", a.heads if a else None, d, like, T)))
    _here(like)
    _ints(positions, "positions", like, T)
    rc = lib.laq_rope(ctypes.byref(plan), code, T, d, _ref(found[0][1]), _ref(found[1][1]), positions.data_ptr(), _ref(found[0][2]), _ref(found[1][2]),
                      _stream(stream))
    if rc != 0:
        raise LaqError(rc, "laq_rope")
    return found[0][0], found[1][0]


def laq_cache_append(cache: PagedCache, k: Optional[torch.Tensor], v: Optional[torch.Tensor], slots: torch.Tensor, q: Optional[torch.Tensor] = None,
                     positions: Optional[torch.Tensor] = None, rope: Optional[Rope] = None, q_out: Optional[torch.Tensor] = None,
                     stream=None) -> Optional[torch.Tensor]:
    """k, v [tokens, Hkv, d] (or one of them; views with contiguous rows are fine; fp32 or bf16, whatever the cache is) into the rows slots [tokens] of the
    cache; tokens whose slot is -1 are left out.  With rope and positions [tokens] k is rotated on the way, and q [tokens, Hq, d], if given, into
    q_out (made if not given; q itself is fine), which is returned."""
    lib = binding._lib or load_library()
    if stream is None and binding._native is not None:
        got = binding._native.cache_append(cache, k, v, slots, q, positions, rope, q_out)
        if got is not None:
            if type(got) is int:
                raise LaqError(got, "laq_cache_append")
            return got[0]
    c = _paged(cache)
    like = k if k is not None else v
    if like is None:
        raise ValueError("k or v is needed")
    if like.dim() != 3:
        raise ValueError("k and v are [tokens, Hkv, d]")
    T = like.shape[0]
    code = _dtype_code(like)
    if like.device != cache.k.device:
        raise ValueError("k and v must live on %s" % cache.k.device)
    hk, hv = _heads(k, "k", c.Hkv, c.d, like, T), _heads(v, "v", c.Hkv, c.d, like, T)
    _ints(slots, "slots", like, T)
    plan = None
    if rope is not None:
        plan = _plan(rope, like)
        if positions is None:
            raise ValueError("rope needs positions")
        _ints(positions, "positions", like, T)
    elif q is not None or positions is not None:
        raise ValueError("q and positions are given with rope")
    if q is None and q_out is not None:
        raise ValueError("q_out without q")
    hq = _heads(q, "q", None, c.d, like, T)
    if q is not None and q_out is None:
        q_out = _empty(stream, *q.shape, dtype=q.dtype, device=q.device)
    ho = _heads(q_out, "q_out", hq.heads if hq else None, c.d, like, T)
    rc = lib.laq_cache_append(ctypes.byref(c), code, T, _ref(hk), _ref(hv), slots.data_ptr(), _ref(plan), positions.data_ptr() if plan is not None else None,
                              _ref(hq), _ref(ho), _stream(stream))
    if rc != 0:
        raise LaqError(rc, "laq_cache_append")
    return q_out


def laq_cache_compact(cache: PagedCache, k: torch.Tensor, v: Optional[torch.Tensor], idx: torch.Tensor, budget: Sequence[int], slots: torch.Tensor,
                      stream=None, block_table: Optional[torch.Tensor] = None, L: Optional[int] = None) -> None:
    """k, v [n, Hkv, L, d] + packed idx (as laq_select writes it) -> the rows slots of the cache: laq_compact into the paged cache.
    slots: one entry per kept row of an instance, for all its KV heads, instance after instance (laq_block_map with add = min(budget, L));
    block_table / L: k, v are paged caches, as for laq_compact."""
    lib = binding._lib or load_library()
    if stream is None and block_table is None and L is None and binding._native is not None:
        got = binding._native.cache_compact(cache, k, v, idx, budget, slots)
        if got is not None:
            if got is not True:
                raise LaqError(got, "laq_cache_compact")
            return
    c = _paged(cache)
    _dev(idx, "idx")
    n, Hkv, L, d, kvs, paged = _cache(k, "k", block_table, L)
    if Hkv != c.Hkv or d != c.d or k.device != cache.k.device:
        raise ValueError("k and the cache differ in KV heads, head size or device")
    if v is not None:
        if v.shape != k.shape or v.dtype != k.dtype or v.stride() != k.stride() or v.device != k.device:
            raise ValueError("k / v mismatch (shape, dtype, strides or device)")
        _aligned(v, "v")
    _aligned(k, "k")
    total, _ = binding.packed_rows(budget, 1, L)
    _ints(idx, "idx", k, total * Hkv), _ints(slots, "slots", k, total)
    sh = _shape(n, Hkv, Hkv, d, L, 1, _dtype_code(k), 0.0, None, 0, "max", kvs, paged)
    rc = lib.laq_cache_compact(ctypes.byref(sh), k.data_ptr(), v.data_ptr() if v is not None else None, idx.data_ptr(), _budget_array(budget, n),
                               ctypes.byref(c), slots.data_ptr(), _stream(stream))
    if rc != 0:
        raise LaqError(rc, "laq_cache_compact")


def laq_cache_load(cache: PagedCache, slots: torch.Tensor, dtype: torch.dtype = torch.bfloat16, k: Optional[torch.Tensor] = None,
                   v: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Rows slots [tokens] of the cache as (k, v) [tokens, Hkv, d] of type dtype (made if not given); rows whose slot is -1 are 0."""
    lib = binding._lib or load_library()
    if stream is None and binding._native is not None:
        got = binding._native.cache_load(cache, slots, dtype, k, v)
        if got is not None:
            if type(got) is int:
                raise LaqError(got, "laq_cache_load")
            return got
    c = _paged(cache)
    _ints(slots, "slots", cache.k, 0)
    T = slots.numel()
    out = []
    for t, name in ((k, "k"), (v, "v")):
        _out(t, name, dtype, T * c.Hkv * c.d, cache.k)
        out.append(t if t is not None else _empty(stream, T, c.Hkv, c.d, dtype=dtype, device=cache.k.device))
    rc = lib.laq_cache_load(ctypes.byref(c), _dtype_code(out[0]), T, slots.data_ptr(), out[0].data_ptr(), out[1].data_ptr(), _stream(stream))
    if rc != 0:
        raise LaqError(rc, "laq_cache_load")
    return out[0], out[1]


def laq_cache_attention_workspace_bytes(cache: PagedCache, Hq: int, dtype: torch.dtype, n: int, n_tokens: int, max_rows: int) -> int:
    code = binding.LAQ_F32 if dtype == torch.float32 else binding.LAQ_BF16
    return int(load_library().laq_cache_attention_workspace_bytes(ctypes.byref(_paged(cache)), _int32(Hq, "Hq"), code, _int32(n, "n"), int(n_tokens),
                                                                 _int32(max_rows, "max_rows")))


def laq_cache_attention(q: torch.Tensor, cache: PagedCache, block_table: torch.Tensor, rows: torch.Tensor, start: Optional[torch.Tensor] = None,
                        max_rows: Optional[int] = None, scale: float = 0.0, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                        want_lse: bool = False, ws: Optional[torch.Tensor] = None, split: bool = True, stream=None):
    """q [tokens, Hq, d] (views with contiguous rows are fine; bf16 with caches of bf16 and float8_e4m3fn, fp32 with all) -> out [tokens, Hq, d] in q's
    dtype: each token's attention over the rows of its request up to its own.  block_table [n, blocks per request], rows [n] (rows held, the tokens' own
    included) and start [n + 1] (tokens start[i] .. start[i+1]-1 are those of request i; None: one token per request) as laq_block_map keeps them.
    max_rows: a bound on the lengths that the launch is planned with (None: what the table holds).  want_lse (or an lse buffer, fp32 [tokens, Hq]):
    returns (out, lse), lse the logarithm of the sum of the exponentials.  split: let the library spread long rows over several workgroups (a
    workspace of laq_cache_attention_workspace_bytes is made if ws is None)."""
    lib = binding._lib or load_library()
    if stream is None and binding._native is not None:
        got = binding._native.cache_attention(q, cache, block_table, rows, start, max_rows, scale, out, lse, want_lse, ws, split)
        if got is not None:
            if type(got) is int:
                raise LaqError(got, "laq_cache_attention")
            return got
    c = _paged(cache)
    if q.dim() != 3:
        raise ValueError("q is [tokens, Hq, d]")
    T, Hq, d = q.shape
    if block_table.dim() != 2 or q.device != cache.k.device:
        raise ValueError("block_table is [n, blocks per request], q lives on %s" % cache.k.device)
    hq = _heads(q, "q", None, c.d, q, T)
    n, width = block_table.shape
    _ints(block_table, "block_table", q, n), _ints(rows, "rows", q, n)
    if start is not None:
        _ints(start, "start", q, n + 1)
    elif T != n:
        raise ValueError("without start there is one token per request")
    most = max(1, _int32(width * c.block_rows if max_rows is None else max_rows, "max_rows"))
    _out(out, "out", q.dtype, T * Hq * d, q)
    _out(lse, "lse", torch.float32, T * Hq, q)
    if out is None:
        out = _empty(stream, T, Hq, d, dtype=q.dtype, device=q.device)
    if lse is None and want_lse:
        lse = _empty(stream, T, Hq, dtype=torch.float32, device=q.device)
    code = _dtype_code(q)
    if ws is not None and (ws.device != q.device or not ws.is_contiguous()):
        raise ValueError("ws must be a dense tensor on %s" % q.device)
    if not split:
        ws = None
    elif ws is None:
        need = int(lib.laq_cache_attention_workspace_bytes(ctypes.byref(c), Hq, code, n, T, most))
        if need:
            ws = _empty(stream, need, dtype=torch.uint8, device=q.device)
    rc = lib.laq_cache_attention(ctypes.byref(c), code, float(scale), n, T, start.data_ptr() if start is not None else None, ctypes.byref(hq),
                                 block_table.data_ptr(), width, rows.data_ptr(), most, out.data_ptr(), lse.data_ptr() if lse is not None else None,
                                 ws.data_ptr() if ws is not None else None, ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream))
    if rc != 0:
        raise LaqError(rc, "laq_cache_attention")
    return (out, lse) if lse is not None else out
