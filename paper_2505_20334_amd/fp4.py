"""Binding of the paged 4-bit cache (``include/laq_fp4.h``) -- argument marshalling only, as in ``binding``.

A cache is four byte tensors (``Fp4Cache``), a pool of blocks that requests own through a block table; the free blocks,
the table, the requests' lengths and the slots of new rows are int32 tensors on the GPU, kept by ``laq_block_map``.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional, Sequence, Tuple

import torch

from . import binding
from .binding import LaqError, _aligned, _budget_array, _cache, _dev, _dtype_code, _empty, _Fp4Cache, _out, _shape, _stream, load_library


class Fp4Cache(NamedTuple):
    """Codes [n_blocks, Hkv, block_rows, d / 2] and scales [n_blocks, Hkv, block_rows, d / 32] of K and of V, uint8 on the GPU.
    Dense, or views of that shape whose last dimension is contiguous (token-major blocks: allocate [n_blocks, block_rows, Hkv, ...]
    and hand over .transpose(1, 2)); K and V have the same strides."""
    k: torch.Tensor
    k_scale: torch.Tensor
    v: torch.Tensor
    v_scale: torch.Tensor


def laq_fp4_cache(n_blocks: int, Hkv: int, block_rows: int, d: int, device="cuda:0") -> Fp4Cache:
    """A cache of zeros."""
    if d % 32 or not 32 <= d <= 256 or block_rows % 16 or min(n_blocks, Hkv, block_rows) < 1:
        raise ValueError("d is a multiple of 32 up to 256, block_rows a multiple of 16")
    return Fp4Cache(*(torch.zeros(n_blocks, Hkv, block_rows, w, dtype=torch.uint8, device=device) for w in (d // 2, d // 32, d // 2, d // 32)))


def laq_block_pool(n_blocks: int, device="cuda:0") -> Tuple[torch.Tensor, torch.Tensor]:
    """(free_blocks, state) of laq_block_map with all blocks free; block 0 is taken first."""
    free = torch.arange(n_blocks - 1, -1, -1, dtype=torch.int32, device=device)
    return free, torch.tensor([n_blocks, 0, 0, 0], dtype=torch.int32, device=device)


def _here(t: torch.Tensor) -> None:
    if t.device.index != torch._C._cuda_getDevice():
        raise ValueError("the tensors live on %s, which is not the current device" % t.device)


def _int32(x, name: str) -> int:
    x = int(x)
    if not -(1 << 31) <= x < 1 << 31:
        raise ValueError("%s is a number of 32 bits" % name)
    return x


def _ints(t: torch.Tensor, name: str, like: torch.Tensor, numel: int) -> torch.Tensor:
    """A dense int32 tensor of at least `numel` entries on the device of `like`."""
    if t.device.type != "cuda":
        raise ValueError("%s must live on the GPU" % name)
    if t.device != like.device or t.dtype != torch.int32 or not t.is_contiguous() or t.numel() < numel:
        raise ValueError("%s must be a dense int32 tensor of at least %d entries on %s" % (name, numel, like.device))
    return t


def _fp4(cache: Fp4Cache) -> _Fp4Cache:
    k, k_scale, v, v_scale = cache
    if k.device.type != "cuda":
        raise ValueError("the cache must live on the GPU")
    _here(k)
    n_blocks, Hkv, block_rows, half = k.shape
    for t, name, like in ((k, "k", k), (v, "v", k), (k_scale, "k_scale", k_scale), (v_scale, "v_scale", k_scale)):
        want = (n_blocks, Hkv, block_rows, half if like is k else half // 16)
        if t.dtype != torch.uint8 or t.device != k.device or t.shape != want or t.stride() != like.stride() or t.stride(3) != 1:
            raise ValueError("%s must be uint8 %s on %s with contiguous rows, K and V with the same strides" % (name, want, k.device))
    strides = (0,) * 6 if k.is_contiguous() and k_scale.is_contiguous() else k.stride()[:3] + k_scale.stride()[:3]
    return _Fp4Cache(k.data_ptr(), k_scale.data_ptr(), v.data_ptr(), v_scale.data_ptr(), n_blocks, Hkv, block_rows, 2 * half, *strides)


def _tokens(t: torch.Tensor, name: str, heads: Optional[int], d: int) -> Tuple[int, int]:
    """A tensor [tokens, heads, d] on the GPU with contiguous rows: its (token, head) strides in elements, zeros if it is dense."""
    if t.device.type != "cuda":
        raise ValueError("%s must live on the GPU" % name)
    if t.dim() != 3 or t.shape[2] != d or (heads is not None and t.shape[1] != heads) or t.stride(2) != 1:
        raise ValueError("%s must be [tokens, %s, %d] with contiguous rows" % (name, heads if heads is not None else "heads", d))
    _aligned(t, name)
    return (0, 0) if t.is_contiguous() else (t.stride(0), t.stride(1))


def laq_block_map(add: torch.Tensor, rows: torch.Tensor, block_table: torch.Tensor, free_blocks: torch.Tensor, state: torch.Tensor,
                  block_rows: int, start: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None, n_slots: Optional[int] = None,
                  stream=None) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """add, rows [n], block_table [n, blocks per request], free_blocks [n_blocks] and state [4] (see laq_block_pool), all int32 on the
    GPU; rows, block_table, free_blocks and state are updated in place.  Returns (start [n + 1], slots [n_slots]), made if n_slots (the
    batch's rows, padding included) is given and they are not; None where they are not wanted.  state[0]: free blocks, state[1]: requests
    refused for want of blocks or table entries (rows as before, slots -1)."""
    lib = binding._lib or load_library()
    if stream is None and binding._native is not None:
        got = binding._native.block_map(add, rows, block_table, free_blocks, state, block_rows, start, slots, n_slots)
        if got is not None:
            if type(got) is int:
                raise LaqError(got, "laq_block_map")
            return got
    n = add.numel()
    _ints(add, "add", rows, n), _ints(rows, "rows", rows, n), _ints(state, "state", rows, 4), _ints(free_blocks, "free_blocks", rows, 1)
    if block_table.dim() != 2 or block_table.shape[0] != n or rows.numel() != n:
        raise ValueError("add and rows are [n], block_table is [n, blocks per request]")
    _ints(block_table, "block_table", rows, n)
    _here(rows)
    if slots is None and n_slots is not None:
        slots = _empty(stream, n_slots, dtype=torch.int32, device=rows.device)
    if start is None and n_slots is not None:
        start = _empty(stream, n + 1, dtype=torch.int32, device=rows.device)
    if slots is not None:
        _ints(slots, "slots", rows, n_slots or 0)
    if start is not None:
        _ints(start, "start", rows, n + 1)
    rc = lib.laq_block_map(n, _int32(block_rows, "block_rows"), free_blocks.numel(), block_table.shape[1], add.data_ptr(), rows.data_ptr(), block_table.data_ptr(),
                           free_blocks.data_ptr(), state.data_ptr(), start.data_ptr() if start is not None else None,
                           slots.data_ptr() if slots is not None else None, slots.numel() if slots is not None else 0, _stream(stream))
    if rc != 0:
        raise LaqError(rc, "laq_block_map")
    return start, slots


def laq_fp4_store(cache: Fp4Cache, k: Optional[torch.Tensor], v: Optional[torch.Tensor], slots: torch.Tensor, stream=None) -> None:
    """k, v [tokens, Hkv, d] (or one of them; views with contiguous rows, e.g. of a fused projection, are fine) into the rows slots [tokens]
    of the cache; tokens whose slot is -1 are left out."""
    lib = binding._lib or load_library()
    if stream is None and binding._native is not None:
        got = binding._native.fp4_store(cache, k, v, slots)
        if got is not None:
            if got is not True:
                raise LaqError(got, "laq_fp4_store")
            return
    c = _fp4(cache)
    like = k if k is not None else v
    if like is None:
        raise ValueError("k or v is needed")
    strides = _tokens(like, "k" if k is not None else "v", c.Hkv, c.d)
    if k is not None and v is not None and (v.shape != k.shape or v.dtype != k.dtype or _tokens(v, "v", c.Hkv, c.d) != strides):
        raise ValueError("k / v mismatch (shape, dtype or strides)")
    _ints(slots, "slots", cache.k, like.shape[0])
    if like.device != cache.k.device:
        raise ValueError("k and v must live on %s" % cache.k.device)
    rc = lib.laq_fp4_store(ctypes.byref(c), _dtype_code(like), like.shape[0], k.data_ptr() if k is not None else None,
                           v.data_ptr() if v is not None else None, *strides, slots.data_ptr(), _stream(stream))
    if rc != 0:
        raise LaqError(rc, "laq_fp4_store")


def laq_fp4_compact(cache: Fp4Cache, k: torch.Tensor, v: Optional[torch.Tensor], idx: torch.Tensor, budget: Sequence[int], slots: torch.Tensor,
                    stream=None, block_table: Optional[torch.Tensor] = None, L: Optional[int] = None) -> None:
    """k, v [n, Hkv, L, d] + packed idx (as laq_select writes it) -> the rows slots of the cache: laq_compact into the 4-bit cache.
    slots: one entry per kept row of an instance, for all its KV heads, instance after instance (laq_block_map with add = min(budget, L));
    block_table / L: k, v are paged caches, as for laq_compact."""
    lib = binding._lib or load_library()
    if stream is None and block_table is None and L is None and binding._native is not None:
        got = binding._native.fp4_compact(cache, k, v, idx, budget, slots)
        if got is not None:
            if got is not True:
                raise LaqError(got, "laq_fp4_compact")
            return
    c = _fp4(cache)
    _dev(idx, "idx")
    n, Hkv, L, d, kvs, paged = _cache(k, "k", block_table, L)
    if Hkv != c.Hkv or d != c.d or k.device != cache.k.device:
        raise ValueError("k and the cache differ in KV heads, head size or device")
    if v is not None:
        if v.shape != k.shape or v.dtype != k.dtype or v.stride() != k.stride():
            raise ValueError("k / v mismatch (shape, dtype or strides)")
        _aligned(v, "v")
    _aligned(k, "k")
    total, _ = binding.packed_rows(budget, 1, L)
    _ints(idx, "idx", k, total * Hkv), _ints(slots, "slots", k, total)
    sh = _shape(n, Hkv, Hkv, d, L, 1, _dtype_code(k), 0.0, None, 0, "max", kvs, paged)
    rc = lib.laq_fp4_compact(ctypes.byref(sh), k.data_ptr(), v.data_ptr() if v is not None else None, idx.data_ptr(), _budget_array(budget, n),
                             ctypes.byref(c), slots.data_ptr(), _stream(stream))
    if rc != 0:
        raise LaqError(rc, "laq_fp4_compact")


def laq_fp4_load(cache: Fp4Cache, slots: torch.Tensor, dtype: torch.dtype = torch.bfloat16, k: Optional[torch.Tensor] = None,
                 v: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Rows slots [tokens] of the cache as (k, v) [tokens, Hkv, d] of type dtype (made if not given); rows whose slot is -1 are 0."""
    lib = binding._lib or load_library()
    if stream is None and binding._native is not None:
        got = binding._native.fp4_load(cache, slots, dtype, k, v)
        if got is not None:
            if type(got) is int:
                raise LaqError(got, "laq_fp4_load")
            return got
    c = _fp4(cache)
    _ints(slots, "slots", cache.k, 0)
    T = slots.numel()
    out = []
    for t, name in ((k, "k"), (v, "v")):
        _out(t, name, dtype, T * c.Hkv * c.d, cache.k)
        out.append(t if t is not None else _empty(stream, T, c.Hkv, c.d, dtype=dtype, device=cache.k.device))
    rc = lib.laq_fp4_load(ctypes.byref(c), _dtype_code(out[0]), T, slots.data_ptr(), out[0].data_ptr(), out[1].data_ptr(), _stream(stream))
    if rc != 0:
        raise LaqError(rc, "laq_fp4_load")
    return out[0], out[1]


def laq_fp4_attention_workspace_bytes(cache: Fp4Cache, Hq: int, dtype: torch.dtype, n: int, n_tokens: int, max_rows: int) -> int:
    code = binding.LAQ_F32 if dtype == torch.float32 else binding.LAQ_BF16
    return int(load_library().laq_fp4_attention_workspace_bytes(ctypes.byref(_fp4(cache)), _int32(Hq, "Hq"), code, _int32(n, "n"), int(n_tokens),
                                                               _int32(max_rows, "max_rows")))


def laq_fp4_attention(q: torch.Tensor, cache: Fp4Cache, block_table: torch.Tensor, rows: torch.Tensor, start: Optional[torch.Tensor] = None,
                      max_rows: Optional[int] = None, scale: float = 0.0, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                      want_lse: bool = False, ws: Optional[torch.Tensor] = None, split: bool = True, stream=None):
    """q [tokens, Hq, d] (views with contiguous rows are fine) -> out [tokens, Hq, d] in q's dtype: each token's attention over the rows of its request
    up to its own.  block_table [n, blocks per request], rows [n] (rows held, the tokens' own included) and start [n + 1] (tokens
    start[i] .. start[i+1]-1 are those of request i; None: one token per request) as laq_block_map keeps them.  max_rows: a bound on the
    lengths that the launch is planned with (None: what the table holds).  want_lse (or an lse buffer, fp32 [tokens, Hq]): returns
    (out, lse), lse the logarithm of the sum of the exponentials.  split: let the library spread long rows over several workgroups (a workspace of
    laq_fp4_attention_workspace_bytes is made if ws is None)."""
    lib = binding._lib or load_library()
    if stream is None and binding._native is not None:
        got = binding._native.fp4_attention(q, cache, block_table, rows, start, max_rows, scale, out, lse, want_lse, ws, split)
        if got is not None:
            if type(got) is int:
                raise LaqError(got, "laq_fp4_attention")
            return got
    c = _fp4(cache)
    strides = _tokens(q, "q", None, c.d)
    T, Hq, d = q.shape
    if block_table.dim() != 2 or q.device != cache.k.device:
        raise ValueError("block_table is [n, blocks per request], q lives on %s" % cache.k.device)
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
        need = int(lib.laq_fp4_attention_workspace_bytes(ctypes.byref(c), Hq, code, n, T, most))
        if need:
            ws = _empty(stream, need, dtype=torch.uint8, device=q.device)
    rc = lib.laq_fp4_attention(ctypes.byref(c), Hq, code, float(scale), n, T, start.data_ptr() if start is not None else None, q.data_ptr(), *strides,
                               block_table.data_ptr(), width, rows.data_ptr(), most, out.data_ptr(), lse.data_ptr() if lse is not None else None,
                               ws.data_ptr() if ws is not None else None, ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream))
    if rc != 0:
        raise LaqError(rc, "laq_fp4_attention")
    return (out, lse) if lse is not None else out
