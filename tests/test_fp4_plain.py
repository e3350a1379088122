"""The plain forms that the 4-bit cache is tested against, pinned; and the refusals of its calls (no GPU needed)."""
import ctypes
import math
import random

import pytest
import torch

import paper_2505_20334_amd as laq
from paper_2505_20334_amd import binding
from fp4_plain import GRID, Allocator, quantise, quantise_block, values

INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3
FAKE = ctypes.c_void_p(0x1000)


def test_the_format_of_a_block_by_its_definition():
    rng = random.Random(5)
    blocks = [[rng.gauss(0, 10.0 ** rng.randint(-20, 20)) for _ in range(32)] for _ in range(200)]
    blocks += [[0.0] * 32, [-0.0] * 32, [2.0 ** -101] * 32, [2.0 ** -102] * 32, [3.38e38] + [1e37] * 31, [math.inf] + [1.0] * 31, [math.nan] + [0.0] * 31]
    for most in (1.0, 1.75, math.nextafter(1.75, 0), 7.0, 6.999):             # the border of the scale
        blocks.append([most] + [most * rng.uniform(-1, 1) for _ in range(31)])
    blocks.append([6.0] + [s * t for t in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0) for s in (1, -1)] + [0.0] * 17)      # ties
    x = torch.tensor(blocks, dtype=torch.float64)
    codes, scales = quantise(x)
    for row, block in enumerate(blocks):
        s, c = quantise_block(block)
        assert scales[row, 0] == s
        assert [int(b) & 15 if j % 2 == 0 else int(b) >> 4 for b in codes[row] for j in (0, 1)] == c
    assert [v for v in values(codes, scales)[-1, 1:15:2].tolist()] == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0]
    # the grid's steps are 2 at most from 4 to 7 (where 6 is the last code), so no number is off by more than 1 where the largest is 5 or more,
    # and by less of a smaller largest one; not beyond 7 * 2^125, where the scale ends
    finite = torch.isfinite(x).all(-1) & (x.abs().amax(-1) > 2.0 ** -98) & (x.abs().amax(-1) < 7 * 2.0 ** 125)
    err = (values(codes, scales) - x).abs()[finite] / x.abs().amax(-1, keepdim=True)[finite]
    assert err.max() <= 1 / 5
    assert quantise_block([6.0] * 32) == (127, [7] * 32) and quantise_block([7.0] * 32) == (128, [6] * 32) and len(GRID) == 8


def test_the_allocator_gives_back_what_it_took():
    a = Allocator(3, 20, 8, 16, range(20))
    before = list(a.free)
    start, slots = a.step([17, 0, 33], 60)
    assert start == [0, 17, 17, 50] and slots[50:] == [-1] * 10 and a.rows == [17, 0, 33]
    assert slots[:17] == [19 * 16 + i for i in range(16)] + [18 * 16] and len(set(slots[:50])) == 50
    a.step([-17, 0, -33], 0)
    assert a.free == before and a.rows == [0, 0, 0]
    assert a.step([16 * 8 + 1, 0, 0], 3)[1] == [-1, -1, -1] and a.refused == 1           # more than the table holds
    a.step([16 * 8, 16 * 8, 16 * 8], 0)                                                  # 24 blocks of 20
    assert a.rows == [128, 128, 0] and a.refused == 1 and len(a.free) == 4


def _cache(**kw):
    base = dict(k=0x1000, k_scale=0x1000, v=0x1000, v_scale=0x1000, n_blocks=8, Hkv=2, block_rows=16, d=128, stride_block=0, stride_head=0, stride_row=0,
                scale_stride_block=0, scale_stride_head=0, scale_stride_row=0)
    base.update(kw)
    return binding._Fp4Cache(*[base[f] for f, _ in binding._Fp4Cache._fields_])


BAD_CACHES = [dict(n_blocks=0), dict(Hkv=0), dict(block_rows=0), dict(block_rows=24), dict(d=16), dict(d=48), dict(d=288), dict(n_blocks=1 << 27),
              dict(k=None), dict(k_scale=None), dict(k=0x1008), dict(v=None), dict(v=0x1004), dict(stride_row=64),
              dict(stride_block=-16, stride_head=1024, stride_row=64, scale_stride_block=128, scale_stride_head=64, scale_stride_row=4),
              dict(stride_block=2048, stride_head=1024, stride_row=48, scale_stride_block=128, scale_stride_head=64, scale_stride_row=4),
              dict(stride_block=2048, stride_head=1024, stride_row=72, scale_stride_block=128, scale_stride_head=64, scale_stride_row=4),
              dict(stride_block=2048, stride_head=1024, stride_row=64, scale_stride_block=128, scale_stride_head=64, scale_stride_row=3)]


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_caches_that_are_refused(bad):
    lib = laq.load_library()
    c = ctypes.byref(_cache(**bad))
    assert lib.laq_fp4_store(c, 1, 4, FAKE, FAKE, 0, 0, FAKE, None) == INVALID
    assert lib.laq_fp4_load(c, 1, 4, FAKE, FAKE, FAKE, None) == INVALID
    assert lib.laq_fp4_attention(c, 8, 1, 0.0, 2, 2, None, FAKE, 0, 0, FAKE, 4, FAKE, 64, FAKE, None, None, 0, None) == INVALID
    sh = binding._shape(1, 2, 2, bad.get("d", 128), 64, 1, 1, 0.0, None, 0)
    assert lib.laq_fp4_compact(ctypes.byref(sh), FAKE, FAKE, FAKE, (ctypes.c_int32 * 1)(8), c, FAKE, None) == INVALID


def test_arguments_that_are_refused():
    lib = laq.load_library()
    c = ctypes.byref(_cache())
    odd = ctypes.c_void_p(0x1008)
    for args in ((2, 4, FAKE, FAKE, 0, 0, FAKE), (1, -1, FAKE, FAKE, 0, 0, FAKE), (1, 4, None, None, 0, 0, FAKE), (1, 4, FAKE, FAKE, 0, 0, None),
                 (1, 4, odd, FAKE, 0, 0, FAKE), (1, 4, FAKE, odd, 0, 0, FAKE), (1, 4, FAKE, FAKE, 256, 0, FAKE), (1, 4, FAKE, FAKE, 256, 127, FAKE),
                 (1, 4, FAKE, FAKE, -256, 128, FAKE), (0, 4, FAKE, FAKE, 258, 128, FAKE)):
        assert lib.laq_fp4_store(c, *args, None) == INVALID
    assert lib.laq_fp4_store(c, 1, 1 << 32, FAKE, FAKE, 0, 0, FAKE, None) == UNSUPPORTED
    assert lib.laq_fp4_store(c, 1, 0, FAKE, FAKE, 0, 0, FAKE, None) == 0                       # nothing to do
    for args in ((2, 4, FAKE, FAKE, FAKE), (1, -1, FAKE, FAKE, FAKE), (1, 4, None, FAKE, FAKE), (1, 4, FAKE, None, None), (1, 4, FAKE, odd, FAKE)):
        assert lib.laq_fp4_load(c, *args, None) == INVALID
    assert lib.laq_fp4_load(c, 1, 0, FAKE, FAKE, FAKE, None) == 0

    bud = (ctypes.c_int32 * 1)(8)
    good = dict(n=1, Hkv=2, d=128, L=64)

    def compact(k=FAKE, v=FAKE, idx=FAKE, budget=bud, slots=FAKE, dtype=1, **kw):
        s = {**good, **kw}
        sh = binding._shape(s["n"], s["Hkv"], s["Hkv"], s["d"], s["L"], 1, dtype, 0.0, None, 0)
        return lib.laq_fp4_compact(ctypes.byref(sh), k, v, idx, budget, c, slots, None)

    for kw in (dict(k=None), dict(idx=None), dict(budget=None), dict(slots=None), dict(k=odd), dict(v=odd), dict(Hkv=1), dict(d=64), dict(dtype=3),
               dict(budget=(ctypes.c_int32 * 1)(0)), dict(L=0)):
        assert compact(**kw) == INVALID, kw

    def attention(Hq=8, dtype=1, scale=0.0, n=2, T=2, start=None, q=FAKE, st=0, sh=0, table=FAKE, width=4, rows=FAKE, most=64, out=FAKE, lse=None, ws=None,
                  ws_bytes=0):
        return lib.laq_fp4_attention(c, Hq, dtype, scale, n, T, start, q, st, sh, table, width, rows, most, out, lse, ws, ws_bytes, None)

    for kw in (dict(Hq=7), dict(Hq=0), dict(Hq=1 << 17), dict(dtype=2), dict(scale=math.nan), dict(scale=math.inf), dict(n=0), dict(T=-1), dict(T=3),
               dict(q=None), dict(q=odd), dict(out=odd), dict(out=None), dict(table=None), dict(rows=None), dict(width=0), dict(most=0), dict(most=65),
               dict(width=1 << 28, most=1), dict(st=1024), dict(st=1024, sh=120 + 4), dict(st=-1024, sh=128), dict(T=1 << 31, start=FAKE)):
        assert attention(**kw) == INVALID, kw
    assert attention(T=0, start=FAKE) == 0
    big = dict(n=1, T=1, width=1 << 16, most=1 << 20)
    need = lib.laq_fp4_attention_workspace_bytes(c, 8, 1, 1, 1, 1 << 20)
    if need:                                         # (a call that long is cut into parts)
        assert attention(**big, ws=FAKE, ws_bytes=need - 1) == WORKSPACE and attention(**big, ws=odd, ws_bytes=need) == WORKSPACE
    assert lib.laq_fp4_attention_workspace_bytes(c, 7, 1, 1, 1, 64) == 0

    def block_map(n=2, br=16, blocks=8, width=4, add=FAKE, rows=FAKE, table=FAKE, free=FAKE, state=FAKE, start=None, slots=None, n_slots=0):
        return lib.laq_block_map(n, br, blocks, width, add, rows, table, free, state, start, slots, n_slots, None)

    for kw in (dict(n=0), dict(br=0), dict(br=8), dict(br=40), dict(blocks=0), dict(width=0), dict(blocks=1 << 28), dict(width=1 << 28), dict(add=None),
               dict(rows=None), dict(table=None), dict(free=None), dict(state=None), dict(n_slots=4), dict(slots=FAKE, n_slots=-1), dict(slots=FAKE, n_slots=1 << 31)):
        assert block_map(**kw) == INVALID, kw


def test_the_binding_refuses_host_tensors_and_sizes():
    host = laq.laq_fp4_cache(4, 2, 16, 64, device="cpu")
    k, i = torch.zeros(3, 2, 64), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: laq.laq_fp4_store(host, k, k, i), lambda: laq.laq_fp4_load(host, i), lambda: laq.laq_fp4_attention(k, host, i.view(4, 1), i),
                 lambda: laq.laq_fp4_compact(host, k[None], None, i, [2], i), lambda: laq.laq_block_map(i, i, i.view(4, 1), i, i, 16)):
        with pytest.raises(ValueError, match="must live on the GPU"):
            call()
    for size in ((4, 2, 16, 48), (4, 2, 20, 64), (0, 2, 16, 64), (4, 2, 16, 288)):
        with pytest.raises(ValueError):
            laq.laq_fp4_cache(*size, device="cpu")


def test_the_library_exports_what_its_second_header_declares(repo_root):
    import os
    import re
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(repo_root, "include", "laq_fp4.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(laq_[a-z0-9_]+)\s*\(", text)))
    assert names == ["laq_block_map", "laq_fp4_attention", "laq_fp4_attention_workspace_bytes", "laq_fp4_compact", "laq_fp4_load", "laq_fp4_store"]
    for name in names:
        assert getattr(laq.load_library(), name) is not None and name in laq.__all__


WIDE = dict(stride_head=1024, stride_row=64, scale_stride_block=128, scale_stride_head=64, scale_stride_row=4)


@pytest.mark.parametrize("bad", [dict(Hkv=32769), dict(stride_block=1 << 32, **WIDE), dict(stride_block=2048, **{**WIDE, "scale_stride_block": 1 << 32}),
                                 dict(stride_block=2048, **{**WIDE, "stride_row": (1 << 27) + 16}),
                                 dict(stride_block=2048, **{**WIDE, "scale_stride_row": (1 << 27) + 1})])
def test_caches_whose_offsets_do_not_fit(bad):
    test_caches_that_are_refused(bad)


def test_calls_that_are_too_large():
    lib = laq.load_library()
    assert lib.laq_block_map(1 << 16, 16, 8, 1 << 15, FAKE, FAKE, FAKE, FAKE, FAKE, None, None, 0, None) == UNSUPPORTED
    c = ctypes.byref(_cache())
    assert lib.laq_fp4_load(c, 1, 1 << 32, FAKE, FAKE, FAKE, None) == UNSUPPORTED
    n = 1 << 23                                          # x 2 KV heads
    assert lib.laq_fp4_attention(c, 2, 1, 0.0, n, n, None, FAKE, 0, 0, FAKE, 4, FAKE, 64, FAKE, None, None, 0, None) == UNSUPPORTED
    # shared out among few workgroups, but for turns that may be more than an int holds
    many = ctypes.byref(_cache(Hkv=32768))
    args = (many, 32768, 1, 0.0, 1024, 1024, None, FAKE, 0, 0, FAKE, (1 << 27) - 1, FAKE, 8192, FAKE, None)
    assert lib.laq_fp4_attention(*args, FAKE, 1 << 62, None) == UNSUPPORTED


def test_batches_without_tokens_need_no_addresses():
    lib = laq.load_library()
    c = ctypes.byref(_cache())
    assert lib.laq_fp4_store(c, 1, 0, None, None, 0, 0, None, None) == 0
    assert lib.laq_fp4_load(c, 1, 0, None, None, None, None) == 0
    assert lib.laq_fp4_attention(c, 8, 1, 0.0, 2, 0, FAKE, None, 0, 0, FAKE, 4, FAKE, 64, None, None, None, 0, None) == 0
    # but sizes that are right
    assert lib.laq_fp4_store(c, 3, 0, None, None, 0, 0, None, None) == INVALID
    assert lib.laq_fp4_load(c, 3, 0, None, None, None, None) == INVALID
    assert lib.laq_fp4_attention(c, 7, 1, 0.0, 2, 0, FAKE, None, 0, 0, FAKE, 4, FAKE, 64, None, None, None, 0, None) == INVALID


def test_the_longest_bounds_are_planned_like_long_ones():
    lib = laq.load_library()
    c = ctypes.byref(_cache(n_blocks=4))
    for Hq, n, T in ((2, 1, 1), (8, 1, 3), (8, 3, 3), (2, 40, 40)):
        long = lib.laq_fp4_attention_workspace_bytes(c, Hq, 1, n, T, 1 << 30)
        for most in ((1 << 31) - 4096, (1 << 31) - 255, (1 << 31) - 16):
            assert lib.laq_fp4_attention_workspace_bytes(c, Hq, 1, n, T, most) >= long > 0
