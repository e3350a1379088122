"""The plain forms that rotary positions and the paged cache of 32, 16 or 8 bits are tested against, pinned; the frequencies; and the refusals of the calls
(no GPU needed)."""
import ctypes
import math
import random
import subprocess
import sys

import pytest
import torch

import paper_2505_20334_amd as laq
import paged_plain as plain
from paper_2505_20334_amd import binding

INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3
FAKE, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008)


def test_the_format_of_a_row_by_its_definition():
    rng = random.Random(5)
    rows = [[rng.gauss(0, 10.0 ** rng.randint(-20, 20)) for _ in range(24)] for _ in range(200)]
    rows += [[0.0] * 24, [-0.0] * 24, [2.0 ** -101] * 24, [3.38e38] + [1e37] * 23, [math.inf] + [1.0] * 23, [math.nan] + [0.0] * 23]
    for most in (1.0, 1.75, math.nextafter(1.75, 2), 448.0, 448.001):          # the border of the scale
        rows.append([most] + [most * rng.uniform(-1, 1) for _ in range(23)])
    rows.append([448.0] + [s * t for t in (17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -11, 1.0625) for s in (1, -1)] + [0.0] * 11)     # ties
    x = torch.tensor(rows, dtype=torch.float64)
    codes, scales = plain.quantise(x)
    for i, row in enumerate(rows):
        s, c = plain.quantise_row(row)
        assert scales[i] == s and codes[i].tolist() == c
    assert plain.values(codes, scales)[-1, 1:13:2].tolist() == [16.0, 20.0, 0.0, 2.0 ** -8, 0.0, 1.0]
    # the type's own conversion, of numbers that 448 reaches
    finite = torch.isfinite(x).all(-1)
    there = (x / torch.exp2(scales.double() - 127)[:, None])[finite]
    assert torch.equal(there.float().to(torch.float8_e4m3fn).view(torch.uint8)[:200], codes[finite][:200])
    err = (plain.values(codes, scales) - x).abs()[finite] / x.abs().amax(-1, keepdim=True)[finite].clamp(min=1e-300)
    assert err[x[finite].abs().amax(-1) > 2.0 ** -90].max() <= 2.0 ** -4
    assert plain.values(torch.tensor([[0x7F, 0xFF, 0x7E, 0x01]], dtype=torch.uint8), torch.tensor([127], dtype=torch.uint8))[0, 2:].tolist() == [448.0, 2.0 ** -9]


def test_a_rotation_by_its_definition():
    x = torch.randn(5, 2, 12, dtype=torch.float64)
    f, p = torch.tensor([0.5, 0.01, 1.0], dtype=torch.float32), torch.tensor([0, 1, -3, 100000, 7])
    half, _ = plain.rotate(x, p, f, "half", 1.0)
    inter, _ = plain.rotate(x, p, f, "interleaved", 2.0)
    for t in range(5):
        for i in range(3):
            by = complex(math.cos(int(p[t]) * float(f[i])), math.sin(int(p[t]) * float(f[i])))
            for h in range(2):
                y = complex(x[t, h, i], x[t, h, i + 3]) * by
                assert abs(y - complex(half[t, h, i], half[t, h, i + 3])) < 1e-12
                y = 2 * complex(x[t, h, 2 * i], x[t, h, 2 * i + 1]) * by
                assert abs(y - complex(inter[t, h, 2 * i], inter[t, h, 2 * i + 1])) < 1e-12
    assert torch.equal(half[..., 6:], x[..., 6:]) and torch.equal(half[0], x[0])
    # the product of a rotated query and a rotated key depends on the distance of their positions
    a, b = plain.rotate(x, p, f, "half", 1.0)[0][..., :6], plain.rotate(x.flip(0), p + 1000, f, "half", 1.0)[0][..., :6]
    c, e = plain.rotate(x, p + 5, f, "half", 1.0)[0][..., :6], plain.rotate(x.flip(0), p + 1005, f, "half", 1.0)[0][..., :6]
    assert torch.allclose((a * b).sum(-1), (c * e).sum(-1), atol=1e-6)


def test_frequencies():
    turns = lambda f, n: f.double() * n / (2 * math.pi)  # noqa: E731
    f = laq.laq_rope_frequencies(64, 10000.0, device="cpu")
    assert f.dtype == torch.float32 and f.shape == (32,) and f[0] == 1 and torch.allclose(f.double(), 10000.0 ** (-torch.arange(32).double() / 32), rtol=1e-7)
    assert torch.equal(laq.laq_rope_frequencies(64, 10000.0, "linear", 4.0, device="cpu"), (f.double() / 4).float())
    base = laq.laq_rope_frequencies(64, 10000.0, "base", 4.0, device="cpu")
    assert base[0] == 1 and abs(float(base[-1] / f[-1]) - 0.25) < 1e-6 and (base[1:] < f[1:]).all()
    for how in ("parts", "ramp"):
        g = laq.laq_rope_frequencies(64, 10000.0, how, 8.0, 4096, 1.0, 32.0, device="cpu")
        assert torch.equal(g[turns(f, 4096) > 40], f[turns(f, 4096) > 40])
        slow = turns(f, 4096) < 0.8
        assert slow.any() and torch.equal(g[slow], (f.double() / 8).float()[slow])
        assert ((g <= f) & (g >= f / 8 * (1 - 1e-6))).all() and (g[1:] < g[:-1]).all()
        assert torch.equal(laq.laq_rope_frequencies(64, 10000.0, how, 1.0, 4096, device="cpu"), f)
    i = int((turns(f, 4096) > 16.5).sum()) - 1            # "parts" by hand
    part = (float(turns(f, 4096)[i]) - 1) / 31
    g = laq.laq_rope_frequencies(64, 10000.0, "parts", 8.0, 4096, 1.0, 32.0, device="cpu")
    assert abs(float(g[i]) - float(f[i]) * (part + (1 - part) / 8)) < 1e-6 * float(f[i])
    # "ramp" by hand: from the index that turns 32 times (rounded down) to the one that turns once (up)
    g = laq.laq_rope_frequencies(64, 10000.0, "ramp", 8.0, 4096, 1.0, 32.0, device="cpu")
    low, high = (64 * math.log(4096 / (t * 2 * math.pi)) / (2 * math.log(10000.0)) for t in (32.0, 1.0))
    low, high = math.floor(low), math.ceil(high)
    mid = (low + high) // 2
    share = (mid - low) / (high - low)
    assert abs(float(g[mid]) - float(f[mid]) * (1 - share + share / 8)) < 1e-6 * float(f[mid])
    for bad in (dict(rot=3), dict(rot=0), dict(rot=64, base=1.0), dict(rot=64, factor=0.5), dict(rot=64, scaling="more"), dict(rot=64, scaling="parts"), dict(rot=2, scaling="base"),
                dict(rot=64, scaling="ramp", trained=4096, slow=4.0, fast=4.0)):
        with pytest.raises(ValueError):
            laq.laq_rope_frequencies(**bad, device="cpu")


def _cache(**kw):
    c = dict(k=0x1000, v=0x2000, k_scale=0x3000, v_scale=0x4000, n_blocks=8, Hkv=2, block_rows=16, d=128, type=2, stride_block=0, stride_head=0, stride_row=0)
    return binding._PagedCache(*{**c, **kw}.values())


def _heads(x=0x1000, heads=2, token=0, head=0):
    return ctypes.byref(binding._Heads(x, heads, token, head))


def _plan(inv_freq=0x1000, rot=64, layout=0, mscale=1.0):
    return ctypes.byref(binding._RopePlan(inv_freq, rot, layout, mscale))


BAD_CACHES = [dict(n_blocks=0), dict(Hkv=0), dict(Hkv=32769), dict(block_rows=0), dict(block_rows=24), dict(d=0), dict(d=12), dict(d=264), dict(type=3), dict(type=-1),
              dict(n_blocks=1 << 28), dict(k=None), dict(v=None), dict(k=0x1008), dict(v=0x1008), dict(k_scale=None), dict(v_scale=0x1004), dict(stride_row=128),
              dict(stride_block=4096, stride_head=2048, stride_row=120), dict(stride_block=4100, stride_head=2048, stride_row=128),
              dict(stride_block=4096, stride_head=2044, stride_row=128), dict(stride_block=-4096, stride_head=2048, stride_row=128),
              dict(stride_block=1 << 60, stride_head=2048, stride_row=128), dict(stride_block=4096, stride_head=2048, stride_row=(1 << 24) + 8)]


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_caches_that_are_refused(bad):
    lib = laq.load_library()
    c = ctypes.byref(_cache(**bad))
    assert lib.laq_cache_append(c, 1, 4, _heads(), _heads(), FAKE, None, None, None, None, None) == INVALID
    assert lib.laq_cache_load(c, 1, 4, FAKE, FAKE, FAKE, None) == INVALID
    assert lib.laq_cache_attention(c, 1, 0.0, 2, 2, None, _heads(heads=8), FAKE, 4, FAKE, 16, FAKE, None, None, 0, None) == INVALID
    sh = binding._shape(1, 2, 2, 128, 64, 1, 1, 0.0, None, 0)
    assert lib.laq_cache_compact(ctypes.byref(sh), FAKE, FAKE, FAKE, (ctypes.c_int32 * 1)(8), c, FAKE, None) == INVALID


def test_arguments_that_are_refused():
    lib = laq.load_library()
    c = ctypes.byref(_cache())

    def append(dtype=1, T=4, k=_heads(), v=_heads(), slots=FAKE, rope=None, positions=None, q=None, q_out=None):
        return lib.laq_cache_append(c, dtype, T, k, v, slots, rope, positions, q, q_out, None)

    q = _heads(heads=8)
    for kw in (dict(dtype=2), dict(T=-1), dict(k=None, v=None), dict(slots=None), dict(k=_heads(0x1008)), dict(v=_heads(0x1008)), dict(k=_heads(heads=3)), dict(v=_heads(heads=1)),
               dict(k=_heads(token=256)), dict(k=_heads(token=256, head=127)), dict(k=_heads(token=-256, head=128)), dict(dtype=0, k=_heads(token=258, head=128)),
               dict(k=_heads(token=1 << 60, head=128)), dict(rope=_plan()), dict(rope=_plan(rot=3), positions=FAKE), dict(rope=_plan(rot=130), positions=FAKE),
               dict(rope=_plan(rot=0), positions=FAKE), dict(rope=_plan(layout=2), positions=FAKE), dict(rope=_plan(mscale=math.nan), positions=FAKE),
               dict(rope=_plan(mscale=math.inf), positions=FAKE), dict(rope=_plan(inv_freq=None), positions=FAKE), dict(q=q, q_out=q),
               dict(rope=_plan(), positions=FAKE, q=q), dict(rope=_plan(), positions=FAKE, q_out=q), dict(rope=_plan(), positions=FAKE, q=q, q_out=_heads(heads=7)),
               dict(rope=_plan(), positions=FAKE, q=_heads(heads=1 << 17), q_out=_heads(heads=1 << 17))):
        assert append(**kw) == INVALID, kw
    assert append(T=(1 << 25) + 1) == UNSUPPORTED
    assert append(T=0) == 0 and append(T=0, k=None, v=None, slots=None) == 0 and append(T=0, dtype=2) == INVALID

    def rope(plan=_plan(), dtype=1, T=4, d=128, q=_heads(), k=None, positions=FAKE, q_out=_heads(), k_out=None):
        return lib.laq_rope(plan, dtype, T, d, q, k, positions, q_out, k_out, None)

    for kw in (dict(plan=None), dict(plan=_plan(rot=130)), dict(dtype=2), dict(T=-1), dict(d=0), dict(d=260), dict(d=132), dict(q=None), dict(q=None, q_out=None), dict(positions=None),
               dict(q_out=None), dict(k=_heads()), dict(k_out=_heads()), dict(q_out=_heads(heads=3)), dict(q_out=_heads(token=132, head=128)), dict(q=_heads(0x1004))):
        assert rope(**kw) == INVALID, kw
    assert rope(T=(1 << 25) + 1) == UNSUPPORTED and rope(T=0, q=_heads(None), q_out=_heads(None)) == 0

    for args in ((2, 4, FAKE, FAKE, FAKE), (1, -1, FAKE, FAKE, FAKE), (1, 4, None, FAKE, FAKE), (1, 4, FAKE, None, None), (1, 4, FAKE, ODD, FAKE)):
        assert lib.laq_cache_load(c, *args, None) == INVALID
    assert lib.laq_cache_load(c, 1, 0, None, None, None, None) == 0 and lib.laq_cache_load(c, 1, (1 << 25) + 1, FAKE, FAKE, FAKE, None) == UNSUPPORTED

    bud = (ctypes.c_int32 * 1)(8)

    def compact(k=FAKE, v=FAKE, idx=FAKE, budget=bud, slots=FAKE, dtype=1, **kw):
        s = {**dict(n=1, Hkv=2, d=128, L=64), **kw}
        sh = binding._shape(s["n"], s["Hkv"], s["Hkv"], s["d"], s["L"], 1, dtype, 0.0, None, 0)
        return lib.laq_cache_compact(ctypes.byref(sh), k, v, idx, budget, c, slots, None)

    for kw in (dict(k=None), dict(idx=None), dict(budget=None), dict(slots=None), dict(k=ODD), dict(v=ODD), dict(Hkv=1), dict(d=64), dict(dtype=3),
               dict(budget=(ctypes.c_int32 * 1)(0)), dict(L=0)):
        assert compact(**kw) == INVALID, kw
    assert compact(L=1 << 30, budget=(ctypes.c_int32 * 1)(1 << 27)) == UNSUPPORTED

    def attention(cache=c, dtype=1, scale=0.0, n=2, T=2, start=None, q=_heads(heads=8), table=FAKE, width=4, rows=FAKE, most=64, out=FAKE, lse=None, ws=None, ws_bytes=0):
        return lib.laq_cache_attention(cache, dtype, scale, n, T, start, q, table, width, rows, most, out, lse, ws, ws_bytes, None)

    for kw in (dict(q=_heads(heads=7)), dict(q=_heads(heads=0)), dict(q=_heads(heads=1 << 17)), dict(dtype=2), dict(scale=math.nan), dict(scale=math.inf), dict(n=0), dict(T=-1),
               dict(T=3), dict(q=None), dict(q=_heads(None, 8)), dict(q=_heads(0x1008, 8)), dict(out=ODD), dict(out=None), dict(table=None), dict(rows=None), dict(width=0), dict(most=0),
               dict(most=65), dict(width=1 << 28, most=1), dict(q=_heads(heads=8, token=1024)), dict(q=_heads(heads=8, token=1024, head=124)), dict(T=1 << 31, start=FAKE)):
        assert attention(**kw) == INVALID, kw
    assert attention(T=0, start=FAKE, q=_heads(None, 8)) == 0 and attention(T=0, start=FAKE, q=_heads(None, 7)) == INVALID
    assert attention(cache=ctypes.byref(_cache(type=0))) == UNSUPPORTED                                   # bf16 queries, fp32 cache
    need = lib.laq_cache_attention_workspace_bytes(c, 8, 1, 1, 1, 1 << 20)
    big = dict(n=1, T=1, width=1 << 16, most=1 << 20)
    assert need > 0 and attention(**big, ws=FAKE, ws_bytes=need - 1) == WORKSPACE and attention(**big, ws=ODD, ws_bytes=need) == WORKSPACE
    assert lib.laq_cache_attention_workspace_bytes(c, 7, 1, 1, 1, 64) == 0
    n = 1 << 24                                                                                           # x 2 KV heads
    assert attention(n=n, T=n, q=_heads(heads=2)) == UNSUPPORTED


def test_workspaces_of_long_bounds_stay_small():
    lib = laq.load_library()
    c = ctypes.byref(_cache(n_blocks=4))
    for Hq, n, T in ((2, 1, 1), (8, 1, 3), (8, 3, 3), (2, 40, 40), (64, 512, 512), (64, 4, 4096)):
        long = lib.laq_cache_attention_workspace_bytes(c, Hq, 1, n, T, 1 << 30)
        # (none for chunks of a prompt, which are not shared out)
        assert (long == 0) == (T == 4096) and long < 1 << 31
        for most in ((1 << 31) - 4096, (1 << 31) - 255, (1 << 31) - 16):
            assert lib.laq_cache_attention_workspace_bytes(c, Hq, 1, n, T, most) == long


def test_the_binding_refuses_host_tensors_and_sizes():
    host = laq.laq_cache(4, 2, 16, 64, device="cpu")
    k, i = torch.zeros(3, 2, 64), torch.zeros(4, dtype=torch.int32)
    rope = laq.Rope(torch.ones(32))
    for call in (lambda: laq.laq_cache_append(host, k, k, i), lambda: laq.laq_cache_load(host, i), lambda: laq.laq_cache_attention(k, host, i.view(4, 1), i),
                 lambda: laq.laq_cache_compact(host, k[None], None, i, [2], i), lambda: laq.laq_rope(k, None, i, rope)):
        with pytest.raises(ValueError, match="must live on the GPU"):
            call()
    for size in ((4, 2, 16, 44), (4, 2, 20, 64), (0, 2, 16, 64), (4, 2, 16, 264)):
        with pytest.raises(ValueError):
            laq.laq_cache(*size, device="cpu")
    with pytest.raises(TypeError):
        laq.laq_cache(4, 2, 16, 64, torch.float16, device="cpu")
    e = laq.laq_cache(4, 2, 16, 64, torch.float8_e4m3fn, device="cpu")
    assert e.k.dtype == torch.float8_e4m3fn and e.k_scale.shape == (4, 2, 16) and host.k_scale is None


SETUP = """
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
import paper_2505_20334_amd as laq
from paper_2505_20334_amd import binding, paged

import ctypes
lib = laq.load_library()
address = lambda name: ctypes.cast(getattr(lib, name), ctypes.c_void_p).value
# (no device here: a device and a stream number as a GPU would give them)
binding._native.bind(address("laq_evict"), address("laq_workspace_bytes"), address("laq_decode_attention"),
                     address("laq_decode_workspace_bytes"), address("laq_qcache_store"), lambda: %d, lambda device: 0)
binding._stream = paged._stream = lambda stream: 0
torch._C._cuda_getDevice = lambda: %d
if not %r:
    binding._native = None

def made(*sizes, dtype=torch.bfloat16):
    return torch.empty(*sizes, dtype=dtype, device="cuda")

def pool(blocks, heads, rows, d, dtype=torch.float8_e4m3fn):
    planes = []
    for _ in range(2):
        planes += [made(blocks, heads, rows, d, dtype=dtype), made(blocks, heads, rows, dtype=torch.uint8) if dtype == torch.float8_e4m3fn else None]
    return laq.PagedCache(*planes)

def ints(*sizes):
    return made(*sizes, dtype=torch.int32)

with FakeTensorMode():
    cache, wide, kv, q, source = pool(8, 2, 16, 128), pool(8, 2, 16, 128, torch.bfloat16), made(3, 2, 128), made(3, 8, 128), made(3, 2, 40, 128)
    rope = laq.Rope(made(64, dtype=torch.float32))
    for call in %r:
        try:
            eval(call)
            print("no exception")
        except Exception as e:
            print("raised", type(e).__name__, str(e).split(chr(10))[0])
"""
GOOD = ["laq.laq_cache_append(cache, kv, kv, ints(3))", "laq.laq_cache_append(wide, kv, None, ints(4), q=q, positions=ints(3), rope=rope)", "laq.laq_cache_load(cache, ints(3))",
        "laq.laq_cache_compact(cache, source, source, ints(200), [10, 20, 30], ints(60))", "laq.laq_cache_attention(q, cache, ints(3, 4), ints(3))",
        "laq.laq_rope(q, kv, ints(3), rope)"]


def outcomes(calls, device=0, native=True):
    res = subprocess.run([sys.executable, "-c", SETUP % (device, device, native, calls)], capture_output=True, text=True, timeout=110)
    assert res.returncode == 0, "the process ended with %d: %s" % (res.returncode, res.stderr[-600:])
    return res.stdout.strip().splitlines()[-len(calls):]


@pytest.mark.parametrize("native", [True, False])
def test_calls_in_order_reach_the_library(native):
    # (which refuses the addresses that tensors without memory have: NULL)
    for got in outcomes(GOOD, native=native):
        assert got.startswith("raised LaqError laq_") and got.endswith("invalid argument (code -1)"), got
    for got in outcomes(GOOD, device=1, native=native):
        assert got.endswith("which is not the current device"), got


BAD = [
    ("laq.laq_cache_append(cache, kv, kv.float(), ints(3))", "v must be"), ("laq.laq_cache_append(cache, kv, kv, ints(2))", "slots"),
    ("laq.laq_cache_append(cache, None, None, ints(3))", "k or v is needed"), ("laq.laq_cache_append(cache, kv[:, :1], None, ints(3))", "k must be"),
    ("laq.laq_cache_append(cache[:3], kv, None, ints(3))", ""), ("laq.laq_cache_append(cache._replace(v=made(8, 2, 16, 128)), kv, None, ints(3))", "v must be"),
    ("laq.laq_cache_append(cache._replace(k_scale=None), kv, None, ints(3))", "k_scale must be"), ("laq.laq_cache_append(wide._replace(k_scale=cache.k_scale), kv, None, ints(3))", "scales"),
    ("laq.laq_cache_append(cache._replace(v_scale=made(8, 2, 32, dtype=torch.uint8)[:, :, ::2]), kv, None, ints(3))", "v_scale must be"),
    ("laq.laq_cache_append(cache, kv.half(), None, ints(3))", ""), ("laq.laq_cache_append(cache, kv, None, ints(3).long())", "slots must be"),
    ("laq.laq_cache_append(cache, kv, kv, ints(3), q=q)", "given with rope"), ("laq.laq_cache_append(cache, kv, kv, ints(3), rope=rope)", "needs positions"),
    ("laq.laq_cache_append(cache, kv, kv, ints(3), positions=ints(2), rope=rope)", "positions must be"), ("laq.laq_cache_append(cache, kv, kv, ints(3), positions=ints(3))", "given with rope"),
    ("laq.laq_cache_append(cache, kv, kv, ints(3), q=q.float(), positions=ints(3), rope=rope)", "q must be"),
    ("laq.laq_cache_append(cache, kv, kv, ints(3), q=q[:2], positions=ints(3), rope=rope)", "q must be"),
    ("laq.laq_cache_append(cache, kv, kv, ints(3), q=q, positions=ints(3), rope=rope, q_out=made(3, 7, 128))", "q_out must be"),
    ("laq.laq_cache_append(cache, kv, kv, ints(3), positions=ints(3), rope=rope, q_out=q)", "q_out without q"),
    ("laq.laq_cache_append(cache, kv, kv, ints(3), positions=ints(3), rope=rope._replace(layout='both'))", "layout"),
    ("laq.laq_cache_append(cache, kv, kv, ints(3), positions=ints(3), rope=rope._replace(inv_freq=made(64)))", "inv_freq"),
    ("laq.laq_rope(None, None, ints(3), rope)", "q or k is needed"), ("laq.laq_rope(q, kv[:2], ints(3), rope)", "k must be"), ("laq.laq_rope(q, None, ints(3), rope, k_out=kv)", "k_out without k"),
    ("laq.laq_rope(q.half(), None, ints(3), rope)", ""), ("laq.laq_rope(q, None, ints(3).long(), rope)", "positions must be"), ("laq.laq_rope(q[0], None, ints(3), rope)", "tokens, heads, d"),
    ("laq.laq_rope(q, None, ints(3), rope, q_out=q.float())", "q_out must be"), ("laq.laq_rope(q, None, ints(3), laq.Rope(made(65, dtype=torch.float32)))", "code -1"),
    ("laq.laq_cache_load(cache, ints(3), torch.float16)", ""), ("laq.laq_cache_load(cache, ints(3), k=made(3, 2, 127))", "k"),
    ("laq.laq_cache_compact(cache, source, source, ints(100), [10, 20, 30], ints(60))", "idx must be"),
    ("laq.laq_cache_compact(cache, source, source, ints(200), [10, 20, 30], ints(50))", "slots must be"),
    ("laq.laq_cache_compact(cache, source, source, ints(200), [10, 20], ints(60))", ""), ("laq.laq_cache_compact(cache, made(3, 4, 40, 128), None, ints(200), [10, 20, 30], ints(60))", "KV heads"),
    ("laq.laq_cache_attention(q, cache, ints(2, 4), ints(2))", "one token per request"), ("laq.laq_cache_attention(q, cache, ints(3, 4), ints(2))", "rows must be"),
    ("laq.laq_cache_attention(q, cache, ints(3, 4), ints(3), start=ints(3))", "start must be"), ("laq.laq_cache_attention(q[..., :64], cache, ints(3, 4), ints(3))", "q must be"),
    ("laq.laq_cache_attention(q, cache, ints(3, 4), ints(3), max_rows=(1 << 32) + 16)", "max_rows"), ("laq.laq_cache_attention(q.half(), cache, ints(3, 4), ints(3))", ""),
    ("laq.laq_cache_attention(q, cache, ints(3, 4), ints(3), out=made(3, 8, 64))", "out"), ("laq.laq_cache_attention(q, cache, ints(3, 4), ints(3), lse=made(3, 8))", "lse"),
    ("laq.laq_cache_attention(q, cache, ints(3, 4), ints(3), ws=torch.empty(64))", "ws"), ("laq.laq_cache_attention(q, pool(8, 2, 0, 128), ints(3, 4), ints(3))", ""),
    ("laq.laq_cache_append(pool(8, 2, 16, 128, torch.float16), kv, kv, ints(3))", "a cache is fp32, bf16 or float8_e4m3fn"),
]


@pytest.mark.parametrize("native", [True, False])
def test_what_is_refused(native):
    for (call, words), got in zip(BAD, outcomes([call for call, _ in BAD], native=native)):
        assert got.startswith("raised ") and words in got, (call, got)


@pytest.mark.parametrize("call", ["torch.vmap(lambda x: laq.laq_cache_append(cache, x, kv, ints(3)))(kv[None])", "torch.vmap(lambda x: laq.laq_cache_load(cache, x))(ints(1, 3))",
                                  "torch.vmap(lambda x: laq.laq_rope(x, None, ints(3), rope))(kv[None])", "torch.vmap(lambda x: laq.laq_cache_attention(x, cache, ints(3, 4), ints(3)))(q[None])",
                                  "torch.vmap(lambda x: laq.laq_cache_compact(cache, x, None, ints(200), [10, 20, 30], ints(60)))(source[None])"])
def test_a_tensor_without_an_address(call):
    assert outcomes([call])[0].startswith("raised RuntimeError Cannot access data pointer")


# what a call makes: number of tensors
MADE = {"laq.laq_cache_load(paged_cache, ints(3), stream=stream)": 2, "laq.laq_rope(made(3, 8, 128), made(3, 2, 128), ints(3), rope, stream=stream)": 2,
        "laq.laq_cache_append(paged_cache, made(3, 2, 128), None, ints(3), q=made(3, 8, 128), positions=ints(3), rope=rope, stream=stream)": 1,
        "laq.laq_cache_attention(made(1, 8, 128), paged_cache, ints(1, 4000), ints(1), want_lse=True, stream=stream)": 3}


@pytest.mark.parametrize("call", list(MADE))
def test_memory_is_taken_under_the_stream_of_the_call(call):
    import test_streams
    setup = test_streams.SETUP.replace("    torch.empty = counted\n", """    paged_cache = laq.PagedCache(made(8, 2, 16, 128), None, made(8, 2, 16, 128), None)
    rope = laq.Rope(made(64, dtype=torch.float32))
    torch.empty = counted
""")
    res = subprocess.run([sys.executable, "-c", setup % ("binding._native = None; " + call)], capture_output=True, text=True, timeout=110)
    assert res.returncode == 0, res.stderr[-800:]
    n = MADE[call]
    own, side, number, default = res.stdout.strip().splitlines()[-4:]
    # (memory of the inputs is made here too, on the current stream: what follows it is the call's)
    tails = [line[1:line.index("]")].replace(" ", "").split(",")[-n:] for line in (own, side, number, default)]
    assert tails == [["0"] * n, ["77"] * n, ["78"] * n, ["0"] * n], (own, side, number, default)
    assert side.endswith(str([0] * n)) and number.endswith(str([0] * n))


def test_the_library_exports_what_its_third_header_declares(repo_root):
    import os
    import re
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(repo_root, "include", "laq_cache.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(laq_[a-z0-9_]+)\s*\(", text)))
    assert names == ["laq_cache_append", "laq_cache_attention", "laq_cache_attention_workspace_bytes", "laq_cache_compact", "laq_cache_load", "laq_rope"]
    for name in names:
        assert getattr(laq.load_library(), name) is not None and name in laq.__all__
