"""The compiled binding of the 4-bit cache's calls, on tensors without memory (no GPU needed): what it does not take ends in
the Python binding's own exception.  Every case runs in a process of its own."""
import subprocess
import sys

import pytest

SETUP = """
import ctypes
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
import paper_2505_20334_amd as laq
from paper_2505_20334_amd import binding, fp4

lib = laq.load_library()
address = lambda name: ctypes.cast(getattr(lib, name), ctypes.c_void_p).value
# (no device here: a device and a stream number as a GPU would give them)
binding._native.bind(address("laq_evict"), address("laq_workspace_bytes"), address("laq_decode_attention"),
                     address("laq_decode_workspace_bytes"), address("laq_qcache_store"), lambda: %s, lambda device: 0)
binding._stream = fp4._stream = lambda stream: 0
torch._C._cuda_getDevice = lambda: %s

def made(*sizes, dtype=torch.bfloat16):
    return torch.empty(*sizes, dtype=dtype, device="cuda")

def pool(blocks, heads, rows, d):
    return laq.Fp4Cache(*(made(blocks, heads, rows, w, dtype=torch.uint8) for w in (d // 2, d // 32, d // 2, d // 32)))

def ints(*sizes):
    return made(*sizes, dtype=torch.int32)

with FakeTensorMode():
    cache, kv, q, source = pool(8, 2, 16, 128), made(3, 2, 128), made(3, 8, 128), made(3, 2, 40, 128)
    try:
        %s
        print("no exception")
    except Exception as e:
        print("raised", type(e).__name__, str(e).split(chr(10))[0])
"""
GOOD = {"store": "laq.laq_fp4_store(cache, kv, kv, ints(3))",
        "load": "laq.laq_fp4_load(cache, ints(3))",
        "compact": "laq.laq_fp4_compact(cache, source, source, ints(200), [10, 20, 30], ints(60))",
        "map": "laq.laq_block_map(ints(3), ints(3), ints(3, 4), ints(8), ints(4), 16, n_slots=5)",
        "attention": "laq.laq_fp4_attention(q, cache, ints(3, 4), ints(3))"}


def outcome(call, device=0):
    res = subprocess.run([sys.executable, "-c", SETUP % (device, device, call)], capture_output=True, text=True, timeout=110)
    assert res.returncode == 0, "the process ended with %d: %s" % (res.returncode, res.stderr[-600:])
    return res.stdout.strip().splitlines()[-1]


@pytest.mark.parametrize("name", list(GOOD))
def test_calls_in_order_reach_the_library(name):
    # (which refuses the addresses that tensors without memory have: NULL)
    assert outcome(GOOD[name]).startswith("raised LaqError laq_") and outcome(GOOD[name]).endswith("invalid argument (code -1)")


@pytest.mark.parametrize("call", ["laq.laq_fp4_store(cache, x, kv, ints(3)), kv", "laq.laq_fp4_load(cache, x), ints(3)", "laq.laq_fp4_attention(x, cache, ints(3, 4), ints(3)), q",
                                  "laq.laq_fp4_compact(cache, x, None, ints(200), [10, 20, 30], ints(60)), source",
                                  "laq.laq_block_map(x, ints(3), ints(3, 4), ints(8), ints(4), 16), ints(3)"])
def test_a_tensor_without_an_address(call):
    call, batch = call.rsplit(", ", 1)
    assert outcome("torch.vmap(lambda x: %s)(%s.unsqueeze(0))" % (call, batch)).startswith("raised RuntimeError Cannot access data pointer")


@pytest.mark.parametrize("name", list(GOOD))
def test_tensors_of_another_device(name):
    assert outcome(GOOD[name], device=1).endswith("which is not the current device")


BAD = [
    ("laq.laq_fp4_store(pool(8, 2, 0, 128), kv, kv, ints(3))", ""), ("laq.laq_fp4_attention(q, pool(8, 2, 0, 128), ints(3, 4), ints(3))", ""),
    ("laq.laq_fp4_store(cache, kv, kv.float(), ints(3))", "mismatch"), ("laq.laq_fp4_store(cache, kv, kv, ints(2))", "slots"),
    ("laq.laq_fp4_store(cache, None, None, ints(3))", "k or v is needed"), ("laq.laq_fp4_store(cache, kv[:, :1], None, ints(3))", "k must be"),
    ("laq.laq_fp4_store(cache[:3], kv, None, ints(3))", ""), ("laq.laq_fp4_store(cache._replace(v=made(8, 2, 16, 64)), kv, None, ints(3))", "v must be uint8"),
    ("laq.laq_fp4_store(cache, kv.half(), None, ints(3))", ""), ("laq.laq_fp4_store(cache, kv, None, ints(3).long())", "slots must be"),
    ("laq.laq_fp4_load(cache, ints(3), torch.float16)", ""), ("laq.laq_fp4_load(cache, ints(3), k=made(3, 2, 127))", "k"),
    ("laq.laq_fp4_compact(cache, source, source, ints(100), [10, 20, 30], ints(60))", "idx must be"),
    ("laq.laq_fp4_compact(cache, source, source, ints(200), [10, 20, 30], ints(50))", "slots must be"),
    ("laq.laq_fp4_compact(cache, source, source, ints(200), [10, 20], ints(60))", ""), ("laq.laq_fp4_compact(cache, made(3, 4, 40, 128), None, ints(200), [10, 20, 30], ints(60))", "KV heads"),
    ("laq.laq_block_map(ints(3), ints(2), ints(3, 4), ints(8), ints(4), 16)", "rows"), ("laq.laq_block_map(ints(3), ints(3), ints(12), ints(8), ints(4), 16)", "block_table"),
    ("laq.laq_block_map(ints(3), ints(3), ints(3, 4), ints(8), ints(3), 16)", "state"),
    ("laq.laq_block_map(ints(3), ints(3), ints(3, 4), ints(8), ints(4), 16, slots=ints(4), n_slots=5)", "slots"),
    ("laq.laq_block_map(ints(3), ints(3), ints(3, 4), ints(8), ints(4), (1 << 32) + 16)", ""),
    ("laq.laq_fp4_attention(q, cache, ints(2, 4), ints(2))", "one token per request"), ("laq.laq_fp4_attention(q, cache, ints(3, 4), ints(2))", "rows must be"),
    ("laq.laq_fp4_attention(q, cache, ints(3, 4), ints(3), start=ints(3))", "start must be"), ("laq.laq_fp4_attention(q[..., :64], cache, ints(3, 4), ints(3))", "q must be"),
    ("laq.laq_fp4_attention(q, cache, ints(3, 4), ints(3), max_rows=(1 << 32) + 16)", "max_rows"),
    ("laq.laq_fp4_attention(q, cache, ints(3, 4), ints(3), out=made(3, 8, 64))", "out"), ("laq.laq_fp4_attention(q, cache, ints(3, 4), ints(3), lse=made(3, 8))", "lse"),
    ("laq.laq_fp4_attention(q, cache, ints(3, 4), ints(3), ws=torch.empty(64))", "ws"),
]


@pytest.mark.parametrize("call,words", BAD)
def test_what_is_refused(call, words):
    got = outcome(call)
    assert got.startswith("raised ") and words in got, got
