"""Where calls that are given a stream take the memory of what they make: under that stream, and kept until the caller's has done with it (on tensors without
memory, no GPU needed).  Every case runs in a process of its own."""
import subprocess
import sys

import pytest

SETUP = """
import contextlib
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
import paper_2505_20334_amd as laq
from paper_2505_20334_amd import binding

binding.load_library()
torch._C._cuda_getDevice = lambda: 0

class Stream:
    def __init__(self, cuda_stream):
        self.cuda_stream = cuda_stream

current = [Stream(0)]
torch.cuda.Stream, torch.cuda.ExternalStream = Stream, Stream
torch.cuda.default_stream = lambda: Stream(0)
torch.cuda.current_stream = lambda: current[-1]

@contextlib.contextmanager
def under(stream):
    current.append(stream)
    yield
    current.pop()

torch.cuda.stream = under
empty, taken, kept = torch.empty, [], []
torch.Tensor.record_stream = lambda t, stream: kept.append(stream.cuda_stream)

def made(*sizes, dtype=torch.bfloat16):
    return empty(*sizes, dtype=dtype, device="cuda")

def ints(*sizes):
    return made(*sizes, dtype=torch.int32)

def counted(*sizes, **kw):
    taken.append(current[-1].cuda_stream)
    return empty(*sizes, **kw)

with FakeTensorMode():
    cache = laq.Fp4Cache(*(made(8, 2, 16, w, dtype=torch.uint8) for w in (64, 4, 64, 4)))
    torch.empty = counted
    for stream in (None, Stream(77), 78, 0):
        try:
            %s
            print("no exception")
        except laq.LaqError as e:                            # the library refuses the addresses that tensors without memory have: NULL
            print(taken, kept)
        taken.clear(), kept.clear()
"""
# what a call makes: number of tensors
CALLS = {"block_map": ("laq.laq_block_map(ints(3), ints(3), ints(3, 4), ints(8), ints(4), 16, n_slots=5, stream=stream)", 2),
         "fp4_load": ("laq.laq_fp4_load(cache, ints(3), stream=stream)", 2),
         "score": ("laq.laq_score(made(1, 8, 8, 128), made(1, 2, 600, 128), stream=stream)", 2),
         "select": ("laq.laq_select(made(1, 2, 600, dtype=torch.float32), [64], 7, 8, stream=stream)", 1),
         "select_sink_recent": ("laq.laq_select_sink_recent(1, 2, 600, [64], 4, stream=stream)", 1),
         "recall": ("laq.laq_recall(ints(128), [64], ints(128), [64], 2, 600, stream=stream)", 2),
         "compact": ("laq.laq_compact(made(1, 2, 600, 128), made(1, 2, 600, 128), ints(128), [64], 8, stream=stream)", 2),
         "evict": ("laq.laq_evict(made(1, 8, 8, 128), made(1, 2, 600, 128), made(1, 2, 600, 128), [64], 7, stream=stream)", 5),
         "decode_attention": ("laq.laq_decode_attention(made(1, 8, 128), made(40000, 128), made(40000, 128), [20000], 2, 30000, stream=stream)", 2),
         "fp4_attention": ("laq.laq_fp4_attention(made(1, 8, 128), cache, ints(1, 4000), ints(1), want_lse=True, stream=stream)", 3)}


@pytest.mark.parametrize("name", list(CALLS))
def test_memory_is_taken_under_the_stream_of_the_call(name):
    call, tensors = CALLS[name]
    # (without the compiled binding, which takes calls on the current stream alone)
    res = subprocess.run([sys.executable, "-c", SETUP % ("binding._native = None; " + call)], capture_output=True, text=True, timeout=110)
    assert res.returncode == 0, res.stderr[-800:]
    own, side, number, default = res.stdout.strip().splitlines()[-4:]
    assert own == "%s []" % ([0] * tensors)
    assert side == "%s %s" % ([77] * tensors, [0] * tensors) and number == "%s %s" % ([78] * tensors, [0] * tensors)
    assert default == "%s %s" % ([0] * tensors, [0] * tensors)


@pytest.mark.gpu
def test_evictions_and_decoding_on_a_busy_stream():
    import torch

    import paper_2505_20334_amd as laq
    gen = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn(2, h, r, 128, generator=gen).bfloat16().cuda() for h, r in ((8, 8), (2, 4096), (2, 4096)))
    budget = [3000, 2000]
    want = laq.laq_evict(q, k, v, budget, 7)
    want_out = laq.laq_decode_attention(q[:, :, 0].contiguous(), want[2], want[3], budget, 2, 4096)
    side, busy = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    for handle in (side, side.cuda_stream):
        with torch.cuda.stream(side):
            for _ in range(20):
                busy = (busy @ busy).clamp(-1, 1)
        got = laq.laq_evict(q, k, v, budget, 7, stream=handle)
        with torch.cuda.stream(side):
            q0 = q[:, :, 0].contiguous()
        out = laq.laq_decode_attention(q0, got[2], got[3], budget, 2, 4096, stream=handle)
        need = laq.laq_workspace_bytes(2, 8, 2, 128, 4096, 8, torch.bfloat16), laq.laq_decode_workspace_bytes(2, 8, 2, 128, 4096, torch.bfloat16, budget)
        others = [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in need for _ in range(8)]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)) and torch.equal(out, want_out)
        del others
