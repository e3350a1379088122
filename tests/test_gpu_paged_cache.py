"""Rotary positions and the paged cache in 32, 16 or 8 bits against their plain forms (needs an MI355X)."""
import math

import pytest
import torch

import fp4_plain
import paged_plain as plain

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


def _laq():
    import paper_2505_20334_amd as laq
    return laq


def _pool(n_blocks, H, br, d, kind, token_major=False, fill=0xA5):
    """A cache whose bytes are all `fill`."""
    laq = _laq()
    planes = []
    for _ in range(2):
        sizes = (n_blocks, br, H, d) if token_major else (n_blocks, H, br, d)
        x = torch.full(sizes[:3] + (d * torch.empty(0, dtype=kind).element_size(),), fill, dtype=torch.uint8, device=DEV).view(kind)
        planes.append(x.transpose(1, 2) if token_major else x)
        planes.append(torch.full((n_blocks, H, br), fill, dtype=torch.uint8, device=DEV) if kind == E4M3 else None)
    return laq.PagedCache(*planes)


def _bytes(t):
    """The bytes of a plane on the CPU, [n_blocks, Hkv, block_rows, bytes of a row]."""
    return t.cpu().contiguous().view(torch.uint8)


def _special(T, H, d, dtype, gen):
    x = torch.randn(T, H, d, generator=gen) * torch.exp2(torch.randint(-6, 7, (T, H, 1), generator=gen).float())
    flat = x.view(-1, d)
    rows = ([0.0] * d, [-0.0] * d, [3e38] + [1e38] * (d - 1), [-3.3e38] + [2e38] * (d - 1), [math.inf] + [1.0] * (d - 1), [1.0] * (d - 1) + [-math.inf],
            [math.nan] * d, [1e-38] * d, [2.0 ** -102] * (d - 1) + [-2.0 ** -99], [1e-45] * d, [448.0] + [2.0 ** -9, 2.0 ** -10, -3 * 2.0 ** -10] * 2 + [464.0] * 0 + [17.0] * (d - 7),
            [1.75] + [-1.0625, 1.1875, 0.0146484375] * 2 + [0.3] * (d - 7), [1.7578125] + [-1.0] * (d - 1), [7.0] + [2.0 ** -15, 3 * 2.0 ** -16] * 3 + [0.1] * (d - 7))
    for i, row in enumerate(rows):
        if 5 * i + 2 < flat.shape[0]:
            flat[5 * i + 2] = torch.tensor(row)
    return x.to(dtype)


def _laid(x, layout, extra=None):
    """x [T, heads, d] on the GPU, dense or as a view."""
    if layout == "fused":                              # beside other heads of the same token
        wide = torch.cat([x, x[:, :1] if extra is None else extra], 1).to(DEV)
        return wide[:, :x.shape[1]]
    if layout == "heads":                              # [heads, T, d]
        return x.transpose(0, 1).contiguous().to(DEV).transpose(0, 1)
    return x.to(DEV)


def _near(got, want, off, what):
    """Element by element; NaN where NaN, infinities where infinities."""
    got, want = got.cpu().double(), want.double()
    same = (got == want) | (got.isnan() & want.isnan())
    bad = ~(same | ((got - want).abs() <= off))
    assert not bad.any(), "%s: %d of %d off, first %s: %r, %r" % (what, int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist(), got[bad][0].item(), want[bad][0].item())


# ---- rotary positions ------------------------------------------------------------------------

ROPE = [  # T, Hq, Hkv, d, rot, layout, memory
    (1, 1, 1, 8, 2, "half", "dense"), (1, 32, 8, 128, 128, "half", "fused"), (3, 5, 2, 64, 64, "interleaved", "heads"), (17, 3, 1, 80, 20, "half", "dense"),
    (17, 3, 1, 80, 20, "interleaved", "fused"), (40, 2, 2, 96, 48, "half", "fused"), (40, 2, 2, 96, 96, "interleaved", "dense"), (5, 71, 1, 256, 256, "half", "dense"),
    (5, 2, 1, 256, 66, "half", "heads"), (9, 4, 4, 72, 72, "half", "dense"), (256, 2, 1, 128, 32, "half", "dense"), (257, 9, 3, 128, 64, "half", "fused"),
    (1030, 3, 2, 40, 40, "half", "dense"), (1030, 7, 1, 128, 126, "half", "fused"), (700, 20, 20, 24, 10, "interleaved", "heads"), (300, 33, 2, 192, 160, "half", "dense"),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,Hq,H,d,rot,layout,memory", ROPE)
def test_rotation(dtype, T, Hq, H, d, rot, layout, memory):
    laq = _laq()
    print("case:", dtype, T, Hq, H, d, rot, layout, memory, flush=True)
    gen = torch.Generator().manual_seed(T * 31 + d + rot)
    q, k = torch.randn(T, Hq, d, generator=gen).to(dtype), (torch.randn(T, H, d, generator=gen) * 5).to(dtype)
    q[0, 0, -1] = -0.0
    far = [0, 1, -1, 1000003, -77777, 2 ** 31 - 1, -2 ** 31, 131071]
    positions = torch.randint(-5, 70000, (T,), generator=gen)
    positions[:len(far)] = torch.tensor(far)[:T]
    rope = laq.Rope(laq.laq_rope_frequencies(rot, 10000.0, device=DEV), layout, 1.0 if d != 96 else 1.2079441541679836)
    qd, kd, pd = _laid(q, memory), _laid(k, memory), positions.int().to(DEV)
    q_out, k_out = laq.laq_rope(qd, kd, pd, rope)
    torch.cuda.synchronize()
    for x, got, name in ((q, q_out, "q"), (k, k_out, "k")):
        want, size = plain.rotate(x, positions, rope.inv_freq.cpu(), layout, rope.mscale)
        _near(got, want, plain.rotation_error(want, size, dtype), name)
        assert torch.equal(got.cpu()[..., rot:], x[..., rot:])
    # alone, in place and into a view: the same bits
    alone, none = laq.laq_rope(None, kd, pd, rope)
    assert alone is None and torch.equal(none, k_out)
    wide = torch.zeros(T, Hq + 3, d, dtype=dtype, device=DEV)
    got, _ = laq.laq_rope(qd, None, pd, rope, q_out=wide[:, 2:2 + Hq])
    assert torch.equal(got, q_out) and not wide[:, :2].any() and not wide[:, -1].any()
    both = laq.laq_rope(qd, kd, pd, rope, q_out=qd, k_out=kd)
    torch.cuda.synchronize()
    assert both[0] is qd and torch.equal(qd, q_out) and torch.equal(kd, k_out)


def test_rotated_back_and_by_nothing():
    laq = _laq()
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(50, 4, 128, generator=gen).to(DEV)
    rope = laq.Rope(laq.laq_rope_frequencies(128, 500000.0, "parts", 8.0, 8192, 1.0, 4.0, device=DEV))
    p = torch.randint(0, 1 << 20, (50,), generator=gen).int().to(DEV)
    there, _ = laq.laq_rope(x, None, p, rope)
    back, _ = laq.laq_rope(there, None, -p, rope)
    # two rotations, four roundings of numbers up to sqrt(2) of a pair each
    size = (x[..., :64].square() + x[..., 64:].square()).sqrt()
    assert ((back - x).abs() <= 12 * 2.0 ** -24 * torch.cat([size, size], -1)).all()
    still, _ = laq.laq_rope(x, None, torch.zeros_like(p), rope)
    assert torch.equal(still, x)


def test_infinite_and_nan_numbers_stay_with_their_pair():
    laq = _laq()
    x = torch.ones(4, 2, 64, device=DEV, dtype=BF16)
    x[1, 0, 3], x[2, 1, 50], x[3, 0, 63] = math.nan, math.inf, math.nan
    rope = laq.Rope(laq.laq_rope_frequencies(48, device=DEV))
    y, _ = laq.laq_rope(x, None, torch.arange(4, dtype=torch.int32, device=DEV) + 5, rope)
    odd = ~torch.isfinite(y)
    want = torch.zeros_like(odd)
    want[1, 0, 3] = want[1, 0, 27] = want[2, 1, 50] = want[3, 0, 63] = True
    assert torch.equal(odd, want)


# ---- rows into the cache and back ------------------------------------------------------------

APPEND = [  # T, H, d, block rows, memory, token major
    (1, 1, 8, 16, "dense", False), (3, 2, 64, 16, "dense", True), (50, 3, 96, 48, "fused", False), (257, 8, 128, 64, "dense", False), (130, 5, 160, 16, "fused", True),
    (77, 1, 72, 256, "heads", False), (200, 2, 256, 32, "fused", False), (64, 4, 192, 128, "heads", True), (300, 3, 80, 16, "dense", False),
]


@pytest.mark.parametrize("kind", [F32, BF16, E4M3])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,H,d,br,memory,token_major", APPEND)
def test_appended_rows_have_the_plain_bits_and_come_back(kind, dtype, T, H, d, br, memory, token_major):
    laq = _laq()
    print("case:", kind, dtype, T, H, d, br, memory, token_major, flush=True)
    gen = torch.Generator().manual_seed(T * 7 + d)
    k, v = _special(T, H, d, dtype, gen), _special(T, H, d, dtype, gen).flip(0)
    n_blocks = -(-T // br) + 2
    slots = torch.randperm(n_blocks * br, generator=gen)[:T].int()
    slots[T // 2::5] = -1                             # some tokens without a place, and some beyond the pool
    slots[T // 3::11] = n_blocks * br + 3
    here = (slots >= 0) & (slots < n_blocks * br)
    cache = _pool(n_blocks, H, br, d, kind, token_major)
    assert laq.laq_cache_append(cache, _laid(k, memory), _laid(v, memory), slots.to(DEV)) is None
    torch.cuda.synchronize()
    b, r = slots[here].long() // br, slots[here].long() % br
    for x, plane, scales in ((k, cache.k, cache.k_scale), (v, cache.v, cache.v_scale)):
        want = torch.full(_bytes(plane).shape, 0xA5, dtype=torch.uint8)
        if kind == E4M3:
            codes, sc = plain.quantise(x[here])
            want_scales = torch.full(scales.shape, 0xA5, dtype=torch.uint8)
            want[b, :, r], want_scales[b, :, r] = codes, sc
            assert torch.equal(scales.cpu(), want_scales)
        else:
            want[b, :, r] = x[here].to(kind).contiguous().view(torch.uint8)
            nan = torch.zeros(want.shape[:3] + (d,), dtype=torch.bool)
            nan[b, :, r] = x[here].isnan()
            got = plane.cpu().contiguous()
            assert got[nan].isnan().all()             # (any NaN is one)
            size = want.shape[3] // d
            same = (_bytes(plane) == want).unflatten(-1, (d, size)).all(-1) | nan
            assert same.all()
        if kind == E4M3:
            assert torch.equal(_bytes(plane), want)
    for out in (BF16, F32):
        kk, vv = laq.laq_cache_load(cache, slots.to(DEV), out)
        torch.cuda.synchronize()
        for x, got in ((k, kk), (v, vv)):
            want = torch.zeros(T, H, d, dtype=torch.float64)
            want[here] = plain.held(x[here], kind)
            _near(got, want.to(out), 0.0, "load")
    # K alone leaves V as it is
    before = [None if t is None else t.clone() for t in cache]
    laq.laq_cache_append(cache, _laid(v, memory), None, slots.to(DEV))
    torch.cuda.synchronize()
    assert torch.equal(_bytes(before[2]), _bytes(cache.v)) and (kind != E4M3 or torch.equal(before[3], cache.v_scale))


@pytest.mark.parametrize("kind", [F32, BF16, E4M3])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,Hq,H,d,rot,layout,br", [(1, 8, 2, 128, 128, "half", 64), (70, 3, 3, 64, 32, "interleaved", 16), (300, 14, 2, 96, 96, "half", 48), (20, 4, 1, 80, 20, "half", 16)])
def test_rows_rotated_on_the_way(kind, dtype, T, Hq, H, d, rot, layout, br):
    laq = _laq()
    print("case:", kind, dtype, T, Hq, H, d, rot, layout, br, flush=True)
    gen = torch.Generator().manual_seed(T + d)
    q, k, v = (torch.randn(T, h, d, generator=gen).to(dtype) for h in (Hq, H, H))
    positions = torch.randint(0, 200000, (T,), generator=gen)
    n_blocks = -(-T // br) + 1
    slots = torch.randperm(n_blocks * br, generator=gen)[:T].int()
    slots[1::4] = -1
    rope = laq.Rope(laq.laq_rope_frequencies(rot, device=DEV), layout, 1.1)
    qkv = torch.cat([q, k, v], 1).to(DEV)
    qd, kd, vd = qkv.split((Hq, H, H), 1)
    cache = _pool(n_blocks, H, br, d, kind)
    pd, sd = positions.int().to(DEV), slots.to(DEV)
    got_q = laq.laq_cache_append(cache, kd, vd, sd, q=qd, positions=pd, rope=rope)
    same_q, same_k = laq.laq_rope(qd, kd, pd, rope)
    kk, vv = laq.laq_cache_load(cache, sd, F32)
    torch.cuda.synchronize()
    assert torch.equal(got_q, same_q)
    here = slots >= 0
    want, size = plain.rotate(k, positions, rope.inv_freq.cpu(), layout, 1.1)
    off = plain.rotation_error(want, size, F32)
    if kind == BF16:                                  # rounded once, from fp32
        off = off + (want.abs() + off) * 2.0 ** -8
    if kind == E4M3:                                  # half a step: 2^-4, or 2^-10 of the scale, which is 2^-7 of the largest magnitude at most
        most = (want.abs() + off).amax(-1, keepdim=True)
        off = off + torch.maximum((want.abs() + off) * 2.0 ** -4, most * 2.0 ** -17)
    _near(kk[here.to(DEV)], want[here], off[here], "k")
    _near(vv[here.to(DEV)], plain.held(v[here], kind), 0.0, "v")
    assert not kk[~here.to(DEV)].any() and not vv[~here.to(DEV)].any()
    if kind == dtype:                                 # rotated and appended apart: the same bits
        apart = _pool(n_blocks, H, br, d, kind)
        laq.laq_cache_append(apart, same_k, vd, sd)
        torch.cuda.synchronize()
        assert torch.equal(_bytes(apart.k), _bytes(cache.k)) and torch.equal(_bytes(apart.v), _bytes(cache.v))
    # queries in place
    assert laq.laq_cache_append(cache, kd, vd, sd, q=qd, positions=pd, rope=rope, q_out=qd) is qd
    torch.cuda.synchronize()
    assert torch.equal(qd, got_q) and torch.equal(kd.cpu(), k)


@pytest.mark.parametrize("kind", [F32, BF16, E4M3])
@pytest.mark.parametrize("dtype,n,H,d,L,budgets,br,layout", [
    (BF16, 1, 8, 128, 300, [64], 64, "dense"), (BF16, 3, 2, 64, 513, [5, 600, 1], 16, "token-major"), (F32, 2, 3, 96, 100, [33, 100], 48, "dense"),
    (F32, 2, 1, 256, 700, [128, 1], 16, "paged"), (BF16, 300, 1, 32, 20, [7] * 150 + [20] * 150, 16, "dense"), (BF16, 1, 4, 80, 77, [77], 32, "dense")])
def test_compacted_rows_have_the_bits_of_appended_ones(kind, dtype, n, H, d, L, budgets, br, layout):
    laq = _laq()
    print("case:", kind, dtype, n, H, d, L, br, layout, flush=True)
    gen = torch.Generator().manual_seed(L + d)
    k, v = torch.randn(n, H, L, d, generator=gen).to(dtype).to(DEV), (3 * torch.randn(n, H, L, d, generator=gen)).to(dtype).to(DEV)
    kept = [min(b, L) for b in budgets]
    idx = [torch.stack([torch.randperm(L, generator=gen)[:b].sort().values for _ in range(H)]).int() for b in kept]
    if n == 3:
        idx[1][0, 3], idx[0][1, 2] = L, -1                # left out
    total = sum(kept)
    n_blocks = -(-total // br) + 2
    slots = torch.randperm(n_blocks * br, generator=gen)[:total].int()
    slots[::9] = -1
    kw, kd, vd = {}, k, v
    if layout == "token-major":
        kd, vd = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v))
    if layout == "paged":
        per = -(-L // 256)
        table = torch.randperm(n * per, generator=gen).view(n, per).int()
        kd, vd = (torch.zeros(n * per, H, 256, d, dtype=dtype, device=DEV) for _ in range(2))
        for i in range(n):
            for b in range(per):
                rows = min(256, L - b * 256)
                kd[table[i, b], :, :rows], vd[table[i, b], :, :rows] = k[i, :, b * 256:b * 256 + rows], v[i, :, b * 256:b * 256 + rows]
        kw = dict(block_table=table.to(DEV), L=L)
    cache, want = _pool(n_blocks, H, br, d, kind), _pool(n_blocks, H, br, d, kind)
    laq.laq_cache_compact(cache, kd, vd, torch.cat([x.flatten() for x in idx]).to(DEV), budgets, slots.to(DEV), **kw)
    first = 0
    for i, b in enumerate(kept):                          # row by row, head by head
        for h in range(H):
            ok = (idx[i][h] >= 0) & (idx[i][h] < L)
            rows = idx[i][h].clamp(0, L - 1).long().to(DEV)
            one = laq.PagedCache(*(None if t is None else t[:, h:h + 1].contiguous() for t in want))
            laq.laq_cache_append(one, k[i, h, rows][:, None], v[i, h, rows][:, None], torch.where(ok, slots[first:first + b], -1).int().to(DEV))
            for t, o in zip(want, one):
                if t is not None:
                    t.view(torch.uint8)[:, h:h + 1] = o.view(torch.uint8)
        first += b
    torch.cuda.synchronize()
    for got, exp in zip(cache, want):
        assert got is None or torch.equal(_bytes(got), _bytes(exp))


# ---- attention -------------------------------------------------------------------------------

class Case:
    """Requests with rows in a shuffled pool whose other rows hold NaN."""

    def __init__(self, dtype, kind, Hq, H, d, br, rows, tokens, seed=0, token_major=False, fused=False, spread=1.0, special=None):
        laq = _laq()
        gen = torch.Generator().manual_seed(seed + sum(rows) + d)
        self.dtype, self.kind, self.Hq, self.H, self.d, self.br, self.rows, self.tokens = dtype, kind, Hq, H, d, br, list(rows), list(tokens)
        n = len(rows)
        have = [-(-r // br) for r in rows]
        self.n_blocks = sum(have) + 2
        order = torch.randperm(self.n_blocks, generator=gen)
        self.width = max(1, max(have)) + 1
        table = torch.full((n, self.width), -1, dtype=torch.int32)
        first = 0
        for i, b in enumerate(have):
            table[i, :b] = order[first:first + b].int()
            first += b
        self.slots = torch.cat([table[i, torch.arange(r) // br] * br + torch.arange(r) % br for i, r in enumerate(rows)] + [torch.zeros(0, dtype=torch.int32)]).int()
        total = sum(rows)
        k = torch.randn(total, H, d, generator=gen) * spread
        v = torch.randn(total, H, d, generator=gen)
        if special is not None:
            special(k, v)
        # every byte that no row is written to: a NaN in each type
        self.cache = _pool(self.n_blocks, H, br, d, kind, token_major, 0xFF)
        if total:
            laq.laq_cache_append(self.cache, k.to(DEV), v.to(DEV), self.slots.to(DEV))
        self.k, self.v = plain.held(k, kind), plain.held(v, kind)
        self.start = [0]
        for t in tokens:
            self.start.append(self.start[-1] + t)
        q = torch.randn(self.start[-1], Hq, d, generator=gen).to(dtype)
        self.q = q.double()
        self.qd = torch.cat([q, q], 1).to(DEV)[:, :Hq] if fused else q.to(DEV)
        self.table, self.rows_d = table.to(DEV), torch.tensor(rows, dtype=torch.int32, device=DEV)
        self.start_d = torch.tensor(self.start, dtype=torch.int32, device=DEV)
        self.hidden = [set() for _ in rows]

    def run(self, start=True, **kw):
        kw.setdefault("max_rows", max(1, max(self.rows)))
        kw.setdefault("want_lse", True)
        return _laq().laq_cache_attention(self.qd, self.cache, self.table, self.rows_d, start=self.start_d if start else None, **kw)

    def check(self, out, lse, scale=None, what=""):
        """Element by element.  With u = 2^-24 (fp32) and A the largest sum of |q k| * scale of a token: a logit is off by at most (d + 4) u A (sums of d
        products in any order, the scale), the maximum's own rounding and the exponential's argument by 2 u A more, the exponential by 2^-22.  A weight
        p is therefore off by e = 2 u (d + 16) A + 2^-22 of it, a sum of L weights in any order by L u more (the parts of a cut one by a few), in numerator and
        denominator.  bf16: every weight in the numerator is rounded, 2^-8 of it at most, and the result, 2^-8."""
        scale = scale or 1.0 / math.sqrt(self.d)
        u, half = 2.0 ** -24, 2.0 ** -8 if self.dtype == BF16 else 2.0 ** -24
        out, lse = out.cpu().double(), lse.cpu().double()
        first = 0
        for i, r in enumerate(self.rows):
            keep = [j for j in range(r) if j not in self.hidden[i]]
            k, v = (x[first:first + r][keep].transpose(0, 1).contiguous() for x in (self.k, self.v))
            first += r
            for t in range(self.tokens[i]):
                tok = self.start[i] + t
                seen = sum(1 for j in keep if j <= r - self.tokens[i] + t)
                o, l, a, A = fp4_plain.attention(self.q[tok], k, v, seen, scale)
                where = "%s request %d token %d" % (what, i, t)
                if seen == 0:
                    assert (out[tok] == 0).all() and (lse[tok] == -math.inf).all(), where
                    continue
                e = (2 * u * (self.d + 16) * A + 2.0 ** -22 + (seen + 64) * u)[:, None]
                tol = (2 * e + half) * a + half * o.abs() + 1e-30
                bad = ~((out[tok] - o).abs() <= tol)
                assert not bad.any(), "%s: %d of %d outputs off, by up to %.3g of the bound" % (where, int(bad.sum()), bad.numel(), float(((out[tok] - o).abs() / tol).max()))
                assert ((lse[tok] - l).abs() <= 2 * e[:, 0] + 4 * u * l.abs()).all(), where
        assert first == sum(self.rows)


ONE = [  # one token per request: (dtype, cache, Hq, H, d, block, lengths)
    (BF16, BF16, 4, 4, 32, 16, [1]), (BF16, BF16, 32, 8, 128, 64, [520]), (BF16, E4M3, 32, 8, 128, 64, [520, 2100]),
    (BF16, BF16, 8, 8, 64, 16, [1, 2, 15, 16, 17, 31, 33, 64, 65]), (BF16, E4M3, 28, 4, 96, 48, [127, 128, 129, 700]), (BF16, BF16, 28, 4, 80, 48, [127, 128, 129, 700]),
    (BF16, BF16, 8, 1, 128, 256, [1000, 3]), (BF16, E4M3, 16, 1, 160, 32, [95, 0, 300]), (BF16, BF16, 17, 1, 128, 16, [70]), (BF16, BF16, 40, 1, 64, 64, [200, 1]),
    (BF16, E4M3, 71, 1, 64, 128, [333]), (BF16, BF16, 6, 2, 192, 16, [257, 255]), (BF16, E4M3, 3, 3, 8, 80, [161]), (BF16, BF16, 8, 2, 256, 64, [63, 1000]),
    (BF16, BF16, 40, 2, 256, 64, [63, 1000]), (BF16, E4M3, 2, 1, 128, 128, [5000, 17, 1025]), (BF16, BF16, 8, 8, 128, 16, [300 + 13 * i for i in range(40)]),
    (BF16, BF16, 32, 8, 64, 64, [4100, 1, 0, 700, 4096, 33, 0, 2000]), (BF16, E4M3, 3, 1, 24, 16, [9000] + [5] * 30),
    (F32, F32, 4, 4, 32, 16, [3, 40]), (F32, F32, 28, 4, 96, 16, [700, 1]), (F32, BF16, 32, 8, 128, 64, [130, 513]), (F32, E4M3, 17, 1, 64, 32, [99]), (F32, F32, 17, 1, 256, 48, [150, 31]),
    (F32, E4M3, 8, 2, 192, 16, [64, 65]), (F32, BF16, 3, 1, 160, 16, [17]), (F32, F32, 1, 1, 128, 256, [3000]), (F32, E4M3, 9, 3, 72, 16, [777, 4000]),
    (F32, BF16, 35, 1, 256, 16, [777, 40]),
]


@pytest.mark.parametrize("dtype,kind,Hq,H,d,br,rows", ONE)
def test_one_token_per_request(dtype, kind, Hq, H, d, br, rows):
    print("case:", dtype, kind, Hq, H, d, br, rows, flush=True)
    c = Case(dtype, kind, Hq, H, d, br, rows, [1] * len(rows), token_major=d % 64 == 0 and br == 64, fused=br == 48)
    c.check(*c.run(start=False), what="parts")
    c.check(*c.run(start=False, split=False), what="whole")
    c.check(*c.run(start=True), what="with start")


MANY = [
    (BF16, BF16, 8, 2, 128, 64, [600, 9, 40, 8], [8, 8, 1, 8]), (BF16, E4M3, 8, 2, 128, 16, [2100, 9], [20, 9]), (BF16, BF16, 32, 8, 128, 64, [700, 300], [130, 77]),
    (BF16, BF16, 4, 4, 64, 16, [257, 64, 3], [257, 64, 3]), (BF16, E4M3, 28, 4, 96, 48, [500], [100]), (BF16, BF16, 7, 1, 80, 32, [90, 0, 50], [3, 0, 50]),
    (BF16, BF16, 3, 3, 256, 16, [300], [60]), (BF16, E4M3, 12, 2, 192, 16, [300, 2], [16, 2]), (BF16, BF16, 2, 2, 40, 16, [100, 20], [30, 25]),
    (F32, F32, 28, 4, 96, 16, [1500, 700], [8, 8]), (F32, F32, 4, 2, 64, 16, [300, 40], [70, 40]), (F32, E4M3, 8, 2, 128, 32, [513], [33]), (F32, BF16, 3, 1, 256, 16, [90], [40]),
    (F32, F32, 6, 1, 256, 16, [90, 700], [40, 3]), (F32, F32, 2, 1, 128, 16, [50, 6], [60, 9]),
]


@pytest.mark.parametrize("dtype,kind,Hq,H,d,br,rows,tokens", MANY)
def test_several_tokens_see_up_to_their_own_row(dtype, kind, Hq, H, d, br, rows, tokens):
    print("case:", dtype, kind, Hq, H, d, br, rows, tokens, flush=True)
    c = Case(dtype, kind, Hq, H, d, br, rows, tokens, token_major=br == 64, fused=br == 48)
    c.check(*c.run(), what="parts")
    c.check(*c.run(split=False), what="whole")


PROMPTS = [  # bf16, enough score rows and columns for the kernel of whole prompts: (cache, Hq, H, d, block, lengths, tokens)
    (BF16, 32, 32, 128, 16, [300, 64, 40, 41], [40, 33, 40, 35]), (E4M3, 32, 32, 128, 64, [300, 200, 40, 129, 37], [40, 64, 40, 65, 1]),
    (BF16, 32, 32, 96, 48, [300, 140, 50, 0], [129, 128, 50, 3]), (E4M3, 16, 16, 80, 16, [200, 130, 50, 90], [130, 129, 60, 0]), (BF16, 32, 32, 64, 32, [500, 300, 70, 90], [64, 64, 70, 80]),
    (E4M3, 32, 32, 24, 16, [150, 64, 70, 90], [64, 64, 70, 80]), (BF16, 32, 8, 128, 64, [700, 300, 129, 600], [130, 120, 110, 100]), (BF16, 14, 2, 128, 256, [513], [513]),
    (E4M3, 28, 4, 128, 16, [1030, 64], [150, 64]), (BF16, 4, 2, 72, 16, [40 + i for i in range(70)], [17 + i % 5 for i in range(70)]), (BF16, 40, 1, 128, 32, [30 + 2 * i for i in range(130)], [1] * 130),
]


@pytest.mark.parametrize("kind,Hq,H,d,br,rows,tokens", PROMPTS)
def test_prompts(kind, Hq, H, d, br, rows, tokens):
    print("case:", kind, Hq, H, d, br, rows, tokens, flush=True)
    c = Case(BF16, kind, Hq, H, d, br, rows, tokens, token_major=br == 64, fused=br == 48)
    got = c.run()
    c.check(*got)
    again = c.run(split=False)
    c.check(*again)
    if _laq().laq_cache_attention_workspace_bytes(c.cache, Hq, BF16, len(rows), sum(tokens), max(rows)) == 0:      # (that kernel shares nothing out)
        assert all(torch.equal(x, y) for x, y in zip(got, again))


@pytest.mark.parametrize("kind", [BF16, E4M3])
def test_blocks_of_prompts_that_are_not_there(kind):
    c = Case(BF16, kind, 32, 32, 128, 32, [300, 200, 70, 90], [40, 50, 60, 90])
    for i, page, bad in ((0, 2, -1), (0, 9, c.n_blocks), (1, 0, 2 ** 31 - 1), (2, 0, -5), (3, 1, c.n_blocks)):
        c.table[i, page] = bad
        c.hidden[i] |= set(range(32 * page, 32 * page + 32))
    c.check(*c.run())


@pytest.mark.parametrize("kind", [BF16, E4M3])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("at", [299, 260, 270, 100, 290])
def test_odd_numbers_of_prompts_reach_those_that_see_them_alone(kind, what, at):
    def put(k, v):
        v[at, 3, 50] = what
        k[300 + 60, 5, 7] = what
    c = Case(BF16, kind, 32, 32, 128, 16, [300, 100, 70, 90], [40, 50, 60, 90], special=put)
    out, lse = c.run()
    torch.cuda.synchronize()
    want, odd_lse = torch.zeros(out.shape, dtype=torch.bool), torch.zeros(lse.shape, dtype=torch.bool)
    first = max(0, at - 260)
    if kind == E4M3:
        want[first:40, 3] = True
    else:
        want[first:40, 3, 50] = True
    # a key with a NaN makes one of every token that sees it; one with an infinity of half of them or so (a weight of 0 otherwise)
    odd_k = ~torch.isfinite(out.cpu())
    odd_k[:40] = False
    got = ~torch.isfinite(out.cpu())
    got[40:] = False
    assert torch.equal(got, want)
    if kind != E4M3:
        x = out.cpu()[first:40, 3, 50]
        assert x.isnan().all() if math.isnan(what) else (x == what).all()
    seen = torch.zeros(out.shape[:2], dtype=torch.bool)
    seen[50:90, 5] = True
    if math.isnan(what) or kind == E4M3:
        assert torch.equal(odd_k.all(-1), seen) and torch.equal(odd_k.any(-1), seen)
    else:
        assert not (odd_k.any(-1) & ~seen).any()


@pytest.mark.parametrize("dtype,kind", [(BF16, BF16), (BF16, E4M3), (F32, F32)])
def test_rows_that_are_not_there(dtype, kind):
    c = Case(dtype, kind, 8, 2, 64, 32, [900, 700, 64], [3, 1, 2])
    n_blocks = c.n_blocks
    for i, page, bad in ((0, 2, -1), (0, 20, n_blocks), (1, 0, 2 ** 31 - 1), (2, 0, -5), (2, 1, n_blocks)):
        c.table[i, page] = bad
        c.hidden[i] |= set(range(32 * page, 32 * page + 32))
    c.check(*c.run(), what="parts")
    c.check(*c.run(split=False), what="whole")


@pytest.mark.parametrize("dtype,kind,tokens", [(BF16, E4M3, 1), (F32, F32, 1), (BF16, BF16, 40)])
def test_lengths_beyond_the_bound_and_beyond_the_table(dtype, kind, tokens):
    c = Case(dtype, kind, 8, 2, 64, 16, [3000, 1500, 2200], [tokens] * 3)
    c.check(*c.run(max_rows=300), what="short bound")
    # a length that the table cannot hold counts as what it holds: 16 rows more, in a block that is not there
    c.rows_d[1] = 2 ** 31 - 1
    c.rows_d[0] = -7
    out, lse = c.run()
    torch.cuda.synchronize()
    last = torch.arange(tokens)
    assert not out[last].any() and (lse[last] == -math.inf).all()
    # (rows 1500 to 1503, which its last block has room for and which were never written, are then request 1's own: NaN)
    assert out[tokens:2 * tokens].isnan().all() and torch.isfinite(out[2 * tokens:]).all()


@pytest.mark.parametrize("dtype,kind", [(BF16, BF16), (F32, E4M3)])
def test_large_logits_scales_and_a_dominant_row(dtype, kind):
    for scale, spread in ((3.0, 4.0), (1e-4, 1.0), (0.7, 30.0)):
        c = Case(dtype, kind, 8, 2, 128, 32, [700, 1300, 40], [1, 1, 5], spread=spread)
        c.check(*c.run(scale=scale), scale=scale, what="scale %g" % scale)


@pytest.mark.parametrize("split", [True, False])
@pytest.mark.parametrize("dtype,kind,tokens,Hq,H,d", [(BF16, BF16, 1, 4, 2, 64), (BF16, BF16, 5, 4, 2, 64), (BF16, E4M3, 30, 4, 2, 64), (BF16, BF16, 30, 8, 2, 160), (BF16, E4M3, 50, 32, 8, 128),
                                                      (F32, F32, 5, 4, 2, 128), (F32, BF16, 30, 4, 2, 64), (F32, E4M3, 20, 8, 2, 160), (F32, F32, 3, 4, 2, 256), (BF16, BF16, 300, 4, 2, 128)])
def test_odd_numbers_in_v_reach_those_that_see_them_alone(split, dtype, kind, tokens, Hq, H, d):
    rows = 700
    inf = math.inf if kind != E4M3 else math.nan              # (a row of 8 bits with an infinity stands for NaN)
    for at, what in ((rows - 1, math.nan), (rows - tokens, inf), (rows - tokens // 2 - 1, -inf), (rows - 1 - min(tokens - 1, 2), math.nan)):
        def put(k, v):
            v[at, 0, d // 2] = what
        c = Case(dtype, kind, Hq, H, d, 16, [rows, 40], [tokens, 1], special=put)
        out, lse = c.run(split=split)
        torch.cuda.synchronize()
        G = Hq // H
        want = torch.zeros(out.shape, dtype=torch.bool)
        first_seer = max(0, at - (rows - tokens))
        if kind == E4M3:
            want[first_seer:tokens, :G] = True
        else:
            want[first_seer:tokens, :G, d // 2] = True
        assert torch.equal(~torch.isfinite(out.cpu()), want), (at, what)
        if kind != E4M3:
            got = out.cpu()[first_seer:tokens, :G, d // 2]
            assert got.isnan().all() if math.isnan(what) else (got == what).all()
        assert torch.isfinite(lse).all()
        # and the others have their values
        c.v[at, 0] = 0 if kind == E4M3 else c.v[at, 0].nan_to_num(0, 0, 0)
        keep = torch.where(want, torch.zeros(()), out.cpu().float())
        fixed = Case.__new__(Case)
        fixed.__dict__.update(c.__dict__)
        for tok in (0, tokens - 1, tokens):
            i, t = (0, tok) if tok < tokens else (1, 0)
            first = 0 if i == 0 else rows
            r = c.rows[i]
            k, v = (x[first:first + r].transpose(0, 1).contiguous() for x in (c.k, c.v))
            o, _, a, A = fp4_plain.attention(c.q[tok], k, v, r - c.tokens[i] + t + 1, 1 / math.sqrt(d))
            e = (2 * 2.0 ** -24 * (d + 16) * A + 2.0 ** -22 + (r + 64) * 2.0 ** -24)[:, None]
            half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
            off = (keep[tok].double() - o).abs() > (2 * e + half) * a + half * o.abs() + 1e-30
            assert not (off & ~want[tok]).any(), (at, what, tok)


@pytest.mark.parametrize("dtype,kind", [(BF16, BF16), (BF16, E4M3), (F32, F32)])
def test_odd_keys_and_queries_stay_with_their_own(dtype, kind):
    def put(k, v):
        k[650, 1, 5] = math.nan
    c = Case(dtype, kind, 8, 2, 128, 16, [700, 40], [60, 1], special=put)
    c.qd[60, 2, 7] = math.inf
    out, lse = c.run()
    torch.cuda.synchronize()
    want = torch.zeros(out.shape[:2], dtype=torch.bool)
    want[10:60, 4:] = True
    want[60, 2] = True
    assert torch.equal(out.isnan().all(-1).cpu(), want) and torch.equal((~torch.isfinite(out)).any(-1).cpu(), want)
    assert torch.equal(~torch.isfinite(lse).cpu(), want)


@pytest.mark.parametrize("dtype,kind,tokens,rows", [(BF16, BF16, [1] * 3, [3000, 17, 900]), (BF16, E4M3, [40, 3, 1], [700, 30, 64]), (F32, F32, [2, 2, 8], [2000, 50, 8])])
def test_replays_give_the_bits_of_eager_calls(dtype, kind, tokens, rows):
    laq = _laq()
    c = Case(dtype, kind, 8, 2, 128, 16, rows, tokens)
    want, want_lse = c.run()
    bytes_ = laq.laq_cache_attention_workspace_bytes(c.cache, 8, dtype, len(rows), c.start[-1], max(rows))
    ws = torch.full((bytes_ + 16,), 0xFF, dtype=torch.uint8, device=DEV)
    out, lse = torch.zeros_like(want), torch.zeros_like(want_lse)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graphs = []
    for _ in range(2):                                # two graphs with one workspace
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            c.run(out=out, lse=lse, ws=ws)
        graphs.append(g)
    for i in range(6):
        out.fill_(7), lse.fill_(7)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        again, _ = c.run(ws=ws)
        torch.cuda.synchronize()
        assert torch.equal(again, want)


def test_another_stream_and_two_at_once():
    c, e = Case(BF16, BF16, 32, 8, 128, 64, [3000, 500], [1, 1]), Case(BF16, E4M3, 8, 2, 64, 16, [2000], [9])
    want, want_e = c.run(), e.run()
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(a):
            x = c.run()
        y = e.run(stream=b)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(x + y, want + want_e))


def test_rows_behind_the_last_sequence_and_batches_without_tokens():
    laq = _laq()
    c = Case(BF16, BF16, 8, 2, 64, 16, [200, 30], [3, 2])
    out, lse = torch.full((9, 8, 64), 5.0, dtype=BF16, device=DEV), torch.full((9, 8), 5.0, device=DEV)
    c.qd = torch.cat([c.qd, torch.full((4, 8, 64), math.nan, dtype=BF16, device=DEV)])
    c.run(out=out, lse=lse)
    torch.cuda.synchronize()
    assert (out[5:] == 5).all() and (lse[5:] == 5).all()
    c.check(out[:5], lse[:5])
    none = torch.zeros(0, 8, 64, dtype=BF16, device=DEV)
    ints = torch.zeros(0, dtype=torch.int32, device=DEV)
    got = laq.laq_cache_attention(none, c.cache, c.table, c.rows_d, start=torch.zeros(3, dtype=torch.int32, device=DEV))
    assert got.shape == (0, 8, 64)
    kv = torch.zeros(0, 2, 64, dtype=BF16, device=DEV)
    rope = laq.Rope(laq.laq_rope_frequencies(64, device=DEV))
    laq.laq_cache_append(c.cache, kv, kv, ints)
    assert laq.laq_cache_append(c.cache, kv, kv, ints, q=none, positions=ints, rope=rope).shape == (0, 8, 64)
    assert laq.laq_rope(none, kv, ints, rope)[1].shape == (0, 2, 64)
    assert laq.laq_cache_load(c.cache, ints)[0].shape == (0, 2, 64)
    torch.cuda.synchronize()


def test_a_start_that_makes_no_sense_stays_in_bounds():
    c = Case(BF16, BF16, 8, 2, 64, 16, [200, 30, 64], [3, 2, 4])
    for start in ([0, 3, 2, 9], [5, 5, 5, 5], [-4, 3, 5, 9], [0, 2 ** 31 - 1, 5, 9], [0, 3, 5, 1000], [2 ** 31 - 1, -2 ** 31, 0, 1], [9, 5, 3, 0]):
        c.start_d.copy_(torch.tensor(start))
        c.run()
        torch.cuda.synchronize()


def test_many_requests_are_found():
    rows = [1 + i * 7 % 50 for i in range(4500)]
    tokens = [min(r, 1 + i % 3) if i % 11 else 0 for i, r in enumerate(rows)]
    c = Case(BF16, BF16, 2, 1, 32, 16, rows, tokens)
    out, lse = c.run()
    some = [0, 1, 63, 64, 65, 4095, 4096, 4097, 4499, 2222]
    torch.cuda.synchronize()
    assert torch.isfinite(out).all()
    firsts = [0]
    for r in rows:
        firsts.append(firsts[-1] + r)
    for i in some:
        for t in range(tokens[i]):
            k, v = (x[firsts[i]:firsts[i + 1]].transpose(0, 1).contiguous() for x in (c.k, c.v))
            o, l, a, _ = fp4_plain.attention(c.q[c.start[i] + t], k, v, rows[i] - tokens[i] + t + 1, 1 / math.sqrt(32))
            got = out[c.start[i] + t].cpu().double()
            assert ((got - o).abs() <= 2.0 ** -8 * (a + o.abs()) + 2.0 ** -14 * a).all(), (i, t)


def test_offsets_beyond_32_bits():
    laq = _laq()
    n_blocks, H, br, d = 70000, 4, 64, 128                # 2.3 * 2^30 numbers a plane
    kind = BF16
    cache = laq.PagedCache(torch.empty(n_blocks, H, br, d, dtype=kind, device=DEV), None, torch.empty(n_blocks, H, br, d, dtype=kind, device=DEV), None)
    gen = torch.Generator().manual_seed(1)
    rows = 130
    k, v = torch.randn(rows, H, d, generator=gen).to(BF16), torch.randn(rows, H, d, generator=gen).to(BF16)
    blocks = [n_blocks - 1, 3, n_blocks - 2]
    table = torch.tensor([blocks], dtype=torch.int32, device=DEV)
    slots = torch.tensor([blocks[j // br] * br + j % br for j in range(rows)], dtype=torch.int32, device=DEV)
    laq.laq_cache_append(cache, k.to(DEV), v.to(DEV), slots)
    kk, vv = laq.laq_cache_load(cache, slots)
    torch.cuda.synchronize()
    assert torch.equal(kk.cpu(), k) and torch.equal(vv.cpu(), v)
    c = Case(BF16, BF16, 8, H, d, br, [rows], [1])
    c.cache, c.table, c.k, c.v = cache, table, k.double(), v.double()
    c.check(*c.run())


@pytest.mark.parametrize("kind", [BF16, E4M3])
def test_evict_into_the_cache_and_decode_on_it(kind):
    """An eviction's rows into the cache, then lookahead steps with rotated queries and keys, each appended and attended to, and dropped again; the loop
    captured gives what it gives step by step."""
    laq = _laq()
    gen = torch.Generator().manual_seed(11)
    n, Hq, H, d, L, W, br, steps = 2, 8, 2, 64, 600, 8, 16, 3
    budgets = [64, 40]
    q, k, v = (torch.randn(n, h, x, d, generator=gen).to(BF16).to(DEV) for h, x in ((Hq, W), (H, L), (H, L)))
    _, idx, k1, v1 = laq.laq_evict(q, k, v, budgets, 7)
    cache = laq.laq_cache(40, H, br, d, kind, device=DEV)
    free, state = laq.laq_block_pool(40, device=DEV)
    rows, table = torch.zeros(n, dtype=torch.int32, device=DEV), torch.full((n, 10), -1, dtype=torch.int32, device=DEV)
    _, slots = laq.laq_block_map(torch.tensor(budgets, dtype=torch.int32, device=DEV), rows, table, free, state, br, n_slots=sum(budgets))
    laq.laq_cache_compact(cache, k, v, idx, budgets, slots)
    rope = laq.Rope(laq.laq_rope_frequencies(d, device=DEV))
    tokens = [tuple(torch.randn(n, h, d, generator=gen).to(BF16).to(DEV) for h in (Hq, H, H)) for _ in range(steps)]
    one = torch.ones(n, dtype=torch.int32, device=DEV)
    new = torch.zeros(n, dtype=torch.int32, device=DEV)
    at = torch.zeros(n, dtype=torch.int32, device=DEV)
    outs = torch.zeros(steps, n, Hq, d, dtype=BF16, device=DEV)
    ws = torch.zeros(laq.laq_cache_attention_workspace_bytes(cache, Hq, BF16, n, n, 100) + 16, dtype=torch.uint8, device=DEV)
    turned = torch.zeros(n, Hq, d, dtype=BF16, device=DEV)

    def loop():
        for t, (qt, kt, vt) in enumerate(tokens):
            laq.laq_block_map(one, rows, table, free, state, br, slots=new)
            at.copy_(one * (L + t))
            laq.laq_cache_append(cache, kt, vt, new, q=qt, positions=at, rope=rope, q_out=turned)
            laq.laq_cache_attention(turned, cache, table, rows, max_rows=100, out=outs[t], ws=ws)
        laq.laq_block_map(-steps * one, rows, table, free, state, br)

    before = free.clone()
    loop()
    torch.cuda.synchronize()
    first = outs.clone()
    assert torch.equal(rows.cpu(), torch.tensor(budgets, dtype=torch.int32)) and torch.equal(free, before) and int(state[1]) == 0
    # against plain attention over what was kept and appended
    r0 = 0
    for i, b in enumerate(budgets):
        kept_k, kept_v = (plain.held(x[r0:r0 + H * b].view(H, b, d).cpu(), kind) for x in (k1, v1))
        r0 += H * b
        for t, (qt, kt, vt) in enumerate(tokens):
            p = torch.tensor([L + t])
            rk, ks = plain.rotate(kt[i:i + 1].cpu(), p, rope.inv_freq.cpu(), "half", 1.0)
            rq, _ = plain.rotate(qt[i:i + 1].cpu(), p, rope.inv_freq.cpu(), "half", 1.0)
            kept_k = torch.cat([kept_k, plain.held(rk[0].float(), kind)[:, None]], 1)
            kept_v = torch.cat([kept_v, plain.held(vt[i].cpu(), kind)[:, None]], 1)
            o, _, a, A = fp4_plain.attention(rq[0].bfloat16().double(), kept_k, kept_v, b + t + 1, 1 / math.sqrt(d))
            # a rotated number next to a border of its type may lie on the other side of it: 2^-3 of a key's number (bf16 2^-7), or a query's 2^-7, in one place of a product
            flip = (2.0 ** -7 + (2.0 ** -3 if kind == E4M3 else 2.0 ** -7)) * A.max() / 8
            got = first[t, i].cpu().double()
            assert ((got - o).abs() <= (2 * flip + 2.0 ** -7) * a + 2.0 ** -8 * o.abs()).all(), (i, t)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        loop()
    for _ in range(4):
        outs.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs, first)
        loop()
        torch.cuda.synchronize()
        assert torch.equal(outs, first)
    # another eviction of what is left: rows read back as the cache holds them
    back = torch.cat([table[i, torch.arange(b, device=DEV) // br] * br + torch.arange(b, device=DEV) % br for i, b in enumerate(budgets)]).int()
    kk, _ = laq.laq_cache_load(cache, back)
    torch.cuda.synchronize()
    assert torch.equal(kk[:64].transpose(0, 1).cpu().double(), plain.held(k1[:H * 64].view(H, 64, d).cpu(), kind))


def test_the_calls_without_the_compiled_binding(monkeypatch):
    laq = _laq()
    from paper_2505_20334_amd import binding
    laq.load_library()
    c = Case(BF16, E4M3, 8, 2, 64, 16, [200, 30], [3, 2])
    gen = torch.Generator().manual_seed(4)
    q, k = torch.randn(5, 4, 64, generator=gen).to(BF16).to(DEV), torch.randn(5, 2, 64, generator=gen).to(BF16).to(DEV)
    p, rope = torch.arange(5, dtype=torch.int32, device=DEV), laq.Rope(laq.laq_rope_frequencies(32, device=DEV), "interleaved")
    src, idx = torch.randn(2, 2, 40, 64, generator=gen).to(BF16).to(DEV), torch.arange(10, dtype=torch.int32, device=DEV).repeat(4)

    def calls():
        cache = _pool(4, 2, 16, 64, E4M3)
        got = list(laq.laq_rope(q, k, p, rope))
        got.append(laq.laq_cache_append(cache, k, k, p, q=q, positions=p, rope=rope))
        laq.laq_cache_compact(cache, src, src, idx, [10, 10], torch.arange(20, 40, dtype=torch.int32, device=DEV))
        got += list(laq.laq_cache_load(cache, torch.arange(-1, 40, dtype=torch.int32, device=DEV), F32)) + list(c.run()) + list(c.run(split=False))
        torch.cuda.synchronize()
        return got
    want = calls()
    monkeypatch.setattr(binding, "_native", None)
    for x, y in zip(want, calls()):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@pytest.mark.parametrize("dtype,kind,tokens,row", [(BF16, BF16, 1, 1 << 24), (F32, F32, 3, 1 << 24), (BF16, E4M3, 40, 1 << 24), (BF16, BF16, 2, (1 << 24) - 8)])
def test_rows_far_apart(dtype, kind, tokens, row):
    laq = _laq()
    d, rows, H = 64, 30, 1
    planes = []
    for _ in range(2):
        flat = torch.empty(32 * row, dtype=torch.uint8 if kind == E4M3 else kind, device=DEV).view(kind)
        planes.append(flat.as_strided((2, H, 16, d), (16 * row, d, row, 1)))
        planes.append(torch.zeros(2, H, 16, dtype=torch.uint8, device=DEV) if kind == E4M3 else None)
    cache = laq.PagedCache(*planes)
    gen = torch.Generator().manual_seed(9)
    k, v = torch.randn(rows, H, d, generator=gen), torch.randn(rows, H, d, generator=gen)
    slots = torch.arange(rows, dtype=torch.int32, device=DEV)
    laq.laq_cache_append(cache, k.to(DEV), v.to(DEV), slots)
    kk, vv = laq.laq_cache_load(cache, slots, F32)
    torch.cuda.synchronize()
    assert torch.equal(kk.cpu().double(), plain.held(k, kind)) and torch.equal(vv.cpu().double(), plain.held(v, kind))
    c = Case(dtype, kind, 2, H, d, 16, [rows], [min(tokens, rows)])
    c.cache, c.table, c.k, c.v = cache, torch.tensor([[0, 1]], dtype=torch.int32, device=DEV), plain.held(k, kind), plain.held(v, kind)
    c.check(*c.run())


@pytest.mark.parametrize("dtype,kind,tokens", [(BF16, BF16, [1, 1, 1]), (F32, E4M3, [3, 1, 2]), (BF16, E4M3, [40, 2, 1])])
def test_as_many_rows_as_a_table_may_hold(dtype, kind, tokens):
    """Lengths next to 2^31: all but the last few blocks are not there."""
    laq = _laq()
    H, d, br = 1, 64, 4096
    long = (1 << 31) - br
    c = Case(dtype, kind, 2, H, d, br, [100, 130, 70], tokens)
    width = long // br
    table = torch.full((3, width), -1, dtype=torch.int32, device=DEV)
    table[:, -1] = c.table[:, 0]
    rows = torch.tensor([long - br + 100, 130, long - br + 70], dtype=torch.int32, device=DEV)
    table[1, 0] = c.table[1, 0]
    c.table, c.rows_d = table, rows
    for max_rows in (long, 4096):
        c.check(*c.run(max_rows=max_rows))
    assert laq.laq_cache_attention_workspace_bytes(c.cache, 2, dtype, 3, sum(tokens), long) < 1 << 30


def test_many_workgroups_of_a_column_on_two_streams_and_in_graphs_with_one_workspace():
    c = Case(BF16, E4M3, 8, 1, 128, 64, [60000], [1])
    e = Case(F32, F32, 8, 2, 64, 16, [9000, 5, 7000], [2, 1, 3])
    want, want_e = c.run(), e.run()
    torch.cuda.synchronize()
    c.check(*want), e.check(*want_e)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        with torch.cuda.stream(a):
            got = c.run()
        with torch.cuda.stream(b):
            got_e = e.run()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got + got_e, want + want_e))
    laq = _laq()
    ws = torch.full((max(laq.laq_cache_attention_workspace_bytes(c.cache, 8, BF16, 1, 1, 60000), laq.laq_cache_attention_workspace_bytes(e.cache, 8, F32, 3, 6, 9000)),), 0xA5,
                    dtype=torch.uint8, device=DEV)
    outs = [tuple(torch.zeros_like(x) for x in w) for w in (want, want_e)]
    graphs = []
    for case, (out, lse) in zip((c, e), outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=a):
            case.run(out=out, lse=lse, ws=ws)
        graphs.append(g)
    for i in range(8):
        for x in outs[i % 2]:
            x.fill_(3)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs[i % 2], (want, want_e)[i % 2]))
        other = (e, c)[i % 2].run(ws=ws)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(other, (want_e, want)[i % 2]))


def test_every_code_and_scale_reads_as_its_number():
    """All scales from 2^-117 to 2^111 and all codes, read back and through the attention of one key."""
    laq = _laq()
    d, br = 256, 16
    scales = list(range(10, 239)) + [255]
    n_blocks = -(-len(scales) // br)
    cache = laq.laq_cache(n_blocks, 1, br, d, E4M3, device=DEV)
    codes = torch.arange(256, dtype=torch.uint8)
    codes[codes & 127 == 127] = 3                         # (NaN)
    cache.k.view(torch.uint8).copy_(codes.expand(n_blocks, 1, br, d)), cache.v.view(torch.uint8).copy_(codes.expand(n_blocks, 1, br, d))
    sc = torch.zeros(n_blocks * br, dtype=torch.uint8)
    sc[:len(scales)] = torch.tensor(scales, dtype=torch.uint8)
    cache.k_scale.copy_(sc.view(n_blocks, 1, br)), cache.v_scale.copy_(sc.view(n_blocks, 1, br))
    slots = torch.arange(len(scales), dtype=torch.int32, device=DEV)
    want = plain.values(codes.expand(len(scales), d), torch.tensor(scales))
    codes_zero = codes & 127 == 0
    for dtype in (F32, BF16):
        kk, vv = laq.laq_cache_load(cache, slots, dtype)
        torch.cuda.synchronize()
        for got in (kk, vv):
            g = got[:-1, 0].cpu().double()
            assert torch.equal(g, want[:-1])
            assert not torch.isfinite(got[-1, 0].cpu()).any()
    # one key: the output is its V (the first row of a block of a request each)
    for dtype in (F32, BF16):
        table = torch.arange(n_blocks, dtype=torch.int32, device=DEV)[:, None].contiguous()
        rows = torch.ones(n_blocks, dtype=torch.int32, device=DEV)
        out = laq.laq_cache_attention(torch.zeros(n_blocks, 1, d, dtype=dtype, device=DEV), cache, table, rows)
        torch.cuda.synchronize()
        assert torch.equal(out[:, 0].cpu().double(), want[::br][:n_blocks])
    assert codes_zero.any()


def _by_definition(c, out, lse, scale=None):
    """Case.check for scores that may be infinite or NaN: a key whose score is -infinity has the weight 0, a token that sees a NaN or +infinity is NaN."""
    scale = scale or 1.0 / math.sqrt(c.d)
    u, half = 2.0 ** -24, 2.0 ** -8 if c.dtype == BF16 else 2.0 ** -24
    out, lse = out.cpu().double(), lse.cpu().double()
    G, first, kinds = c.Hq // c.H, 0, [0, 0, 0]
    for i, r in enumerate(c.rows):
        k, v = (x[first:first + r].transpose(0, 1).repeat_interleave(G, 0) for x in (c.k, c.v))
        first += r
        for t in range(c.tokens[i]):
            tok, seen = c.start[i] + t, r - c.tokens[i] + t + 1
            terms = c.q[tok][:, None] * k[:, :seen] * scale
            s = terms.sum(-1)
            for h in range(c.Hq):
                where = "request %d token %d head %d" % (i, t, h)
                at = s[h] > -math.inf
                if s[h].isnan().any() or (s[h] == math.inf).any():
                    kinds[0] += 1
                    assert out[tok, h].isnan().all() and not torch.isfinite(lse[tok, h]) and lse[tok, h] != -math.inf, where
                elif not at.any():
                    kinds[1] += 1
                    assert (out[tok, h] == 0).all() and lse[tok, h] == -math.inf, where
                else:
                    kinds[2] += 1
                    p, vv = torch.softmax(s[h, at], 0), v[h, :seen][at]
                    o, a, A = p @ vv, p @ vv.abs(), terms[h, at].abs().sum(-1).max()
                    e = 2 * u * (c.d + 16) * A + 2.0 ** -22 + (seen + 64) * u
                    assert ((out[tok, h] - o).abs() <= (2 * e + half) * a + half * o.abs() + 1e-30).all(), where
                    l = torch.logsumexp(s[h, at], 0)
                    assert (lse[tok, h] - l).abs() <= 2 * e + 4 * u * l.abs(), where
    return kinds


ODD = [  # every pair of types, one and two tiles of score rows, each head size, and chunks of prompts: (dtype, cache, Hq, H, d, block, lengths, tokens)
    (BF16, BF16, 8, 2, 128, 16, [300, 40], [1, 1]), (BF16, BF16, 8, 2, 64, 16, [300, 70], [30, 20]), (BF16, E4M3, 8, 2, 128, 64, [300, 40], [1, 1]), (BF16, E4M3, 8, 2, 192, 16, [200, 40], [9, 1]),
    (F32, F32, 8, 2, 128, 16, [300, 40], [1, 1]), (F32, F32, 8, 2, 64, 16, [300, 70], [30, 20]), (F32, E4M3, 8, 2, 128, 16, [300, 40], [1, 1]), (F32, E4M3, 8, 2, 64, 64, [300, 70], [30, 20]),
    (F32, E4M3, 6, 2, 256, 16, [90, 600], [20, 3]), (F32, BF16, 8, 2, 128, 16, [300, 40], [1, 1]), (F32, BF16, 8, 2, 64, 64, [300, 70], [30, 20]), (F32, BF16, 6, 2, 256, 16, [90, 600], [20, 3]),
    (F32, BF16, 28, 4, 96, 48, [700, 1], [8, 1]), (F32, BF16, 2, 2, 24, 16, [2100], [1]), (BF16, BF16, 32, 32, 128, 16, [300, 100, 70, 90], [40, 50, 60, 90]),
    (BF16, E4M3, 64, 64, 64, 64, [150, 64, 70, 90], [64, 64, 70, 80]),
]


@pytest.mark.parametrize("split", [True, False])
@pytest.mark.parametrize("what", [-math.inf, math.inf, math.nan])
@pytest.mark.parametrize("dtype,kind,Hq,H,d,br,rows,tokens", ODD)
def test_infinite_and_nan_keys_have_the_weights_of_their_scores(dtype, kind, Hq, H, d, br, rows, tokens, what, split):
    print("case:", dtype, kind, Hq, H, d, br, rows, tokens, what, split, flush=True)

    def put(k, v):
        for j in (3, 17, rows[0] // 2, rows[0] - 1):
            k[j, 0, d // 2] = what
        k[rows[0] - 1, 1, 0] = what
        k[2, 1, d - 1] = -what
    c = Case(dtype, kind, Hq, H, d, br, rows, tokens, special=put)
    out, lse = c.run(split=split)
    torch.cuda.synchronize()
    kinds = _by_definition(c, out, lse)
    assert kinds[0] and (kinds[2] or Hq == 2)


@pytest.mark.parametrize("split", [True, False])
@pytest.mark.parametrize("dtype,kind,Hq,H,d,br,rows,tokens", ODD)
def test_scores_that_are_all_minus_infinity_give_nothing(dtype, kind, Hq, H, d, br, rows, tokens, split):
    print("case:", dtype, kind, Hq, H, d, br, rows, tokens, split, flush=True)

    def put(k, v):
        k[:rows[0], 0, 0] = -math.inf
    c = Case(dtype, kind, Hq, H, d, br, rows, tokens, special=put)
    c.q[:, :, 0] = (c.q[:, :, 0].abs() + 0.5).to(dtype).double()
    c.qd.copy_(c.q.to(dtype))
    out, lse = c.run(split=split)
    torch.cuda.synchronize()
    kinds = _by_definition(c, out, lse)
    assert kinds[0 if kind == E4M3 else 1] and kinds[2]          # (a row of 8 bits with an infinity stands for NaN)


@pytest.mark.parametrize("split", [True, False])
@pytest.mark.parametrize("what", [-math.inf, math.inf, math.nan])
@pytest.mark.parametrize("dtype,kind,Hq,H,d,br,rows,tokens", ODD)
def test_infinite_and_nan_queries_have_the_weights_of_their_scores(dtype, kind, Hq, H, d, br, rows, tokens, what, split):
    print("case:", dtype, kind, Hq, H, d, br, rows, tokens, what, split, flush=True)

    def put(k, v):
        k[:, 0, 5] = -k[:, 0, 5].abs() - 0.5           # (one sign: all scores of a query with an infinity there are infinities of one sign)
    c = Case(dtype, kind, Hq, H, d, br, rows, tokens, special=put)
    for tok in (0, len(c.q) - 1):
        c.q[tok, 0, 5] = c.q[tok, Hq - 1, d - 2] = what
    c.qd.copy_(c.q.to(dtype))
    out, lse = c.run(split=split)
    torch.cuda.synchronize()
    kinds = _by_definition(c, out, lse)
    assert kinds[1 if what == math.inf else 0] and (kinds[2] or Hq == 2)


@pytest.mark.parametrize("split", [True, False])
@pytest.mark.parametrize("kind,Hq,H,d,br,rows,tokens", [x[1:] for x in ODD if x[0] == F32])
def test_queries_beyond_the_largest_number_of_bf16(kind, Hq, H, d, br, rows, tokens, split):
    print("case:", kind, Hq, H, d, br, rows, tokens, split, flush=True)

    def put(k, v):
        k *= 2.0 ** -100
    c = Case(F32, kind, Hq, H, d, br, rows, tokens, special=put)
    c.q[:, :, 3] = torch.tensor([3.4e38, -3.4028e38]).repeat(Hq // 2).double()
    c.q[0, 0, 3] = torch.finfo(F32).max
    c.qd.copy_(c.q.to(F32))
    c.q = c.q.float().double()
    scale = 2.0 ** -26                                 # (scores of about 2^28)
    c.check(*c.run(split=split, scale=scale), scale=scale)


@pytest.mark.parametrize("dtype,kind,Hq,H,d,n,each", [(BF16, BF16, 8, 2, 64, 3, 3), (F32, E4M3, 8, 2, 128, 3, 9), (BF16, E4M3, 8, 1, 192, 80, 2), (BF16, BF16, 32, 32, 128, 4, 35), (BF16, E4M3, 64, 64, 64, 4, 64),
                                                      (BF16, BF16, 4, 2, 72, 70, 18)])
def test_starts_that_make_no_sense_leave_everything_around_the_output_alone(dtype, kind, Hq, H, d, n, each):
    print("case:", dtype, kind, Hq, H, d, n, each, flush=True)
    c = Case(dtype, kind, Hq, H, d, 16, [each + i * 13 % 90 for i in range(n)], [each] * n)
    T, big = n * each, (1 << 31) - 1
    assert (_laq().laq_cache_attention_workspace_bytes(c.cache, Hq, dtype, n, T, 100) == 0) == (each in (35, 64, 18))      # (both kernels)
    for start in ([0, T, 0, T], [T, 0], [-5, T // 2, T // 2 + 1, 100 * T], [big], [0], [-big, big], [0, T + 1], [T - 1, T, big, -big, T - 2], [T // 2, T // 3, T // 4, T], [0, T] + [T] * (n - 1)):
        values = (start * (n + 1))[:n + 1]
        c.start_d = torch.tensor(values, dtype=torch.int32, device=DEV)
        for split in (True, False):
            bounds, lse = torch.full((T + 60, Hq, d), 5.0, dtype=dtype, device=DEV), torch.full((T + 64, Hq), 5.0, device=DEV)
            c.run(out=bounds[30:30 + T], lse=lse[32:32 + T], split=split)
            torch.cuda.synchronize()
            assert (bounds[:30] == 5.0).all() and (bounds[30 + T:] == 5.0).all() and (lse[:32] == 5.0).all() and (lse[32 + T:] == 5.0).all(), (start, split)
    assert (bounds[30:30 + T] != 5.0).any()            # (the last one: request 0 has all tokens)


CHUNKS = [  # more calls that the kernel of whole prompts takes, each token compared: (cache, Hq, H, d, block, lengths, tokens)
    # numbers of score rows of a group that are no power of two, more than four tiles of a request on average, head sizes that are rounded up
    (BF16, 56, 8, 128, 256, [513], [513]), (E4M3, 140, 20, 128, 16, [430, 64], [150, 64]), (BF16, 112, 16, 80, 64, [300, 150], [150, 130]),
    (E4M3, 64, 64, 80, 16, [200, 130, 50, 90], [130, 129, 60, 0]), (BF16, 32, 32, 80, 32, [200, 130, 50, 90], [130, 129, 50, 1]),
    # columns in the order of lengths: 256 / H of a KV head to a round, the second round backwards.  More than one round, more than two, none whole; no room for one
    (BF16, 64, 32, 64, 16, [700, 200, 90, 300], [300, 200, 90, 64]), (BF16, 64, 64, 32, 64, [900, 300, 500], [300, 129, 40]), (E4M3, 64, 64, 24, 16, [150, 300, 600, 600, 5], [140, 300, 520, 129, 5]),
    (BF16, 64, 64, 72, 16, [520, 150, 150, 600], [520, 150, 150, 129]), (BF16, 260, 260, 16, 16, [300, 41], [140, 40]), (E4M3, 128, 128, 72, 64, [131, 300, 70], [131, 257, 1]),
]


@pytest.mark.parametrize("kind,Hq,H,d,br,rows,tokens", CHUNKS)
def test_chunks_in_any_order_of_lengths(kind, Hq, H, d, br, rows, tokens):
    print("case:", kind, Hq, H, d, br, rows, tokens, flush=True)
    c = Case(BF16, kind, Hq, H, d, br, rows, tokens, token_major=br == 64, fused=br == 32)
    assert _laq().laq_cache_attention_workspace_bytes(c.cache, Hq, BF16, len(rows), sum(tokens), max(rows)) == 0      # (that kernel shares nothing out)
    c.check(*c.run())


EXACT = [  # the calls of bf16 whose weights keep more than bf16's bits: (cache, Hq, H, d, block, lengths, tokens)
    (BF16, 32, 8, 128, 64, [520], [1]), (BF16, 8, 8, 64, 16, [1, 2, 15, 16, 17, 31, 33, 64, 65, 700], [1] * 10), (BF16, 8, 2, 256, 64, [63, 1000], [1, 1]), (BF16, 28, 4, 96, 48, [3000, 700], [1, 1]),
    (E4M3, 32, 8, 128, 64, [520, 2100], [1, 1]), (E4M3, 16, 2, 192, 16, [95, 0, 600], [1, 1, 1]), (E4M3, 8, 2, 64, 48, [900, 40], [4, 4]), (BF16, 8, 2, 128, 64, [600, 9, 40, 8], [8, 8, 1, 8]),
    (BF16, 8, 2, 64, 16, [2000], [20]),
]


@pytest.mark.parametrize("split", [True, False])
@pytest.mark.parametrize("kind,Hq,H,d,br,rows,tokens", EXACT)
def test_the_output_is_what_is_rounded_to_bf16(kind, Hq, H, d, br, rows, tokens, split):
    """Case.check's bounds, but for the weights: two parts of bf16, each rounded by 2^-8 at most, leave 2^-16 of a weight, and the result is rounded once."""
    print("case:", kind, Hq, H, d, br, rows, tokens, split, flush=True)
    c = Case(BF16, kind, Hq, H, d, br, rows, tokens)
    out, _ = c.run(split=split)
    out, u, first = out.cpu().double(), 2.0 ** -24, 0
    for i, r in enumerate(rows):
        k, v = (x[first:first + r].transpose(0, 1).contiguous() for x in (c.k, c.v))
        first += r
        for t in range(tokens[i]):
            seen = r - tokens[i] + t + 1
            o, _, a, A = fp4_plain.attention(c.q[c.start[i] + t], k, v, seen, 1.0 / math.sqrt(d))
            e = (2 * u * (d + 16) * A + 2.0 ** -22 + (seen + 64) * u)[:, None] if seen > 0 else 0.0
            tol = (2 * e + 2.0 ** -16) * a * (1 + 2.0 ** -8) + 2.0 ** -8 * o.abs() + 1e-30
            off = (out[c.start[i] + t] - o).abs()
            assert (off <= tol).all(), "request %d token %d: %d of %d off" % (i, t, int((off > tol).sum()), off.numel())


@pytest.mark.parametrize("dtype,kind,T,Hq,H,d,rot,layout", [
    (BF16, BF16, 513, 8, 2, 128, 128, "half"), (F32, E4M3, 2049, 5, 1, 72, 20, "half"), (BF16, E4M3, 5003, 3, 2, 256, 66, "half"), (F32, BF16, 8193, 4, 4, 64, 64, "interleaved"),
    (BF16, F32, 8195, 2, 1, 192, 192, "half"), (BF16, E4M3, 16381, 32, 8, 128, 128, "half"), (F32, F32, 16381, 28, 4, 96, 40, "half"), (F32, E4M3, 16381, 28, 4, 96, 48, "interleaved")])
def test_long_batches_have_the_bits_of_short_ones(dtype, kind, T, Hq, H, d, rot, layout):
    """Rotated, appended and read back in one call each and 500 tokens at a time, which other shapes of the launch do; the largest go past the caches."""
    laq = _laq()
    print("case:", dtype, kind, T, Hq, H, d, rot, layout, flush=True)
    gen = torch.Generator(device=DEV).manual_seed(T + d)
    qkv = torch.randn(T, Hq + 2 * H, d, generator=gen, device=DEV).to(dtype)
    q, k, v = qkv.split((Hq, H, H), 1)
    positions = torch.randint(-1000, 1 << 20, (T,), generator=gen, device=DEV).int()
    n_blocks = -(-T // 32) + 2
    slots = torch.randperm(n_blocks * 32, generator=gen, device=DEV)[:T].int()
    slots[7::101] = -1
    rope = laq.Rope(laq.laq_rope_frequencies(rot, device=DEV), layout, 1.1)
    at_once, in_parts = _pool(n_blocks, H, 32, d, kind), _pool(n_blocks, H, 32, d, kind)
    got = laq.laq_cache_append(at_once, k, v, slots, q=q, positions=positions, rope=rope)
    got_q, got_k = laq.laq_rope(q, k, positions, rope)
    loaded = laq.laq_cache_load(at_once, slots, dtype)
    for t in range(0, T, 500):
        s = slice(t, t + 500)
        want = laq.laq_cache_append(in_parts, k[s], v[s], slots[s], q=q[s], positions=positions[s], rope=rope)
        want_q, want_k = laq.laq_rope(q[s], k[s], positions[s], rope)
        assert torch.equal(got[s], want) and torch.equal(got_q[s], want) and torch.equal(got_q[s], want_q) and torch.equal(got_k[s], want_k), t
        assert all(torch.equal(x[s], y) for x, y in zip(loaded, laq.laq_cache_load(at_once, slots[s], dtype))), t
    for x, y in zip(at_once, in_parts):
        assert x is None or torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    # in place
    both = laq.laq_rope(q, k, positions, rope, q_out=q, k_out=k)
    torch.cuda.synchronize()
    assert torch.equal(both[0], got_q) and torch.equal(both[1], got_k)


@pytest.mark.parametrize("kind", [F32, BF16, E4M3])
def test_many_compacted_rows_have_the_bits_of_appended_ones(kind):
    """128 MiB of rows, which are read past the caches."""
    laq = _laq()
    gen = torch.Generator(device=DEV).manual_seed(5)
    n, H, d, L, budgets, br = 3, 8, 128, 6200, [6100, 6200, 6001], 64
    k, v = torch.randn(n, H, L, d, generator=gen, device=DEV), torch.randn(n, H, L, d, generator=gen, device=DEV)
    idx = [torch.stack([torch.randperm(L, generator=gen, device=DEV)[:b].sort().values for _ in range(H)]).int() for b in budgets]
    n_blocks = -(-sum(budgets) // br)
    slots = torch.randperm(n_blocks * br, generator=gen, device=DEV)[:sum(budgets)].int()
    cache, want = _pool(n_blocks, H, br, d, kind), _pool(n_blocks, H, br, d, kind)
    laq.laq_cache_compact(cache, k, v, torch.cat([x.flatten() for x in idx]), budgets, slots)
    first = 0
    for i, b in enumerate(budgets):
        rows = idx[i].long()[..., None].expand(-1, -1, d)
        laq.laq_cache_append(want, *(x[i].gather(1, rows).transpose(0, 1) for x in (k, v)), slots[first:first + b])
        first += b
    torch.cuda.synchronize()
    for x, y in zip(cache, want):
        assert x is None or torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@pytest.mark.parametrize("kind,Hq,H,d,n,long,chunk,pad", [(BF16, 32, 8, 128, 20, 3000, 512, 0), (E4M3, 32, 8, 128, 26, 700, 300, 40), (BF16, 8, 2, 64, 70, 400, 1200, 7), (BF16, 32, 8, 128, 16, 900, 1, 240)])
def test_chunks_beside_decoding_requests_and_padding(kind, Hq, H, d, n, long, chunk, pad):
    laq = _laq()
    print("case:", kind, Hq, H, d, n, long, chunk, pad, flush=True)
    tokens = [1] * n
    tokens[n // 2] = chunk
    c = Case(BF16, kind, Hq, H, d, 64, [chunk + 100 if i == n // 2 else 1 + i * 389 % long for i in range(n)], tokens)
    T = c.start[-1]
    out, lse = torch.full((T + pad, Hq, d), 5.0, dtype=BF16, device=DEV), torch.full((T + pad, Hq), 5.0, device=DEV)
    c.qd = torch.cat([c.qd, torch.full((pad, Hq, d), math.nan, dtype=BF16, device=DEV)])
    assert laq.laq_cache_attention_workspace_bytes(c.cache, Hq, BF16, n, T + pad, max(c.rows)) == 0      # (the average number of tokens is that of chunks)
    c.run(out=out, lse=lse)
    torch.cuda.synchronize()
    assert (out[T:] == 5).all() and (lse[T:] == 5).all()
    c.check(out[:T], lse[:T])


CHUNKS8 = [  # 8 bits in the kernel of whole prompts: (Hq, H, d, block, lengths, tokens)
    (64, 64, 128, 64, [300, 200, 40, 129, 37], [40, 64, 40, 65, 1]), (64, 64, 128, 16, [300, 64, 40, 41], [40, 33, 40, 35]), (64, 64, 96, 48, [300, 140, 50, 0], [129, 128, 50, 3]),
    (64, 64, 24, 16, [150, 64, 70, 90], [64, 64, 70, 80]), (64, 64, 64, 32, [500, 300, 70, 90], [64, 64, 70, 80]), (64, 16, 128, 256, [700, 300, 129, 600], [130, 120, 110, 100]),
    (56, 8, 72, 80, [520], [520]), (6, 3, 72, 16, [40 + i for i in range(70)], [17 + i % 5 for i in range(70)]), (80, 2, 128, 128, [30 + 2 * i for i in range(130)], [1] * 130),
]


@pytest.mark.parametrize("Hq,H,d,br,rows,tokens", CHUNKS8)
def test_chunks_over_8_bits(Hq, H, d, br, rows, tokens):
    print("case:", Hq, H, d, br, rows, tokens, flush=True)
    c = Case(BF16, E4M3, Hq, H, d, br, rows, tokens, token_major=br == 64, fused=br == 48)
    assert _laq().laq_cache_attention_workspace_bytes(c.cache, Hq, BF16, len(rows), sum(tokens), max(rows)) == 0
    c.check(*c.run())
    # blocks that are not there
    for i, page, bad in ((0, 0, -1), (len(rows) - 1, 0, c.n_blocks), (0, 1, 2 ** 31 - 1)):
        if page < c.width - 1:
            c.table[i, page] = bad
            c.hidden[i] |= set(range(br * page, br * page + br))
    c.check(*c.run())


@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("d,br", [(128, 16), (128, 64), (40, 32)])
@pytest.mark.parametrize("at", [299, 260, 270, 100, 290])
def test_odd_rows_of_chunks_over_8_bits_reach_those_that_see_them_alone(at, d, br, what):
    def put(k, v):
        v[at, 3, d // 2] = what
        k[300 + 60, 5, 7] = what
    c = Case(BF16, E4M3, 64, 64, d, br, [300, 100, 70, 90], [40, 64, 65, 90], special=put)
    assert _laq().laq_cache_attention_workspace_bytes(c.cache, 64, BF16, 4, 259, 300) == 0
    out, lse = c.run()
    torch.cuda.synchronize()
    want = torch.zeros(out.shape[:2], dtype=torch.bool)
    want[max(0, at - 260):40, 3] = True                # a row of 8 bits with an infinity or a NaN stands for NaN
    want[40 + 24:40 + 64, 5] = True                    # (key 60 of the second request, whose 64 tokens are its rows 36 to 99)
    assert torch.equal(out.isnan().all(-1).cpu(), want) and torch.equal((~torch.isfinite(out)).any(-1).cpu(), want)
    want[:, 3] = False
    assert torch.equal(~torch.isfinite(lse).cpu(), want)


@pytest.mark.parametrize("split", [True, False])
@pytest.mark.parametrize("dtype,kind,Hq,H,d,br,rows,tokens", [x for x in ODD if x[1] != E4M3 and x[4] > 24])
def test_infinities_in_v_that_all_see(dtype, kind, Hq, H, d, br, rows, tokens, split):
    print("case:", dtype, kind, Hq, H, d, br, rows, tokens, split, flush=True)

    def put(k, v):
        first = rows[0] - tokens[0]                    # (keys up to here are seen by every token of request 0)
        for j, e, what in ((0, 3, math.inf), (first, 4, -math.inf), (first // 2, 5, math.nan), (1, 6, math.inf), (first // 3, 6, -math.inf), (first // 4, d - 1, math.inf), (2, d - 1, math.inf)):
            v[j, 0, e] = what
    c = Case(dtype, kind, Hq, H, d, br, rows, tokens, special=put)
    out, lse = c.run(split=split)
    torch.cuda.synchronize()
    got, G = out.cpu()[:tokens[0], :Hq // H], Hq // H
    assert (got[..., 3] == math.inf).all() and (got[..., 4] == -math.inf).all() and got[..., 5].isnan().all() and got[..., 6].isnan().all() and (got[..., d - 1] == math.inf).all()
    odd = torch.zeros(out.shape, dtype=torch.bool)
    odd[:tokens[0], :G, [3, 4, 5, 6, d - 1]] = True
    assert torch.equal(~torch.isfinite(out.cpu()), odd)
    c.v = c.v.nan_to_num(0, 0, 0)                      # and the others have their values
    for tok in range(tokens[0]):
        k, v = (x[:rows[0]].transpose(0, 1).contiguous() for x in (c.k, c.v))
        o, _, _, _ = fp4_plain.attention(c.q[tok], k, v, rows[0] - tokens[0] + tok + 1, 1.0 / math.sqrt(d))
        out[tok] = torch.where(odd[tok], o.to(dtype), out[tok].cpu()).to(DEV)
    c.check(out, lse)
