"""The paged 4-bit cache against its plain form (needs an MI355X): bits of codes and scales, tables and slots, and the
attention to within its roundings."""
import math
import random

import pytest
import torch

import fp4_plain as plain

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def _laq():
    import paper_2505_20334_amd as laq
    return laq


def _pool(n_blocks, H, br, d, token_major=False, fill=0xA5):
    """A cache whose bytes are all `fill`."""
    laq = _laq()
    if not token_major:
        return laq.Fp4Cache(*(torch.full((n_blocks, H, br, w), fill, dtype=torch.uint8, device=DEV) for w in (d // 2, d // 32, d // 2, d // 32)))
    return laq.Fp4Cache(*(torch.full((n_blocks, br, H, w), fill, dtype=torch.uint8, device=DEV).transpose(1, 2) for w in (d // 2, d // 32, d // 2, d // 32)))


def _rows(cache_plane, slots, br):
    """Rows `slots` of a plane, [tokens, H, bytes], on the CPU."""
    p, s = cache_plane.cpu(), slots.cpu().long()
    return p[s // br, :, s % br]


def _special(T, H, d, dtype, gen):
    x = torch.randn(T, H, d, generator=gen) * torch.exp2(torch.randint(-6, 7, (T, H, 1), generator=gen).float())
    flat = x.view(-1, 32)
    for i, block in enumerate(([0.0] * 32, [-0.0] * 32, [3e38] + [1e38] * 31, [-3.3e38] + [2e38] * 31, [math.inf] + [1.0] * 31, [1.0] * 31 + [-math.inf],
                               [math.nan] * 32, [1e-38] * 32, [2.0 ** -102] * 31 + [-2.0 ** -99], [1e-45] * 32, [7.0, 6.0, -5.0, 0.25, -0.25, 0.75] + [3.5] * 26,
                               [1.75, 1.0, -0.3] + [0.0] * 29, [1.7421875] + [-1.0] * 31, [6.0] + [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -5.0] * 3 + [0.1] * 4)):
        if 7 * i + 3 < flat.shape[0]:
            flat[7 * i + 3] = torch.tensor(block)
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,H,d,br,layout,token_major", [
    (1, 1, 32, 16, "dense", False), (3, 2, 64, 16, "dense", True), (50, 3, 96, 48, "fused", False), (257, 8, 128, 64, "dense", False),
    (130, 5, 160, 16, "fused", True), (77, 1, 224, 256, "heads", False), (200, 2, 256, 32, "fused", False), (64, 4, 192, 128, "heads", True)])
def test_stored_rows_have_the_plain_bits_and_come_back(dtype, T, H, d, br, layout, token_major):
    laq = _laq()
    print("case:", dtype, T, H, d, br, layout, token_major, flush=True)
    gen = torch.Generator().manual_seed(T * 7 + d)
    k, v = _special(T, H, d, dtype, gen), _special(T, H, d, dtype, gen).flip(0)
    n_blocks = -(-T // br) + 2
    slots = torch.randperm(n_blocks * br, generator=gen)[:T].int()
    slots[T // 2::5] = -1                             # some tokens without a place, and some beyond the pool
    slots[T // 3::11] = n_blocks * br + 3
    here = (slots >= 0) & (slots < n_blocks * br)
    if layout == "fused":                             # K and V of a token side by side
        kv = torch.stack([k, v], 1).to(DEV)
        kd, vd = kv[:, 0], kv[:, 1]
    elif layout == "heads":                           # [H, T, d]
        kd, vd = (x.transpose(0, 1).contiguous().to(DEV).transpose(0, 1) for x in (k, v))
    else:
        kd, vd = k.to(DEV), v.to(DEV)
    cache = _pool(n_blocks, H, br, d, token_major)
    laq.laq_fp4_store(cache, kd, vd, slots.to(DEV))
    torch.cuda.synchronize()
    untouched = torch.ones(n_blocks * br, dtype=torch.bool)
    untouched[slots[here].long()] = False
    for x, codes, scales in ((k, cache.k, cache.k_scale), (v, cache.v, cache.v_scale)):
        want_c, want_s = plain.quantise(x[here])
        assert torch.equal(_rows(scales, slots[here], br), want_s)
        assert torch.equal(_rows(codes, slots[here], br), want_c)
        for plane in (codes, scales):
            rest = plane.cpu().transpose(1, 2).reshape(n_blocks * br, -1)[untouched]
            assert (rest == 0xA5).all()
    ask = torch.cat([slots, torch.tensor([-1, -(1 << 31), (1 << 31) - 1], dtype=torch.int32)])
    for out_dtype in (BF16, F32):
        got = laq.laq_fp4_load(cache, ask.to(DEV), out_dtype)
        torch.cuda.synchronize()
        for x, y in zip((k, v), got):
            want = torch.zeros(T + 3, H, d, dtype=torch.float64)
            want[:T][here] = plain.values(*plain.quantise(x[here]))
            assert y.dtype == out_dtype and torch.equal(torch.nan_to_num(y.cpu().double(), nan=12345.0), torch.nan_to_num(want, nan=12345.0))
    # one of the two alone
    other = _pool(n_blocks, H, br, d, token_major)
    laq.laq_fp4_store(other, None, vd, slots.to(DEV))
    torch.cuda.synchronize()
    assert torch.equal(other.v.cpu(), cache.v.cpu()) and torch.equal(other.v_scale.cpu(), cache.v_scale.cpu()) and (other.k == 0xA5).all()
    laq.laq_fp4_store(other, kd, None, slots.to(DEV))
    torch.cuda.synchronize()
    assert torch.equal(other.k.cpu(), cache.k.cpu()) and torch.equal(other.k_scale.cpu(), cache.k_scale.cpu())


@pytest.mark.parametrize("dtype,n,H,d,L,budgets,br,layout", [
    (BF16, 1, 8, 128, 600, [64], 16, "dense"), (F32, 2, 2, 64, 300, [300, 1], 64, "dense"), (BF16, 3, 4, 96, 513, [40, 500, 17], 32, "token_major"),
    (BF16, 2, 2, 256, 700, [33, 600], 16, "paged"), (F32, 1, 3, 128, 900, [900], 128, "paged"), (BF16, 300, 1, 32, 20, [1 + i % 20 for i in range(300)], 16, "dense")])
def test_compacted_rows_have_the_bits_of_stored_ones(dtype, n, H, d, L, budgets, br, layout):
    laq = _laq()
    print("case:", dtype, n, H, d, L, br, layout, flush=True)
    gen = torch.Generator().manual_seed(L + d)
    k, v = (torch.randn(n, H, L, d, generator=gen).to(dtype) for _ in range(2))
    idx = torch.cat([torch.rand(H, L, generator=gen).topk(b, -1).indices.sort(-1).values.int().flatten() for b in budgets])
    total = sum(budgets)
    n_blocks = -(-total // br) + 1
    slots = torch.randperm(n_blocks * br, generator=gen)[:total].int()
    slots[5::97] = -1
    kw = {}
    if layout == "paged":
        per = -(-L // 256)
        table = torch.randperm(n * per, generator=gen).view(n, per).int()
        kd, vd = (torch.zeros(n * per, H, 256, d, dtype=dtype) for _ in range(2))
        for x, y in ((k, kd), (v, vd)):
            y[table.long()] = torch.nn.functional.pad(x, (0, 0, 0, per * 256 - L)).view(n, H, per, 256, d).transpose(1, 2)
        kw = dict(block_table=table.to(DEV), L=L)
        kd, vd = kd.to(DEV), vd.to(DEV)
    elif layout == "token_major":
        kd, vd = (x.transpose(1, 2).contiguous().to(DEV).transpose(1, 2) for x in (k, v))
    else:
        kd, vd = k.to(DEV), v.to(DEV)
    cache = _pool(n_blocks, H, br, d)
    laq.laq_fp4_compact(cache, kd, vd, idx.to(DEV), budgets, slots.to(DEV), **kw)
    torch.cuda.synchronize()
    at = 0
    for x, codes, scales in ((k, cache.k, cache.k_scale), (v, cache.v, cache.v_scale)):
        rows, at = [], 0
        for i, b in enumerate(budgets):
            take = idx[at:at + H * b].view(H, b).long()
            at += H * b
            rows.append(torch.stack([x[i, h, take[h]] for h in range(H)], 1))
        want_c, want_s = plain.quantise(torch.cat(rows))
        here = slots >= 0
        assert torch.equal(_rows(codes, slots[here], br), want_c[here]) and torch.equal(_rows(scales, slots[here], br), want_s[here])
    empty = torch.ones(n_blocks * br, dtype=torch.bool)
    empty[slots[slots >= 0].long()] = False
    assert (cache.v.cpu().transpose(1, 2).reshape(n_blocks * br, -1)[empty] == 0xA5).all()
    only_k = _pool(n_blocks, H, br, d)
    laq.laq_fp4_compact(only_k, kd, None, idx.to(DEV), budgets, slots.to(DEV), **kw)
    torch.cuda.synchronize()
    assert torch.equal(only_k.k.cpu(), cache.k.cpu()) and (only_k.v == 0xA5).all()


def test_an_index_outside_of_the_cache_is_left_out():
    laq = _laq()
    k = torch.randn(1, 2, 40, 64, device=DEV)
    cache, slots = _pool(2, 2, 16, 64), torch.arange(3, dtype=torch.int32, device=DEV)
    laq.laq_fp4_compact(cache, k, k, torch.tensor([3, 40, 5, -1, 7, 39], dtype=torch.int32, device=DEV), [3], slots)
    torch.cuda.synchronize()
    got = cache.k.cpu()[0, :, :3]
    assert torch.equal(got[0, 0], plain.quantise(k[0, 0, 3].cpu())[0]) and torch.equal(got[1, 2], plain.quantise(k[0, 1, 39].cpu())[0])
    assert (got[0, 1] == 0xA5).all() and (got[1, 0] == 0xA5).all()


class Mapped:
    """laq_block_map beside the plain allocator."""

    def __init__(self, n, n_blocks, width, br, seed):
        laq = _laq()
        order = torch.randperm(n_blocks, generator=torch.Generator().manual_seed(seed))
        self.want = plain.Allocator(n, n_blocks, width, br, order.tolist())
        self.rows = torch.zeros(n, dtype=torch.int32, device=DEV)
        self.table = torch.full((n, width), -1, dtype=torch.int32, device=DEV)
        self.free, self.state = laq.laq_block_pool(n_blocks, DEV)
        self.free.copy_(order)
        self.br = br

    def step(self, add, n_slots):
        start, slots = _laq().laq_block_map(torch.tensor(add, dtype=torch.int32, device=DEV), self.rows, self.table, self.free, self.state, self.br, n_slots=n_slots)
        torch.cuda.synchronize()
        want_start, want_slots = self.want.step(add, n_slots)
        w = self.want
        assert self.state.tolist() == [len(w.free), w.refused, 0, 0]
        assert self.rows.tolist() == w.rows
        assert self.table.tolist() == w.table
        assert self.free[:len(w.free)].tolist() == w.free
        assert start.tolist() == want_start and slots.tolist() == want_slots
        return start, slots


@pytest.mark.parametrize("n,n_blocks,width,br,most,seed", [
    (1, 4, 4, 16, 40, 1), (3, 1, 2, 16, 20, 2), (7, 200, 30, 32, 300, 3), (64, 500, 12, 16, 60, 4), (64, 9000, 80, 256, 2000, 5), (300, 2500, 20, 48, 200, 6),
    (1024, 3000, 6, 16, 40, 7), (1025, 3000, 6, 16, 40, 8), (2600, 9000, 9, 16, 30, 9)])
def test_block_maps_step_by_step(n, n_blocks, width, br, most, seed):
    print("case:", n, n_blocks, width, br, most, flush=True)
    rng = random.Random(seed)
    m = Mapped(n, n_blocks, width, br, seed)
    for step in range(8):
        kind = step % 4
        if kind == 0:                                 # appended to most requests, in plenty
            add = [rng.choice([0, 1, br, rng.randint(1, most)]) for _ in range(n)]
        elif kind == 1:                               # a token each; some dropped
            add = [rng.choice([1, 1, 1, 0, -rng.randint(1, most)]) for _ in range(n)]
        elif kind == 2:                               # both ways at once, more than there is for some
            add = [rng.choice([-(1 << 31), -most // 2, most, 3, width * br + 1, 0x7fffffff if i == n // 2 else 0]) for i in range(n)]
        else:
            add = [-rng.randint(0, 2 * most) for _ in range(n)]
        appended = sum(max(a, 0) for a in add)
        if appended > 1 << 20:                        # (a plain list of all slots would be long)
            add = [min(a, width * br + 1) for a in add]
            appended = sum(max(a, 0) for a in add)
        m.step(add, rng.choice([appended, appended + 37, appended // 2, 0]))


def test_dropping_what_was_appended_restores_the_list():
    m = Mapped(40, 3000, 200, 16, 3)
    m.step([16 * i + 5 for i in range(40)], 15000)
    before = m.free.clone(), m.state.clone()
    add = [(i * 37) % 200 for i in range(40)]
    m.step(add, sum(add))
    m.step([-a for a in add], 0)
    assert torch.equal(m.free, before[0]) and torch.equal(m.state, before[1])


def test_a_map_of_lengths_and_lists_that_make_no_sense_stays_in_bounds():
    laq = _laq()
    rows = torch.tensor([-5, 1 << 30, 33, 0], dtype=torch.int32, device=DEV)
    table = torch.full((4 + 2, 4), -7, dtype=torch.int32, device=DEV)
    table[2, :3] = torch.tensor([1 << 30, -4, 99999])
    free = torch.full((10,), 1 << 28, dtype=torch.int32, device=DEV)
    state = torch.tensor([1 << 30, 0, 0, 0], dtype=torch.int32, device=DEV)
    add = torch.tensor([16, -64, 20, 5], dtype=torch.int32, device=DEV)
    start, slots = laq.laq_block_map(add, rows, table[:4], free[:6], state, 16, n_slots=50)
    torch.cuda.synchronize()
    assert rows.tolist() == [16, 0, 53, 5] and start.tolist() == [0, 16, 16, 36, 41]
    assert (slots == -1).all()                        # no block that was taken is one of the pool
    assert (table[4:] == -7).all() and (free[6:] == 1 << 28).all()
    # a start longer than an int: it stays at the largest
    big = torch.full((3,), 0x7fffffff, dtype=torch.int32, device=DEV)
    start, slots = laq.laq_block_map(big, rows[:3], table[:3], free[:6], state, 16, n_slots=4)
    torch.cuda.synchronize()
    assert start.tolist() == [0, 0x7fffffff, 0x7fffffff, 0x7fffffff] and (slots == -1).all() and state[1].item() == 3


# ---- attention -----------------------------------------------------------------------------

class Case:
    """A batch with its cache on the CPU (64 bits) and on the GPU."""

    def __init__(self, dtype, Hq, H, d, br, rows, tokens, seed=0, holes=(), token_major=False, fused=False, pad=0, spare=0, peak=1.0, stale=0xFF):
        laq = _laq()
        gen = torch.Generator().manual_seed(seed + d + sum(rows))
        n = len(rows)
        need = [-(-r // br) for r in rows]
        n_blocks = sum(need) + 2
        order = torch.randperm(n_blocks, generator=gen).tolist()
        per = max(1, max(need)) + spare
        # what no row lies in holds scales of 255, which stand for NaN: rows behind a request's last one, other blocks
        cache = _pool(n_blocks, H, br, d, token_major, stale)
        table = torch.full((n, per), -1, dtype=torch.int32)
        slots = []
        for i, r in enumerate(rows):
            table[i, :need[i]] = torch.tensor([order.pop() for _ in range(need[i])], dtype=torch.int32)
            slots += [int(table[i, j // br]) * br + j % br for j in range(r)]
        T = sum(rows)
        channel = torch.where(torch.rand(H, d, generator=gen) < 0.1, 4.0, 1.0)
        self.k, self.v = torch.randn(T, H, d, generator=gen) * channel, torch.randn(T, H, d, generator=gen)
        if T:
            laq.laq_fp4_store(cache, self.k.to(DEV), self.v.to(DEV), torch.tensor(slots, dtype=torch.int32, device=DEV))
        self.kq, self.vq = (plain.values(*plain.quantise(x)) for x in (self.k, self.v))
        self.hidden = [set() for _ in range(n)]       # rows of blocks that are none of the pool
        for i, b, number in holes:
            table[i, b] = number
            self.hidden[i] |= set(range(b * br, (b + 1) * br))
        self.start = torch.tensor([0] + list(tokens), dtype=torch.int32).cumsum(0).int()
        count = int(self.start[-1])
        q = (torch.randn(count + pad, Hq, d, generator=gen) * peak).to(dtype)
        self.q = q.double()
        if fused:                                     # q of a fused projection
            wide = torch.zeros(count + pad, Hq + 2 * H, d, dtype=dtype)
            wide[:, :Hq] = q
            self.qd = wide.to(DEV)[:, :Hq]
        else:
            self.qd = q.to(DEV)
        self.dtype, self.Hq, self.H, self.d, self.rows, self.tokens, self.pad = dtype, Hq, H, d, rows, tokens, pad
        self.cache, self.table, self.rows_d = cache, table.to(DEV), torch.tensor(rows, dtype=torch.int32, device=DEV)
        self.start_d = None if all(t == 1 for t in tokens) and not pad else self.start.to(DEV)

    def run(self, **kw):
        kw.setdefault("max_rows", max(1, max(self.rows)))
        return _laq().laq_fp4_attention(self.qd, self.cache, self.table, self.rows_d, start=self.start_d, want_lse=True, **kw)

    def check(self, out, lse, scale=None, what=""):
        """Element by element.  With u = 2^-24 (fp32) and A the largest sum of |q k| * scale of a token: a logit is off by at most (d + 4) u A (sums of d
        products in any order, the scale), the maximum's own rounding and the exponential's argument by 2 u A more, the exponential by 2^-22; three
        parts of q leave out 2^-24 of each product.  A weight p is therefore off by e = 2 u (d + 16) A + 2^-22 of it, a sum of L weights in any order by L u more (the parts
        of a cut one by a few), in numerator and denominator.  bf16: every weight in the numerator is rounded, 2^-8 of it at most, and the result, 2^-8."""
        scale = scale or 1.0 / math.sqrt(self.d)
        u, half = 2.0 ** -24, 2.0 ** -8 if self.dtype == BF16 else 2.0 ** -24
        out, lse = out.cpu().double(), lse.cpu().double()
        first = 0
        for i, r in enumerate(self.rows):
            keep = [j for j in range(r) if j not in self.hidden[i]]
            k, v = (x[first:first + r][keep].transpose(0, 1).contiguous() for x in (self.kq, self.vq))
            first += r
            for t in range(self.tokens[i]):
                tok = int(self.start[i]) + t
                seen = sum(1 for j in keep if j <= r - self.tokens[i] + t)
                o, l, a, A = plain.attention(self.q[tok], k, v, seen, scale)
                where = "%s request %d token %d" % (what, i, t)
                if seen == 0:
                    assert (out[tok] == 0).all() and (lse[tok] == -math.inf).all(), where
                    continue
                e = (2 * u * (self.d + 16) * A + 2.0 ** -22 + (seen + 64) * u)[:, None]
                tol = (2 * e + half) * a + half * o.abs() + 1e-30
                bad = (out[tok] - o).abs() > tol
                assert not bad.any(), "%s: %d of %d outputs off, by up to %.3g of the bound" % (where, int(bad.sum()), bad.numel(), float(((out[tok] - o).abs() / tol).max()))
                assert ((lse[tok] - l).abs() <= 2 * e[:, 0] + 4 * u * l.abs()).all(), where
        assert first == sum(self.rows)


ONE = [  # one token per request: (dtype, Hq, H, d, block, lengths)
    (BF16, 4, 4, 32, 16, [1]), (BF16, 32, 8, 128, 64, [520]), (BF16, 8, 8, 64, 16, [1, 2, 15, 16, 17, 31, 33, 64, 65]), (BF16, 28, 4, 96, 48, [127, 128, 129, 700]),
    (BF16, 8, 1, 128, 256, [1000, 3]), (BF16, 16, 1, 160, 32, [95, 0, 300]), (BF16, 17, 1, 128, 16, [70]), (BF16, 40, 1, 64, 64, [200, 1]), (BF16, 71, 1, 64, 128, [333]),
    (BF16, 6, 2, 192, 16, [257, 255]), (BF16, 3, 3, 224, 80, [161]), (BF16, 8, 2, 256, 64, [63, 1000]), (BF16, 2, 1, 128, 128, [5000, 17, 1025]),
    (BF16, 8, 8, 128, 16, [300 + 13 * i for i in range(40)]),
    # shared out: columns that end and begin within a share, one request of most rows, many shares of a column, requests of no rows in between
    (BF16, 32, 8, 64, 64, [4100, 1, 0, 700, 4096, 33, 0, 2000] * 2), (BF16, 8, 8, 128, 16, [9000] + [5] * 130), (BF16, 16, 16, 96, 16, [6000, 5990, 257, 513] * 2),
    (F32, 16, 8, 64, 32, [5000, 0, 300, 4999] * 4), (BF16, 40, 8, 256, 64, [4000, 70, 2900, 1] * 2),
    (F32, 4, 4, 32, 16, [3, 40]), (F32, 28, 4, 96, 16, [700, 1]), (F32, 32, 8, 128, 64, [130, 513]), (F32, 17, 1, 64, 32, [99]), (F32, 2, 2, 256, 48, [150, 31]),
    (F32, 8, 2, 192, 16, [64, 65]), (F32, 3, 1, 160, 16, [17]), (F32, 1, 1, 128, 256, [3000]), (F32, 9, 3, 224, 16, [77]),
]


@pytest.mark.parametrize("dtype,Hq,H,d,br,rows", ONE)
def test_one_token_per_request(dtype, Hq, H, d, br, rows):
    print("case:", dtype, Hq, H, d, br, rows, flush=True)
    c = Case(dtype, Hq, H, d, br, rows, [1] * len(rows), token_major=d % 64 == 0 and br == 64, fused=br == 48)
    for split in (True, False):
        out, lse = c.run(split=split)
        torch.cuda.synchronize()
        c.check(out, lse, what="split %s" % split)


MANY = [  # (dtype, Hq, H, d, block, lengths, tokens)
    (BF16, 8, 2, 128, 64, [100, 33, 8], [8, 3, 8]), (BF16, 4, 4, 64, 16, [300], [17]), (BF16, 8, 1, 96, 32, [65, 200, 1], [0, 40, 1]),
    (BF16, 28, 4, 128, 128, [513, 20], [9, 20]), (BF16, 32, 8, 128, 16, [400, 90], [130, 1]), (BF16, 2, 2, 256, 64, [150, 70], [70, 70]),
    (BF16, 5, 1, 160, 16, [100], [50]), (BF16, 16, 4, 64, 64, [1500, 5], [3, 5]), (BF16, 6, 3, 32, 16, [90, 40], [90, 40]),
    (F32, 8, 2, 128, 64, [100, 33, 8], [8, 3, 8]), (F32, 28, 4, 96, 16, [300, 64], [8, 7]), (F32, 4, 2, 256, 32, [90], [40]), (F32, 3, 3, 192, 16, [60], [33]),
    (F32, 2, 1, 64, 16, [250, 30], [100, 30]),
    # tiles of 48 score rows (as many of them as two workgroups a compute unit), the last ones short
    (BF16, 64, 16, 128, 16, [300, 110, 200, 97], [100, 110, 93, 97]), (BF16, 28, 14, 96, 64, [260, 400], [250, 131]), (BF16, 56, 8, 128, 48, [130, 90], [95, 90]),
]


@pytest.mark.parametrize("dtype,Hq,H,d,br,rows,tokens", MANY)
def test_several_tokens_see_up_to_their_own_row(dtype, Hq, H, d, br, rows, tokens):
    print("case:", dtype, Hq, H, d, br, rows, tokens, flush=True)
    c = Case(dtype, Hq, H, d, br, rows, tokens, fused=d == 128, pad=3)
    for split in (True, False):
        out = torch.full((c.qd.shape[0], Hq, d), 77.0, dtype=dtype, device=DEV)
        lse = torch.full((c.qd.shape[0], Hq), 77.0, device=DEV)
        c.run(split=split, out=out, lse=lse)
        torch.cuda.synchronize()
        c.check(out, lse, what="split %s" % split)
        assert (out[-3:] == 77.0).all() and (lse[-3:] == 77.0).all()            # the padding, left as it was


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_that_are_not_there(dtype):
    # requests of no rows, tokens in front of the first row, blocks that are none of the pool at the start, in between and at the end, all blocks missing
    rows, tokens = [0, 3, 100, 100, 70, 40], [2, 7, 3, 1, 70, 5]
    holes = [(2, 0, -1), (3, 1, 1 << 30), (3, 6, -5), (4, 2, 10 ** 6), (5, 0, -1), (5, 1, -(1 << 31)), (5, 2, -1)]
    c = Case(dtype, 8, 2, 128, 16, rows, tokens, holes=holes, spare=2)
    for split in (True, False):
        out, lse = c.run(split=split)
        torch.cuda.synchronize()
        c.check(out, lse, what="split %s" % split)


@pytest.mark.parametrize("dtype,tokens", [(BF16, 1), (F32, 1), (BF16, 40)])
def test_lengths_beyond_the_bound_and_beyond_the_table(dtype, tokens):
    # rows beyond max_rows count; rows beyond what the table holds do not
    c = Case(dtype, 8, 2, 64, 16, [1000, 64], [tokens, min(tokens, 30)])
    for most in (1, 64, 100, 999):
        out, lse = c.run(max_rows=most)
        torch.cuda.synchronize()
        c.check(out, lse, what="max_rows %d" % most)
    full = Case(dtype, 8, 2, 64, 16, [1008, 64], [tokens, min(tokens, 30)])
    full.rows_d[0] = 1 << 30                          # of 63 blocks
    out, lse = full.run(max_rows=1008)
    torch.cuda.synchronize()
    full.check(out, lse)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_large_logits_scales_and_a_dominant_row(dtype):
    # logits of several hundred, of one row alone, scales given
    c = Case(dtype, 8, 2, 128, 32, [500, 90], [1, 6], peak=30.0)
    for scale in (0.0, 0.5, 1e-3):
        out, lse = c.run(scale=scale)
        torch.cuda.synchronize()
        c.check(out, lse, scale=scale or None, what="scale %g" % scale)


@pytest.mark.parametrize("tokens,Hq,H,d", [(1, 4, 2, 64), (5, 4, 2, 64), (30, 4, 2, 64), (30, 8, 2, 160), (50, 128, 32, 128), (3, 4, 2, 256)])
def test_a_nan_in_the_cache_reaches_those_that_see_it(tokens, Hq, H, d):
    laq = _laq()
    print("case:", tokens, Hq, H, d, flush=True)
    c = Case(BF16, Hq, H, d, 16, [50, 60], [tokens, tokens])
    last, G = H - 1, Hq // H                             # the head that gets it, its queries
    nan_row = 59 if tokens == 1 else 60 - tokens // 2 - 1      # of request 1: the last row, or one that the first tokens do not see
    slot = int(c.table[1, nan_row // 16]) * 16 + nan_row % 16
    bad = torch.zeros(1, H, d, device=DEV)
    bad[0, last, 5] = math.inf
    laq.laq_fp4_store(c.cache, None, bad, torch.tensor([slot], dtype=torch.int32, device=DEV))
    out, lse = c.run()
    torch.cuda.synchronize()
    out = out.cpu().view(2, tokens, Hq, d)
    sees = torch.arange(tokens) + 60 - tokens >= nan_row
    assert sees.any() and (tokens == 1 or not sees.all())
    assert torch.isfinite(out[0]).all() and torch.isfinite(out[1, ~sees]).all() and torch.isfinite(out[1, sees][:, :last * G]).all()
    assert torch.isnan(out[1, sees][:, last * G:, :32]).all() and torch.isfinite(out[1, sees][:, last * G:, 32:]).all() and torch.isfinite(lse).all()
    # in K: the logit, and with it everything of the head
    laq.laq_fp4_store(c.cache, bad, torch.ones_like(bad), torch.tensor([slot], dtype=torch.int32, device=DEV))
    out, lse = c.run()
    torch.cuda.synchronize()
    out = out.cpu().view(2, tokens, Hq, d)
    assert torch.isnan(out[1, sees][:, last * G:]).all() and torch.isfinite(out[1, sees][:, :last * G]).all() and torch.isfinite(out[1, ~sees]).all()


def test_infinite_and_nan_queries_stay_with_their_own_head():
    c = Case(BF16, 8, 2, 128, 16, [100, 40], [3, 1])
    want = c.run()[0].cpu()
    q = c.qd.clone()
    q[1, 2, 5] = math.nan
    q[3, 7, 9] = math.inf
    c.qd = q
    got = c.run()[0].cpu()
    same = torch.ones(4, 8, dtype=torch.bool)
    same[1, 2] = same[3, 7] = False
    assert torch.equal(got[same], want[same]) and torch.isnan(got[1, 2]).all()


@pytest.mark.parametrize("dtype,tokens,rows", [(BF16, [1] * 3, [3000, 17, 900]), (BF16, [40, 3, 1], [700, 30, 64]), (F32, [2, 2, 8], [2000, 50, 8])])
def test_replays_give_the_bits_of_eager_calls(dtype, tokens, rows):
    c = Case(dtype, 8, 2, 128, 64, rows, tokens)
    out, lse = torch.empty_like(c.qd), torch.empty(c.qd.shape[0], 8, device=DEV)
    laq = _laq()
    need = laq.laq_fp4_attention_workspace_bytes(c.cache, 8, dtype, 3, c.qd.shape[0], max(rows))
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    c.run(ws=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(out=out, lse=lse, ws=ws)
    for replay in range(5):
        c.qd.normal_()
        c.rows_d[0] = rows[0] - 7 * replay               # lengths change between replays
        ws.random_(0, 256)                               # and nothing is left in the workspace
        want = c.run()
        out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]), "replay %d" % replay


def test_another_stream_and_the_same_bits_twice():
    c = Case(BF16, 16, 4, 128, 32, [2500, 300], [1, 1])
    want = c.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = c.run()
    b = c.run(stream=side)
    torch.cuda.synchronize()
    for x in (a, b):
        assert torch.equal(x[0], want[0]) and torch.equal(x[1], want[1])


def test_offsets_beyond_32_bits():
    # a pool of more than 4 GiB of codes: block numbers near its end
    laq = _laq()
    H, br, d = 8, 256, 256
    per_block = H * br * d // 2
    n_blocks = (1 << 32) // per_block + 40
    codes = [torch.empty(n_blocks, H, br, w, dtype=torch.uint8, device=DEV) for w in (d // 2, d // 32, d // 2, d // 32)]
    for t in codes:
        t[-8:] = 0
    cache = laq.Fp4Cache(*codes)
    gen = torch.Generator().manual_seed(1)
    k, v = (torch.randn(700, H, d, generator=gen) for _ in range(2))
    table = torch.tensor([[n_blocks - 1, n_blocks - 5, n_blocks - 3]], dtype=torch.int32)
    slots = torch.tensor([int(table[0, j // br]) * br + j % br for j in range(700)], dtype=torch.int32, device=DEV)
    laq.laq_fp4_store(cache, k.to(DEV), v.to(DEV), slots)
    got = laq.laq_fp4_load(cache, slots, F32)
    c = Case(BF16, 8, H, d, br, [700], [1])
    c.kq, c.vq = plain.values(*plain.quantise(k)), plain.values(*plain.quantise(v))
    c.cache, c.table = cache, table.to(DEV)
    out, lse = c.run()
    torch.cuda.synchronize()
    assert torch.equal(got[0].cpu().double(), c.kq) and torch.equal(got[1].cpu().double(), c.vq)
    c.check(out, lse)


# ---- together ------------------------------------------------------------------------------

def test_evict_into_the_cache_and_decode_on_it():
    """The method's steps on the 4-bit cache: eviction of a prefill cache, its rows into blocks, tokens appended and attended to in a captured loop,
    lookahead tokens dropped, rows read back for another eviction."""
    laq = _laq()
    gen = torch.Generator().manual_seed(11)
    n, Hq, H, L, d, W, br = 3, 8, 2, 700, 128, 8, 16
    budgets = [200, 90, 64]
    q = (torch.randn(n, Hq, W, d, generator=gen) * 1.5).bfloat16().to(DEV)
    k, v = (torch.randn(n, H, L, d, generator=gen).bfloat16().to(DEV) for _ in range(2))
    scores, idx, k1, v1 = laq.laq_evict(q, k, v, budgets, 7)
    # the same rows into blocks
    n_blocks = 60
    cache = laq.laq_fp4_cache(n_blocks, H, br, d, DEV)
    free, state = laq.laq_block_pool(n_blocks, DEV)
    rows, table = torch.zeros(n, dtype=torch.int32, device=DEV), torch.full((n, 20), -1, dtype=torch.int32, device=DEV)
    start, slots = laq.laq_block_map(torch.tensor(budgets, dtype=torch.int32, device=DEV), rows, table, free, state, br, n_slots=sum(budgets))
    laq.laq_fp4_compact(cache, k, v, idx, budgets, slots)
    kl, vl = laq.laq_fp4_load(cache, slots)
    first = 0
    held = []
    for i, b in enumerate(budgets):
        packed = laq.packed_rows(budgets, H, L)[1][i]
        got = kl[first:first + b].transpose(0, 1).reshape(-1, d).cpu().double()
        assert torch.equal(got, plain.values(*plain.quantise(k1[packed:packed + H * b].cpu())))
        held.append([x[first:first + b].cpu().double() for x in (kl, vl)])
        first += b
    # a captured decoding step: one row appended to each request and attended to
    one = torch.ones(n, dtype=torch.int32, device=DEV)
    qt, kt, vt = (torch.zeros(n, h, d, dtype=BF16, device=DEV) for h in (Hq, H, H))
    out, step_slots = torch.zeros(n, Hq, d, dtype=BF16, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV)
    need = laq.laq_fp4_attention_workspace_bytes(cache, Hq, BF16, n, n, 320)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    saved = [t.clone() for t in (rows, table, free, state)]

    def step():
        laq.laq_block_map(one, rows, table, free, state, br, slots=step_slots)
        laq.laq_fp4_store(cache, kt, vt, step_slots)
        laq.laq_fp4_attention(qt, cache, table, rows, max_rows=320, out=out, ws=ws)

    step()
    for t, s in zip((rows, table, free, state), saved):
        t.copy_(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t in range(20):
        for x in (qt, kt, vt):
            x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        for i in range(n):
            for x, new in zip((0, 1), (kt, vt)):
                held[i][x] = torch.cat([held[i][x], plain.values(*plain.quantise(new[i:i + 1].cpu()))])
            kk, vv = (x.transpose(0, 1).contiguous() for x in held[i])
            want, _, a, _ = plain.attention(qt[i].cpu().double(), kk, vv, kk.shape[1], 1 / math.sqrt(d))
            # (the bound of Case.check with its fp32 part, under 2^-12 here, in full)
            assert ((out[i].cpu().double() - want).abs() <= (2.0 ** -8 + 2.0 ** -12) * a + 2.0 ** -8 * want.abs()).all(), (t, i)
    assert rows.tolist() == [b + 20 for b in budgets] and state[1].item() == 0
    # lookahead tokens of the last 8 steps are dropped; the kept rows of request 0 are read back and evicted once more
    left = state[0].item()
    laq.laq_block_map(torch.full((n,), -8, dtype=torch.int32, device=DEV), rows, table, free, state, br)
    torch.cuda.synchronize()
    assert rows.tolist() == [b + 12 for b in budgets] and state[0].item() >= left
    r = 212
    j = torch.arange(r, device=DEV)
    again, again_v = laq.laq_fp4_load(cache, (table[0].long()[j // br] * br + j % br).int())
    assert torch.equal(again.cpu().double(), held[0][0][:r]) and torch.equal(again_v.cpu().double(), held[0][1][:r])
    kv = again[None].transpose(1, 2), again_v[None].transpose(1, 2)          # a token-major view, as laq_evict reads it
    got = laq.laq_evict(q[:1], *kv, [50], 7)
    want = laq.laq_evict(q[:1], kv[0].contiguous(), kv[1].contiguous(), [50], 7)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))


# ---- calls that the documentation allows ---------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F32])
def test_more_requests_than_are_shared_out(dtype):
    rows = [(i * 37) % 50 for i in range(1100)]
    c = Case(dtype, 2, 1, 32, 16, rows, [1] * 1100)
    for most in (50, 65536):                          # (as long as a bound may make it: spread over workgroups, if that is worth it)
        c.table = torch.nn.functional.pad(c.table, (0, 4096 - c.table.shape[1]), value=-1)
        out, lse = c.run(max_rows=most)
        torch.cuda.synchronize()
        c.check(out, lse, what="max_rows %d" % most)


def test_turns_that_may_be_more_than_an_int_holds():
    # a table of 2^31 rows, nearly, a request, three requests of 128 heads: 2^23 turns of 256 rows for each of 384 columns
    c = Case(BF16, 128, 128, 32, 65536, [300, 40, 0], [1, 1, 1], spare=32766)
    out, lse = c.run(max_rows=8192)
    torch.cuda.synchronize()
    c.check(out, lse)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_start_that_makes_no_sense_stays_in_bounds(dtype):
    c = Case(dtype, 8, 2, 64, 16, [100, 50, 70], [20, 5, 30])
    T, big = 55, (1 << 31) - 1
    for start in ([7, 20, 25, 55], [0, 40, 10, 55], [-5, 20, 25, 1000], [big, big, big, big], [0, 0, 0, 0], [-big, big, -big, big]):
        bounds = torch.full((T + 60, 8, 64), 5.0, dtype=dtype, device=DEV)
        lse = torch.full((T + 60, 8), 5.0, device=DEV)
        c.start_d = torch.tensor(start, dtype=torch.int32, device=DEV)
        for split in (True, False):
            c.run(out=bounds[30:30 + T], lse=lse[30:30 + T], split=split)
            torch.cuda.synchronize()
            for x in (bounds, lse):
                assert (x[:30] == 5.0).all() and (x[30 + T:] == 5.0).all(), start
    assert (bounds[30:30 + T] != 5.0).any()           # (the last one: request 0 has all tokens, or what is left of it)


def test_graphs_that_share_a_workspace():
    # calls of both kinds, captured with one workspace, replayed in any order among eager calls
    cases = [Case(BF16, 8, 2, 128, 64, [3000, 17, 900], [1, 1, 1]), Case(BF16, 8, 8, 64, 16, [5000, 4100] * 8, [1] * 16, seed=3), Case(F32, 8, 2, 64, 32, [2000, 50], [2, 9], seed=5)]
    laq = _laq()
    need = [laq.laq_fp4_attention_workspace_bytes(c.cache, 8, c.dtype, len(c.rows), c.qd.shape[0], max(c.rows)) for c in cases]
    assert all(need)
    ws = torch.zeros(max(need), dtype=torch.uint8, device=DEV)
    graphs, outs = [], []
    for c in cases:
        c.run(ws=ws)
        outs.append((torch.empty_like(c.qd), torch.empty(c.qd.shape[0], 8, device=DEV)))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.run(out=outs[-1][0], lse=outs[-1][1], ws=ws)
        graphs.append(graph)
    for round_, order in enumerate(((0, 1, 2), (2, 2, 1, 0, 1), (1, 0, 0, 2), (0, 2, 1))):
        for c in cases:
            c.qd.normal_()
        want = [c.run() for c in cases]
        for i in order:
            outs[i][0].fill_(3.0)
            graphs[i].replay()
            if round_ % 2:
                cases[(i + 1) % 3].run(ws=ws)
        torch.cuda.synchronize()
        for i, (w, o) in enumerate(zip(want, outs)):
            assert torch.equal(o[0], w[0]) and torch.equal(o[1], w[1]), (round_, i)


def test_two_streams_with_a_workspace_each():
    # calls that are cut, under way at the same time on the same cache
    cases = [Case(BF16, 8, 2, 128, 64, [30000], [1]), Case(BF16, 8, 8, 64, 16, [5000, 4100] * 8, [1] * 16, seed=3)]
    want = [c.run() for c in cases]
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in cases]
    got = [[], []]
    for _ in range(6):
        for i, c in enumerate(cases):
            with torch.cuda.stream(sides[i]):
                got[i].append(c.run())
    torch.cuda.synchronize()
    for i, w in enumerate(want):
        for g in got[i]:
            assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])


def test_batches_without_tokens():
    laq = _laq()
    c = Case(BF16, 8, 2, 64, 16, [20, 5], [0, 0], pad=1)
    nothing = torch.empty(0, 2, 64, dtype=BF16, device=DEV)
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    before = [t.clone() for t in c.cache]
    laq.laq_fp4_store(c.cache, nothing, nothing, none)
    assert [t.shape for t in laq.laq_fp4_load(c.cache, none)] == [(0, 2, 64)] * 2
    out, lse = laq.laq_fp4_attention(c.qd[:0], c.cache, c.table, c.rows_d, start=c.start_d, want_lse=True)
    assert out.shape == (0, 8, 64) and lse.shape == (0, 8)
    out = torch.full((1, 8, 64), 7.0, dtype=BF16, device=DEV)           # padding alone
    c.run(out=out)
    torch.cuda.synchronize()
    assert (out == 7.0).all() and all(torch.equal(x, y) for x, y in zip(before, c.cache))


def test_the_calls_without_the_compiled_binding(monkeypatch):
    from paper_2505_20334_amd import binding
    laq = _laq()
    c = Case(BF16, 8, 2, 64, 16, [600, 50], [2, 3], fused=True)
    idx = torch.arange(2 * 30, dtype=torch.int32, device=DEV) % 30
    n_slots = torch.tensor([20, 5], dtype=torch.int32, device=DEV)

    def calls():
        cache, (free, state) = laq.laq_fp4_cache(40, 2, 16, 64, DEV), laq.laq_block_pool(40, DEV)
        rows, table = torch.zeros(2, dtype=torch.int32, device=DEV), torch.full((2, 20), -1, dtype=torch.int32, device=DEV)
        start, slots = laq.laq_block_map(n_slots, rows, table, free, state, 16, n_slots=30)
        x = torch.linspace(-3, 3, 30 * 2 * 64, device=DEV).view(30, 2, 64)
        laq.laq_fp4_store(cache, x, x.neg(), slots)
        other = laq.laq_fp4_cache(40, 2, 16, 64, DEV)
        laq.laq_fp4_compact(other, x.transpose(0, 1)[None], None, idx, [30], slots)
        return [*cache, *other, *laq.laq_fp4_load(cache, slots, F32), rows, table[0, :2], table[1, :1], free[:37], state, start, slots, *c.run()]

    with_it = calls()
    binding.load_library()
    monkeypatch.setattr(binding, "_native", None)
    without = calls()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(with_it, without))


def test_one_table_row_of_a_request_shared_by_two():
    # two requests on the same blocks (a common prompt): both read them
    c = Case(BF16, 8, 2, 128, 16, [200, 200], [1, 1])
    c.table[1] = c.table[0]
    q = c.qd.clone()
    q[1] = q[0]
    c.qd = q
    out, lse = c.run()
    torch.cuda.synchronize()
    assert torch.equal(out[0], out[1]) and torch.equal(lse[0], lse[1])


# More ranges of a column than the fold has room for the marks of (288 of 16 rows with d >= 128, 160 with d = 64, 96 with d = 32): (dtype, Hq, H, d, lengths,
# tokens).  Shared out: a turn of 256 rows (128 with d > 128) each, 768 shares.  Parts: the last two.
MANY_RANGES = [(BF16, 16, 1, 64, [100000] + [100] * 40, 1), (BF16, 16, 1, 128, [100] * 9 + [131072] + [100] * 9, 1), (BF16, 16, 1, 256, [70000] + [1] * 31, 1),
               (F32, 16, 1, 64, [100000] + [100] * 40, 1), (BF16, 16, 1, 32, [200000], 1), (BF16, 32, 4, 64, [262144], 4)]


@pytest.mark.parametrize("dtype,Hq,H,d,rows,tokens", MANY_RANGES)
def test_more_ranges_than_are_folded_at_once(dtype, Hq, H, d, rows, tokens):
    print("case:", dtype, Hq, H, d, len(rows), max(rows), tokens, flush=True)
    laq = _laq()
    n = len(rows)
    c = Case(dtype, Hq, H, d, 64, rows, [tokens] * n)
    need = laq.laq_fp4_attention_workspace_bytes(c.cache, Hq, dtype, n, n * tokens, max(rows))
    ws = torch.zeros(need, dtype=torch.uint8, device=DEV)
    first = c.run(ws=ws)
    torch.cuda.synchronize()
    c.check(*first, what="eager")
    for again in range(3):                            # same bits every time, whatever lies in the workspace
        ws.random_(0, 256)
        got = c.run(ws=ws)
        torch.cuda.synchronize()
        assert torch.equal(got[0], first[0]) and torch.equal(got[1], first[1]), again
    out, lse = torch.empty_like(c.qd), torch.empty(c.qd.shape[0], Hq, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(out=out, lse=lse, ws=ws)
    longest = rows.index(max(rows))
    for replay in range(4):
        c.qd.normal_()
        c.rows_d[longest] = max(rows) - 9000 * replay
        want = c.run()
        out.fill_(3.0)
        graph.replay()                                # on what the one before left in the workspace
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]), "replay %d" % replay


@pytest.mark.parametrize("row", [100_000_000, 1 << 27])
@pytest.mark.parametrize("dtype,d,tokens", [(BF16, 128, 1), (F32, 64, 1), (BF16, 96, 20), (BF16, 160, 1)])
def test_rows_far_apart(row, dtype, d, tokens):
    # a row-major pool [block_rows, blocks, heads, ..]: the tiles of a step (16 rows each, four of a block) begin up to 48 rows of 2^27 bytes apart
    laq = _laq()
    print("case:", row, dtype, d, tokens, flush=True)
    H, br = 2, 64
    c = Case(dtype, 8, H, d, br, [150, 70, 64], [tokens] * 3)
    blocks = c.cache.k.shape[0]
    buffer = torch.empty(br * row, dtype=torch.uint8, device=DEV)
    planes, at = [], 0
    for plane in c.cache:
        w = plane.shape[3]
        planes.append(buffer.as_strided(plane.shape, (H * w, w, row, 1), at))
        planes[-1].copy_(plane)
        at += -(-blocks * H * w // 16) * 16
    near = c.run()
    c.cache = laq.Fp4Cache(*planes)
    out, lse = c.run()
    torch.cuda.synchronize()
    assert torch.equal(out, near[0]) and torch.equal(lse, near[1])
    c.check(out, lse)


def test_a_workspace_outlives_the_call_on_another_stream():
    # the stream is busy, the call returns, and the caller's stream takes memory of the workspace's size and fills it
    laq = _laq()
    c = Case(BF16, 8, 2, 128, 64, [30000], [1])
    need = laq.laq_fp4_attention_workspace_bytes(c.cache, 8, BF16, 1, 1, 30000)
    want = c.run()
    side, busy = torch.cuda.Stream(), torch.randn(4096, 4096, device=DEV)
    torch.cuda.synchronize()
    for handle in (side, side.cuda_stream):
        with torch.cuda.stream(side):
            for _ in range(20):
                busy = (busy @ busy).clamp(-1, 1)
        got = c.run(stream=handle)
        others = [torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV) for _ in range(8)]
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        del others


@pytest.mark.parametrize("rows,tokens", [([(1 << 31) - 16], [1]), ([(1 << 31) - 16, 100, (1 << 31) - 20], [1, 1, 1]), ([(1 << 31) - 16, 50], [3, 2])])
def test_as_many_rows_as_a_table_may_hold(rows, tokens):
    """2^31 - 16 rows, 511 blocks of which the first 510 are one and the same: K = 0 and V = 1 there, V = 3 in the last one, whose last four rows have
    logits of 51 more and V of their own.  A sum of weights is one of at most 2^17 ones a lane (exact) and of 16 lanes, 4 waves and 1024 ranges: e = 2^-13 of it and of the
    numerator at most, twice that of out.  Logits are 36 * 0.1768 * 8 in 64 bits; the exponent's rounding of 2^-24 * 74 * 2 is 2^-16."""
    laq = _laq()
    print("case:", rows, tokens, flush=True)
    br, width, d, n, tail = 16 * 262657, 511, 32, len(rows), [100.0, 200.0, 400.0, 800.0]
    cache = laq.laq_fp4_cache(2, 1, br, d, DEV)
    k, v = torch.zeros(2 * br, 1, d, device=DEV), torch.ones(2 * br, 1, d, device=DEV)
    v[br:] = 3.0
    k[-4:] = 6.0
    v[-4:] = torch.tensor(tail, device=DEV)[:, None, None]
    laq.laq_fp4_store(cache, k, v, torch.arange(2 * br, dtype=torch.int32, device=DEV))
    tail = plain.values(*plain.quantise(v[-4:, 0].cpu()))[:, 0].tolist()
    table = torch.zeros(n, width, dtype=torch.int32, device=DEV)
    table[:, -1] = 1
    T = sum(tokens)
    start = None if T == n else torch.tensor([0] + tokens, dtype=torch.int32, device=DEV).cumsum(0).int()
    out, lse = laq.laq_fp4_attention(torch.full((T, 1, d), 1.5, device=DEV), cache, table, torch.tensor(rows, dtype=torch.int32, device=DEV), start=start, want_lse=True)
    torch.cuda.synchronize()
    tok, logit = 0, 1.5 * 6.0 * d / math.sqrt(d)
    for r, t in zip(rows, tokens):
        for x in range(t):
            seen = r - t + x + 1
            ordinary = min(seen, br * width - 4)
            weights = [(1.0, min(ordinary, br * 510)), (3.0, max(ordinary - br * 510, 0))] + [(value, math.exp(logit)) for value in tail[:seen - ordinary]]
            total = sum(w for _, w in weights)
            want = sum(value * w for value, w in weights) / total
            assert (out[tok].cpu().double() - want).abs().max() <= 2.0 ** -12 * want, (r, x)
            assert abs(lse[tok].item() - math.log(total)) <= 2.0 ** -12, (r, x)
            tok += 1


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_every_scale_and_code_reads_as_its_number(dtype):
    # row s: all codes with scale s; what the type does not hold is an infinity
    laq = _laq()
    cache = laq.laq_fp4_cache(16, 1, 16, 32, DEV)
    codes = (torch.arange(0, 32, 2) % 16 + 16 * (torch.arange(1, 32, 2) % 16)).to(torch.uint8).expand(256, 16)
    scales = torch.arange(256, dtype=torch.int32).to(torch.uint8)[:, None]
    for plane, x in ((cache.k, codes), (cache.k_scale, scales), (cache.v, codes.flip(1)), (cache.v_scale, scales)):
        plane.copy_(x.view(plane.shape).to(DEV))
    got = laq.laq_fp4_load(cache, torch.arange(256, dtype=torch.int32, device=DEV), dtype)
    torch.cuda.synchronize()
    for y, x in zip(got, (codes, codes.flip(1))):
        want = plain.values(x, scales).to(dtype).double()
        assert torch.equal(torch.nan_to_num(y[:, 0].cpu().double(), nan=12345.0, posinf=math.inf, neginf=-math.inf),
                           torch.nan_to_num(want, nan=12345.0, posinf=math.inf, neginf=-math.inf))


@pytest.mark.parametrize("split", [True, False])
@pytest.mark.parametrize("dtype,tokens,Hq,H,d,long", [(F32, 1, 4, 2, 64, 60), (F32, 5, 4, 2, 128, 60), (F32, 30, 4, 2, 64, 60), (F32, 20, 8, 2, 160, 60), (F32, 3, 4, 2, 256, 60),
                                                      (F32, 6, 8, 2, 96, 3000), (F32, 1, 8, 2, 224, 3000), (BF16, 6, 8, 2, 128, 3000), (BF16, 40, 8, 2, 256, 3000)])
def test_a_nan_of_any_row_reaches_those_that_see_it_alone(split, dtype, tokens, Hq, H, d, long):
    # in V and in K; the last row, one that the first tokens do not see, and one that all see; whole columns and cut ones
    laq = _laq()
    print("case:", dtype, tokens, Hq, H, d, long, split, flush=True)
    G, head, block = Hq // H, H - 1, d // 32 - 1
    for nan_row in {long - 1, long - tokens // 2 - 1, long // 2}:
        c = Case(dtype, Hq, H, d, 16, [50, long], [tokens, tokens])
        clean = [x.cpu() for x in c.run(split=split)]
        slot = torch.tensor([int(c.table[1, nan_row // 16]) * 16 + nan_row % 16], dtype=torch.int32, device=DEV)
        bad = c.v[50 + nan_row][None].clone()
        bad[0, head, 32 * block + 7] = math.nan
        laq.laq_fp4_store(c.cache, None, bad.to(DEV), slot)
        out, lse = (x.cpu() for x in c.run(split=split))
        # (the other blocks of that head keep their bits, and so does everything else)
        want = clean[0].clone().view(2, tokens, Hq, d)
        sees = torch.arange(tokens) + long - tokens >= nan_row
        assert sees.any()
        want[1, sees, head * G:, 32 * block:32 * block + 32] = math.nan
        assert torch.equal(torch.nan_to_num(out.double(), nan=777.0), torch.nan_to_num(want.view_as(out).double(), nan=777.0)), nan_row
        assert torch.equal(lse, clean[1])
        key = c.k[50 + nan_row][None].clone()
        key[0, head, 0] = -math.inf
        laq.laq_fp4_store(c.cache, key.to(DEV), c.v[50 + nan_row][None].to(DEV), slot)
        out, lse = (x.cpu() for x in c.run(split=split))
        want = clean[0].clone().view(2, tokens, Hq, d)
        want[1, sees, head * G:] = math.nan
        want_lse = clean[1].clone().view(2, tokens, Hq)
        want_lse[1, sees, head * G:] = math.nan
        assert torch.equal(torch.nan_to_num(out.double(), nan=777.0), torch.nan_to_num(want.view_as(out).double(), nan=777.0)), nan_row
        assert torch.equal(torch.nan_to_num(lse, nan=777.0), torch.nan_to_num(want_lse.view_as(lse), nan=777.0)), nan_row


@pytest.mark.parametrize("dtype,d", [(F32, 64), (F32, 128), (F32, 256), (BF16, 256)])
def test_infinite_and_nan_queries_of_any_type_stay_with_their_own_head(dtype, d):
    for rows, tokens in (([100, 40], [3, 1]), ([2500, 40], [1, 1]), ([300, 90], [30, 20])):
        c = Case(dtype, 8, 2, d, 16, rows, tokens)
        want = [x.cpu() for x in c.run()]
        q, last = c.qd.clone(), sum(tokens) - 1
        q[0, 2, 5] = math.nan
        q[last, 7, 9] = math.inf
        c.qd = q
        got = [x.cpu() for x in c.run()]
        same = torch.ones(last + 1, 8, dtype=torch.bool)
        same[0, 2] = same[last, 7] = False
        assert torch.equal(got[0][same], want[0][same]) and torch.equal(got[1][same], want[1][same])
        assert torch.isnan(got[0][0, 2]).all() and torch.isnan(got[0][last, 7]).all() and torch.isnan(got[1][0, 2]) and torch.isnan(got[1][last, 7])


def test_long_folds_of_two_streams_and_of_graphs_that_share_a_workspace():
    laq = _laq()
    cases = [Case(BF16, 16, 1, 64, 64, [100000] + [100] * 40, [1] * 41), Case(BF16, 16, 1, 32, 64, [200000], [1], seed=2), Case(BF16, 8, 2, 128, 64, [3000, 17], [1, 1], seed=3)]
    want = [c.run() for c in cases]
    torch.cuda.synchronize()
    sides, got = [torch.cuda.Stream() for _ in cases], [[] for _ in cases]
    for _ in range(6):
        for i, c in enumerate(cases):
            with torch.cuda.stream(sides[i]):
                got[i].append(c.run())
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for w, several in zip(want, got) for g in several for x, y in zip(w, g))
    need = [laq.laq_fp4_attention_workspace_bytes(c.cache, c.Hq, BF16, len(c.rows), c.qd.shape[0], max(c.rows)) for c in cases]
    ws = torch.zeros(max(need), dtype=torch.uint8, device=DEV)
    graphs, outs = [], []
    for c in cases:
        outs.append((torch.empty_like(c.qd), torch.empty(c.qd.shape[0], c.Hq, device=DEV)))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.run(out=outs[-1][0], lse=outs[-1][1], ws=ws)
        graphs.append(graph)
    for order in ((0, 1, 2), (1, 1, 0, 2, 0), (2, 0, 1)):
        for c in cases:
            c.qd.normal_()
        want = [c.run() for c in cases]
        for i in order:
            outs[i][0].fill_(3.0)
            graphs[i].replay()
            cases[(i + 1) % 3].run(ws=ws)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for w, o in zip(want, outs) for x, y in zip(w, o)), order


@pytest.mark.parametrize("dtype,Hq,H,d,rows", [(BF16, 320, 8, 64, [5700, 100] * 8), (F32, 160, 8, 32, [5700, 0, 3, 900] * 5), (BF16, 132, 4, 192, [3000, 2900, 1] * 8)])
def test_shared_out_requests_of_several_tiles(dtype, Hq, H, d, rows):
    # 40, 20 and 33 query heads a KV head: tiles of 16, the last ones short
    print("case:", dtype, Hq, H, d, flush=True)
    c = Case(dtype, Hq, H, d, 32, rows, [1] * len(rows))
    first = c.run()
    torch.cuda.synchronize()
    c.check(*first)
    again = c.run()
    torch.cuda.synchronize()
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_replayed_maps_of_many_workgroups():
    # as many slots as 16 workgroups and more have, appended and dropped in a captured launch each
    laq = _laq()
    n, br, n_blocks, width = 300, 16, 20000, 80
    gen = torch.Generator().manual_seed(4)
    adds = [torch.randint(0, 500, (n,), generator=gen).int().to(DEV) for _ in range(2)]
    state_of = lambda: (torch.zeros(n, dtype=torch.int32, device=DEV), torch.full((n, width), -1, dtype=torch.int32, device=DEV), *laq.laq_block_pool(n_blocks, DEV))  # noqa: E731
    eager, replayed = state_of(), state_of()
    add, back = torch.zeros_like(adds[0]), torch.zeros_like(adds[0])
    start, slots = torch.empty(n + 1, dtype=torch.int32, device=DEV), torch.empty(160000, dtype=torch.int32, device=DEV)
    saved = [t.clone() for t in replayed]
    laq.laq_block_map(add, *replayed, br, start=start, slots=slots)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        laq.laq_block_map(add, *replayed, br, start=start, slots=slots)
        laq.laq_block_map(back, *replayed, br)
    for t, s in zip(replayed, saved):
        t.copy_(s)
    for replay in range(5):
        add.copy_(adds[replay % 2])
        back.copy_(-(adds[replay % 2] // 2))
        graph.replay()
        want = laq.laq_block_map(add, *eager, br, n_slots=160000)
        laq.laq_block_map(back, *eager, br)
        torch.cuda.synchronize()
        assert torch.equal(start, want[0]) and torch.equal(slots, want[1]), replay
        assert torch.equal(replayed[0], eager[0]) and torch.equal(replayed[1], eager[1]) and torch.equal(replayed[3], eager[3])
        held = eager[3][0].item()
        assert torch.equal(replayed[2][:held], eager[2][:held])
