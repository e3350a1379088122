"""The operators around a paged cache held in 4 bits, as measurable cases: their plain forms and the library's calls.

What is kept of an evicted cache lies in a pool of blocks of `block` rows, its numbers in 4 bits with one scale per 32
of them; requests own blocks through a table and grow and shrink from step to step.  Kinds of cases:

  map      laq_block_map: block tables and slot maps from request lengths.  Rows are appended to every request (blocks
           taken from the free list, a slot for every new row) and dropped again: a speculative or lookahead step whose
           tokens are rejected, or a batch that is admitted and released
  store    laq_fp4_store: the rows of new tokens into the cache, by slot (-1: no place, as in a padded batch); read back with laq_fp4_load
  compact  laq_fp4_compact: the rows that an eviction keeps, from the prefill cache into the cache; read back with laq_fp4_load
  attend   laq_fp4_attention: tokens attend to the cache; one per request (decoding), a few (lookahead steps, drafts),
           or a chunk of a prompt

Format of a row of d numbers: blocks of 32; a scale byte s stands for 2^(s-127); a code is a sign and one of the magnitudes
0, .5, 1, 1.5, 2, 3, 4, 6; number 2j of a row lies in the low half of byte j.  The exponent of a block is floor(log2 of its largest
magnitude) - 2, one more from 1.75 times that power of two on, within [-100, 125] (-100 for a block of zeros); a number is rounded to the
nearest code, ties to the even one, the largest code at most.  A block with an infinity or a NaN has s = 255, which stands for NaN.

Fields: heads, kv_heads, d, dtype as in the library's shape; n = requests (or (sequence, layer) instances); block = rows per
block; hi / lo = range of the requests' lengths (or of budgets), spread = how they lie in it: linear (a pyramid of budgets) or
ragged; tokens = new tokens per request; pad = rows of the batch without a place.
"""
import math

import torch

own = False          # run() computes the plain forms, or (True) calls the library

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _map(name=None, **kw):
    case = dict(kind="map", n=32, block=16, hi=2048, lo=128, spread="linear", add_hi=8, add_lo=8)
    return {**case, **kw, **({"name": name} if name else {})}


def _store(name=None, **kw):
    case = dict(kind="store", tokens=64, kv_heads=8, d=128, dtype="bf16", block=64, pad=0, layout="dense")
    return {**case, **kw, **({"name": name} if name else {})}


def _compact(name=None, **kw):
    case = dict(kind="compact", n=1, kv_heads=8, d=128, dtype="bf16", L=4096, hi=128, lo=128, spread="linear", block=64)
    return {**case, **kw, **({"name": name} if name else {})}


def _attend(name=None, **kw):
    case = dict(kind="attend", n=1, heads=32, kv_heads=8, d=128, dtype="bf16", hi=520, lo=520, spread="ragged", tokens=1, block=64)
    return {**case, **kw, **({"name": name} if name else {})}


def listed():
    return [
        # one lookahead step of a batch over pyramid budgets: 8 tokens a request, dropped again; latency is all of it
        _map("map-lookahead-step"),
        # the compacted caches of all layers of eight sequences are given their places, and later released
        _map("map-admit-256", n=256, block=64, hi=0, lo=0, add_hi=2048, add_lo=257),
        # one decoding step of 64 sequences, a layer
        _store("store-step-64"),
        # a prompt of no round length, a layer, by a model that keeps K and V of a token side by side
        _store("store-prompt-16k", tokens=16381, layout="fused"),
        # full-precision rows of another head size, the batch padded
        _store("store-f32-d96", tokens=1000, kv_heads=4, d=96, dtype="f32", block=16, pad=24),
        # one evicted layer
        _compact("compact-layer-4k"),
        # all layers of an evicted prompt, pyramid budgets
        _compact("compact-32layer-8k", n=32, L=8192, hi=2048, lo=128),
        # one decoding step of one layer over a small budget: the smallest call
        _attend("attend-layer-520"),
        # four long caches that were never evicted
        _attend("attend-long-4x131k", n=4, hi=131071, lo=32768),
        # a large batch of unequal lengths
        _attend("attend-batch-128", n=128, hi=8192, lo=1000),
        # a lookahead step of 8 tokens, seven query heads per KV head, full precision, blocks of 16 rows
        _attend("attend-lookahead-f32", n=8, heads=28, kv_heads=4, d=96, dtype="f32", hi=1500, lo=700, tokens=8, block=16),
        # a chunk of 512 prompt tokens of each of four requests over what lies before it
        _attend("attend-chunk-4x512", n=4, hi=8704, lo=2100, tokens=512, block=128),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["map", "store", "compact", "attend"], [15, 15, 15, 55])[0]
    block = rng.choice([16, 32, 64, 128, 256])
    heads, kv_heads = rng.choice([(32, 8), (32, 8), (28, 4), (16, 8), (32, 32), (8, 1)])
    d = rng.choices([128, 64, 96, 256], [60, 20, 10, 10])[0]
    dtype = rng.choices(["bf16", "f32"], [80, 20])[0]
    spread = rng.choice(["linear", "ragged"])
    if kind == "map":
        n = _log_int(rng, 1, 1024)
        add = _log_int(rng, 1, max(1, min(4096, (1 << 19) // n)))
        hi = rng.choice([0, _log_int(rng, 1, 8192)])
        return _map(n=n, block=block, hi=hi, lo=hi // rng.choice([1, 2, 8]), spread=spread, add_hi=add, add_lo=max(1, add // rng.choice([1, 3, 10])))
    if kind == "store":
        return _store(tokens=_log_int(rng, 1, 16384), kv_heads=kv_heads, d=d, dtype=dtype, block=block, pad=rng.choice([0, 0, 1, 37]),
                      layout=rng.choice(["dense", "fused"]))
    hi = _log_int(rng, 1, 2048)
    if kind == "compact":
        L = _log_int(rng, max(64, hi), 16384)
        n = min(_log_int(rng, 1, 64), max(1, (1 << 28) // (kv_heads * L * d)))
        return _compact(n=n, kv_heads=kv_heads, d=d, dtype=dtype, L=L, hi=hi, lo=max(1, hi // rng.choice([1, 2, 16])), spread=spread, block=block)
    tokens = rng.choices([1, rng.randint(2, 16), _log_int(rng, 17, 512)], [60, 20, 20])[0]
    hi = max(_log_int(rng, 1, 65536), tokens)
    n = min(_log_int(rng, 1, 128), max(1, (1 << 28) // (kv_heads * hi * d)), max(1, (1 << 28) // (heads * tokens * hi)))
    return _attend(n=n, heads=heads, kv_heads=kv_heads, d=d, dtype=dtype, hi=hi, lo=max(tokens, hi // rng.choice([1, 3, 20])), spread=spread,
                   tokens=tokens, block=block)


def _lengths(n, hi, lo, spread):
    if spread == "linear":
        return [hi - (hi - lo) * i // max(1, n - 1) for i in range(n)]
    return [hi - int((hi - lo) * (i * 0.6180339887 % 1.0)) for i in range(n)]


def _quantise(x):
    """Codes [.., d / 2] and scales [.., d / 32] (uint8) of rows [.., d]."""
    b = x.float().unflatten(-1, (-1, 32))
    most = b.abs().amax(-1)
    part, power = torch.frexp(most)                       # most = part * 2^power, part in [0.5, 1)
    e = (power - 3 + (part >= 0.875)).clamp(-100, 125)
    e = torch.where(most > 0, e, -100)
    a = torch.ldexp(b.abs(), -e.unsqueeze(-1))
    code = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0) + 8 * torch.signbit(b)
    bad = ~torch.isfinite(b).all(-1)
    code = torch.where(bad.unsqueeze(-1), 0, code).flatten(-2).unflatten(-1, (-1, 2))
    scale = torch.where(bad, 255, e + 127)
    return (code[..., 0] + 16 * code[..., 1]).to(torch.uint8), scale.to(torch.uint8)


def _values(codes, scales):
    """What rows of codes [.., d / 2] and scales [.., d / 32] stand for, in 32 bits."""
    table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=codes.device)
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).unflatten(-1, (-1, 32))
    power = torch.ldexp(torch.ones((), device=codes.device), scales.int() - 127)
    power = torch.where(scales == 255, math.nan, power)
    return (table[c.int()] * power.unsqueeze(-1)).flatten(-2)


def _pool(n_blocks, H, br, d, dev):
    """An empty cache: codes and scales of K, then of V."""
    return [torch.zeros(n_blocks, H, br, w, dtype=torch.uint8, device=dev) for w in (d // 2, d // 32, d // 2, d // 32)]


def _places(lengths, br, n_blocks, gen, dev):
    """A shuffled block table (-1 where a request has no block) and the slot of every row, request by request."""
    per = max(1, max(-(-x // br) for x in lengths))
    have = torch.tensor([-(-x // br) for x in lengths], device=dev)
    order = torch.randperm(n_blocks, generator=gen, device=dev)
    first = torch.cumsum(have, 0) - have
    at = torch.arange(per, device=dev)
    table = torch.where(at < have[:, None], order[(first[:, None] + at).clamp(max=n_blocks - 1)], -1).int()
    rows = torch.arange(max(1, max(lengths)), device=dev)
    slots = table.long()[:, rows // br] * br + rows % br
    return table, slots[rows < torch.tensor(lengths, device=dev)[:, None]].int(), order


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed) * 6151 + 7)
    kind, br = case["kind"], case["block"]
    state = {"kind": kind, "block": br}
    if kind == "map":
        n = case["n"]
        rows = _lengths(n, case["hi"], case["lo"], case["spread"])
        add = _lengths(n, case["add_hi"], case["add_lo"], case["spread"])
        need = [-(-r // br) for r in rows]
        all_need = [-(-(r + a) // br) for r, a in zip(rows, add)]
        n_blocks = sum(all_need) + 5
        table, _, order = _places(rows, br, n_blocks, gen, dev)
        width = max(all_need) + 1
        free = torch.zeros(n_blocks, dtype=torch.int32, device=dev)
        free[:n_blocks - sum(need)] = order[sum(need):].int()
        state.update(rows=torch.tensor(rows, dtype=torch.int32, device=dev), add=torch.tensor(add, dtype=torch.int32, device=dev),
                     table=torch.nn.functional.pad(table, (0, width - table.shape[1]), value=-1).contiguous(), free=free,
                     count=torch.tensor([n_blocks - sum(need), 0, 0, 0], dtype=torch.int32, device=dev),
                     slots=torch.empty(sum(add), dtype=torch.int32, device=dev), start=torch.empty(n + 1, dtype=torch.int32, device=dev))
        state["drop"] = -state["add"]
        return state
    H, d, dt = case["kv_heads"], case["d"], DTYPES[case["dtype"]]
    state.update(dtype=dt)
    # keys have a few large channels, as rotated keys of trained models do
    channel = torch.where(torch.rand(H, 1, d, generator=gen, device=dev) < 0.05, 4.0, 1.0)
    if kind == "store":
        T, pad = case["tokens"], case["pad"]
        n_blocks = -(-T // br) + 3
        _, slots, _ = _places([T], br, n_blocks, gen, dev)
        rows = torch.randn(T + pad, 2, H, d, generator=gen, device=dev)
        rows[:, 0] *= channel[:, 0]
        k, v = rows.to(dt).unbind(1)
        if case["layout"] == "dense":
            k, v = k.contiguous(), v.contiguous()
        slots = slots[torch.randperm(T, generator=gen, device=dev)] if T <= 256 else slots
        state.update(cache=_pool(n_blocks, H, br, d, dev), k=k, v=v, slots=torch.cat([slots, torch.full((pad,), -1, dtype=torch.int32, device=dev)]))
        return state
    n = case["n"]
    lengths = _lengths(n, case["hi"], case["lo"], case["spread"])
    n_blocks = sum(-(-x // br) for x in lengths) + 3
    table, slots, _ = _places(lengths, br, n_blocks, gen, dev)
    if kind == "compact":
        L = case["L"]
        k = torch.randn(n, H, L, d, generator=gen, device=dev, dtype=dt) * channel.to(dt)
        v = torch.randn(n, H, L, d, generator=gen, device=dev, dtype=dt)
        idx = [torch.rand(H, L, generator=gen, device=dev).topk(b, -1).indices.sort(-1).values.int().flatten() for b in lengths]
        state.update(cache=_pool(n_blocks, H, br, d, dev), k=k, v=v, budgets=lengths, idx=torch.cat(idx), slots=slots)
        return state
    Hq, T = case["heads"], case["tokens"]
    cache = _pool(n_blocks, H, br, d, dev)
    step = max(1, (1 << 27) // (H * br * d))
    for b in range(0, n_blocks, step):
        m = min(step, n_blocks - b)
        cache[0][b:b + m], cache[1][b:b + m] = _quantise(torch.randn(m, H, br, d, generator=gen, device=dev) * channel)
        cache[2][b:b + m], cache[3][b:b + m] = _quantise(torch.randn(m, H, br, d, generator=gen, device=dev))
    # requests of a chunk have unequal numbers of tokens; all of one have T
    counts = [T - (i * 5) % max(1, T // 4) for i in range(n)]
    q = torch.randn(sum(counts), Hq, d, generator=gen, device=dev).to(dt)
    state.update(cache=cache, table=table, rows=torch.tensor(lengths, dtype=torch.int32, device=dev), max_rows=max(lengths), q=q, most=max(counts),
                 start=None if T == 1 else torch.tensor([0] + counts, dtype=torch.int32, device=dev).cumsum(0, dtype=torch.int32))
    return state


def _plain_map(s, add, slots, start):
    br, table, free, rows, count = s["block"], s["table"], s["free"], s["rows"].long(), s["count"]
    n, width = table.shape
    held = count[0].long()
    new = (rows + add).clamp(min=0)
    have, want = (rows + br - 1) // br, (new + br - 1) // br
    at = torch.arange(width, device=table.device)
    # blocks that requests give back, the last request's last one first
    back = (at >= want[:, None]) & (at < have[:, None])
    rank = back.flatten().flip(0).cumsum(0).flip(0).view_as(back) - 1
    free[(held + rank)[back]] = table[back]
    held = held + back.sum()
    # blocks that requests take, from the end of the list
    need = torch.where(want <= width, (want - have).clamp(min=0), 0)
    upto = need.cumsum(0)
    fits = (want <= width) & ((need == 0) | (upto <= held))
    need = torch.where(fits, need, 0)
    take = (at >= have[:, None]) & (at < (have + need)[:, None])
    place = held - 1 - (upto - need)[:, None] - (at - have[:, None])
    table[take] = free[place[take]]
    count[0], count[1] = held - need.sum(), (~fits).sum()
    new = torch.where(fits, new, rows)
    s["rows"].copy_(new)
    if slots is not None:
        more = add.long().clamp(min=0)
        start[0] = 0
        start[1:] = more.cumsum(0)
        req = torch.repeat_interleave(torch.arange(n, device=table.device), more, output_size=slots.numel())
        row = rows[req] + torch.arange(slots.numel(), device=table.device) - start[req]
        slots.copy_(torch.where(fits[req], table[req, (row // br).clamp(max=width - 1)] * br + row % br, -1))


def _plain_store(cache, br, k, v, slots):
    here = slots >= 0
    b, r = slots[here].long() // br, slots[here].long() % br
    for rows, codes, scales in ((k, cache[0], cache[1]), (v, cache[2], cache[3])):
        c, sc = _quantise(rows[here])
        codes[b, :, r] = c
        scales[b, :, r] = sc


def _plain_load(cache, br, slots, dt):
    here = (slots >= 0)[:, None, None]
    b, r = slots.clamp(min=0).long() // br, slots.clamp(min=0).long() % br
    return [torch.where(here, _values(codes[b, :, r], scales[b, :, r]), 0.0).to(dt) for codes, scales in (cache[:2], cache[2:])]


def _plain_gather(x, idx, budgets):
    """The rows of the list, all heads of a row together: [rows of all instances, H, d]."""
    n, H, L, d = x.shape
    dev = x.device
    b = torch.tensor(budgets, device=dev)
    inst = torch.repeat_interleave(torch.arange(n, device=dev), b, output_size=sum(budgets))
    first = torch.cumsum(b, 0) - b
    r = torch.arange(sum(budgets), device=dev) - first[inst]
    at = (first[inst] * H + r)[:, None] + torch.arange(H, device=dev) * b[inst][:, None]
    return x[inst[:, None], torch.arange(H, device=dev), idx[at].long()]


def _plain_attend(s):
    q, table, rows, br = s["q"], s["table"].long(), s["rows"].long(), s["block"]
    (T, Hq, d), (n, per) = q.shape, table.shape
    H = s["cache"][0].shape[1]
    G, dev = Hq // H, q.device
    start = torch.arange(n + 1, device=dev) if s["start"] is None else s["start"].long()
    t = torch.arange(s["most"], device=dev)
    live = t < (start[1:] - start[:-1])[:, None]                         # [n, most]
    tok = (start[:-1, None] + t).clamp(max=T - 1)
    # [n, H, rows, d], rows without a block as those of block 0, which nobody sees
    k, v = (_values(codes[table.clamp(min=0)], scales[table.clamp(min=0)]).transpose(1, 2).reshape(n, H, per * br, d)
            for codes, scales in (s["cache"][:2], s["cache"][2:]))
    qg = q.float()[tok].view(n, -1, H, G, d).permute(0, 2, 1, 3, 4).reshape(n, H, -1, d)
    x = torch.matmul(qg, k.transpose(2, 3).contiguous()).view(n, H, -1, G, per * br) * (1.0 / math.sqrt(d))
    last = rows[:, None] - (start[1:] - start[:-1])[:, None] + t         # the row that a token stands at
    seen = (torch.arange(per * br, device=dev) <= last[..., None])[:, None, :, None, :]
    x = x.masked_fill_(~seen, -math.inf)
    m = x.amax(-1, keepdim=True).clamp(min=-3e38)
    x = x.sub_(m).exp_()
    z = x.sum(-1, keepdim=True)
    y = torch.matmul(x.view(n, H, -1, per * br), v).view(n, H, -1, G, d)
    y = torch.where(z > 0, y / z, 0.0)
    lse = (m + z.log()).squeeze(-1)
    y, lse = y.permute(0, 2, 1, 3, 4).reshape(n, -1, Hq, d)[live], lse.permute(0, 2, 1, 3).reshape(n, -1, Hq)[live]
    return y.to(q.dtype), lse


def run(state):
    s = state
    if own:
        import paper_2505_20334_amd as laq
        if s["kind"] == "map":
            laq.laq_block_map(s["add"], s["rows"], s["table"], s["free"], s["count"], s["block"], start=s["start"], slots=s["slots"])
            laq.laq_block_map(s["drop"], s["rows"], s["table"], s["free"], s["count"], s["block"])
            return {k: s[k] for k in ("start", "slots", "rows", "table", "free", "count")}
        cache = laq.Fp4Cache(*s["cache"])
        if s["kind"] == "store":
            laq.laq_fp4_store(cache, s["k"], s["v"], s["slots"])
            k, v = laq.laq_fp4_load(cache, s["slots"], s["dtype"])
            return {"k": k, "v": v}
        if s["kind"] == "compact":
            laq.laq_fp4_compact(cache, s["k"], s["v"], s["idx"], s["budgets"], s["slots"])
            k, v = laq.laq_fp4_load(cache, s["slots"], s["dtype"])
            return {"k": k, "v": v}
        out, lse = laq.laq_fp4_attention(s["q"], cache, s["table"], s["rows"], start=s["start"], max_rows=s["max_rows"], want_lse=True)
        return {"out": out, "lse": lse}
    if s["kind"] == "map":
        _plain_map(s, s["add"], s["slots"], s["start"])
        _plain_map(s, s["drop"], None, None)
        return {k: s[k] for k in ("start", "slots", "rows", "table", "free", "count")}
    if s["kind"] == "store":
        _plain_store(s["cache"], s["block"], s["k"], s["v"], s["slots"])
        k, v = _plain_load(s["cache"], s["block"], s["slots"], s["dtype"])
        return {"k": k, "v": v}
    if s["kind"] == "compact":
        _plain_store(s["cache"], s["block"], _plain_gather(s["k"], s["idx"], s["budgets"]), _plain_gather(s["v"], s["idx"], s["budgets"]), s["slots"])
        k, v = _plain_load(s["cache"], s["block"], s["slots"], s["dtype"])
        return {"k": k, "v": v}
    out, lse = _plain_attend(s)
    return {"out": out, "lse": lse}


def _nearest(x):
    """What rows of [.., d] are stored as, in 64 bits: the scale by powers of two tried one by one, the code by distance."""
    b = x.double().unflatten(-1, (-1, 32))
    most = b.abs().amax(-1, keepdim=True)
    powers = 2.0 ** torch.arange(-100, 126, dtype=torch.float64, device=x.device)
    # the least power of two that the largest magnitude is below 7 times of
    step = powers[torch.searchsorted(powers * 7.0, most, right=True).clamp(max=225)]
    grid = torch.tensor(MAGNITUDES, dtype=torch.float64, device=x.device)
    best, far = torch.zeros_like(b), b.abs() / step
    off = far.clone()                                     # distance to 0, the first code
    for c in range(1, 8):
        d = (far - grid[c]).abs()
        nearer = (d < off) | ((d == off) & (c % 2 == 0))
        best, off = torch.where(nearer, grid[c], best), torch.where(nearer, d, off)
    return (best * step * torch.sign(b)).flatten(-2)


def exact(case, seed):
    if case["kind"] == "map":
        return None                                       # whole numbers
    s = prepare(case, seed)
    if case["kind"] == "store":
        here = (s["slots"] >= 0)[:, None, None]
        return {name: torch.where(here, _nearest(s[name]), 0.0) for name in ("k", "v")}
    if case["kind"] == "compact":
        found = {"k": [], "v": []}
        at, H = 0, case["kv_heads"]
        for i, b in enumerate(s["budgets"]):
            idx = s["idx"][at:at + H * b].view(H, b).long()
            at += H * b
            for name in found:
                found[name].append(torch.stack([_nearest(s[name][i, h, idx[h]]) for h in range(H)], 1))
        return {name: torch.cat(x) for name, x in found.items()}
    grid = torch.tensor(MAGNITUDES, dtype=torch.float64)
    grid = torch.cat([grid, -grid])
    pairs = torch.stack([grid.repeat(16), grid.repeat_interleave(16)], -1).to(s["q"].device)     # by byte
    q, br, d, H = s["q"].double(), s["block"], case["d"], case["kv_heads"]
    G = case["heads"] // H
    start = list(range(case["n"] + 1)) if s["start"] is None else s["start"].tolist()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float64, device=q.device)
    for i, L in enumerate(s["rows"].tolist()):
        T = start[i + 1] - start[i]
        blocks = s["table"][i, :-(-L // br)].long()
        hidden = torch.arange(L, device=q.device)[None, :] > (L - T + torch.arange(T, device=q.device))[:, None]
        for h in range(H):
            k, v = ((pairs[c[blocks, h].reshape(-1, d // 2)[:L].int()].flatten(-2).unflatten(-1, (-1, 32))
                     * torch.exp2(e[blocks, h].reshape(-1, d // 32)[:L].double() - 127)[..., None]).flatten(-2) for c, e in (s["cache"][:2], s["cache"][2:]))
            x = torch.einsum("tgd,ld->tgl", q[start[i]:start[i + 1], h * G:(h + 1) * G], k) / math.sqrt(d)
            x = x.masked_fill(hidden[:, None], -math.inf)
            out[start[i]:start[i + 1], h * G:(h + 1) * G] = torch.einsum("tgl,ld->tgd", torch.softmax(x, -1), v)
            lse[start[i]:start[i + 1], h * G:(h + 1) * G] = torch.logsumexp(x, -1)
    return {"out": out, "lse": lse}


def work(case):
    kind = case["kind"]
    if kind == "map":
        n, br = case["n"], case["block"]
        rows, add = _lengths(n, case["hi"], case["lo"], case["spread"]), _lengths(n, case["add_hi"], case["add_lo"], case["spread"])
        taken = sum(-(-(r + a) // br) - -(-r // br) for r, a in zip(rows, add))
        # lengths read and written twice, the blocks' numbers from the list to the table and back, starts and slots written
        return {"bytes": 4 * (6 * n + 4 * taken + n + 1 + sum(add)), "flops": 0}
    H, d, eb = case["kv_heads"], case["d"], 2 if case["dtype"] == "bf16" else 4
    row = d // 2 + d // 32
    if kind == "store":
        # rows read, stored; read back, written
        T = case["tokens"]
        return {"bytes": 2 * H * (2 * T * row + T * d * eb + (T + case["pad"]) * d * eb) + 8 * (T + case["pad"]), "flops": 0}
    lengths = _lengths(case["n"], case["hi"], case["lo"], case["spread"])
    if kind == "compact":
        T = sum(lengths)
        return {"bytes": 2 * H * T * (2 * row + 2 * d * eb) + 4 * H * T + 8 * T, "flops": 0}
    T, Hq = case["tokens"], case["heads"]
    counts = [T - (i * 5) % max(1, T // 4) for i in range(case["n"])]
    seen = sum(c * (x - c) + c * (c + 1) // 2 for x, c in zip(lengths, counts))
    return {"bytes": sum(lengths) * H * 2 * row + sum(counts) * Hq * (2 * d * eb + 4), "flops": 4 * seen * Hq * d}
