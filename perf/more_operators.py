"""Performance cases of the cache in 8 bits and of prefixes that sequences share: norm with rotation and quantising on the way into the
pages, reading tokens back, attention of one new token over pages in 8 bits, and attention of one new token for sequences whose first
tokens are the same, which are read once for all.

A row of 64 numbers x is held as e4m3 numbers and one exponent s: s is the least whole number with max |x| <= 448 * 2^s, and x / 2^s is
rounded to the nearest e4m3 number.  What is held so is returned as the values that it stands for.

The ranges.  Tokens are whole frames of camera and register tokens (5) and 37 x 37 patches or fewer, one to three hundred frames, or
single tokens of a stream; head dimension 64; 1 to 16 query heads, as many key heads or a divisor of them.  Pages hold 16 to 256 tokens
or a frame.  Batches are 1 to 128 sequences, their own tokens 0 to some thousands behind a prefix, up to 300 frames without one; a
batch has 1 to 6 prefixes of one to a hundred frames.  Tensors are bf16, or fp32 for short sequences; caches of the same type or e4m3.

Queries and keys of the attention cases are what the norm leaves: rows of length sqrt(64) times a gain.

`own` chooses the side: the plain form below (elementary torch operations in 32 bits, in 64 where a value next to a border of the e4m3
numbers would else go to the other side, rounded once at the end), or this package.
"""
import math

import torch

own = False

DIM = 64
SPECIAL = 5  # camera and register tokens of a frame
FRAME = SPECIAL + 37 * 37
SCALE = 1.0 / math.sqrt(DIM)
EPS = 1e-6
GAIN = math.sqrt(2.0)  # learned scale of the norms: logits of queries and keys that do not belong together spread by 2
_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}
_ROW = {"bf16": 2 * DIM, "fp32": 4 * DIM, "e4m3": DIM + 1}  # bytes of a row in a cache


# ---- cases ------------------------------------------------------------------------------------------

def _store(name, op, tokens, heads, kv_heads, norm, axes, page, dtype="bf16", base=100.0, first=0, context=0):
    """first: position of the first token where positions count along the sequence (axes = 1).  context: tokens that are read back."""
    return {"name": name, "op": op, "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "norm": norm, "axes": axes, "page": page,
            "dtype": dtype, "base": base, "first": first, "context": context}


def _load(name, tokens, kv_heads, page, cache="e4m3", dtype="bf16", first=0):
    return {"name": name, "op": "load", "tokens": tokens, "first": first, "kv_heads": kv_heads, "page": page, "cache": cache, "dtype": dtype}


def _attend(name, op, batch, longest, shortest, heads, kv_heads, page, cache="e4m3", dtype="bf16", window=0, sinks=0, frame=1, prefixes=0,
            prefix_longest=0, prefix_shortest=0):
    """window 0: every cached token is visible.  Lengths are spread between the shortest and the longest, those of prefixes as well."""
    return {"name": name, "op": op, "batch": batch, "longest": longest, "shortest": shortest, "heads": heads, "kv_heads": kv_heads, "page": page,
            "cache": cache, "dtype": dtype, "window": window, "sinks": sinks, "frame": frame, "prefixes": prefixes,
            "prefix_longest": prefix_longest, "prefix_shortest": prefix_shortest}


def listed():
    return [
        # one decoding step of 24 streams: the new token normed, turned and stored, then attended from
        _attend("step_24_streams", "step", 24, 2000, 100, 16, 4, 64),
        # a prompt of the benchmark's headline length into the cache; its attention goes over the rows as the cache holds them
        _store("store_100_frames", "store", 100 * FRAME, 16, 16, "layer", 2, 64),
        # a text-like prompt of odd length with shared keys, far along a sequence
        _store("store_odd", "store", 4123, 16, 4, "rms", 1, 100, base=10000.0, first=1000000),
        # one new frame into the cache, and the twelve frames that its attention reads back out of it
        _store("extend_frame", "extend", FRAME, 16, 16, "layer", 2, 64, context=12 * FRAME),
        # a long scan read back whole, a page to a frame
        _load("load_300_frames", 300 * FRAME, 16, FRAME),
        # one stream's query over a short cache: latency
        _attend("paged_e4m3_one", "paged", 1, 8 * FRAME, 8 * FRAME, 16, 16, 64),
        # many streams of unequal length with shared keys, window and sinks
        _attend("paged_e4m3_batch", "paged", 96, 12000, 1, 16, 4, 16, window=4096, sinks=4),
        # two long scans whole in the cache, a page to a frame
        _attend("paged_e4m3_300_frames", "paged", 2, 300 * FRAME, 300 * 1041, 16, 16, FRAME),
        # a few streams that ask about the same short clip: latency
        _attend("prefix_clip", "prefix", 8, 300, 1, 16, 16, 64, cache="bf16", prefixes=1, prefix_longest=4 * FRAME, prefix_shortest=4 * FRAME),
        # many streams on one scan of the headline's length
        _attend("prefix_scan", "prefix", 64, 2000, 10, 16, 16, 64, cache="bf16", prefixes=1, prefix_longest=100 * FRAME, prefix_shortest=100 * FRAME),
        # more of them with shared keys, the cache in 8 bits
        _attend("prefix_scan_e4m3", "prefix", 128, 500, 1, 16, 4, 64, prefixes=1, prefix_longest=100 * FRAME, prefix_shortest=100 * FRAME),
        # streams on five scenes of unequal length, a window of frames and the first frame
        _attend("prefix_scenes", "prefix", 60, 3000, 5, 16, 8, FRAME, window=24, sinks=FRAME, frame=FRAME, prefixes=5, prefix_longest=60 * FRAME,
                prefix_shortest=7 * FRAME + 100),
    ]


_MOST_PAIRS = 128 * 100 * FRAME * 16  # of queries, keys and heads in a drawn case with prefixes
_MOST_CACHED = 300 * (FRAME + 1041) * 16  # cached tokens, times key heads


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    heads = rng.choice([16, 16, 8, rng.randint(1, 16)])
    kv_heads = rng.choice([heads, rng.choice([h for h in range(1, heads + 1) if heads % h == 0])])
    rows, cols = rng.choice([(37, 37), (37, 28), (rng.randint(16, 37), rng.randint(16, 37))])
    frame = SPECIAL + rows * cols
    page = rng.choice([16, 64, 256, frame])
    op = rng.choice(["store", "extend", "load", "step", "paged", "paged", "prefix", "prefix", "prefix"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if op in ("store", "extend"):
        tokens = spread(1, 100000) if op == "store" else spread(1, 4000)
        context = tokens + spread(1, 60000) if op == "extend" else 0
        if dtype == "fp32":  # rows that are normed and turned already
            c = _store("", op, max(1, tokens // 4), heads, kv_heads, "none", 0, page, dtype, context=context)
        else:
            axes = rng.choice([1, 2])
            c = _store("", op, tokens, heads, kv_heads, rng.choice(["rms", "layer"]), axes, page, dtype,
                       100.0 if axes == 2 else rng.choice([10000.0, 500000.0]), rng.choice([0, spread(1, 2000000)]) if axes == 1 else 0, context)
    elif op == "load":
        cache = rng.choice(["e4m3", "e4m3", dtype])
        tokens = spread(1, 300000) // (1 if dtype == "bf16" else 2) + 1
        c = _load("", tokens, kv_heads, page, cache, dtype, rng.choice([0, spread(1, 20000)]))
    else:
        batch = spread(1, 128)
        windowed = rng.random() < 0.4
        one = rng.random() < 0.5
        seen = dict(window=(spread(64, 16384) if one else rng.randint(1, 8)) if windowed else 0, sinks=rng.choice([0, 4, frame]) if windowed else 0,
                    frame=frame if windowed and not one else 1)
        if op == "step":
            longest = spread(1, 4000)
            c = _attend("", op, batch, longest, max(1, int(longest * rng.random())), heads, kv_heads, page, "e4m3", "bf16", **seen)
        elif op == "paged":
            longest = max(1, min(spread(1, 300000), _MOST_CACHED // (batch * kv_heads) // (1 if dtype == "bf16" else 2)))
            c = _attend("", op, batch, longest, max(1, int(longest * rng.random())), heads, kv_heads, page, "e4m3", dtype, **seen)
        else:
            cache = rng.choice([dtype, "e4m3"])
            prefixes = rng.choice([1, 1, 1, rng.randint(2, 6)])
            most = _MOST_PAIRS // (batch * heads) // (1 if dtype == "bf16" else 8)
            scan = max(1, min(spread(200, 137400), most))
            longest = max(0, min(spread(1, 4000) - 1, most))
            c = _attend("", op, batch, longest, int(longest * rng.random()), heads, kv_heads, page, cache, dtype, prefixes=prefixes, prefix_longest=scan,
                        prefix_shortest=max(1, int(scan * rng.random())) if prefixes > 1 else scan, **seen)
    del c["name"]
    return c


# ---- sizes ------------------------------------------------------------------------------------------

def _visible(p, keys, frame, window, sinks):
    """(keys of the first tokens, first key of the window) that the query at position p sees of the first `keys` keys, none of which is behind it."""
    lo = min(keys, max(0, (p // frame - window + 1) * frame)) if window else 0
    return min(sinks, lo), lo


def _between(count, longest, shortest):
    if count < 2:
        return [longest] * count
    step = (longest - shortest) / (count - 1)
    return [int(round(shortest + i * step)) for i in range(count)]


def _lengths(c):
    return _between(c["batch"], c["longest"], c["shortest"])


def _scenes(c):
    """Lengths of the prefixes, and the sequences that each has: [starts[i], starts[i + 1])."""
    n = c["prefixes"]
    return _between(n, c["prefix_longest"], c["prefix_shortest"]), [c["batch"] * i // n for i in range(n + 1)]


def work(c):
    size = 4 if c["dtype"] == "fp32" else 2
    row = DIM * size
    if c["op"] == "load":
        return {"bytes": 2 * c["tokens"] * c["kv_heads"] * (_ROW[c["cache"]] + row), "flops": 2 * c["tokens"] * c["kv_heads"] * DIM}
    if c["op"] in ("store", "extend"):
        n, H, K = c["tokens"], c["heads"], c["kv_heads"]
        stored = 2 * n * K * (_ROW["e4m3"] + (row if c["op"] == "store" else 0))
        back = 2 * c["context"] * K * (_ROW["e4m3"] + row)
        return {"bytes": n * (2 * H + 2 * K) * row + stored + back + 4 * n * (c["axes"] + 1), "flops": n * (H + 2 * K) * DIM * 12}
    H, K = c["heads"], c["kv_heads"]
    seen = pairs = 0
    if c["op"] == "prefix":
        lengths = _lengths(c)
        scans, starts = _scenes(c)
        for i, n in enumerate(scans):
            cut = [_visible(n + m - 1, n, c["frame"], c["window"], c["sinks"]) for m in lengths[starts[i]:starts[i + 1]]]
            pairs += sum(s + n - lo for s, lo in cut)
            if cut:  # read once for all
                seen += max(s for s, _ in cut) + n - min(lo for _, lo in cut)
            for m in lengths[starts[i]:starts[i + 1]]:
                s, lo = _visible(n + m - 1, n + m, c["frame"], c["window"], c["sinks"])
                pairs += m - max(0, lo - n) + max(0, s - n)
                seen += m - max(0, lo - n) + max(0, s - n)
    else:
        for n in _lengths(c):
            s, lo = _visible(n - 1, n, c["frame"], c["window"], c["sinks"])
            pairs += s + n - lo
        seen = pairs
    rows = 2 * c["batch"] * H + (2 * c["batch"] * K if c["op"] == "step" else 0)
    return {"bytes": 2 * seen * K * _ROW[c["cache"]] + rows * row, "flops": 4 * DIM * pairs * H}


# ---- inputs -----------------------------------------------------------------------------------------

def _unit_rows(g, n, gain, dtype=torch.float32):
    x = torch.empty((n, DIM), dtype=dtype, device="cuda")
    for part in x.split(1 << 22):  # no large temporaries
        r = torch.randn((part.shape[0], DIM), generator=g, device="cuda")
        part.copy_(r if gain is None else r * (gain * r.square().mean(1, keepdim=True).rsqrt()))
    return x


def _cache(g, c, pages):
    """Pages that are written already: {"k_cache", "v_cache"}, for e4m3 also {"k_scale", "v_scale"}, the exponents + 127."""
    got, shape = {}, (pages, c["kv_heads"], c["page"])
    for t, gain in (("k", GAIN), ("v", None)):
        if c.get("cache", "e4m3") != "e4m3":
            got[t + "_cache"] = _unit_rows(g, math.prod(shape), gain, _TYPES[c["cache"]]).view(*shape, DIM)
            continue
        codes = torch.empty((math.prod(shape), DIM), dtype=torch.uint8, device="cuda")
        scale = torch.empty(math.prod(shape), dtype=torch.uint8, device="cuda")
        for at in range(0, codes.shape[0], 1 << 21):
            x = _unit_rows(g, min(1 << 21, codes.shape[0] - at), gain)
            s = _exponents(x)
            codes[at:at + x.shape[0]] = (x * torch.exp2(-s)).to(torch.float8_e4m3fn).view(torch.uint8)
            scale[at:at + x.shape[0]] = (s[:, 0] + 127).to(torch.uint8)
        got[t + "_cache"], got[t + "_scale"] = codes.view(torch.float8_e4m3fn).view(*shape, DIM), scale.view(shape)
    return got


def _tables(g, lists, page):
    """Tables of sequences of these lengths, pages in random order, and the number of pages."""
    need = [[-(-n // page) for n in lengths] for lengths in lists]
    order = torch.randperm(max(1, sum(map(sum, need))), generator=g, device="cuda").int()
    tables, at = [], 0
    for of in need:
        table = torch.full((len(of), max(of + [1])), -1, dtype=torch.int32, device="cuda")
        for i, m in enumerate(of):
            table[i, :m] = order[at:at + m]
            at += m
        tables.append(table)
    return tables, order.numel()


def _slots(table, page, places):
    """Slots of the tokens places[i] (int64) of table row i, one row after the other."""
    return torch.cat([table[i, p // page].long() * page + p % page for i, p in enumerate(places)]).int()


def _projected(g, n, c, s):
    """What the projection gives: [tokens, heads, 64], queries, keys and values beside each other, and what norms them."""
    H, K, dtype = c["heads"], c["kv_heads"], _TYPES[c["dtype"]]
    x = torch.empty((n, H + 2 * K, DIM), dtype=dtype, device="cuda")
    for h in range(H + 2 * K):
        x[:, h] = (0.3 + 0.2 * h) * torch.randn((n, DIM), generator=g, device="cuda") + 0.1
    s["q"], s["k"], s["v"] = x[:, :H], x[:, H:H + K], x[:, H + K:]
    norm = c.get("norm", "rms")
    for t in ("q", "k"):
        s[t + "_weight"] = None if norm == "none" else (GAIN + 0.2 * torch.randn((DIM,), generator=g, device="cuda")).to(dtype)
        s[t + "_bias"] = (0.1 * torch.randn((DIM,), generator=g, device="cuda")).to(dtype) if norm == "layer" else None


def _grid_positions(n):
    # patches by row and column from 1 on, camera and register tokens of each frame at 0
    at = torch.arange(n, device="cuda") % FRAME - SPECIAL
    yx = torch.stack([at.div(37, rounding_mode="floor") + 1, at.remainder(37) + 1], dim=1)
    return torch.where(at[:, None] >= 0, yx, torch.zeros_like(yx)).int().contiguous()


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"c": c}
    if c["op"] in ("store", "extend"):
        n, total = c["tokens"], max(c["tokens"], c["context"])
        _projected(g, n, c, s)
        s["positions"] = None if c["axes"] == 0 else _grid_positions(n) if c["axes"] == 2 else (
            c["first"] + torch.arange(n, device="cuda", dtype=torch.int32)).view(n, 1).contiguous()
        (table,), pages = _tables(g, [[total]], c["page"])
        s["pages"] = table[0].contiguous()
        s["slots"] = _slots(table, c["page"], [torch.arange(total - n, total, device="cuda")])
        s.update(_cache(g, c, pages))
        return s
    if c["op"] == "load":
        (table,), pages = _tables(g, [[c["first"] + c["tokens"]]], c["page"])
        s["pages"] = table[0].contiguous()
        s.update(_cache(g, c, pages))
        return s
    lengths = _lengths(c)
    scans, starts = _scenes(c) if c["op"] == "prefix" else ([], [])
    tables, pages = _tables(g, [lengths, scans], c["page"])
    s["page_table"], s["lengths"] = tables[0], torch.tensor(lengths, dtype=torch.int32).cuda()
    s.update(_cache(g, c, pages))
    if c["op"] == "prefix":
        s["prefix_table"] = tables[1]
        s["prefix_lengths"], s["starts"] = (torch.tensor(x, dtype=torch.int32).cuda() for x in (scans, starts))
    if c["op"] == "step":
        _projected(g, c["batch"], c, s)
        last = s["lengths"].long() - 1
        s["positions"] = last.int().view(-1, 1).contiguous()
        s["slots"] = _slots(s["page_table"], c["page"], [last[i:i + 1] for i in range(c["batch"])])
    else:  # as the norm with the rotation leaves it
        s["q"] = _unit_rows(g, c["heads"] * c["batch"], GAIN, _TYPES[c["dtype"]]).view(c["heads"], c["batch"], DIM).transpose(0, 1)
    return s


# ---- the plain forms --------------------------------------------------------------------------------

def _exponents(x):
    """The exponent of every row, [..., 1]."""
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True))  # m in [0.5, 1); 448 = 0.875 * 2^9
    return (e - 9 + (m > 0.875)).clamp(-117, 119).to(x.dtype)


def _put(s, t, slots, x):
    """The rows x [tokens, heads, 64] into the cache of t; returns the values that it holds of them then."""
    e = _exponents(x)
    codes = (x * torch.exp2(-e)).float().to(torch.float8_e4m3fn)
    page, row = slots.long() // s["c"]["page"], slots.long() % s["c"]["page"]
    s[t + "_cache"].view(torch.uint8)[page, :, row] = codes.view(torch.uint8)
    s[t + "_scale"][page, :, row] = (e[..., 0] + 127).to(torch.uint8)
    return codes.float() * torch.exp2(e.float())


def _get(s, t, page, row):
    """Values of the rows at `row` of the pages `page` (of the same shape), [*, heads, 64] in 32 bits."""
    if s[t + "_cache"].dtype != torch.float8_e4m3fn:
        return s[t + "_cache"][page, :, row].float()
    codes = s[t + "_cache"].view(torch.uint8)[page, :, row].view(torch.float8_e4m3fn)
    return codes.float() * torch.exp2(s[t + "_scale"][page, :, row].float() - 127)[..., None]


def _turned(s, t):
    """Rows [tokens, heads, 64] normed and turned, in 64 bits: some of them are then taken to the nearest of few numbers."""
    c, x = s["c"], s[t].double()
    if c.get("norm", "rms") != "none":
        if c.get("norm") == "layer":
            x = x - x.mean(-1, keepdim=True)
        x = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * s[t + "_weight"].double()
        x = x if s[t + "_bias"] is None else x + s[t + "_bias"].double()
    if s["positions"] is None:
        return x
    n, heads, _ = x.shape
    axes = s["positions"].shape[1]
    half = DIM // axes // 2
    freq = c.get("base", 10000.0) ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    angle = s["positions"].double()[:, None, :, None] * freq
    a, b = x.view(n, heads, axes, 2, half).unbind(3)
    return torch.stack([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], dim=3).view(n, heads, DIM)


def _store_plain(s):
    q = _turned(s, "q").transpose(0, 1).to(s["q"].dtype).contiguous()
    k, v = _put(s, "k", s["slots"], _turned(s, "k")), _put(s, "v", s["slots"], s["v"].double())
    return q, *(x.transpose(0, 1).to(s["q"].dtype).contiguous() for x in (k, v))


def _load_plain(s, first, count):
    j = torch.arange(first, first + count, device="cuda")
    page, row = s["pages"].long()[j // s["c"]["page"]], j % s["c"]["page"]
    return tuple(_get(s, t, page, row).transpose(0, 1).to(_TYPES[s["c"]["dtype"]]).contiguous() for t in ("k", "v"))


def _own_keys(s, behind):
    """Keys, values [B, K, keys, 64] and who is seen [B, keys] of the sequences' own tokens, every sequence padded to the longest; `behind` [B]:
    tokens in front of them."""
    c = s["c"]
    n = s["lengths"].long()[:, None]
    p = behind[:, None] + n - 1
    lo = ((p.div(c["frame"], rounding_mode="floor") - c["window"] + 1) * c["frame"] - behind[:, None]).clamp(min=0) if c["window"] else torch.zeros_like(p)
    lo = torch.minimum(lo, n)
    first = torch.minimum((c["sinks"] - behind[:, None]).clamp(min=0), lo)
    i = torch.arange(int(min(max(_lengths(c)), c["window"] * c["frame"] + c["sinks"] if c["window"] else 1 << 40)), device="cuda")
    j = torch.where(i < first, i, i - first + lo)
    seen = j < n
    j = torch.where(seen, j, 0)
    page, row = s["page_table"].gather(1, j // c["page"]).clamp(min=0).long(), j % c["page"]
    return *(_get(s, t, page, row).transpose(1, 2) for t in ("k", "v")), seen


def _paged_plain(s, q):
    c = s["c"]
    B, H, K = c["batch"], c["heads"], c["kv_heads"]
    k, v, seen = _own_keys(s, torch.zeros_like(s["lengths"], dtype=torch.int64))
    x = (q.float().reshape(B, K, H // K, DIM) @ k.transpose(2, 3) * SCALE).masked_fill(~seen[:, None, None], -math.inf)
    p = (x - x.amax(-1, keepdim=True)).exp()
    return (p @ v / p.sum(-1, keepdim=True)).view(B, H, DIM).to(_TYPES[c["dtype"]])


def _prefix_plain(s):
    """The prefixes one after the other, their sequences together; the own tokens of all sequences at once."""
    c = s["c"]
    B, H, K = c["batch"], c["heads"], c["kv_heads"]
    G = H // K
    scans, starts = _scenes(c)
    behind = s["prefix_lengths"].long().repeat_interleave(s["starts"].diff().long(), output_size=B)
    k, v, seen = _own_keys(s, behind)
    q = s["q"].float().reshape(B, K, G, DIM)
    own_x = (q @ k.transpose(2, 3) * SCALE).masked_fill(~seen[:, None, None], -math.inf)
    out = torch.empty((B, H, DIM), dtype=s["q"].dtype, device="cuda")
    for i, n in enumerate(scans):
        a, b = starts[i], starts[i + 1]
        j = torch.arange(n, device="cuda")
        page, row = s["prefix_table"][i].long()[j // c["page"]], j % c["page"]
        pk, pv = (_get(s, t, page, row).transpose(0, 1) for t in ("k", "v"))  # [K, n, 64]
        x = (q[a:b].transpose(0, 1).reshape(K, -1, DIM) @ pk.transpose(1, 2) * SCALE).view(K, b - a, G, n)
        if c["window"]:
            at = (behind[a:b] + s["lengths"][a:b] - 1).div(c["frame"], rounding_mode="floor")[:, None]
            x = x.masked_fill(~((j < c["sinks"]) | (at - j // c["frame"] < c["window"]))[:, None], -math.inf)
        y = own_x[a:b].transpose(0, 1)  # [K, sequences, G, own]
        top = torch.maximum(x.amax(-1, keepdim=True), y.amax(-1, keepdim=True) if y.shape[-1] else torch.full_like(x[..., :1], -math.inf))
        x, y = (x - top).exp(), (y - top).exp()
        o = (x.view(K, -1, n) @ pv).view(K, b - a, G, DIM) + y @ v[a:b].transpose(0, 1)
        o = o / (x.sum(-1, keepdim=True) + y.sum(-1, keepdim=True))
        out[a:b] = o.transpose(0, 1).reshape(b - a, H, DIM).to(out.dtype)
    return out


# ---- one pass ---------------------------------------------------------------------------------------

def run(s):
    c = s["c"]
    if not own:
        if c["op"] == "store":
            return _store_plain(s)
        if c["op"] == "extend":
            return _store_plain(s)[0], *_load_plain(s, 0, c["context"])
        if c["op"] == "load":
            return _load_plain(s, c["first"], c["tokens"])
        if c["op"] == "step":
            q, k, v = _store_plain(s)
            return _paged_plain(s, q.transpose(0, 1)), k, v
        return _paged_plain(s, s["q"]) if c["op"] == "paged" else _prefix_plain(s)
    import paper_2509_07120_amd as bsga

    scales = {t: s[t] for t in ("k_scale", "v_scale") if t in s}
    if c["op"] == "load":
        return bsga.bsga_cache_load(s["k_cache"], s["v_cache"], s["pages"], c["tokens"], first=c["first"], dtype=_TYPES[c["dtype"]], **scales)
    if c["op"] in ("store", "extend", "step"):
        norm = c.get("norm", "rms")
        q, k, v = bsga.bsga_qk_norm_rope_e4m3(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["slots"], s["positions"],
                                              s["q_weight"], s["k_weight"], s["q_bias"], s["k_bias"], norm=None if norm == "none" else norm, eps=EPS,
                                              base=c.get("base", 10000.0), return_rows=c["op"] != "extend")
        if c["op"] == "store":
            return q, k, v
        if c["op"] == "extend":
            return q, *bsga.bsga_cache_load(s["k_cache"], s["v_cache"], s["pages"], c["context"], dtype=_TYPES[c["dtype"]], **scales)
    seen = dict(window=c["window"] or None, sinks=c["sinks"], frame=c["frame"])
    if c["op"] == "step":
        return bsga.bsga_paged_attn_e4m3(q.transpose(0, 1), s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["page_table"], s["lengths"], **seen), k, v
    if c["op"] == "paged":
        return bsga.bsga_paged_attn_e4m3(s["q"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["page_table"], s["lengths"], **seen)
    return bsga.bsga_prefix_attn(s["q"], s["k_cache"], s["v_cache"], s["page_table"], s["lengths"], s["prefix_table"], s["prefix_lengths"], s["starts"],
                                 **scales, **seen)


# ---- what run() returns, from the definitions in 64 bits --------------------------------------------

def _nearest(x):
    """The values that rows x [..., 64] (float64) are held as: 448 = 7 * 2^6 is the largest number; below 2^-6 numbers are 2^-9 apart, from
    there on eight to a power of two."""
    top = x.abs().amax(-1, keepdim=True)
    unit = torch.exp2(torch.ceil(torch.log2(top / 448.0)).clamp(-117, 119))
    unit = torch.where(top > 448.0 * unit, 2 * unit, torch.where(top <= 224.0 * unit, unit / 2, unit))  # (where a logarithm was rounded)
    unit = torch.where(top > 0, unit, torch.ones_like(unit))
    y = x / unit
    apart = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / apart) * apart * unit


def _values(s, t, pages, head, n):
    """Keys or values [n, 64] of one head of the sequence with these pages."""
    pages = pages[:-(-n // s["c"]["page"])].long()
    x = s[t + "_cache"].view(torch.uint8)[pages, head].view(torch.float8_e4m3fn) if t + "_scale" in s else s[t + "_cache"][pages, head]
    x = x.double()
    if t + "_scale" in s:
        x = torch.ldexp(x, (s[t + "_scale"][pages, head].int() - 127)[..., None])
    return x.flatten(0, 1)[:n]


def _exact_rows(s, t):
    """Rows of t [heads, tokens, 64]: normed, and turned as complex factors."""
    c, norm = s["c"], s["c"].get("norm", "rms")
    got = []
    for h in range(s[t].shape[1]):
        x = s[t][:, h].double()
        if norm != "none":
            mean = x.mean(-1, keepdim=True) if norm == "layer" else 0.0
            x = (x - mean) / torch.sqrt(((x - mean) ** 2).mean(-1, keepdim=True) + EPS) * s[t + "_weight"].double()
            if s[t + "_bias"] is not None:
                x = x + s[t + "_bias"].double()
        if s["positions"] is not None:
            axes = s["positions"].shape[1]
            width = DIM // axes
            exponent = torch.arange(0, width, 2, dtype=torch.float64, device="cuda") / width
            angle = s["positions"].double().unsqueeze(-1) / torch.pow(torch.tensor(c.get("base", 10000.0), dtype=torch.float64, device="cuda"), exponent)
            z = x.unflatten(-1, (axes, 2, width // 2))
            z = torch.complex(z[..., 0, :], z[..., 1, :]) * torch.polar(torch.ones_like(angle), angle)
            x = torch.stack([z.real, z.imag], dim=-2).flatten(-3)
        got.append(x)
    return torch.stack(got)


def _exact_attention(s, q, pages, n, front=None):
    """The query q [H, 64] of a sequence with n own tokens, behind those of `front` (keys, values of every head) where it has a prefix."""
    c = s["c"]
    G = c["heads"] // c["kv_heads"]
    out = []
    for h in range(c["kv_heads"]):
        k, v = (_values(s, t, pages, h, n) for t in ("k", "v"))
        if front is not None:
            k, v = torch.cat([front[0][h], k]), torch.cat([front[1][h], v])
        j = torch.arange(k.shape[0], device="cuda")
        if c["window"]:
            kept = (j // c["frame"] + c["window"] > (k.shape[0] - 1) // c["frame"]) | (j < c["sinks"])
            k, v = k[kept], v[kept]
        out.append(torch.softmax(q[h * G:(h + 1) * G].double() @ k.T / 8.0, -1) @ v)
    return torch.cat(out)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c["op"] == "load":
        n = c["first"] + c["tokens"]
        return tuple(torch.stack([_values(s, t, s["pages"], h, n)[c["first"]:] for h in range(c["kv_heads"])]) for t in ("k", "v"))
    if c["op"] in ("store", "extend", "step"):
        q, rows = _exact_rows(s, "q"), {"k": _nearest(_exact_rows(s, "k")), "v": _nearest(s["v"].double().transpose(0, 1))}
        if c["op"] == "store":
            return q, rows["k"], rows["v"]
        if c["op"] == "extend":
            old = c["context"] - c["tokens"]
            return q, *(torch.cat([torch.stack([_values(s, t, s["pages"], h, old) for h in range(c["kv_heads"])]), rows[t]], 1) for t in ("k", "v"))
        out = []
        for i, n in enumerate(_lengths(c)):  # the new token is the last one: behind the others, as the rows that are not in the pages yet
            G, seen = c["heads"] // c["kv_heads"], torch.arange(n, device="cuda")
            seen = (seen // c["frame"] + c["window"] > (n - 1) // c["frame"]) | (seen < c["sinks"]) if c["window"] else seen >= 0
            for h in range(c["kv_heads"]):
                k, v = (torch.cat([_values(s, t, s["page_table"][i], h, n - 1), rows[t][h, i:i + 1]])[seen] for t in ("k", "v"))
                # (the query that the attention gets is in the tensors' type)
                out.append(torch.softmax(q[h * G:(h + 1) * G, i].to(s["q"].dtype).double() @ k.T / 8.0, -1) @ v)
        return torch.cat(out).view(c["batch"], c["heads"], DIM), rows["k"], rows["v"]
    if c["op"] == "paged":
        return torch.stack([_exact_attention(s, s["q"][i], s["page_table"][i], n) for i, n in enumerate(_lengths(c))])
    lengths, out = _lengths(c), []
    scans, starts = _scenes(c)
    for i, n in enumerate(scans):
        front = [[_values(s, t, s["prefix_table"][i], h, n) for h in range(c["kv_heads"])] for t in ("k", "v")]
        out += [_exact_attention(s, s["q"][b], s["page_table"][b], lengths[b], front) for b in range(starts[i], starts[i + 1])]
    return torch.stack(out)
