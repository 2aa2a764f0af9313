"""Performance cases of the streamed attention layer's operators: norms of queries and keys with the position rotation, attention
with a sliding window and first tokens that stay visible, attention of one new token over a paged cache.

The ranges.  Tokens are whole frames of camera and register tokens (5) and a patch grid (37 x 37 or 37 x 28 patches, and smaller
ones), one to a hundred frames, or single tokens of a stream; head dimension 64; 1 to 16 query heads, as many key heads or a divisor
of them; bf16, and fp32 for short sequences.  Windows are counted in frames, or in tokens (frames of one token).  Caches hold up to
300 frames a sequence, in pages of 16 to 256 tokens or of a frame each.

Queries and keys of the attention cases are what the norm leaves: rows of length sqrt(64) times a gain.

`own` chooses the side: the plain form below (elementary torch operations in 32 bits, rounded once at the end), or this package.
"""
import math

import torch

own = False

DIM = 64
SPECIAL = 5  # camera and register tokens of a frame
SCALE = 1.0 / math.sqrt(DIM)
EPS = 1e-6
GAIN = math.sqrt(2.0)  # learned scale of the norms: logits of queries and keys that do not belong together spread by 2
_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ---- cases ------------------------------------------------------------------------------------------

def _norm(name, op, tokens, heads, kv_heads, norm, axes, dtype="bf16", base=100.0, first=0, page=0):
    """first: position of the first token where positions count along the sequence (axes = 1)."""
    return {"name": name, "op": op, "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "norm": norm, "axes": axes,
            "dtype": dtype, "base": base, "first": first, "page": page}


def _window(name, op, queries, keys, heads, kv_heads, frame, window, sinks, dtype="bf16"):
    return {"name": name, "op": op, "queries": queries, "keys": keys, "heads": heads, "kv_heads": kv_heads, "frame": frame,
            "window": window, "sinks": sinks, "dtype": dtype}


def _paged(name, batch, longest, shortest, heads, kv_heads, page, window=0, sinks=0, frame=1, dtype="bf16"):
    """window 0: every cached token is visible.  Lengths are spread between the shortest and the longest."""
    return {"name": name, "op": "paged", "batch": batch, "longest": longest, "shortest": shortest, "heads": heads,
            "kv_heads": kv_heads, "page": page, "window": window, "sinks": sinks, "frame": frame, "dtype": dtype}


def listed():
    return [
        # one decoding step of 24 streams: queries normed and rotated, keys and values straight into the cache's pages
        _norm("norm_rope_step", "norm_step", 24, 16, 4, "rms", 1, base=10000.0, first=131000, page=64),
        # the frames of a short clip between the projection and the attention: layer norm, patch rows and columns as positions
        _norm("norm_rope_8_frames", "norm", 8 * 1374, 16, 16, "layer", 2),
        # the benchmark's headline sequence
        _norm("norm_rope_100_frames", "norm", 100 * 1374, 16, 16, "layer", 2),
        # a training step on a text-like stream of odd length with shared keys, far along a sequence
        _norm("norm_rope_train", "norm_train", 20011, 16, 4, "rms", 1, base=10000.0, first=1000000),
        # one new frame that sees the last 8 frames and the first one: few rows, many keys
        _window("window_new_frame", "window", 1374, 12 * 1374, 16, 16, 1374, 8, 1374),
        # a clip sent through at once, window of 4 frames, camera and register tokens of the first one kept
        _window("window_32_frames", "window", 32 * 1374, 32 * 1374, 16, 16, 1374, 4, SPECIAL),
        # the headline's length
        _window("window_100_frames", "window", 100 * 1374, 100 * 1374, 16, 16, 1374, 4, 1374),
        # a training step: shared keys, window of tokens, odd length
        _window("window_train", "window_train", 20011, 20011, 16, 4, 1, 4096, 4),
        # single precision, as a model is first brought up: two frames, forward and backward
        _window("window_train_fp32", "window_train", 2748, 2748, 16, 16, 1374, 2, 0, dtype="fp32"),
        # one stream's query over a short cache: latency
        _paged("paged_one", 1, 8 * 1374, 8 * 1374, 16, 16, 64),
        # many streams of unequal length with shared keys, window and sinks
        _paged("paged_batch", 96, 12000, 1, 16, 4, 16, window=4096, sinks=4),
        # two long scans whole in the cache, a page to a frame
        _paged("paged_300_frames", 2, 300 * 1374, 300 * 1041, 16, 16, 1374),
    ]


_MOST_PAIRS = 137400 * 6870 * 16 // 2  # of queries, keys and heads in a drawn case
_MOST_CACHED = 300 * (1374 + 1041) * 16  # cached tokens, times key heads


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    heads = rng.choice([16, 16, 8, rng.randint(1, 16)])
    kv_heads = rng.choice([heads, rng.choice([h for h in range(1, heads + 1) if heads % h == 0])])
    rows, cols = rng.choice([(37, 37), (37, 28), (rng.randint(16, 37), rng.randint(16, 37))])
    frame = SPECIAL + rows * cols
    op = rng.choice(["norm", "norm_train", "norm_step", "window", "window", "window_train", "paged", "paged", "paged"])
    if op.startswith("norm"):
        axes = 1 if op == "norm_step" else rng.choice([1, 2])
        norm = rng.choice(["rms", "layer"])
        base = 100.0 if axes == 2 else rng.choice([10000.0, 500000.0])
        first = rng.choice([0, spread(1, 2000000)]) if axes == 1 else 0
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        tokens = spread(1, 300) if op == "norm_step" else spread(200, 20000) if dtype == "fp32" else spread(200, 100000)
        page = rng.choice([16, 64, 256, 100]) if op == "norm_step" else 0
        c = _norm("", op, tokens, heads, kv_heads, norm, axes, dtype, base, first, page)
    elif op.startswith("window"):
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        one = rng.random() < 0.4
        frame = 1 if one else frame
        keys = spread(100, 60000) if dtype == "bf16" else spread(100, 4000)
        window = spread(1, 16384) if one else rng.randint(1, 8)
        sinks = rng.choice([0, rng.randint(1, 64), frame])
        queries = keys if op == "window_train" or rng.random() < 0.5 else max(1, min(keys, spread(1, 2 * keys)))
        most = _MOST_PAIRS // (1 if dtype == "bf16" else 16) // (4 if op == "window_train" else 1)
        while _pairs(queries, keys, frame, window, sinks) * heads > most:
            window, queries = max(1, window // 2), max(1, queries * 3 // 4)
            keys = queries if op == "window_train" else keys
        c = _window("", op, queries, keys, heads, kv_heads, frame, window, sinks, dtype)
    else:
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        batch = spread(1, 128)
        longest = max(1, min(spread(1, 300000), _MOST_CACHED // (batch * kv_heads) // (1 if dtype == "bf16" else 2)))
        shortest = max(1, int(longest * rng.random()))
        windowed = rng.random() < 0.5
        one = rng.random() < 0.5
        c = _paged("", batch, longest, shortest, heads, kv_heads, rng.choice([16, 64, 256, frame]),
                   (spread(64, 16384) if one else rng.randint(1, 8)) if windowed else 0,
                   rng.choice([0, 4, frame]) if windowed else 0, frame if windowed and not one else 1, dtype)
    del c["name"]
    return c


# ---- sizes ------------------------------------------------------------------------------------------

def _visible(p, keys, frame, window, sinks):
    """(keys of the first tokens, first key of the window, end of the window) that the query at position p sees."""
    hi = min(keys, max(0, (p // frame + 1) * frame))
    lo = min(hi, max(0, (p // frame - window + 1) * frame)) if window else 0
    return min(sinks, lo), lo, hi


def _pairs(queries, keys, frame, window, sinks):
    """Queries times the keys that each sees; the queries are the last ones."""
    total, start = 0, keys - queries
    f = start // frame
    while f * frame < keys:  # the queries of a frame see the same keys
        n = min(keys, (f + 1) * frame) - max(start, f * frame)
        s, lo, hi = _visible(f * frame, keys, frame, window, sinks)
        total += n * (s + hi - lo)
        f += 1
    return total


def _lengths(c):
    if c["batch"] == 1:
        return [c["longest"]]
    step = (c["longest"] - c["shortest"]) / (c["batch"] - 1)
    return [int(round(c["shortest"] + i * step)) for i in range(c["batch"])]


def work(c):
    size = 2 if c["dtype"] == "bf16" else 4
    row = DIM * size
    if c["op"].startswith("norm"):
        qk, v = c["tokens"] * (c["heads"] + c["kv_heads"]), c["tokens"] * c["kv_heads"]
        rows = 2 * (qk + v) + (3 * qk + 2 * v if c["op"] == "norm_train" else 0)
        return {"bytes": rows * row + c["tokens"] * 4 * c["axes"], "flops": qk * DIM * (12 + (30 if c["op"] == "norm_train" else 0))}
    if c["op"].startswith("window"):
        pairs = _pairs(c["queries"], c["keys"], c["frame"], c["window"], c["sinks"]) * c["heads"]
        _, lo, _ = _visible(c["keys"] - c["queries"], c["keys"], c["frame"], c["window"], c["sinks"])
        qs, ks = c["queries"] * c["heads"], (c["keys"] - lo + min(c["sinks"], lo)) * c["kv_heads"]  # keys that any query sees
        if c["op"] == "window":
            return {"bytes": (2 * qs + 2 * ks) * row, "flops": 4 * DIM * pairs}
        # forward q k v -> o, backward do o q k v -> dq dk dv; two products forward, five backward
        return {"bytes": (2 * qs + 2 * ks + 4 * qs + 4 * ks) * row, "flops": 14 * DIM * pairs}
    seen = 0
    for n in _lengths(c):
        s, lo, hi = _visible(n - 1, n, c["frame"], c["window"], c["sinks"])
        seen += s + hi - lo
    return {"bytes": (2 * seen * c["kv_heads"] + 2 * c["batch"] * c["heads"]) * row, "flops": 4 * DIM * seen * c["heads"]}


# ---- inputs -----------------------------------------------------------------------------------------

def _positions(c, g):
    n = c["tokens"]
    if c["op"] == "norm_step":  # streams that are not equally far
        return (c["first"] + torch.randint(0, 1000, (n, 1), generator=g, device="cuda")).int()
    if c["axes"] == 1:
        return (c["first"] + torch.arange(n, device="cuda", dtype=torch.int32)).view(n, 1).contiguous()
    # patches by row and column from 1 on, camera and register tokens of each frame at 0
    at = torch.arange(n, device="cuda") % (SPECIAL + 37 * 37) - SPECIAL
    yx = torch.stack([at.div(37, rounding_mode="floor") + 1, at.remainder(37) + 1], dim=1)
    return torch.where(at[:, None] >= 0, yx, torch.zeros_like(yx)).int().contiguous()


def _rows(g, heads, n, dtype, gain=None):
    x = torch.empty((heads, n, DIM), dtype=dtype, device="cuda")
    for h in range(heads):  # a head at a time: no large temporaries
        r = torch.randn((n, DIM), generator=g, device="cuda")
        x[h] = r if gain is None else r * (gain * r.square().mean(1, keepdim=True).rsqrt())
    return x


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype = _TYPES[c["dtype"]]
    H, K = c["heads"], c["kv_heads"]
    s = {"c": c}
    if c["op"].startswith("norm"):
        n = c["tokens"]
        # what the projection gives: [tokens, heads, 64], queries, keys and values beside each other
        x = torch.empty((n, H + 2 * K, DIM), dtype=dtype, device="cuda")
        for h in range(H + 2 * K):
            x[:, h] = (0.3 + 0.2 * h) * torch.randn((n, DIM), generator=g, device="cuda") + 0.1
        s["q"], s["k"], s["v"] = x[:, :H], x[:, H:H + K], x[:, H + K:]
        for t in ("q_weight", "k_weight"):
            s[t] = (GAIN + 0.2 * torch.randn((DIM,), generator=g, device="cuda")).to(dtype)
        for t in ("q_bias", "k_bias"):
            s[t] = (0.1 * torch.randn((DIM,), generator=g, device="cuda")).to(dtype) if c["norm"] == "layer" else None
        s["positions"] = _positions(c, g)
        if c["op"] == "norm_step":
            # every stream has pages of its own; the new token goes somewhere into the last of them
            pages = 2 * n
            s["k_cache"], s["v_cache"] = (torch.randn((pages, K, c["page"], DIM), generator=g, device="cuda").to(dtype) for _ in range(2))
            page = torch.randperm(pages, generator=g, device="cuda")[:n]
            s["slots"] = (page * c["page"] + torch.randint(0, c["page"], (n,), generator=g, device="cuda")).int()
        if c["op"] == "norm_train":
            s["dq"], s["dk"], s["dv"] = (_rows(g, h, n, dtype) for h in (H, K, K))
    elif c["op"].startswith("window"):
        s["q"] = _rows(g, H, c["queries"], dtype, GAIN)
        s["k"] = _rows(g, K, c["keys"], dtype, GAIN)
        s["v"] = _rows(g, K, c["keys"], dtype)
        if c["op"] == "window_train":
            s["dout"] = _rows(g, H, c["queries"], dtype)
    else:
        lengths = _lengths(c)
        need = [-(-n // c["page"]) for n in lengths]
        pages = sum(need)
        order = torch.randperm(pages, generator=g, device="cuda").int()
        table = torch.full((c["batch"], max(need)), -1, dtype=torch.int32, device="cuda")
        at = 0
        for i, m in enumerate(need):
            table[i, :m] = order[at:at + m]
            at += m
        s["page_table"], s["lengths"] = table, torch.tensor(lengths, dtype=torch.int32).cuda()
        s["k_cache"], s["v_cache"] = (_pages(g, pages, K, c["page"], dtype, gain) for gain in (GAIN, None))
        s["q"] = _rows(g, H, c["batch"], dtype, GAIN).transpose(0, 1)  # as the norm with the rotation leaves it
    return s


def _pages(g, pages, heads, page, dtype, gain):
    x = torch.empty((pages * heads * page, DIM), dtype=dtype, device="cuda")
    for part in x.split(1 << 22):
        r = torch.randn((part.shape[0], DIM), generator=g, device="cuda")
        part.copy_(r if gain is None else r * (gain * r.square().mean(1, keepdim=True).rsqrt()))
    return x.view(pages, heads, page, DIM)


# ---- the plain forms --------------------------------------------------------------------------------

def _turns(positions, base):
    """cos and sin of every token's angles, [tokens, 1, axes, 64 / axes / 2]: angles in 64 bits, far positions lose theirs in 32."""
    axes = positions.shape[1]
    half = DIM // axes // 2
    freq = base ** (-torch.arange(half, dtype=torch.float64, device=positions.device) / half)
    angle = positions.double()[:, None, :, None] * freq
    return angle.cos().float(), angle.sin().float()


def _rotate(x, cos, sin):
    n, heads, _ = x.shape
    a, b = x.view(n, heads, cos.shape[2], 2, -1).unbind(3)
    return torch.stack([a * cos - b * sin, b * cos + a * sin], dim=3).view(n, heads, DIM)


def _normed(x, weight, bias, norm):
    """The normed rows, what they are before the weight, and the factor of each row."""
    x = x.float()
    if norm == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
    hat = x * r
    return hat * weight.float() + (0 if bias is None else bias.float()), hat, r


def _norm_plain(s):
    c = s["c"]
    cos, sin = _turns(s["positions"], c["base"])
    out = [_rotate(_normed(s[t], s[t + "_weight"], s[t + "_bias"], c["norm"])[0], cos, sin) for t in ("q", "k")]
    q, k = (x.transpose(0, 1).to(s["q"].dtype).contiguous() for x in out)
    if c["op"] == "norm_step":
        page, row = s["slots"].long() // c["page"], s["slots"].long() % c["page"]
        s["k_cache"][page, :, row] = k.transpose(0, 1)
        s["v_cache"][page, :, row] = s["v"]
        return q, s["k_cache"], s["v_cache"]
    v = s["v"].transpose(0, 1).contiguous()
    return (q, k, v) + (_norm_back_plain(s, cos, sin) if c["op"] == "norm_train" else ())


def _norm_back_plain(s, cos, sin):
    c = s["c"]
    dx, dw = [], []
    for t in ("q", "k"):
        w = s[t + "_weight"].float()
        _, hat, r = _normed(s[t], s[t + "_weight"], s[t + "_bias"], c["norm"])
        g = _rotate(s["d" + t].float().transpose(0, 1), cos, -sin)
        dw.append((g * hat).sum((0, 1), dtype=torch.float64).float())
        if c["norm"] == "layer":
            dw.append(g.sum((0, 1), dtype=torch.float64).float())
        g = g * w
        d = g - hat * (g * hat).mean(-1, keepdim=True)
        if c["norm"] == "layer":
            d = d - g.mean(-1, keepdim=True)
        dx.append((d * r).to(s[t].dtype))
    return tuple(dx) + (s["dv"].transpose(0, 1).contiguous(),) + tuple(dw)


def _window_plain(s):
    """A stretch of queries at a time, against the keys that any of them sees."""
    c = s["c"]
    q, k, v = s["q"], s["k"].float(), s["v"].float()
    H, N, M = c["heads"], c["queries"], c["keys"]
    K, G = c["kv_heads"], c["heads"] // c["kv_heads"]
    train = c["op"] == "window_train"
    out = torch.empty_like(q)
    if train:
        dq, dk, dv = torch.empty_like(q), torch.zeros_like(k), torch.zeros_like(v)
    start, step = M - N, 2048
    for at in range(0, N, step):
        end = min(N, at + step)
        n = end - at
        _, lo, _ = _visible(start + at, M, c["frame"], c["window"], c["sinks"])
        first, _, hi = _visible(start + end - 1, M, c["frame"], c["window"], c["sinks"])
        first = min(first, lo)
        j = torch.cat([torch.arange(first, device="cuda"), torch.arange(lo, hi, device="cuda")])
        ks, vs = k[:, j], v[:, j]
        of_j = j.div(c["frame"], rounding_mode="floor")
        of_i = torch.arange(start + at, start + end, device="cuda").div(c["frame"], rounding_mode="floor")[:, None]
        seen = (of_j <= of_i) & ((of_j > of_i - c["window"]) | (j < c["sinks"]))
        qs = q[:, at:end].float().reshape(K, G * n, DIM)
        x = (qs @ ks.transpose(1, 2) * SCALE).view(K, G, n, -1).masked_fill(~seen, -math.inf)
        p = (x - x.amax(-1, keepdim=True)).exp()
        p = (p / p.sum(-1, keepdim=True)).view(K, G * n, -1)
        del x
        o = p @ vs
        out[:, at:end] = o.view(H, n, DIM).to(q.dtype)
        if train:
            do = s["dout"][:, at:end].float().reshape(K, G * n, DIM)
            dv.index_add_(1, j, p.transpose(1, 2) @ do)
            ds = p * (do @ vs.transpose(1, 2) - (do * o).sum(-1, keepdim=True))
            dq[:, at:end] = (ds @ ks * SCALE).view(H, n, DIM).to(q.dtype)
            dk.index_add_(1, j, ds.transpose(1, 2) @ qs * SCALE)
    return (out, dq, dk.to(q.dtype), dv.to(q.dtype)) if train else out


def _paged_plain(s):
    """Every sequence padded to the one that sees most."""
    c = s["c"]
    B, H, K = c["batch"], c["heads"], c["kv_heads"]
    seen = [_visible(n - 1, n, c["frame"], c["window"], c["sinks"]) for n in _lengths(c)]
    first, lo, hi = (torch.tensor(x, device="cuda")[:, None] for x in zip(*seen))
    i = torch.arange(max(a + b - l for a, l, b in seen), device="cuda")
    j = torch.where(i < first, i, i - first + lo)
    valid = j < hi
    j = torch.where(valid, j, 0)
    page, row = s["page_table"].gather(1, j // c["page"]).long(), j % c["page"]
    k, v = (s[t].transpose(1, 2)[page, row].float().transpose(1, 2) for t in ("k_cache", "v_cache"))  # [B, K, keys, 64]
    x = s["q"].float().reshape(B, K, H // K, DIM) @ k.transpose(2, 3) * SCALE
    x = x.masked_fill(~valid[:, None, None], -math.inf)
    p = (x - x.amax(-1, keepdim=True)).exp()
    o = p @ v / p.sum(-1, keepdim=True)
    return o.view(B, H, DIM).to(s["q"].dtype)


# ---- one pass ---------------------------------------------------------------------------------------

def run(s):
    c = s["c"]
    if not own:
        return _norm_plain(s) if c["op"].startswith("norm") else _window_plain(s) if c["op"].startswith("window") else _paged_plain(s)
    import paper_2509_07120_amd as bsga

    if c["op"].startswith("norm"):
        what = dict(q_bias=s["q_bias"], k_bias=s["k_bias"], norm=c["norm"], eps=EPS, base=c["base"])
        args = (s["q"], s["k"], s["positions"], s["q_weight"], s["k_weight"])
        if c["op"] == "norm_step":
            q = bsga.bsga_qk_norm_rope(*args, v=s["v"], k_cache=s["k_cache"], v_cache=s["v_cache"], slots=s["slots"], **what)[0]
            return q, s["k_cache"], s["v_cache"]
        out = tuple(bsga.bsga_qk_norm_rope(*args, v=s["v"], **what))
        if c["op"] == "norm":
            return out
        dq, dk, dv, dqw, dkw, dqb, dkb = bsga.bsga_qk_norm_rope_bwd(s["dq"], s["dk"], *args, dv=s["dv"], **what)
        return out + (dq, dk, dv) + ((dqw, dqb, dkw, dkb) if c["norm"] == "layer" else (dqw, dkw))
    if c["op"].startswith("window"):
        seen = dict(window=c["window"], sinks=c["sinks"], frame=c["frame"])
        if c["op"] == "window":
            return bsga.bsga_window_attn(s["q"], s["k"], s["v"], **seen)
        out, lse = bsga.bsga_window_attn(s["q"], s["k"], s["v"], return_lse=True, **seen)
        return (out,) + tuple(bsga.bsga_window_attn_bwd(s["dout"], s["q"], s["k"], s["v"], out, lse, **seen))
    return bsga.bsga_paged_attn(s["q"], s["k_cache"], s["v_cache"], s["page_table"], s["lengths"], window=c["window"] or None,
                                sinks=c["sinks"], frame=c["frame"])


# ---- what run() returns, from the definitions in 64 bits --------------------------------------------

def _exact_norm(s):
    c = s["c"]
    n, axes = c["tokens"], c["axes"]
    width = DIM // axes
    # the rotation of a token as complex factors, one for each pair
    exponent = torch.arange(0, width, 2, dtype=torch.float64, device="cuda") / width
    angle = s["positions"].double().unsqueeze(-1) / torch.pow(torch.tensor(c["base"], dtype=torch.float64, device="cuda"), exponent)
    factor = torch.polar(torch.ones_like(angle), angle).unsqueeze(0)  # [1, tokens, axes, width / 2]

    def turn(x, f):  # [heads, tokens, 64]
        z = x.unflatten(-1, (axes, 2, width // 2))
        z = torch.complex(z[..., 0, :], z[..., 1, :]) * f
        return torch.stack([z.real, z.imag], dim=-2).flatten(-3)

    def one(t, h):
        x, w = s[t][:, h:h + 1].transpose(0, 1).double(), s[t + "_weight"].double()
        b = s[t + "_bias"].double() if s[t + "_bias"] is not None else torch.zeros_like(w)
        mean = x.mean(-1, keepdim=True) if c["norm"] == "layer" else torch.zeros_like(x[..., :1])
        dev = torch.sqrt(((x - mean) ** 2).mean(-1, keepdim=True) + EPS)
        return x, w, b, mean, dev

    out, back, sums = {}, {}, []
    for t, heads in (("q", c["heads"]), ("k", c["kv_heads"])):
        ys, dxs = [], []
        dw, db = torch.zeros(DIM, dtype=torch.float64, device="cuda"), torch.zeros(DIM, dtype=torch.float64, device="cuda")
        for h in range(heads):
            x, w, b, mean, dev = one(t, h)
            ys.append(turn((x - mean) / dev * w + b, factor))
            if c["op"] == "norm_train":
                g = turn(s["d" + t][h:h + 1].double(), factor.conj())
                unit = (x - mean) / dev
                dw += (g * unit).sum((0, 1))
                db += g.sum((0, 1))
                gw = g * w
                m = gw.mean(-1, keepdim=True) if c["norm"] == "layer" else 0.0
                dxs.append((gw - m - unit * (gw * unit).mean(-1, keepdim=True)) / dev)
        out[t] = torch.cat(ys)
        if dxs:
            back[t] = torch.cat(dxs).transpose(0, 1)
            sums += [dw, db] if c["norm"] == "layer" else [dw]
    v = s["v"].double()
    if c["op"] == "norm_step":
        caches = []
        for name, new in (("k_cache", out["k"].transpose(0, 1)), ("v_cache", v)):
            cache = s[name].double().transpose(1, 2).flatten(0, 1)
            cache[s["slots"].long()] = new
            caches.append(cache.unflatten(0, (-1, c["page"])).transpose(1, 2).contiguous())
        return (out["q"], *caches)
    got = (out["q"], out["k"], v.transpose(0, 1))
    return got if c["op"] == "norm" else got + (back["q"], back["k"], s["dv"].double().transpose(0, 1), *sums)


def _exact_attention(q, k, v, seen, dout=None):
    """q [g, n, 64] of a key head's queries against k, v [m, 64]; seen [n, m]."""
    weight = torch.where(seen, torch.exp((q @ k.T) / 8.0), torch.zeros((), dtype=torch.float64, device="cuda"))
    weight = weight / weight.sum(-1, keepdim=True)
    o = weight @ v
    if dout is None:
        return o
    dweight = dout @ v.T
    dlogit = weight * (dweight - (weight * dweight).sum(-1, keepdim=True)) / 8.0
    flat = lambda x: x.flatten(0, 1)  # noqa: E731
    return o, dlogit @ k, flat(dlogit).T @ flat(q), flat(weight).T @ flat(dout)


def _exact_window(s):
    c = s["c"]
    if work(c)["flops"] > 2.0e13:  # over about 20 seconds
        return None
    N, M, F = c["queries"], c["keys"], c["frame"]
    G = c["heads"] // c["kv_heads"]
    train = c["op"] == "window_train"
    shape = (c["heads"], N, DIM)
    out = torch.zeros(shape, dtype=torch.float64, device="cuda")
    dq = torch.zeros(shape, dtype=torch.float64, device="cuda") if train else None
    dk, dv = (torch.zeros((c["kv_heads"], M, DIM), dtype=torch.float64, device="cuda") for _ in range(2)) if train else (None, None)
    key = torch.arange(M, device="cuda")
    for rows in torch.arange(N, device="cuda").split(4096):
        own_frame = (rows + (M - N))[:, None] // F
        mask = (key // F <= own_frame) & ((key // F + c["window"] > own_frame) | (key < c["sinks"]))
        cols = mask.any(0).nonzero().flatten()
        mask = mask[:, cols]
        r = slice(int(rows[0]), int(rows[-1]) + 1)
        for h in range(c["kv_heads"]):
            group = slice(h * G, (h + 1) * G)
            args = (s["q"][group, r].double(), s["k"][h, cols].double(), s["v"][h, cols].double(), mask)
            if not train:
                out[group, r] = _exact_attention(*args)
            else:
                out[group, r], dq[group, r], a, b = _exact_attention(*args, s["dout"][group, r].double())
                dk[h, cols] += a
                dv[h, cols] += b
    return (out, dq, dk, dv) if train else out


def _exact_paged(s):
    c = s["c"]
    G = c["heads"] // c["kv_heads"]
    out = []
    for i, n in enumerate(s["lengths"].tolist()):
        pages = s["page_table"][i, :-(-n // c["page"])].long()
        j = torch.arange(n, device="cuda")
        seen = j >= (((n - 1) // c["frame"]) - c["window"] + 1) * c["frame"] if c["window"] else j >= 0
        seen = (seen | (j < c["sinks"]))[None]
        heads = []
        for h in range(c["kv_heads"]):
            k, v = (s[t][pages, h].flatten(0, 1)[:n].double() for t in ("k_cache", "v_cache"))
            heads.append(_exact_attention(s["q"][i, h * G:(h + 1) * G, None].double(), k, v, seen)[:, 0])
        out.append(torch.cat(heads))
    return torch.stack(out)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    return _exact_norm(s) if c["op"].startswith("norm") else _exact_window(s) if c["op"].startswith("window") else _exact_paged(s)
