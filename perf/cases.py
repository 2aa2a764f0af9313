"""Performance cases: the work that a user of this package has it do, through its public entry points.

The ranges.  Tokens are whole frames of camera and register tokens (5) and a patch grid (37 x 37 at
518 x 518 px, 37 x 28 at 518 x 392 px, other grids for other image shapes), 1 to 300 frames; head
dimension 64; 1 to 16 heads (16 for a whole layer, fewer for one rank of a head-sharded one); blocks of
64 and 128 tokens, and query blocks of 128 with key blocks of 64; bf16, and fp32 for short sequences;
thresholds tau from 0.8 to 0.95 and top-k sparsities rho from 0.5 to 0.9.  The values are the
correspondence-structured activations of workload/synthetic.py, drawn on the GPU.

These paths are inference only: none of them has a backward pass.
"""
import math

import torch

import paper_2509_07120_amd as bsga

SPECIAL = 5  # camera and register tokens of a frame
DIM = 64
SCALE = 1.0 / math.sqrt(DIM)


def _case(name, op, frames, rows, cols, heads, block, dtype="bf16", latents=8000, visibility=0.3, tau=0.9, rho=1.0):
    return {"name": name, "op": op, "frames": frames, "rows": rows, "cols": cols, "heads": heads, "block": block,
            "dtype": dtype, "latents": latents, "visibility": visibility, "tau": tau, "rho": rho}


def listed():
    return [
        # one 518 x 518 image: the shortest sequence a model sends through its global attention
        _case("layer_1_frame", "layer", 1, 37, 37, 16, 64, latents=2000, visibility=1.0),
        # an image pair in single precision, as a model is first brought up
        _case("layer_2_frames_fp32", "layer", 2, 37, 37, 16, 64, dtype="fp32", latents=2000, visibility=1.0),
        # a handful of images, small blocks
        _case("layer_8_frames", "layer", 8, 37, 37, 16, 64, latents=2000, visibility=1.0),
        # a short clip, large blocks
        _case("layer_32_frames", "layer", 32, 37, 37, 16, 128),
        # the benchmark's headline: 100 frames, 137,400 tokens
        _case("layer_100_frames", "layer", 100, 37, 37, 16, 128),
        # a long scan at the sparsity that makes such lengths worth while, non-square images
        _case("layer_300_frames_topk", "layer", 300, 37, 28, 16, 128, latents=20000, visibility=0.2, tau=0.0, rho=0.75),
        # special tokens kept dense and apart from the patch tokens, which is how a real model has to run it
        _case("special_100_frames_topk", "special", 100, 37, 37, 16, 128, tau=0.0, rho=0.75),
        # the layers that stay dense
        _case("dense_32_frames", "dense", 32, 37, 37, 16, 128),
        # query blocks of 128 on key blocks of 64, high sparsity
        _case("asym_100_frames_topk", "asym", 100, 37, 37, 16, 128, tau=0.0, rho=0.9),
        # the block map alone, for a program that keeps it for several layers or looks at it
        _case("select_300_frames", "select", 300, 37, 28, 16, 128, latents=20000, visibility=0.2),
        # one of eight ranks of a head-sharded layer: two heads, lists of its own, row sums wanted for a merge
        _case("attention_2_heads", "attention", 32, 37, 37, 2, 128, tau=0.0, rho=0.75),
        # a whole transformer block (norms, projections, MLP) around the layer
        _case("block_8_frames", "block", 8, 37, 37, 16, 128, latents=2000, visibility=1.0, tau=0.0, rho=0.75),
    ]


def draw(rng):
    op = rng.choice(["layer", "layer", "layer", "layer_fp32", "special", "dense", "asym", "select", "attention", "block"])

    def frames(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    rows, cols = rng.choice([(37, 37), (37, 28), (rng.randint(20, 37), rng.randint(20, 37)), (28, 37)])
    heads = rng.choice([16, 16, rng.randint(1, 16)])
    tau, rho = rng.choice([(round(rng.uniform(0.8, 0.95), 3), 1.0), (0.0, round(rng.uniform(0.5, 0.9), 3))])
    few = dict(latents=2000, visibility=1.0)
    if op == "layer":
        if rng.random() < 0.5:
            return _drawn(op, frames(1, 16), rows, cols, heads, 64, tau=tau, rho=rho, **few)
        return _drawn(op, frames(8, 100), rows, cols, heads, 128, tau=tau, rho=rho)
    if op == "layer_fp32":
        return _drawn("layer", frames(1, 4), rows, cols, heads, 64, dtype="fp32", tau=tau, rho=rho, **few)
    if op == "special":
        return _drawn(op, frames(2, 100), rows, cols, heads, 128, tau=tau, rho=rho)
    if op == "dense":
        return _drawn(op, frames(1, 60), rows, cols, heads, 128)
    if op == "asym":
        return _drawn(op, frames(8, 100), rows, cols, heads, 128, tau=tau, rho=rho)
    if op == "select":
        return _drawn(op, frames(2, 300), rows, cols, heads, rng.choice([64, 128]) if rows * cols < 1000 else 128, tau=tau, rho=rho)
    if op == "attention":
        return _drawn(op, frames(4, 64), rows, cols, heads, 128, tau=0.0, rho=round(rng.uniform(0.5, 0.9), 3))
    return _drawn(op, frames(2, 24), rows, cols, 16, 128, tau=tau, rho=rho, **few)


def _drawn(*a, **kw):
    c = _case("", *a, **kw)
    del c["name"]
    return c


# ---- sizes ------------------------------------------------------------------------------------------

def _tokens(c):
    return c["frames"] * (SPECIAL + c["rows"] * c["cols"])


def _ceil(a, b):
    return -(-a // b)


def _blocks(n, block, n_first=None):
    """[(start, length)] of the blocks of a sequence whose parts [0, n_first) and [n_first, n) are blocked apart."""
    n_first = n if n_first is None else n_first
    spans = [(s, min(block, e - s)) for b, e in ((0, n_first), (n_first, n)) for s in range(b, e, block)]
    return spans


def _key_block(c):
    return 64 if c["op"] == "asym" else c["block"]


def _special_mask(c):
    one = torch.zeros(SPECIAL + c["rows"] * c["cols"], dtype=torch.bool)
    one[:SPECIAL] = True
    return one.repeat(c["frames"])


# ---- inputs -----------------------------------------------------------------------------------------

def _activations(c, seed, tensors=("q", "k", "v")):
    """[heads, tokens, 64] each: patch tokens that share a latent are correspondences (see workload/synthetic.py)."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    F, P, H, L = c["frames"], c["rows"] * c["cols"], c["heads"], c["latents"]
    dtype = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    out = {t: torch.empty((H, _tokens(c), DIM), dtype=dtype, device="cuda") for t in tensors}
    for h in range(H):
        z = torch.nn.functional.normalize(torch.randn((L, DIM), generator=g, device="cuda"), dim=1)
        if c["visibility"] >= 1.0:
            latent = torch.randint(0, L, (F, P), generator=g, device="cuda")
        else:
            seen = torch.rand((F, L), generator=g, device="cuda") < c["visibility"]
            ids = seen.to(torch.uint8).argsort(dim=1, descending=True)  # the visible latents of a frame first
            count = seen.sum(dim=1, keepdim=True).clamp(min=1)
            latent = ids.gather(1, (torch.rand((F, P), generator=g, device="cuda") * count).long().clamp(max=L - 1))
        for t in tensors:
            x = torch.randn((F, SPECIAL + P, DIM), generator=g, device="cuda")
            if t != "v":
                x[:, SPECIAL:] = 4.0 * z[latent] + 0.5 * x[:, SPECIAL:]
            out[t][h] = x.view(-1, DIM).to(dtype)
    return [out[t] for t in tensors]


def _lists(c, seed):
    """Kept lists of unequal length, half of each around the row's own place and half anywhere."""
    g = torch.Generator(device="cuda").manual_seed(int(seed) + 1)
    H, nb = c["heads"], _ceil(_tokens(c), c["block"])
    at = torch.arange(nb, device="cuda")
    near = 1.0 - (at[:, None] - at[None, :]).abs() / nb
    score = torch.where(torch.rand((H, nb, nb), generator=g, device="cuda") < 0.5, near, torch.rand((H, nb, nb), generator=g, device="cuda"))
    kept = (1.0 - c["rho"]) * nb * (0.6 + 0.8 * torch.rand((H, nb), generator=g, device="cuda"))
    cnt = kept.long().clamp(1, nb)
    rank = score.argsort(dim=2, descending=True).argsort(dim=2)
    idx = torch.where(rank < cnt[:, :, None], at, nb).sort(dim=2).values
    return torch.where(idx < nb, idx, 0).to(torch.int32).contiguous(), cnt.to(torch.int32).contiguous()


def prepare(case, seed):
    c = case
    s = {"case": c}
    if c["op"] == "block":
        # weights stay with the program; the activations of a scene are new
        s["block"] = bsga.GlobalAttentionBlock(d_model=DIM * c["heads"], heads=c["heads"], block=c["block"], tau=c["tau"],
                                               rho=c["rho"], special=_special_mask(c), seed=0)
        g = torch.Generator(device="cuda").manual_seed(int(seed))
        # tokens of one place in the scene look alike: a few shared directions beside each token's own
        base = torch.randn((c["latents"], DIM * c["heads"]), generator=g, device="cuda")
        pick = torch.randint(0, c["latents"], (_tokens(c),), generator=g, device="cuda")
        x = base[pick] + torch.randn((_tokens(c), DIM * c["heads"]), generator=g, device="cuda")
        s["x"] = x.to(torch.bfloat16)
        return s
    if c["op"] == "select":
        q, k = _activations(c, seed, ("q", "k"))
        nb = _ceil(_tokens(c), c["block"])
        mean = [torch.stack([torch.nn.functional.pad(x[h].double(), (0, 0, 0, nb * c["block"] - _tokens(c))).view(nb, -1, DIM).sum(1)
                             for h in range(c["heads"])]) for x in (q, k)]
        size = torch.full((nb, 1), float(c["block"]), dtype=torch.float64, device="cuda")
        size[-1] = _tokens(c) - (nb - 1) * c["block"]
        s["pools"] = [m / size for m in mean]
        H = c["heads"]
        s["workspace"] = torch.empty(bsga.bsga_select_workspace_bytes(H, nb, nb), dtype=torch.uint8, device="cuda")
        s["out"] = (torch.zeros((H, nb, (nb + 31) // 32), dtype=torch.int32, device="cuda"),
                    torch.zeros((H, nb, nb), dtype=torch.int32, device="cuda"),  # entries past a row's count stay 0
                    torch.zeros((H, nb), dtype=torch.int32, device="cuda"))
        return s
    s["qkv"] = _activations(c, seed)
    if c["op"] == "attention":
        s["lists"] = _lists(c, seed)
    if c["op"] == "special":
        s["plan"] = bsga.SpecialTokenPlan(_special_mask(c), c["block"], "cuda")
    return s


# ---- one pass ---------------------------------------------------------------------------------------

def run(state):
    c, op = state["case"], state["case"]["op"]
    if op == "block":
        return state["block"](state["x"])
    if op == "select":
        return bsga.bsga_select_blocks(*state["pools"], c["tau"], c["rho"], workspace=state["workspace"], out=state["out"])
    q, k, v = state["qkv"]
    if op == "dense":
        return bsga.bsga_dense_attn(q, k, v)
    if op == "attention":
        return bsga.bsga_sparse_attn(q, k, v, c["block"], *state["lists"], return_lse=True)
    # entries of an index list past the row's count are not written, so the lists come as bits and counts
    if op == "special":
        o, _, cnt, bits = bsga.sparse_global_attention_special(q, k, v, state["plan"], c["tau"], c["rho"])
    elif op == "asym":
        q_pool, k_pool = bsga.bsga_pool(q, c["block"]), bsga.bsga_pool(k, _key_block(c))
        bits, idx, cnt = bsga.bsga_select_blocks(q_pool, k_pool, c["tau"], c["rho"])
        o = bsga.bsga_sparse_attn(q, k, v, c["block"], idx, cnt, block_k=_key_block(c))
    else:
        o, _, cnt, bits = bsga.sparse_global_attention(q, k, v, c["block"], c["tau"], c["rho"])
    return o, cnt, bits


# ---- what a pass cannot do without --------------------------------------------------------------------

def _kept(c, nbk):
    """Share of the key blocks a row keeps: about tau where the block distribution is flat, or the top-k floor."""
    return max(min(c["tau"], 1.0), max(1, math.floor(nbk * (1.0 - c["rho"]))) / nbk)


def work(case):
    c = case
    n, H = _tokens(c), c["heads"]
    size = 2 if c["dtype"] == "bf16" else 4
    nbq, nbk = _ceil(n, c["block"]), _ceil(n, _key_block(c))
    tensor = H * n * DIM * size
    scores = 2.0 * H * nbq * nbk * DIM
    maps = 4.0 * H * nbq * (nbk / 32 + 1)  # bits and counts
    attend = 4.0 * H * n * n * DIM
    if c["op"] == "select":
        kept = _kept(c, nbk)
        return {"bytes": 8.0 * H * (nbq + nbk) * DIM + maps + 4.0 * H * nbq * nbk * kept, "flops": scores}
    if c["op"] == "dense":
        return {"bytes": 4.0 * tensor, "flops": attend}
    if c["op"] == "attention":
        kept = 1.0 - c["rho"]
        return {"bytes": 4.0 * tensor + 4.0 * H * n + 4.0 * H * nbq * (nbk * kept + 1), "flops": attend * kept}
    if c["op"] == "block":
        d = H * DIM
        return {"bytes": 2.0 * (2 * n * d + 12 * d * d), "flops": 2.0 * n * 12 * d * d + attend * _kept(c, nbk) + scores}
    return {"bytes": 4.0 * tensor + maps, "flops": attend * _kept(c, nbk) + scores}


def tolerance(case):
    if case["op"] == "select":
        return "exact"
    if case["dtype"] == "fp32":
        return {"rel": 1e-5}
    return {"rel": 1e-2}


# ---- the same in 64 bits ------------------------------------------------------------------------------

def _pool64(x, spans):
    x = x.double()
    return torch.stack([x[s:s + m].mean(0) for s, m in spans])


def _map64(q, k, spans_q, spans_k, tau, rho, dense_q, dense_k):
    """One head's block map [nbq, nbk]; blocks from dense_q / dense_k on are kept whole and not ranked."""
    logits = SCALE * _pool64(q, spans_q) @ _pool64(k, spans_k)[:dense_k].T
    p = torch.softmax(logits, dim=1)
    order = p.sort(dim=1, descending=True, stable=True)
    need = (order.values.cumsum(1) < tau).sum(1) + 1 if tau > 0 else torch.ones(len(spans_q), dtype=torch.long, device=q.device)
    need = need.clamp(min=max(1, math.floor(dense_k * (1.0 - rho))), max=dense_k)
    keep = torch.ones((len(spans_q), len(spans_k)), dtype=torch.bool, device=q.device)
    ranked = torch.arange(dense_k, device=q.device)[None] < need[:, None]
    keep[:, :dense_k] = torch.zeros_like(p, dtype=torch.bool).scatter(1, order.indices, ranked)
    keep[dense_q:] = True
    return keep


def _attend64(q, k, v, spans_q, spans_k, keep):
    """One head: softmax attention of each query block over the key blocks that `keep` (or None: all) names."""
    n = k.shape[0]
    q, k, v = q.double() * SCALE, k.double(), v.double()
    o, lse = torch.empty_like(q), torch.empty(n, dtype=torch.float64, device=q.device)
    member = torch.empty(n, dtype=torch.long, device=q.device)
    for j, (s, m) in enumerate(spans_k):
        member[s:s + m] = j
    piece = 1024  # the product with V is summed over pieces of the keys, so that it fills the card
    for i, (s, m) in enumerate(spans_q):
        at = torch.arange(n, device=q.device) if keep is None else keep[i][member].nonzero().flatten()
        more = -at.numel() % piece
        kk, vv = (torch.nn.functional.pad(x[at], (0, 0, 0, more)) for x in (k, v))
        a = q[s:s + m] @ kk.T
        a[:, at.numel():] = -math.inf
        top = a.amax(1, keepdim=True)
        a = a.sub_(top).exp_()
        total = a.sum(1, keepdim=True)
        parts = a.view(m, -1, piece).transpose(0, 1) @ vv.view(-1, piece, DIM)
        o[s:s + m] = parts.sum(0) / total
        lse[s:s + m] = (top + total.log()).flatten()
    return o, lse


def exact(case, seed):
    c = case
    if c["op"] == "select":
        return None  # bits, indices and counts: compared as they are
    if work(c)["flops"] > 9e13:
        return None
    n, tau, rho = _tokens(c), c["tau"], c["rho"]
    state = prepare(c, seed)
    if c["op"] == "block":
        return _block64(c, state)
    n_first, perm = n, None
    if c["op"] == "special":
        special = _special_mask(c)
        perm = torch.cat([(~special).nonzero().flatten(), special.nonzero().flatten()]).cuda()
        n_first = int((~special).sum())
    spans_q, spans_k = _blocks(n, c["block"], n_first), _blocks(n, _key_block(c), n_first)
    dense_q, dense_k = _ceil(n_first, c["block"]), _ceil(n_first, _key_block(c))
    out, sums = [], []
    for h in range(c["heads"]):
        q, k, v = (x[h] if perm is None else x[h][perm] for x in state["qkv"])
        if c["op"] == "dense":
            keep = None
        elif c["op"] == "attention":
            idx, cnt = (x[h].long() for x in state["lists"])
            listed_ = torch.arange(len(spans_k), device="cuda")[None] < cnt[:, None]
            keep = torch.zeros_like(listed_, dtype=torch.int32).scatter_add_(1, idx, listed_.int()) > 0
        else:
            keep = _map64(q, k, spans_q, spans_k, tau, rho, dense_q, dense_k)
        o, lse = _attend64(q, k, v, spans_q, spans_k, keep)
        if perm is not None:
            o = torch.empty_like(o).index_copy_(0, perm, o)
        out.append(o)
        sums.append(lse)
    o = torch.stack(out)
    if c["op"] == "dense":
        return o
    if c["op"] == "attention":
        return o, torch.stack(sums)
    return o, None, None


def _block64(c, state):
    m, x, n = state["block"], state["x"].double(), _tokens(c)
    D, H = x.shape[1], c["heads"]

    def norm(y, ln):
        return torch.nn.functional.layer_norm(y, (D,), ln.weight.double(), ln.bias.double(), ln.eps)

    def linear(y, w, b):
        return y @ w.double().T + b.double()

    special = _special_mask(c)
    perm = torch.cat([(~special).nonzero().flatten(), special.nonzero().flatten()]).cuda()
    n_first = int((~special).sum())
    spans = _blocks(n, c["block"], n_first)
    nb1 = _ceil(n_first, c["block"])
    qkv = linear(norm(x, m.ln1)[perm], m.w_qkv, m.b_qkv).view(n, 3, H, DIM).permute(1, 2, 0, 3)
    heads = []
    for h in range(H):
        q, k, v = qkv[0][h], qkv[1][h], qkv[2][h]
        keep = _map64(q, k, spans, spans, c["tau"], c["rho"], nb1, nb1)
        heads.append(_attend64(q, k, v, spans, spans, keep)[0])
    o = torch.stack(heads, dim=1).reshape(n, D)
    y = linear(o, m.w_out, m.b_out)
    x = x + torch.empty_like(y).index_copy_(0, perm, y)
    mid = torch.nn.functional.gelu(linear(norm(x, m.ln2), m.w_fc1, m.b_fc1))
    return x + linear(mid, m.w_fc2, m.b_fc2)
