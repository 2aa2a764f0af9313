"""Attention of one new token for sequences that share their first tokens, against the definition in float64 on the tokens of both one after the other; bounds as
in test_gpu_window.py (its check())."""
import math

import pytest
import torch

from tests.test_gpu_e4m3 import cached, queries, values
from tests.test_gpu_window import TYPES, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_2509_07120_amd as pkg
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return pkg


def draw(scans, starts, lengths, H, K, page, cache, dtype, seed=0, gain=1.0):
    """(arguments of bsga_prefix_attn, scales, keys and values [K, n, 64] of every sequence, the prefix's first)."""
    kc, vc, ks, vs, table, seqs = cached(list(lengths) + list(scans), K, page, seed, gain=gain)
    B = len(lengths)
    scales = dict(k_scale=ks, v_scale=vs)
    if cache != "e4m3":
        kc, vc = (values(c, s).to(TYPES[cache]) for c, s in ((kc, ks), (vc, vs)))
        scales = {}
    whole = []
    for b in range(B):
        of = [g for g in range(len(scans)) if starts[g] <= b < starts[g + 1]]
        whole.append([torch.cat([seqs[B + of[0]][t], seqs[b][t]], 1) if of else seqs[b][t] for t in range(2)])
    ints = [torch.tensor(x, dtype=torch.int32).cuda() for x in (lengths, scans, starts)]
    args = [queries(B, H, TYPES[dtype], seed, gain=1.0), kc, vc, table[:B].contiguous(), ints[0], table[B:].contiguous(), ints[1], ints[2]]
    return args, scales, whole


def visible(n, window, sinks, frame):
    j = torch.arange(n, device="cuda")
    return j >= 0 if window is None else ((n - 1) // frame - j // frame < window) | (j < sinks)


def check_all(o, lse, q, whole, window=None, sinks=0, frame=1):
    for b, (k, v) in enumerate(whole):
        n = k.shape[1]
        if n == 0:
            assert bool((o[b] == 0).all()) and (lse is None or bool((lse[b] == -math.inf).all()))
            continue
        check(o[b][:, None], None if lse is None else lse[b][:, None], q[b][:, None], k, v, visible(n, window, sinks, frame)[None])


CASES = [  # prefixes, starts, own lengths, heads, key heads, page, window, sinks, frame, cache, type
    ([1], [0, 1], [0], 1, 1, 16, None, 0, 1, "bf16", "bf16"),
    ([100], [0, 3], [5, 0, 64], 4, 2, 16, None, 0, 1, "bf16", "bf16"),
    ([700], [0, 9], [1, 2, 3, 100, 0, 40, 33, 32, 31], 16, 16, 64, None, 0, 1, "e4m3", "bf16"),
    ([3001], [0, 40], list(range(40)), 8, 2, 64, None, 0, 1, "bf16", "bf16"),
    ([5000], [0, 70], [7] * 70, 16, 4, 37, None, 0, 1, "e4m3", "bf16"),             # 280 queries to a key head
    ([333, 1, 0, 900], [1, 4, 4, 6, 9], [3, 10, 0, 5, 80, 1, 0, 2, 9, 600, 0], 6, 2, 16, None, 0, 1, "bf16", "bf16"),   # sequences without a prefix at both ends
    ([333, 1, 0, 900], [1, 4, 4, 6, 9], [3, 10, 0, 5, 80, 1, 0, 2, 9, 600, 0], 6, 2, 16, None, 0, 1, "e4m3", "fp32"),
    ([2000], [0, 20], [1, 50, 100, 150, 300] * 4, 4, 4, 100, 200, 3, 1, "bf16", "bf16"),   # windows that begin in the prefix, or behind it
    ([2000], [0, 20], [1, 50, 100, 150, 300] * 4, 8, 1, 100, 200, 3, 1, "e4m3", "bf16"),
    ([4122, 2748], [0, 5, 12], [1, 1374, 1375, 3000, 20, 7, 1, 2, 3, 4, 5, 2000], 4, 2, 1374, 2, 1374, 1374, "bf16", "bf16"),
    ([4122, 2748], [0, 5, 12], [1, 1374, 1375, 3000, 20, 7, 1, 2, 3, 4, 5, 2000], 4, 2, 1374, 2, 5, 1374, "e4m3", "bf16"),
    ([300], [0, 6], [1, 400, 3, 700, 5, 6], 3, 1, 16, 64, 1000, 1, "bf16", "bf16"),      # more sinks than there are prefix tokens
    ([900], [0, 7], [3, 0, 17, 1, 90, 5, 2], 5, 5, 24, None, 0, 1, "fp32", "fp32"),
    ([900], [0, 7], [3, 1, 17, 1, 90, 5, 2], 10, 2, 24, 100, 2, 1, "fp32", "fp32"),
    ([6000], [0, 2], [100, 3], 40, 2, 1, None, 0, 1, "bf16", "bf16"),                    # a page to a token, 20 heads to a key head
    ([50] * 70, list(range(0, 141, 2)), [4] * 140, 2, 1, 16, None, 0, 1, "bf16", "bf16"),  # more prefixes than lanes
    ([137], [0, 130], [1] * 130, 1, 1, 16, None, 0, 1, "bf16", "bf16"),                  # one query a sequence
]


@pytest.mark.parametrize("scans,starts,lengths,H,K,page,window,sinks,frame,cache,dtype", CASES)
def test_against_the_definition(B, scans, starts, lengths, H, K, page, window, sinks, frame, cache, dtype):
    args, scales, whole = draw(scans, starts, lengths, H, K, page, cache, dtype)
    what = dict(window=window, sinks=sinks, frame=frame)
    o, lse = B.bsga_prefix_attn(*args, **scales, return_lse=True, **what)
    assert o.shape == (len(lengths), H, 64) and o.is_contiguous()
    check_all(o, lse, args[0], whole, window, sinks, frame)
    assert torch.equal(B.bsga_prefix_attn(args[0].contiguous(), *args[1:], **scales, **what), o)


@pytest.mark.parametrize("cache,dtype", [("bf16", "bf16"), ("e4m3", "bf16"), ("e4m3", "fp32"), ("fp32", "fp32")])
def test_no_prefix_is_attention_over_pages(B, cache, dtype):
    args, scales, whole = draw([], [0], [300, 0, 41], 4, 2, 16, cache, dtype)
    o, lse = B.bsga_prefix_attn(*args, **scales, return_lse=True)
    check_all(o, lse, args[0], whole)
    # prefixes that have no tokens, or no sequences
    args, scales, whole = draw([0, 50], [0, 3, 3], [300, 0, 41], 4, 2, 16, cache, dtype)
    o, lse = B.bsga_prefix_attn(*args, **scales, return_lse=True)
    check_all(o, lse, args[0], whole)


@pytest.mark.parametrize("cache,dtype", [("bf16", "bf16"), ("e4m3", "bf16"), ("fp32", "fp32")])
@pytest.mark.parametrize("gain", [2.0 ** -20, 4.0, 16.0])
def test_logits_of_any_size(B, cache, dtype, gain):
    args, scales, whole = draw([900], [0, 3], [40, 1, 0], 4, 2, 32, cache, dtype, gain=gain)
    o, lse = B.bsga_prefix_attn(*args, **scales, return_lse=True)
    check_all(o, lse, args[0], whole)


@pytest.mark.parametrize("cache,dtype", [("bf16", "bf16"), ("e4m3", "bf16"), ("fp32", "fp32")])
@pytest.mark.parametrize("scale", [2.0 ** -100, 2.0 ** -20, 3.0])
@pytest.mark.parametrize("sequences", [4, 30, 100])
def test_scales_of_logits(B, cache, dtype, scale, sequences):
    args, scales, whole = draw([500], [0, sequences], [i % 7 for i in range(sequences)], 2, 2, 32, cache, dtype)
    o, lse = B.bsga_prefix_attn(*args, **scales, return_lse=True, softmax_scale=scale)
    for b, (k, v) in enumerate(whole):
        check(o[b][:, None], lse[b][:, None], args[0][b][:, None], k, v, torch.ones((1, k.shape[1]), dtype=torch.bool, device="cuda"), scale)


@pytest.mark.parametrize("sequences", [4, 30, 100])
@pytest.mark.parametrize("byte", [63, 207])
def test_values_of_any_size(B, byte, sequences):
    """Rows whose values have the smallest and the largest scale that is written, beside others: what each stands for."""
    args, scales, whole = draw([700], [0, sequences], [i % 5 for i in range(sequences)], 2, 2, 16, "e4m3", "bf16")
    vs = scales["v_scale"]
    vs.masked_fill_(vs != 255, byte)
    some = torch.rand(vs.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)) < 0.2
    mixed = torch.where(some & (vs != 255), byte + (8 if byte < 127 else -8), vs).to(torch.uint8)
    scales["v_scale"] = mixed
    o = B.bsga_prefix_attn(*args, **scales)
    kc, vc, table, n, pt = args[1], args[2], args[3], args[4].tolist(), args[5]
    for b in range(sequences):
        rows = [torch.cat([values(c[t].view(torch.uint8), s[t]).transpose(0, 1).reshape(2, -1, 64)[:, :m] for t, m in
                           ((pt[0, :44].long(), 700), (table[b, :-(-n[b] // 16)].long(), n[b]))], 1) for c, s in ((kc, scales["k_scale"]), (vc, mixed))]
        f = 2.0 ** (127 - byte)
        check((o[b].double() * f).float().bfloat16()[:, None], None, args[0][b][:, None], rows[0], rows[1] * f,
              torch.ones((1, rows[0].shape[1]), dtype=torch.bool, device="cuda"))


def test_sums_that_grow(B):
    """Logits that rise along the prefix, far beyond the first ones, and many keys of nearly one logit: the reference follows."""
    for cache in ("bf16", "e4m3"):
        for sequences in (4, 30, 100):
            args, scales, whole = draw([9000], [0, sequences], [1] * sequences, 1, 1, 64, cache, "bf16")
            pages = args[5][0, :-(-9000 // 64)].long()
            up = torch.arange(pages.numel(), device="cuda")
            if cache == "e4m3":  # a power of two every few pages, and values of small scales
                scales["k_scale"][pages] = (112 + up // 14).clamp(max=130).to(torch.uint8)[:, None, None].expand_as(scales["k_scale"][pages])
                scales["v_scale"][pages] = 90
                k, v = (values(c[pages].view(torch.uint8), s[pages]).transpose(0, 1).reshape(1, -1, 64)[:, :9000] for c, s in
                        ((args[1], scales["k_scale"]), (args[2], scales["v_scale"])))
                f = 2.0 ** 37
            else:
                args[1][pages] *= (0.05 * up)[:, None, None, None].to(args[1].dtype)
                k, v = (c[pages].transpose(0, 1).reshape(1, -1, 64)[:, :9000] for c in (args[1], args[2]))
                f = 1.0
            args[4].zero_()
            o, lse = B.bsga_prefix_attn(*args, **scales, return_lse=True)
            for b in range(sequences):
                check((o[b].double() * f).float().bfloat16()[:, None], lse[b][:, None], args[0][b][:, None], k, v * f,
                      torch.ones((1, 9000), dtype=torch.bool, device="cuda"))


@pytest.mark.parametrize("queries_of_a_head", [3, 60, 300])
@pytest.mark.parametrize("cache,dtype", [("bf16", "bf16"), ("e4m3", "bf16"), ("fp32", "fp32")])
def test_the_rows_it_sees_decide(B, cache, dtype, queries_of_a_head):
    """Values that are not numbers, in prefix tokens that some sequences see and others do not: those that see them become NaN or infinite where they are, the others stay as
    they were up to the order of sums."""
    n = queries_of_a_head
    lengths = [1 + i * 60 // n for i in range(n)]
    args, scales, whole = draw([400], [0, n], lengths, 2, 2, 16, cache, dtype)
    what = dict(window=100, sinks=2)
    clean = B.bsga_prefix_attn(*args, **scales, **what)
    check_all(clean, None, args[0], whole, 100, 2)
    j = 330  # seen by queries at positions below 430: the first half of them
    page, row = int(args[5][0, j // 16]), j % 16
    kc, vc = args[1], args[2]
    if cache == "e4m3":
        kc.view(torch.uint8)[page, 0, row], vc.view(torch.uint8)[page, 1, row, 7] = 0x7f, 0xff
    else:
        kc[page, 0, row], vc[page, 1, row, 7] = math.nan, math.inf
    hidden = int(args[5][0, 200 // 16])  # seen by nobody
    if cache == "e4m3":
        kc.view(torch.uint8)[hidden], vc.view(torch.uint8)[hidden] = 0x7f, 0x7f
    else:
        kc[hidden], vc[hidden] = math.nan, math.inf
    o = B.bsga_prefix_attn(*args, **scales, **what)
    sees = torch.tensor([400 + m - 1 - j < 100 for m in lengths], device="cuda")
    assert bool(sees.any()) and not bool(sees.all())
    assert bool(o[sees, 0].isnan().all()) and bool((o[sees, 1, 7].isnan() if cache == "e4m3" else o[sees, 1, 7] == math.inf).all())
    rest = torch.ones(64, dtype=torch.bool, device="cuda")
    rest[7] = False
    for b in range(n):  # the same definition, with the bad number of its own head left out of what is compared
        k, v = (x.clone() for x in whole[b])
        if bool(sees[b]):
            k, v, got, q = k[1:], v[1:].clone(), o[b, 1:], args[0][b, 1:]
            v[:, j, 7] = 0
            got = torch.where(rest, got, 0)
            v = torch.where(rest, v, 0)
            check(got[:, None], None, q[:, None], k, v, visible(k.shape[1], 100, 2, 1)[None])
        else:
            check(o[b][:, None], None, args[0][b][:, None], k, v, visible(k.shape[1], 100, 2, 1)[None])


def test_numbers_that_do_not_fit(B):
    """Lengths beyond the tables, below zero, page numbers and starts that do not exist: nothing outside the tensors is read."""
    args, scales, whole = draw([64], [0, 3], [64, 64, 64], 2, 1, 16, "bf16", "bf16")
    args[3], args[5] = args[3][:, :4].contiguous(), args[5][:, :4].contiguous()
    want = B.bsga_prefix_attn(*args)
    more = [a.clone() for a in args]
    more[4][0], more[6][0], more[7][1] = 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1
    assert torch.equal(B.bsga_prefix_attn(*more), want)
    more[7][0] = -2 ** 31
    assert torch.equal(B.bsga_prefix_attn(*more), want)
    more[3][1, 1], more[5][0, 2] = -2 ** 31, 2 ** 31 - 1
    args[3][1, 1], args[5][0, 2] = 0, args[1].shape[0] - 1
    assert torch.equal(B.bsga_prefix_attn(*more), B.bsga_prefix_attn(*args))
    none = [a.clone() for a in args]
    none[4].fill_(-3)
    none[6].fill_(-3)
    assert bool((B.bsga_prefix_attn(*none) == 0).all())


def test_nothing_to_do(B):
    args, _, _ = draw([64], [0, 2], [64, 64], 2, 1, 16, "bf16", "bf16")
    q, kc, vc, table, n, pt, pn, st = args
    assert B.bsga_prefix_attn(q[:0], kc, vc, table[:0], n[:0], pt, pn, st).shape == (0, 2, 64)
    o, lse = B.bsga_prefix_attn(q, kc[:0], vc[:0], table, n, pt, pn, st, return_lse=True)
    assert bool((o == 0).all()) and bool((lse == -math.inf).all())
    empty = B.bsga_prefix_attn(q, kc, vc, table[:, :0].contiguous(), n, pt, pn, st)
    assert torch.equal(empty, B.bsga_prefix_attn(q, kc, vc, table, n * 0, pt, pn, st))


def test_another_stream_and_a_graph(B):
    args, scales, _ = draw([700, 90], [0, 5, 8], [10, 0, 30, 500, 7, 3, 2, 1], 8, 2, 16, "e4m3", "bf16")
    call = lambda: B.bsga_prefix_attn(*args, **scales, window=600, sinks=3)  # noqa: E731
    want = call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for i in range(4):
        args[0].mul_(1.0 + 0.25 * i)
        args[4].sub_(1)
        args[6].sub_(5)
        args[7][1].sub_(1)  # lengths and who has which prefix are read when the graph runs
        graph.replay()
        torch.cuda.synchronize()
        assert bool(got.isfinite().all()) and torch.equal(got.clone(), call())
