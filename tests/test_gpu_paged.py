"""Attention of one new token over a paged cache against the definition in float64; bounds as in test_gpu_window.py (its check())."""
import math

import pytest
import torch

from tests.test_gpu_window import TYPES, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_2509_07120_amd as pkg
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return pkg


def draw(lengths, H, K, page, dtype, seed=0, spare=3, gain=1.0):
    """(q [B, H, 64] view, caches, table, lengths): pages in random order, rows that no sequence has and table entries past the end hold rubbish."""
    g = torch.Generator(device="cuda").manual_seed(seed + sum(lengths) + page + H)
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + spare
    kc, vc = (torch.full((pages, K, page, 64), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    table = torch.full((len(lengths), max(need) + 2), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    table[:, -1] = -7
    order = torch.randperm(pages, generator=g, device="cuda").int()
    at, seqs = 0, []
    for b, n in enumerate(lengths):
        table[b, :need[b]] = order[at:at + need[b]]
        k, v = ((s * torch.randn((K, n, 64), generator=g, device="cuda")).to(dtype) for s in (gain, 1.0))
        for i in range(need[b]):
            p, part = int(order[at + i]), slice(i * page, min((i + 1) * page, n))
            kc[p, :, :part.stop - part.start], vc[p, :, :part.stop - part.start] = k[:, part], v[:, part]
        at += need[b]
        seqs.append((k, v))
    q = (gain * torch.randn((H, len(lengths), 64), generator=g, device="cuda")).to(dtype).transpose(0, 1)
    return q, kc, vc, table, torch.tensor(lengths, dtype=torch.int32).cuda(), seqs


def visible(n, window, sinks, frame):
    j = torch.arange(n, device="cuda")
    if window is None:
        return j >= 0
    return ((n - 1) // frame - j // frame < window) | (j < sinks)


CASES = [  # lengths, heads, key heads, page, window, sinks, frame, type
    ([1], 1, 1, 16, None, 0, 1, "bf16"),
    ([0, 1, 2, 31, 32, 33, 0, 129], 4, 2, 16, None, 0, 1, "bf16"),
    ([700, 5, 64, 1], 16, 1, 64, 100, 4, 1, "bf16"),
    ([5000], 16, 16, 64, None, 0, 1, "bf16"),
    ([2000, 1999, 1], 40, 2, 37, None, 0, 1, "bf16"),           # 20 heads to a key head: two workgroups
    ([4500, 100], 2, 1, 1, None, 0, 1, "bf16"),                 # a page to a token
    ([3000, 2500, 7], 3, 3, 1374, 2, 5, 1374, "bf16"),
    ([4000, 3999], 8, 4, 100, 3, 130, 50, "bf16"),
    ([1000, 90], 4, 4, 16, 64, 1000, 1, "bf16"),                # more sinks than there are keys before the window
    ([300] * 70, 8, 1, 16, None, 0, 1, "bf16"),
    ([1, 0, 17, 400], 4, 2, 16, None, 0, 1, "fp32"),
    ([1500, 33], 17, 1, 24, 200, 3, 1, "fp32"),
    ([5000], 2, 2, 256, None, 0, 1, "fp32"),
]


@pytest.mark.parametrize("lengths,H,K,page,window,sinks,frame,dtype", CASES)
def test_against_the_definition(B, lengths, H, K, page, window, sinks, frame, dtype):
    q, kc, vc, table, n, seqs = draw(lengths, H, K, page, TYPES[dtype])
    what = dict(window=window, sinks=sinks, frame=frame)
    o, lse = B.bsga_paged_attn(q, kc, vc, table, n, return_lse=True, **what)
    assert o.shape == (len(lengths), H, 64) and o.is_contiguous()
    for b, (k, v) in enumerate(seqs):
        if lengths[b] == 0:
            assert bool((o[b] == 0).all()) and bool((lse[b] == -math.inf).all())
            continue
        check(o[b][:, None], lse[b][:, None], q[b][:, None], k, v, visible(lengths[b], window, sinks, frame)[None])
    assert torch.equal(B.bsga_paged_attn(q.contiguous(), kc, vc, table, n, **what), o)
    # no room past the longest sequence: other splits, the same result up to the order of sums
    tight = table[:, :max(1, max(-(-x // page) for x in lengths))].contiguous()
    o2 = B.bsga_paged_attn(q, kc, vc, tight, n, **what)
    for b, (k, v) in enumerate(seqs):
        if lengths[b] > 0:
            check(o2[b][:, None], None, q[b][:, None], k, v, visible(lengths[b], window, sinks, frame)[None])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("gain", [0.0, 6.0, 12.0])
def test_logits_of_any_size(B, dtype, gain):
    q, kc, vc, table, n, seqs = draw([900, 40], 4, 2, 32, TYPES[dtype], gain=gain)
    o, lse = B.bsga_paged_attn(q, kc, vc, table, n, return_lse=True)
    for b, (k, v) in enumerate(seqs):
        check(o[b][:, None], lse[b][:, None], q[b][:, None], k, v, torch.ones((1, k.shape[1]), dtype=torch.bool, device="cuda"))


def test_the_rows_it_sees_decide(B):
    """Keys that are not numbers: where they are seen the result is not one either, elsewhere nothing changes."""
    q, kc, vc, table, n, seqs = draw([500, 500], 4, 2, 16, torch.bfloat16)
    clean = B.bsga_paged_attn(q, kc, vc, table, n, window=100, sinks=2)
    hidden, seen = int(table[0, 300 // 16]), int(table[1, 450 // 16])
    kc[hidden], vc[hidden] = float("nan"), float("inf")
    kc[seen, 0, 450 % 16, 5] = float("nan")
    o = B.bsga_paged_attn(q, kc, vc, table, n, window=100, sinks=2)
    assert torch.equal(o[0], clean[0]) and torch.equal(o[1, 2:], clean[1, 2:]) and bool(o[1, :2].isnan().all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [1, 37, 500])
def test_an_infinite_last_value(B, dtype, n):
    """It has a weight above zero: its number becomes infinite, by its sign, and the others stay as they were."""
    q, kc, vc, table, lengths, _ = draw([n], 4, 2, 16, TYPES[dtype])
    clean = B.bsga_paged_attn(q, kc, vc, table, lengths)
    page, row = int(table[0, (n - 1) // 16]), (n - 1) % 16
    vc[page, 0, row, 5], vc[page, 1, row, 40] = math.inf, -math.inf
    o = B.bsga_paged_attn(q, kc, vc, table, lengths)
    assert bool((o[0, :2, 5] == math.inf).all()) and bool((o[0, 2:, 40] == -math.inf).all())
    o[0, :2, 5], o[0, 2:, 40] = clean[0, :2, 5], clean[0, 2:, 40]
    assert torch.equal(o, clean)


def test_lengths_and_pages_that_do_not_exist(B):
    """Lengths beyond the table and below zero are clamped, and so are page numbers: nothing outside the cache is read."""
    q, kc, vc, table, n, seqs = draw([64, 64, 64], 2, 1, 16, torch.bfloat16, spare=0)
    table = table[:, :4].contiguous()
    want = B.bsga_paged_attn(q, kc, vc, table, n)
    n2 = n.clone()
    n2[0], n2[1] = 2 ** 31 - 1, -5
    o = B.bsga_paged_attn(q, kc, vc, table, n2)
    assert torch.equal(o[0], want[0]) and torch.equal(o[2], want[2]) and bool((o[1] == 0).all())
    bad = table.clone()
    bad[0, 1], bad[0, 2] = -2 ** 31, 2 ** 31 - 1
    ok = table.clone()
    ok[0, 1], ok[0, 2] = 0, kc.shape[0] - 1
    assert torch.equal(B.bsga_paged_attn(q, kc, vc, bad, n), B.bsga_paged_attn(q, kc, vc, ok, n))


def test_nothing_to_do(B):
    q, kc, vc, table, n, _ = draw([64, 64], 2, 1, 16, torch.bfloat16)
    assert B.bsga_paged_attn(q[:0], kc, vc, table[:0], n[:0]).shape == (0, 2, 64)
    o, lse = B.bsga_paged_attn(q, kc[:0], vc[:0], table, n, return_lse=True)
    assert bool((o == 0).all()) and bool((lse == -math.inf).all())
    assert bool((B.bsga_paged_attn(q, kc, vc, table[:, :0].contiguous(), n) == 0).all())


def test_a_cache_past_32_bits(B):
    """Pages whose bytes lie past 2^32 and rows past 2^31 numbers: 40,000 pages of 16 heads x 64 tokens."""
    pages, K, page = 40000, 16, 64
    kc, vc = (torch.empty((pages, K, page, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q, ks, vs, table, n, seqs = draw([200, 130], 16, K, page, torch.bfloat16)
    at = torch.randperm(300, generator=torch.Generator().manual_seed(3))[:ks.shape[0]].cuda() + pages - 300
    kc[at], vc[at] = ks, vs
    moved = table.clone()
    inside = (table >= 0) & (table < ks.shape[0])
    moved[inside] = at.int()[table[inside].long()]
    assert torch.equal(B.bsga_paged_attn(q, kc, vc, moved, n), B.bsga_paged_attn(q, ks, vs, table, n))


def test_another_stream_and_a_graph(B):
    q, kc, vc, table, n, _ = draw([700, 5, 300], 8, 2, 16, torch.bfloat16)
    want = B.bsga_paged_attn(q, kc, vc, table, n)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = B.bsga_paged_attn(q, kc, vc, table, n)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = B.bsga_paged_attn(q, kc, vc, table, n)
    for i in range(4):
        q.mul_(1.0 + 0.25 * i)
        n.sub_(1)  # lengths are read when the graph runs
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, B.bsga_paged_attn(q, kc, vc, table, n))
