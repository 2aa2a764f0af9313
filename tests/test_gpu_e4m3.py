"""The cache in 8 bits: rows on their way into it, back out of it, and attention over it, against the definition in float64.

Bounds.  A row that is neither normed nor turned is quantised exactly as the definition says, bit for bit.  Otherwise the row that is quantised is off by the norm's and
the rotation's 2^-19 of the terms that are added up (test_gpu_norm_rope.py), and the number by half a step more, 2^-4 of it or 2^(s - 10); what a number stands for
has no error of its own, in bf16 or fp32.  Attention over such rows: as test_gpu_window.py (its check()) on what they stand for; a value's scale is a power of two and
changes no rounding."""
import math

import pytest
import torch

from tests.test_gpu_norm_rope import _forward
from tests.test_gpu_window import TYPES, check

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def B():
    import paper_2509_07120_amd as pkg
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return pkg


def exponents(x):
    """s of every row of x [..., 64], by the finite numbers."""
    x = x.double()
    top = torch.where(x.isfinite(), x.abs(), 0).amax(-1)
    m, e = torch.frexp(top)  # 448 = 0.875 * 2^9
    return torch.where(top > 0, e - 9 + (m > 0.875), -64).clamp(-64, 80)


def quantised(x):
    """(values in float64, s) that the rows are held as."""
    s = exponents(x)
    x = x.double()
    unit = torch.exp2(s.double())[..., None]
    y = x / unit
    y = torch.where(x.isfinite(), y.clamp(-448, 448), math.nan)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * unit, s


def values(codes, scale):
    """What [..., 64] numbers and [...] exponent bytes stand for, float64."""
    return torch.ldexp(codes.view(torch.uint8).cpu().view(E4M3).double(), (scale.cpu().int() - 127)[..., None]).to(codes.device)


def empty_cache(pages, K, page):
    """Caches and scales full of a byte that is never written with such a scale."""
    kc, vc = (torch.full((pages, K, page, 64), 0x55, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2))
    return kc, vc, *(torch.full((pages, K, page), 3, dtype=torch.uint8, device="cuda") for _ in range(2))


def cached(lengths, K, page, seed=0, spare=3, gain=1.0):
    """(caches, scales, table, values of every sequence [K, n, 64]): pages in random order; rows that no sequence has hold NaN, table entries past the end rubbish."""
    g = torch.Generator(device="cuda").manual_seed(seed + sum(lengths) + page)
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + spare
    x = [torch.randint(0, 0x7f, (pages, K, page, 64), generator=g, device="cuda").to(torch.uint8) for _ in range(2)]  # finite ones up to 448
    for t in x:
        t.add_(128 * torch.randint(0, 2, t.shape, generator=g, device="cuda").to(torch.uint8))
    # (numbers of e4m3 at random are spread over their exponents; a scale of 2^-7 makes the largest of 64 about 3)
    scale = [torch.randint(119, 122, (pages, K, page), generator=g, device="cuda").to(torch.uint8) for _ in range(2)]
    if gain != 1.0:
        scale[0] = (scale[0].int() + int(math.log2(gain))).to(torch.uint8)
    table = torch.full((len(lengths), max(need + [0]) + 2), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    table[:, -1] = -7
    order = torch.randperm(pages, generator=g, device="cuda").int()
    at, seqs, used = 0, [], torch.zeros((pages, page), dtype=torch.bool, device="cuda")
    for b, n in enumerate(lengths):
        table[b, :need[b]] = order[at:at + need[b]]
        of = order[at:at + need[b]].long()
        at += need[b]
        rows = torch.arange(need[b] * page, device="cuda").view(need[b], page) < n
        used[of] = rows
        seqs.append([values(x[t][of], scale[t][of]).transpose(0, 1).reshape(K, -1, 64)[:, :n] for t in range(2)])
    for t in range(2):
        x[t].masked_fill_(~used[:, None, :, None], 0x7f)
        scale[t].masked_fill_(~used[:, None], 255)
    return x[0].view(E4M3), x[1].view(E4M3), scale[0], scale[1], table, seqs


ROWS = [("bf16", 1, 1, 16), ("bf16", 77, 2, 16), ("fp32", 300, 3, 100), ("bf16", 1031, 16, 64), ("fp32", 65, 1, 1)]


@pytest.mark.parametrize("dtype,N,K,page", ROWS)
def test_rows_as_they_are(B, dtype, N, K, page):
    """Bit for bit, with numbers of every size, rows of zeros, infinities and NaN; other rows of the cache stay as they were."""
    g = torch.Generator(device="cuda").manual_seed(N)
    pages = -(-N // page) + 2
    size = torch.exp2(torch.randint(-140, 120, (N, 2 * K, 1), generator=g, device="cuda").double())
    x = (torch.randn((N, 2 * K, 64), generator=g, device="cuda").double() * size).float()
    x[0, 0] = 0.0
    if N > 20:
        x[3, 0, 5], x[3, 0, 6], x[4, K, 7] = math.inf, -math.inf, math.nan
        x[5] = math.inf
        x[6, 0] = torch.finfo(torch.float32).max / 2  # within the largest scale's clamp, and rounds
        x[7, 0, :8] = torch.tensor([448.0, 449.0, 432.0, 464.0, 1.0625, 1.1875, 2.0 ** -9, 1.5 * 2.0 ** -10])  # next to a scale's border, ties
        x[7, 0, 8:] = 0.0
        x[8, 0] = x[7, 0]
        x[8, 0, 1] = 0.0
    x = x.to(TYPES[dtype])
    if N > 20:
        x[9, 0], x[9, K] = torch.finfo(x.dtype).max, torch.finfo(x.dtype).tiny
    k, v = x[:, :K], x[:, K:]
    cache = empty_cache(pages, K, page)
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:N].int()
    if N > 20:
        slots[10], slots[11], slots[12] = -1, pages * page, 2 ** 31 - 1
    q, kr, vr = B.bsga_qk_norm_rope_e4m3(None, k, v, *cache, slots, norm=None, return_rows=True)
    assert q is None
    inside = (slots >= 0) & (slots < pages * page)
    for t, rows, got, codes, scale in (("k", k, kr, cache[0], cache[2]), ("v", v, vr, cache[1], cache[3])):
        want, s = quantised(rows.cpu())
        assert torch.equal(got.transpose(0, 1).double().cpu().nan_to_num(7e300), want.nan_to_num(7e300)), t
        at, row = slots[inside].long() // page, slots[inside].long() % page
        assert torch.equal(values(codes[at, :, row], scale[at, :, row]).cpu().nan_to_num(7e300), want[inside.cpu()].nan_to_num(7e300)), t
        assert torch.equal(scale[at, :, row].cpu().int(), (s + 127)[inside.cpu()].int())
        left = torch.ones((pages, page), dtype=torch.bool, device="cuda")
        left[at, row] = False
        assert bool((scale.transpose(1, 2)[left] == 3).all()) and bool((codes.view(torch.uint8).transpose(1, 2)[left] == 0x55).all())
    # without rows: the same cache
    again = empty_cache(pages, K, page)
    assert B.bsga_qk_norm_rope_e4m3(None, k, v, *again, slots, norm=None) == (None, None, None)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(cache, again))


@pytest.mark.parametrize("dtype,N,H,K,norm,axes,base", [("bf16", 1, 1, 1, "rms", 1, 1e4), ("bf16", 333, 6, 2, "layer", 2, 100.0), ("fp32", 130, 4, 4, "rms", 1, 5e5),
                                                        ("fp32", 97, 3, 1, "layer", 1, 1e4), ("bf16", 2011, 16, 16, "layer", 2, 100.0), ("bf16", 64, 2, 1, None, 2, 50.0)])
def test_normed_and_turned(B, dtype, N, H, K, norm, axes, base):
    t = TYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(N + H)
    x = (torch.randn((N, H + 2 * K, 64), generator=g, device="cuda") * 2 + 0.5).to(t)
    q, k, v = x[:, :H], x[:, H:H + K], x[:, H + K:]
    w = [None if norm is None else (1 + 0.3 * torch.randn(64, generator=g, device="cuda")).to(t) for _ in range(2)]
    b = [(0.2 * torch.randn(64, generator=g, device="cuda")).to(t) if norm == "layer" else None for _ in range(2)]
    positions = torch.randint(-1000, 2000000 if axes == 1 else 40, (N, axes), generator=g, device="cuda").int()
    what = dict(q_weight=w[0], k_weight=w[1], q_bias=b[0], k_bias=b[1], norm=norm, base=base)
    pages = -(-N // 24)
    cache = empty_cache(pages, K, 24)
    slots = torch.randperm(pages * 24, generator=g, device="cuda")[:N].int()
    q_out, kr, vr = B.bsga_qk_norm_rope_e4m3(q, k, v, *cache, slots, positions, return_rows=True, **what)
    assert torch.equal(q_out, B.bsga_qk_norm_rope(q, k, positions, **what)[0])
    assert torch.equal(vr.transpose(0, 1).double().cpu(), quantised(v.cpu())[0])
    at, row = slots.long() // 24, slots.long() % 24
    got = values(cache[0][at, :, row], cache[2][at, :, row])
    assert torch.equal(got, kr.transpose(0, 1).double())
    assert torch.equal(values(cache[1][at, :, row], cache[3][at, :, row]), vr.transpose(0, 1).double())
    want, slack = (y.transpose(0, 1) for y in _forward(k.double(), w[1], b[1], positions, norm, 1e-6, base))
    s = cache[2][at, :, row].double() - 127
    top, off = want.abs().amax(-1), slack.amax(-1)
    assert bool((top - off <= 448 * torch.exp2(s)).all()) and bool((top + off > 224 * torch.exp2(s)).all())  # the least scale
    half = torch.maximum(2.0 ** -4 * (want.abs() + slack), torch.exp2(s - 10)[..., None])
    assert bool(((got - want).abs() <= half + slack).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("norm,axes,base,mean", [("rms", 1, 1e4, 0.0), ("layer", 2, 100.0, 0.0), ("layer", 1, 5e5, 30.0), ("rms", 0, 1e4, 0.0), (None, 2, 100.0, 0.0)])
def test_keys_are_the_nearest_numbers(B, dtype, norm, axes, base, mean):
    """No key goes to the other side of a border between two numbers: two million of them, bit for bit what the definition in float64 makes (which is itself off
    by 2^-40 at positions up to 4096, so that one number in 2^37 may differ)."""
    g = torch.Generator(device="cuda").manual_seed(int(base) + axes)
    N, K, page = 8192, 4, 64
    k = (torch.randn((N, K, 64), generator=g, device="cuda") * torch.exp2(torch.randint(-3, 4, (N, K, 1), generator=g, device="cuda")) + mean).to(TYPES[dtype])
    w = (1 + 0.2 * torch.randn(64, generator=g, device="cuda")).to(TYPES[dtype]) if norm else None
    bias = (0.3 * torch.randn(64, generator=g, device="cuda")).to(TYPES[dtype]) if norm == "layer" else None
    positions = torch.randint(0, 4097, (N, axes), generator=g, device="cuda").int() if axes else None
    slots = torch.randperm(N, generator=g, device="cuda").int()
    kc, vc, ks, vs = empty_cache(N // page, K, page)
    rows = B.bsga_qk_norm_rope_e4m3(None, k, k, kc, vc, ks, vs, slots, positions, k_weight=w, k_bias=bias, norm=norm, base=base, return_rows=True)[1]
    x = k.double()
    if norm:
        x = x - x.mean(-1, keepdim=True) if norm == "layer" else x
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w.double()
        x = x if bias is None else x + bias.double()
    if axes:
        half = 32 // axes
        angle = positions.double()[:, None, :, None] * base ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
        a, b = x.view(N, K, axes, 2, half).unbind(3)
        x = torch.stack([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], 3).view(N, K, 64)
    want, s = quantised(x)
    page_of, row_of = slots.long() // page, slots.long() % page
    assert torch.equal(ks[page_of, :, row_of].int(), (s + 127).int())
    assert torch.equal(values(kc, ks)[page_of, :, row_of], want)
    assert torch.equal(rows.transpose(0, 1).double(), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,K,page,first,count", [(1, 1, 16, 0, 1), (100, 3, 16, 7, 60), (1400, 2, 1374, 1370, 30), (500, 16, 64, 0, 500), (70, 4, 1, 3, 64), (200, 1, 24, 200, 0)])
def test_tokens_read_back(B, n, K, page, first, count, dtype):
    t = TYPES[dtype]
    kc, vc, ks, vs, table, [(k, v)] = cached([n], K, page)
    got = B.bsga_cache_load(kc, vc, table[0, :-2].contiguous(), count, first, ks, vs, dtype=t)
    for x, want in zip(got, (k, v)):
        assert x.shape == (K, count, 64) and torch.equal(x, want[:, first:first + count].to(t))
    # into a larger tensor, and from a cache of the tensors' own type
    wide = torch.full((2, K, count + 9, 64), 5.0, dtype=t, device="cuda")
    into = tuple(w[:, 4:4 + count] for w in wide)
    assert B.bsga_cache_load(kc, vc, table[0, :-2].contiguous(), count, first, ks, vs, out=into)[0] is into[0]
    assert all(torch.equal(a, b) for a, b in zip(into, got)) and bool((wide[:, :, :4] == 5).all()) and bool((wide[:, :, 4 + count:] == 5).all())
    plain = [values(c, s).to(t) for c, s in ((kc, ks), (vc, vs))]
    assert all(torch.equal(a, b) for a, b in zip(B.bsga_cache_load(*plain, table[0, :-2].contiguous(), count, first), got))


def test_tokens_without_a_page_are_zeros(B):
    kc, vc, ks, vs, table, [(k, v)] = cached([100], 2, 16)
    pages = table[0, :7].clone()
    pages[1], pages[3], pages[5] = -1, kc.shape[0], -2 ** 31
    gone = torch.zeros(100, dtype=torch.bool, device="cuda")
    for p in (1, 3, 5):
        gone[16 * p:16 * p + 16] = True
    got = B.bsga_cache_load(kc, vc, pages, 100, 0, ks, vs)
    for x, want in zip(got, (k, v)):
        assert bool((x[:, gone] == 0).all()) and torch.equal(x[:, ~gone], want[:, ~gone].bfloat16())


CASES = [  # lengths, heads, key heads, page, window, sinks, frame, type
    ([1], 1, 1, 16, None, 0, 1, "bf16"),
    ([0, 1, 2, 31, 32, 33, 63, 64, 65, 0, 129], 4, 2, 16, None, 0, 1, "bf16"),
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


def visible(n, window, sinks, frame):
    j = torch.arange(n, device="cuda")
    return j >= 0 if window is None else ((n - 1) // frame - j // frame < window) | (j < sinks)


def queries(n, H, dtype, seed=0, gain=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed + H)
    return (gain * torch.randn((H, n, 64), generator=g, device="cuda")).to(dtype).transpose(0, 1)


@pytest.mark.parametrize("lengths,H,K,page,window,sinks,frame,dtype", CASES)
def test_attention(B, lengths, H, K, page, window, sinks, frame, dtype):
    kc, vc, ks, vs, table, seqs = cached(lengths, K, page)
    q, n = queries(len(lengths), H, TYPES[dtype]), torch.tensor(lengths, dtype=torch.int32).cuda()
    what = dict(window=window, sinks=sinks, frame=frame)
    o, lse = B.bsga_paged_attn_e4m3(q, kc, vc, ks, vs, table, n, return_lse=True, **what)
    assert o.shape == (len(lengths), H, 64) and o.is_contiguous()
    tight = table[:, :max(1, max(-(-x // page) for x in lengths))].contiguous()  # other splits
    o2 = B.bsga_paged_attn_e4m3(q, kc, vc, ks, vs, tight, n, **what)
    for b, (k, v) in enumerate(seqs):
        if lengths[b] == 0:
            assert bool((o[b] == 0).all()) and bool((lse[b] == -math.inf).all())
            continue
        seen = visible(lengths[b], window, sinks, frame)[None]
        check(o[b][:, None], lse[b][:, None], q[b][:, None], k, v, seen)
        check(o2[b][:, None], None, q[b][:, None], k, v, seen)
    assert torch.equal(B.bsga_paged_attn_e4m3(q.contiguous(), kc, vc, ks, vs, table, n, **what), o)


@pytest.mark.parametrize("coded", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lengths,H,K,width,window", [([3000, 2000, 1000, 1], 4, 4, 2000, None), ([40] * 9 + [0, 1500] + [7] * 10, 6, 2, 500, None),
                                                      ([900, 30, 2600, 0, 1], 40, 2, 1000, None), ([5000] + [1] * 15, 2, 1, 320, 3000)])
def test_tables_wider_than_their_sequences(B, lengths, H, K, width, window, dtype, coded):
    """Many stretches that no sequence has, or the longest alone."""
    kc, vc, ks, vs, table, seqs = cached(lengths, K, 16)
    table = torch.cat([table, torch.full((len(lengths), width), -1, dtype=torch.int32, device="cuda")], 1)[:, :width].contiguous()
    q, n = queries(len(lengths), H, TYPES[dtype]), torch.tensor(lengths, dtype=torch.int32).cuda()
    if coded:
        o, lse = B.bsga_paged_attn_e4m3(q, kc, vc, ks, vs, table, n, window=window, return_lse=True)
    else:
        kc, vc = (values(c, s).to(TYPES[dtype]) for c, s in ((kc, ks), (vc, vs)))
        o, lse = B.bsga_paged_attn(q, kc, vc, table, n, window=window, return_lse=True)
    for b, (k, v) in enumerate(seqs):
        if lengths[b] == 0:
            assert bool((o[b] == 0).all()) and bool((lse[b] == -math.inf).all())
        else:
            check(o[b][:, None], lse[b][:, None], q[b][:, None], k, v, visible(lengths[b], window, 0, 1)[None])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("gain", [2.0 ** -20, 4.0, 16.0])
def test_logits_of_any_size(B, dtype, gain):
    kc, vc, ks, vs, table, seqs = cached([900, 40], 2, 32, gain=gain)
    q = queries(2, 4, TYPES[dtype])
    o, lse = B.bsga_paged_attn_e4m3(q, kc, vc, ks, vs, table, torch.tensor([900, 40], dtype=torch.int32).cuda(), return_lse=True)
    for b, (k, v) in enumerate(seqs):
        check(o[b][:, None], lse[b][:, None], q[b][:, None], k, v, torch.ones((1, k.shape[1]), dtype=torch.bool, device="cuda"))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("byte", [63, 207])
def test_values_of_any_size(B, dtype, byte):
    """Rows whose values have the smallest and the largest scale that is written: the same bits, times the power of two."""
    kc, vc, ks, vs, table, _ = cached([200], 2, 16)
    vs.masked_fill_(vs != 255, byte)
    q, n = queries(1, 4, TYPES[dtype]), torch.tensor([200], dtype=torch.int32).cuda()
    o = B.bsga_paged_attn_e4m3(q, kc, vc, ks, vs, table, n)
    want = B.bsga_paged_attn_e4m3(q, kc, vc, ks, torch.where(vs == 255, vs, 127).to(torch.uint8), table, n)
    assert torch.equal(o.double() * 2.0 ** (127 - byte), want.double())
    of = table[0, :13].long()
    k, v = (values(c[of], s[of]).transpose(0, 1).reshape(2, -1, 64)[:, :200] for c, s in ((kc, ks), (vc, vs)))
    check(want[0][:, None], None, q[0][:, None], k, v * 2.0 ** (127 - byte), torch.ones((1, 200), dtype=torch.bool, device="cuda"))


def test_the_rows_it_sees_decide(B):
    kc, vc, ks, vs, table, _ = cached([500, 500], 2, 16)
    q, n = queries(2, 4, torch.bfloat16), torch.tensor([500, 500], dtype=torch.int32).cuda()
    args = (q, kc, vc, ks, vs, table, n)
    clean = B.bsga_paged_attn_e4m3(*args, window=100, sinks=2)
    hidden, seen = int(table[0, 300 // 16]), int(table[1, 450 // 16])
    kc.view(torch.uint8)[hidden], vc.view(torch.uint8)[hidden], ks[hidden], vs[hidden] = 0x7f, 0xff, 255, 255
    kc.view(torch.uint8)[seen, 0, 450 % 16, 5] = 0x7f
    o = B.bsga_paged_attn_e4m3(*args, window=100, sinks=2)
    assert torch.equal(o[0], clean[0]) and torch.equal(o[1, 2:], clean[1, 2:]) and bool(o[1, :2].isnan().all())


def test_lengths_and_pages_that_do_not_exist(B):
    kc, vc, ks, vs, table, _ = cached([64, 64, 64], 1, 16, spare=0)
    table = table[:, :4].contiguous()
    q, n = queries(3, 2, torch.bfloat16), torch.tensor([64, 64, 64], dtype=torch.int32).cuda()
    want = B.bsga_paged_attn_e4m3(q, kc, vc, ks, vs, table, n)
    n2 = torch.tensor([2 ** 31 - 1, -5, 64], dtype=torch.int32).cuda()
    o = B.bsga_paged_attn_e4m3(q, kc, vc, ks, vs, table, n2)
    assert torch.equal(o[0], want[0]) and torch.equal(o[2], want[2]) and bool((o[1] == 0).all())
    bad, ok = table.clone(), table.clone()
    bad[0, 1], bad[0, 2], ok[0, 1], ok[0, 2] = -2 ** 31, 2 ** 31 - 1, 0, kc.shape[0] - 1
    assert torch.equal(B.bsga_paged_attn_e4m3(q, kc, vc, ks, vs, bad, n), B.bsga_paged_attn_e4m3(q, kc, vc, ks, vs, ok, n))


def test_nothing_to_do(B):
    kc, vc, ks, vs, table, _ = cached([64, 64], 1, 16)
    q, n = queries(2, 2, torch.bfloat16), torch.tensor([64, 64], dtype=torch.int32).cuda()
    assert B.bsga_paged_attn_e4m3(q[:0], kc, vc, ks, vs, table[:0], n[:0]).shape == (0, 2, 64)
    o, lse = B.bsga_paged_attn_e4m3(q, kc[:0], vc[:0], ks[:0], vs[:0], table, n, return_lse=True)
    assert bool((o == 0).all()) and bool((lse == -math.inf).all())
    x = torch.randn((0, 1, 64), dtype=torch.bfloat16, device="cuda")
    got = B.bsga_qk_norm_rope_e4m3(x, x, x, kc, vc, ks, vs, n[:0], norm=None, return_rows=True)
    assert all(t.shape == (1, 0, 64) for t in got)


def test_a_cache_past_32_bits(B):
    """Pages whose bytes lie past 2^32: 72,000 pages of 16 heads x 64 tokens, 4.7 GB each."""
    pages, K, page = 72000, 16, 64
    kc, vc = (torch.empty((pages, K, page, 64), dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2))
    ks, vs = (torch.empty((pages, K, page), dtype=torch.uint8, device="cuda") for _ in range(2))
    k0, v0, s0, s1, table, _ = cached([200, 130], K, page)
    at = torch.randperm(300, generator=torch.Generator().manual_seed(3))[:k0.shape[0]].cuda() + pages - 300
    for big, small in ((kc, k0), (vc, v0), (ks, s0), (vs, s1)):
        big.view(torch.uint8)[at] = small.view(torch.uint8)
    moved = table.clone()
    inside = (table >= 0) & (table < k0.shape[0])
    moved[inside] = at.int()[table[inside].long()]
    q, n = queries(2, 16, torch.bfloat16), torch.tensor([200, 130], dtype=torch.int32).cuda()
    assert torch.equal(B.bsga_paged_attn_e4m3(q, kc, vc, ks, vs, moved, n), B.bsga_paged_attn_e4m3(q, k0, v0, s0, s1, table, n))
    far, near = (B.bsga_cache_load(*c, t[0, :4].contiguous(), 200, 0, *s) for c, t, s in (((kc, vc), moved, (ks, vs)), ((k0, v0), table, (s0, s1))))
    assert all(torch.equal(a, b) for a, b in zip(far, near))
    x = torch.randn((40, K, 64), device="cuda").bfloat16()
    slots = ((pages - 1) * page + 10 + torch.arange(40, device="cuda")).int()
    _, rows, _ = B.bsga_qk_norm_rope_e4m3(None, x, x, kc, vc, ks, vs, slots, norm=None, return_rows=True)
    assert torch.equal(values(kc[-1, :, 10:50], ks[-1, :, 10:50]), rows.double())


def test_another_stream_and_a_graph(B):
    K, H, page = 2, 8, 16
    kc, vc, ks, vs, table, _ = cached([700, 5, 300], K, page)
    n = torch.tensor([700, 5, 300], dtype=torch.int32).cuda()
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((3, H + 2 * K, 64), generator=g, device="cuda").bfloat16()
    slots = torch.tensor([int(table[b, (m - 1) // page]) * page + (m - 1) % page for b, m in enumerate(n.tolist())], dtype=torch.int32).cuda()
    positions = (n - 1).view(3, 1).contiguous()

    def step():
        q, kr, _ = B.bsga_qk_norm_rope_e4m3(x[:, :H], x[:, H:H + K], x[:, H + K:], kc, vc, ks, vs, slots, positions, return_rows=True)
        return B.bsga_paged_attn_e4m3(q.transpose(0, 1), kc, vc, ks, vs, table, n), kr, *B.bsga_cache_load(kc, vc, table[0, :40].contiguous(), 600, 30, ks, vs)

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(4):
        x.mul_(1.0 + 0.25 * i).add_(0.125)
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in got]
        assert all(torch.equal(a, b) for a, b in zip(kept, step()))
