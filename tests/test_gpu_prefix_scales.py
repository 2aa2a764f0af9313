"""Attention with a shared prefix over a cache in 8 bits whose values have scales far apart, against the definition in float64: a key counts by its logit, whatever the size
of its value.  Bounds as in test_gpu_window.py (its check()): a value's scale is a power of two and changes no rounding of its weight; where it is added to a logit before the
exponential, a number of up to 64 powers of two in 32 bits, it is off by 2^-23 of that, 2^-17.5 of the weight, and the four sums of the logit it is in by 2^-17, together less than the
2^-18 (2 + size) there is for logits and sums where a logit's terms add up to 1.5 and more, as they do here."""
import math

import pytest
import torch

from tests.test_gpu_e4m3 import values
from tests.test_gpu_prefix import B, draw, visible  # noqa: F401
from tests.test_gpu_window import check

pytestmark = pytest.mark.gpu


def _rows(c, scale, table, n, page):
    of = table[:-(-n // page)].long()
    return values(c[of], scale[of]).transpose(0, 1).reshape(c.shape[1], -1, 64)[:, :n]


def _check(B, args, scales, scans, lengths, page, most, window=None, sinks=0):  # noqa: F811
    """One prefix.  Results and values times 2^(127 - most) are numbers of ordinary size."""
    o, lse = B.bsga_prefix_attn(*args, **scales, window=window, sinks=sinks, return_lse=True)
    f = 2.0 ** (127 - most)
    got = (o.double() * f).to(o.dtype)
    for b, n in enumerate(lengths):
        k, v = (torch.cat([_rows(c, s, args[5][0], scans, page), _rows(c, s, args[3][b], n, page)], 1) for c, s in
                ((args[1], scales["k_scale"]), (args[2], scales["v_scale"])))
        check(got[b][:, None], lse[b][:, None], args[0][b][:, None], k, v * f, visible(k.shape[1], window, sinks, 1)[None])


@pytest.mark.parametrize("sequences", [4, 30, 100])  # tiles of 16, 32 and 64 queries
@pytest.mark.parametrize("where", ["rows", "halves"])
@pytest.mark.parametrize("least,most", [(63, 207), (63, 190), (63, 144), (63, 143), (0, 130), (20, 100), (1, 207), (40, 40)])
def test_value_scales_far_apart(B, least, most, where, sequences):  # noqa: F811
    """Half of the value rows have one scale, half the other; those of the least that is written are rows of zeros, which is where it comes from."""
    lengths = [3 * i % 50 for i in range(sequences)]
    args, scales, _ = draw([700], [0, sequences], lengths, 2, 2, 16, "e4m3", "bf16")
    codes, scale, table = args[2].view(torch.uint8), scales["v_scale"], args[5][0]
    held = scale != 255
    if where == "rows":
        small = torch.rand(scale.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)) < 0.5
    else:  # whole stretches and waves of small ones, the prefix's first
        small = torch.zeros_like(held)
        small[table[:22].long()] = True
    scale.copy_(torch.where(held, torch.where(small, least, most), scale))
    if least == 63:
        codes.masked_fill_((small & held)[..., None], 0)
    _check(B, args, scales, 700, lengths, 16, most)


@pytest.mark.parametrize("sequences", [30, 100])
@pytest.mark.parametrize("window", [None, 150])
def test_one_large_value(B, window, sequences):  # noqa: F811
    """One row of 448 * 2^80 in the prefix, zeros and ordinary rows otherwise; with a window, some sequences see it and some do not."""
    lengths = [1 + i % 60 for i in range(sequences)]
    args, scales, _ = draw([700], [0, sequences], lengths, 4, 2, 16, "e4m3", "bf16")
    codes, scale, table = args[2].view(torch.uint8), scales["v_scale"], args[5][0]
    held = scale != 255
    zero = (torch.rand(scale.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)) < 0.5) & held
    codes.masked_fill_(zero[..., None], 0)
    scale.masked_fill_(zero, 63)
    j = 580
    codes[int(table[j // 16]), 0, j % 16], scale[int(table[j // 16]), 0, j % 16] = 0x7e, 207
    o, lse = B.bsga_prefix_attn(*args, **scales, window=window, sinks=3 if window else 0, return_lse=True)
    for b, n in enumerate(lengths):
        k, v = (torch.cat([_rows(c, s, table, 700, 16), _rows(c, s, args[3][b], n, 16)], 1) for c, s in ((args[1], scales["k_scale"]), (args[2], scale)))
        seen = visible(700 + n, window, 3 if window else 0, 1)
        for head in range(2):  # (of each key head for itself: the other's values are of ordinary size)
            f = 2.0 ** -80 if head == 0 and bool(seen[j]) else 1.0
            of = slice(2 * head, 2 * head + 2)
            check((o[b, of].double() * f).to(o.dtype)[:, None], lse[b, of][:, None], args[0][b, of][:, None], k[head:head + 1], v[head:head + 1] * f, seen[None])


@pytest.mark.parametrize("least,most", [(63, 207), (63, 143), (0, 130)])
def test_tiles_of_queries_agree(B, least, most):  # noqa: F811
    """The same sequences, few and many to a prefix, and each over one table: alike up to the roundings of two results."""
    lengths = [5] * 40
    args, scales, _ = draw([640], [0, 40], lengths, 2, 1, 16, "e4m3", "bf16")
    scale = scales["v_scale"]
    scale.copy_(torch.where(scale != 255, torch.where(torch.arange(16, device="cuda") % 3 == 0, least, most), scale))
    many = B.bsga_prefix_attn(*args, **scales)
    few = args[:]
    few[0], few[3], few[4] = args[0][:5], args[3][:5].contiguous(), args[4][:5].contiguous()
    few[7] = torch.tensor([0, 5], dtype=torch.int32).cuda()
    few = B.bsga_prefix_attn(*few, **scales)
    pages = torch.cat([args[5][:, :40].expand(40, -1), args[3][:, :1]], 1).contiguous()
    alone = B.bsga_paged_attn_e4m3(args[0], args[1], args[2], **scales, page_table=pages, lengths=args[4] + 640)
    # each is off by at most 2^-8 of sum p |v| for the weights' roundings and 2^-8 of the result for its own (and 2^-16 for logits and sums), and sum p |v| of at most
    # the largest value
    bound = 2 * (2 * 2.0 ** -8 + 2.0 ** -16) * 448 * 2.0 ** (most - 127)
    assert float((many.double() - alone.double()).abs().max()) <= bound and float((many[:5].double() - few.double()).abs().max()) <= bound
    assert math.isfinite(float(many.double().abs().max()))
