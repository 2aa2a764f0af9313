"""Bookkeeping of tokens that several sequences of the paged cache begin with, which is the host's: no GPU is needed."""
import pytest
import torch

E4M3 = torch.float8_e4m3fn


def _cache(*args, **kw):
    import paper_2509_07120_amd as pkg
    return pkg.PagedCache(*args, device="cpu", **kw)


def _state(c):
    return (c.page_table.tolist(), c.lengths.tolist(), list(c._free), [list(p) for p in c._pages], list(c._length), list(c._shared), list(c._behind),
            None if c.prefixes is None else [t.tolist() for t in c.prefixes])


def test_tensors_in_8_bits():
    c = _cache(2, 5, 3, page=4, dtype=E4M3)
    assert c.k.dtype == c.v.dtype == E4M3 and c.k.shape == (5, 3, 4, 64) and c.k.is_contiguous() and not bool(c.v.view(torch.uint8).any())
    assert set(c.scales) == {"k_scale", "v_scale"} and all(t.dtype == torch.uint8 and t.shape == (5, 3, 4) for t in c.scales.values())
    assert _cache(2, 5, 3, page=4).scales == {}


def test_share():
    c = _cache(6, 20, 1, page=4)
    c.grow([0, 0, 10, 0, 0, 7])
    pages = [list(p) for p in c._pages]
    c.share(2, [2, 3])
    assert c.lengths.tolist() == [0, 0, 0, 0, 0, 7] and c.behind.tolist() == [0, 0, 10, 10, 0, 0] and c.page_table[2].tolist() == [-1] * 20
    table, lengths, starts = c.prefixes
    assert starts.tolist() == [0, 2, 4] and lengths.tolist() == [0, 10] and table.tolist() == [[-1] * 3, pages[2]]
    assert all(t.dtype == torch.int32 for t in c.prefixes)
    c.share(5, [4, 5])
    table, lengths, starts = c.prefixes
    assert starts.tolist() == [0, 2, 4, 6] and lengths.tolist() == [0, 10, 7] and table.tolist() == [[-1] * 3, pages[2], pages[5] + [-1]]
    assert len(c._free) == 20 - 3 - 2 and sorted(c._free + pages[2] + pages[5]) == list(range(20))
    slots = c.grow([1, 0, 1, 1, 2, 5])
    assert len(set(s // 4 for s in slots.tolist()) & set(pages[2] + pages[5])) == 0 and c.lengths.tolist() == [1, 0, 1, 1, 2, 5]


def test_share_in_front_and_with_others_only():
    c = _cache(4, 20, 1, page=4)
    c.grow([0, 0, 0, 9])
    c.share(3, [0, 1])
    assert c.prefixes[2].tolist() == [0, 2] and c.prefixes[1].tolist() == [9] and c.behind.tolist() == [9, 9, 0, 0] and c._length == [0] * 4
    c.grow([0, 0, 0, 5])  # it has tokens of its own again, and can give them away
    c.share(3, [2])
    assert c.prefixes[2].tolist() == [0, 2, 3] and c.behind.tolist() == [9, 9, 5, 0]


def test_share_refuses():
    c = _cache(5, 30, 1, page=4)
    c.grow([9, 0, 0, 30, 0])
    for b, sequences, text in ((0, [], "neighbours"), (0, [1, 3], "neighbours"), (0, [2, 1], "neighbours"), (0, [4, 5], "neighbours"), (0, [-1, 0], "neighbours"),
                               (1, [1, 2], "no tokens"), (0, [2, 3], "none yet"), (3, [0, 1], "none yet")):
        before = _state(c)
        with pytest.raises(ValueError, match=text):
            c.share(b, sequences)
        assert _state(c) == before
    c.share(0, [0, 1])
    before = _state(c)
    for b, sequences, text in ((3, [1, 2, 3], "none yet"), (0, [2], "no tokens")):
        with pytest.raises(ValueError, match=text):
            c.share(b, sequences)
        assert _state(c) == before
    c.trim(2)
    with pytest.raises(ValueError, match="freed"):
        c.share(3, [2, 3])


@pytest.mark.parametrize("window", [1, 2, 3, 7])
@pytest.mark.parametrize("sinks", [0, 1, 5, 30])
@pytest.mark.parametrize("frame", [1, 3, 10])
@pytest.mark.parametrize("page", [1, 4])
def test_trim_and_check_behind_shared_tokens(window, sinks, frame, page):
    for n in range(1, 50, 7):
        c = _cache(2, 120, 1, page=page, dtype=torch.float32)
        c.grow([17, 0])
        c.share(0, [0, 1])
        c.grow([0, n])
        c.trim(window, sinks, frame)
        seen = {j for p in range(17 + n - 1, 17 + n + 40) for j in range(17 + n) if j // frame <= p // frame and (p // frame - j // frame < window or j < sinks)}
        kept = {i for i, p in enumerate(c._pages[1]) if p >= 0}
        assert kept == {(j - 17) // page for j in seen if j >= 17} | {(n - 1) // page}
        assert all(p >= 0 for p in c._shared[0][2])
        for w, s, f in ((window, sinks, frame), (None, 0, 1), (9, 2, 4), (2, 40, 1)):
            p = 17 + n
            needs = [j for j in range(17, p) if j // f <= p // f and (w is None or p // f - j // f < w or j < s)]
            if any(c._pages[1][(j - 17) // page] < 0 for j in needs):
                with pytest.raises(ValueError, match="sequence 1.*freed"):
                    c.check_seen(w, s, f)
            else:
                c.check_seen(w, s, f)


def test_what_fails_is_taken_back():
    """(on the CPU: the layer gets as far as the norm, which wants device tensors)"""
    import paper_2509_07120_amd as pkg
    for dtype in (torch.float32, E4M3):
        layer = pkg.StreamAttention(2, 1, window=9, dtype=torch.float32, device="cpu")
        c = _cache(3, 30, 1, page=4, dtype=dtype)
        c.grow([10, 0, 3])
        c.share(0, [0, 1])
        for call in (lambda: layer.extend(torch.zeros(9, 128), c, 1), lambda: layer.extend(torch.zeros(9, 128), c, 2), lambda: layer.step(torch.zeros(3, 128), c)):
            before = _state(c)
            with pytest.raises((ValueError, RuntimeError)):
                call()
            assert _state(c) == before
        with pytest.raises(ValueError, match="not empty"):
            layer.prefill(torch.zeros(9, 128), c, 1)
