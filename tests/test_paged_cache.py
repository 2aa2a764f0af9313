"""Bookkeeping of the paged cache, which is the host's: no GPU is needed."""
import pytest
import torch


def _cache(*args, **kw):
    import paper_2509_07120_amd as pkg
    return pkg.PagedCache(*args, device="cpu", **kw)


def _state(c):
    return c.page_table.tolist(), c.lengths.tolist(), list(c._free), [list(p) for p in c._pages], list(c._length)


def test_trim_without_a_window_frees_nothing():
    c = _cache(2, 5, 1, page=4)
    c.grow([6, 3])
    before = _state(c)
    assert c.trim(None) == 0 and c.trim(window=None, sinks=3, frame=2) == 0
    assert _state(c) == before


@pytest.mark.parametrize("window,sinks,frame", [(0, 0, 1), (-1, 0, 1), (2, -1, 1), (2, 0, 0), (2, 0, -3), (None, -1, 1), (None, 0, 0)])
def test_trim_refuses_what_the_attention_refuses(window, sinks, frame):
    """(0 is "no limit" at the C interface: taken as a window of nothing it would free tokens that are seen, the last ones among them)"""
    c = _cache(1, 3, 1, page=4)
    c.grow([6])
    before = _state(c)
    with pytest.raises(ValueError, match="window|sinks|frame"):
        c.trim(window, sinks, frame)
    assert _state(c) == before
    assert c.grow([3]).tolist() == [6, 7, 8]


@pytest.mark.parametrize("window", [1, 2, 3, 7])
@pytest.mark.parametrize("sinks", [0, 1, 5, 9])
@pytest.mark.parametrize("frame", [1, 3, 10])
@pytest.mark.parametrize("page", [1, 4, 7])
def test_trim_keeps_what_later_queries_see(window, sinks, frame, page):
    for n in range(1, 60, 4):
        c = _cache(1, 80, 1, page=page, dtype=torch.float32)
        c.grow([n])
        c.trim(window, sinks, frame)
        seen = {j for p in range(n - 1, n + 40) for j in range(n) if j // frame <= p // frame and (p // frame - j // frame < window or j < sinks)}
        assert all(c._pages[0][j // page] >= 0 for j in seen)
        kept = {i for i, p in enumerate(c._pages[0]) if p >= 0}
        assert kept == {j // page for j in seen} | {(n - 1) // page}  # and nothing else


def test_trim_takes_freed_pages_out_of_the_table():
    c = _cache(2, 9, 1, page=4)
    c.grow([23, 10])
    assert c.trim(5, sinks=2) > 0
    assert c.page_table[0].tolist() == [0, -1, -1, -1, 4, 5] + [-1] * 3  # tokens 18 to 22 and the first 2 stay
    assert c.page_table[1].tolist() == [6, 7, 8] + [-1] * 6
    assert sorted(c.grow([0, 12]).tolist()) == sorted([4 * 8 + 2, 4 * 8 + 3] + [4 * p + i for p in (3, 2) for i in range(4)] + [4, 5])
    assert c.page_table[0].tolist() == [0, -1, -1, -1, 4, 5] + [-1] * 3


@pytest.mark.parametrize("trimmed", [(5, 2, 1), (2, 0, 3), (1, 7, 4), (3, 9, 2)])
@pytest.mark.parametrize("page", [1, 4])
def test_windows_that_see_freed_tokens(trimmed, page):
    """check_seen(), against the rule itself for the next token of every sequence."""
    for window, sinks, frame in [(w, s, f) for w in (None, 1, 2, 3, 5, 6, 40) for s in (0, 2, 3, 7, 20) for f in (1, 2, 3, 4)]:
        c = _cache(2, 200, 1, page=page)
        c.check_seen(window, sinks, frame)  # nothing there, nothing freed
        c.grow([23, 2])
        c.check_seen(window, sinks, frame)
        c.trim(*trimmed)
        c.grow([6, 6])
        c.trim(*trimmed)
        bad = False
        for b, p in ((0, 29), (1, 8)):
            seen = [j for j in range(p) if j // frame <= p // frame and (window is None or p // frame - j // frame < window or j < sinks)]
            bad |= any(c._pages[b][j // page] < 0 for j in seen)
        if bad:
            with pytest.raises(ValueError, match="sequence [01].*freed"):
                c.check_seen(window, sinks, frame)
        else:
            c.check_seen(window, sinks, frame)


def test_a_step_asks_before_it_grows():
    import paper_2509_07120_amd as pkg
    layer = pkg.StreamAttention(2, 1, window=9, dtype=torch.float32, device="cpu")
    c = _cache(1, 9, 1, page=4, dtype=torch.float32)
    c.grow([20])
    c.trim(3)
    before = _state(c)
    with pytest.raises(ValueError, match="freed"):
        layer.step(torch.zeros(1, 128), c)
    assert _state(c) == before


@pytest.mark.parametrize("counts", [[1, 1, 1], [0, 9, 0], [30, 0, 3], [3, 4, 5], [0, 0, 0]])
def test_what_fails_behind_grow_is_taken_back(counts):
    c = _cache(3, 30, 1, page=4)
    c.grow([7, 0, 12])
    c.trim(2)
    before, slots = _state(c), []
    with pytest.raises(KeyError):
        with c.growing(counts) as got:
            slots.append(got.tolist())
            assert c._length == [a + b for a, b in zip([7, 0, 12], counts)]
            raise KeyError
    assert _state(c) == before
    with c.growing(counts) as got:
        assert got.tolist() == slots[0]  # the same places as the first time
    assert c.lengths.tolist() == [a + b for a, b in zip([7, 0, 12], counts)]


def test_a_prompt_and_a_step_that_fail_leave_the_cache_as_it_was():
    """(on the CPU: the layer gets as far as the norm, which wants device tensors)"""
    import paper_2509_07120_amd as pkg
    layer = pkg.StreamAttention(2, 1, window=9, dtype=torch.float32, device="cpu")
    c = _cache(2, 9, 1, page=4, dtype=torch.float32)
    for call in (lambda: layer.prefill(torch.zeros(9, 128), c, 1), lambda: layer.prefill(torch.zeros(9, 64), c, 1),
                 lambda: layer.step(torch.zeros(2, 128), c), lambda: layer.step(torch.zeros(2, 128), c, torch.zeros(3, dtype=torch.int32))):
        before = _state(c)
        with pytest.raises((ValueError, RuntimeError)):
            call()
        assert _state(c) == before
