"""The streamed layer on a cache whose pages that no later token sees have been freed: the same outputs, bit for bit, as on the same cache with all of its pages, whatever the
freed pages hold by then (a key that a query does not see has no part in its result)."""
import pytest
import torch

from tests.test_gpu_stream_e4m3 import B, _x  # noqa: F401

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


def _spoil(cache, pages):
    """What a sequence that got the freed pages might leave there."""
    for t in (cache.k, cache.v):
        if cache.scales:
            t.view(torch.uint8)[pages] = 0x7f
        else:
            t[pages] = float("nan")
    for t in cache.scales.values():
        t[pages] = 254


def _trim(cache, layer):
    before = set(cache._free)
    n = cache.trim(**layer.seen)
    gone = sorted(set(cache._free) - before)
    assert len(gone) == n
    if n:
        _spoil(cache, torch.tensor(gone, device="cuda"))
    return n


@pytest.mark.parametrize("coded", [True, False])
@pytest.mark.parametrize("dtype,frame,window,sinks", [(torch.bfloat16, 1, 40, 3), (torch.float32, 1, 40, 0), (torch.bfloat16, 10, 2, 10), (torch.bfloat16, 50, 1, 5),
                                                      (torch.float32, 20, 3, 70), (torch.bfloat16, 1, 130, 65)])
def test_prompt_frames_and_tokens(B, dtype, frame, window, sinks, coded):  # noqa: F811
    layer = B.StreamAttention(4, 2, window=window, sinks=sinks, frame=frame, dtype=dtype)
    trimmed, whole = (B.PagedCache(2, 100, 2, page=16, dtype=E4M3 if coded else dtype) for _ in range(2))
    xs = [_x(n, 256, dtype, n) for n in (700, 400)]
    freed, at = 0, [300, 1]
    for c in (trimmed, whole):
        for b in range(2):
            layer.prefill(xs[b][:at[b]], c, b)
    for n, b in ((20, 0), (1, 0), (200, 1), (100, 0), (0, 0), (37, 1), (63, 0)):
        freed += _trim(trimmed, layer)
        parts = [layer.extend(xs[b][at[b]:at[b] + n], c, b) for c in (trimmed, whole)]
        assert bool(parts[1].isfinite().all()) and torch.equal(*parts)
        at[b] += n
        freed += _trim(trimmed, layer)
        x = torch.stack([xs[i][at[i]] for i in range(2)])
        steps = [layer.step(x, c) for c in (trimmed, whole)]
        assert bool(steps[1].isfinite().all()) and torch.equal(*steps)
        at = [i + 1 for i in at]
    assert freed > 0 and trimmed.lengths.tolist() == whole.lengths.tolist() == at


@pytest.mark.parametrize("coded", [True, False])
@pytest.mark.parametrize("frame,window,sinks", [(1, 60, 3), (25, 2, 25), (1, 20, 130), (1, 90, 3)])
def test_sequences_that_begin_alike(B, frame, window, sinks, coded):  # noqa: F811
    layer = B.StreamAttention(4, 2, window=window, sinks=sinks, frame=frame)
    trimmed, whole = (B.PagedCache(5, 100, 2, page=16, dtype=E4M3 if coded else torch.bfloat16) for _ in range(2))
    first, xs = _x(100, 256, torch.bfloat16, 5), [_x(300, 256, torch.bfloat16, 10 + b) for b in range(5)]
    for c in (trimmed, whole):
        layer.prefill(first, c, 1)
        c.share(1, [1, 2, 3])
        layer.prefill(xs[4][:90], c, 4)
    freed, at = 0, [0, 0, 0, 0, 90]
    for n, b in ((40, 2), (100, 3), (7, 4), (90, 2), (30, 3)):
        freed += _trim(trimmed, layer)
        parts = [layer.extend(xs[b][at[b]:at[b] + n], c, b) for c in (trimmed, whole)]
        assert bool(parts[1].isfinite().all()) and torch.equal(*parts)
        at[b] += n
        freed += _trim(trimmed, layer)
        x = torch.stack([xs[i][at[i]] for i in range(5)])
        steps = [layer.step(x, c) for c in (trimmed, whole)]
        assert bool(steps[1].isfinite().all()) and torch.equal(*steps)
        at = [i + 1 for i in at]
    assert freed > 0
