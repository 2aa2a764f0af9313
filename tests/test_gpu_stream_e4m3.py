"""The streamed attention layer on a cache in 8 bits, with a new frame on a cache, and with sequences that begin with the same tokens.

What the cache holds is read back and taken as given: outputs are the definition in float64 over it, with the queries that the layer's own norm gives.  They are O(1): a few
bf16 roundings of values up to about 4, 12 * 2^-8, as for the layer on a cache of its own type (fp32: of 2^-24, a thousand terms, 2^-13)."""
import pytest
import torch

from tests.test_gpu_window import attend, seen_by

pytestmark = pytest.mark.gpu
BARS = {torch.bfloat16: 12 * 2.0 ** -8, torch.float32: 2.0 ** -13}


@pytest.fixture(scope="module")
def B():
    import paper_2509_07120_amd as pkg
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return pkg


def _x(n, d, dtype, seed=1):
    return torch.randn((n, d), generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


@torch.no_grad()
def _want(B, layer, cache, x, b, start):
    """The layer's outputs for x, the tokens from `start` on of sequence b, over what the cache holds of it."""
    k, v = cache.load(b, dtype=x.dtype)
    q, k0, _ = layer._split(torch.nn.functional.linear(x, layer.w_qkv, layer.b_qkv))
    positions = torch.arange(start, start + x.shape[0], device="cuda", dtype=torch.int32)
    q = B.bsga_qk_norm_rope(q, k0, positions, **layer._norms())[0]
    n, m = x.shape[0], start + x.shape[0]
    s = layer.seen
    o = attend(q, k[:, :m], v[:, :m], seen_by(n, m, s["window"], s["sinks"], s["frame"], start), 0.125)[0]
    return o.transpose(0, 1).reshape(n, -1) @ layer.w_out.double().T + layer.b_out.double()


def _near(o, want, dtype):
    err = float((o.double() - want).abs().max())
    assert err <= BARS[dtype], err


@pytest.mark.parametrize("coded", [True, False])
@pytest.mark.parametrize("dtype,norm,frame,window,sinks", [(torch.bfloat16, "rms", 1, 40, 3), (torch.float32, "layer", 1, None, 0), (torch.bfloat16, "layer", 10, 2, 10),
                                                           (torch.bfloat16, "rms", 100, 1, 5)])
def test_prompt_frames_and_tokens(B, dtype, norm, frame, window, sinks, coded):
    layer = B.StreamAttention(4, 2, window=window, sinks=sinks, frame=frame, norm=norm, dtype=dtype)
    cache = B.PagedCache(2, 60, 2, page=16, dtype=torch.float8_e4m3fn if coded else dtype)
    xs = [_x(n, 256, dtype, n) for n in (300, 97)]
    _near(layer.prefill(xs[0][:100], cache, 0), _want(B, layer, cache, xs[0][:100], 0, 0), dtype)
    at = 100
    for n in (10, 1, 39, 0, 50):  # a new frame, a token, parts of a prompt
        o = layer.extend(xs[0][at:at + n], cache, 0)
        assert o.shape == (n, 256)
        if n:
            _near(o, _want(B, layer, cache, xs[0][at:at + n], 0, at), dtype)
        at += n
    _near(layer.extend(xs[1][:90], cache, 1), _want(B, layer, cache, xs[1][:90], 1, 0), dtype)  # also as a first prompt
    for i in range(3):
        o = layer.step(torch.stack([xs[0][at + i], xs[1][90 + i]]), cache)
        for b, j in ((0, at + i), (1, 90 + i)):
            _near(o[b:b + 1], _want(B, layer, cache, xs[b][j:j + 1], b, j), dtype)
    assert cache.lengths.tolist() == [at + 3, 93]
    if window is not None:
        cache.trim(window, sinks, frame)
        o = layer.extend(xs[0][at + 3:at + 23], cache, 0)
        assert bool(o.isfinite().all())
        if not coded:  # the same as all at once (whole frames)
            if frame == 1:
                whole = layer(xs[0][:at + 23]).detach()
                assert float((o.double() - whole[at + 3:].double()).abs().max()) <= BARS[dtype]


def test_a_prompt_in_parts_is_the_prompt(B):
    """On a cache of the layer's type: rows of whole frames, by what forward() gives for the whole."""
    for frame, window, sinks in ((1, 50, 2), (20, 3, 20), (1, None, 0)):
        layer = B.StreamAttention(4, 1, window=window, sinks=sinks, frame=frame)
        x = _x(200, 256, torch.bfloat16)
        whole = layer(x).detach()
        cache = B.PagedCache(1, 20, 1, page=16)
        o = torch.cat([layer.extend(part, cache, 0) for part in x.split((40, 20, 100, 40))])
        assert float((o.double() - whole.double()).abs().max()) <= BARS[torch.bfloat16]


@pytest.mark.parametrize("coded", [True, False])
@pytest.mark.parametrize("frame,window,sinks", [(1, None, 0), (1, 60, 3), (25, 2, 25)])
def test_sequences_that_begin_alike(B, frame, window, sinks, coded):
    dtype = torch.bfloat16
    layer = B.StreamAttention(4, 2, window=window, sinks=sinks, frame=frame, dtype=dtype)
    cache = B.PagedCache(6, 80, 2, page=16, dtype=torch.float8_e4m3fn if coded else dtype)
    first, second = _x(100, 256, dtype, 5), _x(75, 256, dtype, 6)
    layer.prefill(first, cache, 1)
    layer.prefill(second, cache, 4)
    cache.share(1, [1, 2, 3])
    cache.share(4, [4])
    own = [_x(40, 256, dtype, 10 + b) for b in range(6)]
    starts = [0, 100, 100, 100, 75, 0]
    _near(layer.extend(own[2][:25], cache, 2), _want(B, layer, cache, own[2][:25], 2, 100), dtype)
    layer.prefill(own[0][:25], cache, 0)
    taken = [25, 0, 25, 0, 0, 0]
    for _ in range(4):
        x = torch.stack([own[b][taken[b]] for b in range(6)])
        o = layer.step(x, cache)
        for b in range(6):
            _near(o[b:b + 1], _want(B, layer, cache, x[b:b + 1], b, starts[b] + taken[b]), dtype)
            taken[b] += 1
    assert cache.lengths.tolist() == taken
    with pytest.raises(ValueError, match="not empty"):
        layer.prefill(own[3], cache, 3)
    if window is not None:
        cache.trim(window, sinks, frame)
        x = torch.stack([own[b][taken[b]] for b in range(6)])
        assert bool(layer.step(x, cache).isfinite().all())


def test_a_step_in_a_graph(B):
    """Growing is the host's and stays outside: the operators of a step, replayed while lengths, slots and inputs change."""
    layer = B.StreamAttention(4, 2, window=64, sinks=2)
    cache = B.PagedCache(3, 60, 2, page=16, dtype=torch.float8_e4m3fn)
    layer.prefill(_x(70, 256, torch.bfloat16), cache, 0)
    cache.share(0, [0, 1, 2])
    x, slots = torch.zeros((3, 256), dtype=torch.bfloat16, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")

    def operators():
        q, k, v = layer._split(torch.nn.functional.linear(x, layer.w_qkv, layer.b_qkv))
        q = layer._store(q, k, v, cache.lengths + cache.behind - 1, cache, slots).transpose(0, 1)
        return B.bsga_prefix_attn(q, cache.k, cache.v, cache.page_table, cache.lengths, *cache.prefixes, **cache.scales, **layer.seen)

    slots.copy_(cache.grow([1, 1, 1]))
    with torch.no_grad():
        operators()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = operators()
        for i in range(5):
            slots.copy_(cache.grow([1, i % 2, 1]) if i % 2 else cache.grow([1, 1, 1]))
            x.copy_(_x(3, 256, torch.bfloat16, 20 + i))
            graph.replay()
            torch.cuda.synchronize()
            kept = got.clone()
            assert bool(kept.isfinite().all()) and torch.equal(kept, operators())
