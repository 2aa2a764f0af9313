"""The streamed attention layer and its cache where they can go wrong: nothing to do, frees and refusals between steps, long prompts."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_2509_07120_amd as pkg
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return pkg


def _x(n, d, dtype, seed=1):
    return torch.randn((n, d), generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def test_norm_of_no_tokens_into_caches(B):
    x = torch.empty((0, 3, 64), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    pos, slots = (torch.empty(s, dtype=torch.int32, device="cuda") for s in ((0, 2), (0,)))
    caches = [torch.randn((4, 3, 16, 64), device="cuda").bfloat16() for _ in range(2)]
    want = [c.clone() for c in caches]
    q, k, v = B.bsga_qk_norm_rope(x, x, pos, w, w, v=x, k_cache=caches[0], v_cache=caches[1], slots=slots)
    assert q.shape == (3, 0, 64) and k is caches[0] and v is caches[1]
    assert all(torch.equal(c, c0) for c, c0 in zip(caches, want))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_empty_prompt(B, dtype):
    layer = B.StreamAttention(4, 2, window=40, sinks=3, dtype=dtype)
    cache = B.PagedCache(2, 8, 2, page=16, dtype=dtype)
    x = _x(5, 256, dtype)
    assert layer.prefill(x[:0], cache, 0).shape == (0, 256) and layer(x[:0]).shape == (0, 256)
    assert cache.lengths.tolist() == [0, 0]
    whole = layer(x).detach()
    bar = 12 * 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -13  # outputs of O(1), a few roundings of values up to about 4
    for i in range(5):
        o = layer.step(x[i:i + 1].repeat(2, 1), cache)
        assert float((o.double() - whole[i].double()).abs().max()) <= bar
