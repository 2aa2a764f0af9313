"""The streamed attention layer and its cache where they can go wrong: nothing to do, frees and refusals between steps, long prompts."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_2509_07120_amd as pkg
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return pkg


def test_norm_of_no_tokens_into_caches(B):
    x = torch.empty((0, 3, 64), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    pos, slots = (torch.empty(s, dtype=torch.int32, device="cuda") for s in ((0, 2), (0,)))
    caches = [torch.randn((4, 3, 16, 64), device="cuda").bfloat16() for _ in range(2)]
    want = [c.clone() for c in caches]
    q, k, v = B.bsga_qk_norm_rope(x, x, pos, w, w, v=x, k_cache=caches[0], v_cache=caches[1], slots=slots)
    assert q.shape == (3, 0, 64) and k is caches[0] and v is caches[1]
    assert all(torch.equal(c, c0) for c, c0 in zip(caches, want))
