"""Windows and first tokens of more than there is, up to what 64 bits hold: the results without a limit, bit for bit."""
import pytest
import torch

from tests.test_gpu_window import TYPES, B, draw  # noqa: F401

pytestmark = pytest.mark.gpu
HUGE = [(1 << 30) - 1, (1 << 31) + 3, (1 << 32) + 5, 10 ** 12, (1 << 63) - 1]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("frame", [1, 4, 1024, 1374])
def test_pages(B, dtype, frame):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(frame)
    width, page = 80, 64
    caches = [torch.randn((2 * width, 2, page, 64), generator=g, device="cuda").to(TYPES[dtype]) for _ in range(2)]
    q = torch.randn((3, 4, 64), generator=g, device="cuda").to(TYPES[dtype])
    table = torch.randint(0, 2 * width, (3, width), generator=g, device="cuda").int()
    lengths = torch.tensor([4999, 1, 3000], dtype=torch.int32, device="cuda")
    want = B.bsga_paged_attn(q, *caches, table, lengths, frame=frame, return_lse=True)
    for seen in [dict(window=w) for w in HUGE] + [dict(window=HUGE[i], sinks=HUGE[-1 - i]) for i in range(5)] + [dict(window=1, sinks=s) for s in HUGE]:
        got = B.bsga_paged_attn(q, *caches, table, lengths, frame=frame, return_lse=True, **seen)
        assert all(torch.equal(x, y) for x, y in zip(got, want)), seen


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("frame", [1, 64, 1024])
def test_window_and_gradient(B, dtype, frame):  # noqa: F811
    q, k, v = draw(2, 1, 1500, 1700, TYPES[dtype])
    dout = torch.randn_like(q)
    results = []
    for seen in [dict()] + [dict(window=w) for w in HUGE]:
        o, lse = B.bsga_window_attn(q, k, v, frame=frame, return_lse=True, **seen)
        results.append([o, lse, *B.bsga_window_attn_bwd(dout, q, k, v, o, lse, frame=frame, **seen)])
    assert all(torch.equal(x, y) for r in results[1:] for x, y in zip(r, results[0]))
