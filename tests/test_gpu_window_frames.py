"""Attention with a window counted in long frames: waves whose rows belong to two frames, so that whole tiles are seen by some of their rows and by
the others not at all; in float64 against the definition, with the bounds of test_gpu_window.py."""
import pytest
import torch

from tests.test_gpu_window import B, check, draw, seen_by  # noqa: F401

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H,K,N,M,frame,window,sinks,q_start", [
    (2, 1, 1500, 1500, 300, 2, 0, None),     # rows without a maximum while others of their wave are far ahead
    (2, 2, 1500, 1500, 300, 2, 5, None),     # all begin with the first tokens
    (1, 1, 1500, 1500, 300, 1, 300, None),   # the first frame stays visible: two ranges, tiles that only rows of the later frame leave out
    (3, 3, 900, 1500, 257, 3, 130, None),    # boundaries inside tiles
    (2, 2, 700, 1500, 400, 2, 0, -333),      # rows before the first key see nothing
    (8, 2, 640, 640, 320, 1, 0, None),       # frames that are tiles
    (2, 2, 700, 700, 350, None, 0, None),    # no window
])
def test_rows_of_two_frames(B, H, K, N, M, frame, window, sinks, q_start, dtype):  # noqa: F811
    q, k, v = draw(H, K, N, M, TYPES[dtype], seed=3)
    o, lse = B.bsga_window_attn(q, k, v, window=window, sinks=sinks, frame=frame, q_start=q_start, return_lse=True)
    check(o, lse, q, k, v, seen_by(N, M, window, sinks, frame, q_start))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_bad_frame_stays_with_those_that_see_it(B, bad):  # noqa: F811
    N, frame = 1500, 300
    q, k, v = draw(2, 2, N, N, torch.bfloat16, seed=4)
    seen = seen_by(N, N, 2, 0, frame, None)
    k2, v2 = k.clone(), v.clone()
    k2[:, 100], v2[:, 150] = bad, bad
    o = B.bsga_window_attn(q, k2, v2, window=2, frame=frame)
    apart = ~(seen[:, 100] | seen[:, 150])
    assert int(apart.sum()) == 900
    check(o[:, apart], None, q[:, apart], k, v, seen[apart])
    assert not bool(o[:, seen[:, 150]].isfinite().any())


@pytest.mark.parametrize("H,K", [(1, 1), (2, 2), (3, 1), (4, 4), (6, 3), (8, 8), (12, 4)])
def test_every_number_of_heads_reaches_every_row(B, H, K):  # noqa: F811
    """The launch deals units to the chip's eight parts by the number of heads."""
    N = 2600
    q, k, v = draw(H, K, N, N, torch.bfloat16, seed=H)
    o, lse = B.bsga_window_attn(q, k, v, window=70, sinks=3, return_lse=True)
    check(o, lse, q, k, v, seen_by(N, N, 70, 3, 1, None))
