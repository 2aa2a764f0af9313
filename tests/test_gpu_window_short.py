"""Attention with windows that are short beside the queries of a workgroup, where waves go by themselves; bounds as in test_gpu_window.py."""
import pytest
import torch

from tests.test_gpu_window import B, check, draw, seen_by  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,K,N,M,window,sinks,frame", [
    (3, 1, 129, 129, 1, 0, 1),
    (2, 2, 1153, 1200, 70, 0, 1),
    (4, 2, 2001, 2001, 5, 3, 13),
    (2, 1, 3000, 3000, 300, 65, 1),
    (1, 1, 6001, 6001, 2, 130, 64),      # the longest frame of such a launch
    (1, 1, 3000, 3000, 2, 130, 65),      # and the first that is not
    (8, 8, 2048, 2048, None, 0, 1),      # 32 tiles for the last 256 queries
    (8, 8, 2049, 2049, None, 0, 1),
])
def test_short_windows(B, H, K, N, M, window, sinks, frame):  # noqa: F811
    q, k, v = draw(H, K, N, M, torch.bfloat16, layout="tokens")
    what = dict(window=window, sinks=sinks, frame=frame)
    o, lse = B.bsga_window_attn(q, k, v, return_lse=True, **what)
    check(o, lse, q, k, v, seen_by(N, M, window, sinks, frame, None))
    assert torch.equal(B.bsga_window_attn(q, k, v, **what), o)


def test_rows_that_are_not_finite(B):  # noqa: F811
    """A value that is not a number reaches the queries that see it, and no others (those of the same tile are computed again one by one, with sums in
    another order)."""
    q, k, v = draw(2, 1, 1500, 1500, torch.bfloat16)
    clean = v.clone()
    v[0, 700, 3] = float("nan")
    o = B.bsga_window_attn(q, k, v, window=40)
    seen = seen_by(1500, 1500, 40, 0, 1, None)
    touched = seen[:, 700]
    assert int(touched.sum()) == 40 and bool(o[:, touched, 3].isnan().all())
    check(o[:, ~touched], None, q[:, ~touched], k, clean, seen[~touched])
    rest = torch.arange(64, device="cuda") != 3
    check(o[:, touched][..., rest], None, q[:, touched], k, clean[..., rest], seen[touched])
