"""Attention with a window where values are infinite, not numbers, or huge: rows that see them.  Bounds as in test_gpu_window."""
import pytest
import torch

from tests.test_gpu_window import TYPES, B, check, draw, seen_by  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N", [90, 111, 600])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_rows_that_see_a_value_that_is_not_finite(B, dtype, bad, N):  # noqa: F811
    """Key 40 is such a row, or value 41: none of the results of a query that sees it is finite, those of the others are the formula's."""
    q, k, v = draw(2, 1, N, N, TYPES[dtype])
    seen = seen_by(N, N, 70, 3, 1, None)
    for key, value in ((True, False), (False, True), (True, True)):
        k2, v2 = k.clone(), v.clone()
        touched = torch.zeros(N, dtype=torch.bool, device="cuda")
        if key:
            k2[0, 40] = bad
            touched |= seen[:, 40]
        if value:
            v2[0, 41] = bad
            touched |= seen[:, 41]
        assert bool(touched.any()) and not bool(touched.all())
        o, lse = B.bsga_window_attn(q, k2, v2, window=70, sinks=3, return_lse=True)
        assert not bool(o[:, touched].isfinite().any())
        check(o[:, ~touched], lse[:, ~touched], q[:, ~touched], k, v, seen[~touched])
        if key:  # (64 products of an infinity with numbers of both signs, or of a NaN)
            assert bool(lse[:, seen[:, 40]].isnan().all())
        elif value:
            check(torch.zeros_like(o[:, touched]), lse[:, touched], q[:, touched], k, torch.zeros_like(v), seen[touched])
    alone = seen[:, 41] & ~seen[:, 40]
    assert bool(alone.any()) == (N > 110)  # query 110 is past key 40, not past key 41


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N", [90, 600])
def test_rows_that_see_a_huge_value(B, dtype, N):  # noqa: F811
    """A value of 1e36: results of that size, by the formula."""
    q, k, v = draw(2, 1, N, N, TYPES[dtype])
    v[0, 41] = 1e36
    seen = seen_by(N, N, 70, 3, 1, None)
    o, lse = B.bsga_window_attn(q, k, v, window=70, sinks=3, return_lse=True)
    assert float(o[:, seen[:, 41]].abs().min()) > 1e30
    check(o, lse, q, k, v, seen)
