"""Gradient of the norm with the rotation: the number of heads of a tensor that is not there cannot make the workspace's size 0.  No GPU is needed."""
import pytest

from tests.test_norm_rope_refusals import A, B, _err  # noqa: F401


@pytest.mark.parametrize("absent,heads,kv_heads", [("q", -1, 2), ("q", 65536, 2), ("k", 4, -1), ("k", 4, 1 << 30)])
def test_heads_of_an_absent_tensor(B, absent, heads, kv_heads):  # noqa: F811
    q, k = (None, A) if absent == "q" else (A, None)
    assert B.lib.bsga_qk_norm_rope_bwd_workspace_bytes(100, heads, kv_heads) == 0
    for room in (0, 16, 1 << 30):
        assert B.lib.bsga_qk_norm_rope_bwd(q, k, None, q, k, *(64,) * 4, 0, 100, heads, kv_heads, 64, 1, 1e-6, A, A, A, 1, 1e4, q, k, None, *(64,) * 6, A, A,
                                           room, None) == 1 and "heads" in _err(B)


def test_no_heads_of_an_absent_tensor(B):  # noqa: F811
    """0 is a number of heads of a tensor that is not there: the call gets as far as its workspace."""
    need = B.lib.bsga_qk_norm_rope_bwd_workspace_bytes(100, 0, 2)
    assert need > 0
    assert B.lib.bsga_qk_norm_rope_bwd(None, A, None, None, A, *(64,) * 4, 0, 100, 0, 2, 64, 1, 1e-6, A, A, A, 1, 1e4, None, A, None, *(64,) * 6, A, A,
                                       need - 1, None) == 3 and "needed" in _err(B)
