"""The norm with the rotation on no tokens: tensors without elements have no address, caches and weights do.  No GPU is needed."""
import pytest

from tests.test_norm_rope_refusals import A, B, _err  # noqa: F401


def _forward(B, q, k, v, slots, q_out, k_out, v_out):  # noqa: F811
    return B.lib.bsga_qk_norm_rope(q, k, v, *(64, 64) * 3, 0, 0, 4, 2, 64, 1, 1e-6, A, None, A, None, None, 1, 1e4, slots, 4, 16, q_out, k_out, v_out, None)


@pytest.mark.parametrize("v_cache", [A, None])
@pytest.mark.parametrize("slots", [A, None])  # (slots without elements have no address either)
def test_into_caches(B, slots, v_cache):  # noqa: F811
    assert _forward(B, None, None, None, slots, None, A, v_cache) == 0, _err(B)


def test_gradients_with_room_for_them(B):  # noqa: F811
    none = (None,) * 5
    assert B.lib.bsga_qk_norm_rope_bwd(*none, *(64,) * 4, 0, 0, 4, 2, 64, 1, 1e-6, A, A, None, 1, 1e4, A, A, A, *(64,) * 6, None, None, 0, None) == 0, _err(B)

