"""Strides whose bytes pass 64 bits, or any memory: refused by the streamed layer's entry points, not taken for what is left of them.  No GPU is needed."""
import pytest

from tests.test_norm_rope_refusals import A, B, _err  # noqa: F401

WRAPS = [(1 << 40) + 8, 1 << 60, 1 << 61, 1 << 62, (1 << 62) + 64, (1 << 63) - 64]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("stride", WRAPS)
@pytest.mark.parametrize("which", range(6))
def test_every_stride(B, which, stride, dtype):  # noqa: F811
    st = [64] * 6
    st[which] = stride
    lib = B.lib
    assert lib.bsga_qk_norm_rope(A, A, A, *st, dtype, 100, 4, 2, 64, 1, 1e-6, A, None, A, None, A, 1, 1e4, None, 0, 0, A, A, A, None) == 1 and "16 bytes" in _err(B)
    assert lib.bsga_window_attn(A, A, A, *st, dtype, 4, 2, 100, 100, 64, 0.125, 0, 1, 10, 0, A, None, None, 0, None) == 1 and "stride" in _err(B)
    assert lib.bsga_window_attn_bwd(A, A, A, A, *st, A, A, dtype, 4, 2, 100, 100, 64, 0.125, 0, 1, 10, 0, A, A, A, None, 0, None) == 1 and "stride" in _err(B)
    grads = lambda x, into: lib.bsga_qk_norm_rope_bwd(A, A, A, A, A, *x, dtype, 100, 4, 2, 64, 1, 1e-6, A, A, A, 1, 1e4, A, A, A, *into, A, None, 0, None)  # noqa: E731
    assert grads([64] * 4, st) == 1 and "strides" in _err(B)
    if which < 4:
        assert grads(st[:4], [64] * 6) == 1 and "strides" in _err(B)
    if which < 2:
        assert lib.bsga_paged_attn(A, *st[:2], A, A, dtype, 3, 4, 2, 64, A, 10, A, 20, 16, 0.125, 1, 0, 0, A, None, A, 1 << 40, None) == 1 and "q must" in _err(B)
