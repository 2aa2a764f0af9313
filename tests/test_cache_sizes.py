"""Sizes of a paged cache whose product does not fit 64 bits: refused, not taken for what is left of the product.  No GPU is needed."""
import pytest

from tests.test_norm_rope_refusals import A, B, _err  # noqa: F401

WRAPS = [((1 << 48), 65536), ((1 << 48) + 1, 65536), ((1 << 62) + 1, 4), ((1 << 63) - 1, 2)]  # 2^64, 2^64 + 65536, 2^64 + 4, 2^64 - 2


@pytest.mark.parametrize("pages,page", WRAPS)
def test_norm_into_pages(B, pages, page):  # noqa: F811
    """(No tokens: nothing is launched either way.)"""
    assert B.lib.bsga_qk_norm_rope(None, A, None, *(64, 64) * 3, 0, 0, 4, 2, 64, 1, 1e-6, None, None, A, None, A, 1, 1e4, A, pages, page, None, A, None,
                                   None) == 1 and "2^31" in _err(B)


@pytest.mark.parametrize("width,page", WRAPS)
def test_page_table(B, width, page):  # noqa: F811
    assert B.lib.bsga_paged_attn(A, 256, 64, A, A, 0, 0, 4, 2, 64, A, width, A, 20, page, 0.125, 1, 0, 0, A, None, A, 1 << 40, None) == 1 and "2^30" in _err(B)
    assert B.lib.bsga_paged_attn_workspace_bytes(0, 3, 4, 2, width, 20, page, 1, 0, 0) == 0
