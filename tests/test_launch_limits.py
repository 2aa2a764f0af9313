"""Calls whose launch would have 2^32 threads or more in a row, which the runtime does not take, are refused by name before anything is launched: no GPU is needed."""
from tests.test_e4m3_refusals import _paged
from tests.test_norm_rope_refusals import A, B, _err  # noqa: F401


def test_reading_back(B):  # noqa: F811
    def call(n):
        return B.lib.bsga_cache_load(A, A, A, A, 2, 100, 1, 1, 64, A, 1 << 30, 0, n, 0, A, A, n * 64, n * 64, None)

    for n in ((1 << 30) - 63, 1 << 30):
        assert call(n) == 2 and "one launch" in _err(B)


def test_attention_over_pages(B):  # noqa: F811
    # a page to a token: a stretch's page numbers have to fit, so that 20,000 tokens are 11 stretches, whose join has a workgroup to a row
    big = dict(b=65535, width=20000, page=1, pages=1 << 20, wsb=1 << 60)
    assert _paged(B, h=257, kh=1, st=(257 * 64, 64), **big) == 2 and "one launch" in _err(B)

    def own(b, h, kh, width):
        return B.lib.bsga_paged_attn(A, h * 64, 64, A, A, 0, b, h, kh, 64, A, width, A, 1 << 20, 1, 0.125, 1, 0, 0, A, None, A, 1 << 60, None)

    assert own(65535, 257, 1, 20000) == 2 and "one launch" in _err(B)
    # up to eight stretches: sixteen rows to a workgroup
    assert own(65535, 4112, 1, 6000) == 2 and "one launch" in _err(B)
