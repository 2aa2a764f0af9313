"""Windows and first tokens that pass 32 bits, in frames or in tokens, mean what they say: more than there is.  How a call over pages is dealt out shows in
the workspace that it asks for.  No GPU is needed."""
import pytest

from tests.test_norm_rope_refusals import B  # noqa: F401

HUGE = [(1 << 30) - 1, 1 << 30, (1 << 31) - 1, 1 << 31, (1 << 31) + 3, 1 << 32, (1 << 32) + 5, 10 ** 12, (1 << 62) + 1, (1 << 63) - 1]


@pytest.mark.parametrize("frame", [1, 2, 4, 1024, 1374, 1 << 24])
@pytest.mark.parametrize("dtype", [0, 1])
def test_pages(B, dtype, frame):  # noqa: F811
    def size(window, sinks, batch=3, width=1000):
        return B.lib.bsga_paged_attn_workspace_bytes(dtype, batch, 16, 4, width, 4000, 64, frame, window, sinks)

    for width in (17, 1000, 16000):
        for batch in (1, 3, 100):
            all_keys = size(0, 0, batch, width)
            assert all_keys > 0 or batch == 100  # (so many sequences fill the chip on their own)
            for window in HUGE:
                assert size(window, 0, batch, width) == size(window, 5, batch, width) == size(window, (1 << 63) - 1, batch, width) == all_keys, window
            for sinks in HUGE:
                assert size(1, sinks, batch, width) == all_keys, sinks


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("frame", [1, 64, 1000, 1024, 1 << 20])
def test_gradient(B, dtype, frame):  # noqa: F811
    """Keys of every frame are seen up to the last query, whatever the window's tokens come to in 32 bits."""
    def size(window):
        return B.lib.bsga_window_attn_bwd_workspace_bytes(dtype, 2, 2, 6000, 6000, 0, frame, window, 0)

    for window in [6000, 1 << 22, (1 << 26) - 1] + HUGE:
        assert size(window) == size(0), window
