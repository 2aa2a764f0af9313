"""What attention over a paged cache refuses, and what workspaces it asks for, before anything is launched: no GPU is needed."""
import pytest
import torch

from tests.test_norm_rope_refusals import A, B, _err, _OnDevice  # noqa: F401


def test_arguments(B):  # noqa: F811
    def call(q=A, st=(256, 64), k=A, v=A, dt=0, b=3, h=4, kh=2, d=64, table=A, width=10, lengths=A, pages=20, page=16, scale=0.125, frame=1, window=0,
             sinks=0, out=A, ws=A, wsb=1 << 40):
        return B.lib.bsga_paged_attn(q, *st, k, v, dt, b, h, kh, d, table, width, lengths, pages, page, scale, frame, window, sinks, out, None, ws,
                                     wsb, None)

    assert call(dt=2) == 1 and "dtype" in _err(B)
    assert call(d=128) == 2 and "head_dim" in _err(B)
    assert call(b=-1) == 1 and call(b=65536) == 1 and "batch" in _err(B)
    assert call(h=0) == 1 and call(kh=0) == 1 and call(kh=3) == 1 and "multiple of kv_heads" in _err(B)
    assert call(page=0) == 1 and call(page=65537) == 1 and "page" in _err(B)
    assert call(pages=-1) == 1 and "n_pages" in _err(B)
    assert call(width=-1) == 1 and call(width=1 << 27) == 1 and "2^30" in _err(B)
    assert call(frame=0) == 1 and "frame" in _err(B)
    assert call(window=-1) == 1 and "window" in _err(B)
    assert call(sinks=-1) == 1 and "sinks" in _err(B)
    for scale in (0.0, float("nan")):
        assert call(scale=scale) == 1 and "softmax_scale" in _err(B)
    assert call(q=None) == 1 and call(q=A + 8) == 1 and call(st=(60, 64)) == 1 and "q must" in _err(B)
    for name in ("k", "v", "table", "lengths"):
        assert call(**{name: None}) == 1 and "non-null" in _err(B)
    assert call(out=None) == 1 and call(k=A + 8) == 1 and "aligned" in _err(B)
    need = B.lib.bsga_paged_attn_workspace_bytes(0, 3, 4, 2, 1000, 20, 16, 1, 0, 0)
    assert need > 0 and call(width=1000, wsb=need - 1) == 3 and call(width=1000, ws=None) == 3 and "needed" in _err(B)
    assert call(ws=A + 4) == 1 and "aligned" in _err(B)
    assert call(b=0) == 0


def test_workspaces(B):  # noqa: F811
    f = B.lib.bsga_paged_attn_workspace_bytes
    assert f(0, 0, 4, 2, 10, 20, 16, 1, 0, 0) == 0 and f(5, 3, 4, 2, 10, 20, 16, 1, 0, 0) == 0
    for batch in (1, 3, 4096, 65535):
        for width, page in ((0, 16), (1, 1), (1 << 20, 16), (1 << 14, 65536), (300, 1374), (1 << 30, 1)):
            for seen in ((1, 0, 0), (1, 1, 0), (1374, 8, 1374), (1 << 24, 1 << 60, 1 << 60)):
                # 65 numbers for each row and stretch, and a stretch is 128 keys at least
                assert 0 <= f(0, batch, 16, 4, width, 100, page, *seen) <= 65 * 4 * batch * 16 * (width * page // 128 + 1)


def test_tensors(B):  # noqa: F811
    t = _OnDevice
    q, c, table, n = t((3, 4, 64)), t((20, 2, 16, 64)), t((3, 10), torch.int32), t((3,), torch.int32)
    f = B.bsga_paged_attn
    with pytest.raises(TypeError, match="unsupported dtype"):
        f(t((3, 4, 64), torch.float16), c, c, table, n)
    with pytest.raises(ValueError, match="q must be a device"):
        f(torch.empty((3, 4, 64), dtype=torch.bfloat16), c, c, table, n)
    with pytest.raises(ValueError, match="contiguous rows"):
        f(t((3, 4, 64, 1)), c, c, table, n)
    with pytest.raises(TypeError, match="v_cache"):
        f(q, c, t((20, 2, 16, 64), torch.float32), table, n)
    with pytest.raises(ValueError, match="v_cache"):
        f(q, c, t((20, 2, 8, 64)), table, n)
    with pytest.raises(ValueError, match="k_cache"):
        f(q, t((20, 2, 16, 64), index=1), c, table, n)
    with pytest.raises(TypeError, match="page_table"):
        f(q, c, c, t((3, 10), torch.int64), n)
    with pytest.raises(ValueError, match="lengths"):
        f(q, c, c, table, t((2,), torch.int32))
    with pytest.raises(ValueError, match="window"):
        f(q, c, c, table, n, window=0)
