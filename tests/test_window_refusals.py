"""What attention with a window refuses, and what workspaces it asks for, before anything is launched: no GPU is needed."""
import pytest
import torch

from tests.test_norm_rope_refusals import A, B, _err, _OnDevice  # noqa: F401


def test_forward(B):  # noqa: F811
    def call(q=A, k=A, v=A, st=(64, 6400) * 3, dt=0, h=4, kh=2, n=100, m=100, d=64, scale=0.125, start=0, frame=1, window=10, sinks=0, out=A, ws=None,
             wsb=0):
        return B.lib.bsga_window_attn(q, k, v, *st, dt, h, kh, n, m, d, scale, start, frame, window, sinks, out, None, ws, wsb, None)

    assert call(dt=2) == 1 and "dtype" in _err(B)
    assert call(d=128) == 2 and "head_dim" in _err(B)
    assert call(h=0) == 1 and call(h=65536) == 1 and call(kh=0) == 1 and call(kh=3) == 1 and "multiple of kv_heads" in _err(B)
    assert call(n=-1) == 1 and call(m=(1 << 24) + 1) == 1 and "n_k" in _err(B)
    assert call(start=-(1 << 24) - 1) == 1 and call(start=(1 << 25) + 1) == 1 and "q_start" in _err(B)
    assert call(frame=0) == 1 and "frame" in _err(B)
    assert call(window=-1) == 1 and "window" in _err(B)
    assert call(sinks=-1) == 1 and "sinks" in _err(B)
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert call(scale=scale) == 1 and "softmax_scale" in _err(B)
    assert call(q=None) == 1 and "q must" in _err(B)
    assert call(k=A + 8) == 1 and "k must" in _err(B)
    assert call(v=None) == 1 and "v must" in _err(B)
    assert call(st=(60, 6400, 64, 6400, 64, 6400)) == 1 and call(st=(64, 6400, 1 << 23, 6400, 64, 6400)) == 1 and "stride" in _err(B)
    assert call(out=None) == 1 and call(out=A + 4) == 1 and "out" in _err(B)
    assert call(n=0) == 0


def test_backward(B):  # noqa: F811
    def call(do=A, q=A, k=A, v=A, st=(64, 6400) * 3, out=A, lse=A, dt=0, h=4, kh=2, n=100, m=100, d=64, scale=0.125, seen=(0, 1, 10, 0), dq=A, dk=A,
             dv=A, ws=A, wsb=1 << 40):
        return B.lib.bsga_window_attn_bwd(do, q, k, v, *st, out, lse, dt, h, kh, n, m, d, scale, *seen, dq, dk, dv, ws, wsb, None)

    assert call(dt=7) == 1 and call(d=32) == 2 and call(kh=3) == 1 and call(seen=(0, 0, 10, 0)) == 1 and call(scale=0.0) == 1
    for name in ("do", "out", "lse", "dq"):
        assert call(**{name: None}) == 1 and "dout" in _err(B)
    assert call(dk=None) == 1 and call(dv=A + 8) == 1 and "dk and dv" in _err(B)
    assert call(q=None) == 1 and call(v=A + 8) == 1
    need = B.lib.bsga_window_attn_bwd_workspace_bytes(0, 4, 2, 100, 100, 0, 1, 10, 0)
    assert need >= 4 * 100 * 8 and call(wsb=need - 1) == 3 and call(ws=None) == 3 and "needed" in _err(B)
    assert call(ws=A + 4) == 1 and "aligned" in _err(B)
    assert call(n=0, m=0) == 0


def test_workspaces(B):  # noqa: F811
    f, b = B.lib.bsga_window_attn_workspace_bytes, B.lib.bsga_window_attn_bwd_workspace_bytes
    assert f(0, 16, 137400, 137400, 0, 1374, 4, 1374) == 0  # enough rows without splits
    assert f(0, 16, 1, 100000, 99999, 1, 0, 0) > 0
    assert f(0, 0, 10, 10, 0, 1, 0, 0) == 0 and f(9, 4, 10, 10, 0, 1, 0, 0) == 0 and f(0, 4, 10, 10, 0, 0, 0, 0) == 0
    for n, m in ((0, 100), (100, 0), (0, 0), (1, 1), (1, 100000), (137400, 137400), (1 << 24, 1)):
        for seen in ((0, 1, 0, 0), (0, 1374, 4, 1374), (-50, 1, 7, 1 << 40), (1 << 25, 1 << 24, 1 << 60, 3)):
            for h, kh in ((16, 16), (16, 1), (1, 1)):
                assert 0 <= f(0, h, n, m, *seen) < 1 << 31
                assert h * n * 8 <= b(1, h, kh, n, m, *seen) < 1 << 38


def test_tensors(B):  # noqa: F811
    t = _OnDevice
    q, k = t((4, 8, 64)), t((2, 8, 64))
    with pytest.raises(ValueError, match="q must be a device"):
        B.bsga_window_attn(torch.empty((4, 8, 64), dtype=torch.bfloat16), k, k)
    with pytest.raises(TypeError, match="v must be"):
        B.bsga_window_attn(q, k, t((2, 8, 64), torch.float32))
    with pytest.raises(TypeError, match="unsupported dtype"):
        B.bsga_window_attn(t((4, 8, 64), torch.float16), k, k)
    with pytest.raises(ValueError, match="same device"):
        B.bsga_window_attn(q, t((2, 8, 64), index=1), k)
    with pytest.raises(ValueError, match="k and v"):
        B.bsga_window_attn(q, k, t((2, 9, 64)))
    with pytest.raises(ValueError, match="q must be.*contiguous rows"):
        B.bsga_window_attn(t((4, 8, 64, 1)), k, k)
    with pytest.raises(ValueError, match="window"):
        B.bsga_window_attn(q, k, k, window=0)
    with pytest.raises(ValueError, match="out must"):
        B.bsga_window_attn(q, k, k, out=t((4, 9, 64)))
    with pytest.raises(ValueError, match="lse must"):
        B.bsga_window_attn_bwd(q, q, k, k, q, t((4, 9), torch.float32))
