"""What the norm with the rotation refuses, before anything is launched: no GPU is needed."""
import pytest
import torch

A = 0x1000  # a fake, 16-byte aligned, non-null pointer


@pytest.fixture(scope="module")
def B():
    import paper_2509_07120_amd as pkg
    return pkg


def _err(B):
    return B.lib.bsga_last_error().decode()


def test_forward(B):
    def call(q=A, k=A, v=A, st=(64, 64) * 3, dt=0, n=100, h=4, kh=2, d=64, norm=1, eps=1e-6, qw=A, qb=None, kw=A, kb=None, pos=A, axes=1,
             base=1e4, slots=None, pages=0, page=0, qo=A, ko=A, vo=A):
        return B.lib.bsga_qk_norm_rope(q, k, v, *st, dt, n, h, kh, d, norm, eps, qw, qb, kw, kb, pos, axes, base, slots, pages, page, qo,
                                       ko, vo, None)

    assert call(dt=2) == 1 and "dtype" in _err(B)
    assert call(d=128) == 2 and "head_dim" in _err(B)
    assert call(n=-1) == 1 and call(n=(1 << 24) + 1) == 1 and "n_tokens" in _err(B)
    assert call(q=None, k=None, v=None, qo=None, ko=None, vo=None) == 1 and "nothing to do" in _err(B)
    assert call(norm=3) == 1 and "norm" in _err(B)
    assert call(eps=-1.0) == 1 and call(eps=float("nan")) == 1 and "eps" in _err(B)
    assert call(axes=3) == 1 and "axes" in _err(B)
    assert call(axes=0) == 1 and call(pos=None) == 1 and "positions" in _err(B)
    assert call(base=0.0) == 1 and call(base=float("inf")) == 1 and "base" in _err(B)
    assert call(h=0) == 1 and "heads of q" in _err(B)
    assert call(kh=65536) == 1 and "heads of k" in _err(B)
    assert call(q=A + 8) == 1 and call(st=(60, 64, 64, 64, 64, 64)) == 1 and call(st=(64, 64, 64, -64, 64, 64)) == 1 and "16 bytes" in _err(B)
    assert call(st=(4, 64, 64, 64, 64, 64), dt=1, n=0) == 0  # 16 bytes of fp32
    assert call(qw=A + 4) == 1 and "aligned" in _err(B)
    assert call(qb=A) == 1 and "bias" in _err(B)
    assert call(norm=0) == 1 and "weight" in _err(B)
    assert call(qo=None) == 1 and call(v=None) == 1 and "its output" in _err(B)
    assert call(ko=A + 8) == 1 and "outputs" in _err(B)
    assert call(slots=A, pages=4, page=0) == 1 and "page" in _err(B)
    assert call(slots=A, pages=0, page=16) == 1 and call(slots=A, pages=1 << 27, page=16) == 1 and "2^31" in _err(B)
    assert call(n=0) == 0  # nothing to do, nothing launched


def test_backward(B):
    def call(dq=A, dk=A, dv=A, q=A, k=A, st=(64,) * 4, dt=0, n=100, h=4, kh=2, d=64, norm=1, eps=1e-6, qw=A, kw=A, pos=A, axes=1, base=1e4,
             dqi=A, dki=A, dvi=A, ost=(64,) * 6, dw=A, ws=A, wsb=1 << 30):
        return B.lib.bsga_qk_norm_rope_bwd(dq, dk, dv, q, k, *st, dt, n, h, kh, d, norm, eps, qw, kw, pos, axes, base, dqi, dki, dvi, *ost,
                                           dw, ws, wsb, None)

    assert call(dq=None) == 1 and call(dki=None) == 1 and call(dvi=None) == 1 and "both sides" in _err(B)
    assert call(dv=A + 8) == 1
    assert call(dqi=A + 8) == 1 and "aligned" in _err(B)
    assert call(ost=(64, 64, 64, 4, 64, 64)) == 1 and "strides" in _err(B)
    assert call(norm=0, qw=None, kw=None) == 1 and "weights" in _err(B)
    need = B.lib.bsga_qk_norm_rope_bwd_workspace_bytes(100, 4, 2)
    assert need > 0 and call(wsb=need - 1) == 3 and call(ws=None) == 3 and "needed" in _err(B)
    assert call(ws=A + 4) == 1 and "aligned" in _err(B)
    assert call(d=32) == 2 and call(dt=5) == 1
    assert call(n=0, dw=None) == 0
    assert B.lib.bsga_qk_norm_rope_bwd_workspace_bytes(0, 4, 2) == 0 and B.lib.bsga_qk_norm_rope_bwd_workspace_bytes(5, -1, 2) == 0


class _OnDevice(torch.Tensor):
    """Stands in for a device tensor."""
    @staticmethod
    def __new__(cls, shape, dtype=torch.bfloat16, index=0):
        return torch.Tensor._make_subclass(cls, torch.empty(shape, dtype=dtype))

    def __init__(self, shape, dtype=torch.bfloat16, index=0):
        self.index_ = index

    is_cuda = property(lambda self: True)

    def get_device(self):
        return self.index_


def test_tensors(B):
    t = _OnDevice
    q, k = t((8, 4, 64)), t((8, 2, 64))
    f = B.bsga_qk_norm_rope
    with pytest.raises(ValueError, match="device"):
        f(torch.empty((8, 4, 64)), k)
    with pytest.raises(TypeError, match="k must be"):
        f(q, t((8, 2, 64), torch.float32))
    with pytest.raises(ValueError, match="k must be.*tokens"):
        f(q, t((9, 2, 64)))
    with pytest.raises(ValueError, match="same device"):
        f(q, t((8, 2, 64), index=1))
    with pytest.raises(ValueError, match="heads"):
        f(q, k, v=t((8, 4, 64)))
    with pytest.raises(ValueError, match="norm must be"):
        f(q, k, norm="batch")
    with pytest.raises(TypeError, match="positions"):
        f(q, k, t((8, 1), torch.int64))
    with pytest.raises(ValueError, match="positions"):
        f(q, k, t((7, 1), torch.int32))
    with pytest.raises(TypeError, match="q_weight"):
        f(q, k, None, t((64,), torch.float32))
    with pytest.raises(ValueError, match="k_weight"):
        f(q, k, None, None, t((32,)))
    with pytest.raises(ValueError, match="caches go with slots"):
        f(q, k, k_cache=t((3, 2, 16, 64)))
    slots = t((8,), torch.int32)
    with pytest.raises(ValueError, match="slots need"):
        f(q, k, slots=slots)
    with pytest.raises(ValueError, match="slots must"):
        f(q, k, slots=t((7,), torch.int32), k_cache=t((3, 2, 16, 64)))
    with pytest.raises(ValueError, match="k_cache must"):
        f(q, k, slots=slots, k_cache=t((3, 4, 16, 64)))
    with pytest.raises(ValueError, match="v_cache must"):
        f(q, k, v=t((8, 2, 64)), slots=slots, k_cache=t((3, 2, 16, 64)), v_cache=t((3, 2, 8, 64)))
    with pytest.raises(ValueError, match="dk must"):
        B.bsga_qk_norm_rope_bwd(t((4, 8, 64)), t((4, 8, 64)), q, k)
