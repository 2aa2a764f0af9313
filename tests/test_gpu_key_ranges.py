"""Keys of any size on their way into a cache in 8 bits, against the definition in float64, bit for bit (which is itself off by 2^-40 at these positions, so that one number
in 2^37 may differ): rows whose squares, or whose sum, are not numbers of 32 bits."""
import pytest
import torch

from tests.test_gpu_e4m3 import B, empty_cache, quantised, values  # noqa: F401
from tests.test_gpu_window import TYPES

pytestmark = pytest.mark.gpu


def _want(k, w, bias, positions, norm, eps, base=1e4):
    x = k.double()
    if norm == "layer":
        x = x - x.mean(-1, keepdim=True)
    x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * w.double()
    if bias is not None:
        x = x + bias.double()
    if positions is None:
        return x
    half = 32
    angle = positions.double()[:, None, :, None] * base ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    a, b = x.view(*k.shape[:2], 1, 2, half).unbind(3)
    return torch.stack([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], 3).view(k.shape)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("axes", [0, 1])
@pytest.mark.parametrize("size,eps", [(1.0, 1e-6), (2e18, 1e-6), (3e18, 1e-6), (1e19, 1e-6), (1e37, 0.0), (1e-12, 0.0), (1e-15, 0.0), (1e-19, 0.0), (1e-21, 0.0), (1e-23, 0.0),
                                      (1e-36, 0.0), (1e-21, 1e-42), (1e-6, 1e-40), (1e19, 1e39)])
def test_rows_of_any_size(B, size, eps, norm, axes, dtype):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(axes + 2 * len(norm))
    N, K, page = 200, 2, 40
    k = (size * torch.randn((N, K, 64), generator=g, device="cuda").double()).to(TYPES[dtype])
    k[::7] = torch.randn((len(range(0, N, 7)), K, 64), generator=g, device="cuda").to(k.dtype)  # ordinary rows between them
    w = (1 + 0.2 * torch.randn(64, generator=g, device="cuda")).to(k.dtype)
    bias = (0.3 * torch.randn(64, generator=g, device="cuda")).to(k.dtype) if norm == "layer" and axes else None
    positions = torch.randint(0, 4097, (N, 1), generator=g, device="cuda").int() if axes else None
    slots = torch.randperm(N, generator=g, device="cuda").int()
    kc, vc, ks, vs = empty_cache(N // page, K, page)
    rows = B.bsga_qk_norm_rope_e4m3(None, k, k, kc, vc, ks, vs, slots, positions, k_weight=w, k_bias=bias, norm=norm, eps=eps, return_rows=True)[1]
    want, s = quantised(_want(k, w, bias, positions, norm, eps))
    at, row = slots.long() // page, slots.long() % page
    assert torch.equal(ks[at, :, row].int(), (s + 127).int())
    assert torch.equal(values(kc, ks)[at, :, row], want)
    assert torch.equal(rows.transpose(0, 1).double(), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("mean,spread", [(1.0, 1e-3), (100.0, 1.0), (3e4, 1.0), (1e6, 4.0)])
def test_a_mean_far_above_what_is_left(B, mean, spread, dtype):  # noqa: F811
    """Layer norm: what the mean is off by, in units of the result."""
    g = torch.Generator(device="cuda").manual_seed(3)
    N, K, page = 4000, 2, 40
    k = (mean + spread * torch.randn((N, K, 64), generator=g, device="cuda")).to(TYPES[dtype])
    w, bias = ((x + 0.2 * torch.randn(64, generator=g, device="cuda")).to(k.dtype) for x in (1.0, 0.0))
    positions = torch.randint(0, 4097, (N, 1), generator=g, device="cuda").int()
    slots = torch.randperm(N, generator=g, device="cuda").int()
    kc, vc, ks, vs = empty_cache(N // page, K, page)
    B.bsga_qk_norm_rope_e4m3(None, k, k, kc, vc, ks, vs, slots, positions, k_weight=w, k_bias=bias, norm="layer")
    want, s = quantised(_want(k, w, bias, positions, "layer", 1e-6))
    at, row = slots.long() // page, slots.long() % page
    assert torch.equal(ks[at, :, row].int(), (s + 127).int())
    assert torch.equal(values(kc, ks)[at, :, row], want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("weight,size", [(1e30, 1.0), (1e35, 1e-35), (1e-30, 1.0), (3e12, 1e-36)])
def test_weights_of_any_size(B, weight, size, dtype):  # noqa: F811
    """What a number loses below 2^-126 before the weight comes back behind it: an eps of 10^12 keeps rows of small numbers small until then."""
    g = torch.Generator(device="cuda").manual_seed(5)
    N, K, page = 200, 2, 40
    k = (size * torch.randn((N, K, 64), generator=g, device="cuda").double()).to(TYPES[dtype])
    w = (weight * (1 + 0.2 * torch.randn(64, generator=g, device="cuda").double())).to(k.dtype)
    positions = torch.randint(0, 4097, (N, 1), generator=g, device="cuda").int()
    slots = torch.randperm(N, generator=g, device="cuda").int()
    kc, vc, ks, vs = empty_cache(N // page, K, page)
    B.bsga_qk_norm_rope_e4m3(None, k, k, kc, vc, ks, vs, slots, positions, k_weight=w, norm="rms", eps=1e12)
    want, s = quantised(_want(k, w, None, positions, "rms", 1e12))
    at, row = slots.long() // page, slots.long() % page
    assert torch.equal(ks[at, :, row].int(), (s + 127).int())
    assert torch.equal(values(kc, ks)[at, :, row], want)
