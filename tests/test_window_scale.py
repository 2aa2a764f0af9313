"""Scales whose reciprocal does not fit beside a logarithm: the gradient, which begins its sums with -lse / scale, refuses them.  No GPU is needed."""
import math

import pytest

from tests.test_norm_rope_refusals import A, B, _err  # noqa: F401


def _backward(B, scale, room):  # noqa: F811
    return B.lib.bsga_window_attn_bwd(A, A, A, A, *(64, 6400) * 3, A, A, 0, 4, 2, 100, 100, 64, scale, 0, 1, 10, 0, A, A, A, A, room, None)


@pytest.mark.parametrize("scale", [1.5e-45, 1e-40, 2.0 ** -126, 4.8e-38, math.nextafter(2.0 ** -120, 0.0) * (1 - 2.0 ** -23)])
def test_too_small(B, scale):  # noqa: F811
    assert _backward(B, scale, 0) == 1 and "softmax_scale" in _err(B)


@pytest.mark.parametrize("scale", [2.0 ** -120, 1e-30, 0.125, 1e30])
def test_as_small_as_it_may_be(B, scale):  # noqa: F811
    assert _backward(B, scale, 0) == 3 and "needed" in _err(B)  # on to the workspace
