"""Norms of queries and keys with the rotation by position, and their gradient, against the definition in float64.

Bounds.  The kernels compute in fp32.  A row's mean and sum of squares are sums of 64 terms in a tree (at most 6 + 16 roundings of 2^-24),
the factor takes a square root and a division, angles are off by 2^-25 turns at most and their sine and cosine by a few units in the last
place: together less than 2^-19 of the terms that are added up (|n1| + |n2| for a pair; what the mean takes off counts with the
size of x and of the mean).  Then one rounding to the tensors' type, eps / 2 of the value.  The gradient adds a sum over the row, 2^-18 of its terms;
gradients of weights are sums of fp32 products over at most a few hundred terms a lane, 2^-16 of the terms' absolute sum."""
import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def B():
    import paper_2509_07120_amd as pkg
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return pkg


def _turn(x, positions, base, sign=1):
    """x [heads, tokens, 64] float64, positions [tokens, axes] or None."""
    if positions is None:
        return x
    axes = positions.shape[1]
    half = 32 // axes
    parts = []
    for s in range(axes):
        angle = positions[:, s, None].double() * base ** (-torch.arange(half, device=x.device).double() / half)
        a, b = x[..., 2 * half * s:2 * half * s + half], x[..., 2 * half * s + half:2 * half * (s + 1)]
        parts += [a * angle.cos() - sign * b * angle.sin(), b * angle.cos() + sign * a * angle.sin()]
    return torch.cat(parts, -1)


def _stats(x, norm, eps):
    if norm is None:
        return x, torch.ones_like(x[..., :1]), torch.zeros_like(x[..., :1])
    mean = x.mean(-1, keepdim=True) if norm == "layer" else torch.zeros_like(x[..., :1])
    r = ((x - mean).square().mean(-1, keepdim=True) + eps) ** -0.5
    return (x - mean) * r, r, mean


def _forward(x, w, b, positions, norm, eps, base):
    """(result, slack) for x [tokens, heads, 64] float64."""
    x = x.transpose(0, 1)
    h, r, mean = _stats(x, norm, eps)
    w = torch.ones(64, dtype=torch.float64, device=x.device) if w is None else w.double()
    b = torch.zeros(64, dtype=torch.float64, device=x.device) if b is None else b.double()
    size = ((x.abs() + mean.abs()) * r * w.abs() + b.abs())
    size = size + size.roll(32, -1) + size.roll(16, -1) + size.roll(-16, -1)  # (its partner's is among them)
    return _turn(h * w + b, positions, base), 2.0 ** -19 * size


def _backward(x, g, w, positions, norm, eps, base):
    """(dx, slack, dw, db, slack of these two) for x [tokens, heads, 64] and g [heads, tokens, 64], float64."""
    x = x.transpose(0, 1)
    h, r, mean = _stats(x, norm, eps)
    g = _turn(g, positions, base, -1)
    size = g.abs() + g.abs().roll(32, -1) + g.abs().roll(16, -1) + g.abs().roll(-16, -1)
    hsize = (x.abs() + mean.abs()) * r
    dw, db, dslack = (g * h).sum((0, 1)), g.sum((0, 1)), 2.0 ** -16 * (size * (hsize + 1)).sum((0, 1))
    w = torch.ones(64, dtype=torch.float64, device=x.device) if w is None else w.double()
    gw, size = g * w, size * w.abs()
    if norm is None:
        dx, slack = gw, size
    else:
        dx = gw - (gw.mean(-1, keepdim=True) if norm == "layer" else 0) - h * (gw * h).mean(-1, keepdim=True)
        dx, slack = dx * r, (size + size.mean(-1, keepdim=True) + hsize * (size * hsize).mean(-1, keepdim=True)) * r
    return dx.transpose(0, 1), 2.0 ** -18 * slack.transpose(0, 1), dw, db, dslack


def _close(got, want, slack):
    err = (got.double() - want).abs()
    bound = slack + torch.finfo(got.dtype).eps / 2 * (want.abs() + slack) + 1e-38
    assert got.shape == want.shape and bool((err <= bound).all()), float((err - bound).max())


def _draw(N, H, K, dtype, seed=0, layout="packed"):
    g = torch.Generator(device="cuda").manual_seed(1000 * N + 10 * H + K + seed)
    heads = H + 2 * K
    x = (torch.randn((N, heads, 64), generator=g, device="cuda") * (0.2 + torch.arange(heads, device="cuda")[:, None]) + 0.3).to(dtype)
    if layout == "heads":  # [heads, tokens, 64], as the linear layer of this package gives it
        x = x.transpose(0, 1).contiguous().transpose(0, 1)
    if layout == "gaps":  # rows that do not touch
        wide = torch.full((N + 3, heads + 1, 72), float("nan"), dtype=dtype, device="cuda")
        wide[:N, :heads, 8:] = x
        x = wide[:N, :heads, 8:]
    w = [(1 + 0.3 * torch.randn(64, generator=g, device="cuda")).to(dtype) for _ in range(2)]
    b = [(0.3 * torch.randn(64, generator=g, device="cuda")).to(dtype) for _ in range(2)]
    return x[:, :H], x[:, H:H + K], x[:, H + K:], w, b, g


CASES = [  # tokens, heads, key heads, norm, axes, type, layout
    (1, 1, 1, "rms", 1, "bf16", "packed"),
    (1, 16, 16, "layer", 2, "fp32", "packed"),
    (63, 3, 1, "layer", 1, "bf16", "gaps"),
    (64, 16, 4, "rms", 2, "bf16", "heads"),
    (65, 5, 5, None, 1, "bf16", "packed"),
    (129, 2, 1, "rms", 0, "fp32", "gaps"),
    (777, 16, 16, "layer", 2, "bf16", "packed"),
    (1374, 15, 3, "rms", 1, "fp32", "heads"),
    (5003, 16, 4, "layer", 1, "bf16", "packed"),
    (9001, 11, 11, "rms", 2, "bf16", "packed"),
]


def _positions(N, axes, g, far):
    if axes == 0:
        return None
    p = torch.randint(-50, 2000, (N, axes), generator=g, device="cuda").int()
    p[0] = far
    return p


@pytest.mark.parametrize("N,H,K,norm,axes,dtype,layout", CASES)
def test_forward(B, N, H, K, norm, axes, dtype, layout):
    q, k, v, w, b, g = _draw(N, H, K, TYPES[dtype], layout=layout)
    if norm is None:
        w = [None, None]
    if norm != "layer":
        b = [None, None]
    for far in (0, 2 ** 31 - 1, -2 ** 31):
        pos = _positions(N, axes, g, far)
        qo, ko, vo = B.bsga_qk_norm_rope(q, k, pos, w[0], w[1], b[0], b[1], v=v, norm=norm, eps=1e-5, base=500.0)
        _close(qo, *_forward(q.double(), w[0], b[0], pos, norm, 1e-5, 500.0))
        _close(ko, *_forward(k.double(), w[1], b[1], pos, norm, 1e-5, 500.0))
        assert torch.equal(vo, v.transpose(0, 1))
    qo, ko, none = B.bsga_qk_norm_rope(q, k, pos, norm=norm, eps=1e-5)
    assert none is None
    _close(qo, *_forward(q.double(), None, None, pos, norm, 1e-5, 10000.0))
    _close(ko, *_forward(k.double(), None, None, pos, norm, 1e-5, 10000.0))


@pytest.mark.parametrize("N,H,K,norm,axes,dtype,layout", CASES)
def test_backward(B, N, H, K, norm, axes, dtype, layout):
    q, k, v, w, b, g = _draw(N, H, K, TYPES[dtype], layout=layout)
    if norm is None:
        w = [None, None]
    if norm != "layer":
        b = [None, None]
    pos = _positions(N, axes, g, 1234567)
    dq, dk, dv = (torch.randn((h, N, 64), generator=g, device="cuda").to(TYPES[dtype]) for h in (H, K, K))
    what = dict(norm=norm, eps=1e-5, base=300.0)
    got = B.bsga_qk_norm_rope_bwd(dq, dk, q, k, pos, w[0], w[1], b[0], b[1], dv=dv, **what)
    for t, (x, d) in enumerate(((q, dq), (k, dk))):
        dx, slack, dw, db, dslack = _backward(x.double(), d.double(), w[t], pos, norm, 1e-5, 300.0)
        _close(got[t], dx, slack)
        for mine, want, given in ((got[3 + t], dw, w[t]), (got[5 + t], db, b[t])):
            assert (mine is None) == (given is None)
            if given is not None:
                assert mine.dtype == torch.float32
                _close(mine, want, dslack)
    assert torch.equal(got[2], dv.transpose(0, 1))
    assert got[0].untyped_storage().data_ptr() == got[2].untyped_storage().data_ptr() and got[0].stride(0) == (H + 2 * K) * 64
    again = B.bsga_qk_norm_rope_bwd(dq, dk, q, k, pos, w[0], w[1], b[0], b[1], dv=dv, **what)
    assert all(x is None or torch.equal(x, y) for x, y in zip(got, again))


@pytest.mark.parametrize("norm,axes", [("rms", 1), ("layer", 2), ("rms", 0)])
def test_gradient_against_differences(B, norm, axes):
    """The slope of sum(g y) along random directions, from the definition in float64 a step of 1e-6 to either side: the difference is off by the
    third derivative times 1e-12 and by rounding, 2^-52 / 1e-6 of the sum's terms; the gradient by its own 2^-18 of them."""
    N, H, K = 37, 4, 2
    q, k, v, w, b, g = _draw(N, H, K, torch.float32, seed=5)
    pos = _positions(N, axes, g, 77)
    bias = b if norm == "layer" else [None, None]
    dq, dk = (torch.randn((h, N, 64), generator=g, device="cuda") for h in (H, K))
    got = B.bsga_qk_norm_rope_bwd(dq, dk, q, k, pos, w[0], w[1], bias[0], bias[1], norm=norm, eps=1e-5, base=300.0)
    for t, (x, d) in enumerate(((q, dq), (k, dk))):
        args = [x.double(), w[t].double()] + ([bias[t].double()] if norm == "layer" else [])
        grads = [got[t], got[3 + t]] + ([got[5 + t]] if norm == "layer" else [])
        along = [torch.randn(a.shape, generator=g, device="cuda").double() for a in args]

        def loss(s):
            moved = [a + s * z for a, z in zip(args, along)]
            y, _ = _forward(moved[0], moved[1], moved[2] if norm == "layer" else None, pos, norm, 1e-5, 300.0)
            return (y * d.double()).sum(), (y * d.double()).abs().sum()

        slope = float((loss(1e-6)[0] - loss(-1e-6)[0]) / 2e-6)
        mine = float(sum((a.double() * z).sum() for a, z in zip(grads, along)))
        size = float(sum((a.double() * z).abs().sum() for a, z in zip(grads, along)))
        assert abs(slope - mine) <= 2.0 ** -16 * size + 1e-8 * float(loss(0)[1])


@pytest.mark.parametrize("dtype,page,K", [("bf16", 16, 4), ("fp32", 7, 1), ("bf16", 1, 3)])
def test_into_the_pages_of_a_cache(B, dtype, page, K):
    N, H, pages = 37, 4, 60
    q, k, v, w, b, g = _draw(N, H, K, TYPES[dtype])
    pos = _positions(N, 1, g, 5)
    kc, vc = (torch.randn((pages, K, page, 64), generator=g, device="cuda").to(TYPES[dtype]) for _ in range(2))
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:N].int()
    slots[3], slots[4], slots[5], slots[6] = -1, pages * page, 2 ** 31 - 1, -2 ** 31
    if slots.numel() > 7:
        slots[7] = pages * page - 1 if not bool((slots == pages * page - 1).any()) else slots[7]
    want_k, want_v = kc.clone(), vc.clone()
    qo, ko, vo = B.bsga_qk_norm_rope(q, k, pos, w[0], w[1], v=v)
    for i, s in enumerate(slots.tolist()):
        if 0 <= s < pages * page:
            want_k[s // page, :, s % page], want_v[s // page, :, s % page] = ko[:, i], vo[:, i]
    q2, k2, v2 = B.bsga_qk_norm_rope(q, k, pos, w[0], w[1], v=v, k_cache=kc, v_cache=vc, slots=slots)
    assert k2 is kc and v2 is vc and torch.equal(q2, qo)
    assert torch.equal(kc, want_k) and torch.equal(vc, want_v)  # every other token of the caches is as it was


def test_rows_that_are_not_numbers_stay_where_they_are(B):
    q, k, v, w, b, g = _draw(70, 3, 3, torch.bfloat16)
    pos = _positions(70, 1, g, 5)
    clean = B.bsga_qk_norm_rope(q, k, pos, w[0], w[1], b[0], b[1], v=v, norm="layer")
    q, k = q.clone(), k.clone()
    q[5, 1, 7], k[69, 2, 63], q[0, 0, 0] = float("nan"), float("inf"), 3e38
    out = B.bsga_qk_norm_rope(q, k, pos, w[0], w[1], b[0], b[1], v=v, norm="layer")
    bad_q, bad_k = torch.zeros(3, 70, dtype=torch.bool, device="cuda"), torch.zeros(3, 70, dtype=torch.bool, device="cuda")
    bad_q[1, 5], bad_q[0, 0], bad_k[2, 69] = True, True, True
    assert bool(out[0][1, 5].isnan().all()) and bool(out[1][2, 69].isnan().all()) and not bool(out[0][0, 0].isnan().any())
    assert torch.equal(out[0][~bad_q], clean[0][~bad_q]) and torch.equal(out[1][~bad_k], clean[1][~bad_k])


def test_constant_and_zero_rows(B):
    """A row of one value: the layer norm's variance is 0, eps holds the factor, the bias is left; a row of zeros under rms is zeros."""
    x = torch.full((4, 2, 64), 3.0, device="cuda")
    b = torch.randn(64, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    out = B.bsga_qk_norm_rope(x, x, q_bias=b, k_bias=b, norm="layer")
    assert bool((out[0] == b).all())
    assert bool((B.bsga_qk_norm_rope(torch.zeros_like(x), x)[0] == 0).all())


def test_no_tokens(B):
    x = torch.empty((0, 3, 64), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    pos = torch.empty((0, 2), dtype=torch.int32, device="cuda")
    q, k, v = B.bsga_qk_norm_rope(x, x, pos, w, w, v=x)
    assert q.shape == (3, 0, 64) and v.shape == (3, 0, 64)
    d = torch.empty((3, 0, 64), dtype=torch.bfloat16, device="cuda")
    got = B.bsga_qk_norm_rope_bwd(d, d, x, x, pos, w, w, dv=d)
    assert bool((got[3] == 0).all()) and bool((got[4] == 0).all())


def test_another_stream_and_a_graph(B):
    q, k, v, w, b, g = _draw(1374, 16, 4, torch.bfloat16)
    pos = _positions(1374, 2, g, 5)
    dq, dk, dv = (torch.randn((h, 1374, 64), generator=g, device="cuda").bfloat16() for h in (16, 4, 4))

    def step():
        out = B.bsga_qk_norm_rope(q, k, pos, w[0], w[1], b[0], b[1], v=v, norm="layer")
        return list(out) + list(B.bsga_qk_norm_rope_bwd(dq, dk, q, k, pos, w[0], w[1], b[0], b[1], dv=dv, norm="layer"))

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(4):
        q.mul_(1.0 + 0.25 * i)
        dq.neg_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, step()))
