"""The gradient of attention with a sliding window against its formula in float64 and against differences.

Bounds.  With P exact, dV = P^T dO, dS = P (dP - D), dQ = scale dS K, dK = scale dS^T Q.  The kernels' P is off by 2^-18 (2 + L), L the
largest sum |q k| scale (as in the forward pass, twice: products and lse), dP - D by 2^-18 of sum |dO V| + sum |dO O|, and in bf16 O is rounded (2^-8 of
sum |dO O|, half a step of eight significant bits); then P and dS are rounded to bf16 for the last product (2^-8) and the result is rounded
(eps / 2).  So an error of e_P = 2^-17 (2 + L) (+ 2^-8 in bf16) relative to each P, and for dS the same of P (sum |dO V| + sum |dO O|); added up over absolute values."""
import math

import pytest
import torch

from tests.test_gpu_window import CASES, TYPES, B, draw, seen_by  # noqa: F401

pytestmark = pytest.mark.gpu


def gradients(dout, q, k, v, seen, scale):
    """(dq, dk, dv) and the bounds' sums for each, float64."""
    H, G = q.shape[0], q.shape[0] // k.shape[0]
    bf16 = q.dtype == torch.bfloat16
    do, q, k, v = dout.double(), q.double(), k.double().repeat_interleave(G, 0), v.double().repeat_interleave(G, 0)
    x = torch.where(seen, q @ k.transpose(1, 2) * scale, -math.inf)
    size = torch.where(seen, q.abs() @ k.abs().transpose(1, 2) * scale, 0).amax((1, 2), keepdim=True)
    top = x.amax(-1, keepdim=True)
    p = torch.where(seen, (x - torch.where(top == -math.inf, 0, top)).exp(), 0)
    s = p.sum(-1, keepdim=True)
    p = torch.where(s > 0, p / s, 0)
    o = p @ v
    D, absD = (do * o).sum(-1, keepdim=True), (do * o).abs().sum(-1, keepdim=True)
    ds = p * (do @ v.transpose(1, 2) - D)
    absds = p * (do.abs() @ v.abs().transpose(1, 2) + absD)
    half = torch.finfo(torch.bfloat16).eps / 2
    eP = 2.0 ** -17 * (2 + size) + (half if bf16 else 0)
    # dS's own rounding is of dS; what comes from P, dP and D is of the terms
    eS = 2.0 ** -17 * (2 + size) * absds + (half * (ds.abs() + p * absD) if bf16 else 0)
    fold = lambda t: t.view(H // G, G, *t.shape[1:]).sum(1)  # noqa: E731
    want = (ds @ k * scale, fold(ds.transpose(1, 2) @ q) * scale, fold(p.transpose(1, 2) @ do))
    slack = (eS @ k.abs() * scale, fold(eS.transpose(1, 2) @ q.abs()) * scale, fold((eP * p).transpose(1, 2) @ do.abs()))
    return want, slack


def check(got, want, slack, keep=None):
    for g, w, s in zip(got, want, slack):
        eps = torch.finfo(g.dtype).eps / 2
        err, bound = (g.double() - w).abs(), 1.02 * s + eps * (w.abs() + s) + 1e-30
        assert g.shape == w.shape and bool((err <= bound).all()), float((err - bound).max())


@pytest.mark.parametrize("H,K,N,M,window,sinks,frame,q_start,dtype,layout", CASES)
def test_backward(B, H, K, N, M, window, sinks, frame, q_start, dtype, layout):  # noqa: F811
    q, k, v = draw(H, K, N, M, TYPES[dtype], layout=layout)
    dout = draw(H, K, N, M, TYPES[dtype], seed=99)[0]
    what = dict(window=window, sinks=sinks, frame=frame, q_start=q_start)
    out, lse = B.bsga_window_attn(q, k, v, return_lse=True, **what)
    got = B.bsga_window_attn_bwd(dout, q, k, v, out, lse, **what)
    seen = seen_by(N, M, window, sinks, frame, q_start)
    check(got, *gradients(dout, q, k, v, seen, 0.125))
    unseen = ~seen.any(0)
    assert bool((got[1][:, unseen] == 0).all()) and bool((got[2][:, unseen] == 0).all())
    assert all(torch.equal(x, y) for x, y in zip(got, B.bsga_window_attn_bwd(dout, q, k, v, out, lse, **what)))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_many_queries_of_the_first_tokens(B, dtype):  # noqa: F811
    """Few first tokens that every query sees: their queries are dealt out to many workgroups."""
    N = 6000 if dtype == "bf16" else 2500
    q, k, v = draw(2, 1, N, N, TYPES[dtype])
    dout = draw(2, 1, N, N, TYPES[dtype], seed=3)[0]
    out, lse = B.bsga_window_attn(q, k, v, window=200, sinks=130, return_lse=True)
    got = B.bsga_window_attn_bwd(dout, q, k, v, out, lse, window=200, sinks=130)
    check(got, *gradients(dout, q, k, v, seen_by(N, N, 200, 130, 1, None), 0.125))


@pytest.mark.parametrize("K", [4, 1])
def test_against_differences(B, K):  # noqa: F811
    """The slope of sum(dout o) along random directions, from the definition in float64 a step of 1e-6 to either side: off by the third
    derivative times 1e-12 and by rounding, 2^-52 / 1e-6 of the sum's terms.  The gradient's own bound is 2^-17 (2 + L) of the terms, see above."""
    H, N = 4, 150
    q, k, v = draw(H, K, N, N, torch.float32)
    dout = draw(H, K, N, N, torch.float32, seed=5)[0]
    out, lse = B.bsga_window_attn(q, k, v, window=40, sinks=3, return_lse=True)
    grads = B.bsga_window_attn_bwd(dout, q, k, v, out, lse, window=40, sinks=3)
    seen = seen_by(N, N, 40, 3, 1, None)
    g = torch.Generator(device="cuda").manual_seed(1)
    along = [torch.randn(t.shape, generator=g, device="cuda").double() for t in (q, k, v)]

    def loss(step):
        a, b, c = (t.double() + step * z for t, z in zip((q, k, v), along))
        b, c = b.repeat_interleave(H // K, 0), c.repeat_interleave(H // K, 0)
        p = (a @ b.transpose(1, 2) / 8).masked_fill(~seen, -math.inf).softmax(-1)
        return (p @ c * dout.double()).sum(), (p @ c * dout.double()).abs().sum()

    slope = float((loss(1e-6)[0] - loss(-1e-6)[0]) / 2e-6)
    mine = float(sum((x.double() * z).sum() for x, z in zip(grads, along)))
    _, slack = gradients(dout, q, k, v, seen, 0.125)
    allowed = float(sum((s * z.abs()).sum() for s, z in zip(slack, along)))
    assert abs(slope - mine) <= allowed + 1e-8 * float(loss(0)[1])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_values_in_masked_places(B, dtype, bad):  # noqa: F811
    """A key that is not a number reaches the gradients of the queries that see it, and through them those of the keys that these see; a query that is not,
    those of the keys that it sees."""
    N = 500
    q, k, v = draw(2, 2, N, N, TYPES[dtype])
    dout = draw(2, 2, N, N, TYPES[dtype], seed=3)[0]
    seen = seen_by(N, N, 70, 0, 1, None)
    q, k, v = q.clone(), k.clone(), v.clone()
    clean = [t.clone() for t in (q, k, v)]
    k[0, 200], v[1, 200], q[0, 400] = bad, bad, bad
    out, lse = B.bsga_window_attn(q, k, v, window=70, return_lse=True)
    got = B.bsga_window_attn_bwd(dout, q, k, v, out, lse, window=70)
    want, slack = gradients(dout, *clean, seen, 0.125)
    hit = seen[:, 200].clone()
    hit[400] = True
    keys_hit = seen[hit].any(0)
    assert not bool(hit.all()) and not bool(keys_hit.all())
    check([got[0][:, ~hit], got[1][:, ~keys_hit], got[2][:, ~keys_hit]],
          [want[0][:, ~hit], want[1][:, ~keys_hit], want[2][:, ~keys_hit]], [slack[0][:, ~hit], slack[1][:, ~keys_hit], slack[2][:, ~keys_hit]])


def test_no_queries_and_no_keys(B):  # noqa: F811
    q, k, v = draw(2, 2, 70, 70, torch.bfloat16)
    none = q[:, :0].contiguous()
    dq, dk, dv = B.bsga_window_attn_bwd(none, q[:, :0], k, v, none, torch.empty((2, 0), device="cuda"))
    assert dq.shape == (2, 0, 64) and bool((dk == 0).all()) and bool((dv == 0).all())
    o, lse = B.bsga_window_attn(q, k[:, :0], v[:, :0], q_start=0, return_lse=True)
    dq, dk, dv = B.bsga_window_attn_bwd(q, q, k[:, :0], v[:, :0], o, lse, q_start=0)
    assert bool((dq == 0).all()) and dk.shape == (2, 0, 64)


def test_a_graph(B):  # noqa: F811
    q, k, v = draw(4, 2, 900, 900, torch.bfloat16)
    dout = draw(4, 2, 900, 900, torch.bfloat16, seed=3)[0]

    def step():
        out, lse = B.bsga_window_attn(q, k, v, window=300, sinks=4, return_lse=True)
        return B.bsga_window_attn_bwd(dout, q, k, v, out, lse, window=300, sinks=4)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(4):
        q.mul_(1.0 + 0.25 * i)
        dout.neg_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, step()))
