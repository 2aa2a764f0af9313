"""Guard bytes around every output and workspace of the streamed attention layer's entry points: lengths that end inside tiles, pages and workgroups,
launches whole and in parts."""
import pytest
import torch

from tests.test_gpu_canaries import B, Guarded  # noqa: F401

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float32]


def ptr(x):
    return None if x is None else (x.view if isinstance(x, Guarded) else x).data_ptr()


def whole(*outs):
    torch.cuda.synchronize()
    for x in outs:
        assert x.intact(), "guard bytes were overwritten"


def room(n):
    return Guarded((max(n, 16),), torch.uint8)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,H,K,axes", [(1, 1, 1, 1), (77, 6, 2, 2), (1031, 4, 4, 1)])
def test_norm_and_rotation(B, N, H, K, axes, dtype):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(N)
    x = torch.randn((N, H + 2 * K, 64), device="cuda", generator=g).to(dtype)
    q, k, v = x[:, :H], x[:, H:H + K], x[:, H + K:]
    w = [torch.randn(64, device="cuda", generator=g).to(dtype) for _ in range(2)]
    positions = torch.randint(0, 5000, (N, axes), device="cuda", generator=g).int()
    code, t, st = int(dtype == torch.float32), x.stride(0), torch.cuda.current_stream().cuda_stream
    outs = [Guarded((h, N, 64), dtype) for h in (H, K, K)]
    assert B.lib.bsga_qk_norm_rope(ptr(q), ptr(k), ptr(v), t, 64, t, 64, t, 64, code, N, H, K, 64, 1, 1e-6, ptr(w[0]), None, ptr(w[1]), None,
                                   ptr(positions), axes, 10000.0, None, 0, 0, *map(ptr, outs), st) == 0
    whole(*outs)

    page = 16  # into the pages of a cache, with slots past its end
    pages = -(-N // page) + 1
    caches = [Guarded((pages, K, page, 64), dtype) for _ in range(2)]
    slots = torch.randperm(pages * page, device="cuda", generator=g)[:N].int()
    slots[0] = pages * page
    slots[-1] = -1
    q_out = Guarded((H, N, 64), dtype)
    assert B.lib.bsga_qk_norm_rope(ptr(q), ptr(k), ptr(v), t, 64, t, 64, t, 64, code, N, H, K, 64, 1, 1e-6, ptr(w[0]), None, ptr(w[1]), None,
                                   ptr(positions), axes, 10000.0, ptr(slots), pages, page, ptr(q_out), *map(ptr, caches), st) == 0
    whole(q_out, *caches)

    grads = [Guarded((N, h, 64), dtype) for h in (H, K, K)]
    d_weights, space = Guarded((4, 64), torch.float32), room(B.lib.bsga_qk_norm_rope_bwd_workspace_bytes(N, H, K))
    dq, dk, dv = (torch.randn((h, N, 64), device="cuda", generator=g).to(dtype) for h in (H, K, K))
    assert B.lib.bsga_qk_norm_rope_bwd(ptr(dq), ptr(dk), ptr(dv), ptr(q), ptr(k), t, 64, t, 64, code, N, H, K, 64, 1, 1e-6, ptr(w[0]), ptr(w[1]),
                                       ptr(positions), axes, 10000.0, *map(ptr, grads), H * 64, 64, K * 64, 64, K * 64, 64, ptr(d_weights),
                                       ptr(space), space.n, st) == 0
    whole(*grads, d_weights, space)
    assert all(bool(x.view.float().isfinite().all()) for x in outs + grads + [d_weights])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,K,N,M,frame,window,sinks,start", [(1, 1, 1, 1, 1, 0, 0, 0), (4, 2, 33, 1999, 1, 500, 4, 1966), (2, 1, 611, 611, 129, 2, 7, 0),
                                                             (1, 1, 5, 9000, 1, 0, 0, 8995), (3, 3, 300, 200, 10, 3, 0, -100)])
def test_attention_with_a_window(B, H, K, N, M, frame, window, sinks, start, dtype):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(N)
    q, dout = (torch.randn((H, N, 64), device="cuda", generator=g).to(dtype) for _ in range(2))
    k, v = (torch.randn((K, M, 64), device="cuda", generator=g).to(dtype) for _ in range(2))
    code, st = int(dtype == torch.float32), torch.cuda.current_stream().cuda_stream
    seen = (start, frame, window, sinks)
    strides = (64, N * 64, 64, M * 64, 64, M * 64)
    out, lse = Guarded((H, N, 64), dtype), Guarded((H, N), torch.float32)
    space = room(B.lib.bsga_window_attn_workspace_bytes(code, H, N, M, *seen))
    for x in (space, None):
        assert B.lib.bsga_window_attn(ptr(q), ptr(k), ptr(v), *strides, code, H, K, N, M, 64, 0.125, *seen, ptr(out), ptr(lse), ptr(x),
                                      0 if x is None else x.n, st) == 0
        whole(out, lse, space)
    grads = [Guarded((h, n, 64), dtype) for h, n in ((H, N), (K, M), (K, M))]
    space = room(B.lib.bsga_window_attn_bwd_workspace_bytes(code, H, K, N, M, *seen))
    assert B.lib.bsga_window_attn_bwd(ptr(dout), ptr(q), ptr(k), ptr(v), *strides, ptr(out), ptr(lse), code, H, K, N, M, 64, 0.125, *seen,
                                      *map(ptr, grads), ptr(space), space.n, st) == 0
    whole(*grads, space)
    assert all(bool(x.view.float().isfinite().all()) for x in grads + [out])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths,H,K,page,window,sinks", [((1,), 1, 1, 16, 0, 0), ((0, 17, 1000, 333), 6, 2, 16, 0, 0), ((5000, 4999), 16, 2, 64, 0, 0),
                                                          ((700, 90), 4, 4, 32, 128, 4)])
def test_attention_over_pages(B, lengths, H, K, page, window, sinks, dtype):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(H)
    n, width = len(lengths), max(-(-x // page) for x in lengths) + 1
    pages = n * width
    kc, vc = (torch.randn((pages, K, page, 64), device="cuda", generator=g).to(dtype) for _ in range(2))
    table = torch.randperm(pages, device="cuda", generator=g).int().view(n, width)
    q = torch.randn((n, H, 64), device="cuda", generator=g).to(dtype)
    code, st = int(dtype == torch.float32), torch.cuda.current_stream().cuda_stream
    out, lse = Guarded((n, H, 64), dtype), Guarded((n, H), torch.float32)
    space = room(B.lib.bsga_paged_attn_workspace_bytes(code, n, H, K, width, pages, page, 1, window, sinks))
    known = torch.tensor(lengths, dtype=torch.int32).cuda()
    assert B.lib.bsga_paged_attn(ptr(q), H * 64, 64, ptr(kc), ptr(vc), code, n, H, K, 64, ptr(table), width, ptr(known), pages, page, 0.125, 1, window,
                                 sinks, ptr(out), ptr(lse), ptr(space), space.n, st) == 0
    whole(out, lse, space)
    assert bool(out.view.float().isfinite().all())
