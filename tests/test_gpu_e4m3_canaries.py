"""Guard bytes around every output and workspace of the entry points on caches in 8 bits and shared prefixes: lengths that end inside tiles, pages and workgroups."""
import pytest
import torch

from tests.test_gpu_canaries import B, Guarded  # noqa: F401
from tests.test_gpu_e4m3 import cached
from tests.test_gpu_stream_canaries import TYPES, ptr, room, whole

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,H,K,axes", [(1, 1, 1, 1), (77, 6, 2, 2), (1031, 4, 4, 1)])
def test_norm_and_rotation_and_back(B, N, H, K, axes, dtype):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(N)
    x = torch.randn((N, H + 2 * K, 64), device="cuda", generator=g).to(dtype)
    q, k, v = x[:, :H], x[:, H:H + K], x[:, H + K:]
    positions = torch.randint(0, 5000, (N, axes), device="cuda", generator=g).int()
    code, t, st = int(dtype == torch.float32), x.stride(0), torch.cuda.current_stream().cuda_stream
    page = 16
    pages = -(-N // page) + 1
    caches = [Guarded((pages, K, page, 64), torch.uint8) for _ in range(2)]
    scales = [Guarded((pages, K, page), torch.uint8) for _ in range(2)]
    slots = torch.randperm(pages * page, device="cuda", generator=g)[:N].int()
    slots[0] = pages * page
    slots[-1] = -1
    outs = [Guarded((h, N, 64), dtype) for h in (H, K, K)]
    assert B.lib.bsga_qk_norm_rope_e4m3(ptr(q), ptr(k), ptr(v), t, 64, t, 64, t, 64, code, N, H, K, 64, 1, 1e-6, None, None, None, None, ptr(positions), axes,
                                        10000.0, ptr(slots), pages, page, *map(ptr, outs), *map(ptr, caches), *map(ptr, scales), st) == 0
    whole(*outs, *caches, *scales)
    assert all(bool(x.view.float().isfinite().all()) for x in outs)
    table = torch.arange(pages, device="cuda").int()
    back = [Guarded((K, N, 64), dtype) for _ in range(2)]
    assert B.lib.bsga_cache_load(*map(ptr, caches), *map(ptr, scales), 2, pages, page, K, 64, ptr(table), pages, 0, N, code, *map(ptr, back), N * 64, N * 64,
                                 st) == 0
    whole(*back)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths,scans,starts,H,K,page,window,sinks", [((1,), (1,), (0, 1), 1, 1, 16, 0, 0), ((0, 17, 1000, 333), (70,), (1, 3), 6, 2, 16, 0, 0),
                                                                       ((50, 49) * 50, (5000,), (0, 100), 16, 2, 64, 0, 0),
                                                                       ((700, 90, 3), (600, 3), (0, 2, 3), 4, 4, 32, 128, 4)])
def test_attention(B, lengths, scans, starts, H, K, page, window, sinks, dtype):  # noqa: F811
    kc, vc, ks, vs, table, _ = cached(list(lengths) + list(scans), K, page)
    n, code, st = len(lengths), int(dtype == torch.float32), torch.cuda.current_stream().cuda_stream
    q = torch.randn((n, H, 64), device="cuda", generator=torch.Generator(device="cuda").manual_seed(H)).to(dtype)
    out, lse = Guarded((n, H, 64), dtype), Guarded((n, H), torch.float32)
    own, scan, of, begin = table[:n].contiguous(), table[n:].contiguous(), *(torch.tensor(x, dtype=torch.int32).cuda() for x in (lengths, starts))
    sizes = torch.tensor(scans, dtype=torch.int32).cuda()
    width, pages = table.shape[1], kc.shape[0]
    space = room(B.lib.bsga_paged_attn_e4m3_workspace_bytes(code, n, H, K, width, pages, page, 1, window, sinks))
    assert B.lib.bsga_paged_attn_e4m3(ptr(q), H * 64, 64, ptr(kc), ptr(vc), ptr(ks), ptr(vs), code, n, H, K, 64, ptr(own), width, ptr(of), pages, page, 0.125, 1,
                                      window, sinks, ptr(out), ptr(lse), ptr(space), space.n, st) == 0
    whole(out, lse, space)
    assert bool(out.view.float().isfinite().all())
    space = room(B.lib.bsga_prefix_attn_workspace_bytes(code, 2, n, H, K, width, len(scans), width, pages, page, 1, window, sinks))
    assert B.lib.bsga_prefix_attn(ptr(q), H * 64, 64, ptr(kc), ptr(vc), ptr(ks), ptr(vs), code, 2, n, H, K, 64, ptr(own), width, ptr(of), ptr(scan), width, ptr(sizes),
                                  ptr(begin), len(scans), pages, page, 0.125, 1, window, sinks, ptr(out), ptr(lse), ptr(space), space.n, st) == 0
    whole(out, lse, space)
    assert bool(out.view.float().isfinite().all())
