"""What the operators on caches in 8 bits and on shared prefixes refuse, and what workspaces they ask for, before anything is launched: no GPU is needed."""
import pytest
import torch

from tests.test_norm_rope_refusals import A, B, _err, _OnDevice  # noqa: F401

E4M3 = torch.float8_e4m3fn


def test_norm_and_rotation(B):  # noqa: F811
    def call(q=A, k=A, v=A, st=(64, 64) * 3, dt=0, n=100, h=4, kh=2, d=64, norm=1, eps=1e-6, qw=A, qb=None, kw=A, kb=None, pos=A, axes=1,
             base=1e4, slots=A, pages=10, page=16, qo=A, kr=A, vr=A, kc=A, vc=A, ks=A, vs=A):
        return B.lib.bsga_qk_norm_rope_e4m3(q, k, v, *st, dt, n, h, kh, d, norm, eps, qw, qb, kw, kb, pos, axes, base, slots, pages, page, qo, kr, vr, kc,
                                            vc, ks, vs, None)

    assert call(dt=2) == 1 and "dtype" in _err(B)
    assert call(d=128) == 2 and "head_dim" in _err(B)
    assert call(n=-1) == 1 and call(n=(1 << 24) + 1) == 1 and "n_tokens" in _err(B)
    assert call(q=None, k=None, v=None, qo=None, kr=None, vr=None) == 1 and "nothing to do" in _err(B)
    assert call(qo=None) == 1 and call(k=None) == 1 and "go with their inputs" in _err(B)
    for name in ("kc", "vc", "ks", "vs"):
        assert call(**{name: None}) == 1 and "its cache" in _err(B)
    assert call(k=None, kr=None) == 1 and "its cache" in _err(B)
    assert call(kr=A + 8) == 1 and "outputs" in _err(B)
    assert call(vc=A + 8) == 1 and "caches" in _err(B)
    assert call(slots=None) == 1 and "slots" in _err(B)
    assert call(page=0) == 1 and call(pages=0) == 1 and call(pages=1 << 27) == 1 and "2^31" in _err(B)
    assert call(st=(64, 64, 60, 64, 64, 64)) == 1 and "16 bytes" in _err(B)
    assert call(norm=2, kb=A + 4) == 1 and "aligned" in _err(B)
    assert call(n=0) == 0 and call(n=0, kr=None, vr=None, slots=None) == 0


def test_reading_back(B):  # noqa: F811
    def call(k=A, v=A, ks=A, vs=A, cdt=2, pages=20, page=16, kh=2, d=64, table=A, width=10, first=0, n=100, dt=0, ko=A, vo=A, kst=6400, vst=6400):
        return B.lib.bsga_cache_load(k, v, ks, vs, cdt, pages, page, kh, d, table, width, first, n, dt, ko, vo, kst, vst, None)

    assert call(dt=2) == 1 and "dtype" in _err(B)
    assert call(cdt=1) == 1 and call(cdt=0, dt=1) == 1 and call(cdt=3) == 1 and "8 bits or" in _err(B)
    assert call(d=32) == 2 and "head_dim" in _err(B)
    assert call(kh=0) == 1 and call(kh=32768) == 1 and "kv_heads" in _err(B)
    assert call(page=0) == 1 and call(page=65537) == 1 and "page" in _err(B)
    assert call(pages=-1) == 1 and "n_pages" in _err(B)
    assert call(width=-1) == 1 and call(width=1 << 27) == 1 and "2^30" in _err(B)
    for first, n in ((-1, 5), (0, -1), (0, 161), (100, 61), (161, 0), (1 << 62, 1), (1, (1 << 63) - 1)):
        assert call(first=first, n=n) == 1 and "do not lie" in _err(B)
    for name in ("k", "v", "table", "ko", "vo"):
        assert call(**{name: None}) == 1 and "non-null" in _err(B)
    assert call(ks=None) == 1 and call(vs=None) == 1 and "scale" in _err(B)
    assert call(k=A + 8) == 1 and call(vo=A + 8) == 1 and "aligned" in _err(B)
    assert call(kst=60) == 1 and call(vst=-64) == 1 and "strides" in _err(B)
    assert call(kst=6336) == 1 and call(vst=0) == 1 and "overlap" in _err(B)
    assert call(n=0) == 0 and call(first=160, n=0) == 0


def _paged(B, **kw):  # noqa: F811
    a = dict(q=A, st=(256, 64), k=A, v=A, ks=A, vs=A, dt=0, b=3, h=4, kh=2, d=64, table=A, width=10, lengths=A, pages=20, page=16, scale=0.125, frame=1, window=0,
             sinks=0, out=A, ws=A, wsb=1 << 40)
    assert set(kw) <= set(a)
    a.update(kw)
    return B.lib.bsga_paged_attn_e4m3(a["q"], *a["st"], a["k"], a["v"], a["ks"], a["vs"], a["dt"], a["b"], a["h"], a["kh"], a["d"], a["table"], a["width"],
                                      a["lengths"], a["pages"], a["page"], a["scale"], a["frame"], a["window"], a["sinks"], a["out"], None, a["ws"],
                                      a["wsb"], None)


def _prefix(B, **kw):  # noqa: F811
    a = dict(q=A, st=(256, 64), k=A, v=A, ks=A, vs=A, dt=0, cdt=2, b=3, h=4, kh=2, d=64, table=A, width=10, lengths=A, pt=A, pw=50, pl=A, starts=A, n=2, pages=20,
             page=16, scale=0.125, frame=1, window=0, sinks=0, out=A, ws=A, wsb=1 << 40)
    assert set(kw) <= set(a)
    a.update(kw)
    return B.lib.bsga_prefix_attn(a["q"], *a["st"], a["k"], a["v"], a["ks"], a["vs"], a["dt"], a["cdt"], a["b"], a["h"], a["kh"], a["d"], a["table"], a["width"],
                                  a["lengths"], a["pt"], a["pw"], a["pl"], a["starts"], a["n"], a["pages"], a["page"], a["scale"], a["frame"], a["window"],
                                  a["sinks"], a["out"], None, a["ws"], a["wsb"], None)


@pytest.mark.parametrize("of", [_paged, _prefix])
def test_attention(B, of):  # noqa: F811
    def call(**kw):
        return of(B, **kw)

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
    assert call(ks=None) == 1 and call(vs=None) == 1 and "scale" in _err(B)
    assert call(out=None) == 1 and call(k=A + 8) == 1 and "aligned" in _err(B)
    assert call(width=1000, wsb=100) == 3 and call(width=1000, ws=None) == 3 and "needed" in _err(B)
    assert call(ws=A + 4) == 1 and "aligned" in _err(B)
    assert call(b=0) == 0


def test_prefixes(B):  # noqa: F811
    assert _prefix(B, cdt=1) == 1 and _prefix(B, cdt=0, dt=1) == 1 and _prefix(B, cdt=7) == 1 and "8 bits or" in _err(B)
    assert _prefix(B, n=-1) == 1 and _prefix(B, n=65536) == 1 and "prefixes" in _err(B)
    assert _prefix(B, pw=-1) == 1 and _prefix(B, pw=(1 << 26) - 9) == 1 and "2^30" in _err(B)
    for name in ("pt", "pl", "starts"):
        assert _prefix(B, **{name: None}) == 1 and "non-null" in _err(B)
    assert _prefix(B, b=65535, h=65535, kh=1) == 2 and "too many" in _err(B)
    assert _prefix(B, b=65535, width=1 << 20, page=1, pages=1 << 30, h=16, kh=16) == 2 and "one launch" in _err(B)
    for scale in (2.0 ** -101, 1e-45, float("inf")):
        assert _prefix(B, scale=scale) == 1 and "softmax_scale" in _err(B)


def test_workspaces(B):  # noqa: F811
    f, g = B.lib.bsga_paged_attn_e4m3_workspace_bytes, B.lib.bsga_prefix_attn_workspace_bytes
    assert f(0, 0, 4, 2, 10, 20, 16, 1, 0, 0) == 0 and f(5, 3, 4, 2, 10, 20, 16, 1, 0, 0) == 0
    assert g(0, 2, 0, 4, 2, 10, 1, 10, 20, 16, 1, 0, 0) == 0 and g(0, 1, 3, 4, 2, 10, 1, 10, 20, 16, 1, 0, 0) == 0
    for batch in (1, 3, 4096, 16000):
        for width, page in ((0, 16), (1, 1), (1 << 20, 16), (1 << 13, 65536), (300, 1374), (1 << 29, 1)):
            for seen in ((1, 0, 0), (1, 1, 0), (1374, 8, 1374), (1 << 24, 1 << 60, 1 << 60)):
                # 65 numbers for each row and stretch, and a stretch is 128 keys at least
                most = 65 * 4 * batch * 16 * (width * page // 128 + 1)
                assert 0 <= f(0, batch, 16, 4, width, 100, page, *seen) <= most
                assert 0 < g(0, 2, batch, 16, 4, width, 3, width, 100, page, *seen) <= 2 * most


def test_tensors(B):  # noqa: F811
    t = _OnDevice
    c, s, i = t((20, 2, 16, 64), E4M3), t((20, 2, 16), torch.uint8), lambda *shape: t(shape, torch.int32)  # noqa: E731
    q, x = t((3, 4, 64)), t((7, 2, 64))

    def store(q=t((7, 4, 64)), k=x, v=x, kc=c, vc=c, ks=s, vs=s, slots=i(7)):
        return B.bsga_qk_norm_rope_e4m3(q, k, v, kc, vc, ks, vs, slots)

    for kw, error, text in ((dict(k=t((7, 2, 64), torch.float16)), TypeError, "unsupported dtype"), (dict(v=t((6, 2, 64))), ValueError, "v must"),
                            (dict(q=t((7, 4, 64), torch.float32)), TypeError, "q must"), (dict(slots=i(8)), ValueError, "slots"),
                            (dict(slots=t((7,), torch.int64)), TypeError, "slots"), (dict(kc=t((20, 2, 16, 64))), TypeError, "k_cache"),
                            (dict(vc=t((20, 2, 8, 64), E4M3)), ValueError, "v_cache"), (dict(kc=t((20, 3, 16, 64), E4M3), vc=t((20, 3, 16, 64), E4M3)), ValueError, "k_cache"),
                            (dict(ks=t((20, 2, 16), torch.int8)), TypeError, "k_scale"), (dict(vs=t((20, 2, 8), torch.uint8)), ValueError, "v_scale"),
                            (dict(vs=None), ValueError, "v_scale"), (dict(kc=t((20, 2, 16, 64), E4M3, index=1)), ValueError, "k_cache")):
        with pytest.raises(error, match=text):
            store(**kw)

    load = B.bsga_cache_load
    with pytest.raises(ValueError, match="k_scale"):
        load(c, c, i(5), 10)
    with pytest.raises(TypeError, match="pages"):
        load(c, c, t((5,), torch.int64), 10, 0, s, s)
    with pytest.raises(ValueError, match="pages must"):
        load(c, c, i(1, 5), 10, 0, s, s)
    with pytest.raises(TypeError, match="unsupported dtype"):
        load(c, c, i(5), 10, 0, s, s, dtype=torch.float16)
    with pytest.raises(TypeError, match="as it is"):
        load(t((20, 2, 16, 64)), t((20, 2, 16, 64)), i(5), 10, dtype=torch.float32)
    with pytest.raises(ValueError, match="scales go with"):
        load(t((20, 2, 16, 64)), t((20, 2, 16, 64)), i(5), 10, 0, s, s)
    with pytest.raises(ValueError, match=r"out\[1\]"):
        load(c, c, i(5), 10, 0, s, s, out=(t((2, 10, 64)), t((2, 11, 64))))
    with pytest.raises(TypeError, match=r"out\[1\]"):
        load(c, c, i(5), 10, 0, s, s, out=(t((2, 10, 64)), t((2, 10, 64), torch.float32)))

    paged = B.bsga_paged_attn_e4m3
    with pytest.raises(TypeError, match="k_cache"):
        paged(q, t((20, 2, 16, 64)), c, s, s, i(3, 10), i(3))
    with pytest.raises(ValueError, match="k_scale"):
        paged(q, c, c, None, s, i(3, 10), i(3))
    with pytest.raises(ValueError, match="lengths"):
        paged(q, c, c, s, s, i(3, 10), i(2))
    with pytest.raises(ValueError, match="page_table"):
        paged(q, c, c, s, s, i(30), i(3))
    with pytest.raises(ValueError, match="window"):
        paged(q, c, c, s, s, i(3, 10), i(3), window=0)
    with pytest.raises(ValueError, match="contiguous rows"):
        paged(t((3, 4, 64, 1)), c, c, s, s, i(3, 10), i(3))

    def prefix(q=q, c=c, pt=i(2, 5), pl=i(2), st=i(3), **kw):
        return B.bsga_prefix_attn(q, c, c, i(3, 10), i(3), pt, pl, st, **kw)

    scales = dict(k_scale=s, v_scale=s)
    for kw, error, text in ((dict(), ValueError, "k_scale"), (dict(c=t((20, 2, 16, 64)), **scales), ValueError, "scales go with"),
                            (dict(c=t((20, 2, 16, 64), torch.float32)), TypeError, "k_cache"), (dict(pt=i(5), **scales), ValueError, "prefix_table"),
                            (dict(pl=i(3), **scales), ValueError, "prefix_lengths"), (dict(st=i(2), **scales), ValueError, "starts"),
                            (dict(st=t((3,), torch.int64), **scales), TypeError, "starts"), (dict(window=0, **scales), ValueError, "window")):
        with pytest.raises(error, match=text):
            prefix(**kw)


def test_another_device_and_workspaces(B, monkeypatch):  # noqa: F811
    t = _OnDevice
    c, s, i, x = t((20, 2, 16, 64), E4M3), t((20, 2, 16), torch.uint8), lambda *shape: t(shape, torch.int32), t((3, 2, 64))  # noqa: E731

    def store():
        B.bsga_qk_norm_rope_e4m3(x, x, x, c, c, s, s, i(3))

    def load():
        B.bsga_cache_load(c, c, i(5), 10, 0, s, s)

    def paged(**kw):
        B.bsga_paged_attn_e4m3(t((3, 4, 64)), c, c, s, s, i(3, 10), i(3), **kw)

    def prefix(**kw):
        B.bsga_prefix_attn(t((3, 4, 64)), c, c, i(3, 10), i(3), i(2, 5), i(2), i(3), s, s, **kw)

    for call in (paged, prefix):
        scattered = t((1 << 10, 1 << 10), torch.uint8).t()
        scattered.index_ = 0
        for workspace in (torch.empty(1 << 20, dtype=torch.uint8), t((1 << 20,), torch.uint8, index=1), scattered):
            with pytest.raises(ValueError, match="workspace must"):
                call(workspace=workspace)
    monkeypatch.setattr(B.binding, "_current_device", lambda: 1)
    for call in (store, load, paged, prefix):
        with pytest.raises(ValueError, match="current device"):
            call()
