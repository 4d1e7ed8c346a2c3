"""Host-side checks of the paged cache's entry points and of windowed prompts: refusals and empty calls, without a GPU."""
import ctypes
import os

import pytest
import torch

import paper_2506_19505_amd as antkv
from paper_2506_19505_amd.binding import _Geom

OK, EINVAL, EUNSUPPORTED, EWORKSPACE = 0, 1, 2, 3
FAKE, OTHER, ODD = (ctypes.c_void_p(x) for x in (4096, 8192, 4098))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(antkv.lib_path()):
        from paper_2506_19505_amd.build import build
        build()
    return antkv.load_library()


def _g(B=2, Hq=8, Hkv=2, D=128, d=8, C=256):
    return _Geom(B, Hq, Hkv, D, d, C)


# every call below is refused before anything is enqueued, or has nothing to do

def _map(lib, R=2, held=FAKE, new=FAKE, table=FAKE, cap=4, n_pages=8, page=16, free=FAKE, n_free=8, at=None, T=4, ctx=OTHER, qs=FAKE,
         slot=FAKE, status=FAKE):
    return lib.antkv_page_map(R, held, new, table, cap, n_pages, page, free, n_free, at, T, ctx, qs, slot, status, None)


@pytest.mark.parametrize("bad,code", [
    (dict(page=8), EUNSUPPORTED), (dict(page=48), EUNSUPPORTED), (dict(page=512), EUNSUPPORTED), (dict(page=0), EINVAL),
    (dict(page=-16), EINVAL), (dict(n_pages=0), EINVAL), (dict(n_pages=1 << 27, page=16), EINVAL), (dict(R=-1), EINVAL), (dict(R=8193), EUNSUPPORTED),
    (dict(cap=0), EINVAL), (dict(cap=(1 << 26) + 1, page=16), EINVAL), (dict(n_free=-1), EINVAL), (dict(T=-1), EINVAL), (dict(T=1 << 31), EINVAL),
    (dict(held=None), EINVAL), (dict(new=None), EINVAL), (dict(table=None), EINVAL), (dict(free=None), EINVAL), (dict(ctx=None), EINVAL),
    (dict(qs=None), EINVAL), (dict(slot=None), EINVAL), (dict(status=None), EINVAL), (dict(at=FAKE), EINVAL), (dict(ctx=FAKE), EINVAL)])
def test_page_map_refusals(lib, bad, code):
    assert _map(lib, **bad) == code


def _store(lib, g=None, k=FAKE, v=OTHER, xt=256, xh=128, T=4, slot=FAKE, kp=FAKE, vp=OTHER, n_pages=8, page=16):
    return lib.antkv_page_store(ctypes.byref(g or _g()), k, v, xt, xh, T, slot, kp, vp, n_pages, page, None)


@pytest.mark.parametrize("bad,code", [
    (dict(g=_g(D=64)), EUNSUPPORTED), (dict(g=_g(Hq=16)), EUNSUPPORTED), (dict(page=24), EUNSUPPORTED), (dict(n_pages=0), EINVAL), (dict(T=-1), EINVAL),
    (dict(T=1 << 30), EINVAL), (dict(k=None), EINVAL), (dict(v=ODD), EINVAL), (dict(slot=None), EINVAL), (dict(vp=FAKE), EINVAL), (dict(xt=255), EINVAL),
    (dict(xh=-128), EINVAL), (dict(T=0, k=None), OK)])
def test_page_store_refusals(lib, bad, code):
    assert _store(lib, **bad) == code


def _load(lib, g=None, kp=FAKE, vp=FAKE, n_pages=8, page=16, table=FAKE, cap=4, ctx=None, first=0, N=8, k=FAKE, v=OTHER, xb=2048, xh=1024, xt=128):
    return lib.antkv_page_load(ctypes.byref(g or _g()), kp, vp, n_pages, page, table, cap, ctx, first, N, k, v, xb, xh, xt, None)


@pytest.mark.parametrize("bad,code", [
    (dict(N=65), EINVAL), (dict(first=60, N=5), EINVAL), (dict(first=-1), EINVAL), (dict(first=65, N=0), EINVAL), (dict(N=-1), EINVAL), (dict(page=0), EINVAL),
    (dict(page=20), EUNSUPPORTED), (dict(cap=0), EINVAL), (dict(table=None), EINVAL), (dict(kp=None), EINVAL), (dict(v=FAKE), EINVAL), (dict(k=ODD), EINVAL),
    (dict(xt=64), EINVAL), (dict(xb=4), EINVAL), (dict(N=0, k=None), OK), (dict(first=64, N=0), OK), (dict(g=_g(B=0)), OK)])
def test_page_load_refusals(lib, bad, code):
    assert _load(lib, **bad) == code


def _attn(lib, g=None, q=FAKE, qt=1024, qh=128, T=4, qs=FAKE, ctx=FAKE, table=FAKE, cap=4, kp=FAKE, vp=FAKE, n_pages=8, page=16, scale=0.1, window=0,
          sink=0, out=FAKE, rm=None, rs=None, ws=FAKE, wsb=1 << 40):
    return lib.antkv_page_attn(ctypes.byref(g or _g()), q, qt, qh, T, qs, ctx, table, cap, kp, vp, n_pages, page, scale, window, sink, out, rm, rs, ws,
                               wsb, None)


@pytest.mark.parametrize("bad,code", [
    (dict(g=_g(Hq=16)), EUNSUPPORTED), (dict(g=_g(Hq=7)), EINVAL), (dict(g=_g(B=8193)), EUNSUPPORTED), (dict(page=17), EUNSUPPORTED), (dict(n_pages=-1), EINVAL), (dict(T=-1), EINVAL),
    (dict(T=1 << 28), EINVAL), (dict(cap=0), EINVAL), (dict(cap=1 << 27), EINVAL), (dict(window=-1), EINVAL), (dict(window=(1 << 30) + 1), EINVAL), (dict(sink=-1), EINVAL),
    (dict(scale=0.0), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(rm=FAKE), EINVAL), (dict(rs=FAKE), EINVAL), (dict(q=None), EINVAL),
    (dict(q=ODD), EINVAL), (dict(out=ODD), EINVAL), (dict(kp=ODD), EINVAL), (dict(qs=None), EINVAL), (dict(ctx=None), EINVAL), (dict(table=None), EINVAL),
    (dict(qt=4), EINVAL), (dict(qh=-8), EINVAL), (dict(ws=None), EWORKSPACE), (dict(ws=ctypes.c_void_p(4096 + 128)), EWORKSPACE), (dict(wsb=1000), EWORKSPACE),
    (dict(T=0, q=None), OK), (dict(g=_g(B=0)), OK)])
def test_page_attn_refusals(lib, bad, code):
    assert _attn(lib, **bad) == code


def test_page_attn_workspace(lib):
    need = lambda g, T: lib.antkv_page_attn_workspace(ctypes.byref(g), T)
    assert need(_g(D=64), 4) == 0 and need(_g(), 0) == 0 and need(_g(B=0), 4) == 0 and need(_g(), 1 << 30) == 0
    for hkv in (1, 2, 7, 8, 100, 300, 600):
        sizes = [need(_g(B=3, Hq=4 * hkv, Hkv=hkv), T) for T in (1, 2, 31, 63, 64, 65, 255, 700, 768, 1000, 100000)]
        assert sizes == sorted(sizes) and sizes[0] > 0              # more tokens never need less
    sizes = [need(_g(), T) for T in (1, 100000)]
    assert sizes[-1] < 300 << 20                                    # partial sums of the cut requests, not of every row
    assert _attn(lib, T=4, wsb=need(_g(), 4) - 1) == EWORKSPACE


def _window(lib, g=None, q=FAKE, k=FAKE, v=FAKE, N=8, Nq=8, scale=0.1, window=4, sink=0, out=FAKE, rm=None, rs=None):
    return lib.antkv_prefill_attn_window(ctypes.byref(g or _g()), q, k, v, N, Nq, scale, window, sink, out, rm, rs, None)


@pytest.mark.parametrize("bad,code", [
    (dict(window=0), EINVAL), (dict(window=-5), EINVAL), (dict(sink=-1), EINVAL), (dict(N=0, Nq=0), EINVAL), (dict(Nq=9), EINVAL), (dict(Nq=0), EINVAL),
    (dict(N=(1 << 30) + 1), EINVAL), (dict(scale=-1.0), EINVAL), (dict(rm=FAKE), EINVAL), (dict(q=None), EINVAL), (dict(v=ODD), EINVAL), (dict(out=ODD), EINVAL),
    (dict(g=_g(D=64)), EUNSUPPORTED), (dict(g=_g(B=0), q=None), OK)])
def test_prefill_attn_window_refusals(lib, bad, code):
    assert _window(lib, **bad) == code


def test_bindings_refuse_host_tensors_and_wrong_shapes():
    geom = antkv.Geometry(1, 8, 2, 8)
    half, ints = lambda *s: torch.zeros(s, dtype=torch.float16), lambda *s: torch.zeros(s, dtype=torch.int32)
    pools = half(4, 2, 16, 128), half(4, 2, 16, 128)
    with pytest.raises(ValueError):
        antkv.page_map(ints(1), ints(1), ints(1, 4), 16, 4, ints(4), 1)
    with pytest.raises(ValueError):
        antkv.page_store(geom, half(1, 2, 128), half(1, 2, 128), ints(1), *pools)
    with pytest.raises(ValueError):
        antkv.page_load(geom, *pools, ints(1, 4), 8)
    with pytest.raises(ValueError):
        antkv.page_attn(geom, half(1, 8, 128), 0.1, ints(2), ints(1), ints(1, 4), *pools)
    with pytest.raises(ValueError):
        antkv.prefill_attn_window(geom, half(1, 8, 4, 128), half(1, 2, 4, 128), half(1, 2, 4, 128), 0.1, 4)


def test_batches_beyond_a_grid(lib):
    one = _g(Hq=8, Hkv=8)
    assert _store(lib, T=(1 << 28) + 1) == EINVAL
    assert _attn(lib, T=(1 << 27) + 1) == EINVAL
    assert lib.antkv_page_attn_workspace(ctypes.byref(_g()), (1 << 27) + 1) == 0 < lib.antkv_page_attn_workspace(ctypes.byref(_g()), 1 << 27)
    assert _attn(lib, g=one, n_pages=1 << 26) == EINVAL              # (2^33 rows of a head)
    assert _window(lib, N=1 << 30, Nq=1 << 30) == _window(lib, g=one, N=1 << 30, Nq=1 << 30) == _window(lib, g=one, N=1 << 28, Nq=1 << 28) == EINVAL


def test_as_many_pairs_of_request_and_head_as_there_may_be(lib):
    """8192 requests of ordinary numbers of heads: what is refused here is the workspace, or nothing is to be done."""
    for B, hkv in ((8192, 8), (2048, 32), (8192, 128)):
        g = _g(B=B, Hq=hkv, Hkv=hkv)
        assert lib.antkv_page_attn_workspace(ctypes.byref(g), 8192) > 0
        assert _attn(lib, g=g, wsb=1000) == EWORKSPACE
        assert _load(lib, g=g, N=0) == _store(lib, g=g, T=0) == _attn(lib, g=g, T=0) == OK
    g = _g(B=8192, Hq=129, Hkv=129)
    assert lib.antkv_page_attn_workspace(ctypes.byref(g), 1) == 0
    assert _load(lib, g=g, N=0) == _store(lib, g=g, T=0) == _attn(lib, g=g, T=0) == EUNSUPPORTED
    assert _window(lib, g=_g(B=8192, Hq=8, Hkv=8), q=None) == EUNSUPPORTED


def test_a_workspace_that_would_be_refused_is_not_made():
    for geom, T in ((antkv.Geometry(8193, 8, 2, 8), 1), (antkv.Geometry(1, 8, 2, 8), 1 << 28), (antkv.Geometry(1, 6, 1, 8), 4), (antkv.Geometry(1, 8, 2, 8), -1)):
        with pytest.raises(ValueError):
            antkv.page_attn_workspace(geom, T, "cpu")
    assert antkv.page_attn_workspace(antkv.Geometry(1, 8, 2, 8), 0, "cpu").numel() > 0


@pytest.mark.parametrize("hkv", [1, 2, 64])
def test_page_store_of_a_grid_and_a_row_more(lib, hkv):
    """2^29 rows are 2^24 workgroups of 256 threads, 2^32 threads: one workgroup too many."""
    assert _store(lib, g=_g(Hq=hkv, Hkv=hkv), T=(1 << 29) // hkv) == EINVAL
