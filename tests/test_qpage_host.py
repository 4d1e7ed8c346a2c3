"""Host-side checks of the 8-bit pages' and the rotary positions' entry points: refusals and empty calls, without a GPU."""
import ctypes
import os

import pytest
import torch

import paper_2506_19505_amd as antkv
from paper_2506_19505_amd.binding import _Geom

OK, EINVAL, EUNSUPPORTED, EWORKSPACE = 0, 1, 2, 3
FAKE, OTHER, ODD, ODD2 = (ctypes.c_void_p(x) for x in (4096, 8192, 4098, 4104))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(antkv.lib_path()):
        from paper_2506_19505_amd.build import build
        build()
    return antkv.load_library()


def _g(B=2, Hq=8, Hkv=2, D=128, d=8, C=256):
    return _Geom(B, Hq, Hkv, D, d, C)


# every call below is refused before anything is enqueued, or has nothing to do

def _store(lib, g=None, k=FAKE, v=OTHER, xt=256, xh=128, T=4, slot=FAKE, kp=FAKE, vp=OTHER, ks=FAKE, vs=OTHER, n_pages=8, page=16):
    return lib.antkv_qpage_store(ctypes.byref(g or _g()), k, v, xt, xh, T, slot, kp, vp, ks, vs, n_pages, page, None)


@pytest.mark.parametrize("bad,code", [
    (dict(g=_g(D=64)), EUNSUPPORTED), (dict(g=_g(Hq=16)), EUNSUPPORTED), (dict(page=24), EUNSUPPORTED), (dict(page=8), EUNSUPPORTED), (dict(n_pages=0), EINVAL),
    (dict(T=-1), EINVAL), (dict(T=1 << 31), EINVAL), (dict(k=None), EINVAL), (dict(v=ODD), EINVAL), (dict(slot=None), EINVAL), (dict(vp=FAKE), EINVAL),
    (dict(ks=None), EINVAL), (dict(vs=None), EINVAL), (dict(vs=FAKE), EINVAL), (dict(ks=ODD), EINVAL), (dict(kp=ODD2), EINVAL), (dict(xt=255), EINVAL),
    (dict(xh=-128), EINVAL), (dict(n_pages=1 << 27), EINVAL), (dict(T=0, k=None), OK)])
def test_qpage_store_refusals(lib, bad, code):
    assert _store(lib, **bad) == code


@pytest.mark.parametrize("hkv,most", [(1, (1 << 28) - 16), (4, (1 << 28) - 16), (5, (1 << 27) - 16), (64, (1 << 24) - 16)])
def test_qpage_store_of_a_grid_and_a_row_more(lib, hkv, most):
    """16 rows of four heads to a workgroup, fewer than 2^24 of them."""
    g = _g(Hq=hkv, Hkv=hkv)
    assert _store(lib, g=g, T=most + 1) == EINVAL and _store(lib, g=g, T=most, slot=None) == EINVAL
    assert (most // 16) * ((hkv + 3) // 4) < 1 << 24 <= (most // 16 + 1) * ((hkv + 3) // 4)


def _load(lib, g=None, kp=FAKE, vp=FAKE, ks=FAKE, vs=FAKE, n_pages=8, page=16, table=FAKE, cap=4, ctx=None, first=0, N=8, k=FAKE, v=OTHER, xb=2048, xh=1024,
          xt=128):
    return lib.antkv_qpage_load(ctypes.byref(g or _g()), kp, vp, ks, vs, n_pages, page, table, cap, ctx, first, N, k, v, xb, xh, xt, 0, None)


@pytest.mark.parametrize("bad,code", [
    (dict(N=65), EINVAL), (dict(first=60, N=5), EINVAL), (dict(first=-1), EINVAL), (dict(first=65, N=0), EINVAL), (dict(N=-1), EINVAL), (dict(page=0), EINVAL),
    (dict(page=20), EUNSUPPORTED), (dict(cap=0), EINVAL), (dict(table=None), EINVAL), (dict(kp=None), EINVAL), (dict(ks=None), EINVAL), (dict(vs=ODD), EINVAL),
    (dict(v=FAKE), EINVAL), (dict(k=ODD), EINVAL), (dict(xt=64), EINVAL), (dict(xb=4), EINVAL), (dict(N=0, k=None), OK), (dict(first=64, N=0), OK),
    (dict(g=_g(B=0)), OK)])
def test_qpage_load_refusals(lib, bad, code):
    assert _load(lib, **bad) == code


def _attn(lib, g=None, q=FAKE, qt=1024, qh=128, T=4, qs=FAKE, ctx=FAKE, table=FAKE, cap=4, kp=FAKE, vp=FAKE, ks=FAKE, vs=FAKE, n_pages=8, page=16, scale=0.1,
          window=0, sink=0, out=FAKE, rm=None, rs=None, ws=FAKE, wsb=1 << 40):
    return lib.antkv_qpage_attn(ctypes.byref(g or _g()), q, qt, qh, T, qs, ctx, table, cap, kp, vp, ks, vs, n_pages, page, scale, window, sink, out, rm, rs,
                                ws, wsb, None)


@pytest.mark.parametrize("bad,code", [
    (dict(g=_g(Hq=16)), EUNSUPPORTED), (dict(g=_g(Hq=7)), EINVAL), (dict(g=_g(B=8193)), EUNSUPPORTED), (dict(page=17), EUNSUPPORTED), (dict(n_pages=-1), EINVAL), (dict(T=-1), EINVAL),
    (dict(T=1 << 28), EINVAL), (dict(cap=0), EINVAL), (dict(cap=1 << 27), EINVAL), (dict(window=-1), EINVAL), (dict(window=(1 << 30) + 1), EINVAL), (dict(sink=-1), EINVAL),
    (dict(scale=0.0), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(rm=FAKE), EINVAL), (dict(rs=FAKE), EINVAL), (dict(q=None), EINVAL),
    (dict(q=ODD), EINVAL), (dict(out=ODD), EINVAL), (dict(kp=ODD), EINVAL), (dict(ks=None), EINVAL), (dict(vs=None), EINVAL), (dict(vs=ODD), EINVAL), (dict(qs=None), EINVAL),
    (dict(ctx=None), EINVAL), (dict(table=None), EINVAL), (dict(g=_g(Hkv=8), n_pages=1 << 26), EINVAL), (dict(qt=4), EINVAL), (dict(qh=-8), EINVAL), (dict(ws=None), EWORKSPACE),
    (dict(ws=ctypes.c_void_p(4096 + 128)), EWORKSPACE), (dict(wsb=1000), EWORKSPACE), (dict(T=0, q=None), OK), (dict(g=_g(B=0)), OK)])
def test_qpage_attn_refusals(lib, bad, code):
    assert _attn(lib, **bad) == code


def test_qpage_attn_workspace(lib):
    need = lambda g, T: lib.antkv_qpage_attn_workspace(ctypes.byref(g), T)
    assert need(_g(D=64), 4) == 0 and need(_g(), 0) == 0 and need(_g(B=0), 4) == 0 and need(_g(), 1 << 30) == 0 and need(_g(B=8193), 1) == 0
    for hkv in (1, 2, 7, 8, 100, 300, 600):
        sizes = [need(_g(B=3, Hq=4 * hkv, Hkv=hkv), T) for T in (1, 2, 31, 63, 64, 65, 255, 700, 768, 1000, 100000)]
        assert sizes == sorted(sizes) and sizes[0] > 0              # more tokens never need less
    assert _attn(lib, T=4, wsb=need(_g(), 4) - 1) == EWORKSPACE
    for geom, T in ((antkv.Geometry(8193, 8, 2, 8), 1), (antkv.Geometry(1, 8, 2, 8), 1 << 28), (antkv.Geometry(1, 6, 1, 8), 4), (antkv.Geometry(1, 8, 2, 8), -1)):
        with pytest.raises(ValueError):
            antkv.qpage_attn_workspace(geom, T, "cpu")


# ------------------------------------------------------------------------------------------------ rotary positions

def _rope(lib, g=None, q=FAKE, qs=(0, 1024, 128), k=FAKE, ks=(0, 256, 128), T=4, pos=None, starts=None, ctx=None, pos0=0, freqs=FAKE, rot=128, style=0, amp=1.0,
          inv=0, qo=OTHER, qos=(4096, 1024, 128), ko=ctypes.c_void_p(16384), kos=(4096, 256, 128)):
    return lib.antkv_rope(ctypes.byref(g or _g()), q, *qs, k, *ks, T, pos, starts, ctx, pos0, freqs, rot, style, amp, inv, qo, *qos, ko, *kos, None)


@pytest.mark.parametrize("bad,code", [
    (dict(g=_g(D=64)), EUNSUPPORTED), (dict(g=_g(Hq=7)), EINVAL), (dict(rot=0), EINVAL), (dict(rot=-16), EINVAL), (dict(rot=17), EINVAL), (dict(rot=144), EINVAL),
    (dict(rot=24), EUNSUPPORTED), (dict(rot=2), EUNSUPPORTED), (dict(style=2), EINVAL), (dict(style=-1), EINVAL), (dict(amp=float("nan")), EINVAL),
    (dict(amp=float("inf")), EINVAL), (dict(T=-1), EINVAL), (dict(T=1 << 30), EINVAL), (dict(T=1 << 31, g=_g(B=1)), EINVAL), (dict(pos0=-1), EINVAL),
    (dict(pos0=(1 << 40) + 1), EINVAL), (dict(starts=FAKE), EINVAL), (dict(ctx=FAKE), EINVAL), (dict(starts=FAKE, ctx=FAKE, pos=FAKE), EINVAL),
    (dict(starts=FAKE, ctx=FAKE, g=_g(B=8193)), EUNSUPPORTED), (dict(q=None, qo=None, k=None, ko=None), EINVAL), (dict(q=None), EINVAL), (dict(ko=None), EINVAL),
    (dict(freqs=None), EINVAL), (dict(freqs=ctypes.c_void_p(4100)), EINVAL), (dict(q=ODD), EINVAL), (dict(ko=ODD), EINVAL), (dict(qs=(0, 4, 128)), EINVAL),
    (dict(ks=(-8, 256, 128)), EINVAL), (dict(kos=(4096, 64, 128)), EINVAL), (dict(qos=(0, 1024, 128)), EINVAL), (dict(qo=FAKE), EINVAL), (dict(ko=OTHER), EINVAL),
    (dict(qo=ctypes.c_void_p(4096), q=OTHER, k=FAKE), EINVAL), (dict(T=0, q=None, qo=None), OK), (dict(g=_g(B=0), freqs=None), OK)])
def test_rope_refusals(lib, bad, code):
    assert _rope(lib, **bad) == code


@pytest.mark.parametrize("bad,code", [
    (dict(rot=0), EINVAL), (dict(rot=130), EINVAL), (dict(rot=40), EUNSUPPORTED), (dict(base=1.0), EINVAL), (dict(base=float("nan")), EINVAL),
    (dict(base=float("inf")), EINVAL), (dict(factor=0.0), EINVAL), (dict(factor=-2.0), EINVAL), (dict(trained=-1.0), EINVAL),
    (dict(trained=float("nan")), EINVAL), (dict(trained=8192.0, slow=4.0, fast=4.0), EINVAL), (dict(trained=8192.0, slow=-1.0), EINVAL),
    (dict(trained=8192.0, fast=float("inf")), EINVAL), (dict(freqs=None), EINVAL), (dict(freqs=ctypes.c_void_p(4100)), EINVAL)])
def test_rope_freqs_refusals(lib, bad, code):
    a = dict(rot=128, base=1e4, factor=1.0, trained=0.0, slow=1.0, fast=4.0, freqs=FAKE)
    a.update(bad)
    assert lib.antkv_rope_freqs(*a.values(), None) == code


def test_bindings_refuse_host_tensors_and_wrong_shapes():
    geom = antkv.Geometry(1, 8, 2, 8)
    half, ints = lambda *s: torch.zeros(s, dtype=torch.float16), lambda *s: torch.zeros(s, dtype=torch.int32)
    pools = [torch.zeros((4, 2, 16, 128), dtype=torch.float8_e4m3fn) for _ in "kv"] + [torch.zeros((4, 2, 1)) for _ in "kv"]
    with pytest.raises(ValueError):
        antkv.qpage_store(geom, half(1, 2, 128), half(1, 2, 128), ints(1), *pools)
    with pytest.raises(ValueError):
        antkv.qpage_load(geom, *pools, ints(1, 4), 8)
    with pytest.raises(ValueError):
        antkv.qpage_attn(geom, half(1, 8, 128), 0.1, ints(2), ints(1), ints(1, 4), *pools)
    with pytest.raises(ValueError):
        antkv.rope(geom, half(1, 8, 128), None, torch.zeros(64, dtype=torch.float64))
    with pytest.raises(ValueError):
        antkv.rope_freqs(128, device="cpu")
