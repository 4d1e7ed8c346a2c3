"""GPU checks of rotary positions against 64 bits.

Tolerance per value: half a step of fp16, 2^-11 of it (2^-25 below 2^-14), and of the pair's size |x_a| + |x_b| (times the amplitude) 1e-6: the
turn is rounded to fp32 (pi 2^-24 of angle), sine and cosine to fp32 with a few units of error (2^-22), products and sum to fp32 (3 x 2^-24)."""
import math

import numpy as np
import pytest
import torch

import paper_2506_19505_amd as antkv

pytestmark = pytest.mark.gpu

D = 128


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def randn(seed, *shape):
    return torch.randn(shape, dtype=torch.float16, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


def exact_freqs(rot, base=10000.0, factor=1.0, trained=0, slow=1.0, fast=4.0):
    out = []
    for i in range(rot // 2):
        f = base ** (-2 * i / rot)
        w = 0.0 if not trained else min(1.0, max(0.0, (trained * f / (2 * math.pi) - slow) / (fast - slow)))
        out.append(f * (w + (1 - w) / factor))
    return torch.tensor(out, dtype=torch.float64)


def exact(x, pos, freqs, style, amplitude=1.0, inverse=False):
    """x [.., T, D] (rows of positions pos [T], or [B, 1, T]) in 64 bits, and the size of each value's pair."""
    rot = 2 * freqs.shape[0]
    angle = pos.double()[..., None] * freqs.to(pos.device) * (-1 if inverse else 1)
    c, s = angle.cos() * amplitude, angle.sin() * amplitude
    x = x.double()
    a = torch.arange(rot // 2, device=x.device) * (1 if style else 2)
    b = a + (rot // 2 if style else 1)
    y, size = x.clone(), torch.zeros_like(x)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    size[..., a] = size[..., b] = (x[..., a].abs() + x[..., b].abs()) * abs(amplitude)
    return y, size


def compare(got, x, pos, freqs, style, amplitude=1.0, inverse=False):
    want, size = exact(x, pos, freqs, style, amplitude, inverse)
    assert ((got.double() - want).abs() <= 2.0 ** -11 * want.abs() + 2.0 ** -25 + 1e-6 * size).all(), ((got.double() - want).abs() - 2.0 ** -11 * want.abs()).max()
    rot = 2 * freqs.shape[0]
    assert torch.equal(got[..., rot:], x[..., rot:])


@pytest.mark.parametrize("rot", [16, 32, 96, 128])
@pytest.mark.parametrize("base,factor,trained,slow,fast", [(10000.0, 1.0, 0, 1, 4), (500000.0, 8.0, 8192, 1, 4), (10000.0, 4.0, 0, 1, 4), (10000.0, 32.0, 4096, 0, 32),
                                                           (1.5, 0.5, 1, 0.1, 0.2)])
def test_rope_freqs(rot, base, factor, trained, slow, fast):
    got = antkv.rope_freqs(rot, base, factor, trained, slow, fast).cpu()
    want = exact_freqs(rot, base, factor, trained, slow, fast)
    assert got.shape == want.shape and (got / want - 1).abs().max() <= 1e-14


@pytest.mark.parametrize("style", [0, 1])
@pytest.mark.parametrize("rot", [16, 32, 48, 64, 96, 112, 128])
@pytest.mark.parametrize("Hq,Hkv,T", [(8, 2, 1), (8, 8, 5), (4, 1, 67), (28, 7, 33), (32, 8, 700)])
def test_rope_one_sequence(Hq, Hkv, T, rot, style):
    q, k = randn(T, T, Hq + 2 * Hkv, D)[:, :Hq], randn(T + 1, T, Hkv, D)          # out of a fused projection, and by itself
    freqs = antkv.rope_freqs(rot)
    pos = torch.arange(T, device="cuda")
    for inverse, amplitude, pos0 in ((False, 1.0, 0), (True, 1.25, 123457)):
        qo, ko = antkv.rope(antkv.Geometry(1, Hq, Hkv, 8), q, k, freqs, style=style, inverse=inverse, amplitude=amplitude, pos0=pos0)
        for got, x in ((qo, q), (ko, k)):
            compare(got.transpose(0, 1), x.transpose(0, 1), pos + pos0, freqs, style, amplitude, inverse)


@pytest.mark.parametrize("B,Hq,Hkv,T", [(1, 8, 2, 9), (3, 4, 4, 130), (2, 14, 7, 1), (5, 2, 1, 1000)])
def test_rope_dense(B, Hq, Hkv, T):
    """Prompts as prompt attention has them, positions of their own (negative and far ones among them) and from pos0 on."""
    q, k, freqs, geom = randn(1, B, Hq, T, D), randn(2, B, Hkv, T, D), antkv.rope_freqs(128, 500000.0, 8.0, 8192), antkv.Geometry(B, Hq, Hkv, 8)
    pos = torch.randint(-50, 1 << 20, (B, T), device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).to(torch.int32)
    qo, ko = antkv.rope(geom, q, k, freqs, pos=pos, style=1)
    compare(qo, q, pos[:, None], freqs, 1)
    compare(ko, k, pos[:, None], freqs, 1)
    none, ko = antkv.rope(geom, None, k, freqs, pos0=70, style=0, inverse=True)
    assert none is None
    compare(ko, k, torch.arange(70, 70 + T, device="cuda"), freqs, 0, inverse=True)
    qo, none = antkv.rope(geom, q, None, freqs, style=0)
    assert none is None
    compare(qo, q, torch.arange(T, device="cuda"), freqs, 0)


def batch_positions(ctx, new):
    return torch.cat([torch.arange(c - n, c) for c, n in zip(ctx, new)]).cuda()


@pytest.mark.parametrize("R,most,pad,seed", [(1, 1, 0, 0), (1, 50, 3, 1), (64, 1, 0, 2), (65, 3, 5, 3), (300, 2, 1, 4), (5, 700, 2, 5), (4097, 1, 0, 6), (8192, 2, 3, 7)])
def test_rope_packed(R, most, pad, seed):
    """Batches as page_map makes them: requests without rows first, last and in a row, rows behind the last one left alone."""
    rng = np.random.default_rng(seed)
    new = rng.integers(0 if R > 1 else 1, most + 1, R)
    if R > 4:
        new[[0, 1, R // 2, R - 1]] = 0
    ctx = new + rng.integers(0, 100000, R)
    starts, total = np.concatenate([[0], np.cumsum(new)]), int(new.sum())
    T, Hq, Hkv = total + pad, 4, 2
    q, k, freqs = randn(seed, T, Hq, D), randn(seed + 1, T, Hkv, D), antkv.rope_freqs(64)
    outs = [torch.full_like(x, 7.0) for x in (q, k)]
    antkv.rope(antkv.Geometry(R, Hq, Hkv, 8), q, k, freqs, q_start=ints(starts), ctx_len=ints(ctx), style=1, q_out=outs[0], k_out=outs[1])
    pos = batch_positions(ctx.tolist(), new.tolist())
    for got, x in zip(outs, (q, k)):
        compare(got[:total].transpose(0, 1), x[:total].transpose(0, 1), pos, freqs, 1)
        assert (got[total:] == 7.0).all()


def test_rope_packed_starts_that_do_not_ascend():
    """Whatever the arrays hold, nothing outside the batch is read or written, and rows of proper requests come first."""
    q, freqs, geom = randn(1, 20, 8, D), antkv.rope_freqs(), antkv.Geometry(3, 8, 2, 8)
    guard = torch.full((22, 8, D), 7.0, dtype=torch.float16, device="cuda")
    want = antkv.rope(geom, q, None, freqs, q_start=ints([0, 5, 5, 5]), ctx_len=ints([90, 60, 50]))[0]
    for starts in ([0, 5, 900, 10 ** 9], [0, 5, -7, -9], [7, 9, 9, 9], [-5, 5, 5, 5]):
        antkv.rope(geom, q, None, freqs, q_start=ints(starts), ctx_len=ints([90, 60, 50]), q_out=guard[1:21])
        assert (guard[0] == 7.0).all() and (guard[21] == 7.0).all()
        if starts[:2] == [0, 5] and starts[2] >= 5:
            assert torch.equal(guard[1:6], want[:5])
        if starts[0] == 7:
            assert (guard[1:8] == 7.0).all() and (guard[10:] == 7.0).all()
        guard.fill_(7.0)


def test_rope_in_place_and_strided():
    x = randn(5, 40, 12, D)
    freqs, geom = antkv.rope_freqs(96), antkv.Geometry(1, 8, 2, 8)
    want = antkv.rope(geom, x[:, :8], x[:, 8:10], freqs, pos0=9, style=1)
    y = x.clone()
    q, k = y[:, :8], y[:, 8:10]
    got = antkv.rope(geom, q, k, freqs, pos0=9, style=1, q_out=q, k_out=k)
    assert got[0] is q and torch.equal(y[:, :8], want[0]) and torch.equal(y[:, 8:10], want[1]) and torch.equal(y[:, 10:], x[:, 10:])
    one = x[3:4, :1].expand(40, 8, D)                                # a row that all tokens and heads share
    spread = torch.full((8, 41, 2 * D), 7.0, dtype=torch.float16, device="cuda")
    antkv.rope(geom, one, None, freqs, style=0, q_out=spread[:, :40, :D].transpose(0, 1))
    compare(spread[:, :40, :D], one.transpose(0, 1), torch.arange(40, device="cuda"), freqs, 0)
    assert (spread[:, 40] == 7.0).all() and (spread[:, :, D:] == 7.0).all()


@pytest.mark.parametrize("style", [0, 1])
def test_rope_far_positions(style):
    """Angles of 2^31 radians: their reduction in 64 bits leaves 1e-6 of a turn (2^31 / 2 pi turns, three roundings of 2^-53 each)."""
    freqs, geom = antkv.rope_freqs(), antkv.Geometry(1, 4, 1, 8)
    x = randn(6, 300, 4, D)
    pos = torch.arange((1 << 31) - 300, 1 << 31, device="cuda")
    got = antkv.rope(geom, x, None, freqs, pos=pos.to(torch.int32), style=style)[0]
    compare(got.transpose(0, 1), x.transpose(0, 1), pos, freqs, style)


def test_rope_inverse_undoes_and_is_the_gradient():
    """Back and forth: two roundings of each value, 2^-11 of the pair's length each.  Gradient of a weighted sum: against differences of the formula in
    64 bits, which is linear, so that they are exact but for their own rounding."""
    T, Hq = 50, 4
    x, w, freqs, geom = randn(7, T, Hq, D), randn(8, T, Hq, D), antkv.rope_freqs(64, 10000.0, 4.0), antkv.Geometry(1, Hq, 1, 8)
    for style in (0, 1):
        there = antkv.rope(geom, x, None, freqs, pos0=1000, style=style, amplitude=1.5)[0]
        back = antkv.rope(geom, there, None, freqs, pos0=1000, style=style, amplitude=1 / 1.5, inverse=True)[0]
        _, size = exact(x, torch.zeros(T, Hq, device="cuda"), freqs, style)
        assert ((back - x).double().abs() <= 2 * 2.0 ** -11 * (size + x.double().abs()) + 1e-6).all()
        grad = antkv.rope(geom, w, None, freqs, pos0=1000, style=style, amplitude=1.5, inverse=True)[0]
        pos = torch.arange(1000, 1000 + T, device="cuda")
        f = lambda z: (exact(z.transpose(0, 1), pos, freqs, style, 1.5)[0] * w.transpose(0, 1).double()).sum(-1)
        for c in (0, 1, 31, 32, 63, 64, 127):
            step = torch.zeros(D, dtype=torch.float64, device="cuda")
            step[c] = 0.5
            diff = f(x.double() + step) - f(x.double() - step)          # [Hq, T]
            g = grad.transpose(0, 1)[..., c].double() if c < 64 else (w * 1.0).transpose(0, 1)[..., c].double()
            bound = 2.0 ** -11 * diff.abs() + 1e-5
            assert ((g - diff).abs() <= bound).all(), (style, c)


def test_rope_captured_and_on_another_stream():
    """One captured call replayed over other lengths and rows, eager work between, checked against eager calls; and a call on a side stream."""
    R, T, Hq, Hkv = 3, 12, 8, 2
    geom, freqs = antkv.Geometry(R, Hq, Hkv, 8), antkv.rope_freqs(128, 10000.0, 8.0, 8192)
    q, k = randn(9, T, Hq, D), randn(10, T, Hkv, D)
    starts, ctx = ints([0, 4, 8, 12]), ints([50, 60, 70])
    outs = [torch.zeros_like(q), torch.zeros_like(k)]
    call = lambda o: antkv.rope(geom, q, k, freqs, q_start=starts, ctx_len=ctx, style=1, q_out=o[0], k_out=o[1])
    call(outs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(outs)
    for i, s in enumerate(([0, 4, 8, 12], [0, 0, 1, 12], [0, 10, 12, 12], [0, 1, 2, 3])):
        q.normal_()
        k.normal_()
        starts.copy_(ints(s))
        ctx.copy_(ints([100 * i + 20, 33, 5000]))
        for o in outs:
            o.fill_(float(i))
        want = [o.clone() for o in outs]
        call(want)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), i
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x = q * 2
        got = antkv.rope(geom, x, k, freqs, q_start=starts, ctx_len=ctx, style=1, q_out=torch.zeros_like(q), k_out=torch.zeros_like(k))
    side.synchronize()
    want = antkv.rope(geom, q * 2, k, freqs, q_start=starts, ctx_len=ctx, style=1, q_out=torch.zeros_like(q), k_out=torch.zeros_like(k))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_rope_of_many_rows():
    """More groups of tokens than a grid has workgroups for: all rows are turned."""
    T = (1 << 20) * 2 + 77
    x = randn(11, 1, 1, D).expand(T, 1, D)
    freqs = antkv.rope_freqs(16)
    got = antkv.rope(antkv.Geometry(1, 1, 1, 8), None, x, freqs, style=1)[1]
    for a in (0, 1 << 20, T - 5000):
        compare(got[a:a + 5000].transpose(0, 1), x[a:a + 5000].transpose(0, 1), torch.arange(a, a + got[a:a + 5000].shape[0], device="cuda"), freqs, 1)


def test_rope_turns_keys_as_the_decode_over_keys_before_rope():
    """decode over keys stored before RoPE, every token an anchor, against decode over the same keys turned here: two roundings of fp16 apart."""
    B, Hq, Hkv, N = 2, 8, 2, 300
    geom, gen = antkv.Geometry(B, Hq, Hkv, 8), 13
    k, v, q = randn(gen, B, Hkv, N, D), randn(gen + 1, B, Hkv, N, D), randn(gen + 2, B, Hq, D)
    cb = randn(gen + 3, Hkv, 16, 256, 8)
    codes = antkv.encode(geom, k, cb), antkv.encode(geom, v, cb)
    idx = torch.arange(N, dtype=torch.int32, device="cuda").expand(B, Hkv, N).contiguous()
    for style in (0, 1):
        want = antkv.decode_attn_prerope(geom, q, D ** -0.5, *codes, cb, cb, idx, k, idx, v, rope_style=style, pos0=40)
        turned = antkv.rope(geom, None, k, antkv.rope_freqs(), pos0=40, style=style)[1]
        got = antkv.decode_attn(geom, q, D ** -0.5, *codes, cb, cb, idx, turned, idx, v)
        err = (got.double() - want.double()).norm(dim=-1) / want.double().norm(dim=-1)
        assert err.max() <= 4e-3                                    # either is within 2e-3 of the exact result
