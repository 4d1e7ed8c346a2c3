"""GPU checks of what pages of 8 bits hold, exactly: every number of fp16 under every scale, every byte through every growth of its scale, and rows
of blocks that lie between each other in the batch."""
import numpy as np
import pytest
import torch

import paper_2506_19505_amd as antkv
from test_gpu_qpages import Pools, gen_of, randn

pytestmark = pytest.mark.gpu

D = 128


def geometry(Hkv):
    return antkv.Geometry(1, Hkv, Hkv, 8)


def held(pools, scales):
    """Pools whose blocks hold all finite values and both NaN of e4m3 (rows 0 and 1, the others zeros) under the given scales [n_pages]."""
    codes = torch.arange(256, device="cuda").to(torch.uint8)
    for b, s, w, ws in zip(pools.bytes, pools.scales, pools.want, pools.want_scales):
        b.view(torch.uint8).zero_()
        b.view(torch.uint8)[:, :, :2] = codes.view(2, D)
        s.copy_(scales[:, None, None])
        w.copy_(b.float().double())
        ws.copy_(s.double())


@pytest.mark.parametrize("exponents", [range(-32, -18), range(-18, -4), range(-4, 9)])
def test_every_half_under_every_scale(exponents):
    """All numbers of fp16 as rows 1 .. 15 of blocks that go on under a scale from 2^-32 to 2^8: those that it is enough for leave it as it is, others make
    it grow.  In V a row's sizes are cut at 448 of the scale first, so that it stays: down to values that are subnormal in e4m3, or nothing."""
    codes = torch.arange(65536, device="cuda").to(torch.int16).view(torch.float16).view(512, 1, D)
    # numbers of about one size side by side, and small ones beside large ones (every 35th row)
    x = torch.cat([codes, codes.view(-1)[torch.randperm(65536, device="cuda", generator=gen_of(7))].view(512, 1, D), torch.zeros((11, 1, D), dtype=torch.float16, device="cuda")])
    n_blocks = x.shape[0] // 15
    assert x.shape[0] == 15 * n_blocks
    slot = [16 * (t // 15) + 1 + t % 15 for t in range(x.shape[0])]
    for e in exponents:
        scale = 2.0 ** e
        pools = Pools(n_blocks, 1, 16)
        held(pools, torch.full((n_blocks,), scale, device="cuda"))
        cut = torch.where(x.isfinite(), x.float().clamp(-448 * scale, 448 * scale), x.float()).half()
        # (448 x 2^-32 lies between two halves: the lower one)
        cut = torch.where(cut.isfinite() & (cut.float().abs() > 448 * scale), torch.copysign(torch.full_like(cut, 2.0 ** -24), cut), cut)
        pools.store(geometry(1), x, cut, slot)
        pools.check(f"2^{e}")
        assert (pools.scales[1] == scale).all()


def test_every_byte_through_every_growth():
    """A block of all values of e4m3 goes on with a row whose largest size needs a scale of its own, from each of the 41 to each of them: what is there is
    rounded to the larger one, or left."""
    exps = [(a, b) for a in range(-32, 9) for b in range(-32, 9)]
    pools = Pools(len(exps), 1, 16)
    held(pools, torch.tensor([2.0 ** a for a, _ in exps], device="cuda"))
    k = torch.zeros((len(exps), 1, D), dtype=torch.float16, device="cuda")
    # of a scale 2^b: 225 .. 448 of it (2^-24, the least number, of the least one; 61440 of the largest)
    k[:, 0, 5] = torch.tensor([min(2.0 ** b * 256, 61440.0) for _, b in exps], device="cuda").half()
    v = k.clone()
    v[:, 0, 9], v[:, 0, 100] = -v[:, 0, 5], v[:, 0, 5] / 2
    pools.store(geometry(1), k, v, [16 * i + 15 for i in range(len(exps))])
    pools.check()
    for s in pools.scales:
        assert torch.equal(s.view(-1).cpu(), torch.tensor([2.0 ** max(a, b) for a, b in exps]))


# a wave looks for first rows among 1, 2, 2, 8, 16 and 16 rows of these batches
@pytest.mark.parametrize("T,Hkv", [(300, 2), (1000, 5), (3000, 2), (7000, 3), (9000, 3), (12000, 1)])
def test_rows_of_blocks_between_each_other(T, Hkv):
    """Each block's rows lie within 16 rows of the batch but not side by side: those of two or three blocks alternate, some rows have no slot, blocks lack
    some of their rows, the first one too (what they then hold goes on: nothing here, under no scale)."""
    rng = np.random.default_rng(T)
    groups, t, n_blocks = [], 0, 0
    while t < T:                                                    # 16 rows of the batch, shared out among one to four blocks
        n = min(16, T - t)
        of = rng.integers(0, rng.integers(1, 5), n)
        row = np.full(n, -1)
        for b in range(4):
            at = np.flatnonzero(of == b)
            row[at] = 16 * (n_blocks + b) + rng.permutation(16)[:len(at)]
        row[rng.random(n) < 0.1] = -1
        n_blocks += 4
        groups.append(row)
        t += n
    slots = np.concatenate(groups)
    order = rng.permutation(n_blocks)                               # blocks anywhere in the pool
    slots = np.where(slots >= 0, order[slots // 16] * 16 + slots % 16, -1)
    lead = int(rng.integers(1, 16))                                 # (so that they begin inside what a wave looks at)
    slots = np.concatenate([np.full(lead, -1), slots])[:T]
    gen, page = gen_of(T), 32
    pools = Pools(-(-n_blocks // 2), Hkv, page)
    k, v = randn(gen, T, Hkv, D), randn(gen, T, Hkv, D) * 3
    pools.store(geometry(Hkv), k, v, slots.tolist())
    pools.check("first")
    # once more, the slots of a group in another order: every block goes on or begins anew
    again = slots.copy()
    for a in range(lead, T, 16):
        rng.shuffle(again[a:a + 16])
    pools.store(geometry(Hkv), v, k * 20, again.tolist())
    pools.check("second")


@pytest.mark.parametrize("new", [1, 8, 300])
def test_scales_that_are_no_powers_of_two(new):
    """Loading and attention take a positive normal scale for the power of two at or below it, in narrow blocks and in wide ones, bit for bit."""
    Hq, Hkv, page, n = 8, 2, 32, 700
    gen, geom = gen_of(new), antkv.Geometry(1, Hq, Hkv, 8)
    q = randn(gen, new, Hq, D)
    pools = Pools(24, Hkv, page, seed=new)
    table = torch.randperm(24, device="cuda", generator=gen).to(torch.int32)[None]
    even = [s.clone() for s in pools.scales]
    for s in pools.scales:                                          # 1.0 to 1.99 of them
        s.mul_(1 + 0.99 * torch.rand(s.shape, device="cuda", generator=gen))
    args = lambda scales: (*pools.bytes, *scales)
    starts, ctx = torch.tensor([0, new], dtype=torch.int32, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda")
    want, got = ((*antkv.qpage_load(geom, *args(s), table, n), *antkv.qpage_attn(geom, q, 0.001, starts, ctx, table, *args(s), want_stats=True)) for s in (even, pools.scales))
    assert all(x.isfinite().all() for x in want)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
