"""GPU checks of the cache in pages of 8 bits against plain implementations: what is stored and loaded exactly, attention against 64 bits
over the values that the pages hold, with the tolerances of the FP16 pages (the arithmetic behind the conversion, which is exact, is the same)."""
import numpy as np
import pytest
import torch

import paper_2506_19505_amd as antkv
from test_gpu_pages import BATCHES, D, OUT_TOL, SCALE, compare, exact, gen_of, ints, one_way, randn

pytestmark = pytest.mark.gpu

E4M3, NAN = torch.float8_e4m3fn, float("nan")


# ------------------------------------------------------------------------------------------------ the definition

def scale_of(amax):
    """float64: the least power of two from 2^-32 to 2^8 through which amax is at most 448."""
    s = torch.full_like(amax, 2.0 ** -32)
    for e in range(-31, 9):
        s = torch.where(amax > 448 * 2.0 ** (e - 1), 2.0 ** e, s)
    return s


def round_to(y):
    """float64 to the nearest e4m3 value, ties to even; NaN stays."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def held_rows(x, s):
    """What rows x (float64 [.., D]) are held as under scales s, as values of e4m3."""
    fine = torch.where(x.isfinite(), x.clamp(-61440, 61440), 0)
    return torch.where(x.isfinite(), round_to(fine / s), NAN)


def amax_of(x):
    return torch.where(x.isfinite(), x.abs().clamp(max=61440), 0).amax((-1, -2))


def plain_store(x, slot, values, scales):
    """x float64 [T, Hkv, D] to values float64 [n, Hkv, page, D] (of e4m3, not yet scaled) and scales float64 [n, Hkv, page / 16], block by block."""
    n, Hkv, page, _ = values.shape
    blocks = {}
    for t, s in enumerate(slot):
        if 0 <= s < n * page:
            blocks.setdefault(s // 16, []).append((t, s % 16))
    for b, rows in blocks.items():
        p, o = b // (page // 16), b % (page // 16)
        ts, offs = [t for t, _ in rows], [i for _, i in rows]
        need = scale_of(amax_of(x[ts].transpose(0, 1)))                              # [Hkv]
        block = values[p, :, 16 * o:16 * o + 16]                                     # a view
        if 0 not in offs:
            was = scales[p, :, o]                                                    # (one that nobody made counts as the least)
            was = torch.where((torch.frexp(was).mantissa == 0.5) & (was >= 2.0 ** -32) & (was <= 2.0 ** 8), was, 2.0 ** -32)
            grown = torch.maximum(need, was)
            block.copy_(torch.where(block.isnan(), block, round_to(block * (was / grown)[:, None, None])))
            need = grown
        block[:, offs] = held_rows(x[ts].transpose(0, 1), need[:, None, None])
        scales[p, :, o] = need


class Pools:
    """Pages of 8 bits on the GPU, and what they should hold."""

    def __init__(self, n_pages, Hkv, page, seed=None):
        self.n, self.Hkv, self.page = n_pages, Hkv, page
        self.bytes = [torch.full((n_pages, Hkv, page, D), 127, dtype=torch.uint8, device="cuda").view(E4M3) for _ in "kv"]
        self.scales = [torch.full((n_pages, Hkv, page // 16), NAN, device="cuda") for _ in "kv"]
        if seed is not None:
            gen = gen_of(seed)
            for b, s in zip(self.bytes, self.scales):
                codes = torch.randint(0, 127, b.shape, device="cuda", generator=gen) + 128 * torch.randint(0, 2, b.shape, device="cuda", generator=gen)
                b.view(torch.uint8).copy_(codes.to(torch.uint8))
                s.copy_(torch.exp2(torch.randint(-12, 2, s.shape, device="cuda", generator=gen).float()))
        self.want = [b.float().double() for b in self.bytes]
        self.want_scales = [s.double() for s in self.scales]

    def args(self):
        return *self.bytes, *self.scales

    def store(self, geom, k, v, slot):
        antkv.qpage_store(geom, k, v, ints(slot), *self.args())
        for x, w, s in zip((k, v), self.want, self.want_scales):
            plain_store(x.double(), slot, w, s)

    def check(self, what=""):
        for got, s, w, ws, name in zip(self.bytes, self.scales, self.want, self.want_scales, "kv"):
            touched = ~ws.isnan()
            assert torch.equal(s.double()[touched], ws[touched]) and torch.equal(s.isnan(), ws.isnan()), f"{what} {name}: scales"
            got = got.float().double()
            assert torch.equal(got.isnan(), w.isnan()) and torch.equal(got[~w.isnan()], w[~w.isnan()]), f"{what} {name}: values"


# ------------------------------------------------------------------------------------------------ storing

@pytest.mark.parametrize("T,Hkv,page,at,fused", [(1, 1, 16, 0, False), (1, 8, 64, 0, True), (7, 2, 16, 0, True), (16, 2, 32, 0, False), (31, 7, 32, 0, False), (33, 3, 128, 16, True),
                                                 (1000, 8, 256, 0, True), (4100, 4, 16, 0, False), (3000, 3, 64, 48, True), (20000, 1, 16, 0, False)])
def test_qpage_store_of_whole_blocks(T, Hkv, page, at, fused):
    """Rows from the start of a block on, into pages that held anything; negative slots and slots behind the pool are skipped."""
    gen = gen_of(T)
    n_pages = (T + at) // page + 4
    pools = Pools(n_pages, Hkv, page)
    if fused:
        qkv = randn(gen, T, 6 * Hkv, D)
        k, v = qkv[:, 4 * Hkv:5 * Hkv], qkv[:, 5 * Hkv:]
    else:
        k, v = randn(gen, T, Hkv, D), randn(gen, Hkv, T, D).transpose(0, 1).contiguous()
    order = np.random.default_rng(T).permutation(n_pages)
    pos = np.arange(at, at + T)
    slot = order[pos // page] * page + pos % page
    if T > 40:
        slot[-2:] = -1, n_pages * page
        slot[T // 2] = -5                                           # (the block around it has 15 rows)
    pools.store(antkv.Geometry(1, Hkv, Hkv, 8), k, v, slot.tolist())
    pools.check()


@pytest.mark.parametrize("size", [1.0, 1e-5, 3e-7, 500.0, 20000.0])
def test_qpage_store_of_all_sizes(size):
    """Values from fp16's smallest to its largest, blocks of zeros, and largest values at the borders between scales."""
    gen, Hkv, T = gen_of(3), 2, 256
    pools = Pools(T // 16, Hkv, 16)
    k = (torch.randn((T, Hkv, D), device="cuda", generator=gen) * size).clamp(-65504, 65504).half()
    v = k.clone()
    k[:16] = 0
    for b, top in enumerate((448, 448.25, 447.75, 449, 224, 224.125, 223.9, 61440, 61472, 65504, 57344, 57376, 2.0 ** -24, 7 * 2.0 ** -24, 28672)):
        block = slice(16 * b, 16 * b + 16)
        v[block] = v[block].clamp(-top, top)
        v[16 * b + 5, 1, 7] = -top
    pools.store(antkv.Geometry(1, Hkv, Hkv, 8), k, v, range(T))
    pools.check()
    dense = antkv.qpage_load(antkv.Geometry(1, Hkv, Hkv, 8), *pools.args(), ints([range(T // 16)]), T)
    for x, got, s in zip((k, v), dense, pools.scales):
        got, x = got[0].transpose(0, 1).double(), x.double()
        unit = s.double()[:, :, 0].repeat_interleave(16, 0)[..., None]
        assert got.isfinite().all()                                 # whatever the scale, an fp16 number
        assert ((got - x).abs() <= torch.maximum(x.abs() / 16, 2.0 ** -10 * unit)).all()


def test_qpage_store_every_half():
    """All numbers of fp16, their signs, infinities and NaN, a block for 2048 of them; each next to a 1."""
    codes = torch.arange(65536, device="cuda").to(torch.int16).view(torch.float16)
    x = codes.view(32, 16, 1, D).flatten(0, 1).contiguous()
    y = x.clone()
    y[::16, 0, 0] = 1.0
    pools = Pools(32, 1, 16)
    pools.store(antkv.Geometry(1, 1, 1, 8), x, y, range(512))
    pools.check()


def test_qpage_store_a_token_at_a_time():
    """Blocks that go on from step to step: scales grow, and rows that are there are rounded to the new one; 64 requests at different places."""
    gen, R, Hkv, page = gen_of(4), 64, 3, 32
    geom, pools = antkv.Geometry(R, Hkv, Hkv, 8), Pools(2 * R, Hkv, page)
    pos = [r % 23 for r in range(R)]
    # what a request held before
    first = [(r, j) for r in range(R) for j in range(pos[r])]
    pools.store(geom, randn(gen, len(first), Hkv, D) * 0.1, randn(gen, len(first), Hkv, D), [2 * r * page + j for r, j in first])
    pools.check("before")
    for step in range(20):
        size = torch.exp2(torch.randint(-6, 5, (R, 1, 1), device="cuda", generator=gen).float()).half()
        k, v = randn(gen, R, Hkv, D) * size, randn(gen, R, Hkv, D) * size
        pools.store(geom, k, v, [(2 * r + pos[r] // page) * page + pos[r] % page for r in range(R)])
        pos = [p + 1 for p in pos]
        pools.check(f"step {step}")


@pytest.mark.parametrize("chunks", [[5, 20, 1, 1, 30, 7], [16, 16, 17, 15], [1] * 40, [40, 3, 200, 1, 50]])
def test_qpage_store_in_chunks(chunks):
    """A prompt in chunks that begin and end inside blocks; the error over all of its growing: that of the rounding at the end and 2^-9 of the scale."""
    gen, Hkv, page, T = gen_of(5), 2, 64, sum(chunks)
    geom, pools = antkv.Geometry(1, Hkv, Hkv, 8), Pools(T // page + 2, Hkv, page)
    size = torch.exp2(torch.linspace(-8, 6, T, device="cuda"))[:, None, None].half()
    k, v, at = randn(gen, T, Hkv, D) * size, randn(gen, T, Hkv, D) * size.flip(0), 0
    for n in chunks:
        pools.store(geom, k[at:at + n], v[at:at + n], range(at, at + n))
        at += n
        pools.check(f"at {at}")
    for x, got, s in zip((k, v), antkv.qpage_load(geom, *pools.args(), ints([range(pools.n)]), T), pools.scales):
        unit = s.transpose(1, 2).reshape(-1, Hkv).double().repeat_interleave(16, 0)[:T, :, None]
        err = (got[0].transpose(0, 1).double() - x.double()).abs()
        assert (err <= torch.maximum(x.double().abs() / 16, 2.0 ** -10 * unit) + 2.0 ** -9 * unit).all()


def test_qpage_store_rows_of_a_block_in_any_order():
    gen, Hkv, page = gen_of(6), 2, 32
    geom, pools = antkv.Geometry(1, Hkv, Hkv, 8), Pools(40, Hkv, page)
    rng = np.random.default_rng(6)
    slots = []
    for b in rng.permutation(80)[:70]:
        slots += (16 * b + rng.permutation(16)[:rng.integers(1, 17)]).tolist()
    T = len(slots)
    pools.store(geom, randn(gen, T, Hkv, D), randn(gen, T, Hkv, D) * 3, slots)
    # blocks that began without their first row hold what was there, under no scale: rounded as if under the least one
    for got, s, w, ws in zip(pools.bytes, pools.scales, pools.want, pools.want_scales):
        for b in sorted({x // 16 for x in slots}):
            p, o = b // 2, b % 2
            rows = [x % 16 for x in slots if x // 16 == b]
            assert s[p, :, o].isfinite().all()
            if 0 in rows:
                assert torch.equal(s[p, :, o].double(), ws[p, :, o])
                assert torch.equal(got[p, :, 16 * o:16 * o + 16].float().double()[:, rows], w[p, :, 16 * o:16 * o + 16][:, rows])


def test_qpage_store_scales_that_nobody_made():
    """A block that goes on under a scale that is none (not a power of two in range) takes the new rows' own."""
    gen, Hkv = gen_of(7), 1
    geom = antkv.Geometry(1, Hkv, Hkv, 8)
    k = randn(gen, 1, 1, D)
    need = scale_of(amax_of(k.double().transpose(0, 1)))
    for odd in (NAN, float("inf"), -1.0, 0.0, 3.0, 2.0 ** -33, 512.0, 1e-40, -0.0):
        pools = Pools(1, 1, 16, seed=8)
        for s in pools.scales:
            s.fill_(odd)
        antkv.qpage_store(geom, k, k, ints([3]), *pools.args())
        for b, s in zip(pools.bytes, pools.scales):
            assert s.item() == need.item()
            assert torch.equal(b[0, 0, 3].float().double(), held_rows(k[0, 0].double(), need))


def test_qpage_store_what_is_not_finite():
    """Infinities and NaN are held as NaN and leave the scale alone, in new rows and in rows that are rounded again."""
    gen, Hkv = gen_of(9), 2
    geom, pools = antkv.Geometry(1, Hkv, Hkv, 8), Pools(2, Hkv, 16)
    k, v = randn(gen, 20, Hkv, D), randn(gen, 20, Hkv, D)
    k[2, 0, 5], k[3, 1, :], v[0, 0, 127], v[15, :, 64] = float("inf"), NAN, -float("inf"), NAN
    k[16:18] = NAN                                                  # a block without a number in it
    v[19, 1, 3] = float("inf")
    pools.store(geom, k[:10], v[:10], range(10))
    pools.check("first")
    pools.store(geom, k[10:] * 64, v[10:] * 64, range(10, 20))
    pools.check("second")


def test_qpage_store_nothing():
    geom, pools = antkv.Geometry(1, 2, 2, 8), Pools(2, 2, 16, seed=1)
    none = torch.zeros((0, 2, D), dtype=torch.float16, device="cuda")
    pools.store(geom, none, none, [])
    pools.store(geom, randn(gen_of(1), 3, 2, D), randn(gen_of(1), 3, 2, D), [-1, -7, 32])
    pools.check()


def test_qpage_store_of_the_largest_batch():
    """As many rows as a grid has, all of them the same one and nearly all without a slot."""
    T, Hkv = (1 << 24) - 16, 64
    gen = gen_of(92)
    k, v = (randn(gen, 1, Hkv, D).expand(T, Hkv, D) for _ in "kv")
    pools = Pools(4, Hkv, 16)
    slot = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    slot[0], slot[T // 2], slot[-1] = 0, 48, 16
    antkv.qpage_store(antkv.Geometry(1, Hkv, Hkv, 8), k, v, slot, *pools.args())
    for x, w, s in zip((k, v), pools.want, pools.want_scales):
        plain_store(x[:3].double(), [0, 48, 16], w, s)
    pools.check()


# ------------------------------------------------------------------------------------------------ loading

@pytest.mark.parametrize("B,Hkv,page,N,first", [(1, 1, 16, 1, 0), (2, 8, 16, 100, 0), (3, 2, 64, 333, 5), (1, 7, 256, 700, 300), (5, 3, 32, 31, 33), (1, 8, 64, 5000, 1)])
def test_qpage_load(B, Hkv, page, N, first):
    cap = (first + N) // page + 2
    pools, gen = Pools(B * cap + 1, Hkv, page, seed=N), gen_of(N)
    table = torch.randperm(B * cap + 1, device="cuda", generator=gen)[:B * cap].view(B, cap).to(torch.int32)
    lens = [first + N + 5 if b == 0 else max(0, first + N - 7 * b) for b in range(B)]
    pos = torch.arange(first, first + N, device="cuda")
    dense = []
    for b, s in zip(pools.bytes, pools.scales):
        values = (b.float().double().view(-1, Hkv, page // 16, 16, D) * s.double()[..., None, None]).view(-1, Hkv, page, D)
        dense.append(values[table[:, pos // page].long(), :, pos % page].transpose(1, 2).half())
        assert torch.equal(dense[-1].double(), values[table[:, pos // page].long(), :, pos % page].transpose(1, 2))       # fp16 numbers, all of them
    geom = antkv.Geometry(B, Hkv, Hkv, 8)
    whole = antkv.qpage_load(geom, *pools.args(), table, N, first=first)
    assert all(torch.equal(g, d) for g, d in zip(whole, dense))
    before = randn(gen, B, Hkv, N, D), randn(gen, B, Hkv, N, D)
    table[0, -2], table[0, 0] = -1, pools.n                         # pages that are none
    there = (pos < ints(lens)[:, None]) & (table[:, pos // page] >= 0) & (table[:, pos // page] < pools.n)
    got = antkv.qpage_load(geom, *pools.args(), table, N, first=first, ctx_len=ints(lens), k=before[0].clone(), v=before[1].clone())
    for g, d, b in zip(got, dense, before):
        assert torch.equal(g, torch.where(there[:, None, :, None], d, b))
    made = antkv.qpage_load(geom, *pools.args(), table, N, first=first, ctx_len=ints(lens))
    half = antkv.qpage_load(geom, *pools.args(), table, N, first=first, ctx_len=ints(lens), v=before[1].clone())
    for g, d in zip((*made, half[0]), (*dense, dense[0])):
        assert torch.equal(g, torch.where(there[:, None, :, None], d, 0))
    assert torch.equal(half[1], got[1])


# ------------------------------------------------------------------------------------------------ attention

class ByteCache:
    """Pages of a batch of requests whose values are k[r], v[r] fp16 [Hkv, ctx, D]; what no request holds is NaN, scales too."""

    def __init__(self, seed, ctx, Hkv, page, extra=2):
        gen = gen_of(seed)
        counts = [-(-c // page) for c in ctx]
        self.page, self.ctx, self.n_pages = page, ctx, sum(counts) + 3
        self.pools = Pools(self.n_pages, Hkv, page)
        self.k, self.v = [randn(gen, Hkv, c, D) for c in ctx], [randn(gen, Hkv, c, D) for c in ctx]
        for k in self.k:
            k[..., 5::32] *= 10                                     # channels that stand out, as keys have them
        self.table = torch.full((len(ctx), max(counts, default=0) + extra), -1, dtype=torch.int32, device="cuda")
        order = torch.randperm(self.n_pages, device="cuda", generator=gen).to(torch.int32)
        used = 0
        for r, n in enumerate(counts):
            self.table[r, :n] = order[used:used + n]
            used += n
        self.fill()

    def fill(self):
        """Rows into the pages, and k and v to what the pages then hold."""
        for r, c in enumerate(self.ctx):
            if c == 0:
                continue
            j = torch.arange(c, device="cuda")
            ids, off = self.table[r].long()[j // self.page], j % self.page
            for x, b, s in ((self.k[r], *[a[0] for a in (self.pools.bytes, self.pools.scales)]), (self.v[r], *[a[1] for a in (self.pools.bytes, self.pools.scales)])):
                rows = torch.zeros((x.shape[0], -(-c // 16) * 16, D), dtype=torch.float64, device="cuda")
                rows[:, :c] = x.double()
                scale = scale_of(amax_of(rows.view(x.shape[0], -1, 16, D)))                                # [Hkv, blocks]
                held = held_rows(rows.view(x.shape[0], -1, 16, D), scale[..., None, None]).view(x.shape[0], -1, D)[:, :c]
                each = scale.repeat_interleave(16, 1)[:, :c]
                b.view(torch.uint8)[ids, :, off] = held.to(E4M3).view(torch.uint8).transpose(0, 1)
                s[ids, :, off // 16] = each.float().transpose(0, 1)
                x.copy_((held * each[..., None]).half())


def check_attn(c, new, Hq, window=0, n_sink=0, q=None, pad=0, seed=1, scale=SCALE, hidden=None, workspace=None, ctx=None, each=1):
    """Every row of the batch against 64 bits; rows behind the last request stay as they are."""
    Hkv, R, T = c.pools.Hkv, len(new), sum(new) + pad
    G = Hq // Hkv
    if q is None:
        q = randn(gen_of(seed), T, Hq, D)
    starts = np.concatenate([[0], np.cumsum(new)])
    out = torch.full((T, Hq, D), 7.0, dtype=torch.float16, device="cuda")
    geom = antkv.Geometry(R, Hq, Hkv, 8)
    args = geom, q, scale, ints(starts), ints(ctx or c.ctx), c.table, *c.pools.args()
    got, top, total = antkv.qpage_attn(*args, window=window, n_sink=n_sink, out=out, want_stats=True, workspace=workspace)
    assert got is out and (out[starts[-1]:] == 7.0).all()
    lean = antkv.qpage_attn(*args, window=window, n_sink=n_sink)
    assert lean[1] is None and torch.equal(lean[0][:starts[-1]].view(torch.int16), out[:starts[-1]].view(torch.int16))
    for r, n in enumerate(new):
        a, b = int(starts[r]), int(starts[r + 1])
        pos = torch.arange((ctx or c.ctx)[r] - n, (ctx or c.ctx)[r], device="cuda")
        for h in range(0, Hq if n else 0, each):
            want = exact(q[a:b, h], c.k[r][h // G], c.v[r][h // G], pos, window, n_sink, scale, None if hidden is None else hidden[r])
            compare((out[a:b, h], top[h, a:b], total[h, a:b]), want, f"request {r}, head {h}")
    return out


@pytest.mark.parametrize("window,n_sink", [(0, 0), (1, 0), (40, 4), (100, 37), (64, 0), (5000, 3)])
@pytest.mark.parametrize("Hq,Hkv,page,ctx,new", BATCHES)
def test_qpage_attn(Hq, Hkv, page, ctx, new, window, n_sink):
    check_attn(ByteCache(len(ctx) + page, ctx, Hkv, page), new, Hq, window, n_sink, pad=3)


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("Hq,Hkv,ctx,new,window,n_sink", [(4, 1, [40000], [1], 0, 0), (4, 1, [33000, 70000], [40, 1], 0, 0), (4, 2, [66000], [3], 60000, 100),
                                                          (2, 2, [35000], [300], 0, 0)])
def test_qpage_attn_long(Hq, Hkv, page, ctx, new, window, n_sink):
    """More key tiles than a workgroup looks pages up for at a time, and ranges of them."""
    check_attn(ByteCache(page, ctx, Hkv, page), new, Hq, window, n_sink)


def test_qpage_attn_many_requests():
    """More requests than threads of a workgroup, most of them with a token, some with none."""
    rng = np.random.default_rng(3)
    ctx = rng.integers(1, 90, 700).tolist()
    new = [int(min(c, n)) for c, n in zip(ctx, rng.integers(0, 3, 700))]
    check_attn(ByteCache(5, ctx, 1, 16), new, 2)


def test_qpage_attn_wide_batch():
    """Enough rows for workgroups of eight waves; requests of one token among long chunks."""
    for window, n_sink in ((0, 0), (200, 5)):
        check_attn(ByteCache(9, [1500, 900, 2000, 1, 400], 8, 32), [1500, 1, 300, 1, 0], 32, window, n_sink, pad=5)


def test_qpage_attn_a_workgroup_per_block():
    """Many blocks: of many requests of few tokens, in shares, and of a long prompt, each a workgroup of its own."""
    rng = np.random.default_rng(4)
    ctx = rng.integers(1, 300, 300).tolist()
    check_attn(ByteCache(6, ctx, 8, 16), [1 + (r % 7 == 0) * min(c - 1, 40) for r, c in enumerate(ctx)], 16, each=3)
    for window, n_sink in ((0, 0), (700, 40)):
        check_attn(ByteCache(7, [8300, 40], 8, 64), [8250, 1], 32, window, n_sink, each=7)


def test_qpage_attn_long_prompts():
    for window, n_sink in ((0, 0), (300, 40)):
        check_attn(ByteCache(51, [4100, 4097], 8, 32), [4100, 4093], 32, window, n_sink, pad=5, each=11)


@pytest.mark.parametrize("window,n_sink", [(0, 0), (90, 40)])
@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (4, 2), (3, 3)])
def test_qpage_attn_a_token_each_on_average(Hq, Hkv, window, n_sink):
    """No more rows than requests, but uneven ones: some have many blocks of 32 rows, some none."""
    ctx = [600, 1, 70, 2000, 33, 64] + [5] * 94
    check_attn(ByteCache(61, ctx, Hkv, 32), [40, 1, 0, 33, 17, 0] + [0] * 90 + [5, 0, 1, 1], Hq, window, n_sink, pad=2)
    check_attn(ByteCache(62, [3000] + [9] * 129, Hkv, 16), [130] + [0] * 129, Hq, window, n_sink)


def test_qpage_attn_scores_far_apart():
    """Scores over a few hundred log2 units: the softmax reference moves many times per row; and one key far above many others."""
    c = ByteCache(4, [900, 333], 2, 16)
    check_attn(c, [300, 1], 8, q=(randn(gen_of(8), 301, 8, D).float() * 12).half())
    c = ByteCache(6, [9000], 2, 64)
    q = randn(gen_of(9), 1, 8, D)
    for g in range(2):
        c.k[0][g] *= 0.01
        c.k[0][g, 4000] = (q[0, 4 * g:4 * g + 4].sum(0) * 0.55).half()
    c.fill()
    check_attn(c, [1], 8, q=q)


def test_qpage_attn_sizes_of_blocks():
    """Blocks whose scales lie up to 2^20 apart, K and V each in an order of its own."""
    for ctx, new in (([1000], [1]), ([1000, 500], [300, 40])):
        c = ByteCache(14, ctx, 2, 32)
        for r, n in enumerate(ctx):
            size = torch.exp2((torch.arange(n, device="cuda") // 16 * 7 % 21 - 17).float())[:, None].half()
            c.k[r].mul_(size)
            c.v[r].mul_(size.flip(0) * 8)
        c.fill()
        check_attn(c, new, 8)


def test_qpage_attn_strided_queries():
    c = ByteCache(4, [200, 100], 2, 16)
    check_attn(c, [30, 1], 8, q=randn(gen_of(3), 31, 12, D)[:, :8])
    check_attn(c, [30, 1], 8, q=randn(gen_of(3), 8, 31, D).transpose(0, 1))


@pytest.mark.parametrize("window,n_sink", [(0, 0), (50, 10)])
def test_qpage_attn_hidden_values_take_no_part(window, n_sink):
    """NaN in K and V: rows that see them get what the formula gives, the others nothing of them."""
    c = ByteCache(4, [150, 90, 400], 2, 16)
    c.v[0][:, 100, 3], c.v[0][:, 100, 77], c.v[0][:, 101, 3], c.v[0][0, 60, 9], c.v[0][1, 12, 9] = NAN, NAN, NAN, NAN, NAN
    c.k[1][:, 89] = NAN                                             # seen by the last row only
    c.v[1][:, 88] = NAN
    c.v[2][:, 300:310] = NAN
    c.fill()
    q, new, starts = randn(gen_of(5), 90 + 150 + 200, 8, D), [150, 90, 200], [0, 150, 240, 440]
    out, top, total = antkv.qpage_attn(antkv.Geometry(3, 8, 2, 8), q, SCALE, ints(starts), ints(c.ctx), c.table, *c.pools.args(), window=window, n_sink=n_sink,
                                       want_stats=True)
    for r, n in enumerate(new):
        a, b = starts[r], starts[r + 1] - (r == 1)                  # (the row that sees a NaN key is looked at below)
        for h in range(8):
            pos = torch.arange(c.ctx[r] - n, c.ctx[r] - (r == 1), device="cuda")
            compare((out[a:b, h], top[h, a:b], total[h, a:b]), exact(q[a:b, h], c.k[r][h // 4], c.v[r][h // 4], pos, window, n_sink), f"request {r}, head {h}")
    assert out[239].isnan().all() and total[:, 239].isnan().all()


@pytest.mark.parametrize("window,n_sink", [(0, 0), (17000, 40)])
def test_qpage_attn_hidden_values_far_apart(window, n_sink):
    """NaN in edge tiles of the first and of later turns of the loop over keys: rows that see them, rows that do not."""
    c = ByteCache(31, [34000], 1, 32)
    for at in (3, 39, 33850, 33999):
        c.v[0][0, at, at % D] = NAN
    if window:
        c.v[0][0, 16900, 7] = NAN                                   # behind the left edge of some rows
    c.fill()
    check_attn(c, [200], 2, window, n_sink)


@pytest.mark.parametrize("ctx,new,top,gain", [([300], [1], 5, 4), ([300], [300], 170, 4), ([290, 300], [60, 1], 170, 4), ([6000], [1], 4000, 24), ([9000], [100], 5000, 24),
                                              ([4000, 5000], [1, 200], 3000, 24)])
def test_qpage_attn_nan_of_little_weight(ctx, new, top, gain):
    """A value that a row sees is in its result whatever its weight: 65 and 391 log2 units below the largest, in tiles that all rows see and in
    ones that some do, where sums of waves and of pieces meet."""
    c = ByteCache(82, ctx, 2, 16)
    q = torch.cat([one_way(gen_of(82 + r), c.k[r], top, gain, n, 8) for r, n in enumerate(new)])
    for r, v in enumerate(c.v):
        for i, at in enumerate((3, 40, 100, ctx[r] // 2, ctx[r] - 129, ctx[r] - 20)):
            v[:, at, 7 * i + 1] = NAN
    c.fill()
    check_attn(c, new, 8, q=q)


def test_qpage_attn_pages_that_are_none():
    """Keys of such pages, and behind the table's end, are not seen; a row that sees nothing is zero."""
    page, ctx, new = 16, [200, 64, 90, 50], [40, 64, 90, 1]
    c = ByteCache(4, ctx, 2, page)
    c.table[0, 3], c.table[0, 12] = -1, c.n_pages                   # positions 48 .. 63 and 192 .. 207
    c.table[1, 0] = 1 << 30                                         # rows 0 .. 15 of the second request see nothing
    c.table[2, :] = -1
    hidden = [torch.zeros(n, dtype=torch.bool, device="cuda") for n in ctx]
    hidden[0][48:64], hidden[0][192:], hidden[1][:16], hidden[2][:] = True, True, True, True
    out = check_attn(c, new, 8, hidden=hidden)
    assert (out[40:56] == 0).all() and (out[104:194] == 0).all()
    for p in (32, 64):
        c = ByteCache(4, [200, 300], 2, p)
        c.table[0, 1], c.table[1, 0] = -7, c.n_pages + 5
        hidden = [torch.zeros(n, dtype=torch.bool, device="cuda") for n in (200, 300)]
        hidden[0][p:2 * p], hidden[1][:p] = True, True
        check_attn(c, [100, 300], 8, hidden=hidden, window=150, n_sink=70)


def test_qpage_attn_lengths_beyond_the_table():
    """A context longer than the table's row holds, one shorter than its rows, and none at all."""
    c = ByteCache(4, [96, 20, 30], 2, 16, extra=0)                  # 6 entries a row
    k, v = ([torch.cat([x, torch.zeros(2, 30, D, dtype=torch.float16, device="cuda")], dim=1) for x in y] for y in (c.k, c.v))
    q, new, ctx, starts = randn(gen_of(2), 60, 8, D), [20, 30, 10], [110, 20, 0], [0, 20, 50, 60]
    out, top, total = antkv.qpage_attn(antkv.Geometry(3, 8, 2, 8), q, SCALE, ints(starts), ints(ctx), c.table, *c.pools.args(), want_stats=True)
    for r in range(3):
        a, b = starts[r], starts[r + 1]
        pos = torch.arange(ctx[r] - new[r], ctx[r], device="cuda")  # negative ones see nothing
        hidden = torch.arange(k[r].shape[1], device="cuda") >= min(ctx[r], 96)
        for h in range(8):
            compare((out[a:b, h], top[h, a:b], total[h, a:b]), exact(q[a:b, h], k[r][h // 4], v[r][h // 4], pos, 0, 0, hidden=hidden), f"{r} {h}")


def test_qpage_attn_starts_that_are_no_starts():
    """Rows that are no request's are never followed; requests that overlap write nothing."""
    c = ByteCache(41, [100, 60, 90], 2, 16)
    q, geom = randn(gen_of(41), 20, 8, D), antkv.Geometry(3, 8, 2, 8)
    run = lambda starts: antkv.qpage_attn(geom, q, SCALE, ints(starts), ints(c.ctx), c.table, *c.pools.args())[0]
    want = run([0, 5, 5, 5])
    for starts in ([0, 5, 3, 3], [0, 5, 900, 10 ** 9], [0, 5, -7, -9]):
        assert torch.equal(run(starts)[:3].view(torch.int16), want[:3].view(torch.int16)), starts
    out = torch.full((20, 8, D), 7.0, dtype=torch.float16, device="cuda")
    antkv.qpage_attn(geom, q, SCALE, ints([0, 20, 0, 20]), ints(c.ctx), c.table, *c.pools.args(), out=out)
    assert (out == 7.0).all()


def test_qpage_attn_as_many_requests_as_there_may_be():
    """8192 requests on 8 KV heads, more than 65535 pairs of them: attention, and their rows out of the pages."""
    rng = np.random.default_rng(91)
    R, Hkv, page = 8192, 8, 16
    ctx = rng.integers(1, 40, R).tolist()
    new = [0 if r % 5 == 0 else min(c, 1 + 30 * (r % 97 == 0)) for r, c in enumerate(ctx)]
    pools, gen = Pools(3 * R, Hkv, page, seed=91), gen_of(91)
    table = torch.randperm(3 * R, device="cuda", generator=gen).to(torch.int32).view(R, 3).contiguous()
    starts = np.concatenate([[0], np.cumsum(new)])
    q, geom = randn(gen, int(starts[-1]), 2 * Hkv, D), antkv.Geometry(R, 2 * Hkv, Hkv, 8)
    q *= 0.01                                                       # (values up to 448 x 2)
    out, top, total = antkv.qpage_attn(geom, q, SCALE, ints(starts), ints(ctx), table, *pools.args(), want_stats=True)
    k, v = antkv.qpage_load(geom, *pools.args(), table, 39, ctx_len=ints(ctx))
    assert out.isfinite().all()
    for r in [*range(0, R, 97), R - 2, R - 1]:
        a, b, n = int(starts[r]), int(starts[r + 1]), ctx[r]
        pos = torch.arange(n - new[r], n, device="cuda")
        for h in range(r % 3, 2 * Hkv if new[r] else 0, 3):
            compare((out[a:b, h], top[h, a:b], total[h, a:b]), exact(q[a:b, h], k[r, h // 2, :n], v[r, h // 2, :n], pos, 0, 0), f"request {r}, head {h}")
        for x, b8, s in zip((k, v), pools.bytes, pools.scales):
            rows = (b8[table[r].long()].float() * s[table[r].long()].repeat_interleave(16, 2)[..., None]).transpose(0, 1).flatten(1, 2)
            assert torch.equal(x[r, :, :n], rows[:, :n].half()) and (x[r, :, n:] == 0).all()


def test_qpage_attn_requests_that_share_pages():
    c = ByteCache(72, [100, 64, 80], 2, 16)
    for r in (1, 2):
        c.table[r, :4] = c.table[0, :4]
        c.k[r][:, :64], c.v[r][:, :64] = c.k[0][:, :64], c.v[0][:, :64]
    check_attn(c, [1, 20, 10], 8)


@pytest.mark.parametrize("ctx,new", [([3000, 1, 700] + [20] * 37, [1, 1, 90] + [1] * 37), ([40000] + [20] * 39, [1] * 40)])
def test_qpage_attn_tables_of_great_capacity(ctx, new):
    """Tables for so many tokens that a batch might cost more than the shares can count: a workgroup per block, of many turns too."""
    c = ByteCache(53, ctx, 2, 256)
    table = torch.full((40, 1 << 22), -1, dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = c.table
    c.table = table
    check_attn(c, new, 8)


def test_qpage_attn_same_bits_whatever_the_workspace_held():
    c = ByteCache(4, [9000, 700, 1], 2, 64)
    first = check_attn(c, [1, 100, 1], 8)
    for fill in (0, 1, 255):
        ws = antkv.qpage_attn_workspace(antkv.Geometry(3, 8, 2, 8), 102, "cuda").fill_(fill)
        again = check_attn(c, [1, 100, 1], 8, workspace=ws)
        assert torch.equal(first.view(torch.int16), again.view(torch.int16))


def test_qpage_attn_on_two_streams():
    caches = [ByteCache(s, [3000 + s, 50], 2, 16) for s in (0, 1)]
    qs = [randn(gen_of(s), 33, 8, D) for s in (0, 1)]
    geom, starts = antkv.Geometry(2, 8, 2, 8), ints([0, 1, 33])
    args = [(geom, q, SCALE, starts, ints(c.ctx), c.table, *c.pools.args()) for c, q in zip(caches, qs)]
    want = [antkv.qpage_attn(*a)[0] for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(antkv.qpage_attn(*args[i])[0])
    torch.cuda.synchronize()
    assert all(torch.equal(x.view(torch.int16), want[i].view(torch.int16)) for i in range(2) for x in got[i])


def test_qpools_of_more_than_32_bits():
    """Pages whose bytes lie beyond 2^32: stored, loaded and read as those of a small pool."""
    Hkv, page, n_pages = 8, 256, 18000                              # 4.7e9 bytes to a pool
    big = [torch.empty((n_pages, Hkv, page, D), dtype=torch.uint8, device="cuda").view(E4M3) for _ in "kv"] + [torch.empty((n_pages, Hkv, page // 16), device="cuda") for _ in "kv"]
    assert big[0].numel() > 1 << 32
    ctx, new, gen = [700, 300], [1, 300], gen_of(21)
    geom, T = antkv.Geometry(2, 4 * Hkv, Hkv, 8), sum(ctx)
    k, v = randn(gen, T, Hkv, D), randn(gen, T, Hkv, D)
    pos = np.concatenate([np.arange(n) for n in ctx])
    small, tables = Pools(6, Hkv, page), ([[4, 0, 5], [2, 3, 1]], [[17999, 9000, 17], [4096, 16500, 8192]])
    outs = []
    for pools, table in ((small.args(), tables[0]), (big, tables[1])):
        pages = np.concatenate([np.asarray(table[r])[np.arange(n) // page] for r, n in enumerate(ctx)])
        antkv.qpage_store(geom, k, v, ints(pages * page + pos % page), *pools)
        q = randn(gen_of(22), sum(new), 4 * Hkv, D)
        outs.append((*antkv.qpage_load(geom, *pools, ints(table), 700, ctx_len=ints(ctx)),
                     antkv.qpage_attn(geom, q, SCALE, ints([0, 1, 301]), ints(ctx), ints(table), *pools)[0]))
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(*outs)) and outs[0][2].isfinite().all()


# ------------------------------------------------------------------------------------------------ all of them together

def test_prompts_in_chunks_through_rope_and_bytes_until_they_are_codes():
    """Two prompts in uneven chunks beside a request that decodes: rope, store, attention over what was stored; then out of the pages, turned
    back, and through selection and encoding.  Attention against 64 bits over the pages' own values; those against the rows that went in."""
    Hq, Hkv, page, n_pages, d = 8, 2, 32, 40, 8
    gen, steps = gen_of(11), [[0, 0, 56], [100, 64, 1], [1, 136, 1], [232, 0, 1], [0, 0, 1]]
    lens = [sum(s[r] for s in steps) for r in range(3)]
    K, V, Q = ([randn(gen, h, n, D) for n in lens] for h in (Hkv, Hkv, Hq))
    geom, one, freqs = antkv.Geometry(3, Hq, Hkv, d), antkv.Geometry(1, Hq, Hkv, d), antkv.rope_freqs(128, 10000.0, 4.0, 200)
    turned = lambda X, r, first, n: antkv.rope(one, X[r][None, :, first:first + n].contiguous() if X is Q else None,
                                               X[r][None, :, first:first + n].contiguous() if X is K else None, freqs, pos0=first, style=1)
    pools = Pools(n_pages, Hkv, page)
    table, free = torch.full((3, 16), -1, dtype=torch.int32, device="cuda"), torch.randperm(n_pages, device="cuda", generator=gen).to(torch.int32)
    done, at, held, stats = [0, 0, 0], None, ints([0, 0, 0]), [[], [], []]
    for new in steps:
        T = sum(new) + 2                                            # (a padded batch)
        rows = lambda X: torch.cat([X[r][:, done[r]:done[r] + n] for r, n in enumerate(new)] + [X[0][:, :2]], dim=1).transpose(0, 1).contiguous()
        held, q_start, slot, at = antkv.page_map(held, ints(new), table, page, n_pages, free, T, free_at=at)
        q, k, v = rows(Q), rows(K), rows(V)
        antkv.rope(geom, q, k, freqs, q_start=q_start, ctx_len=held, style=1, q_out=q, k_out=k)
        a = 0
        for r, n in enumerate(new):                                 # packed rows turn as dense ones do
            if n:
                assert torch.equal(q[a:a + n].transpose(0, 1), turned(Q, r, done[r], n)[0][0]) and torch.equal(k[a:a + n].transpose(0, 1), turned(K, r, done[r], n)[1][0])
            a += n
        antkv.qpage_store(geom, k, v, slot, *pools.args())
        out, top, total = antkv.qpage_attn(geom, q, SCALE, q_start, held, table, *pools.args(), want_stats=True)
        done = [x + n for x, n in zip(done, new)]
        dk, dv = antkv.qpage_load(geom, *pools.args(), table, max(done), ctx_len=held)
        a = 0
        for r, n in enumerate(new):
            for h in range(Hq if n else 0):
                want = exact(q[a:a + n, h], dk[r, h // 4, :done[r]], dv[r, h // 4, :done[r]], torch.arange(done[r] - n, done[r], device="cuda"), 0, 0)
                compare((out[a:a + n, h], top[h, a:a + n], total[h, a:a + n]), want, f"{new} {r} {h}")
            stats[r].append((top[:, a:a + n], total[:, a:a + n]))
            a += n
    assert held.tolist() == done == lens and at.tolist()[1] == 0
    for r in range(2):
        n = lens[r]
        kd, vd = antkv.qpage_load(one, *pools.args(), table[r:r + 1], n)
        kt = turned(K, r, 0, n)[1]
        for got, x, s in ((kd, kt, pools.scales[0]), (vd, V[r][None, :, :n], pools.scales[1])):
            j = torch.arange(n, device="cuda")
            unit = s[table[r].long()[j // page], :, j % page // 16].transpose(0, 1).double()[None, ..., None]
            assert ((got.double() - x.double()).abs() <= torch.maximum(x.double().abs() / 16, 2.0 ** -10 * unit) + 2.0 ** -9 * unit).all()
        # back to where keys were before RoPE: a rounding more on either side of those of the pages
        plain = antkv.rope(one, None, kd, freqs, style=1, inverse=True)[1]
        err = (plain.double() - K[r][None, :, :n].double()).norm(dim=-1) / K[r][None, :, :n].double().norm(dim=-1)
        assert err.max() <= 2.0 ** -4 + 3 * 2.0 ** -11              # e4m3: half a step at most of each value, so of their norm
        qt = turned(Q, r, 0, n)[0]
        top, total = (torch.cat([s[i] for s in stats[r]], dim=1)[None].contiguous() for i in range(2))
        idx_k, idx_v, ans_k, ans_v = antkv.anchor_select(one, qt, kd, SCALE, 4)
        assert all(((x[..., 1:] - x[..., :-1]) > 0).all() and (x >= 0).all() and (x < n).all() for x in (idx_k, idx_v))
        cb = randn(gen, Hkv, D // d, 256, d)
        codes_k, codes_v = antkv.encode(one, plain, cb), antkv.encode(one, vd, cb)
        rows_k, rows_v = antkv.gather_rows(one, plain, idx_k), antkv.gather_rows(one, vd, idx_v)
        step = antkv.decode_attn_prerope(one, qt[:, :, -1].contiguous(), SCALE, codes_k, codes_v, cb, cb, idx_k, rows_k, idx_v, rows_v, rope_style=1)
        assert step.isfinite().all()


@pytest.mark.parametrize("most", [1, 100])
def test_captured_step_replayed_over_other_lengths(most):
    """Map, rope, store and attention captured in two graphs that share a workspace, replayed over contexts whose lengths change places and size
    (other numbers of pieces per block), eager steps between: every replay against the eager step on copies, bit for bit."""
    Hq, Hkv, page, R, own = 8, 2, 16, 4, 200
    T = R - 1 + most
    gen, geom, freqs = gen_of(93), antkv.Geometry(R, Hq, Hkv, 8), antkv.rope_freqs(64)
    n_pages = R * own + 40
    pools = Pools(n_pages, Hkv, page, seed=94)
    order = torch.randperm(n_pages, device="cuda", generator=gen).to(torch.int32)
    whole, free = order[:R * own].view(R, own), order[R * own:].contiguous()
    table, held, new = whole.clone(), ints([0] * R), ints([1] * R)
    q, k, v = randn(gen, T, Hq, D), randn(gen, T, Hkv, D), randn(gen, T, Hkv, D)
    ws, out = antkv.qpage_attn_workspace(geom, T, "cuda"), torch.empty((T, Hq, D), dtype=torch.float16, device="cuda")
    qr, kr = torch.empty_like(q), torch.empty_like(k)

    def step(table, kp, vp, ks, vs, out, qr, kr, ws):
        lens, q_start, slot, _ = antkv.page_map(held, new, table, page, n_pages, free, T)
        antkv.rope(geom, q, k, freqs, q_start=q_start, ctx_len=lens, style=0, q_out=qr, k_out=kr)
        antkv.qpage_store(geom, kr, v, slot, kp, vp, ks, vs)
        antkv.qpage_attn(geom, qr, SCALE / 100, q_start, lens, table, kp, vp, ks, vs, out=out, workspace=ws)

    state = [table, *pools.args(), out, qr, kr]
    step(*state, ws)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(*state, ws)
        graphs.append(graph)
    lengths = [[3000, 900, 40, 5], [5, 40, 900, 3000], [40, 3000, 5, 900], [20, 30, 5, 40], [700, 5, 40, 2900], [3000, 5, 40, 900], [1, 15, 60, 3000]]
    for i in range(2 * len(lengths)):                               # (an odd number of them: each goes to both graphs)
        ctx = lengths[i % len(lengths)]
        fresh = [1] * R
        fresh[int(np.argmax(ctx)) if i % 3 else int(np.argsort(ctx)[-2])] = most
        held.copy_(ints([max(c - n, 0) for c, n in zip(ctx, fresh)]))
        new.copy_(ints(fresh))
        table.copy_(whole)
        for x in (q, k, v):
            x.normal_()
        eager = [t.clone() for t in state]
        step(*eager, antkv.qpage_attn_workspace(geom, T, "cuda"))
        graphs[i & 1].replay()
        torch.cuda.synchronize()
        raw = lambda t: t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])
        for got, want in zip(state, eager):
            assert torch.equal(raw(got), raw(want)), f"replay {i}"
        assert out.isfinite().all()


def test_a_step_on_another_stream():
    Hq, Hkv, page, n_pages, n = 8, 2, 16, 40, 500
    gen, geom, one = gen_of(51), antkv.Geometry(1, Hq, Hkv, 8), ints([n])
    k, v, q = randn(gen, n, Hkv, D), randn(gen, n, Hkv, D), randn(gen, n, Hq, D)
    free = torch.randperm(n_pages, device="cuda", generator=gen).to(torch.int32)

    def step():
        pools = [torch.zeros((n_pages, Hkv, page, D), device="cuda").to(E4M3) for _ in "kv"] + [torch.zeros((n_pages, Hkv, page // 16), device="cuda") for _ in "kv"]
        table = torch.full((1, n_pages), -1, dtype=torch.int32, device="cuda")
        ctx, starts, slot, _ = antkv.page_map(ints([0]), one, table, page, n_pages, free, n)
        freqs = antkv.rope_freqs(128, 500000.0)
        qr, kr = antkv.rope(geom, q, k, freqs, q_start=starts, ctx_len=ctx)
        antkv.qpage_store(geom, kr, v, slot, *pools)
        out = antkv.qpage_attn(geom, qr, SCALE, starts, ctx, table, *pools, window=90, n_sink=3)[0]
        return out, *antkv.qpage_load(geom, *pools, table, n), *pools[2:]

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(3):
            got = step()
    side.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, want)) and got[0].isfinite().all()
