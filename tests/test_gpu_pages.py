"""GPU checks of the paged FP16 cache and of windowed prompts against plain implementations: integers exactly, attention against
64 bits.

Attention tolerances: the weights and the output are rounded to fp16, 2^-11 relative each, the scores are fp32 sums of 128 exact
products and the rest is fp32: 2^-10 + 1e-4 relative L2 per row.  Row maxima are such scores (1e-5 at the magnitudes used, as a
share of them beyond 1), row sums fp32 sums of exponentials of them (1e-4)."""
import numpy as np
import pytest
import torch

import paper_2506_19505_amd as antkv

pytestmark = pytest.mark.gpu

D = 128
SCALE = D ** -0.5
OUT_TOL = 2.0 ** -10 + 1e-4


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def gen_of(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(gen, *shape):
    return torch.randn(shape, dtype=torch.float16, device="cuda", generator=gen)


# ------------------------------------------------------------------------------------------------ page_map

def plain_map(held, new, table, page, n_pages, free, at, T):
    table, cap = table.copy(), table.shape[1]
    R, slots, starts, missing, take = len(held), [], [0], 0, at
    ok = lambda p: p if 0 <= p < n_pages else -1
    for r in range(R):
        h, n = max(0, held[r]), max(0, new[r])
        has, need = min(cap, -(-h // page)), min(cap, -(-(h + n) // page))
        short = starts[-1] + n > T or h + n > cap * page
        for i in range(has, need):
            short |= take >= len(free)
            table[r, i] = ok(free[take]) if take < len(free) else -1
            take += 1
        for j in range(h, h + n):
            p = ok(table[r, j // page]) if j // page < cap else -1
            slots.append(p * page + j % page if p >= 0 else -1)
        if n and h % page and h // page < cap:
            short |= ok(table[r, h // page]) < 0
        missing += bool(n and short)
        starts.append(starts[-1] + n)
    slots = (slots + [-1] * T)[:T]
    ctx = [max(0, h) + max(0, n) for h, n in zip(held, new)]
    return ctx, starts, slots, table, [min(take, len(free)), missing]


def check_map(held, new, page, cap, T, free_count=None, at=None, seed=0, spoil=None):
    rng = np.random.default_rng(seed)
    R = len(held)
    has = [min(cap, -(-max(0, h) // page)) for h in held]
    n_pages = sum(has) + sum(-(-max(0, n) // page) + 1 for n in new) + 5
    order = rng.permutation(n_pages)
    table = rng.integers(-9, 1 << 20, (R, cap)).astype(np.int32)    # what is behind a row's pages is anything
    used = 0
    for r in range(R):
        table[r, :has[r]] = order[used:used + has[r]]
        used += has[r]
    free = order[used:].astype(np.int32)
    if free_count is not None:
        free = free[:free_count]
    if spoil:
        spoil(table, free)
    want = plain_map(held, new, table, page, n_pages, free, at or 0, T)
    dev_table = ints(table)
    got = antkv.page_map(ints(held), ints(new), dev_table, page, n_pages, ints(free), T, free_at=None if at is None else ints([at, 77]))
    for g, w, what in zip((got[0], got[1], got[2], dev_table, got[3]), want, ("ctx_len", "q_start", "slot", "table", "status")):
        np.testing.assert_array_equal(g.cpu().numpy(), np.asarray(w, dtype=np.int64), err_msg=what)


@pytest.mark.parametrize("R,page,longest,most_new,seed", [(1, 16, 1, 1, 0), (1, 64, 5000, 3000, 1), (5, 16, 40, 40, 2), (64, 32, 3000, 1, 3), (256, 16, 500, 3, 4),
                                                          (257, 64, 900, 90, 5), (1000, 128, 1000, 40, 6), (8192, 16, 60, 2, 7), (7, 256, 9000, 9000, 8)])
def test_page_map(R, page, longest, most_new, seed):
    rng = np.random.default_rng(100 + seed)
    held = rng.integers(0, longest + 1, R)
    new = rng.integers(0, most_new + 1, R)
    held[rng.random(R) < 0.2] = 0
    on_edge = rng.random(R) < 0.2
    held[on_edge] = held[on_edge] // page * page                    # pages that are just full
    new[rng.random(R) < 0.2] = 0
    cap = int(max(-(-(held + new) // page))) + 2
    for T in {int(new.sum()), int(new.sum()) + 13}:                 # a padded batch too
        check_map(held.tolist(), new.tolist(), page, cap, T, seed=seed)
    check_map(held.tolist(), new.tolist(), page, cap, int(new.sum()), at=3, seed=seed)


def test_page_map_without_room():
    held, new = [10, 33, 0, 16, 100], [20, 31, 5, 16, 60]
    T = sum(new)
    for count in (0, 1, 3, 5):
        check_map(held, new, 16, 12, T, free_count=count)
    check_map(held, new, 16, 4, T)                                  # table rows too short
    check_map(held, new, 16, 12, T - 20)                            # the batch too short
    check_map(held, new, 16, 12, 0)
    check_map([-5, 3, 2147483600], [4, -7, 30], 16, 4, 34)          # no lengths that a request has
    check_map(held, new, 16, 12, T, at=1000)

    def spoil(table, free):
        table[0, 0], table[1, 2], free[1], free[2] = -3, 1 << 30, -1, 1 << 20
    held2 = [10, 33, 0, 16, 100]
    rng_spoiled = dict(held=held2, new=[20, 31, 0, 0, 0], page=16, cap=12, T=51, spoil=spoil)
    check_map(**rng_spoiled)


def test_page_map_of_no_request():
    out = antkv.page_map(ints([]), ints([]), torch.zeros((0, 4), dtype=torch.int32, device="cuda"), 16, 8, ints([1, 2]), 3, free_at=ints([1]))
    assert out[1].tolist() == [0] and out[2].tolist() == [-1] * 3 and out[3].tolist() == [1, 0]


def test_page_map_goes_on_without_the_host():
    """Steps that take each other's status and lengths, written alternately into two sets of arrays."""
    R, page, n_pages = 3, 16, 64
    table, free = torch.full((R, 12), -1, dtype=torch.int32, device="cuda"), torch.randperm(n_pages, device="cuda").to(torch.int32)
    held, at, new = ints([0] * R), None, ints([5, 0, 17])
    outs = [None, None]
    for step in range(8):
        outs[step & 1] = antkv.page_map(held, new, table, page, n_pages, free, 22, free_at=at, out=outs[step & 1])
        held, _, slot, at = outs[step & 1]
        assert slot.unique().numel() == 22
    assert held.tolist() == [40, 0, 136] and at.tolist() == [3 + 9, 0]
    assert sorted(table[table >= 0].tolist()) == sorted(free[:12].tolist())


# ------------------------------------------------------------------------------------------------ page_store, page_load

@pytest.mark.parametrize("T,Hkv,page,fused", [(1, 1, 16, False), (1, 8, 64, True), (7, 2, 16, True), (31, 7, 32, False), (33, 3, 128, True),
                                              (1000, 8, 256, True), (4097, 4, 16, False)])
def test_page_store(T, Hkv, page, fused):
    gen = gen_of(T)
    n_pages = T // page + 3
    kp, vp = randn(gen, n_pages, Hkv, page, D), randn(gen, n_pages, Hkv, page, D)
    if fused:                                                       # Q, K and V heads of a token side by side
        x = randn(gen, T, 6 * Hkv, D)
        k, v = x[:, 4 * Hkv:5 * Hkv], x[:, 5 * Hkv:]
    else:                                                           # heads first
        k, v = randn(gen, Hkv, T, D).transpose(0, 1), randn(gen, Hkv, T, D).transpose(0, 1)
    slot = torch.randperm(n_pages * page, device="cuda", generator=gen)[:T].to(torch.int32)
    if T > 4:
        slot[1], slot[2], slot[3] = -1, n_pages * page, -2 ** 31
    want = [p.clone() for p in (kp, vp)]
    for t, s in enumerate(slot.tolist()):
        if 0 <= s < n_pages * page:
            want[0][s // page, :, s % page] = k[t]
            want[1][s // page, :, s % page] = v[t]
    antkv.page_store(antkv.Geometry(1, Hkv, Hkv, 8), k, v, slot, kp, vp)
    assert torch.equal(kp, want[0]) and torch.equal(vp, want[1])


@pytest.mark.parametrize("B,Hkv,page,N,first", [(1, 1, 16, 1, 0), (2, 8, 16, 67, 0), (3, 7, 64, 130, 5), (1, 4, 256, 1000, 700), (5, 2, 32, 33, 31)])
def test_page_load(B, Hkv, page, N, first):
    gen = gen_of(N)
    cap = -(-(first + N) // page) + 1
    n_pages = B * cap + 2
    kp, vp = randn(gen, n_pages, Hkv, page, D), randn(gen, n_pages, Hkv, page, D)
    table = torch.randperm(n_pages, device="cuda", generator=gen)[:B * cap].view(B, cap).to(torch.int32).contiguous()
    lens = [first + N + 9, first, first + N // 2, 0, -4][:B]
    geom = antkv.Geometry(B, 4 * Hkv, Hkv, 8)
    pos = torch.arange(first, first + N, device="cuda")
    dense = [p[table.long()[:, pos // page], :, pos % page].transpose(1, 2) for p in (kp, vp)]
    k, v = antkv.page_load(geom, kp, vp, table, N, first=first)
    assert torch.equal(k, dense[0]) and torch.equal(v, dense[1])
    before = randn(gen, B, Hkv, N, D), randn(gen, B, Hkv, N, D)
    table[0, -2], table[0, 0] = -1, n_pages                         # pages that are none
    there = (pos < ints(lens)[:, None]) & (table[:, (pos // page)] >= 0) & (table[:, (pos // page)] < n_pages)
    got = antkv.page_load(geom, kp, vp, table, N, first=first, ctx_len=ints(lens), k=before[0].clone(), v=before[1].clone())
    for g, d, b in zip(got, dense, before):
        assert torch.equal(g, torch.where(there[:, None, :, None], d, b))


# ------------------------------------------------------------------------------------------------ attention

def exact(q, k, v, pos, window, n_sink, scale=SCALE, hidden=None):
    """64 bits: q [n, D] at positions pos [n], k, v [C, D] -> out, row_max, row_sum; a hidden value takes no part, whatever it is."""
    j = torch.arange(k.shape[0], device="cuda")
    p = pos[:, None]
    seen = j <= p
    if window:
        seen &= (j > p - window) | (j < n_sink)
    if hidden is not None:
        seen &= ~hidden
    s = torch.where(seen, scale * (q.double() @ torch.where(seen.any(0)[:, None], k, 0).double().t().contiguous()), -float("inf"))
    m = s.amax(-1) if k.shape[0] else torch.full((q.shape[0],), -float("inf"), dtype=torch.float64, device="cuda")
    e = torch.where(seen, torch.exp(s - torch.where(m == -float("inf"), 0, m)[:, None]), 0.0)
    fine = torch.where(v.isfinite() & seen.any(0)[:, None], v, 0).double()
    out = (e @ fine) / torch.where(e.sum(-1) > 0, e.sum(-1), 1.0)[:, None]
    for value, there in ((float("inf"), v == float("inf")), (-float("inf"), v == -float("inf")), (float("nan"), v.isnan())):
        out = torch.where(seen.double() @ there.double() > 0, out + value, out)
    return out, m, e.sum(-1)


def compare(got, want, what=""):
    out, top, total = (x.double() for x in got)
    w_out, w_top, w_total = want
    assert torch.equal(out.isfinite(), w_out.isfinite()) and torch.equal(out.isnan(), w_out.isnan()), what
    bad = ~w_out.isfinite() & ~w_out.isnan()
    assert torch.equal(out[bad], w_out[bad]), what
    clean = w_out.isfinite()
    a, b = torch.where(clean, out, 0), torch.where(clean, w_out, 0)
    err = (a - b).norm(dim=-1)
    assert (err <= OUT_TOL * b.norm(dim=-1)).all(), f"{what}: relative L2 {(err / b.norm(dim=-1).clamp(min=1e-30)).max().item():.2e}"
    none = w_top == -float("inf")
    assert torch.equal(top == -float("inf"), none) and (total[none] == 0).all() and (out[none] == 0).all(), what
    assert ((top - w_top)[~none].abs() <= 1e-5 * w_top[~none].abs().clamp(min=1)).all(), what
    assert ((total / w_total - 1)[~none].abs() <= 1e-4).all(), what


class Cache:
    """Pages of a batch of requests whose rows are k[r], v[r] [Hkv, ctx, D]; what no request holds is NaN."""

    def __init__(self, seed, ctx, Hkv, page, extra=2):
        gen = gen_of(seed)
        counts = [-(-c // page) for c in ctx]
        self.page, self.ctx, self.n_pages = page, ctx, sum(counts) + 3
        self.k_pages = torch.full((self.n_pages, Hkv, page, D), float("nan"), dtype=torch.float16, device="cuda")
        self.v_pages = torch.full_like(self.k_pages, float("nan"))
        self.k, self.v = [randn(gen, Hkv, c, D) for c in ctx], [randn(gen, Hkv, c, D) for c in ctx]
        self.table = torch.full((len(ctx), max(counts, default=0) + extra), -1, dtype=torch.int32, device="cuda")
        order = torch.randperm(self.n_pages, device="cuda", generator=gen).to(torch.int32)
        used = 0
        for r, n in enumerate(counts):
            self.table[r, :n] = order[used:used + n]
            used += n
        self.fill()

    def fill(self):
        for r, c in enumerate(self.ctx):
            if c == 0:
                continue
            j = torch.arange(c, device="cuda")
            ids = self.table[r].long()[j // self.page]
            self.k_pages[ids, :, j % self.page] = self.k[r].transpose(0, 1)
            self.v_pages[ids, :, j % self.page] = self.v[r].transpose(0, 1)


def check_attn(c, new, Hq, window=0, n_sink=0, q=None, pad=0, seed=1, scale=SCALE, hidden=None, workspace=None, ctx=None, each=1):
    """Every row of the batch against 64 bits; rows behind the last request stay as they are."""
    Hkv, R, T = c.k_pages.shape[1], len(new), sum(new) + pad
    G = Hq // Hkv
    if q is None:
        q = randn(gen_of(seed), T, Hq, D)
    starts = np.concatenate([[0], np.cumsum(new)])
    out = torch.full((T, Hq, D), 7.0, dtype=torch.float16, device="cuda")
    geom = antkv.Geometry(R, Hq, Hkv, 8)
    got, top, total = antkv.page_attn(geom, q, scale, ints(starts), ints(ctx or c.ctx), c.table, c.k_pages, c.v_pages, window=window, n_sink=n_sink,
                                      out=out, want_stats=True, workspace=workspace)
    assert got is out and (out[starts[-1]:] == 7.0).all()
    lean = antkv.page_attn(geom, q, scale, ints(starts), ints(ctx or c.ctx), c.table, c.k_pages, c.v_pages, window=window, n_sink=n_sink)
    assert lean[1] is None and torch.equal(lean[0][:starts[-1]].view(torch.int16), out[:starts[-1]].view(torch.int16))
    for r, n in enumerate(new):
        a, b = int(starts[r]), int(starts[r + 1])
        pos = torch.arange((ctx or c.ctx)[r] - n, (ctx or c.ctx)[r], device="cuda")
        for h in range(0, Hq if n else 0, each):
            want = exact(q[a:b, h], c.k[r][h // G], c.v[r][h // G], pos, window, n_sink, scale, None if hidden is None else hidden[r])
            compare((out[a:b, h], top[h, a:b], total[h, a:b]), want, f"request {r}, head {h}")
    return out


# one token and many, groups of 1, 2 and 4, heads that are no multiple of 8, contexts that end inside a page, a tile, at their ends;
# requests without tokens, with one key
BATCHES = [
    (8, 2, 16, [1], [1]), (8, 2, 16, [17], [1]), (4, 4, 64, [33, 64, 1, 65], [1, 1, 1, 1]), (8, 8, 32, [40, 7], [40, 7]), (14, 7, 16, [100, 31, 32], [1, 31, 0]),
    (8, 2, 128, [300, 129, 5], [300, 3, 0]), (16, 8, 256, [700, 20, 256], [33, 20, 200]), (32, 8, 64, [2500], [1]), (4, 1, 16, [1000, 900, 800, 31], [1, 64, 65, 31]),
    (2, 2, 32, [511, 512, 513], [129, 128, 127]), (28, 7, 64, [5000, 60], [9, 60]), (8, 2, 16, [4100], [2]), (8, 8, 16, [2000, 3], [257, 1]),
]


@pytest.mark.parametrize("window,n_sink", [(0, 0), (1, 0), (40, 4), (100, 37), (64, 0), (5000, 3)])
@pytest.mark.parametrize("Hq,Hkv,page,ctx,new", BATCHES)
def test_page_attn(Hq, Hkv, page, ctx, new, window, n_sink):
    check_attn(Cache(len(ctx) + page, ctx, Hkv, page), new, Hq, window, n_sink, pad=3)


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("Hq,Hkv,ctx,new,window,n_sink", [(4, 1, [40000], [1], 0, 0), (4, 1, [33000, 70000], [40, 1], 0, 0), (4, 2, [66000], [3], 60000, 100),
                                                          (2, 2, [35000], [300], 0, 0)])
def test_page_attn_long(Hq, Hkv, page, ctx, new, window, n_sink):
    """More key tiles than a workgroup looks pages up for at a time, and ranges of them."""
    check_attn(Cache(page, ctx, Hkv, page), new, Hq, window, n_sink)


def test_page_attn_many_requests():
    """More requests than threads of a workgroup, most of them with a token, some with none."""
    rng = np.random.default_rng(3)
    ctx = rng.integers(1, 90, 700).tolist()
    new = [int(min(c, n)) for c, n in zip(ctx, rng.integers(0, 3, 700))]
    check_attn(Cache(5, ctx, 1, 16), new, 2)


def test_page_attn_wide_batch():
    """Enough rows for workgroups of eight waves; requests of one token among long chunks."""
    check_attn(Cache(9, [1500, 900, 2000, 1, 400], 8, 32), [1500, 1, 300, 1, 0], 32, pad=5)
    check_attn(Cache(9, [1500, 900, 2000, 1, 400], 8, 32), [1500, 1, 300, 1, 0], 32, window=200, n_sink=5)


def test_page_attn_a_workgroup_per_block():
    """Many blocks: of many requests of few tokens, in shares, and of a long prompt, each a workgroup of its own."""
    rng = np.random.default_rng(4)
    ctx = rng.integers(1, 300, 300).tolist()
    check_attn(Cache(6, ctx, 8, 16), [1 + (r % 7 == 0) * min(c - 1, 40) for r, c in enumerate(ctx)], 16, each=3)
    check_attn(Cache(7, [8300, 40], 8, 64), [8250, 1], 32, each=7)
    check_attn(Cache(7, [8300, 40], 8, 64), [8250, 1], 32, window=700, n_sink=40, each=7)


def test_page_attn_scores_far_apart():
    """Scores over a few hundred log2 units: the softmax reference moves many times per row; and one key far above many others."""
    c = Cache(4, [900, 333], 2, 16)
    q = (randn(gen_of(8), 301, 8, D).float() * 12).half()
    check_attn(c, [300, 1], 8, q=q)
    c = Cache(6, [9000], 2, 64)
    q = randn(gen_of(9), 1, 8, D)
    for g in range(2):
        c.k[0][g] *= 0.01
        c.k[0][g, 4000] = (q[0, 4 * g:4 * g + 4].sum(0) * 0.55).half()
    c.fill()
    check_attn(c, [1], 8, q=q)


def test_page_attn_strided_queries():
    c = Cache(4, [200, 100], 2, 16)
    x = randn(gen_of(3), 31, 12, D)
    check_attn(c, [30, 1], 8, q=x[:, :8])
    check_attn(c, [30, 1], 8, q=randn(gen_of(3), 8, 31, D).transpose(0, 1))


@pytest.mark.parametrize("window,n_sink", [(0, 0), (50, 10)])
def test_page_attn_hidden_values_take_no_part(window, n_sink):
    """Infinities and NaN in K and V: rows that see them get what the formula gives, the others nothing of them."""
    c = Cache(4, [150, 90, 400], 2, 16)
    inf, nan = float("inf"), float("nan")
    c.v[0][:, 100, 3], c.v[0][:, 100, 77], c.v[0][:, 101, 3] = inf, nan, -inf
    c.v[0][0, 60, 9], c.v[0][1, 12, 9] = -inf, inf                 # just outside the sinks, and outside a window
    c.k[1][:, 89] = nan                                            # seen by the last row only
    c.v[1][:, 88] = nan
    c.v[2][:, 300:310] = inf
    c.fill()
    q = randn(gen_of(5), 90 + 150 + 200, 8, D)
    new = [150, 90, 200]
    starts = [0, 150, 240, 440]
    geom = antkv.Geometry(3, 8, 2, 8)
    out, top, total = antkv.page_attn(geom, q, SCALE, ints(starts), ints(c.ctx), c.table, c.k_pages, c.v_pages, window=window, n_sink=n_sink, want_stats=True)
    for r, n in enumerate(new):
        a, b = starts[r], starts[r + 1] - (r == 1)                  # (the row that sees a NaN key is looked at below)
        for h in range(8):
            pos = torch.arange(c.ctx[r] - n, c.ctx[r] - (r == 1), device="cuda")
            compare((out[a:b, h], top[h, a:b], total[h, a:b]), exact(q[a:b, h], c.k[r][h // 4], c.v[r][h // 4], pos, window, n_sink), f"request {r}, head {h}")
    assert out[239].isnan().all() and total[:, 239].isnan().all()


def test_page_attn_pages_that_are_none():
    """Keys of such pages, and behind the table's end, are not seen; a row that sees nothing is zero."""
    page, ctx, new = 16, [200, 64, 90, 50], [40, 64, 90, 1]
    c = Cache(4, ctx, 2, page)
    c.table[0, 3], c.table[0, 12] = -1, c.n_pages                   # positions 48 .. 63 and 192 .. 207
    c.table[1, 0] = 1 << 30                                         # rows 0 .. 15 of the second request see nothing
    c.table[2, :] = -1
    hidden = [torch.zeros(n, dtype=torch.bool, device="cuda") for n in ctx]
    hidden[0][48:64], hidden[0][192:], hidden[1][:16], hidden[2][:] = True, True, True, True
    out = check_attn(c, new, 8, hidden=hidden)
    assert (out[40:56] == 0).all() and (out[104:194] == 0).all()
    for p in (32, 64):
        c = Cache(4, [200, 300], 2, p)
        c.table[0, 1], c.table[1, 0] = -7, c.n_pages + 5
        hidden = [torch.zeros(n, dtype=torch.bool, device="cuda") for n in (200, 300)]
        hidden[0][p:2 * p], hidden[1][:p] = True, True
        check_attn(c, [100, 300], 8, hidden=hidden, window=150, n_sink=70)


def test_page_attn_lengths_beyond_the_table():
    """A context longer than the table's row holds, one shorter than its rows, and none at all."""
    c = Cache(4, [96, 20, 30], 2, 16, extra=0)                      # 6 entries a row
    k = [torch.cat([x, torch.zeros(2, 30, D, dtype=torch.float16, device="cuda")], dim=1) for x in c.k]
    v = [torch.cat([x, torch.zeros(2, 30, D, dtype=torch.float16, device="cuda")], dim=1) for x in c.v]
    q, new, ctx = randn(gen_of(2), 60, 8, D), [20, 30, 10], [110, 20, 0]
    starts = [0, 20, 50, 60]
    out, top, total = antkv.page_attn(antkv.Geometry(3, 8, 2, 8), q, SCALE, ints(starts), ints(ctx), c.table, c.k_pages, c.v_pages, want_stats=True)
    for r in range(3):
        a, b = starts[r], starts[r + 1]
        pos = torch.arange(ctx[r] - new[r], ctx[r], device="cuda")  # negative ones see nothing
        hidden = torch.arange(k[r].shape[1], device="cuda") >= min(ctx[r], 96)
        for h in range(8):
            compare((out[a:b, h], top[h, a:b], total[h, a:b]), exact(q[a:b, h], k[r][h // 4], v[r][h // 4], pos, 0, 0, hidden=hidden), f"{r} {h}")


def test_page_attn_same_bits_whatever_the_workspace_held():
    c = Cache(4, [9000, 700, 1], 2, 64)
    first = check_attn(c, [1, 100, 1], 8)
    for fill in (0, 1, 255):
        ws = antkv.page_attn_workspace(antkv.Geometry(3, 8, 2, 8), 102, "cuda").fill_(fill)
        again = check_attn(c, [1, 100, 1], 8, workspace=ws)
        assert torch.equal(first.view(torch.int16), again.view(torch.int16))


def test_page_attn_on_two_streams():
    caches = [Cache(s, [3000 + s, 50], 2, 16) for s in (0, 1)]
    qs = [randn(gen_of(s), 33, 8, D) for s in (0, 1)]
    geom, starts = antkv.Geometry(2, 8, 2, 8), ints([0, 1, 33])
    args = [(geom, q, SCALE, starts, ints(c.ctx), c.table, c.k_pages, c.v_pages) for c, q in zip(caches, qs)]
    want = [antkv.page_attn(*a)[0] for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(antkv.page_attn(*args[i])[0])
    torch.cuda.synchronize()
    assert all(torch.equal(x.view(torch.int16), want[i].view(torch.int16)) for i in range(2) for x in got[i])


def test_pools_of_more_than_32_bits():
    """Pages whose bytes, and whose elements, lie beyond 2^32: stored, loaded and read as those of a small pool."""
    Hkv, page, n_pages = 8, 256, 18000                              # 4.7e9 elements to a pool
    kp, vp = (torch.empty((n_pages, Hkv, page, D), dtype=torch.float16, device="cuda") for _ in "kv")
    assert kp.numel() > 1 << 32
    ctx, new, gen = [700, 300], [1, 300], gen_of(21)
    c = Cache(21, ctx, Hkv, page, extra=0)
    table = ints([[17999, 9000, 17], [4096, 16500, 8192]])
    geom, T = antkv.Geometry(2, 4 * Hkv, Hkv, 8), sum(ctx)
    k, v = (torch.cat(x, dim=1).transpose(0, 1).contiguous() for x in (c.k, c.v))
    pos = np.concatenate([np.arange(n) for n in ctx])
    pages = np.concatenate([table[r].cpu().numpy()[np.arange(n) // page] for r, n in enumerate(ctx)])
    antkv.page_store(geom, k, v, ints(pages * page + pos % page), kp, vp)
    got_k, got_v = antkv.page_load(geom, kp, vp, table, 700, ctx_len=ints(ctx))
    for r, n in enumerate(ctx):
        assert torch.equal(got_k[r, :, :n], c.k[r]) and torch.equal(got_v[r, :, :n], c.v[r])
    q, starts = randn(gen, sum(new), 4 * Hkv, D), ints([0, 1, 301])
    small = antkv.page_attn(geom, q, SCALE, starts, ints(ctx), c.table, c.k_pages, c.v_pages)[0]
    assert torch.equal(antkv.page_attn(geom, q, SCALE, starts, ints(ctx), table, kp, vp)[0].view(torch.int16), small.view(torch.int16))


@pytest.mark.parametrize("window,n_sink", [(0, 0), (17000, 40)])
def test_page_attn_hidden_values_far_apart(window, n_sink):
    """Values that are not finite, in edge tiles of the first and of later turns of the loop over keys: rows that see them, rows that do not."""
    c = Cache(31, [34000], 1, 32)
    rows = 200                                                      # positions 33800 .. 33999
    for at, x in ((3, "inf"), (39, "nan"), (33850, "-inf"), (33999, "nan")):
        c.v[0][0, at, at % D] = float(x)
    if window:
        c.v[0][0, 16900, 7] = float("inf")                          # behind the left edge of some rows
    c.fill()
    check_attn(c, [rows], 2, window, n_sink)


def test_page_attn_starts_that_do_not_ascend():
    """Row numbers that are no request's rows are never followed: what lies between proper starts is right."""
    c = Cache(41, [100, 60, 90], 2, 16)
    q, geom = randn(gen_of(41), 20, 8, D), antkv.Geometry(3, 8, 2, 8)
    want = antkv.page_attn(geom, q, SCALE, ints([0, 5, 5, 5]), ints(c.ctx), c.table, c.k_pages, c.v_pages)[0]
    for starts in ([0, 5, 3, 3], [0, 5, 900, 10 ** 9], [0, 5, -7, -9]):
        got = antkv.page_attn(geom, q, SCALE, ints(starts), ints(c.ctx), c.table, c.k_pages, c.v_pages)[0]
        assert torch.equal(got[:3].view(torch.int16), want[:3].view(torch.int16)), starts


def test_page_attn_requests_that_overlap_write_nothing():
    c, R = Cache(42, [50] * 100, 2, 16), 100
    q, out = randn(gen_of(42), 30, 8, D), torch.full((30, 8, D), 7.0, dtype=torch.float16, device="cuda")
    for r in (100, 60):
        antkv.page_attn(antkv.Geometry(r, 8, 2, 8), q, SCALE, ints([0, 30] * (r // 2) + [0]), ints(c.ctx[:r]), c.table[:r], c.k_pages, c.v_pages, out=out)
        assert (out == 7.0).all()


def test_page_attn_long_prompts():
    """Blocks enough for a workgroup each: prompts of one length, and one beside a short one, in a window and without."""
    for window, n_sink in ((0, 0), (300, 40)):
        check_attn(Cache(51, [4100, 4097], 8, 32), [4100, 4093], 32, window, n_sink, pad=5, each=11)
        check_attn(Cache(52, [9000, 30], 8, 64), [8800, 2], 32, window, n_sink, each=11)


@pytest.mark.parametrize("window,n_sink", [(0, 0), (90, 40)])
@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (4, 2), (3, 3)])
def test_page_attn_a_token_each_on_average(Hq, Hkv, window, n_sink):
    """No more rows than requests, but uneven ones: some have many blocks of 32 rows, some none."""
    ctx = [600, 1, 70, 2000, 33, 64] + [5] * 94
    check_attn(Cache(61, ctx, Hkv, 32), [40, 1, 0, 33, 17, 0] + [0] * 90 + [5, 0, 1, 1], Hq, window, n_sink, pad=2)
    check_attn(Cache(62, [3000] + [9] * 129, Hkv, 16), [130] + [0] * 129, Hq, window, n_sink)


def test_page_attn_as_many_requests_as_there_may_be():
    """8192 requests, most of a token or none, in 128 looks at their lengths."""
    rng = np.random.default_rng(71)
    ctx = rng.integers(1, 60, 8192).tolist()
    new = [0 if r % 5 == 0 else min(c, 1 + 30 * (r % 97 == 0)) for r, c in enumerate(ctx)]
    ctx[8000], new[8000] = 5000, 70
    c = Cache(71, ctx, 1, 16)
    starts = np.concatenate([[0], np.cumsum(new)])
    q, geom = randn(gen_of(71), int(starts[-1]), 2, D), antkv.Geometry(8192, 2, 1, 8)
    out, top, total = antkv.page_attn(geom, q, SCALE, ints(starts), ints(ctx), c.table, c.k_pages, c.v_pages, want_stats=True)
    assert out.isfinite().all()
    for r in [*range(0, 8192, 97), 8000, 8191]:
        a, b = int(starts[r]), int(starts[r + 1])
        pos = torch.arange(ctx[r] - new[r], ctx[r], device="cuda")
        for h in range(2 if new[r] else 0):
            compare((out[a:b, h], top[h, a:b], total[h, a:b]), exact(q[a:b, h], c.k[r][0], c.v[r][0], pos, 0, 0), f"request {r}, head {h}")


def test_page_attn_requests_that_share_pages():
    """The same pages in the tables of three requests, as a common beginning."""
    c = Cache(72, [100, 64, 80], 2, 16)
    for r in (1, 2):
        c.table[r, :4] = c.table[0, :4]
        c.k[r][:, :64], c.v[r][:, :64] = c.k[0][:, :64], c.v[0][:, :64]
    check_attn(c, [1, 20, 10], 8)


def test_page_attn_tables_of_great_capacity():
    """Tables for so many tokens that a batch might cost more than the shares can count."""
    c = Cache(53, [3000, 1, 700] + [20] * 37, 2, 256)
    table = torch.full((40, 1 << 22), -1, dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = c.table
    c.table = table
    check_attn(c, [1, 1, 90] + [1] * 37, 8)


def test_a_step_on_another_stream():
    """Map, store, attention, load and a windowed prompt on a stream of their own, each reading what the one before has written."""
    Hq, Hkv, page, n_pages, n = 8, 2, 16, 40, 500
    gen, geom, one = gen_of(51), antkv.Geometry(1, Hq, Hkv, 8), ints([n])
    k, v, q = randn(gen, n, Hkv, D), randn(gen, n, Hkv, D), randn(gen, n, Hq, D)
    free = torch.randperm(n_pages, device="cuda", generator=gen).to(torch.int32)

    def step():
        kp, vp = (torch.zeros((n_pages, Hkv, page, D), dtype=torch.float16, device="cuda") for _ in "kv")
        table = torch.full((1, n_pages), -1, dtype=torch.int32, device="cuda")
        ctx, starts, slot, _ = antkv.page_map(ints([0]), one, table, page, n_pages, free, n)
        antkv.page_store(geom, k, v, slot, kp, vp)
        out = antkv.page_attn(geom, q, SCALE, starts, ctx, table, kp, vp, window=90, n_sink=3)[0]
        dk, dv = antkv.page_load(geom, kp, vp, table, n)
        dense = antkv.prefill_attn_window(geom, q.transpose(0, 1)[None].contiguous(), dk, dv, SCALE, 90, 3, want_stats=False)[0]
        return out, dk, dv, dense

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(3):
            got = step()
    side.synchronize()
    assert all(torch.equal(g.view(torch.int16), w.view(torch.int16)) for g, w in zip(got, want))
    a, b = want[0].transpose(0, 1).double(), want[3][0].double()
    assert ((a - b).norm(dim=-1) <= 2 * OUT_TOL * b.norm(dim=-1)).all()


# ------------------------------------------------------------------------------------------------ windowed prompts

@pytest.mark.parametrize("window,n_sink", [(1, 0), (1, 1), (7, 4), (32, 0), (33, 32), (128, 70), (10 ** 9, 10 ** 9)])
@pytest.mark.parametrize("B,Hq,Hkv,N,Nq", [(1, 8, 2, 1, 1), (2, 4, 4, 33, 33), (1, 4, 2, 257, 100), (1, 8, 2, 700, 700), (3, 2, 2, 95, 95), (1, 7, 7, 130, 1),
                                           (48, 8, 8, 70, 70)])
def test_prefill_attn_window(B, Hq, Hkv, N, Nq, window, n_sink):
    gen = gen_of(N)
    q, k, v = randn(gen, B, Hq, Nq, D), randn(gen, B, Hkv, N, D), randn(gen, B, Hkv, N, D)
    out, top, total = antkv.prefill_attn_window(antkv.Geometry(B, Hq, Hkv, 8), q, k, v, SCALE, window, n_sink)
    pos, G = torch.arange(N - Nq, N, device="cuda"), Hq // Hkv
    for b in range(B):
        for h in range(Hq):
            compare((out[b, h], top[b, h], total[b, h]), exact(q[b, h], k[b, h // G], v[b, h // G], pos, min(window, N), n_sink), f"{b} {h}")
    assert torch.equal(out, antkv.prefill_attn_window(antkv.Geometry(B, Hq, Hkv, 8), q, k, v, SCALE, window, n_sink, want_stats=False)[0])


@pytest.mark.parametrize("Hq,Hkv,N,Nq,window,n_sink", [(4, 1, 33000, 40, 32990, 3), (32, 8, 3001, 3001, 600, 4), (16, 16, 2000, 2000, 300, 1)])
def test_prefill_attn_window_long(Hq, Hkv, N, Nq, window, n_sink):
    gen = gen_of(N)
    q, k, v = randn(gen, 1, Hq, Nq, D), randn(gen, 1, Hkv, N, D), randn(gen, 1, Hkv, N, D)
    out, top, total = antkv.prefill_attn_window(antkv.Geometry(1, Hq, Hkv, 8), q, k, v, SCALE, window, n_sink)
    pos, G = torch.arange(N - Nq, N, device="cuda"), Hq // Hkv
    for h in range(0, Hq, 3):
        compare((out[0, h], top[0, h], total[0, h]), exact(q[0, h], k[0, h // G], v[0, h // G], pos, window, n_sink), f"head {h}")


def test_prefill_attn_window_hidden_values_take_no_part():
    gen, N = gen_of(1), 300
    q, k, v = randn(gen, 1, 4, N, D), randn(gen, 1, 2, N, D), randn(gen, 1, 2, N, D)
    v[0, 0, 200, 5], v[0, 0, 100, 6], v[0, 1, 299], v[0, 1, 3, 8] = float("inf"), float("nan"), -float("inf"), float("nan")
    out, top, total = antkv.prefill_attn_window(antkv.Geometry(1, 4, 2, 8), q, k, v, SCALE, 20, 4)
    for h in range(4):
        compare((out[0, h], top[0, h], total[0, h]), exact(q[0, h], k[0, h // 2], v[0, h // 2], torch.arange(N, device="cuda"), 20, 4), f"head {h}")


def test_prefill_attn_window_of_everything_is_prefill_attn():
    gen = gen_of(2)
    q, k, v = randn(gen, 2, 8, 300, D), randn(gen, 2, 2, 500, D), randn(gen, 2, 2, 500, D)
    geom = antkv.Geometry(2, 8, 2, 8)
    a, b = antkv.prefill_attn_window(geom, q, k, v, SCALE, 500), antkv.prefill_attn(geom, q, k, v, SCALE)
    assert ((a[0].double() - b[0].double()).norm(dim=-1) <= 2 * OUT_TOL * b[0].double().norm(dim=-1)).all()
    assert (a[1] - b[1]).abs().max() <= 2e-5 and (a[2] / b[2] - 1).abs().max() <= 2e-4


# ------------------------------------------------------------------------------------------------ together

def test_prompts_in_chunks_until_they_are_codes():
    """Two prompts through pages in uneven chunks beside a request that decodes; then, dense, through selection and encoding to a
    decode step over codes: the same as from the dense prompt."""
    Hq, Hkv, page, n_pages, d = 8, 2, 16, 64, 8
    gen, lens, chunks = gen_of(11), [333, 200, 60], [[100, 64, 1], [1, 136, 1], [232, 0, 1], [0, 0, 1]]
    K, V, Q = ([randn(gen, h, n + 4, D) for n in lens] for h in (Hkv, Hkv, Hq))
    geom = antkv.Geometry(3, Hq, Hkv, d)
    kp, vp = (torch.full((n_pages, Hkv, page, D), float("nan"), dtype=torch.float16, device="cuda") for _ in "kv")
    table, free = torch.full((3, 24), -1, dtype=torch.int32, device="cuda"), torch.randperm(n_pages, device="cuda", generator=gen).to(torch.int32)
    done, at = [0, 0, 0], None
    outs, stats = [[], [], []], [[], [], []]
    steps = [[0, 0, 56]] + chunks                                   # the third request's prompt first
    held = ints(done)
    for new in steps:
        T = sum(new) + 2                                            # (a padded batch)
        rows = lambda X: torch.cat([X[r][:, done[r]:done[r] + n] for r, n in enumerate(new)] + [X[0][:, :2]], dim=1).transpose(0, 1).contiguous()
        held, q_start, slot, at = antkv.page_map(held, ints(new), table, page, n_pages, free, T, free_at=at)
        antkv.page_store(geom, rows(K), rows(V), slot, kp, vp)
        out, top, total = antkv.page_attn(geom, rows(Q), SCALE, q_start, held, table, kp, vp, want_stats=True)
        assert at.tolist()[1] == 0
        a = 0
        for r, n in enumerate(new):
            outs[r].append(out[a:a + n])
            stats[r].append((top[:, a:a + n], total[:, a:a + n]))
            a += n
            done[r] += n
    assert held.tolist() == done == [333, 200, 60]
    for r in range(2):
        n = done[r]
        one = antkv.Geometry(1, Hq, Hkv, d)
        q, k, v = (X[r][None, :, :n].contiguous() for X in (Q, K, V))
        want, w_top, w_total = antkv.prefill_attn(one, q, k, v, SCALE)
        got = torch.cat(outs[r]).transpose(0, 1)
        assert ((got.double() - want[0].double()).norm(dim=-1) <= 2 * OUT_TOL * want[0].double().norm(dim=-1)).all()
        k2, v2 = antkv.page_load(one, kp, vp, table[r:r + 1], n)
        assert torch.equal(k2, k) and torch.equal(v2, v)
        top, total = (torch.cat([s[i] for s in stats[r]], dim=1)[None].contiguous() for i in range(2))
        idx_k, idx_v, ans_k, ans_v = antkv.anchor_select(one, q, k2, SCALE, 4, row_max=top, row_sum=total)
        _, _, w_k, w_v = antkv.anchor_select(one, q, k, SCALE, 4, row_max=w_top, row_sum=w_total)
        assert (ans_k / w_k - 1).abs().max() <= 1e-3 and (ans_v / w_v - 1).abs().max() <= 1e-3
        cb = randn(gen, Hkv, D // d, 256, d)
        codes_k, codes_v = antkv.encode(one, k2, cb), antkv.encode(one, v2, cb)
        assert torch.equal(codes_k, antkv.encode(one, k, cb)) and torch.equal(codes_v, antkv.encode(one, v, cb))
        rows_k, rows_v = antkv.gather_rows(one, k2, idx_k), antkv.gather_rows(one, v2, idx_v)
        step = antkv.decode_attn(one, q[:, :, -1].contiguous(), SCALE, codes_k, codes_v, cb, cb, idx_k, rows_k, idx_v, rows_v)
        assert step.isfinite().all()


def test_captured_step_replayed_with_other_lengths():
    """A decode step (map, store, attention) captured once and replayed over growing contexts, eager steps between: each replay against
    the same step called eagerly on copies.  Twice in two graphs that share a workspace."""
    Hq, Hkv, page, n_pages, R = 8, 2, 16, 400, 4
    gen, geom = gen_of(12), antkv.Geometry(R, Hq, Hkv, 8)
    ctx = [1, 15, 900, 3000]
    pools = randn(gen, n_pages, Hkv, page, D), randn(gen, n_pages, Hkv, page, D)
    counts = [-(-c // page) for c in ctx]
    order = torch.randperm(n_pages, device="cuda", generator=gen).to(torch.int32)
    table = torch.full((R, 200), -1, dtype=torch.int32, device="cuda")
    for r in range(R):
        table[r, :counts[r]] = order[sum(counts[:r]):sum(counts[:r + 1])]
    free, at = order[sum(counts):].contiguous(), ints([0, 0])
    held, new = ints(ctx), ints([1] * R)
    q, k, v = randn(gen, R, Hq, D), randn(gen, R, Hkv, D), randn(gen, R, Hkv, D)
    ws = antkv.page_attn_workspace(geom, R, "cuda")
    out = torch.empty((R, Hq, D), dtype=torch.float16, device="cuda")

    def step(held, at, table, kp, vp, out, ws):
        lens, q_start, slot, status = antkv.page_map(held, new, table, page, n_pages, free, R, free_at=at)
        antkv.page_store(geom, k, v, slot, kp, vp)
        antkv.page_attn(geom, q, SCALE, q_start, lens, table, kp, vp, out=out, workspace=ws)
        return lens, status

    step(held.clone(), at.clone(), table.clone(), pools[0].clone(), pools[1].clone(), out.clone(), ws)     # (loads the library)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            res = step(held, at, table, *pools, out, ws)
            held.copy_(res[0])
            at.copy_(res[1])
        graphs.append(graph)
    for i in range(8):
        for x in (q, k, v):
            x.normal_()
        new.copy_(ints([1, 1, 0 if i == 5 else 1, 1]))
        eager = [t.clone() for t in (held, at, table, *pools, out)]
        want = step(*eager, antkv.page_attn_workspace(geom, R, "cuda"))
        graphs[i & 1].replay()
        torch.cuda.synchronize()
        rows = int(new.sum())
        assert torch.equal(held, want[0]) and torch.equal(at, want[1]) and torch.equal(table, eager[2])
        assert torch.equal(pools[0], eager[3]) and torch.equal(pools[1], eager[4])
        assert torch.equal(out[:rows].view(torch.int16), eager[5][:rows].view(torch.int16)), f"replay {i}"
        assert out[:rows].isfinite().all()


# ------------------------------------------------------------------------------------------------ visible infinities

def one_way(gen, k, top, gain, rows, Hq):
    """Queries all of about one direction, and keys k [Hkv, C, D] of which number `top` scores 16.3 gain log2 units more than the others."""
    base = torch.where(torch.rand(D, device="cuda", generator=gen) < 0.5, 1.0, -1.0)
    k.copy_((0.05 * k.float()).half())
    if gain:
        k[:, top] = (gain * base).half()
    return (base + 0.1 * randn(gen, rows, Hq, D).float()).half()


def spread_odd(v, keys):
    """inf, -inf and NaN at the given keys of v [Hkv, C, D], each in a channel of its own, and one channel with inf and -inf."""
    for i, key in enumerate(keys):
        v[:, key, 7 * i + 1] = (float("inf"), -float("inf"), float("nan"))[i % 3]
    v[:, keys[0], 127], v[:, keys[-1], 127] = float("inf"), -float("inf")


@pytest.mark.parametrize("Hq,Hkv,ctx", [(8, 2, 5000), (1, 1, 1300), (4, 1, 20000)])
def test_page_attn_infinities_in_pieces_of_a_row(Hq, Hkv, ctx):
    """One token whose keys are cut into pieces, no multiple of 16 of them: an infinity in the last one, which is read again in place of those missing."""
    c = Cache(81, [ctx], Hkv, 16)
    spread_odd(c.v[0], [ctx - 40, ctx - 70, ctx - 100])
    c.fill()
    check_attn(c, [1], Hq)


@pytest.mark.parametrize("top", [5, 170])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (150, 70)])
@pytest.mark.parametrize("ctx,new", [([300], [1]), ([300], [300]), ([290, 300], [60, 1])])
def test_page_attn_infinities_of_little_weight(ctx, new, window, n_sink, top):
    """A value that a row sees is in its result whatever its weight: 65 log2 units below the largest (nothing, in fp16), in a tile that all
    rows see and in one that some do."""
    c = Cache(82, ctx, 2, 16)
    q = torch.cat([one_way(gen_of(82 + r), c.k[r], top, 4, n, 8) for r, n in enumerate(new)])
    for v in c.v:
        spread_odd(v, [3, 40, 100, 150, 171, 220, 280])
    c.fill()
    check_attn(c, new, 8, window, n_sink, q=q)


@pytest.mark.parametrize("gain", [4, 24])
@pytest.mark.parametrize("N,Nq,window,n_sink,top", [(500, 500, 300, 40, 20), (500, 500, 500, 0, 400), (33000, 40, 32990, 33, 17000), (33000, 40, 32990, 33, 20)])
def test_prefill_attn_window_infinities_of_little_weight(N, Nq, window, n_sink, top, gain):
    """The same over a dense prompt, up to 391 log2 units (nothing, in fp32), and over more key tiles than are looked up at a time: the softmax
    reference moves that far after, or long before, the value is seen."""
    gen = gen_of(83)
    k, v = randn(gen, 2, N, D), randn(gen, 2, N, D)
    q = one_way(gen, k, top, gain, Nq, 4)
    spread_odd(v, [2, 50, N // 2 - 10, N // 2 + 300 if N > 1000 else 260, N - 100, N - 64, N - 5])
    q = q.transpose(0, 1).contiguous()
    out, row_max, row_sum = antkv.prefill_attn_window(antkv.Geometry(1, 4, 2, 8), q[None], k[None], v[None], SCALE, window, n_sink)
    for h in range(4):
        compare((out[0, h], row_max[0, h], row_sum[0, h]), exact(q[h], k[h // 2], v[h // 2], torch.arange(N - Nq, N, device="cuda"), window, n_sink), f"head {h}")


@pytest.mark.parametrize("gain", [0, 4, 24])
@pytest.mark.parametrize("ctx,new,top", [([300], [1], 5), ([300], [1], 170), ([6000], [1], 10), ([6000], [1], 4000), ([9000], [100], 30), ([9000], [100], 5000),
                                         ([4000, 5000], [1, 200], 3000)])
def test_page_attn_infinities_where_sums_meet(ctx, new, top, gain):
    """Sums of waves and of pieces whose weights beside the others are nothing in fp32 (391 log2 units) hold infinities: they stay."""
    c = Cache(84, ctx, 2, 16)
    q = torch.cat([one_way(gen_of(84 + r), c.k[r], top, gain, n, 8) for r, n in enumerate(new)])
    for r, v in enumerate(c.v):
        n = ctx[r]
        spread_odd(v, [3, 45, n // 3, n // 2, n - 250, n - 100, n - 6])
    c.fill()
    check_attn(c, new, 8, q=q)


@pytest.mark.parametrize("gain", [0, 4, 24])
def test_page_attn_infinities_in_turns_of_a_row(gain):
    """A token on more key tiles than a workgroup looks up at a time, all of them its own (a table of great capacity)."""
    c = Cache(85, [40000] + [20] * 39, 1, 256)
    q = torch.cat([one_way(gen_of(85), c.k[0], 36000, gain, 1, 4), randn(gen_of(86), 39, 4, D)])
    spread_odd(c.v[0], [3, 20000, 32700, 33000, 36001, 39990])
    c.fill()
    table = torch.full((40, 1 << 22), -1, dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = c.table
    c.table = table
    check_attn(c, [1] * 40, 4, q=q)


# ------------------------------------------------------------------------------------------------ many requests of many heads

def test_as_many_requests_as_there_may_be_of_eight_heads():
    """8192 requests on 8 KV heads, more than 65535 pairs of them: attention, and their rows out of the pages."""
    rng = np.random.default_rng(91)
    R, Hkv, page = 8192, 8, 16
    ctx = rng.integers(1, 40, R).tolist()
    new = [0 if r % 5 == 0 else min(c, 1 + 30 * (r % 97 == 0)) for r, c in enumerate(ctx)]
    c = Cache(91, ctx, Hkv, page, extra=0)
    starts = np.concatenate([[0], np.cumsum(new)])
    q, geom = randn(gen_of(91), int(starts[-1]), 2 * Hkv, D), antkv.Geometry(R, 2 * Hkv, Hkv, 8)
    out, top, total = antkv.page_attn(geom, q, SCALE, ints(starts), ints(ctx), c.table, c.k_pages, c.v_pages, want_stats=True)
    k, v = antkv.page_load(geom, c.k_pages, c.v_pages, c.table, 39, ctx_len=ints(ctx))
    assert out.isfinite().all()
    for r in [*range(0, R, 97), R - 2, R - 1]:
        a, b = int(starts[r]), int(starts[r + 1])
        pos = torch.arange(ctx[r] - new[r], ctx[r], device="cuda")
        for h in range(r % 3, 2 * Hkv if new[r] else 0, 3):
            compare((out[a:b, h], top[h, a:b], total[h, a:b]), exact(q[a:b, h], c.k[r][h // 2], c.v[r][h // 2], pos, 0, 0), f"request {r}, head {h}")
        assert torch.equal(k[r, :, :ctx[r]], c.k[r]) and torch.equal(v[r, :, :ctx[r]], c.v[r])
        assert (k[r, :, ctx[r]:] == 0).all() and (v[r, :, ctx[r]:] == 0).all()


def test_page_store_of_the_largest_batch():
    """As many rows as a grid has, all of them the same one and nearly all without a slot."""
    T, Hkv = (1 << 23) - 1, 64
    gen = gen_of(92)
    k, v = (randn(gen, 1, Hkv, D).expand(T, Hkv, D) for _ in "kv")
    kp, vp = (torch.zeros((4, Hkv, 16, D), dtype=torch.float16, device="cuda") for _ in "kv")
    slot = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    slot[0], slot[T // 2], slot[-1] = 5, 63, 30
    antkv.page_store(antkv.Geometry(1, Hkv, Hkv, 8), k, v, slot, kp, vp)
    for x, pages in ((k, kp), (v, vp)):
        want = torch.zeros_like(pages)
        for s in (5, 63, 30):
            want[s // 16, :, s % 16] = x[0]
        assert torch.equal(pages, want)


# ------------------------------------------------------------------------------------------------ replays over other pieces

@pytest.mark.parametrize("most", [1, 100])
def test_captured_step_replayed_over_other_numbers_of_pieces(most):
    """A step captured in two graphs that share a workspace, replayed over contexts whose lengths change places and size: a share's arrival
    word meets blocks of 9, 3, 8 and one piece (tokens of their own: contexts of 3000 and 900 end in share 15, or 12, by turns), of single
    tokens, and with a chunk of 100 among them."""
    Hq, Hkv, page, R, own = 8, 2, 16, 4, 200
    T = R - 1 + most
    gen, geom = gen_of(93), antkv.Geometry(R, Hq, Hkv, 8)
    n_pages = R * own + 40
    pools = [randn(gen, n_pages, Hkv, page, D) for _ in "kv"]
    order = torch.randperm(n_pages, device="cuda", generator=gen).to(torch.int32)
    whole, free = order[:R * own].view(R, own), order[R * own:].contiguous()
    table, held, new = whole.clone(), ints([0] * R), ints([1] * R)
    q, k, v = randn(gen, T, Hq, D), randn(gen, T, Hkv, D), randn(gen, T, Hkv, D)
    ws = antkv.page_attn_workspace(geom, T, "cuda")
    out = torch.empty((T, Hq, D), dtype=torch.float16, device="cuda")

    def step(table, kp, vp, out, ws):
        lens, q_start, slot, _ = antkv.page_map(held, new, table, page, n_pages, free, T)
        antkv.page_store(geom, k, v, slot, kp, vp)
        antkv.page_attn(geom, q, SCALE, q_start, lens, table, kp, vp, out=out, workspace=ws)

    step(table, *pools, out, ws)                                    # (loads the library)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(table, *pools, out, ws)
        graphs.append(graph)
    lengths = [[3000, 900, 40, 5], [5, 40, 900, 3000], [40, 3000, 5, 900], [900, 5, 3000, 40], [20, 30, 5, 40], [700, 5, 40, 2900], [2900, 40, 5, 700],
               [3000, 5, 40, 900], [1, 15, 60, 3000]]
    for i in range(2 * len(lengths)):                               # (an odd number of them: each goes to both graphs)
        ctx = lengths[i % len(lengths)]
        fresh = [1] * R
        fresh[int(np.argmax(ctx)) if i % 3 else int(np.argsort(ctx)[-2])] = most
        held.copy_(ints([max(c - n, 0) for c, n in zip(ctx, fresh)]))
        new.copy_(ints(fresh))
        table.copy_(whole)
        for x in (q, k, v):
            x.normal_()
        eager = [t.clone() for t in (table, *pools, out)]
        step(*eager, antkv.page_attn_workspace(geom, T, "cuda"))
        graphs[i & 1].replay()
        torch.cuda.synchronize()
        for got, want in zip((table, *pools, out), eager):
            assert torch.equal(got.view(torch.int16), want.view(torch.int16)), f"replay {i}"
        assert out.isfinite().all()
    cache = [p.clone() for p in pools]                              # the last step against 64 bits
    ctx, starts = [max(c, n) for c, n in zip(ctx, fresh)], np.concatenate([[0], np.cumsum(fresh)])
    for r in range(R):
        j = torch.arange(ctx[r], device="cuda")
        kr, vr = (p[table[r].long()[j // page], :, j % page].transpose(0, 1) for p in cache)
        a, b = int(starts[r]), int(starts[r + 1])
        for h in range(Hq):
            want = exact(q[a:b, h], kr[h // 4], vr[h // 4], j[ctx[r] - fresh[r]:], 0, 0)[0]
            assert ((out[a:b, h].double() - want).norm(dim=-1) <= OUT_TOL * want.norm(dim=-1)).all(), (r, h)


# ------------------------------------------------------------------------------------------------ large scores

@pytest.mark.parametrize("ctx,new", [([900], [1]), ([900], [300])])
def test_scores_of_great_size(ctx, new):
    """Scores of 4.5e7, at which log2 units come in steps of four: equal ones share the row, one above the others has it."""
    gen, n = gen_of(94), new[0]
    base = torch.where(torch.rand(D, device="cuda", generator=gen) < 0.5, 1.0, -1.0)
    for tops in (range(900), [500], [3, 899], [40]):
        c = Cache(94, ctx, 2, 16)
        c.k[0].mul_(0.01)
        c.k[0][:, list(tops)] = (2000 * base).half()
        c.fill()
        q = (2000 * base).half().expand(n, 8, D)
        check_attn(c, new, 8, q=q)
        dense = antkv.prefill_attn_window(antkv.Geometry(1, 8, 2, 8), q.transpose(0, 1)[None].contiguous(), c.k[0][None].contiguous(), c.v[0][None].contiguous(), SCALE, 700, 30)
        pos = torch.arange(900 - n, 900, device="cuda")
        for h in range(8):
            compare([x[0, h] for x in dense], exact(q[:, h], c.k[0][h // 4], c.v[0][h // 4], pos, 700, 30), f"{tops} {h}")
