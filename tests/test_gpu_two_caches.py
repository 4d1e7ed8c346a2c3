"""GPU checks of both caches side by side: one workspace for the attention over either, called and captured in turn, and rows captured on their way out."""
import numpy as np
import pytest
import torch

import paper_2506_19505_amd as antkv
import test_gpu_pages as halves
import test_gpu_qpages as eights
from test_gpu_pages import D, SCALE, gen_of, ints, randn

pytestmark = pytest.mark.gpu

HQ, HKV = 8, 2


def bits(t):
    return t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


@pytest.mark.parametrize("ctx,new", [([9000, 700, 1], [1, 100, 1]), ([9000, 40], [1, 1]), ([5000], [300])])
def test_one_workspace_for_both_caches(ctx, new):
    """What one cache's launches leave in the workspace (arrival words, partial sums) lies under the other's words: eager calls in turn, then two captured
    ones that are replayed in turn, all with the bits of calls that have a workspace of their own."""
    geom, T = antkv.Geometry(len(ctx), HQ, HKV, 8), sum(new)
    a, b = halves.Cache(111, ctx, HKV, 16), eights.ByteCache(112, ctx, HKV, 16)
    q, starts, lens = randn(gen_of(113), T, HQ, D), ints(np.concatenate([[0], np.cumsum(new)])), ints(ctx)
    both = [lambda out, ws: antkv.page_attn(geom, q, SCALE, starts, lens, a.table, a.k_pages, a.v_pages, out=out, workspace=ws)[0],
            lambda out, ws: antkv.qpage_attn(geom, q, SCALE, starts, lens, b.table, *b.pools.args(), out=out, workspace=ws)[0]]
    want = [f(None, None).clone() for f in both]
    assert all(w.isfinite().all() for w in want) and not torch.equal(*want)
    need = max(antkv.page_attn_workspace(geom, T, "cuda").numel(), antkv.qpage_attn_workspace(geom, T, "cuda").numel())
    ws = torch.randint(0, 256, (need,), dtype=torch.uint8, device="cuda", generator=gen_of(114))
    outs = [torch.empty_like(q) for _ in both]
    for i in (0, 1, 1, 0, 0, 1, 0, 1):
        outs[i].fill_(7.0)
        both[i](outs[i], ws)
        assert torch.equal(bits(outs[i]), bits(want[i])), i
    torch.cuda.synchronize()
    graphs = []
    for f, out in zip(both, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            f(out, ws)
        graphs.append(graph)
    for n, i in enumerate((1, 0, 0, 1, 0, 1, 1, 0)):
        outs[i].fill_(7.0)
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(bits(outs[i]), bits(want[i])), (n, i)
        if n % 3 == 2:                                              # an eager call of either between
            for j, f in enumerate(both):
                assert torch.equal(bits(f(None, ws)), bits(want[j]))


def test_rows_on_their_way_out_captured():
    """Rows out of 8-bit pages and turned back, in one graph, replayed over other lengths, tables and bytes; arrays made here, and given ones."""
    R, N, page, n_pages = 3, 90, 32, 20
    geom, freqs, gen = antkv.Geometry(R, HKV, HKV, 8), antkv.rope_freqs(96), gen_of(115)
    pools = eights.Pools(n_pages, HKV, page, seed=116)
    table, lens = torch.zeros((R, 4), dtype=torch.int32, device="cuda"), ints([N] * R)
    given = [torch.zeros((R, HKV, N, D), dtype=torch.float16, device="cuda") for _ in "kv"]

    def call(given):
        k, v = antkv.qpage_load(geom, *pools.args(), table, N, first=5, ctx_len=lens)
        antkv.qpage_load(geom, *pools.args(), table, N, first=5, ctx_len=lens, k=given[0], v=given[1])
        return k, v, antkv.rope(geom, None, k, freqs, pos0=5, style=1, inverse=True)[1]

    call(given)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = call(given)
    for i, n in enumerate(([95, 40, 0], [5, 6, 200], [-3, 95, 70], [60, 60, 60])):
        table.copy_(torch.randperm(n_pages, device="cuda", generator=gen)[:4 * R].view(R, 4))
        table[i % R, i % 4] = -1
        lens.copy_(ints(n))
        for s in pools.scales:
            s.copy_(torch.exp2(torch.randint(-9, 3, s.shape, device="cuda", generator=gen).float()))
        for g in given:
            g.fill_(float(i))
        mine = [g.clone() for g in given]
        want = call(mine)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(bits(x), bits(y)) for x, y in zip((*outs, *given), (*want, *mine))), i
        assert want[2].isfinite().all()
