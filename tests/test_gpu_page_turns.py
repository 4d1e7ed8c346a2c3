"""GPU checks of pieces of more key tiles than a workgroup looks up at a time (512 tiles of a wide block, 1024 of a narrow one): the turns behind the
first one, in both caches, against 64 bits with the tolerances of the other attention tests."""
import pytest
import torch

import test_gpu_pages as halves
import test_gpu_qpages as eights
from test_gpu_pages import D, gen_of, randn

pytestmark = pytest.mark.gpu

CACHES = [(halves.Cache, halves.check_attn, 0), (eights.ByteCache, eights.check_attn, 2)]           # and log2 of a wide key tile's cost
PAGE, GREAT = 256, 1 << 22                                          # a table's entries for 2^30 tokens


def with_a_great_table(c):
    table = torch.full((len(c.ctx), GREAT), -1, dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = c.table
    c.table = table


def a_workgroup_per_block(T, R, G, waves, shift):
    """Where the costs of all blocks might not fit an int, nothing is cut: a piece has all of its block's key tiles."""
    return T * G // (32 * waves) + min(R, T) > (1 << 30) // ((GREAT * PAGE // 32 + 32) << shift)


def spoil(c, odd, at, window):
    """Values that are not finite: among the sinks, behind the left edge of some rows, on both sides of tile 512, in later turns, near the end."""
    if not odd:
        return
    n = c.ctx[0]
    keys = [3, 90, n - at, n // 4, 16383, 16384, n // 2, n - 2000, n - 40, n - 2]
    if window:
        keys.append(n - at - window + 60)
    for i, key in enumerate(keys):
        x = float(("nan", "inf", "-inf")[i % 3]) if isinstance(c, halves.Cache) else float("nan")
        c.v[0][:, key, 11 * i + 1] = x
    c.fill()


@pytest.mark.parametrize("odd", [False, True])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (36000, 100)])
@pytest.mark.parametrize("cache", CACHES)
def test_wide_blocks_of_four_waves(cache, window, n_sink, odd):
    """40 tokens among single ones: a block of 128 rows on 1250 key tiles, and the one behind it, in which two waves have no rows."""
    make, check, shift = cache
    ctx, new = [40000] + [20] * 39, [40] + [1] * 39
    assert sum(new) * 4 < 1024 * len(new) and a_workgroup_per_block(sum(new), len(new), 4, 4, shift) and 40000 // 32 > 2 * 512
    c = make(101, ctx, 2, PAGE)
    spoil(c, odd, 40, window)
    with_a_great_table(c)
    check(c, new, 8, window, n_sink)


@pytest.mark.parametrize("odd", [False, True])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (36000, 100)])
@pytest.mark.parametrize("cache", CACHES)
def test_wide_blocks_of_eight_waves(cache, window, n_sink, odd):
    """2010 tokens of one request: blocks of 256 rows on up to 1250 key tiles, the last one with waves without rows."""
    make, check, shift = cache
    T = 2010
    assert T * 4 >= 1024 and a_workgroup_per_block(T, 1, 4, 8, shift) and (40000 - T) // 32 > 2 * 512 and 0 < T * 4 % 256 < 224
    c = make(102, [40000], 1, PAGE)
    spoil(c, odd, T, window)
    with_a_great_table(c)
    check(c, [T], 4, window, n_sink, each=3)


@pytest.mark.parametrize("odd", [False, True])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (30000, 100)])
@pytest.mark.parametrize("cache", CACHES)
def test_a_chunk_of_a_long_prompt(cache, window, n_sink, odd):
    """2048 tokens of 32 heads on 32768 keys: 32 blocks of a KV head in 32 shares, so that a piece has about as many key tiles as a block, 1000 (in the window 940)."""
    make, check, _ = cache
    c = make(103, [32768], 8, 64)
    spoil(c, odd, 2048, window)
    check(c, [2048], 32, window, n_sink, each=7)


@pytest.mark.parametrize("odd", [False, True])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (38000, 100)])
@pytest.mark.parametrize("cache", CACHES)
def test_narrow_blocks(cache, window, n_sink, odd):
    """Eight tokens of a request, 32 rows, on 1250 key tiles: a wave has 256 of the first turn and up to 57 of the second."""
    make, check, shift = cache
    ctx, new = [40000] + [20] * 39, [8] + [1] * 39
    assert a_workgroup_per_block(sum(new), len(new), 4, 4, shift) and 38000 // 32 > 1024
    c = make(104, ctx, 2, PAGE)
    spoil(c, odd, 8, window)
    with_a_great_table(c)
    check(c, new, 8, window, n_sink)


@pytest.mark.parametrize("cache", CACHES)
def test_a_reference_that_moves_in_later_turns(cache):
    """Keys far above all before them in the second and in the third turn: what the turns before have summed is scaled down, to nothing in fp32 by the last."""
    make, check, shift = cache
    ctx, new = [40000] + [20] * 39, [40] + [1] * 39
    c = make(105, ctx, 2, PAGE)
    base = torch.where(torch.rand(D, device="cuda", generator=gen_of(105)) < 0.5, 1.0, -1.0)
    q = (base + 0.1 * randn(gen_of(106), sum(new), 8, D).float()).half()
    c.k[0].copy_((0.05 * c.k[0].float()).half())
    for key, gain in ((100, 1), (20000, 4), (35000, 12)):
        c.k[0][:, key] = (gain * base).half()
    c.fill()
    with_a_great_table(c)
    check(c, new, 8, q=q)
