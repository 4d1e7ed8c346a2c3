"""GPU checks of rotary positions for more groups of tokens than a grid has workgroups, with the tolerance of the other rope tests."""
import pytest
import torch

import paper_2506_19505_amd as antkv
from test_gpu_rope import D, compare, ints, randn

pytestmark = pytest.mark.gpu

MOST_GROUPS = 1 << 20
H = 17                                                              # heads: 16 threads to a row, 256 to a workgroup, so that it has one token


def test_rope_of_more_tokens_than_a_grid_has_workgroups():
    """A workgroup's second pass: rows on both sides of the border, and the last ones."""
    assert 256 // 16 // H <= 1
    T = MOST_GROUPS + 77
    x = randn(11, 1, 1, D).expand(T, H, D)
    freqs = antkv.rope_freqs()
    got = antkv.rope(antkv.Geometry(1, H, H, 8), None, x, freqs, style=1)[1]
    for a in (0, MOST_GROUPS - 50, T - 40):
        n = min(100, T - a)
        compare(got[a:a + n].transpose(0, 1), x[a:a + n].transpose(0, 1), torch.arange(a, a + n, device="cuda"), freqs, 1)
    # every row: those at one position are alike in all heads
    assert torch.equal(got, got[:, :1].expand(T, H, D))


def test_rope_of_a_packed_batch_of_more_tokens_than_a_grid_has_workgroups():
    """The same of requests; rows that are nobody's lie behind the border where the first pass had a request's, and the other way round."""
    T, lead, end = MOST_GROUPS + 77, 30, MOST_GROUPS + 50
    x = randn(12, 1, 1, D).expand(T, H, D)
    freqs = antkv.rope_freqs(64)
    out = torch.full((T, H, D), 7.0, dtype=torch.float16, device="cuda")
    starts, ctx = [lead, MOST_GROUPS - 5, MOST_GROUPS + 10, end], [1 << 21, 100, 3000]
    antkv.rope(antkv.Geometry(3, H, H, 8), None, x, freqs, q_start=ints(starts), ctx_len=ints(ctx), k_out=out)
    assert (out[:lead] == 7.0).all() and (out[end:] == 7.0).all()
    for r in range(3):
        a, b = starts[r], starts[r + 1]
        for i in (a, max(a, b - 40)):
            j = min(b, i + 40)
            pos = torch.arange(ctx[r] - (b - i), ctx[r] - (b - j), device="cuda")
            compare(out[i:j].transpose(0, 1), x[i:j].transpose(0, 1), pos, freqs, 0)
