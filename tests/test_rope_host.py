"""Host-side check of what rope does with tensors that record gradients, without a GPU."""
import pytest
import torch

import paper_2506_19505_amd as antkv


@pytest.mark.parametrize("which", ["q", "k", "both", "result"])
def test_rope_refuses_to_drop_gradients(which):
    """Rows that gradients are asked of: their turned copies would have none.  Without gradients the call goes on to its other checks."""
    geom, freqs = antkv.Geometry(1, 8, 2, 8), torch.zeros(64, dtype=torch.float64)
    q, k = torch.zeros((3, 8, 128), dtype=torch.float16), torch.zeros((3, 2, 128), dtype=torch.float16)
    if which in ("q", "both", "result"):
        q.requires_grad_()
    if which in ("k", "both"):
        k.requires_grad_()
    if which == "result":
        q = q * 2
    for rows in ((q, k), (q, None) if q.requires_grad else (None, k)):
        with pytest.raises(ValueError, match="inverse"):
            antkv.rope(geom, *rows, freqs)
        for quiet in (torch.no_grad, torch.inference_mode):
            with quiet(), pytest.raises(ValueError, match="device"):
                antkv.rope(geom, *rows, freqs)
    with pytest.raises(ValueError, match="device"):
        antkv.rope(geom, q.detach(), k.detach(), freqs)
