"""Batched serving over caches of 8 bits and logits before sampling, at the
shapes where another path of a kernel begins.  Oracle, checks and tolerances are
test_gpu_serving8.py's, where nothing else is said.
"""
import numpy as np
import pytest
import torch

from paper_2605_08755_amd import laq
from test_gpu_serving import dev, f16, say
from test_gpu_serving8 import DEV, adjust_case, adjust_check, to_dev

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------
# logits before sampling
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("R,V,H,N,mask", [(1, 5, 3, 2, True), (3, 4001, 60, 5, True), (5, 8200, 0, 0, False),
                                          (300, 7001, 64, 4, True), (2, 70001, 17000, 300, True)])
def test_adjust_into_columns_beside_the_logits(R, V, H, N, mask):
    """Logits and out as columns of one array, either first, and as rows of
    unlike strides between each other: the bits of a call with arrays of their
    own, nothing beside out written."""
    say("adjust columns", R, V, H, N, mask)
    rng = np.random.default_rng(R + V)
    logits, a = adjust_case(rng, R, V, H, N, mask)
    d = to_dev(a)
    want = laq.adjust_logits(dev(logits), **d)
    torch.cuda.synchronize()
    adjust_check(logits, a, want.cpu().numpy())
    for gap in (0, 3, 8):
        for first in (True, False):
            both = torch.full((R, 2 * V + gap + 5), 7.0, dtype=torch.float16, device=DEV)
            x, y = both[:, :V], both[:, V + gap:2 * V + gap]
            if not first:
                x, y = y, x
            x.copy_(dev(logits))
            before = both.clone()
            got = laq.adjust_logits(x, **d, out=y)
            torch.cuda.synchronize()
            assert got.data_ptr() == y.data_ptr() and torch.equal(y.view(torch.int16), want.view(torch.int16))
            y.copy_(before[:, V + gap:2 * V + gap] if first else before[:, :V])
            assert torch.equal(both.view(torch.int16), before.view(torch.int16))
    # out's rows between the logits', whose stride is twice theirs: row i of out at V + i 2 V, of the logits at i 4 V
    flat = torch.full((4 * V * (R + 1),), 7.0, dtype=torch.float16, device=DEV)
    x, y = flat.as_strided((R, V), (4 * V, 1)), flat.as_strided((R, V), (2 * V, 1), V)
    x.copy_(dev(logits))
    laq.adjust_logits(x, **d, out=y)
    torch.cuda.synchronize()
    assert torch.equal(y.view(torch.int16), want.view(torch.int16)) and torch.equal(x.view(torch.int16), dev(logits).view(torch.int16))
    with pytest.raises(laq.LaqError):
        laq.adjust_logits(x, **d, out=flat.as_strided((R, V), (4 * V, 1), V - 1))
