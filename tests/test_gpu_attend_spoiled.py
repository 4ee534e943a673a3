"""Queries that are not finite: NaN where they see a token, nothing where they see none, and no other row takes notice."""
import numpy as np
import pytest
import torch

from test_gpu_attend import TYPES, World

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dim", [32, 128, 256])
@pytest.mark.parametrize("counts", [[1, 1], [150, 140]], ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_queries_that_are_not_finite(dtype, counts, dim, bad):
    w = World([300, 200], 2, dim, 22)
    w.queries(counts, 4, dtype)
    w.c.k[..., 5] = -3                                   # a product with minus infinity could be minus infinity throughout
    mask = np.ones((2, 300), np.uint8)
    mask[0] = 0                                          # the first sequence sees nothing
    mask[1, :150] = 0
    m = torch.from_numpy(mask).cuda()
    clean, free = w.got(False, mask=m), w.got(True)
    n, rows = counts[0], sum(counts)
    hit = torch.zeros((rows, 4), dtype=torch.bool)
    hit[0, 1] = hit[rows - 1, 2] = True
    w.q[0, 1, 5] = bad
    w.q[rows - 1, 2, 5] = bad
    hit = hit.cuda()
    out, lse = w.got(False, mask=m)
    assert not out[:n].any() and bool((lse[:n] == -float("inf")).all())
    hit[0, 1] = False
    assert bool(out[hit].isnan().all()) and bool(lse[hit].isnan().all())
    assert torch.equal(out[~hit], clean[0][~hit]) and torch.equal(lse[~hit], clean[1][~hit])
    hit[0, 1] = True
    out, lse = w.got(True)
    assert bool(out[hit].isnan().all()) and bool(lse[hit].isnan().all())
    assert torch.equal(out[~hit], free[0][~hit]) and torch.equal(lse[~hit], free[1][~hit])
