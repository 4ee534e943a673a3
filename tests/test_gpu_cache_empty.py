"""A pool without pages, and tables without entries: what sequences hold before anything was stored."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("pages,entries", [(0, 0), (0, 3), (2, 0)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16], ids=str)
def test_nothing_is_held(dtype, pages, entries):
    from paper_2210_09887_amd import ops
    c = ops.GpuCache.empty(pages, 2, 40)
    before = c.k.random_(-128, 128).clone(), c.v.random_(-128, 128).clone()
    table, starts, n = ints([[0] * entries] * 2), ints([0, 3, 133]), ints([100, 150])
    assert table.shape == (2, entries)
    x = torch.randn((133, 2, 40), device="cuda").to(dtype)
    c.store(x, x, table, starts, ints([0, 20]), 130)
    assert torch.equal(c.k, before[0]) and torch.equal(c.v, before[1])
    for t in c.read(table, starts, ints([0, 20]), 130, 133, dtype):
        assert t.shape == x.shape and not t.any()
    for rows in (133, 1):                                # .. and one query
        q, s = torch.randn((rows, 6, 40), device="cuda").to(dtype), starts if rows > 1 else ints([0, 0, 1])
        for kw in (dict(), dict(causal=True), dict(causal=True, window=7), dict(mask=torch.ones((2, 150), dtype=torch.bool, device="cuda"))):
            out, lse = c.attend(q, table, s, n, rows, 150, **kw)
            assert not out.any() and bool((lse == -float("inf")).all())
