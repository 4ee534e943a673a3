"""The cache of 8-bit pages: codes and scales against the formula, to the bit, and the values read back."""
import numpy as np
import pytest
import torch

from cache_ref import PAGE, RefCache

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def make(pages, heads, dim, fill=True):
    from paper_2210_09887_amd import ops
    c = ops.GpuCache.empty(pages, heads, dim)
    if fill:                                             # what pages hold before they are first used does not matter
        c.k.random_(-128, 128)
        c.v.random_(-128, 128)
        c.k_scale.fill_(float("nan"))
        c.v_scale.fill_(float("nan"))
    return c, RefCache(pages, heads, dim), RefCache(pages, heads, dim)


def same(c, rk, rv, table, lengths):
    k, v = c.k.cpu().numpy(), c.v.cpu().numpy()
    ks, vs = c.k_scale.cpu().numpy(), c.v_scale.cpu().numpy()
    for row, n in zip(table, lengths):
        for i in range(min(len(row), -(-n // PAGE))):
            p, m = row[i], min(PAGE, n - i * PAGE)
            if 0 <= p < len(ks):
                assert np.array_equal(ks[p], rk.scale[p], equal_nan=True) and np.array_equal(vs[p], rv.scale[p], equal_nan=True), (p, ks[p], rk.scale[p])
                assert np.array_equal(k[p, :, :m, :c.dim], rk.codes[p, :, :m]), f"keys of page {p}"
                assert np.array_equal(v[p, :, :c.dim, :m].transpose(0, 2, 1), rv.codes[p, :, :m]), f"values of page {p}"


def put(c, rk, rv, table, counts, held, dtype, g, amp=1.0, views=False):
    T = sum(counts)
    both = (amp * torch.randn((T, 2, c.heads, c.dim + (1 if views else 0)), generator=g)).to(dtype)[..., int(views):]
    k, v = both[:, 0], both[:, 1]
    starts = np.concatenate([[0], np.cumsum(counts)]).astype(int)
    bd = torch.empty((T, 2, c.heads, c.dim + (1 if views else 0)), dtype=dtype, device="cuda")[..., int(views):]
    bd.copy_(both)
    c.store(bd[:, 0], bd[:, 1], ints(table), ints(starts.tolist()), ints(held), max(counts, default=0))
    rk.store(k.double().numpy(), table, starts, held)
    rv.store(v.double().numpy(), table, starts, held)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("heads,dim", [(1, 8), (3, 32), (2, 40), (2, 64), (1, 72), (2, 96), (1, 128), (1, 160), (1, 192), (2, 200), (1, 256)])
def test_codes_and_scales(heads, dim, dtype):
    """Prompts of odd lengths, then a few tokens, then one at a time: pages that are begun, filled and begun anew."""
    g = torch.Generator().manual_seed(dim)
    c, rk, rv = make(16, heads, dim)
    table = [[3, 9, 1, -1], [0, 2, -1, -1], [15, 4, 5, 6]]
    held = [0, 0, 0]
    for counts, amp in (([1, 63, 130], 1.0), ([70, 3, 62], 3.0), ([1, 1, 1], 1.0), ([1, 0, 1], 40.0), ([2, 1, 0], 41.0), ([60, 5, 1], 0.5), ([1, 1, 1], 45.0)):
        put(c, rk, rv, table, counts, held, dtype, g, amp, views=amp == 3.0)
        held = [a + b for a, b in zip(held, counts)]
        same(c, rk, rv, table, held)
    # the values back, whole sequences and a piece of each
    for first, n in (([0, 0, 0], held), ([1, 64, 7], [min(held[0] - 1, 65), held[1] - 64, 100])):
        starts = np.concatenate([[0], np.cumsum(n)]).astype(int)
        k, v = c.read(ints(table), ints(starts.tolist()), ints(first), max(n), int(starts[-1]), dtype)
        for got, r in ((k, rk), (v, rv)):
            for s in range(3):
                want, _ = r.values(table[s], first[s] + n[s])
                want = torch.from_numpy(want[first[s]:]).float().to(dtype)       # code * scale is rounded to 32 bits, then to the type
                assert torch.equal(got[starts[s]:starts[s + 1]].cpu(), want)


def test_zeros_small_values_and_values_that_are_not_finite():
    g = torch.Generator().manual_seed(1)
    c, rk, rv = make(4, 2, 32)
    table = [[1, 2]]
    put(c, rk, rv, table, [5], [0], torch.float32, g, 0.0)
    same(c, rk, rv, table, [5])
    put(c, rk, rv, table, [5], [5], torch.float32, g, 1e-44)                     # the scale is a number of few bits, or zero
    same(c, rk, rv, table, [10])
    put(c, rk, rv, table, [5], [10], torch.float32, g, 1e37)
    same(c, rk, rv, table, [15])
    x = torch.randn((3, 2, 32), generator=g).cuda()
    for bad in (float("nan"), float("inf"), float("-inf")):
        x[1, 1, 7] = bad
        c.store(x, x, ints(table), ints([0, 3]), ints([15]), 3)
        rk.store(x.double().cpu().numpy(), table, [0, 3], [15])
        rv.store(x.double().cpu().numpy(), table, [0, 3], [15])
        assert bool(c.k_scale[1, 1].isnan()) and bool(c.k_scale[1, 0].isfinite())
        k, v = c.read(ints(table), ints([0, 18]), ints([0]), 18, 18, torch.float32)
        assert bool(k[:, 1].isnan().all()) and bool(k[:, 0].isfinite().all())
        put(c, rk, rv, table, [2], [18], torch.float32, g)                       # stays so ..
        assert bool(c.v_scale[1, 1].isnan())
        put(c, rk, rv, table, [20], [0], torch.float32, g)                       # .. until the page is stored from its start again
        same(c, rk, rv, table, [20])


@pytest.mark.parametrize("amp", [1e-37, 3e-38, 1e-39, 1e-42])
def test_scales_without_a_finite_reciprocal(amp):
    """Values so small that their scale is subnormal: codes as the quotients say, to the bit."""
    g = torch.Generator().manual_seed(3)
    c, rk, rv = make(2, 2, 40)
    for counts, held in (([70], [0]), ([5], [70])):
        put(c, rk, rv, [[1, 0]], counts, held, torch.float32, g, amp)
        same(c, rk, rv, [[1, 0]], [held[0] + counts[0]])


def test_a_page_that_grows_at_every_token_stays_within_its_bound():
    """64 tokens, each a little larger than the last: half a code for the last rounding and half of 0.8 + 0.64 + .. = 4 for the earlier ones."""
    c, rk, rv = make(1, 1, 32)
    x = torch.randn((64, 1, 32), generator=torch.Generator().manual_seed(2))
    x = x / x.abs().amax(2, keepdim=True) * (1.02 ** torch.arange(64.0))[:, None, None]
    for t in range(64):
        c.store(x[t:t + 1].cuda(), x[t:t + 1].cuda(), ints([[0]]), ints([0, 1]), ints([t]), 1)
    k, v = c.read(ints([[0]]), ints([0, 64]), ints([0]), 64, 64, torch.float32)
    for got, scale in ((k, c.k_scale), (v, c.v_scale)):
        assert float((got.cpu() - x).abs().max()) <= 2.501 * float(scale.max()) and float(scale.max()) <= 1.25 * float(x.abs().max()) / 127 * 1.001


def test_tokens_without_a_page_are_left_out():
    g = torch.Generator().manual_seed(3)
    c, rk, rv = make(3, 1, 32)
    before = c.k.clone(), c.v.clone()
    table = [[-1, 1], [2, 7], [1 << 30, -5]]
    put(c, rk, rv, table, [100, 200, 70], [0, 0, 0], torch.float16, g)
    same(c, rk, rv, table, [100, 200, 70])
    assert torch.equal(c.k[0], before[0][0]) and torch.equal(c.v[0], before[1][0])
    starts = ints([0, 100, 300, 370])
    k, v = c.read(ints(table), starts, ints([0, 0, 0]), 200, 370, torch.float32)
    for got, r in ((k, rk), (v, rv)):
        for s, (a, b) in enumerate(((0, 100), (100, 300), (300, 370))):
            assert np.array_equal(got[a:b].cpu().numpy(), r.values(table[s], b - a)[0].astype(np.float32))
    # rows beyond the maps are not touched, whatever starts say; max_new bounds a sequence
    x = torch.ones((10, 1, 32), device="cuda")
    c.store(x, x, ints([[0, 1]]), ints([0, 90]), ints([0]), 90)
    assert bool((c.k[0, 0, :10] == 127).all()) and bool((c.k[0, 0, 10:] == before[0][0, 0, 10:]).all())
    c.store(2 * x, 2 * x, ints([[0, 1]]), ints([0, 10]), ints([0]), 4)
    assert bool((c.k[0, 0, 4:10] == 127).all()) and abs(float(c.k_scale[0]) - 2 / 127) < 1e-6


def test_pages_beyond_four_gibibytes():
    from paper_2210_09887_amd import ops
    c = ops.GpuCache.empty(33000, 8, 256)                # 4.3 GB of keys, as much of values
    x = torch.randn((70, 8, 256), generator=torch.Generator().manual_seed(4))
    table = ints([[32999, 16500]])
    c.store(x.cuda(), x.cuda(), table, ints([0, 70]), ints([0]), 70)
    k, v = c.read(table, ints([0, 70]), ints([0]), 70, 70, torch.float32)
    assert torch.equal(k, v) and float((k.cpu() - x).abs().max()) < 0.51 * float(c.k_scale[32999].max())
    r = RefCache(2, 8, 256)
    r.store(x.double().numpy(), [[0, 1]], [0, 70], [0])
    assert np.array_equal(c.k[32999].cpu().numpy(), r.codes[0]) and np.array_equal(c.k_scale[16500].cpu().numpy(), r.scale[1])


def test_refusals():
    from paper_2210_09887_amd import ops
    c, _, _ = make(2, 2, 32)
    x, t, s, h = torch.zeros((3, 2, 32), device="cuda"), ints([[0]]), ints([0, 3]), ints([0])
    for bad in (lambda: ops.GpuCache.empty(2, 2, 30), lambda: ops.GpuCache.empty(2, 2, 264), lambda: ops.GpuCache(c.k, c.k, c.k_scale, c.v_scale, 40),
                lambda: ops.GpuCache(c.k, c.v, c.k_scale.half(), c.v_scale, 32), lambda: c.store(x, x, t.long(), s, h, 3), lambda: c.store(x, x, t, s[:1], h, 3),
                lambda: c.store(x, x.half(), t, s, h, 3), lambda: c.store(x[:, :1], x[:, :1], t, s, h, 3), lambda: c.store(x, x, t, s, h.cpu(), 3),
                lambda: c.store(x.transpose(1, 2), x, t, s, h, 3), lambda: c.read(t, s, h, 3, 3, torch.int8)):
        with pytest.raises(ValueError):
            bad()
    assert [t.shape for t in c.read(t, ints([0, 0]), h, 0, 0, torch.float16)] == [(0, 2, 32)] * 2
