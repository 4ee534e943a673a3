"""Attention over the cache of 8-bit pages against the formula in 64 bits."""
import numpy as np
import pytest
import torch

from cache_ref import PAGE, RefCache, attend

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]
EPS = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class World:
    """Sequences of the given lengths in a cache of their own, with the pages in no order; codes and scales drawn directly."""

    def __init__(self, lengths, kv_heads, dim, seed=0, spare=2, v_amp=1.0):
        from paper_2210_09887_amd import ops
        r = np.random.default_rng(seed)
        n = [-(-v // PAGE) for v in lengths]
        self.pages, self.lengths, self.kv, self.dim = sum(n) + spare, lengths, kv_heads, dim
        ids = r.permutation(self.pages)
        most = max(1, max(n, default=1))
        self.table = np.full((len(lengths), most), -1)
        at = 0
        for s, k in enumerate(n):
            self.table[s, :k] = ids[at:at + k]
            at += k
        self.c = ops.GpuCache.empty(self.pages, kv_heads, dim)
        self.k, self.v = RefCache(self.pages, kv_heads, dim), RefCache(self.pages, kv_heads, dim)
        for ref, codes, scale, amp, last in ((self.k, self.c.k, self.c.k_scale, 1.0, False), (self.v, self.c.v, self.c.v_scale, v_amp, True)):
            codes.random_(-127, 128)                     # the channels beyond dim hold something, too
            ref.codes[:] = np.clip(np.rint(r.standard_normal(ref.codes.shape) * 40), -127, 127)
            ref.scale[:] = np.exp(r.standard_normal(ref.scale.shape) * 0.5) / 40 * amp
            x = torch.from_numpy(ref.codes.transpose(0, 1, 3, 2) if last else ref.codes).to(torch.int8)
            (codes[:, :, :dim] if last else codes[..., :dim]).copy_(x)
            scale.copy_(torch.from_numpy(ref.scale))
        self.r = r

    def queries(self, counts, heads, dtype, amp=1.5):
        self.counts, self.starts = counts, np.concatenate([[0], np.cumsum(counts)]).astype(int)
        self.q = torch.from_numpy(self.r.standard_normal((int(self.starts[-1]), heads, self.dim)) * amp).to(dtype)
        return self.q

    def want(self, causal, window=0, mask=None, scale=None, rows=None):
        scale = float(np.float32(self.dim ** -0.5 if scale is None else scale))
        out, lse = [], []
        for s, n in enumerate(self.lengths):
            (k, there), (v, _) = self.k.values(self.table[s], n), self.v.values(self.table[s], n)
            q = self.q[self.starts[s]:self.starts[s + 1]].double().numpy()
            o, e = attend(q, k, v, there, causal, window, None if mask is None else mask[s], scale)
            out.append(o)
            lse.append(e)
        return np.concatenate(out), np.concatenate(lse)

    def got(self, causal, window=0, mask=None, scale=None, **kw):
        return self.c.attend(self.q.cuda(), ints(self.table.tolist()), ints(self.starts.tolist()), ints(self.lengths), max(self.counts, default=0), max(self.lengths, default=0),
                             scale, causal, window, mask, **kw)

    def check(self, causal, window=0, mask=None, scale=None):
        out, lse = self.got(causal, window, None if mask is None else torch.from_numpy(mask).cuda(), scale)
        want, wl = self.want(causal, window, mask, scale)
        compare(out, lse, want, wl, self)


def compare(out, lse, want, wl, w):
    u = EPS[out.dtype]
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.array_equal(np.isneginf(lse), np.isneginf(wl))
    live = ~np.isneginf(wl)
    assert not out[~live].any()
    # logits of size up to 40 from products that are exact in 32 bits and sums and exponents that are not: 40 * 8 * 2^-24 of every
    # probability; probabilities as halves (or two): 2^-12 (2^-23) each, rounded at random; the result once
    logit = 8 * 2.0 ** -24 * max(1.0, float(np.abs(wl[live]).max(initial=0)) + 40)
    assert np.abs(lse[live] - wl[live]).max(initial=0) < 2 * logit
    half = 2.0 ** -23 if u == 2.0 ** -24 else 2.0 ** -11
    size = np.abs(want).max(initial=0) + float(w.v.scale.max()) * 127
    assert (np.abs(out - want) - u * np.abs(want)).max(initial=0) < (2 * logit + half) * size
    norm = np.linalg.norm(want)
    assert norm == 0 or np.linalg.norm(out - want) / norm < 1.5 * u + 4 * logit + half


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("dim", [8, 32, 40, 64, 80, 96, 128, 160, 192, 200, 256])
def test_head_sizes_and_types(dim, dtype):
    w = World([1, 63, 64, 65, 200, 700], 2, dim, dim)
    w.queries([1, 1, 1, 1, 1, 1], 6, dtype)
    w.check(True)
    w.queries([1, 3, 0, 5, 2, 9], 6, dtype)
    w.check(True)
    w.check(False)


@pytest.mark.parametrize("kv,heads", [(1, 1), (3, 3), (1, 7), (2, 32), (4, 12), (1, 40)])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_shared_heads(kv, heads, dtype):
    w = World([130, 5], kv, 64, heads)
    w.queries([1, 2], heads, dtype)
    w.check(True)
    w.queries([40, 5], heads, dtype)
    w.check(True)
    w.check(False, mask=(w.r.random((2, 131)) < 0.5).astype(np.uint8))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("window", [0, 1, 64, 100])
@pytest.mark.parametrize("counts", [[1, 1], [7, 20], [150, 333]], ids=str)
def test_causal_and_windows(counts, window, dtype):
    w = World([517, 333], 2, 64, window)
    w.queries(counts, 4, dtype)
    w.check(True, window)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("counts", [[1, 1, 1], [100, 130, 65]], ids=str)
def test_masks_and_rows_that_see_nothing(counts, dtype):
    w = World([300, 129, 200], 2, 32, 5)
    w.queries(counts, 4, dtype)
    mask = (w.r.random((3, 307)) < 0.3).astype(np.uint8)
    mask[1] = 0
    mask[2, :190] = 0
    for row in (307, 320):
        m = np.zeros((3, row), np.uint8)
        m[:, :307] = mask * 3
        w.check(False, mask=m)
        w.check(True, mask=m)
        w.check(True, 40, mask=m)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_empty_sequences_and_more_queries_than_tokens(dtype):
    w = World([0, 10, 3, 0], 1, 64, 6)
    w.queries([4, 0, 40, 1], 2, dtype)
    w.check(True)
    w.check(False)
    w.queries([0, 0, 0, 0], 2, dtype)
    out, lse = w.got(True)
    assert out.shape == (0, 2, 64) and lse.shape == (0, 2)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("counts", [[1, 1], [90, 200]], ids=str)
def test_tokens_without_a_page_are_not_there(counts, dtype):
    w = World([500, 300], 2, 64, 7)
    w.table[0, 0], w.table[0, 3], w.table[1, :] = -1, w.pages, -7
    w.queries(counts, 4, dtype)
    w.check(False)
    w.check(True)
    w.table = np.ascontiguousarray(w.table[:, :3])       # a table that is shorter than the sequences
    w.check(True)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("counts,lengths", [([1, 1], [20000, 7000]), ([3, 1], [4097, 64]), ([70, 500], [5000, 3001])], ids=str)
def test_long_sequences(counts, lengths, dtype):
    w = World(lengths, 1, 64, 8)
    w.queries(counts, 2, dtype)
    w.check(True)


@pytest.mark.parametrize("v_amp", [1e-20, 1e-6, 1e6, 1e20])
@pytest.mark.parametrize("counts", [[1], [200]], ids=str)
def test_values_of_any_size(counts, v_amp):
    """The probabilities are halves: their products with the scales would not be."""
    for dtype in (torch.float32, torch.bfloat16):
        w = World([1000], 2, 32, 9, v_amp=v_amp)
        w.v.scale[w.table[0, 3]] = 0                     # a page of zeros
        w.v.scale[w.table[0, 5]] *= 1000
        w.c.v_scale.copy_(torch.from_numpy(w.v.scale))
        w.queries(counts, 2, dtype)
        w.check(True)


@pytest.mark.parametrize("amp", [1e-30, 1e-4, 1e4, 1e30])
@pytest.mark.parametrize("counts", [[1], [200]], ids=str)
def test_queries_of_any_size(counts, amp):
    for dtype in (torch.float32, torch.bfloat16):
        w = World([300], 2, 64, 10)
        w.queries(counts, 4, dtype, amp)
        w.q[0] = 0
        w.check(True, scale=0.2 / amp if amp > 1e-20 else 1e30 * 0.2)


@pytest.mark.parametrize("counts", [[1], [150]], ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_one_token_outweighs_all_others(counts, dtype):
    """Logits of several hundred: the maximum moves late, everything before it fades to nothing."""
    w = World([400], 1, 32, 11)
    w.queries(counts, 1, dtype)
    w.check(True, scale=20.0)
    w.check(True, scale=-20.0)
    w.check(True, scale=0.0)


@pytest.mark.parametrize("counts", [[1, 1], [130, 70]], ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_hidden_tokens_have_no_influence_and_bad_ones_reach_those_that_see_them(counts, dtype):
    w = World([400, 200], 2, 32, 12)
    w.queries(counts, 2, dtype)
    mask = np.ones((2, 400), np.uint8)
    mask[0, 64:128] = 0
    clean = w.got(True, mask=torch.from_numpy(mask).cuda())
    bad = int(w.table[0, 1])
    w.c.k_scale[bad] = float("nan")
    w.c.v_scale[bad] = float("nan")
    got = w.got(True, mask=torch.from_numpy(mask).cuda())
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])
    out, lse = w.got(True)                               # without the mask the page is seen by every query of the first sequence
    n = counts[0]
    assert bool(out[:n].isnan().all()) and bool(lse[:n].isnan().all()) and bool(out[n:].isfinite().all())
    w.c.k_scale[bad] = 0.01                              # values alone
    out, lse = w.got(True)
    assert bool(out[:n].isnan().all()) and bool(lse.isfinite().all()) and bool(out[n:].isfinite().all())
    if n > 100:                                          # causal: rows before the page do not see it
        last = int(w.table[0, 6])
        w.c.v_scale[bad] = 0.01
        w.c.v_scale[last] = float("nan")
        out, _ = w.got(True)
        first_hit = 6 * PAGE - (400 - n)
        assert bool(out[:first_hit].isfinite().all()) and bool(out[first_hit:n].isnan().all())
    # a query that is not finite spoils its own row only
    w.c.v_scale[:] = 0.01
    clean = w.got(True)
    w.q[0, 0, 3] = float("nan")
    out, _ = w.got(True)
    assert bool(out[0, 0].isnan().all()) and torch.equal(out[0, 1], clean[0][0, 1]) and torch.equal(out[1:], clean[0][1:])


@pytest.mark.parametrize("counts", [[1, 2], [100, 61]], ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_strides_and_bounds(counts, dtype):
    """Queries as a slice of a projection that begins at any element, output into a slice; bounds larger than anything there is."""
    w = World([333, 64], 2, 40, 13)
    w.queries(counts, 4, dtype)
    out, lse = w.got(True)
    T = sum(counts)
    t, s, n = ints(w.table.tolist()), ints(w.starts.tolist()), ints(w.lengths)
    for at in (0, 3, 8):
        big = torch.zeros((T, 4 * 40 + 16), dtype=dtype, device="cuda")
        q = big[:, at:at + 160].view(T, 4, 40)
        q.copy_(w.q)
        into = torch.full((T, 4, 48), 5.0, dtype=dtype, device="cuda")
        o, e = w.c.attend(q, t, s, n, max(counts), 333, causal=True, out=into[..., :40])
        assert torch.equal(o, out) and torch.equal(e, lse) and bool((into[..., 40:] == 5).all())
        o, e = w.c.attend(q, t, s, n, 10 * max(counts) + 100, 5000, causal=True)
        compare(o, e, *w.want(True), w)
        o, e = w.c.attend(q, t, s, n, max(counts), 333, causal=True, out=q)      # in place
        assert torch.equal(o, out)


def test_the_same_bits_twice_and_on_another_stream():
    w = World([3000, 1700], 2, 128, 14)
    for counts in ([1, 1], [300, 129]):
        w.queries(counts, 8, torch.bfloat16)
        first = w.got(True)
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            again = w.got(True)
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_pages_beyond_four_gibibytes():
    from paper_2210_09887_amd import ops
    c = ops.GpuCache.empty(33000, 8, 256)
    x = torch.randn((70, 8, 256), generator=torch.Generator().manual_seed(15)).cuda()
    for ids in ([32999, 16500], [1, 2]):
        c.store(x, x, ints([ids]), ints([0, 70]), ints([0]), 70)
    for q in (x[:1], x):
        far, near = (c.attend(q, ints([ids]), ints([0, len(q)]), ints([70]), len(q), 70, causal=True) for ids in ([32999, 16500], [1, 2]))
        assert torch.equal(far[0], near[0]) and torch.equal(far[1], near[1]) and bool(far[0].isfinite().all())


def test_captured_in_a_graph():
    w = World([900, 400], 2, 64, 16)
    for counts in ([1, 1], [100, 200]):
        w.queries(counts, 4, torch.float16)
        q, t, s, n = w.q.cuda(), ints(w.table.tolist()), ints(w.starts.tolist()), ints(w.lengths)
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            w.c.attend(q, t, s, n, max(counts), 900, causal=True)
        st.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            out, lse = w.c.attend(q, t, s, n, max(counts), 900, causal=True)
        for k in range(3):
            n.sub_(10 * k)
            q.mul_(0.9)
            g.replay()
            torch.cuda.synchronize()
            want = w.c.attend(q, t, s, n, max(counts), 900, causal=True)
            torch.cuda.synchronize()
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1]), k


def test_stored_and_read_by_the_attention():
    """Tokens put in one after the other are what a prompt put in at once is, as far as the scales of a growing page let them."""
    from paper_2210_09887_amd import ops
    g = torch.Generator().manual_seed(17)
    T, kv, heads, dim = 150, 2, 4, 64
    k, v = torch.randn((2, T, kv, dim), generator=g).cuda()
    q = torch.randn((T, heads, dim), generator=g).cuda()
    c = ops.GpuCache.empty(3, kv, dim)
    table = ints([[2, 0, 1]])
    rows = []
    for t in range(T):
        c.store(k[t:t + 1], v[t:t + 1], table, ints([0, 1]), ints([t]), 1)
        rows.append(c.attend(q[t:t + 1], table, ints([0, 1]), ints([t + 1]), 1, T, causal=True)[0])
    one = torch.cat(rows)
    s = torch.einsum("thd,shd->hts", q.double().cpu(), k.double().cpu().repeat_interleave(2, 1)) * dim ** -0.5
    s.masked_fill_(torch.ones(T, T).triu(1).bool(), -float("inf"))
    want = torch.einsum("hts,shd->thd", torch.softmax(s, -1), v.double().cpu().repeat_interleave(2, 1))
    # codes of 3 / 127 of a deviation, off by half a step and a little more, uniformly: about a hundredth
    assert float((one.double().cpu() - want).norm() / want.norm()) < 0.03


def test_refusals():
    w = World([10], 2, 32, 18)
    w.queries([3], 4, torch.float16)
    q, t, s, n = w.q.cuda(), ints(w.table.tolist()), ints([0, 3]), ints([10])
    m = torch.ones((1, 10), dtype=torch.uint8, device="cuda")
    for bad in (lambda: w.c.attend(q.double(), t, s, n, 3, 10), lambda: w.c.attend(q[..., :16], t, s, n, 3, 10), lambda: w.c.attend(q, t, s, n.long(), 3, 10),
                lambda: w.c.attend(q, t, s[:1], n, 3, 10), lambda: w.c.attend(q, t, s, n, 3, 11, mask=m), lambda: w.c.attend(q, t, s, n, 3, 10, mask=m.float()),
                lambda: w.c.attend(q, t, s, n, 3, 10, mask=m.cpu()), lambda: w.c.attend(q, t, s, n, 3, 10, out=q[:2]), lambda: w.c.attend(q.cpu(), t, s, n, 3, 10)):
        with pytest.raises(ValueError):
            bad()
    from paper_2210_09887_amd import binding as B
    for bad in (lambda: w.c.attend(q[:, :3], t, s, n, 3, 10), lambda: w.c.attend(q, t, s, n, 3, 10, window=4), lambda: w.c.attend(q, t, s, n, 3, 10, float("nan"))):
        with pytest.raises(B.MdcnnError):
            bad()


@pytest.mark.parametrize("counts", [[1], [150]], ids=str)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)      # (the results are smaller than halves resolve)
@pytest.mark.parametrize("v_amp", [1e-12, 1.0, 1e12])
def test_pages_of_zeros_first_last_and_between(v_amp, dtype, counts):
    """Pages whose values are all zeros count in the sum of the exponentials and nowhere else, whatever comes before or after them."""
    for zeros in ([0, 1, 2, 3, 4, 5], [0], [10, 11, 12, 13, 14, 15], [1, 5, 9], list(range(15)), list(range(16))):
        w = World([1000], 1, 32, 19, v_amp=v_amp)
        for k in zeros:
            w.v.scale[w.table[0, k]] = 0
            w.k.scale[w.table[0, k]] *= 2
        w.c.v_scale.copy_(torch.from_numpy(w.v.scale))
        w.c.k_scale.copy_(torch.from_numpy(w.k.scale))
        w.queries(counts, 2, dtype)
        if len(zeros) == 16:
            out, lse = w.got(False)
            assert not out.any() and bool(lse.isfinite().all())
        else:
            w.check(False)
