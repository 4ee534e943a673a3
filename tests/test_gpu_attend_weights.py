"""Attention where one token outweighs all others: the others' weights keep their bits, and with them what they add up to."""
import math

import pytest
import torch

from cache_ref import PAGE

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]
EPS = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
HEADS, DIM = 8, 32


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def check_sink(tokens, queries, copies, gap, equal, sink_value, dtype, floor):
    """The first of `tokens` tokens has a logit about `gap` above the others', which are all equal or a deviation of one apart; its values are zeros or like theirs.
    `copies` sequences read the same pages with the same queries: with many of them a block goes over a whole sequence.

    Bounds: a weight is a half (one of fp32 calls two) down to `floor` of the largest, whatever it is; logits of up to G from products and sums in 32 bits, 8 * 2^-24 G;
    sums over the pages in 32 bits, four terms a page; the result rounded once."""
    from paper_2210_09887_amd import ops
    g = torch.Generator().manual_seed(tokens + queries)
    pages, scale = -(-tokens // PAGE), DIM ** -0.5
    k = torch.zeros((tokens, HEADS, DIM))
    if not equal:
        k[1:, :, 1:] = torch.randint(-20, 21, (tokens - 1, HEADS, DIM - 1), generator=g).float()
    k[0, :, 0] = 100
    v = torch.randint(20, 128, (tokens, HEADS, DIM), generator=g).float()
    if sink_value == "zero":
        v[0] = 0
    q = torch.randn((queries, HEADS, DIM), generator=g) / (0.115 * math.sqrt(DIM - 1) * scale)
    q[..., 0] = gap / scale
    q = q.to(dtype)
    c = ops.GpuCache.empty(pages, HEADS, DIM)
    pad = pages * PAGE - tokens
    lay = lambda t: torch.cat((t, torch.full((pad, HEADS, DIM), 77.0))).view(pages, PAGE, HEADS, DIM).permute(0, 2, 1, 3).to(torch.int8)  # noqa: E731
    c.k.copy_(lay(k))
    c.v.copy_(lay(v).transpose(2, 3))
    c.k_scale.fill_(0.01)
    c.v_scale.fill_(0.01)
    table = ints([list(range(pages))] * copies)
    starts = ints([queries * i for i in range(copies + 1)])
    out, lse = c.attend(q.cuda().repeat(copies, 1, 1), table, starts, ints([tokens] * copies), queries, tokens)
    held = float(torch.tensor(0.01))                     # the scales as they are held
    score = torch.einsum("qhd,thd->hqt", q.double(), k.double()) * (held * float(torch.tensor(scale)))
    top = score.amax(2, keepdim=True)
    p = torch.exp(score - top)
    total = p.sum(2, keepdim=True)
    values = v.double().transpose(0, 1) * held
    want = (p / total) @ values
    if dtype == torch.float16 and float(want.abs().min()) < 2.0 ** -14:
        return                                           # (halves do not resolve such results)
    half = 2.0 ** -22 if dtype == torch.float32 else 2.0 ** -11
    arithmetic = (8 * (abs(gap) + 6) + 4 * pages + 16) * 2.0 ** -24
    bound = EPS[dtype] * want.abs() + ((half * p).clamp(min=floor) / total) @ values.abs() + arithmetic * ((p / total) @ values.abs())
    got, logs = out.double().cpu().view(copies, queries, HEADS, DIM).transpose(1, 2), lse.double().cpu().view(copies, queries, HEADS).transpose(1, 2)
    worst = float(((got - want).abs() / bound).max())
    print(f"{dtype} {tokens} tokens, {queries} queries, gap {gap}, {'equal' if equal else 'uneven'}, sink {sink_value}: {worst:.3f} of the bound, "
          f"relative {float((got[0] - want).norm() / want.norm()):.2e}", flush=True)
    assert worst < 1
    assert float((logs - (top + total.log())[..., 0]).abs().max()) < 2 * arithmetic * (1 + abs(gap) / 8)


SHAPES = [(768, 1, 1), (4096, 1, 1), (4096, 130, 1), (2048, 130, 48), (16384, 1, 256)]     # .. the last two: one block goes over a whole sequence


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("tokens,queries,copies", SHAPES)
@pytest.mark.parametrize("gap", [0.0, 10.0, 12.0, 14.0, 17.5, 20.0])
def test_tokens_beside_one_that_outweighs_them(tokens, queries, copies, gap, dtype):
    for equal in (True, False):
        for sink_value in ("zero", "usual"):
            check_sink(tokens, queries, copies, gap, equal, sink_value, dtype, 2.0 ** -35)


@pytest.mark.parametrize("tokens,queries,copies", SHAPES)
@pytest.mark.parametrize("gap", [14.0, 17.5, 20.0, 24.0])
def test_weights_of_fp32_calls_keep_two_halves_of_bits(tokens, queries, copies, gap):
    """The second half holds 2^11 times what the first leaves: 22 bits down to 2^-24 of the largest weight and a step of 2^-45 of it from there."""
    for equal in (True, False):
        for sink_value in ("zero", "usual"):
            check_sink(tokens, queries, copies, gap, equal, sink_value, torch.float32, 2.0 ** -46)


@pytest.mark.parametrize("size", [1e-27, 1e-20, 1e-9, 1.0, 1e9, 1e20, 1e33])
@pytest.mark.parametrize("queries,pages", [(1, 1), (1, 7), (130, 1), (130, 7)])
def test_values_of_any_size_keep_the_bits_of_fp32(queries, pages, size):
    """All logits are zero: a result is the mean of codes times scales.  Its error: weights of 22 bits (4 * 2^-24), their exponent (16 beside the largest: 6) and
    power (2), sums of 16 terms and over waves and pages (12), inverse and quotient (4); 32 * 2^-24 in all.  64 heads have scales of their own."""
    from paper_2210_09887_amd import ops
    g = torch.Generator().manual_seed(pages)
    heads, n = 64, 64 * pages
    c = ops.GpuCache.empty(pages, heads, DIM)
    codes = torch.randint(20, 128, (pages, heads, DIM, PAGE), generator=g, dtype=torch.int8)
    scale = torch.exp(2 * torch.rand((pages, heads), generator=g)) * size
    c.k.fill_(0)
    c.k_scale.fill_(1)
    c.v.copy_(codes)
    c.v_scale.copy_(scale)
    out, lse = c.attend(torch.zeros((queries, heads, DIM), device="cuda"), ints([list(range(pages))]), ints([0, queries]), ints([n]), queries, n)
    want = (codes.double() * scale.double()[..., None, None]).sum((0, 3)) / n
    worst = float(((out.double().cpu() - want).abs() / want).max()) * 2 ** 24
    print(f"{queries} queries, {pages} pages, values of {size:.0e}: {worst:.1f} * 2^-24", flush=True)
    assert worst < 32
    assert float((lse.double().cpu() - math.log(n)).abs().max()) < 32 * 2.0 ** -24 + 2.0 ** -24 * math.log(n) + 2.0 ** -24 * abs(math.log(size) - 10)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("queries", [1, 130])
@pytest.mark.parametrize("zeros_first", [False, True])
@pytest.mark.parametrize("gap", [0.0, 10.0, 16.0, 20.0, 24.0, 30.0, 50.0, 80.0])
def test_pages_of_zeros_above_values_as_small_as_they_count(gap, zeros_first, queries, dtype):
    """Values of 2^-99 in the pages of one half, zeros with logits that lie `gap` higher in the other's: the sum of the exponentials stays finite, and right.
    Errors: logits 8 * 2^-24 gap, sums over 8 pages and waves 32 * 2^-24, T of 100 in units of log 2, rounded with the log-sum: 2 * 2^-18."""
    from paper_2210_09887_amd import ops
    pages, n = 8, 512
    c = ops.GpuCache.empty(pages, HEADS, DIM)
    c.k.fill_(0)
    c.v.fill_(100)
    low, high = (slice(4, 8), slice(0, 4)) if zeros_first else (slice(0, 4), slice(4, 8))
    c.k[high, :, :, 0] = 100
    c.k_scale.fill_(0.01)
    c.v_scale[low] = 2.0 ** -99
    c.v_scale[high] = 0
    q = torch.zeros((queries, HEADS, DIM))
    q[..., 0] = gap * math.sqrt(DIM)
    q = q.to(dtype)
    out, lse = c.attend(q.cuda(), ints([list(range(pages))]), ints([0, queries]), ints([n]), queries, n)
    real = float(q[0, 0, 0]) / math.sqrt(DIM)
    total = 256 * (1 + math.exp(real))
    assert float((lse.double().cpu() - math.log(total)).abs().max()) < (8 * gap + 32) * 2.0 ** -24 + 2 * 2.0 ** -18
    # a result below 2^-126 may be anything down to zero
    want = 100 * 2.0 ** -99 * 256 / total
    u = 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8
    assert float((out.double().cpu() - want).abs().max()) < want * (u + 2.0 ** -10 + 16 * gap * 2.0 ** -24) + 2.0 ** -126


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=str)
@pytest.mark.parametrize("dim", [32, 128, 256])
def test_few_queries_are_rounded_once(dim, dtype):
    """Up to 16 rows: weights of 22 bits and sums in 32 leave (8 * 8 + 4 + 16) * 2^-24 of a result whose values are all positive, so that no more of
    them lie on the wrong side of a rounding than twice that in units of the type."""
    from paper_2210_09887_amd import ops
    g = torch.Generator().manual_seed(dim)
    seqs, n = 64, 5
    c = ops.GpuCache.empty(seqs, HEADS, dim)
    k = torch.randint(-127, 128, (seqs, HEADS, PAGE, dim), generator=g, dtype=torch.int8)
    v = torch.randint(20, 128, (seqs, HEADS, dim, PAGE), generator=g, dtype=torch.int8)
    c.k.copy_(k)
    c.v.copy_(v)
    c.k_scale.fill_(1 / 64)
    c.v_scale.fill_(1 / 64)
    q = torch.randn((seqs, HEADS, dim), generator=g).to(dtype)
    out, _ = c.attend(q.cuda(), ints([[i] for i in range(seqs)]), ints(list(range(seqs + 1))), ints([n] * seqs), 1, n)
    score = (k[:, :, :n].double() / 64 @ q.double()[..., None])[..., 0] * float(torch.tensor(dim ** -0.5))
    assert float(score.abs().max()) < 8
    want = (v[..., :n].double() / 64 @ torch.softmax(score, -1)[..., None])[..., 0]
    wrong = float((out.cpu() != want.to(dtype)).double().mean())
    bound = 2 * 84 * 2.0 ** -24 / EPS[dtype]
    print(f"{dtype} {dim}: {wrong:.5f} of the results rounded the wrong way, bound {bound:.5f}", flush=True)
    assert wrong < bound
