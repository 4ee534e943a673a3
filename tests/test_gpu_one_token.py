"""One token whose heads lie first, [heads, 1, dim] seen as [1, heads, dim]: its token stride is that of a head and counts for nothing."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def heads_first(heads, dim, dtype, seed, extra=0):
    """The token, and the same in rows side by side; extra: elements between the heads, so that torch does not call it contiguous."""
    t = torch.randn((heads, 1, dim + extra), generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()[..., :dim].transpose(0, 1)
    assert t.stride(0) == t.stride(1) == dim + extra
    return t, t.clone(memory_format=torch.contiguous_format).reshape(-1).view(1, heads, dim)


@pytest.mark.parametrize("extra", [0, 8, 3])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_rotary(dtype, interleaved, extra):
    from paper_2210_09887_amd import ops
    (q, qs), (k, ks) = heads_first(6, 64, dtype, 1, extra), heads_first(2, 64, dtype, 2, extra)
    pos, steps = ints([12345]), ops.rotary_steps(48)
    want = ops.rotary((qs, ks), pos, steps, interleaved=interleaved)
    got = ops.rotary((q, k), pos, steps, interleaved=interleaved)
    into = heads_first(6, 64, dtype, 3, extra)[0], heads_first(2, 64, dtype, 4, extra)[0]
    ops.rotary((q, k), pos, steps, interleaved=interleaved, out=into)
    for g, i, w in zip(got, into, want):
        assert torch.equal(g, w) and torch.equal(i, w)
    ops.rotary((q, k), pos, steps, interleaved=interleaved, out=(q, k))
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_rotary_gradient():
    from paper_2210_09887_amd import ops
    q, _ = heads_first(6, 64, torch.float32, 5)
    d, ds = heads_first(6, 64, torch.float32, 6)
    pos, steps = ints([77]), ops.rotary_steps(64)
    q.requires_grad_()
    y, = ops.rotary_turn((q,), pos, steps)
    y.backward(d)
    assert torch.equal(q.grad, ops.rotary((ds,), pos, steps, inverse=True)[0])


@pytest.mark.parametrize("extra", [0, 8, 3])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_cache_and_attention(dtype, extra):
    from paper_2210_09887_amd import ops
    (k, ks), (v, vs), (q, qs) = heads_first(2, 64, dtype, 7, extra), heads_first(2, 64, dtype, 8, extra), heads_first(6, 64, dtype, 9, extra)
    caches = []
    for a, b in ((k, v), (ks, vs)):
        c = ops.GpuCache.empty(2, 2, 64)
        for t in (c.k, c.v, c.k_scale, c.v_scale):
            t.fill_(1)
        c.store(a, b, ints([[1, 0]]), ints([0, 1]), ints([70]), 1)
        caches.append(c)
    c, w = caches
    assert all(torch.equal(a, b) for a, b in ((c.k, w.k), (c.v, w.v), (c.k_scale, w.k_scale), (c.v_scale, w.v_scale)))
    how = ints([[1, 0]]), ints([0, 1]), ints([71]), 1, 71
    want, got, into = w.attend(qs, *how, causal=True), c.attend(q, *how, causal=True), heads_first(6, 64, dtype, 10, extra)[0]
    lse = c.attend(q, *how, causal=True, out=into)[1]
    assert torch.equal(got[0], want[0]) and torch.equal(into, want[0]) and torch.equal(got[1], want[1]) and torch.equal(lse, want[1])
    c.attend(q, *how, causal=True, out=q)
    assert torch.equal(q, want[0])
