"""Cache and rotary positions captured in a graph, and on a stream that is not the current one."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def draw(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).cuda()


def on_another_stream(call):
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = call()
    s.synchronize()
    return got


def captured(call):
    """(graph, what its replays write)"""
    on_another_stream(call)
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g, stream=s):
        got = call()
    return g, got


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary(interleaved, dtype):
    from paper_2210_09887_amd import ops
    q, k = draw(1, 70, 6, 64).to(dtype), draw(2, 70, 2, 64).to(dtype)
    pos, steps = ints(list(range(70))), ops.rotary_steps(48)
    call = lambda: ops.rotary((q, k), pos, steps, interleaved=interleaved)  # noqa: E731
    want = call()
    assert all(torch.equal(a, b) for a, b in zip(on_another_stream(call), want))
    g, got = captured(call)
    for n in range(3):
        q.mul_(1.5)
        pos.add_(1000 * n)
        g.replay()
        torch.cuda.synchronize()
        want = call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), n


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("counts", [[1, 1], [130, 70]], ids=str)
def test_store_and_read(counts, dtype):
    from paper_2210_09887_amd import ops
    T, starts, table, held = sum(counts), ints([0, counts[0], sum(counts)]), ints([[5, 0, 3, 6], [1, 2, 4, 7]]), ints([3, 60])
    back, first = [63, 124], ints([0, 0])
    x, y = draw(3, T, 2, 40).to(dtype), draw(4, T, 2, 40).to(dtype)

    def fresh():
        c = ops.GpuCache.empty(8, 2, 40)
        for t in (c.k, c.v, c.k_scale, c.v_scale):
            t.zero_()
        return c

    def call(c):
        c.store(x, y, table, starts, held, max(counts))
        return c.read(table, ints_of, first, max(back), sum(back), dtype)

    ints_of = ints([0, back[0], sum(back)])
    c, d = fresh(), fresh()
    want, got = call(c), on_another_stream(lambda: call(d))
    for a, b in zip((c.k, c.v, c.k_scale, c.v_scale, *want), (d.k, d.v, d.k_scale, d.v_scale, *got)):
        assert torch.equal(a, b)
    e, f = fresh(), fresh()
    g, got = captured(lambda: call(e))
    for t in (e.k, e.v, e.k_scale, e.v_scale):           # (what the call before the capture has stored)
        t.zero_()
    for n in range(4):                                   # scales grow and codes are rounded again, in both alike
        x.mul_(1.3)
        held.add_(counts[0] if n < 2 and counts[0] == 1 else 0)
        g.replay()
        torch.cuda.synchronize()
        want = call(f)
        torch.cuda.synchronize()
        for a, b in zip((e.k, e.v, e.k_scale, e.v_scale, *got), (f.k, f.v, f.k_scale, f.v_scale, *want)):
            assert torch.equal(a, b), n
