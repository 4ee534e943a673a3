"""Rotary positions against the formula in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

EPS = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def reference(x, pos, freqs, axes, interleaved, magnitude, inverse=False):
    """x [T, h, D] in 64 bits, pos [T, axes], freqs one list per axis."""
    n = len(freqs[0])
    angle = torch.cat([pos[:, a:a + 1].double() * torch.tensor(freqs[a], dtype=torch.float64) for a in range(axes)], 1)[:, None]
    c, s = magnitude * torch.cos(angle), magnitude * torch.sin(angle) * (-1 if inverse else 1)
    R, y = 2 * axes * n, x.clone()
    even, odd = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    a, b = x[..., even], x[..., odd]
    y[..., even], y[..., odd] = a * c - b * s, a * s + b * c
    return y


def plain_freqs(n, axes, base=10000.0):
    return [[base ** (-i / n) for i in range(n)] for _ in range(axes)]


def check(got, want, x):
    # one rounding of the result; sine and cosine to 4 * 2^-24, three more roundings in the sum, relative to the pair's length
    u = EPS[got.dtype]
    size = x.double().abs().amax(-1, keepdim=True) * 1.5
    assert float(((got.double().cpu() - want).abs() - u * want.abs() - 16 * 2.0 ** -24 * size).max()) <= 0


CASES = [(1, 1, 1, 2, 2, 1), (1, 3, 1, 64, 64, 1), (7, 4, 2, 64, 32, 1), (5, 2, 2, 40, 24, 3), (33, 8, 1, 80, 80, 2), (129, 5, 5, 96, 50, 1), (300, 3, 1, 256, 256, 4), (1000, 2, 1, 7, 6, 1),
         (2048, 16, 4, 128, 128, 1)]


@pytest.mark.parametrize("dtype", list(EPS), ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_sizes_layouts_and_types(case, interleaved, dtype):
    from paper_2210_09887_amd import ops
    T, hq, hk, D, R, axes = case
    g = torch.Generator().manual_seed(1)
    q, k = (torch.randn((T, h, D), generator=g).to(dtype) for h in (hq, hk))
    pos = torch.randint(-1000, 100000, (T, axes), generator=g, dtype=torch.int32)
    steps = ops.rotary_steps(R, axes)
    freqs = plain_freqs(R // 2 // axes, axes)
    for inverse in (False, True):
        out = ops.rotary((q.cuda(), k.cuda()), pos.cuda(), steps, axes, interleaved, 1.25, inverse)
        for x, y in zip((q, k), out):
            check(y, reference(x.double(), pos, freqs, axes, interleaved, 1.25, inverse), 1.25 * x)
    one, = ops.rotary((q.cuda(),), pos.cuda(), steps, axes, interleaved, 1.25, True)
    assert torch.equal(one, out[0])
    qc, kc = q.cuda(), k.cuda()
    same = ops.rotary((qc, kc), pos.cuda(), steps, axes, interleaved, 1.25, True, out=(qc, kc))
    assert same[0].data_ptr() == qc.data_ptr() and torch.equal(qc, out[0]) and torch.equal(kc, out[1])


def test_positions_at_the_ends_of_the_range():
    """The angle is exact at any position: integers, compared with integers of Python."""
    from paper_2210_09887_amd import ops
    pos = torch.tensor([0, 1, -1, 2 ** 20, -2 ** 20, 2 ** 31 - 1, -2 ** 31, 123456789], dtype=torch.int32)
    steps = ops.rotary_steps(64)
    x = torch.zeros((len(pos), 1, 64))
    x[..., :32] = 1.0
    y, = ops.rotary((x.cuda(),), pos.cuda(), steps)
    y = y.double().cpu()[:, 0]
    for t, p in enumerate(pos.tolist()):
        for i, s in enumerate(steps.tolist()):
            turn = (p * s % (1 << 64)) / 2.0 ** 64 * 2 * math.pi
            assert abs(y[t, i] - math.cos(turn)) < 4 * 2.0 ** -24 and abs(y[t, 32 + i] - math.sin(turn)) < 4 * 2.0 ** -24


@pytest.mark.parametrize("dtype", list(EPS), ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
def test_strides(interleaved, dtype):
    """Slices of one projection, heads before tokens, a projection that begins at an odd element, into a slice of a larger tensor."""
    from paper_2210_09887_amd import ops
    T, D = 37, 32
    g = torch.Generator().manual_seed(2)
    both = torch.randn((T, 6 * D + 3), generator=g).to(dtype).cuda()
    pos = torch.arange(T, dtype=torch.int32, device="cuda") * 11
    steps = ops.rotary_steps(24)
    for at in (0, 1, 2):
        q, k = both[:, at:at + 4 * D].view(T, 4, D), both[:, at + 4 * D:at + 6 * D].view(T, 2, D)
        want = ops.rotary((q.contiguous(), k.contiguous()), pos, steps, interleaved=interleaved)
        got = ops.rotary((q, k), pos, steps, interleaved=interleaved)
        first = ops.rotary((q.transpose(0, 1).contiguous().transpose(0, 1), k), pos, steps, interleaved=interleaved)
        out = torch.full((T, 7 * D), 9.0, dtype=dtype, device="cuda")
        ops.rotary((q, k), pos, steps, interleaved=interleaved, out=(out[:, :4 * D].view(T, 4, D), out[:, 4 * D:6 * D].view(T, 2, D)))
        for i, w in enumerate(want):
            assert torch.equal(got[i], w) and torch.equal(first[i], w)
        assert torch.equal(out[:, :4 * D].view(T, 4, D), want[0]) and torch.equal(out[:, 4 * D:6 * D].view(T, 2, D), want[1]) and bool((out[:, 6 * D:] == 9).all())
        heads_first = torch.empty((4, T, D), dtype=dtype, device="cuda").transpose(0, 1)
        ops.rotary((q,), pos, steps, interleaved=interleaved, out=(heads_first,))
        assert torch.equal(heads_first, want[0])


def test_scalings_turn_as_their_formulas_say():
    from paper_2210_09887_amd import ops
    n, pos = 16, torch.tensor([[5000], [70000]], dtype=torch.int32)
    x = torch.randn((2, 1, 32), generator=torch.Generator().manual_seed(3))
    f = plain_freqs(n, 1)[0]
    keep = [min(1.0, max(0.0, (2048 * v / (2 * math.pi) - 2) / 14)) for v in f]
    for kw, freqs in ((dict(scaling="linear", factor=8.0), [v / 8 for v in f]), (dict(scaling="base", factor=8.0), plain_freqs(n, 1, 10000.0 * 8.0 ** (n / (n - 1)))[0]),
                      (dict(scaling="parts", factor=8.0, original=2048, slow=2.0, fast=16.0), [v * k + v / 8 * (1 - k) for v, k in zip(f, keep)])):
        y, = ops.rotary((x.cuda(),), pos.cuda(), ops.rotary_steps(32, **kw))
        check(y, reference(x.double(), pos, [freqs], 1, False, 1.0), x)


def test_gradient_is_the_transposed_turn():
    from paper_2210_09887_amd import ops
    g = torch.Generator().manual_seed(4)
    q, k, dq, dk = (torch.randn((9, h, 48), generator=g).cuda() for h in (4, 2, 4, 2))
    pos, steps = torch.arange(27, dtype=torch.int32, device="cuda").view(9, 3), ops.rotary_steps(36, 3)
    q.requires_grad_()
    k.requires_grad_()
    out = ops.rotary_turn((q, k), pos, steps, 3, True, 1.5)
    (out[0] * dq).sum().backward(retain_graph=True)
    (out[1] * dk).sum().backward()
    want = ops.rotary((dq, dk), pos, steps, 3, True, 1.5, inverse=True)
    assert torch.equal(q.grad, want[0]) and torch.equal(k.grad, want[1])
    # <R x, d> = <x, R' d>
    a, b = float((out[0].double() * dq.double()).sum()), float((q.double() * want[0].double()).sum())
    assert abs(a - b) < 2.0 ** -18 * float(q.norm() * dq.norm())


def test_a_map_that_the_loss_leaves_out_and_no_second_gradient():
    from paper_2210_09887_amd import ops
    q, k = (torch.randn((7, 3, 16), device="cuda", requires_grad=True) for _ in range(2))
    pos, steps = torch.arange(7, dtype=torch.int32, device="cuda"), ops.rotary_steps(16)
    out = ops.rotary_turn((q, k), pos, steps)
    d = torch.randn_like(out[0])
    out[0].backward(d, retain_graph=True)
    assert torch.equal(q.grad, ops.rotary((d,), pos, steps, inverse=True)[0]) and not bool(k.grad.any())
    g, = torch.autograd.grad(out[0], q, d.clone().requires_grad_(), create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


def test_no_tokens_and_refusals():
    from paper_2210_09887_amd import ops
    steps, pos = ops.rotary_steps(8), torch.zeros(3, dtype=torch.int32, device="cuda")
    e = torch.empty((0, 2, 8), device="cuda")
    assert ops.rotary((e,), pos[:0], steps)[0].shape == e.shape
    x = torch.zeros((3, 2, 8), device="cuda")
    for bad in (lambda: ops.rotary((x.cpu(),), pos, steps), lambda: ops.rotary((x,), pos.long(), steps), lambda: ops.rotary((x,), pos[:2], steps),
                lambda: ops.rotary((x,), pos, steps.int()), lambda: ops.rotary((x, x, x), pos, steps), lambda: ops.rotary((x, x.half()), pos, steps),
                lambda: ops.rotary((x.transpose(1, 2),), pos, steps), lambda: ops.rotary((x,), pos.cpu(), steps), lambda: ops.rotary((x,), pos, steps, out=(x[:2],)),
                lambda: ops.rotary_steps(8, scaling="other")):
        with pytest.raises(ValueError):
            bad()
