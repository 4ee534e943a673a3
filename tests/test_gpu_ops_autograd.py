"""What the operators do under autograd: the calls without gradients refuse tensors that require one."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def world():
    """Calls by name, each of tensors that may require a gradient, by name; with what they are given."""
    from paper_2210_09887_amd import ops
    g = torch.Generator().manual_seed(1)
    draw = lambda *s: torch.randn(s, generator=g).cuda()  # noqa: E731
    c, pos, steps = ops.GpuCache.empty(1, 2, 16), ints([0, 1, 2]), ops.rotary_steps(16)
    c.store(draw(3, 2, 16), draw(3, 2, 16), ints([[0]]), ints([0, 3]), ints([0]), 3)
    x, gamma, beta = draw(2, 3, 4, 8), draw(8), draw(8)
    _, mean, rstd = ops.group_norm(x, 2, gamma, beta)
    attend = lambda q, out=None: c.attend(q, ints([[0]]), ints([0, 3]), ints([3]), 3, 3, out=out)  # noqa: E731
    return {
        "group_norm": (lambda x, gamma, beta, out: ops.group_norm(x, 2, gamma, beta, out=out), dict(x=x, gamma=gamma, beta=beta, out=draw(2, 3, 4, 8))),
        "group_norm_backward": (lambda x, dy, mean, rstd, gamma, beta: ops.group_norm_backward(x, dy, mean, rstd, 2, gamma, beta),
                                dict(x=x, dy=draw(2, 3, 4, 8), mean=mean, rstd=rstd, gamma=gamma, beta=beta)),
        "rotary": (lambda q, k, out: ops.rotary((q, k), pos, steps, out=(out, torch.empty_like(k))), dict(q=draw(3, 4, 16), k=draw(3, 2, 16), out=draw(3, 4, 16))),
        "store": (lambda k, v: c.store(k, v, ints([[0]]), ints([0, 3]), ints([0]), 3), dict(k=draw(3, 2, 16), v=draw(3, 2, 16))),
        "attend": (attend, dict(q=draw(3, 4, 16), out=draw(3, 4, 16))),
    }


@pytest.mark.parametrize("name", ["group_norm", "group_norm_backward", "rotary", "store", "attend"])
def test_tensors_that_require_a_gradient_are_refused_where_there_is_none(name):
    call, tensors = world()[name]
    call(**tensors)
    for which, t in tensors.items():
        given = dict(tensors)
        given[which] = t.clone().requires_grad_()
        with pytest.raises(ValueError, match=f"{name} gives no gradients"):
            call(**given)
        with torch.no_grad():
            call(**given)
        call(**{**given, which: given[which].detach()})
        with torch.inference_mode():
            call(**given)


def test_the_calls_for_autograd_take_them():
    from paper_2210_09887_amd import ops
    x = torch.randn((2, 3, 4, 8), device="cuda", requires_grad=True)
    q = torch.randn((3, 4, 16), device="cuda", requires_grad=True)
    (ops.group_norm_act(x, 2, act="silu").sum() + ops.rotary_turn((q,), ints([0, 1, 2]), ops.rotary_steps(16))[0].sum()).backward()
    assert x.grad is not None and q.grad is not None


@pytest.mark.parametrize("name", ["group_norm", "rotary", "attend"])
def test_autograd_knows_what_is_written_over(name):
    """A tensor that a product has saved for its gradient, then written by the call."""
    call, tensors = world()[name]
    for kept in (False, True):
        w = torch.ones_like(tensors["out"]).requires_grad_()
        a = 2 * w
        b = a * a
        version = a._version
        if not kept:
            call(**{**tensors, "out": a.detach()})
            assert a._version > version
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                b.sum().backward()
        else:                                            # written elsewhere: the gradient is there
            call(**tensors)
            b.sum().backward()
            assert torch.equal(w.grad, 8 * w.detach())


def test_autograd_knows_that_a_store_writes_the_pages():
    from paper_2210_09887_amd import ops
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            c = ops.GpuCache.empty(1, 2, 16)
            x = torch.randn((3, 2, 16), device="cuda")
            c.store(x, x, ints([[0]]), ints([0, 3]), ints([0]), 3)
    c = ops.GpuCache.empty(1, 2, 16)
    before = [t._version for t in (c.k, c.v, c.k_scale, c.v_scale)]
    c.store(x.clone(), x.clone(), ints([[0]]), ints([0, 3]), ints([0]), 3)
    assert all(t._version > n for t, n in zip((c.k, c.v, c.k_scale, c.v_scale), before))
