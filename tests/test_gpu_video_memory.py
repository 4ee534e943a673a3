"""The example that runs group norm, rotary positions, the cache and its attention together: a memory of a video's frames."""
import math

import numpy as np
import pytest
import torch

from cache_ref import attend

pytestmark = pytest.mark.gpu


def _head64(head, x, pos):
    """The head in 64 bits for autograd: x [h, w, C], pos [h * w, 3]."""
    h, w, c = x.shape
    z = x.reshape(h * w, head.groups, -1)
    z = (z - z.mean((0, 2), keepdim=True)) / torch.sqrt(z.var((0, 2), unbiased=False, keepdim=True) + 1e-5)
    u = z.reshape(h * w, c) * head.gamma + head.beta
    y = (u * torch.sigmoid(u) @ head.weight).view(h * w, -1, head.dim)
    q, k, v = y.split([head.q_heads, head.kv_heads, head.kv_heads], 1)
    turned = head.dim // 8 * 6
    n = turned // 6
    f = 100.0 ** (-torch.arange(n, dtype=torch.float64) / n)
    a = (pos.double()[:, :, None] * f).flatten(1)[:, None]

    def turn(m):
        p, r = m[..., :turned // 2], m[..., turned // 2:turned]
        return torch.cat((p * a.cos() - r * a.sin(), p * a.sin() + r * a.cos(), m[..., turned:]), -1)

    return turn(q), turn(k), v


class _Like:
    def __init__(self, head):
        for n in ("q_heads", "kv_heads", "dim", "groups"):
            setattr(self, n, getattr(head, n))
        self.gamma, self.beta, self.weight = (p.detach().double().cpu().requires_grad_() for p in head.parameters)


def test_the_heads_loss_and_gradients():
    """Against the formulas in 64 bits.  Features in float32, so every step is off by a few 2^-24 of sums of at most 96 terms: 1e-4 of a gradient's
    norm leaves a factor of ten."""
    from examples.video_memory import Head, loss_of, positions_of, same_of
    g = torch.Generator().manual_seed(1)
    h, w, c = 5, 7, 32
    head = Head(c, q_heads=4, kv_heads=2, dim=16, groups=4)
    with torch.no_grad():
        head.gamma += 0.2 * torch.randn(c, generator=g).cuda()
        head.beta += 0.2 * torch.randn(c, generator=g).cuda()
    x = [torch.randn((h, w, c), generator=g) for _ in range(2)]
    pos = [positions_of(h, w, (s * 2 - 1, -s), s, "cpu") for s in range(2)]
    same = same_of(h, w, (-1, 0), (1, -1), "cpu")
    assert sorted(set(same.tolist()))[0] == -1 and int((same >= 0).sum()) == 3 * 6
    loss = loss_of(head, (x[0].cuda(), pos[0].cuda()), (x[1].cuda(), pos[1].cuda()), same.cuda())
    loss.backward()
    like = _Like(head)
    q, _, _ = _head64(like, x[1].double(), pos[1])
    _, k, _ = _head64(like, x[0].double(), pos[0])
    logits = torch.stack([q[:, i] @ k[:, i // 2].t() for i in range(4)])[:, same >= 0] / math.sqrt(16)
    want = torch.nn.functional.cross_entropy(logits.flatten(0, 1), same[same >= 0].repeat(4))
    want.backward()
    assert abs(float(loss) - float(want)) < 1e-5 * float(want)
    for p, r in zip(head.parameters, (like.gamma, like.beta, like.weight)):
        far = float((p.grad.double().cpu() - r.grad).norm() / r.grad.norm())
        assert far < 1e-4, far


@pytest.mark.parametrize("h,w", [(1, 1), (5, 7), (8, 8), (9, 15)])
def test_memory_holds_the_last_frames(h, w):
    """Reads after each of five frames, three of which are held: against 64 bits over the values the pages hold.  The result is rounded to half precision: 2^-11 of
    each value, and the attention's own weights and values are rounded to half as well; 3e-3 of the norm is four of those."""
    from examples.video_memory import VideoMemory
    g = torch.Generator().manual_seed(h * w)
    n, kv, q_heads, dim = h * w, 2, 6, 40
    memory, kept = VideoMemory(3, n, kv, dim), []
    out, lse = memory.read(torch.randn((n, q_heads, dim), generator=g).half().cuda())
    assert float(out.abs().max()) == 0 and bool((lse == -math.inf).all())
    for t in range(5):
        k, v = (torch.randn((n, kv, dim), generator=g).half().cuda() for _ in range(2))
        visible = (torch.rand(n, generator=g) < 0.8).to(torch.uint8)
        visible[0] = 1
        memory.put(k, v, visible.cuda() if t % 2 else None)
        slot = t % 3
        back = memory.cache.read(memory.table[slot], memory.starts, memory.none_held, n, n, torch.float32)
        kept.append((slot, *(b.double().cpu().numpy() for b in back), visible.numpy().astype(bool) if t % 2 else np.ones(n, bool)))
        held = sorted(kept[-3:], key=lambda f: f[0])
        q = torch.randn((n, q_heads, dim), generator=g).half()
        out, lse = memory.read(q.cuda())
        kk, vv, see = (np.concatenate([f[i] for f in held]) for i in (1, 2, 3))
        want, want_lse = attend(q.double().numpy(), kk, vv, np.ones(len(see), bool), False, 0, see, dim ** -0.5)
        far = np.linalg.norm(out.double().cpu().numpy() - want) / np.linalg.norm(want)
        assert far < 3e-3, (t, far)
        assert np.abs(lse.cpu().numpy() - want_lse).max() < 5e-3


def test_labels_are_carried():
    """A small video, start to end: training lowers the loss, and the labels of the first frame come through better than by chance (one in eight)."""
    from examples.video_memory import main
    losses, untrained, right = main(["--size", "128", "--frames", "5", "--steps", "12"])
    assert all(math.isfinite(x) for x in losses) and losses[-1] < losses[0]
    assert len(right) == len(untrained) == 4 and min(right) > 0.25
