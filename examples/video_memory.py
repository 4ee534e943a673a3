"""Labels carried through a moving-camera video by a memory of its past frames.

A sparse network gives every frame's feature map (`GpuNet`).  Behind it a head makes queries, keys and values of the pixels:
group norm with silu, one projection, rotary positions - row and column of the pixel in the world, which the camera's shifts give, and the
frame's number.  Keys and values of past frames are kept in 8 bits in the pages of a `GpuCache`; a new frame's pixels
read the labels of what they resemble.  The head is trained so that a pixel finds itself in the frame before.

    python examples/video_memory.py [--size 512] [--frames 12] [--steps 30]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from inputs import build_net, build_sequence  # noqa: E402
from paper_2210_09887_amd import ops  # noqa: E402
from paper_2210_09887_amd.runtime import GpuNet  # noqa: E402

PAGE = 64


class Head:
    """Queries, keys and values of a feature map's pixels.  Parameters in float32; the maps are made in the features' type."""

    def __init__(self, channels, q_heads=8, kv_heads=2, dim=64, groups=32, seed=0, device="cuda:0"):
        g = torch.Generator().manual_seed(seed)
        self.q_heads, self.kv_heads, self.dim, self.groups = q_heads, kv_heads, dim, groups
        n = (q_heads + 2 * kv_heads) * dim
        self.gamma, self.beta = torch.ones(channels, device=device), torch.zeros(channels, device=device)
        self.weight = (torch.randn((channels, n), generator=g) * channels ** -0.5).to(device)
        self.steps = ops.rotary_steps(turned=dim // 8 * 6, axes=3, base=100.0, device=device)
        self.parameters = [self.gamma, self.beta, self.weight]
        for p in self.parameters:
            p.requires_grad_()

    def __call__(self, features, positions):
        """features [h, w, C], positions [h * w, 3] int32 -> q [h * w, q_heads, dim], k, v [h * w, kv_heads, dim]"""
        h, w, c = features.shape
        x = ops.group_norm_act(features[None], self.groups, self.gamma, self.beta, act="silu").view(h * w, c)
        y = (x @ self.weight.to(x.dtype)).view(h * w, -1, self.dim)
        q, k, v = y.split([self.q_heads, self.kv_heads, self.kv_heads], 1)
        q, k = ops.rotary_turn((q, k), positions, self.steps, axes=3)
        return q, k, v


class VideoMemory:
    """The last `frames` frames of a video, a frame's pixels on pages of its own."""

    def __init__(self, frames, pixels, kv_heads, dim, device="cuda:0"):
        self.frames, self.pixels, self.per = frames, pixels, -(-pixels // PAGE)
        self.cache = ops.GpuCache.empty(frames * self.per, kv_heads, dim, device)
        self.table = torch.arange(frames * self.per, dtype=torch.int32, device=device).view(frames, 1, self.per)
        self.whole = self.table.view(1, -1)
        self.mask = torch.zeros((1, frames * self.per * PAGE), dtype=torch.uint8, device=device)    # zero: no pixel there, or none to be seen
        self.starts = torch.tensor([0, pixels], dtype=torch.int32, device=device)
        self.none_held = torch.zeros(1, dtype=torch.int32, device=device)
        self.lengths = [torch.tensor([n * self.per * PAGE], dtype=torch.int32, device=device) for n in range(frames + 1)]
        self.count = 0                                                                             # frames that were ever put

    def put(self, k, v, visible=None):
        """A frame in place of the oldest; visible: [pixels], zero for pixels that are not to be read."""
        at = self.count % self.frames
        self.cache.store(k, v, self.table[at], self.starts, self.none_held, self.pixels)
        row = self.mask[0, at * self.per * PAGE:][:self.pixels]
        row.fill_(1) if visible is None else row.copy_(visible)
        self.count += 1

    def read(self, q):
        """(out, lse) of every pixel's queries over the frames held; zeros and -inf while there is none."""
        held = min(self.count, self.frames)
        return self.cache.attend(q, self.whole, self.starts, self.lengths[held], self.pixels, held * self.per * PAGE, mask=self.mask)


def positions_of(h, w, origin, t, device="cuda:0"):
    """Row and column in the world and frame number of every pixel, int32 [h * w, 3]."""
    y = torch.arange(h, dtype=torch.int32, device=device) + origin[0]
    x = torch.arange(w, dtype=torch.int32, device=device) + origin[1]
    return torch.stack((y[:, None].expand(h, w), x[None].expand(h, w), torch.full((h, w), t, dtype=torch.int32, device=device)), -1).view(h * w, 3)


def regions_of(positions, size, labels):
    """The labels that the first frame comes with: squares of `size` pixels of the world."""
    return (positions[:, 0].div(size, rounding_mode="floor") + 3 * positions[:, 1].div(size, rounding_mode="floor")) % labels


def features_of(size, frames, seed_net=3):
    """Feature maps [h, w, C] of a moving-camera video and the view's origin for each, in pixels of the map."""
    net, seq = build_net(seed_net, H=size, W=size), build_sequence(3, n_frames=frames, H=size, W=size)
    gpu = GpuNet(net)
    maps, origins, at = [], [], [0, 0]
    for t in range(frames):
        shift = [int(n) for n in seq.shifts[t]]
        at = [at[0] + shift[0], at[1] + shift[1]]
        out, _ = gpu.frame(torch.from_numpy(seq.frames[t]).cuda(), *shift)
        maps.append(gpu.split_outputs(out)[0].clone())
        origins.append(tuple(at))
    torch.cuda.synchronize()
    gpu.close()
    return maps, origins


def loss_of(head, before, now, same):
    """How badly the pixels of `now` find themselves among those of `before`: same[i] is the pixel of `before` at the place of pixel i, -1 if out of view."""
    q, _, _ = head(*now)
    _, k, _ = head(*before)
    per = head.q_heads // head.kv_heads
    seen = same >= 0
    logits = torch.stack([q[:, i].float() @ k[:, i // per].float().t() for i in range(head.q_heads)])[:, seen] * head.dim ** -0.5
    return torch.nn.functional.cross_entropy(logits.flatten(0, 1), same[seen].repeat(head.q_heads))


def same_of(h, w, before, now, device="cuda:0"):
    """The pixel of the earlier view at the world's place of every pixel of the later one, -1 where it lies outside."""
    p = positions_of(h, w, (now[0] - before[0], now[1] - before[1]), 0, device).long()
    inside = (p[:, 0] >= 0) & (p[:, 0] < h) & (p[:, 1] >= 0) & (p[:, 1] < w)
    return torch.where(inside, p[:, 0] * w + p[:, 1], -1)


def train(head, maps, origins, steps, rate=3e-3):
    h, w, _ = maps[0].shape
    opt = torch.optim.Adam(head.parameters, lr=rate)
    losses = []
    for i in range(steps):
        t = 1 + i % (len(maps) - 1)
        pair = [(maps[s], positions_of(h, w, origins[s], s)) for s in (t - 1, t)]
        loss = loss_of(head, *pair, same_of(h, w, origins[t - 1], origins[t]))
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(float(loss.detach()))
    return losses


@torch.no_grad()
def carry(head, maps, origins, labels=8, region=6, memory_frames=4):
    """Carries the first frame's labels through the video.  Returns each later frame's share of right labels among the pixels the first frame has seen."""
    h, w, _ = maps[0].shape
    memory, right = VideoMemory(memory_frames, h * w, head.kv_heads, head.dim), []
    for t, (features, origin) in enumerate(zip(maps, origins)):
        pos = positions_of(h, w, origin, t)
        q, k, v = head(features, pos)
        truth = regions_of(pos, region, labels)
        if t == 0:
            found, known = truth, torch.ones(h * w, dtype=torch.uint8, device=q.device)
        else:
            out, lse = memory.read(q)
            found = out[..., :labels].float().sum(1).argmax(-1)
            known = torch.isfinite(lse).all(1).to(torch.uint8)
            seen = same_of(h, w, origins[0], origin) >= 0
            right.append(float((found == truth)[seen].float().mean()) if bool(seen.any()) else 1.0)
        v = v.clone()
        v[..., :labels] = torch.nn.functional.one_hot(found.long(), labels)[:, None]            # a pixel's value begins with its label
        memory.put(k, v, known)
    return right


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--size", type=int, default=512)
    p.add_argument("--frames", type=int, default=12)
    p.add_argument("--steps", type=int, default=30)
    a = p.parse_args(argv)
    maps, origins = features_of(a.size, a.frames)
    head = Head(maps[0].shape[2])
    untrained = carry(head, maps, origins)
    losses = train(head, maps, origins, a.steps)
    right = carry(head, maps, origins)
    print(f"{a.frames} frames of {a.size} x {a.size}, maps {tuple(maps[0].shape)}: loss {losses[0]:.3f} -> {losses[-1]:.3f} in {a.steps} steps")
    print("labels right, frame by frame: before training " + " ".join(f"{r:.2f}" for r in untrained) + " | after " + " ".join(f"{r:.2f}" for r in right))
    return losses, untrained, right


if __name__ == "__main__":
    main()
