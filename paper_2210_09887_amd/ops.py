"""Operators behind the feature maps, on device tensors: group norm with an activation, rotary positions, a cache of
keys and values in 8 bits and the attention that reads it.

Argument marshalling only: shapes, strides and types are taken from the tensors, outputs and workspaces come from torch, the
work is enqueued on the current stream of the tensors' device.  `group_norm_act` is the same for autograd.
"""
from __future__ import annotations

import torch

from . import binding as B

_DTYPE = {torch.float32: B.MDCNN_F32, torch.float16: B.MDCNN_F16, torch.bfloat16: B.MDCNN_BF16}
_ACT = {"none": B.MDCNN_ACT_NONE, "relu": B.MDCNN_ACT_RELU, "silu": B.MDCNN_ACT_SILU}


def _stream(dev):
    return torch.cuda.current_stream(dev).cuda_stream


def _need(ok, text):
    if not ok:
        raise ValueError(text)


def _on(dev, **tensors):
    """Every given tensor is on the GPU `dev`: a pointer of another device would be read there."""
    _need(dev.type == "cuda", "mdcnn needs GPU tensors: there is no CPU path")
    for name, t in tensors.items():
        _need(t is None or t.device == dev, f"{name} is on {None if t is None else t.device}, not on {dev}")


def _floats(name, t, n):
    _need(t is None or (t.dtype == torch.float32 and t.numel() == n and t.is_contiguous()), f"{name}: {n} contiguous float32 values")


def _beside(t):
    """The last extent's elements lie side by side."""
    return t.stride(-1) == 1 or t.shape[-1] == 1 or t.numel() == 0


def _ptr(t):
    return None if t is None else t.data_ptr()


def _work(nbytes, dev):
    return torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes else None


# -- group norm -----------------------------------------------------------------------------------------------------------
def _map(name, t, like=None):
    _need(t.dim() == 4 and (like is None or t.shape == like.shape), f"{name}: a map [N, H, W, C]" + ("" if like is None else f" of shape {tuple(like.shape)}"))
    _need(t.dtype in _DTYPE and (like is None or t.dtype == like.dtype), f"{name}: float32, float16 or bfloat16" + ("" if like is None else ", as x"))
    _need(_beside(t), f"{name}: channels last")
    return B.mdcnn_strides(t.stride(0), t.stride(1), t.stride(2))


def _norm_desc(x, groups, gamma, beta, eps, act):
    _need(act in _ACT, f"act: one of {', '.join(_ACT)}")
    xs = _map("x", x)
    N, H, W, C = x.shape
    _on(x.device, gamma=gamma, beta=beta)
    _floats("gamma", gamma, C)
    _floats("beta", beta, C)
    return B.mdcnn_group_norm_desc(N, H, W, C, int(groups), _DTYPE[x.dtype], _ACT[act], eps, _ptr(gamma), _ptr(beta), xs, xs, xs)


def group_norm(x, groups, gamma=None, beta=None, eps=1e-5, act="none", out=None):
    """y = act(gamma (x - mean) / sqrt(variance + eps) + beta) over every image and group of channels of x [N, H, W, C].

    x may be a view with any strides as long as its channels lie side by side.  Returns (y, mean, rstd), the statistics
    [N, groups] in float32."""
    d = _norm_desc(x, groups, gamma, beta, eps, act)
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    _on(x.device, out=out)
    d.ys = _map("out", out, x)
    n = B.mdcnn_group_norm_bytes(d)
    stats = torch.empty((2, x.shape[0], int(groups)), dtype=torch.float32, device=x.device)
    work = _work(n, x.device)
    with torch.cuda.device(x.device):
        B.mdcnn_group_norm(d, x.data_ptr(), out.data_ptr(), stats[0].data_ptr(), stats[1].data_ptr(), _ptr(work), n, _stream(x.device))
    return out, stats[0], stats[1]


def group_norm_backward(x, dy, mean, rstd, groups, gamma=None, beta=None, act="none"):
    """Gradients (dx, dgamma, dbeta) of group_norm from the gradient dy of y and the statistics it returned."""
    d = _norm_desc(x, groups, gamma, beta, 0.0, act)
    _on(x.device, dy=dy, mean=mean, rstd=rstd)
    d.ds = _map("dy", dy, x)
    _floats("mean", mean, x.shape[0] * int(groups))
    _floats("rstd", rstd, x.shape[0] * int(groups))
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    d.ys = _map("dx", dx, x)
    n = B.mdcnn_group_norm_bytes(d, True)
    grads = torch.empty((2, x.shape[3]), dtype=torch.float32, device=x.device)
    work = _work(n, x.device)
    with torch.cuda.device(x.device):
        B.mdcnn_group_norm_backward(d, x.data_ptr(), dy.data_ptr(), mean.data_ptr(), rstd.data_ptr(), dx.data_ptr(), grads[0].data_ptr(), grads[1].data_ptr(),
                                    _ptr(work), n, _stream(x.device))
    return dx, grads[0], grads[1]


class _GroupNormAct(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, groups, gamma, beta, eps, act):
        y, mean, rstd = group_norm(x, groups, gamma, beta, eps, act)
        ctx.save_for_backward(x, gamma, beta, mean, rstd)
        ctx.how = groups, act
        return y

    @staticmethod
    def backward(ctx, dy):
        x, gamma, beta, mean, rstd = ctx.saved_tensors
        groups, act = ctx.how
        if not _beside(dy):
            dy = dy.contiguous()
        dx, dgamma, dbeta = group_norm_backward(x, dy, mean, rstd, groups, gamma, beta, act)
        return dx, None, None if gamma is None else dgamma, None if beta is None else dbeta, None, None


def group_norm_act(x, groups, gamma=None, beta=None, eps=1e-5, act="none"):
    """y of group_norm for autograd: gradients of x, gamma and beta."""
    return _GroupNormAct.apply(x, groups, gamma, beta, eps, act)


# -- rotary positions -------------------------------------------------------------------------------------------------------
_SCALING = {"none": B.MDCNN_ROTARY_PLAIN, "linear": B.MDCNN_ROTARY_LINEAR, "base": B.MDCNN_ROTARY_BASE, "parts": B.MDCNN_ROTARY_PARTS}


def rotary_steps(turned, axes=1, base=10000.0, scaling="none", factor=1.0, original=4096, slow=1.0, fast=32.0, device="cuda:0"):
    """The frequencies of `turned` channels on `axes` positions as `rotary` takes them: an int64 tensor of turned / 2 steps in
    2^64ths of a turn (the upper half of the range as negative numbers).

    scaling: "none"; "linear" all turns slowed by factor; "base" the base raised so that the slowest pair is slowed by factor;
    "parts" pairs that turn fewer than `slow` times within `original` positions slowed by factor, more than `fast` times not at all."""
    _need(scaling in _SCALING, f"scaling: one of {', '.join(_SCALING)}")
    steps = B.mdcnn_rotary_table(B.mdcnn_rotary_desc(int(turned), int(axes), base, _SCALING[scaling], factor, original, slow, fast))
    return torch.tensor([n - (1 << 64) if n >= 1 << 63 else n for n in steps], dtype=torch.int64, device=device)


def _heads(name, t, dtype, dim, tokens):
    _need(t.dim() == 3 and t.shape[0] == tokens and t.shape[2] == dim, f"{name}: [{tokens}, heads, {dim}]")
    _need(t.dtype == dtype, f"{name}: {dtype}")
    _need(_beside(t), f"{name}: channels side by side")


def rotary(maps, positions, steps, axes=1, interleaved=False, magnitude=1.0, inverse=False, out=None):
    """Turns the first 2 * len(steps) channels of every head of one or two maps [tokens, heads, dim] (queries and keys; any strides, channels side by
    side) by positions [tokens] or [tokens, axes] int32; the others are copied.  Returns new tensors, or `out` (which may be `maps`
    themselves).  inverse=True turns back by the same angles, times magnitude: the gradient."""
    first = maps[0]
    tokens, dim, dev = first.shape[0], first.shape[-1], first.device
    _need(1 <= len(maps) <= 2, "maps: one or two")
    _need(first.dtype in _DTYPE, "maps: float32, float16 or bfloat16")
    _need(positions.dtype == torch.int32 and positions.is_contiguous() and positions.numel() == tokens * axes, f"positions: {tokens} x {axes} contiguous int32 values")
    _need(steps.dtype == torch.int64 and steps.dim() == 1 and steps.is_contiguous(), "steps: contiguous int64 values of rotary_steps")
    if out is None:
        out = [torch.empty(m.shape, dtype=m.dtype, device=dev) for m in maps]
    _on(dev, positions=positions, steps=steps, **{f"maps[{i}]": m for i, m in enumerate(maps)}, **{f"out[{i}]": m for i, m in enumerate(out)})
    _need(len(out) == len(maps), "out: one tensor for each map")
    hs = []
    for i, (x, y) in enumerate(zip(maps, out)):
        _heads(f"maps[{i}]", x, first.dtype, dim, tokens)
        _heads(f"out[{i}]", y, first.dtype, dim, tokens)
        _need(x.shape[1] == y.shape[1], "out: as many heads as maps")
        hs.append(B.mdcnn_heads(x.data_ptr(), y.data_ptr(), x.shape[1], x.stride(0), x.stride(1), y.stride(0), y.stride(1)))
    with torch.cuda.device(dev):
        B.mdcnn_rotary(hs, tokens, dim, _DTYPE[first.dtype], positions.data_ptr(), axes, steps.data_ptr(), 2 * steps.numel(), interleaved, inverse, magnitude, _stream(dev))
    return list(out)


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, positions, steps, axes, interleaved, magnitude, *maps):
        ctx.save_for_backward(positions, steps)
        ctx.how = axes, interleaved, magnitude
        return tuple(rotary(maps, positions, steps, axes, interleaved, magnitude))

    @staticmethod
    def backward(ctx, *grads):
        positions, steps = ctx.saved_tensors
        axes, interleaved, magnitude = ctx.how
        grads = [g if _beside(g) else g.contiguous() for g in grads]
        return (None, None, None, None, None, *rotary(grads, positions, steps, axes, interleaved, magnitude, inverse=True))


def rotary_turn(maps, positions, steps, axes=1, interleaved=False, magnitude=1.0):
    """`rotary` for autograd: gradients of the maps."""
    return list(_Rotary.apply(positions, steps, axes, interleaved, magnitude, *maps))


# -- the cache --------------------------------------------------------------------------------------------------------------
class GpuCache:
    """Keys and values in pages of 64 tokens, 8 bits a value with one scale for each page and head.

    k: int8 [pages, heads, 64, pitch], v: int8 [pages, heads, pitch, 64], pitch the next of 32, 64, 96, 128, 192, 256 to `dim`; k_scale, v_scale:
    float32 [pages, heads].  The tensors are the caller's (`GpuCache.empty` makes them).  Which pages are whose is the caller's too: `table` int32
    [sequences, max_pages] of the calls says in which page tokens 64 i .. 64 i + 63 of a sequence lie; entries outside the pool hold no page."""

    def __init__(self, k, v, k_scale, v_scale, dim):
        pages, heads, dev = k.shape[0], k.shape[1], k.device
        pitch = B.mdcnn_cache_pitch(dim)
        _need(pitch > 0, "dim: a multiple of 8 from 8 to 256")
        _need(k.dtype == v.dtype == torch.int8 and k.shape == (pages, heads, 64, pitch) and v.shape == (pages, heads, pitch, 64), f"k, v: int8 [pages, heads, 64, {pitch}] and [pages, heads, {pitch}, 64]")
        _need(k_scale.dtype == v_scale.dtype == torch.float32 and k_scale.shape == v_scale.shape == (pages, heads), "k_scale, v_scale: float32 [pages, heads]")
        _need(all(t.is_contiguous() for t in (k, v, k_scale, v_scale)), "k, v, k_scale, v_scale: contiguous")
        _on(dev, v=v, k_scale=k_scale, v_scale=v_scale)
        self.k, self.v, self.k_scale, self.v_scale, self.dim, self.heads, self.device = k, v, k_scale, v_scale, int(dim), heads, dev
        self._desc = (pages, heads, int(dim), k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr())

    @classmethod
    def empty(cls, pages, heads, dim, device="cuda:0"):
        pitch = B.mdcnn_cache_pitch(dim)
        _need(pitch > 0, "dim: a multiple of 8 from 8 to 256")
        codes = torch.empty((2, pages, heads, 64 * pitch), dtype=torch.int8, device=device)
        scales = torch.empty((2, pages, heads), dtype=torch.float32, device=device)
        return cls(codes[0].view(pages, heads, 64, pitch), codes[1].view(pages, heads, pitch, 64), scales[0], scales[1], dim)

    def _cache(self, table, **per_sequence):
        _need(table.dtype == torch.int32 and table.dim() == 2 and table.is_contiguous(), "table: contiguous int32 [sequences, max_pages]")
        n = table.shape[0]
        for name, t in per_sequence.items():
            _need(t.dtype == torch.int32 and t.is_contiguous() and t.numel() == n + (name == "starts"), f"{name}: {n + (name == 'starts')} contiguous int32 values")
        _on(self.device, table=table, **per_sequence)
        return B.mdcnn_cache_desc(*self._desc, table.data_ptr(), n, table.shape[1])

    def _side(self, name, t):
        _need(t.dim() == 3 and t.shape[1] == self.heads and t.shape[2] == self.dim and _beside(t), f"{name}: [tokens, {self.heads}, {self.dim}], channels side by side")
        return B.mdcnn_heads(t.data_ptr(), t.data_ptr(), self.heads, t.stride(0), t.stride(1), t.stride(0), t.stride(1))

    def store(self, k, v, table, starts, held, max_new):
        """Puts new tokens [tokens, heads, dim] into their pages: sequence s has tokens starts[s] .. starts[s + 1] - 1, which follow the held[s]
        that it has already.  max_new: no sequence has more new tokens."""
        _need(k.dtype == v.dtype and k.dtype in _DTYPE and k.shape == v.shape, "k, v: float32, float16 or bfloat16 of one shape")
        _on(self.device, k=k, v=v)
        c = self._cache(table, starts=starts, held=held)
        with torch.cuda.device(self.device):
            B.mdcnn_cache_store(c, self._side("k", k), self._side("v", v), k.shape[0], starts.data_ptr(), held.data_ptr(), max_new, _DTYPE[k.dtype], _stream(self.device))

    def read(self, table, starts, first, max_new, tokens, dtype):
        """The values of tokens first[s] .. of every sequence s, starts[s + 1] - starts[s] of them, as (k, v) [tokens, heads, dim]; tokens = starts[-1]."""
        _need(dtype in _DTYPE, "dtype: float32, float16 or bfloat16")
        k, v = (torch.empty((tokens, self.heads, self.dim), dtype=dtype, device=self.device) for _ in range(2))
        c = self._cache(table, starts=starts, first=first)
        with torch.cuda.device(self.device):
            if tokens:
                B.mdcnn_cache_read(c, self._side("k", k), self._side("v", v), k.shape[0], starts.data_ptr(), first.data_ptr(), max_new, _DTYPE[dtype], _stream(self.device))
        return k, v

    def attend(self, q, table, starts, lengths, max_new, max_len, scale=None, causal=False, window=0, mask=None, out=None):
        """Attention of queries [tokens, q_heads, dim] (q_heads a multiple of heads) over the cache: sequence s has the queries starts[s] ..
        starts[s + 1] - 1 and lengths[s] tokens in the cache; max_new and max_len are bounds on both.  scale: of the logits, dim ** -0.5 if not given.
        causal: the queries are the last tokens of their sequence and see nothing behind themselves, with window > 0 only the `window`
        tokens up to themselves.  mask: uint8 or bool [sequences, >= max_len], zero: token hidden.  Returns (out, lse): [tokens, q_heads,
        dim] in the type of q and the natural logarithms of the sums [tokens, q_heads] in float32; zeros and -inf where a query sees nothing."""
        _need(q.dtype in _DTYPE and q.dim() == 3 and q.shape[2] == self.dim and _beside(q), f"q: [tokens, q_heads, {self.dim}] float32, float16 or bfloat16, channels side by side")
        tokens, heads, _ = q.shape
        c = self._cache(table, starts=starts, lengths=lengths)
        if out is None:
            out = torch.empty((tokens, heads, self.dim), dtype=q.dtype, device=self.device)
        _need(out.shape == q.shape and out.dtype == q.dtype and _beside(out), "out: as q")
        _on(self.device, q=q, out=out, mask=mask)
        how = B.mdcnn_attend_desc(starts.data_ptr(), lengths.data_ptr(), tokens, max_new, max_len, self.dim ** -0.5 if scale is None else scale, causal, window)
        if mask is not None:
            _need(mask.dtype in (torch.uint8, torch.bool) and mask.dim() == 2 and mask.shape[0] == table.shape[0] and mask.shape[1] >= max_len and mask.stride(1) == 1 and mask.stride(0) >= max_len,
                  f"mask: uint8 or bool [{table.shape[0]}, {max_len} or more]")
            how.mask_dev, how.mask_row = mask.data_ptr(), mask.stride(0)
        n = B.mdcnn_cache_attend_bytes(c, how, heads)
        work = _work(n, self.device)
        lse = torch.empty((tokens, heads), dtype=torch.float32, device=self.device)
        side = B.mdcnn_heads(q.data_ptr(), out.data_ptr(), heads, q.stride(0), q.stride(1), out.stride(0), out.stride(1))
        with torch.cuda.device(self.device):
            B.mdcnn_cache_attend(c, how, side, _DTYPE[q.dtype], lse.data_ptr(), _ptr(work), n, _stream(self.device))
        return out, lse
