"""Operators behind the feature maps, on device tensors: group norm with an activation, rotary positions, a cache of
keys and values in 8 bits and the attention that reads it.

Argument marshalling only: shapes, strides and types are taken from the tensors, outputs and workspaces come from torch, the
work is enqueued on the current stream of the tensors' device.  `group_norm_act` and `rotary_turn` are the same for autograd; the other calls know no
gradients and refuse tensors that require one while autograd records.

A call on a small map is as long as its way through the host, so what follows from shapes, strides and types alone - the checks, the description
for the library, the size of the workspace - is worked out once for each combination (the cached `_.._plan` functions); pointers are
filled into a copy.
"""
from __future__ import annotations

import functools

import torch
from torch.autograd.function import once_differentiable

from . import binding as B

_DTYPE = {torch.float32: B.MDCNN_F32, torch.float16: B.MDCNN_F16, torch.bfloat16: B.MDCNN_BF16}
_ACT = {"none": B.MDCNN_ACT_NONE, "relu": B.MDCNN_ACT_RELU, "silu": B.MDCNN_ACT_SILU}
_PLANS = 512                                             # combinations of shapes that are remembered


def _need(ok, text):
    if not ok:
        raise ValueError(text)


def _refuse_devices(dev, **tensors):
    _need(dev.type == "cuda", "mdcnn needs GPU tensors: there is no CPU path")
    for name, t in tensors.items():
        _need(t is None or t.device == dev, f"{name} is on {None if t is None else t.device}, not on {dev}")


def _on(dev, *tensors):
    """Whether every given tensor is on the GPU `dev`: a pointer of another device would be read there."""
    return dev.type == "cuda" and all([t is None or t.device == dev for t in tensors])


def _recorded(*tensors):
    """Whether autograd would record what is done with these tensors."""
    return torch.is_grad_enabled() and any([t is not None and t.requires_grad for t in tensors])


def _refuse_gradients(call, instead):
    raise ValueError(f"{call} gives no gradients, and a tensor requires one: {instead}detach it or call under torch.no_grad()")


def _written(*tensors):
    """Tells autograd that these tensors of the caller's hold other values now: what it saved of them is no longer there."""
    torch.autograd.graph.increment_version(tensors)


def _floats(name, t, n):
    _need(t is None or (t.dtype == torch.float32 and t.numel() == n and t.is_contiguous()), f"{name}: {n} contiguous float32 values")


def _beside(shape, stride):
    """The last extent's elements lie side by side."""
    return stride[-1] == 1 or shape[-1] == 1 or 0 in shape


def _ptr(t):
    return None if t is None else t.data_ptr()


def _like(t):
    return torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


def _call(call, dev, *args):
    """call(*args, stream) with `dev` as the current device and its current stream."""
    index = dev.index
    if index == torch.cuda.current_device():
        call(*args, torch._C._cuda_getCurrentRawStream(index))
    else:
        with torch.cuda.device(index):
            call(*args, torch._C._cuda_getCurrentRawStream(index))


# -- group norm -----------------------------------------------------------------------------------------------------------
def _strides(name, shape, stride, like):
    _need(len(shape) == 4 and shape == like, f"{name}: a map [N, H, W, C]" + ("" if shape is like else f" of shape {tuple(like)}"))
    _need(_beside(shape, stride), f"{name}: channels last")
    return B.mdcnn_strides(*stride[:3])


@functools.lru_cache(_PLANS)
def _norm_plan(shape, dtype, groups, act, eps, x_stride, y_stride, d_stride=None, backward=False):
    """(description without pointers, bytes of workspace)"""
    _need(dtype in _DTYPE, "x: float32, float16 or bfloat16")
    _need(act in _ACT, f"act: one of {', '.join(_ACT)}")
    xs = _strides("x", shape, x_stride, shape)
    ys = _strides("dx" if backward else "out", shape, y_stride, shape)
    ds = _strides("dy", shape, d_stride, shape) if backward else xs
    d = B.mdcnn_group_norm_desc(*shape, groups, _DTYPE[dtype], _ACT[act], eps, None, None, xs, ys, ds)
    return d, B.mdcnn_group_norm_bytes(d, backward)


def group_norm(x, groups, gamma=None, beta=None, eps=1e-5, act="none", out=None):
    """y = act(gamma (x - mean) / sqrt(variance + eps) + beta) over every image and group of channels of x [N, H, W, C].

    x may be a view with any strides as long as its channels lie side by side.  Returns (y, mean, rstd), the statistics
    [N, groups] in float32."""
    dev, shape, dtype = x.device, x.shape, x.dtype
    if not _on(dev, gamma, beta, out):
        _refuse_devices(dev, gamma=gamma, beta=beta, out=out)
    if _recorded(x, gamma, beta, out):
        _refuse_gradients("group_norm", "use group_norm_act, ")
    given = out is not None
    if given:
        _need(out.shape == shape and out.dtype == dtype, "out: as x")
    else:
        out = _like(x)
    plan, n = _norm_plan(shape, dtype, groups, act, eps, x.stride(), out.stride())
    _floats("gamma", gamma, shape[3])
    _floats("beta", beta, shape[3])
    d = B.mdcnn_group_norm_desc.from_buffer_copy(plan)
    d.gamma_dev, d.beta_dev = _ptr(gamma), _ptr(beta)
    mean = torch.empty((shape[0], groups), dtype=torch.float32, device=dev)
    rstd = torch.empty_like(mean)
    work = torch.empty(n, dtype=torch.uint8, device=dev) if n else None
    _call(B.mdcnn_group_norm, dev, d, x.data_ptr(), out.data_ptr(), mean.data_ptr(), rstd.data_ptr(), _ptr(work), n)
    if given:
        _written(out)
    return out, mean, rstd


def group_norm_backward(x, dy, mean, rstd, groups, gamma=None, beta=None, act="none"):
    """Gradients (dx, dgamma, dbeta) of group_norm from the gradient dy of y and the statistics it returned."""
    dev, shape, dtype = x.device, x.shape, x.dtype
    if not _on(dev, dy, mean, rstd, gamma, beta):
        _refuse_devices(dev, dy=dy, mean=mean, rstd=rstd, gamma=gamma, beta=beta)
    if _recorded(x, dy, mean, rstd, gamma, beta):
        _refuse_gradients("group_norm_backward", "")
    _need(dy.shape == shape and dy.dtype == dtype, "dy: as x")
    dx = _like(x)
    plan, n = _norm_plan(shape, dtype, groups, act, 0.0, x.stride(), dx.stride(), dy.stride(), True)
    _floats("gamma", gamma, shape[3])
    _floats("beta", beta, shape[3])
    _floats("mean", mean, shape[0] * groups)
    _floats("rstd", rstd, shape[0] * groups)
    d = B.mdcnn_group_norm_desc.from_buffer_copy(plan)
    d.gamma_dev, d.beta_dev = _ptr(gamma), _ptr(beta)
    dgamma = torch.empty(shape[3], dtype=torch.float32, device=dev)
    dbeta = torch.empty_like(dgamma)
    work = torch.empty(n, dtype=torch.uint8, device=dev) if n else None
    _call(B.mdcnn_group_norm_backward, dev, d, x.data_ptr(), dy.data_ptr(), mean.data_ptr(), rstd.data_ptr(), dx.data_ptr(), dgamma.data_ptr(), dbeta.data_ptr(), _ptr(work), n)
    return dx, dgamma, dbeta


class _GroupNormAct(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, groups, gamma, beta, eps, act):
        y, mean, rstd = group_norm(x, groups, gamma, beta, eps, act)
        ctx.save_for_backward(x, gamma, beta, mean, rstd)
        ctx.how = groups, act
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, gamma, beta, mean, rstd = ctx.saved_tensors
        groups, act = ctx.how
        if not _beside(dy.shape, dy.stride()):
            dy = dy.contiguous()
        dx, dgamma, dbeta = group_norm_backward(x, dy, mean, rstd, groups, gamma, beta, act)
        return dx, None, None if gamma is None else dgamma.view_as(gamma), None if beta is None else dbeta.view_as(beta), None, None


def group_norm_act(x, groups, gamma=None, beta=None, eps=1e-5, act="none"):
    """y of group_norm for autograd: gradients of x, gamma and beta (which may have any shape of C values); not differentiable twice."""
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


@functools.lru_cache(_PLANS)
def _heads_plan(name, like, x_shape, x_stride, y_shape, y_stride):
    _need(len(x_shape) == 3 and x_shape[0] == like[0] and x_shape[2] == like[2] and _beside(x_shape, x_stride), f"{name}: [{like[0]}, heads, {like[2]}], channels side by side")
    _need(y_shape == x_shape and _beside(y_shape, y_stride), f"the output of {name}: of its shape, channels side by side")
    return B.mdcnn_heads(None, None, x_shape[1], x_stride[0], x_stride[1], y_stride[0], y_stride[1])


def _heads(name, x, y, like):
    h = B.mdcnn_heads.from_buffer_copy(_heads_plan(name, like, x.shape, x.stride(), y.shape, y.stride()))
    h.x_dev, h.y_dev = x.data_ptr(), y.data_ptr()
    return h


def rotary(maps, positions, steps, axes=1, interleaved=False, magnitude=1.0, inverse=False, out=None):
    """Turns the first 2 * len(steps) channels of every head of one or two maps [tokens, heads, dim] (queries and keys; any strides, channels side by
    side) by positions [tokens] or [tokens, axes] int32; the others are copied.  Returns new tensors, or `out` (which may be `maps`
    themselves).  inverse=True turns back by the same angles, times magnitude: the gradient."""
    first = maps[0]
    shape, dev, dtype = first.shape, first.device, first.dtype
    _need(1 <= len(maps) <= 2 and (out is None or len(out) == len(maps)), "maps: one or two, out: as many")
    given = out is not None
    out = list(out) if given else [_like(m) for m in maps]
    if not _on(dev, positions, steps, *maps, *out):
        _refuse_devices(dev, positions=positions, steps=steps, **{f"maps[{i}]": m for i, m in enumerate(maps)}, **{f"out[{i}]": m for i, m in enumerate(out)})
    if _recorded(*maps, *out):
        _refuse_gradients("rotary", "use rotary_turn, ")
    _need(dtype in _DTYPE and all([m.dtype == dtype for m in (*maps, *out)]), "maps and out: float32, float16 or bfloat16, all of one type")
    hs = [_heads("the first map" if i == 0 else "the second map", x, y, shape) for i, (x, y) in enumerate(zip(maps, out))]
    _need(positions.dtype == torch.int32 and positions.is_contiguous() and positions.numel() == shape[0] * axes, f"positions: {shape[0]} x {axes} contiguous int32 values")
    _need(steps.dtype == torch.int64 and steps.dim() == 1 and steps.is_contiguous(), "steps: contiguous int64 values of rotary_steps")
    _call(B.mdcnn_rotary, dev, hs, shape[0], shape[2], _DTYPE[dtype], positions.data_ptr(), axes, steps.data_ptr(), 2 * steps.numel(), interleaved, inverse, magnitude)
    if given:
        _written(*out)
    return out


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, positions, steps, axes, interleaved, magnitude, *maps):
        ctx.save_for_backward(positions, steps)
        ctx.how = axes, interleaved, magnitude
        return tuple(rotary(maps, positions, steps, axes, interleaved, magnitude))

    @staticmethod
    @once_differentiable
    def backward(ctx, *grads):
        positions, steps = ctx.saved_tensors
        axes, interleaved, magnitude = ctx.how
        grads = [g if _beside(g.shape, g.stride()) else g.contiguous() for g in grads]
        return (None, None, None, None, None, *rotary(grads, positions, steps, axes, interleaved, magnitude, inverse=True))


def rotary_turn(maps, positions, steps, axes=1, interleaved=False, magnitude=1.0):
    """`rotary` for autograd: gradients of the maps; not differentiable twice."""
    return list(_Rotary.apply(positions, steps, axes, interleaved, magnitude, *maps))


# -- the cache --------------------------------------------------------------------------------------------------------------
def _per_sequence(name, t, n):
    _need(t.dtype == torch.int32 and t.is_contiguous() and t.numel() == n, f"{name}: {n} contiguous int32 values")


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
        _refuse_devices(dev, v=v, k_scale=k_scale, v_scale=v_scale)
        self.k, self.v, self.k_scale, self.v_scale, self.dim, self.heads, self.device = k, v, k_scale, v_scale, int(dim), heads, dev
        self._plan = B.mdcnn_cache_desc(pages, heads, int(dim), k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), None, 0, 0)

    @classmethod
    def empty(cls, pages, heads, dim, device="cuda:0"):
        pitch = B.mdcnn_cache_pitch(dim)
        _need(pitch > 0, "dim: a multiple of 8 from 8 to 256")
        codes = torch.empty((2, pages, heads, 64 * pitch), dtype=torch.int8, device=device)
        scales = torch.empty((2, pages, heads), dtype=torch.float32, device=device)
        return cls(codes[0].view(pages, heads, 64, pitch), codes[1].view(pages, heads, pitch, 64), scales[0], scales[1], dim)

    def _cache(self, table):
        _need(table.dtype == torch.int32 and table.dim() == 2 and table.is_contiguous(), "table: contiguous int32 [sequences, max_pages]")
        c = B.mdcnn_cache_desc.from_buffer_copy(self._plan)
        c.table_dev = table.data_ptr()
        c.n_seq, c.max_pages = table.shape
        return c

    def store(self, k, v, table, starts, held, max_new):
        """Puts new tokens [tokens, heads, dim] into their pages: sequence s has tokens starts[s] .. starts[s + 1] - 1, which follow the held[s]
        that it has already.  max_new: no sequence has more new tokens."""
        dev, shape = self.device, k.shape
        if not _on(dev, k, v, table, starts, held):
            _refuse_devices(dev, k=k, v=v, table=table, starts=starts, held=held)
        if _recorded(k, v):
            _refuse_gradients("store", "")
        _need(k.dtype == v.dtype and k.dtype in _DTYPE and v.shape == shape and len(shape) == 3 and shape[1:] == (self.heads, self.dim),
              f"k, v: [tokens, {self.heads}, {self.dim}] float32, float16 or bfloat16, of one type")
        c = self._cache(table)
        _per_sequence("starts", starts, c.n_seq + 1)
        _per_sequence("held", held, c.n_seq)
        _call(B.mdcnn_cache_store, dev, c, _heads("k", k, k, shape), _heads("v", v, v, shape), shape[0], starts.data_ptr(), held.data_ptr(), max_new, _DTYPE[k.dtype])
        _written(self.k, self.v, self.k_scale, self.v_scale)

    def read(self, table, starts, first, max_new, tokens, dtype):
        """The values of tokens first[s] .. of every sequence s, starts[s + 1] - starts[s] of them, as (k, v) [tokens, heads, dim]; tokens = starts[-1]."""
        dev = self.device
        if not _on(dev, table, starts, first):
            _refuse_devices(dev, table=table, starts=starts, first=first)
        _need(dtype in _DTYPE, "dtype: float32, float16 or bfloat16")
        c = self._cache(table)
        _per_sequence("starts", starts, c.n_seq + 1)
        _per_sequence("first", first, c.n_seq)
        k = torch.empty((tokens, self.heads, self.dim), dtype=dtype, device=dev)
        v = torch.empty_like(k)
        _call(B.mdcnn_cache_read, dev, c, _heads("k", k, k, k.shape), _heads("v", v, v, k.shape), tokens, starts.data_ptr(), first.data_ptr(), max_new, _DTYPE[dtype])
        return k, v

    def attend(self, q, table, starts, lengths, max_new, max_len, scale=None, causal=False, window=0, mask=None, out=None):
        """Attention of queries [tokens, q_heads, dim] (q_heads a multiple of heads) over the cache: sequence s has the queries starts[s] ..
        starts[s + 1] - 1 and lengths[s] tokens in the cache; max_new and max_len are bounds on both.  scale: of the logits, dim ** -0.5 if not given.
        causal: the queries are the last tokens of their sequence and see nothing behind themselves, with window > 0 only the `window`
        tokens up to themselves.  mask: uint8 or bool [sequences, >= max_len], zero: token hidden.  Returns (out, lse): [tokens, q_heads,
        dim] in the type of q and the natural logarithms of the sums [tokens, q_heads] in float32; zeros and -inf where a query sees nothing."""
        dev, shape = self.device, q.shape
        if not _on(dev, q, table, starts, lengths, mask, out):
            _refuse_devices(dev, q=q, table=table, starts=starts, lengths=lengths, mask=mask, out=out)
        if _recorded(q, out):
            _refuse_gradients("attend", "")
        _need(q.dtype in _DTYPE and len(shape) == 3 and shape[2] == self.dim, f"q: [tokens, q_heads, {self.dim}] float32, float16 or bfloat16")
        given = out is not None
        if given:
            _need(out.shape == shape and out.dtype == q.dtype, "out: as q")
        else:
            out = _like(q)
        c = self._cache(table)
        _per_sequence("starts", starts, c.n_seq + 1)
        _per_sequence("lengths", lengths, c.n_seq)
        how = B.mdcnn_attend_desc(starts.data_ptr(), lengths.data_ptr(), shape[0], max_new, max_len, self.dim ** -0.5 if scale is None else scale, causal, window)
        if mask is not None:
            _need(mask.dtype in (torch.uint8, torch.bool) and mask.dim() == 2 and mask.shape[0] == c.n_seq and mask.shape[1] >= max_len and mask.stride(1) == 1 and mask.stride(0) >= max_len,
                  f"mask: uint8 or bool [{c.n_seq}, {max_len} or more]")
            how.mask_dev, how.mask_row = mask.data_ptr(), mask.stride(0)
        n = B.mdcnn_cache_attend_bytes(c, how, shape[1], _DTYPE[q.dtype])
        work = torch.empty(n, dtype=torch.uint8, device=dev) if n else None
        lse = torch.empty(shape[:2], dtype=torch.float32, device=dev)
        _call(B.mdcnn_cache_attend, dev, c, how, _heads("q", q, out, shape), _DTYPE[q.dtype], lse.data_ptr(), _ptr(work), n)
        if given:
            _written(out)
        return out, lse
