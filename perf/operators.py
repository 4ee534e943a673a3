"""Cases of the operators that read a memory of past frames (or a prompt) behind the feature maps of a network.

A case names one of four operators and its sizes:

  norm    group norm with an activation on a map [N, H, W, C]; `train`: with its gradients
  rotary  rotary positions of queries and keys, both slices of one projection; `train`: with the gradient (the transposed turn)
  cache   keys and values of new tokens put into pages of 8-bit codes with a scale per page and head; the pages they went to,
          read back as values
  attend  attention of queries over such pages: one query per sequence, the pixels of a frame, or a prompt

`run` computes them either in their plain form (`own` false: elementary torch operations in 32 bits) or through the calls of
`paper_2210_09887_amd.ops` (`own` true).  A page holds 64 tokens; keys lie [page, head, token, channel], values [page, head,
channel, token], channels padded to the next of 32, 64, 96, 128, 192, 256.
"""
from __future__ import annotations

import math
import random

import torch

own = False

PAGE = 64
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def _norm(name, N, H, W, C, groups, dtype, act="silu", train=False, crop=False):
    return dict({"name": name} if name else {}, op="norm", N=N, H=H, W=W, C=C, groups=groups, dtype=dtype, act=act, train=train, crop=crop)


def _rotary(name, tokens, heads, kv_heads, dim, turned, dtype, axes=1, interleaved=False, factor=1.0, far=4096, train=False):
    return dict({"name": name} if name else {}, op="rotary", tokens=tokens, heads=heads, kv_heads=kv_heads, dim=dim, turned=turned, dtype=dtype, axes=axes,
                interleaved=interleaved, factor=factor, far=far, train=train)


def _cache(name, seqs, new_lo, new_hi, held_lo, held_hi, kv_heads, dim, dtype):
    return dict({"name": name} if name else {}, op="cache", seqs=seqs, new_lo=new_lo, new_hi=new_hi, held_lo=held_lo, held_hi=held_hi, kv_heads=kv_heads, dim=dim, dtype=dtype)


def _attend(name, seqs, new_lo, new_hi, len_lo, len_hi, heads, kv_heads, dim, dtype, causal=True, window=0, masked=False):
    return dict({"name": name} if name else {}, op="attend", seqs=seqs, new_lo=new_lo, new_hi=new_hi, len_lo=len_lo, len_hi=len_hi, heads=heads, kv_heads=kv_heads, dim=dim,
                dtype=dtype, causal=causal, window=window, masked=masked)


def listed():
    return [
        # the lowest branch of the pose network behind a camera, 384 x 288 / 32: a map so small that the call itself counts
        _norm("norm_low_branch", 1, 12, 9, 256, 32, "f16"),
        # training on feature maps of no round size (296 x 424 / 8) in fp32, three channels to a group
        _norm("norm_train_ragged", 3, 37, 53, 96, 32, "f32", train=True),
        # training on a batch of maps at a quarter of 512 x 512, bf16: the whole of it is memory traffic
        _norm("norm_train_batch", 16, 128, 128, 256, 32, "bf16", train=True),
        # one new token for each of 48 sequences
        _rotary("rotary_step", 48, 32, 8, 128, 128, "bf16", far=16384),
        # training on the pixels of eight frames of 48 x 36, turned by row, column and frame; frames further apart than in training
        _rotary("rotary_frames_train", 13824, 8, 8, 32, 24, "f32", axes=3, interleaved=True, factor=4.0, far=65536, train=True),
        # one new token for each of 48 sequences goes into pages that are mostly begun
        _cache("cache_step", 48, 1, 1, 0, 16383, 8, 128, "bf16"),
        # prompts of 300 to 6000 tokens, some behind a beginning that the cache holds already
        _cache("cache_prompts", 4, 300, 6000, 0, 2000, 8, 128, "f16"),
        # one token of one short sequence, fp32: latency
        _attend("attend_one", 1, 1, 1, 700, 700, 8, 2, 64, "f32"),
        # one token for each of 48 sequences of 1 to 16384 tokens, four query heads to a head of the cache
        _attend("attend_step", 48, 1, 1, 1, 16384, 32, 8, 128, "bf16"),
        # one token for each of two very long sequences
        _attend("attend_long", 2, 1, 1, 150001, 150001, 16, 2, 128, "f16"),
        # the 48 x 36 pixels of a frame of two videos read the eight frames before it, but for the pixels that left the view
        _attend("attend_frame", 2, 1728, 1728, 13824, 13824, 8, 8, 32, "f16", causal=False, masked=True),
        # the next piece of prompts, behind what the cache holds of them
        _attend("attend_prompts", 3, 900, 4096, 1800, 8192, 32, 8, 128, "bf16"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(["norm", "norm", "rotary", "cache", "attend", "attend", "attend"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if op == "norm":
        groups = rng.choice([1, 4, 8, 16, 32])
        C = groups * _log(rng, 1 if groups > 4 else 8, 32 if groups < 32 else 16)
        H, W = _log(rng, 5, 200), _log(rng, 5, 200)
        N = max(1, min(_log(rng, 1, 32), 67_000_000 // (H * W * C)))
        return _norm(None, N, H, W, C, groups, dtype, rng.choice(["none", "relu", "silu"]), rng.random() < 0.5, rng.random() < 0.3)
    dim = rng.choice([32, 40, 64, 64, 80, 96, 128, 128, 128, 192, 256])
    if op == "rotary":
        axes = rng.choice([1, 1, 2, 3])
        kv = rng.choice([1, 2, 4, 8])
        turned = 2 * axes * max(1, round(dim * rng.choice([0.25, 0.5, 1.0, 1.0]) / (2 * axes)))
        turned -= 2 * axes if turned > dim else 0
        heads = kv * rng.choice([1, 2, 4])
        tokens = _log(rng, 1, max(1, min(60000, 60_000_000 // (dim * (heads + kv)))))
        return _rotary(None, tokens, heads, kv, dim, turned, dtype, axes, rng.random() < 0.5, rng.choice([1.0, 1.0, 4.0, 16.0]), _log(rng, 64, 1 << 20), rng.random() < 0.5)
    kv = rng.choice([1, 2, 3, 4, 8])
    if op == "cache":
        seqs = _log(rng, 1, 64)
        hi = _log(rng, 1, max(1, min(8000, 24_000_000 // (seqs * kv * dim))))
        held = _log(rng, 1, max(1, min(16000, 100_000_000 // (seqs * kv * dim))))
        return _cache(None, seqs, rng.randint(1, hi), hi, 0, held, kv, dim, dtype)
    heads = kv * rng.choice([1, 1, 2, 3, 4, 7, 8])
    way = rng.choice(["step", "step", "few", "prompt", "frame"])
    if way in ("step", "few"):
        seqs = _log(rng, 1, 64)
        longest = _log(rng, 2, max(2, min(150000, 150_000_000 // (seqs * kv * dim))))
        new = 1 if way == "step" else rng.randint(2, 8)
        return _attend(None, seqs, 1, new, rng.randint(1, longest), longest, heads, kv, dim, dtype, window=rng.choice([0, 0, 0, rng.randint(1, longest)]))
    seqs = rng.randint(1, 4)
    pairs = min(3_200_000_000, int(4e11 / dim)) // (heads * seqs)
    new = _log(rng, 20, min(4096, math.isqrt(pairs)))
    most = max(new, min(16384, pairs // new, 20_000_000 // (seqs * kv * dim)))
    longest = _log(rng, new, most)
    return _attend(None, seqs, rng.randint(1, new), new, rng.randint(new, longest), longest, heads, kv, dim, dtype, causal=way == "prompt",
                   window=rng.choice([0, 0, rng.randint(1, longest)]) if way == "prompt" else 0, masked=way == "frame")


def _spread(n, lo, hi):
    """n whole numbers from lo to hi, evenly apart in their logarithm."""
    return [round((lo + 1) * ((hi + 1) / (lo + 1)) ** ((i + 1) / n if n == 1 else i / (n - 1))) - 1 for i in range(n)]


def _pitch(dim):
    return next(p for p in (32, 64, 96, 128, 192, 256) if p >= dim)


def _attend_sizes(case):
    new = _spread(case["seqs"], case["new_lo"], case["new_hi"])
    return new, [max(a, b) for a, b in zip(new, _spread(case["seqs"], case["len_lo"], case["len_hi"]))]


def _starts(counts):
    return torch.tensor([0] + counts, dtype=torch.int32).cumsum(0, dtype=torch.int32).cuda()


# -- what a program has in hand ------------------------------------------------------------------------------------------
def _pages(case, g, r, lengths):
    """Pages of the sequences in no order, with a few to spare: codes as normal values give them, scales that differ from page to page."""
    pages = [-(-n // PAGE) for n in lengths]
    total, most, kv, pitch = sum(pages) + 3, max(1, max(pages)), case["kv_heads"], _pitch(case["dim"])
    ids = list(range(total))
    r.shuffle(ids)
    table = torch.full((len(lengths), most), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = torch.tensor(ids[at:at + n], dtype=torch.int32)
        at += n

    def codes(*shape):
        return (torch.randn(shape, device="cuda", generator=g, dtype=torch.float16) * 40).round_().clamp_(-127, 127).to(torch.int8)

    def scales():
        return torch.exp(0.3 * torch.randn((total, kv), device="cuda", generator=g)) / 40

    return dict(k=codes(total, kv, PAGE, pitch), v=codes(total, kv, pitch, PAGE), k_scale=scales(), v_scale=scales(), table=table.cuda())


def prepare(case, seed):
    r = random.Random(seed)
    g = torch.Generator(device="cuda").manual_seed(r.randrange(1 << 31))
    dt = TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=g)

    s = {"case": case}
    if case["op"] == "norm":
        N, H, W, C = (case[k] for k in "NHWC")
        big = (N, H + 3, W + 5, C) if case["crop"] else (N, H, W, C)              # a crop of a larger map keeps its strides
        s["x"] = (normal(*big) * (0.5 + torch.rand(C, device="cuda", generator=g)) + normal(C)).to(dt)[:, big[1] - H:, big[2] - W:]
        s["gamma"], s["beta"] = 1 + 0.2 * normal(C), 0.2 * normal(C)
        s["dy"] = normal(N, H, W, C).to(dt) if case["train"] else None
    elif case["op"] == "rotary":
        T, h, k, D = case["tokens"], case["heads"], case["kv_heads"], case["dim"]
        both = normal(T, (h + k) * D).to(dt)
        s["q"], s["k"] = both[:, :h * D].view(T, h, D), both[:, h * D:].view(T, k, D)
        s["pos"] = torch.randint(-case["far"] // 8 if case["axes"] > 1 else 0, case["far"], (T, case["axes"]), device="cuda", generator=g, dtype=torch.int32)
        s["steps"] = torch.tensor([_step(f) for f in _frequencies(case)], dtype=torch.int64).cuda()
        s["dq"], s["dk"] = (normal(T, h, D).to(dt), normal(T, k, D).to(dt)) if case["train"] else (None, None)
    elif case["op"] == "cache":
        B, kv, D = case["seqs"], case["kv_heads"], case["dim"]
        new, held = _spread(B, case["new_lo"], case["new_hi"]), _spread(B, case["held_lo"], case["held_hi"])
        r.shuffle(new)
        r.shuffle(held)
        s.update(_pages(case, g, r, [a + b for a, b in zip(new, held)]))
        T = sum(new)
        both = (normal(T, 2 * kv * D) * (0.5 + torch.rand(2 * kv * D, device="cuda", generator=g))).to(dt)
        s["new_k"], s["new_v"] = both[:, :kv * D].view(T, kv, D), both[:, kv * D:].view(T, kv, D)
        s["starts"], s["held"], s["max_new"] = _starts(new), torch.tensor(held, dtype=torch.int32).cuda(), max(new)
        first = [n // PAGE * PAGE for n in held]                                  # the pages that get tokens, from their first token on
        back = [a + b - c for a, b, c in zip(held, new, first)]
        s["back_starts"], s["back_first"], s["back_max"], s["back"] = _starts(back), torch.tensor(first, dtype=torch.int32).cuda(), max(back), sum(back)
    else:
        B = case["seqs"]
        new, lengths = _attend_sizes(case)
        order = list(range(B))
        r.shuffle(order)
        new, lengths = [new[i] for i in order], [lengths[i] for i in order]
        s.update(_pages(case, g, r, lengths))
        s["q"] = (1.5 * normal(sum(new), case["heads"], case["dim"])).to(dt)
        s["starts"], s["lengths"] = _starts(new), torch.tensor(lengths, dtype=torch.int32).cuda()
        s["max_new"], s["max_len"] = max(new), max(lengths)
        s["mask"] = None
        if case["masked"]:                                                        # runs of pixels that are out of view
            m = torch.rand((B, -(-max(lengths) // 37)), device="cuda", generator=g) < 0.7
            s["mask"] = m.repeat_interleave(37, 1)[:, :max(lengths)].to(torch.uint8).contiguous()
    return s


def _step(frequency):
    """Radians per position as a fraction of a turn in 64 bits (wraps like the turn does)."""
    n = int(round(frequency / (2 * math.pi) * 2.0 ** 64)) % (1 << 64)
    return n - (1 << 64) if n >= 1 << 63 else n


def _frequencies(case):
    """Of the turned pairs, axis by axis: base 10000, slow turns stretched by `factor` (by how often they turn within 4096 positions: less than once
    by the whole factor, more than 32 times not at all)."""
    n = case["turned"] // 2 // case["axes"]

    def one(i):
        f = 10000.0 ** (-i / n)
        keep = min(1.0, max(0.0, (4096 * f / (2 * math.pi) - 1) / 31))
        return f * keep + f / case["factor"] * (1 - keep)

    return [one(i) for _ in range(case["axes"]) for i in range(n)]


def _magnitude(case):
    return 0.1 * math.log(case["factor"]) + 1.0


# -- one pass ----------------------------------------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2210_09887_amd import ops
    c = s["case"]
    if c["op"] == "norm":
        y, mean, rstd = ops.group_norm(s["x"], c["groups"], s["gamma"], s["beta"], 1e-5, c["act"])
        if not c["train"]:
            return y, mean, rstd
        return (y, mean, rstd, *ops.group_norm_backward(s["x"], s["dy"], mean, rstd, c["groups"], s["gamma"], s["beta"], c["act"]))
    if c["op"] == "rotary":
        kw = dict(axes=c["axes"], interleaved=c["interleaved"], magnitude=_magnitude(c))
        out = ops.rotary((s["q"], s["k"]), s["pos"], s["steps"], **kw)
        if not c["train"]:
            return out
        return (*out, *ops.rotary((s["dq"], s["dk"]), s["pos"], s["steps"], inverse=True, **kw))
    if "handle" not in s:                                                         # a program keeps it as long as the pages
        s["handle"] = ops.GpuCache(s["k"], s["v"], s["k_scale"], s["v_scale"], c["dim"])
    if c["op"] == "cache":
        s["handle"].store(s["new_k"], s["new_v"], s["table"], s["starts"], s["held"], s["max_new"])
        return s["handle"].read(s["table"], s["back_starts"], s["back_first"], s["back_max"], s["back"], TYPES[c["dtype"]])
    return s["handle"].attend(s["q"], s["table"], s["starts"], s["lengths"], s["max_new"], s["max_len"], causal=c["causal"], window=c["window"], mask=s["mask"])


def _run_plain(s):
    c = s["case"]
    return {"norm": _plain_norm, "rotary": _plain_rotary, "cache": _plain_cache, "attend": _plain_attend}[c["op"]](s, c, TYPES[c["dtype"]])


def _plain_norm(s, c, dt):
    N, P, G = c["N"], c["H"] * c["W"], c["groups"]
    shape = s["x"].shape
    x = s["x"].float().reshape(N, P, G, -1)
    mean = x.mean((1, 3), keepdim=True)
    d = x - mean
    rstd = torch.rsqrt((d * d).mean((1, 3), keepdim=True) + 1e-5)
    z = (d * rstd).reshape(N * P, -1)
    u = z * s["gamma"] + s["beta"]
    gate = torch.sigmoid(u) if c["act"] == "silu" else None
    y = u * gate if c["act"] == "silu" else u.clamp(min=0) if c["act"] == "relu" else u
    out = y.to(dt).reshape(shape), mean.reshape(N, G), rstd.reshape(N, G)
    if not c["train"]:
        return out
    du = s["dy"].float().reshape(N * P, -1)
    du = du * (gate * (1 + u * (1 - gate))) if c["act"] == "silu" else du * (u > 0) if c["act"] == "relu" else du
    dgamma, dbeta = (du * z).sum(0), du.sum(0)
    t = (du * s["gamma"]).reshape(N, P, G, -1)
    z = z.reshape(N, P, G, -1)
    dx = rstd * (t - t.mean((1, 3), keepdim=True) - z * (t * z).mean((1, 3), keepdim=True))
    return (*out, dx.to(dt).reshape(shape), dgamma, dbeta)


def _turned(x, cos, sin, c, dt):
    R = c["turned"]
    f = x[..., :R].float()
    a, b = (f[..., 0::2], f[..., 1::2]) if c["interleaved"] else (f[..., :R // 2], f[..., R // 2:])
    a, b = a * cos - b * sin, a * sin + b * cos
    f = torch.stack((a, b), -1).flatten(-2) if c["interleaved"] else torch.cat((a, b), -1)
    return torch.cat((f.to(dt), x[..., R:]), -1)


def _plain_rotary(s, c, dt):
    pos = s["pos"].long().repeat_interleave(c["turned"] // 2 // c["axes"], 1)
    angle = ((pos * s["steps"]) >> 32).float() * (2 * math.pi / 2 ** 32)
    cos, sin = torch.cos(angle)[:, None] * _magnitude(c), torch.sin(angle)[:, None] * _magnitude(c)
    out = _turned(s["q"], cos, sin, c, dt), _turned(s["k"], cos, sin, c, dt)
    if not c["train"]:
        return out
    return (*out, _turned(s["dq"], cos, -sin, c, dt), _turned(s["dk"], cos, -sin, c, dt))


def _where(starts, first, total):
    """Sequence and position of each of `total` tokens that lie one sequence behind the other."""
    i = torch.arange(total, device="cuda")
    b = torch.searchsorted(starts[1:].long(), i, right=True)
    return b, first[b].long() + i - starts[b]


def _plain_store(codes, scale, new, s, token_last):
    D = s["case"]["dim"]
    b, at = _where(s["starts"], s["held"], new.shape[0])
    page, slot = s["table"][b, at // PAGE].long(), at % PAGE
    x = new.float()
    need = torch.zeros_like(scale).index_reduce_(0, page, x.abs().amax(2), "amax") / 127
    grows = (s["held"] % PAGE > 0) & (s["starts"][1:] > s["starts"][:-1])        # the first page of a sequence's new tokens holds some already
    begun = s["table"].gather(1, (s["held"] // PAGE).long().clamp(max=s["table"].shape[1] - 1)[:, None])[:, 0].long().clamp(min=0)
    before = scale[begun]
    after = torch.where(need[begun] <= before, before, torch.maximum(need[begun], 1.25 * before))
    ratio = torch.where(after > 0, before / after, torch.zeros_like(after))
    kept = codes[begun]
    codes[begun] = torch.where(grows[:, None, None, None], torch.round(kept.float() * ratio[:, :, None, None]).to(torch.int8), kept)
    touched = torch.zeros(scale.shape[0], dtype=torch.bool, device="cuda").index_fill_(0, page, True)
    scale.copy_(torch.where(touched[:, None], need, scale))
    scale[begun] = torch.where(grows[:, None], after, scale[begun])
    by = scale[page][:, :, None]
    q = torch.where(by > 0, torch.round(x / by).clamp(-127, 127), torch.zeros_like(x)).to(torch.int8)
    if token_last:
        codes[page, :, :D, slot] = q
    else:
        codes[page, :, slot, :D] = q


def _plain_cache(s, c, dt):
    D = c["dim"]
    _plain_store(s["k"], s["k_scale"], s["new_k"], s, False)
    _plain_store(s["v"], s["v_scale"], s["new_v"], s, True)
    b, at = _where(s["back_starts"], s["back_first"], s["back"])
    page, slot = s["table"][b, at // PAGE].long(), at % PAGE
    k = s["k"][page, :, slot, :D].float() * s["k_scale"][page][:, :, None]
    v = s["v"][page, :, :D, slot].float() * s["v_scale"][page][:, :, None]
    return k.to(dt), v.to(dt)


def _plain_attend(s, c, dt):
    B, D, kv, g = c["seqs"], c["dim"], c["kv_heads"], c["heads"] // c["kv_heads"]
    n, L = s["max_new"], s["max_len"]
    ids = s["table"].long().clamp(min=0)
    k = (s["k"][ids].float() * s["k_scale"][ids][..., None, None]).permute(0, 2, 1, 3, 4).reshape(B * kv, -1, s["k"].shape[3])[:, :L, :D]
    v = (s["v"][ids].float() * s["v_scale"][ids][..., None, None]).permute(0, 2, 1, 4, 3).reshape(B * kv, -1, s["k"].shape[3])[:, :L, :D]
    starts, lengths = s["starts"].long(), s["lengths"].long()
    count = starts[1:] - starts[:-1]
    i, j = torch.arange(n, device="cuda"), torch.arange(L, device="cuda")
    row = (starts[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)
    q = s["q"].float()[row].reshape(B, n, kv, g, D).permute(0, 2, 1, 3, 4).reshape(B * kv, n * g, D)
    sees = (j < lengths[:, None])[:, None].expand(B, n, L)
    if c["causal"]:
        at = (lengths - count)[:, None] + i
        sees = sees & (j <= at[:, :, None])
        if c["window"]:
            sees = sees & (j > at[:, :, None] - c["window"])
    if s["mask"] is not None:
        sees = sees & (s["mask"] != 0)[:, None]
    score = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(D ** -0.5).view(B, kv, n, g, L)
    score.masked_fill_(~sees[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.bmm(p.view(B * kv, n * g, L), v.contiguous()).view(B, kv, n, g, D)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    lse = (top + total.log())[..., 0]
    live = i < count[:, None]
    return o.permute(0, 2, 1, 3, 4).reshape(B, n, kv * g, D)[live].to(dt), lse.permute(0, 2, 1, 3).reshape(B, n, kv * g)[live]


# -- work and exact values ----------------------------------------------------------------------------------------------
def work(case):
    e, op = SIZE[case["dtype"]], case["op"]
    if op == "norm":
        values = case["N"] * case["H"] * case["W"] * case["C"]
        return {"bytes": float(values * e * (5 if case["train"] else 2) + case["C"] * 8), "flops": float(values * (30 if case["train"] else 10))}
    if op == "rotary":
        values = case["tokens"] * (case["heads"] + case["kv_heads"]) * case["dim"] * (2 if case["train"] else 1)
        return {"bytes": float(2 * values * e + case["tokens"] * case["axes"] * 4), "flops": float(3 * values)}
    if op == "cache":
        new, held = _spread(case["seqs"], case["new_lo"], case["new_hi"]), _spread(case["seqs"], case["held_lo"], case["held_hi"])
        width = 2 * case["kv_heads"] * case["dim"]
        kept = sum(n % PAGE for n in held)
        return {"bytes": float(width * (sum(new) * (e + 1) + (sum(new) + kept) * (1 + e))), "flops": float(width * 4 * sum(new))}
    new, lengths = _attend_sizes(case)
    w = case["window"]

    def pairs(n, length):
        if not case["causal"]:
            return n * length
        return sum(max(0, min(length - n + i + 1, w or length)) for i in range(n))

    read = sum(min(length, w + n) if w else length for n, length in zip(new, lengths))
    seen = sum(pairs(n, length) for n, length in zip(new, lengths)) * (0.7 if case["masked"] else 1.0)
    width = case["heads"] * case["dim"]
    return {"bytes": float(2 * read * case["kv_heads"] * case["dim"] + 2 * sum(new) * width * e + 4 * sum(new) * case["heads"]), "flops": float(4 * width * seen)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "rotary": _exact_rotary, "cache": _exact_cache, "attend": _exact_attend}[case["op"]](s, case)


def _exact_norm(s, c):
    N, H, W, C, G = c["N"], c["H"], c["W"], c["C"], c["groups"]
    gamma, beta = s["gamma"].double(), s["beta"].double()
    mean = torch.stack([m.double().mean((0, 1)).view(G, -1).mean(1) for m in s["x"]])
    wide = mean.repeat_interleave(C // G, 1)[:, None, None]
    rstd = torch.stack([((m.double() - a) ** 2).mean((0, 1)).view(G, -1).mean(1) for m, a in zip(s["x"], wide)]).add(1e-5).rsqrt()
    z = (s["x"].double() - wide) * rstd.repeat_interleave(C // G, 1)[:, None, None]
    u = z * gamma + beta
    if c["act"] == "silu":
        y, slope = u / (1 + torch.exp(-u)), (1 + torch.exp(-u) * (1 + u)) / (1 + torch.exp(-u)) ** 2
    elif c["act"] == "relu":
        y, slope = u.clamp(min=0), (u > 0).double()
    else:
        y, slope = u, torch.ones_like(u)
    if not c["train"]:
        return y, mean, rstd
    du = s["dy"].double() * slope
    one = (du * gamma).sum((1, 2)).view(N, G, -1).sum(2) / (H * W * C // G)
    two = (du * gamma * z).sum((1, 2)).view(N, G, -1).sum(2) / (H * W * C // G)
    one, two, scale = (t.repeat_interleave(C // G, 1)[:, None, None] for t in (one, two, rstd))
    return y, mean, rstd, scale * (du * gamma - one - z * two), (du * z).sum((0, 1, 2)), du.sum((0, 1, 2))


def _exact_rotary(s, c):
    per, R = c["turned"] // 2 // c["axes"], c["turned"]
    f = torch.tensor(_frequencies(c), dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.full((1,), _magnitude(c), dtype=torch.float64, device="cuda"),
                       torch.cat([s["pos"][:, a:a + 1].double() * f[a * per:(a + 1) * per] for a in range(c["axes"])], 1))[:, None]

    def of(x, by):
        x = x.double()
        pair = torch.complex(x[..., 0:R:2], x[..., 1:R:2]) if c["interleaved"] else torch.complex(x[..., :R // 2], x[..., R // 2:R])
        pair = torch.view_as_real((pair * by).resolve_conj())
        return torch.cat((pair.flatten(-2) if c["interleaved"] else pair.transpose(-1, -2).flatten(-2), x[..., R:]), -1)

    out = of(s["q"], turn), of(s["k"], turn)
    return (*out, of(s["dq"], turn.conj()), of(s["dk"], turn.conj())) if c["train"] else out


def _exact_cache(s, c):
    """The state is codes and scales of 32 bits: quotients in 64 bits, scales rounded as they are held."""
    D = c["dim"]
    starts, held, first, table = s["starts"].tolist(), s["held"].tolist(), s["back_first"].tolist(), s["table"].tolist()
    got = []
    for codes, scales, new, last in ((s["k"], s["k_scale"], s["new_k"], False), (s["v"], s["v_scale"], s["new_v"], True)):
        out = []
        for b in range(c["seqs"]):
            x, n = new[starts[b]:starts[b + 1]].double(), held[b]
            ids = table[b][first[b] // PAGE:-(-(n + x.shape[0]) // PAGE)]
            for k, page in enumerate(ids):
                lo, hi = first[b] + k * PAGE, first[b] + (k + 1) * PAGE
                part = x[max(0, lo - n):max(0, hi - n)]
                scale = (part.abs().amax((0, 2)).float() / 127).double()
                if lo < n:
                    old = codes[page].double()[:, :D].transpose(1, 2) if last else codes[page].double()[:, :, :D]
                    old = old[:, :n - lo].transpose(0, 1)
                    was = scales[page].double()
                    scale = torch.where(scale <= was, was, torch.maximum(scale, (1.25 * was).float().double()))
                    old = torch.round((old * (was / scale).float().double()[:, None]).float()).double()
                    out.append(old * scale[:, None])
                out.append(torch.round(part / scale[:, None].clamp(min=1e-300)).clamp(-127, 127) * scale[:, None])
        got.append(torch.cat(out))
    return tuple(got)


def _exact_attend(s, c):
    D, kv, g = c["dim"], c["kv_heads"], c["heads"] // c["kv_heads"]
    starts, lengths = s["starts"].tolist(), s["lengths"].tolist()
    out = torch.zeros((starts[-1], c["heads"], D), dtype=torch.float64, device="cuda")
    lse = torch.full((starts[-1], c["heads"]), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(c["seqs"]):
        n, L = starts[b + 1] - starts[b], lengths[b]
        ids = s["table"][b, :-(-L // PAGE)].long()
        at = L - n + torch.arange(n, device="cuda")[:, None]
        j = torch.arange(L, device="cuda")[None]
        hidden = (j > at) if c["causal"] else torch.zeros((n, L), dtype=torch.bool, device="cuda")
        if c["window"]:
            hidden = hidden | (j <= at - c["window"])
        if s["mask"] is not None:
            hidden = hidden | (s["mask"][b, :L] == 0)[None]
        for h in range(kv):
            k = (s["k"][ids, h].double() * s["k_scale"][ids, h].double()[:, None, None]).reshape(-1, s["k"].shape[3])[:L, :D]
            v = (s["v"][ids, h].double() * s["v_scale"][ids, h].double()[:, None, None]).transpose(1, 2).reshape(-1, s["k"].shape[3])[:L, :D]
            for m in range(h * g, (h + 1) * g):
                a = (s["q"][starts[b]:starts[b + 1], m].double() @ k.T) / math.sqrt(D)
                a[hidden] = -math.inf
                lse[starts[b]:starts[b + 1], m] = torch.logsumexp(a, 1)
                w = torch.exp(a - lse[starts[b]:starts[b + 1], m][:, None])
                out[starts[b]:starts[b + 1], m] = torch.nan_to_num(w) @ v
    return out, lse
