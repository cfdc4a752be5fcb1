"""Timed cases of the operators that take decoded images into a sequence model: pixels to patch tokens, the positions of
those tokens on several axes (time, height, width), and the queries and keys that carry the positions.

  patches      tokens of the images of a decoded record: each image's rectangle resampled to whole patches, normalised,
               laid out patch after patch (in blocks of merge x merge patches)
  positions    positions of packed sequences of text and image or clip grids, and where each sequence goes on
  rotate       queries and keys rotated by the angles of their tokens' positions; `inverse` is the gradient's direction
  norm         the same behind a root-mean-square norm of every head, in one pass
  norm_grad    its backward pass: gradients of queries, keys and both norms' weights

A case names an operator, its sizes and types:

  n, shape, patch, merge, crop   images, their sizes (the benchmark's workloads: imagenet, celeba, ham), pixels of a
                                 patch's side, patches of a block's side, whether they are cropped and mirrored
  seqs, segs, clips              sequences, segments in each, whether grids have several frames
  b, s, hq, hk, dim, rot         sequences, tokens, heads of queries and keys, their size, how much of it is rotated
  pairs                          half: (i, i + rot / 2); next: (2 i, 2 i + 1)
  axes                           which axis turns pair i: runs (sections of 1/4, 3/8, 3/8), turns (i mod 3), two (rows and
                                 columns, each with the whole range of frequencies), one (plain positions)
  packed                         queries and keys are slices of one projection's output
  far                            positions reach up to this
"""
from __future__ import annotations

import math
import random

import torch

own = False

MEAN, STD = (0.485, 0.456, 0.406), (0.229, 0.224, 0.225)
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"f16": 2, "bf16": 2, "f32": 4}
EPS = 1e-6
DEVICE = "cuda:0"


def _patches(name, n, shape, patch, merge, crop, dtype):
    return {"name": name, "op": "patches", "n": n, "shape": shape, "patch": patch, "merge": merge, "crop": crop, "dtype": dtype}


def _positions(name, seqs, segs, clips):
    return {"name": name, "op": "positions", "seqs": seqs, "segs": segs, "clips": clips}


def _heads(name, op, b, s, hq, hk, dim, rot, pairs, axes, dtype, packed=False, inverse=False, far=32768):
    return {"name": name, "op": op, "b": b, "s": s, "hq": hq, "hk": hk, "dim": dim, "rot": rot, "pairs": pairs, "axes": axes,
            "dtype": dtype, "packed": packed, "inverse": inverse, "far": far}


def listed():
    return [
        # one request's few images: launch latency
        _patches("patches_4_celeba", 4, "celeba", 14, 2, False, "bf16"),
        # a whole ImageNet-shaped record at native resolution, the benchmark's 1024 images; the largest of its kind
        _patches("patches_1024_imagenet", 1024, "imagenet", 14, 2, False, "bf16"),
        # random-resized crops and flips of large images, another patch size, single precision
        _patches("patches_96_ham_crop_f32", 96, "ham", 16, 1, True, "f32"),
        # a prompt of some images and the text between them
        _positions("positions_8", 8, 9, False),
        # a long training batch of packed sequences with images and clips
        _positions("positions_512_clips", 512, 17, True),
        # one new token of each running request, grouped heads, far positions
        _heads("rotate_single_64", "rotate", 64, 1, 32, 8, 128, 128, "half", "runs", "bf16", far=1_000_000),
        # a prompt of odd length, rotated in the other pairing, out of one projection's output
        _heads("rotate_prompt_8191", "rotate", 1, 8191, 32, 8, 128, 128, "next", "turns", "f16", packed=True),
        # the gradient of an image encoder's rotation: rows and columns, heads of 80, single precision
        _heads("rotate_inverse_f32", "rotate", 3, 4001, 16, 16, 80, 80, "half", "two", "f32", inverse=True, far=128),
        # one new token of each running request behind the norms
        _heads("norm_single_16", "norm", 16, 1, 32, 8, 128, 128, "half", "runs", "bf16", packed=True, far=262_144),
        # a long prompt with many images; the largest
        _heads("norm_prompt_32768", "norm", 1, 32768, 32, 8, 128, 128, "half", "runs", "bf16", packed=True, far=262_144),
        # a short training sequence, heads partly rotated, single precision
        _heads("norm_grad_257_f32", "norm_grad", 2, 257, 12, 4, 64, 32, "next", "one", "f32"),
        # an image encoder's training step: packed images, heads of 72, rows and columns
        _heads("norm_grad_16384", "norm_grad", 1, 16384, 16, 16, 72, 72, "half", "two", "bf16", far=128),
    ]


def draw(rng: random.Random):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["patches", "positions", "rotate", "norm", "norm", "norm_grad", "norm_grad"])
    if op == "patches":
        shape = rng.choice(["imagenet", "celeba", "ham"])
        c = _patches("", spread(1, 256 if shape == "ham" else 768), shape, rng.choice([8, 14, 14, 16, 16, 28, 32]), rng.choice([1, 1, 2, 2, 3]),
                     rng.random() < 0.5, rng.choice(["f16", "bf16", "bf16", "f32"]))
    elif op == "positions":
        c = _positions("", spread(1, 512), spread(4, 17), rng.random() < 0.5)
    else:
        dim = rng.choice([32, 48, 64, 64, 72, 80, 96, 112, 128, 128, 192, 256])
        hk = rng.choice([1, 2, 4, 8, 8, 16])
        hq = hk * rng.choice([1, 1, 2, 3, 4, 8])
        dtype = rng.choice(["f16", "bf16", "bf16", "f32"])
        most = 32768 * 40 * 128 * 2 // (dim * (hq + hk) * BYTES[dtype] * (2 if op == "norm_grad" else 1))
        s = 1 if rng.random() < 0.25 else spread(2, min(65536, most))
        b = spread(1, max(1, min(256, most // s)))
        axes = rng.choice(["runs", "turns", "two", "one"])
        rot = dim if rng.random() < 0.7 else dim // 4 * 2
        c = _heads("", op, b, s, hq, hk, dim, rot, rng.choice(["half", "next"]), axes, dtype, packed=rng.random() < 0.5,
                   inverse=op == "rotate" and rng.random() < 0.5, far=spread(64, 1_000_000))
    del c["name"]
    return c


# ---- sizes that belong to a case --------------------------------------------------------------------------------------


def _images(case):
    """Per image: offset, width, height, x0, y0, w, h, rows, cols, flip."""
    rng = random.Random(1000 * case["n"] + case["patch"])
    unit, at, got = case["patch"] * case["merge"], 0, []
    for _ in range(case["n"]):
        if case["shape"] == "imagenet":
            W, H = (16 * int(round(rng.uniform(256, 500) / 16.0)) for _ in range(2))
        else:
            W, H = (178, 218) if case["shape"] == "celeba" else (600, 450)
        x0, y0, w, h, flip = 0, 0, W, H, 0
        if case["crop"]:
            w, h = (max(1, int(side * math.sqrt(rng.uniform(0.08, 1.0)))) for side in (W, H))
            x0, y0, flip = rng.randint(0, W - w), rng.randint(0, H - h), rng.randint(0, 1)
        rows, cols = (case["merge"] * max(1, int(round(side / unit))) for side in (h, w))
        got.append((at, W, H, x0, y0, w, h, rows, cols, flip))
        at += (3 * W * H + 127) // 128 * 128
    return got, at + 16


def _segments(case):
    """Rows of time (or tokens), height, width, sequence: text has no height and width."""
    rng = random.Random(100 * case["seqs"] + case["segs"])
    got = []
    for b in range(case["seqs"]):
        for j in range(case["segs"]):
            if j % 2 == 0:
                got.append((rng.randint(0, 120), 0, 0, b))
            else:
                got.append((rng.randint(2, 8) if case["clips"] and rng.random() < 0.3 else 1, rng.randint(4, 18), rng.randint(4, 18), b))
    return got


def _tokens(segment):
    t, h, w, _ = segment
    return t * h * w if h and w else t


def _turns(case):
    """(frequency, axis) of every pair."""
    half = case["rot"] // 2
    if case["axes"] == "two":
        each = (half + 1) // 2
        return [(10000.0 ** (-(i % each) / each), i // each) for i in range(half)]
    freq = [1_000_000.0 ** (-i / half) for i in range(half)]
    first, second = half // 4, half // 4 + half * 3 // 8
    axis = {"runs": lambda i: 0 if i < first else 1 if i < second else 2, "turns": lambda i: i % 3, "one": lambda i: 0}[case["axes"]]
    return [(f, axis(i)) for i, f in enumerate(freq)]


# ---- inputs -----------------------------------------------------------------------------------------------------------


class _State:
    pass


def prepare(case, seed):
    s = _State()
    s.case = case
    gen = torch.Generator(device=DEVICE).manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, device=DEVICE, generator=gen)

    if case["op"] == "patches":
        table, size = _images(case)
        s.images = torch.tensor(table, dtype=torch.int64, device=DEVICE)
        count = s.images[:, 7] * s.images[:, 8]
        image = torch.repeat_interleave(torch.arange(len(table), device=DEVICE), count)
        local = torch.arange(image.numel(), device=DEVICE) - (torch.cumsum(count, 0) - count)[image]
        s.index = torch.stack([image, local], 1).to(torch.int32)
        # smooth waves under noise, as photographs have
        wave = torch.arange(size, device=DEVICE, dtype=torch.float32).mul_(2 * math.pi / 911.0).add_(float(seed % 628) / 100).sin_()
        s.rgb = wave.mul_(50).add_(128).add_(randn(size).mul_(10)).clamp_(0, 255).to(torch.uint8)
        return s
    if case["op"] == "positions":
        rows = _segments(case)
        # texts and grids of the case, dealt to their places by the seed
        rng, kinds = random.Random(seed), {False: [r[:3] for r in rows if not r[1]], True: [r[:3] for r in rows if r[1]]}
        for kind in kinds.values():
            rng.shuffle(kind)
        rows = [(*kinds[h > 0].pop(), b) for _, h, _, b in rows]
        s.n_tokens, s.n_sequences = sum(map(_tokens, rows)), case["seqs"]
        s.rows, s.segments = rows, torch.tensor(rows, dtype=torch.int32, device=DEVICE)
        return s
    b, n, hq, hk, dim, dtype = case["b"], case["s"], case["hq"], case["hk"], case["dim"], DTYPES[case["dtype"]]
    if case["packed"]:
        qkv = randn(b, n, hq + 2 * hk, dim).mul_(1.5).to(dtype)
        s.q, s.k = qkv[:, :, :hq], qkv[:, :, hq:hq + hk]
    else:
        s.q, s.k = randn(b, n, hq, dim).mul_(1.5).to(dtype), randn(b, n, hk, dim).mul_(1.5).to(dtype)
    turns = _turns(case)
    s.inv_freq = torch.tensor([f for f, _ in turns], dtype=torch.float64, device=DEVICE)
    s.axes = torch.tensor([a for _, a in turns], dtype=torch.int32, device=DEVICE)
    n_axes = {"one": 1, "two": 2}.get(case["axes"], 3)
    s.positions = torch.randint(0, case["far"] + 1, (n_axes, b, n), device=DEVICE, generator=gen, dtype=torch.int32)
    if case["op"] != "rotate":
        s.wq, s.wk = (randn(dim).mul_(0.2).add_(1).to(dtype) for _ in range(2))
    if case["op"] == "norm_grad":
        s.gq, s.gk = randn(b, n, hq, dim).to(dtype), randn(b, n, hk, dim).to(dtype)
    return s


# ---- plain forms ------------------------------------------------------------------------------------------------------


def _plain_patches(s):
    p, m, dtype = s.case["patch"], s.case["merge"], DTYPES[s.case["dtype"]]
    local = s.index[:, 1].long()
    off, W, _, x0, y0, w, h, rows, cols, flip = s.images[s.index[:, 0].long()].unbind(1)
    block, rest = local // (m * cols), local % (m * cols)
    row, col = block * m + rest % (m * m) // m, rest // (m * m) * m + rest % m
    at = torch.arange(p, device=local.device)

    def taps(out, size, side):           # whole numbers: where a border lies is exact
        num = ((2 * out + 1) * side[:, None] - size[:, None]).clamp(min=0)
        num = torch.minimum(num, (side[:, None] - 1) * 2 * size[:, None])
        lo = num // (2 * size[:, None])
        return lo, torch.minimum(lo + 1, side[:, None] - 1), (num - lo * 2 * size[:, None]).float() / (2 * size[:, None]).float()

    ox = col[:, None] * p + at
    ox = torch.where(flip[:, None] != 0, (cols * p)[:, None] - 1 - ox, ox)
    xa, xb, fx = taps(ox, cols * p, w)
    ya, yb, fy = taps(row[:, None] * p + at, rows * p, h)
    channel = torch.arange(3, device=local.device)[None, :, None, None]

    def pixels(y, x):
        return s.rgb[off[:, None, None, None] + ((y0[:, None] + y)[:, None, :, None] * W[:, None, None, None]
                                                 + (x0[:, None] + x)[:, None, None, :]) * 3 + channel].float()

    fx, fy = fx[:, None, None, :], fy[:, None, :, None]
    top = pixels(ya, xa) * (1 - fx) + pixels(ya, xb) * fx
    low = pixels(yb, xa) * (1 - fx) + pixels(yb, xb) * fx
    v = top * (1 - fy) + low * fy
    mean, std = (torch.tensor(c, device=v.device)[None, :, None, None] for c in (MEAN, STD))
    return ((v / 255.0 - mean) / std).to(dtype).reshape(local.numel(), 3 * p * p)


def _plain_positions(s):
    t, h, w, seq = s.segments.long().T.contiguous()
    text = h * w == 0
    count = torch.where(text, t, t * h * w)
    extent = torch.where(text, t, torch.maximum(t, torch.maximum(h, w)))
    total = torch.cumsum(extent, 0) - extent                   # of all segments before, whatever their sequence
    first = torch.searchsorted(seq, torch.arange(s.n_sequences, device=seq.device))
    base = total - total[first][seq]
    row = torch.repeat_interleave(torch.arange(seq.numel(), device=seq.device), count, output_size=s.n_tokens)
    local = torch.arange(s.n_tokens, device=seq.device) - (torch.cumsum(count, 0) - count)[row]
    hh, ww = h[row].clamp(min=1), w[row].clamp(min=1)
    grid = torch.stack([local // (hh * ww), local // ww % hh, local % ww])
    positions = base[row] + torch.where(text[row], local.expand(3, -1), grid)
    ends = torch.zeros(s.n_sequences, dtype=torch.int64, device=seq.device).scatter_reduce(0, seq, base + extent, "amax")
    return positions.to(torch.int32), ends.to(torch.int32)


def _angles(s):
    angle = s.positions[s.axes.long()].double().permute(1, 2, 0) * s.inv_freq      # far positions: 64 bits
    return angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]


def _turned(x, cos, sin, rot, pairs):
    half = rot // 2
    if pairs == "half":
        a, b = x[..., :half], x[..., half:rot]
        return torch.cat([a * cos - b * sin, a * sin + b * cos, x[..., rot:]], -1)
    a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), x[..., rot:]], -1)


def _plain_rotate(s):
    c = s.case
    cos, sin = _angles(s)
    sin = -sin if c["inverse"] else sin
    return {n: _turned(x.float(), cos, sin, c["rot"], c["pairs"]).to(x.dtype) for n, x in (("q", s.q), ("k", s.k))}


def _plain_norm(s):
    c = s.case
    cos, sin = _angles(s)
    got = {}
    for n, x, weight in (("q", s.q, s.wq), ("k", s.k, s.wk)):
        v = x.float()
        v = v * torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS) * weight.float()
        got[n] = _turned(v, cos, sin, c["rot"], c["pairs"]).to(x.dtype)
    return got


def _plain_norm_grad(s):
    c = s.case
    cos, sin = _angles(s)
    got = {}
    for n, x, weight, g in (("q", s.q, s.wq, s.gq), ("k", s.k, s.wk, s.gk)):
        v, w = x.float(), weight.float()
        d = _turned(g.float(), cos, -sin, c["rot"], c["pairs"])           # the gradient behind the norm
        r = torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS)
        u = v * r
        got["d" + n] = (r * (d * w - u * (d * w * u).mean(-1, keepdim=True))).to(x.dtype)
        got["dw" + n] = (d * u).sum((0, 1, 2)).to(weight.dtype)
    return got


# ---- the framework's operators ----------------------------------------------------------------------------------------


def _own(s):
    import paper_1911_00472_b200 as P
    c = s.case
    if c["op"] == "patches":
        return P.patch_tokens(s.rgb, s.images, s.index, c["patch"], MEAN, STD, merge=c["merge"], dtype=DTYPES[c["dtype"]])
    if c["op"] == "positions":
        return P.token_positions(s.segments, s.n_tokens, s.n_sequences)
    next_ = c["pairs"] == "next"
    if c["op"] == "rotate":
        q, k = P.rotate(s.q, s.k, s.positions, s.inv_freq, s.axes, interleaved=next_, inverse=c["inverse"])
        return {"q": q, "k": k}
    if c["op"] == "norm":
        q, k = P.norm_rotate(s.q, s.k, s.wq, s.wk, s.positions, s.inv_freq, s.axes, eps=EPS, interleaved=next_)
        return {"q": q, "k": k}
    dq, dk, dwq, dwk = P.norm_rotate_backward(s.gq, s.gk, s.q, s.k, s.wq, s.wk, s.positions, s.inv_freq, s.axes, eps=EPS, interleaved=next_)
    return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}


def run(s):
    if own:
        return _own(s)
    return {"patches": _plain_patches, "positions": _plain_positions, "rotate": _plain_rotate, "norm": _plain_norm, "norm_grad": _plain_norm_grad}[s.case["op"]](s)


# ---- work and definition ----------------------------------------------------------------------------------------------


def work(case):
    """Each input read once, each output written once."""
    if case["op"] == "patches":
        table, _ = _images(case)
        values = sum(r[7] * r[8] for r in table) * 3.0 * case["patch"] ** 2
        read = sum(3.0 * r[5] * r[6] for r in table) + 80.0 * len(table) + 8.0 * sum(r[7] * r[8] for r in table)
        return {"bytes": read + values * BYTES[case["dtype"]], "flops": 11.0 * values}
    if case["op"] == "positions":
        rows = _segments(case)
        return {"bytes": 16.0 * len(rows) + 12.0 * sum(map(_tokens, rows)) + 4.0 * case["seqs"], "flops": 6.0 * sum(map(_tokens, rows))}
    tokens, heads, size = case["b"] * case["s"], case["hq"] + case["hk"], BYTES[case["dtype"]]
    values = float(tokens * heads * case["dim"])
    passes = 3 if case["op"] == "norm_grad" else 2
    n_axes = {"one": 1, "two": 2}.get(case["axes"], 3)
    extra = 4.0 * n_axes * tokens + 6.0 * case["rot"] + (4.0 if case["op"] == "norm" else 8.0 if case["op"] == "norm_grad" else 0.0) * case["dim"] * size
    return {"bytes": passes * values * size + extra, "flops": values * {"rotate": 3.0, "norm": 7.0, "norm_grad": 14.0}[case["op"]]}


def _exact_patches(s):
    """Image by image: the resampling as two matrices, rows and columns."""
    c = s.case
    p, m, dev = c["patch"], c["merge"], s.rgb.device

    def matrix(out, side, flip):
        centre = (torch.arange(out, device=dev, dtype=torch.float64) + 0.5) * side / out - 0.5
        centre = centre.clamp(0, side - 1)
        tent = (1 - (centre[:, None] - torch.arange(side, device=dev, dtype=torch.float64)).abs()).clamp(min=0)
        return tent.flip(0) if flip else tent

    got = []
    mean, std = (torch.tensor(v, device=dev, dtype=torch.float64)[:, None, None] for v in (MEAN, STD))
    for off, W, H, x0, y0, w, h, rows, cols, flip in _images(c)[0]:
        image = s.rgb[off:off + 3 * W * H].view(H, W, 3)[y0:y0 + h, x0:x0 + w].permute(2, 0, 1).double()
        v = matrix(rows * p, h, 0) @ image @ matrix(cols * p, w, flip).T
        v = (v / 255 - mean) / std
        v = v.view(3, rows // m, m, p, cols // m, m, p).permute(1, 4, 2, 5, 0, 3, 6)
        got.append(v.reshape(rows * cols, 3 * p * p))
    return torch.cat(got)


def _exact_positions(s):
    """Segment by segment, as a reader of the sequence counts."""
    axes, ends, at, now = ([], [], []), [0] * s.n_sequences, 0, 0
    for t, h, w, seq in s.rows:
        at, now = (at if seq == now else 0), seq
        if not h or not w:
            for a in axes:
                a.extend(range(at, at + t))
            at += t
        else:
            for i in range(t):
                for j in range(h):
                    axes[0].extend([at + i] * w)
                    axes[1].extend([at + j] * w)
                    axes[2].extend(range(at, at + w))
            at += max(t, h, w)
        ends[seq] = at
    return torch.tensor(axes, dtype=torch.int32, device=DEVICE), torch.tensor(ends, dtype=torch.int32, device=DEVICE)


def _exact_heads(s):
    """Pairs as complex numbers times a number of length one; the backward pass by differentiation of the forward."""
    c = s.case
    half, rot, dim = c["rot"] // 2, c["rot"], c["dim"]
    angle = torch.stack([s.positions[a].double() * f for f, a in _turns(c)], -1)[:, :, None]
    unit = torch.polar(torch.ones_like(angle), -angle if c["inverse"] else angle)

    def forward(x, weight):
        if weight is not None:
            x = weight * x / torch.sqrt((x * x).sum(-1, keepdim=True) / dim + EPS)
        parts = x[..., :rot].unflatten(-1, (2, half)).transpose(-1, -2) if c["pairs"] == "half" else x[..., :rot].unflatten(-1, (half, 2))
        z = torch.view_as_real(torch.view_as_complex(parts.contiguous()) * unit)
        z = z.transpose(-1, -2) if c["pairs"] == "half" else z
        return torch.cat([z.reshape(*x.shape[:-1], rot), x[..., rot:]], -1)

    got = {}
    for n in ("q", "k"):
        x = getattr(s, n).double()
        if c["op"] == "rotate":
            got[n] = forward(x, None)
            continue
        weight = getattr(s, "w" + n).double()
        if c["op"] == "norm":
            got[n] = forward(x, weight)
            continue
        x, weight = x.requires_grad_(), weight.requires_grad_()
        got["d" + n], got["dw" + n] = torch.autograd.grad(forward(x, weight), (x, weight), getattr(s, "g" + n).double())
    return got


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_patches(s) if case["op"] == "patches" else _exact_positions(s) if case["op"] == "positions" else _exact_heads(s)
