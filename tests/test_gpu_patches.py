"""Patch tokens and token positions against plain forms in 64 bits, and the path from a record to a training step.

Tolerance of a token's value (v / 255 - mean) / std: the weights of the taps and each of the two mixes are off by at most
3 u of 255 (u = 2^-24; where a sample falls is worked out in whole numbers), scaling and shifting by 3 u of their
terms: 16 u (1 / std + |mean / std|) is taken, and half a step of the output type.  Positions are whole numbers: equal."""
from concurrent.futures import ThreadPoolExecutor

import numpy as np
import pytest
import torch

import pcr_synth
import paper_1911_00472_b200 as P
from oracle import pcr_oracle as O

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
MEAN, STD = (0.485, 0.456, 0.406), (0.229, 0.224, 0.225)
DTYPES = [torch.bfloat16, torch.float16, torch.float32]


class Info:
    def __init__(self, out_offset, width, height):
        self.out_offset, self.width, self.height = out_offset, width, height


def matrix(out, side, flip=0):
    """Rows of bilinear weights, by the definition: half-pixel centres, the edge pixels repeated."""
    centre = np.clip((np.arange(out) + 0.5) * side / out - 0.5, 0, side - 1)
    m = np.maximum(0, 1 - np.abs(centre[:, None] - np.arange(side)))
    return m[::-1] if flip else m


def tokens_of(image, crop, grid, patch, merge):
    x0, y0, w, h, flip = crop
    rows, cols = grid
    v = image[y0:y0 + h, x0:x0 + w].astype(np.float64).transpose(2, 0, 1)
    v = matrix(rows * patch, h) @ v @ matrix(cols * patch, w, flip).T
    v = (v / 255 - np.array(MEAN)[:, None, None]) / np.array(STD)[:, None, None]
    order = [(r, c) for rb in range(0, rows, merge) for cb in range(0, cols, merge) for r in range(rb, rb + merge) for c in range(cb, cb + merge)]
    return np.stack([v[:, r * patch:(r + 1) * patch, c * patch:(c + 1) * patch].reshape(-1) for r, c in order])


def check(got, want):
    want = torch.from_numpy(want).to(got.device)
    per = torch.tensor([(1 + abs(m)) / s for m, s in zip(MEAN, STD)], dtype=torch.float64, device=got.device)
    slack = 16 * U * per.repeat_interleave(got.shape[1] // 3)
    off = (got.double() - want).abs()
    allowed = torch.finfo(got.dtype).eps / 2 * want.abs() + slack
    assert got.shape == want.shape and bool((off <= allowed).all()), float((off / allowed).max())


def images(sizes, seed=0):
    """(images, info, buffer) of random images, at offsets that are multiples of 4 and not of 128 only."""
    rng = np.random.default_rng(seed)
    pics = [rng.integers(0, 256, (h, w, 3), dtype=np.uint8) for w, h in sizes]
    at, info = 0, []
    for p in pics:
        info.append(Info(at, p.shape[1], p.shape[0]))
        at += p.size + rng.integers(0, 9)
    buf = np.zeros(at, dtype=np.uint8)
    for p, i in zip(pics, info):
        buf[i.out_offset:i.out_offset + p.size] = p.reshape(-1)
    return pics, info, torch.from_numpy(buf[:info[-1].out_offset + pics[-1].size].copy()).cuda()     # (nothing behind the last pixel)


SIZES = [(37, 53), (1, 1), (14, 14), (200, 9), (3, 301), (64, 64), (128, 96)]


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("patch,merge", [(14, 2), (16, 1), (1, 1), (3, 3), (7, 2), (5, 1), (32, 1), (17, 1), (28, 2), (8, 4), (2, 1)])
def test_sizes(patch, merge, dtype):
    pics, info, rgb = images(SIZES, patch)
    whole = [(0, 0, i.width, i.height, 0) for i in info]
    rng = np.random.default_rng(patch + merge)
    cut = []
    for i in info:
        w, h = rng.integers(1, i.width + 1), rng.integers(1, i.height + 1)
        cut.append((rng.integers(0, i.width - w + 1), rng.integers(0, i.height - h + 1), w, h, rng.integers(0, 2)))
    for crops in (whole, cut):
        plan = P.patch_plan(info, patch, merge=merge, crops=np.array(crops))
        got = P.patch_tokens(rgb, plan.images, plan.index, patch, MEAN, STD, merge=merge, dtype=dtype)
        check(got, np.concatenate([tokens_of(p, c, g, patch, merge) for p, c, g in zip(pics, crops, plan.grids)]))


def test_grids_of_any_size_order_of_tokens_and_parts():
    pics, info, rgb = images(SIZES[:4])
    grids = np.array([(6, 2), (2, 2), (4, 8), (2, 14)])
    plan = P.patch_plan(info, 14, merge=2, grids=grids)
    crops = [(0, 0, i.width, i.height, 0) for i in info]
    want = np.concatenate([tokens_of(p, c, g, 14, 2) for p, c, g in zip(pics, crops, grids)])
    check(P.patch_tokens(rgb, plan.images, plan.index, 14, MEAN, STD, merge=2), want)
    # any order of the tokens, some twice; an output that is given; one token; none
    pick = torch.randperm(len(want), device="cuda")[:37].repeat(2)
    out = torch.empty(74, 588, dtype=torch.float16, device="cuda")
    got = P.patch_tokens(rgb, plan.images, plan.index[pick].contiguous(), 14, MEAN, STD, merge=2, dtype=torch.float16, out=out)
    assert got is out
    check(got, want[pick.cpu().numpy()])
    check(P.patch_tokens(rgb, plan.images, plan.index[5:6].contiguous(), 14, MEAN, STD, merge=2), want[5:6])
    assert P.patch_tokens(rgb, plan.images, plan.index[:0].contiguous(), 14, MEAN, STD).shape == (0, 588)
    # outputs that start at any element
    for shift in (1, 2, 4):
        room = torch.full((74 * 588 + 8,), 9.0, dtype=torch.float16, device="cuda")
        got = P.patch_tokens(rgb, plan.images, plan.index[pick].contiguous(), 14, MEAN, STD, merge=2, dtype=torch.float16,
                             out=room[shift:shift + 74 * 588].view(74, 588))
        assert torch.equal(got, out) and bool((room[:shift] == 9).all()) and bool((room[shift + 74 * 588:] == 9).all())


def test_large_resampling_ratios():
    # one image so large, or so stretched, that the taps' arithmetic takes more than 32 bits
    pics, info, rgb = images([(20000, 3), (5, 5)])
    plan = P.patch_plan(info, 32, merge=1, grids=np.array([(1, 1600), (1, 1700)]))
    want = np.concatenate([tokens_of(p, (0, 0, i.width, i.height, 0), g, 32, 1) for p, i, g in zip(pics, info, plan.grids)])
    check(P.patch_tokens(rgb, plan.images, plan.index, 32, MEAN, STD, dtype=torch.float32), want)


@pytest.mark.parametrize("patch", [14, 16, 9])
@pytest.mark.parametrize("scale", [0.4, 0.99, 1.01, 1.7, 2.3, 5.0])
def test_resampling_by_any_factor(patch, scale):
    # neighbouring columns one source pixel apart, two or none, or further; source rows that repeat or are left out
    pics, info, rgb = images([(211, 173), (96, 64)], 4)
    crops = np.array([(3, 5, 200, 160, 0), (0, 0, 95, 63, 1)])
    grids = np.maximum(1, np.round(crops[:, [3, 2]] / (patch * scale)).astype(int))
    plan = P.patch_plan(info, patch, crops=crops, grids=grids)
    want = np.concatenate([tokens_of(p, c, g, patch, 1) for p, c, g in zip(pics, crops, grids)])
    for dtype in DTYPES:
        check(P.patch_tokens(rgb, plan.images, plan.index, patch, MEAN, STD, dtype=dtype), want)


@pytest.mark.parametrize("patch", [14, 16, 9])
@pytest.mark.parametrize("flip", [0, 1])
def test_end_of_the_buffer(patch, flip):
    """Images whose last pixel is the buffer's, of 0 to 3 bytes beyond a whole word: nothing behind it counts."""
    for w, h in [(61, 43), (61, 44), (62, 45), (63, 47), (1, 1), (5, 1), (1, 3)]:
        pics, info, _ = images([(8, 3), (w, h)], w)
        pics, info = pics[1:], [Info(0, w, h)]
        n = pics[0].size
        for grid in [(max(1, h // patch), max(1, w // patch)), (5, 6), (1, 2)]:
            crop = (0, 0, w, h, flip)
            plan = P.patch_plan(info, patch, crops=np.array([crop]), grids=np.array([grid]))
            got = []
            for behind in (0, 255):
                room = torch.full((n + 64,), behind, dtype=torch.uint8, device="cuda")
                room[:n] = torch.from_numpy(pics[0].reshape(-1)).cuda()
                got.append(P.patch_tokens(room[:n], plan.images, plan.index, patch, MEAN, STD, dtype=torch.float32))
            assert torch.equal(got[0], got[1])
            check(got[0], tokens_of(pics[0], crop, grid, patch, 1))


def test_graphs_and_streams():
    """Captured and replayed on other pixels, and on a stream of its own."""
    pics, info, rgb = images(SIZES)
    plan = P.patch_plan(info, 14, merge=2)
    segments = plan.segments(merged=True)
    T = len(plan.index) // 4
    want = P.patch_tokens(rgb, plan.images, plan.index, 14, MEAN, STD, merge=2)
    at, after = P.token_positions(segments, T, len(info))
    work = torch.zeros_like(rgb)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = P.patch_tokens(work, plan.images, plan.index, 14, MEAN, STD, merge=2)
        got_at, got_after = P.token_positions(segments, T, len(info))
    work.copy_(rgb)
    graph.replay()
    assert torch.equal(got, want) and torch.equal(got_at, at) and torch.equal(got_after, after)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = P.patch_tokens(rgb, plan.images, plan.index, 14, MEAN, STD, merge=2, stream=side)
    got_at, got_after = P.token_positions(segments, T, len(info), stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want) and torch.equal(got_at, at) and torch.equal(got_after, after)


def test_entries_that_do_not_fit_give_zeros():
    pics, info, rgb = images(SIZES[:3])
    plan = P.patch_plan(info, 14, merge=2)
    good = P.patch_tokens(rgb, plan.images, plan.index, 14, MEAN, STD, merge=2)
    big = 1 << 40
    for row, col, value in [(0, 0, rgb.numel() - 10), (0, 0, -4), (0, 0, big), (0, 1, 38 * 53), (0, 1, 0), (0, 2, big), (0, 3, -1), (0, 3, 1), (0, 4, 2 * big),
                            (0, 5, 0), (0, 5, 38), (0, 6, -3), (0, 7, 0), (0, 7, 3), (0, 8, big), (0, 8, -2), (0, 9, 2)]:
        bad = plan.images.clone()
        bad[row, col] = value
        got = P.patch_tokens(rgb, bad, plan.index, 14, MEAN, STD, merge=2)
        mine = plan.index[:, 0] == row
        assert bool((got[mine] == 0).all()), (col, value)
        assert torch.equal(got[~mine], good[~mine])
    index = plan.index.clone()
    index[0, 0], index[1, 0], index[2, 1], index[3, 1], index[4, 0] = 3, -1, 1 << 30, -1, 1 << 30
    got = P.patch_tokens(rgb, plan.images, index, 14, MEAN, STD, merge=2)
    assert bool((got[:5] == 0).all()) and torch.equal(got[5:], good[5:])


def test_refusals():
    pics, info, rgb = images(SIZES[:3])
    plan = P.patch_plan(info, 14, merge=2)
    ok = (rgb, plan.images, plan.index)
    for args in ((rgb.float(), *ok[1:]), (rgb, plan.images.int(), plan.index), (rgb, plan.images[:, :9], plan.index), (rgb, plan.images, plan.index.long()),
                 (rgb, plan.images.cpu(), plan.index), (rgb[::2], *ok[1:])):
        with pytest.raises(ValueError):
            P.patch_tokens(*args, 14, MEAN, STD)
    for patch, kw in ((0, {}), (33, {}), (14, dict(merge=0)), (14, dict(merge=65))):
        with pytest.raises(P.PcrError):
            P.patch_tokens(*ok, patch, MEAN, STD, **kw)
    with pytest.raises(P.PcrError):
        P.patch_tokens(*ok, 14, MEAN, (0.2, 0.0, 0.2))
    with pytest.raises(P.PcrError):                       # pixels are read as aligned words
        P.patch_tokens(rgb[1:], plan.images, plan.index, 14, MEAN, STD)
    with pytest.raises(ValueError):
        P.patch_tokens(*ok, 14, MEAN, STD, dtype=torch.float64)
    seg = plan.segments()
    for bad in (seg.long(), seg[:, :3], seg.t()):
        with pytest.raises(ValueError):
            P.token_positions(bad, 10, 3)
    with pytest.raises(ValueError):
        P.token_positions(seg, 10, 3, out=torch.empty(3, 9, dtype=torch.int32, device="cuda"))
    for kw in (dict(merge=0), dict(time_step=-1), dict(time_step=1 << 21)):
        with pytest.raises(P.PcrError):
            P.token_positions(seg, 10, 3, **kw)
    with pytest.raises((P.PcrError, RuntimeError)):
        P.token_positions(seg, -1, 3)
    torch.cuda.synchronize()


# ---- positions ----------------------------------------------------------------------------------------------------------


def positions_of(rows, n_sequences, merge=1, time_step=1, restart=False):
    out, after, at, now = [], [0] * n_sequences, 0, None
    for t, h, w, seq in rows:
        t = max(t, 0)
        if seq != now or restart:
            at, now = 0, seq
        if h <= 0 or w <= 0:
            out += [(at + i,) * 3 for i in range(t)]
            at += t
        elif t:
            m = merge if h % merge == 0 and w % merge == 0 else 1
            for f in range(t):
                out += [(at + f * time_step, at + y, at + x) for yb in range(0, h, m) for xb in range(0, w, m)
                        for y in range(yb, yb + m) for x in range(xb, xb + m)]
            at += max((t - 1) * time_step, h - 1, w - 1) + 1
        if 0 <= seq < n_sequences:
            after[seq] = at
    return np.array(out, dtype=np.int64).reshape(-1, 3).T, np.array(after)


def check_positions(rows, n_sequences, **kw):
    segments = torch.tensor(rows, dtype=torch.int32, device="cuda").reshape(-1, 4)
    want, after = positions_of(rows, n_sequences, **kw)
    got, next_ = P.token_positions(segments, want.shape[1], n_sequences, **kw)
    assert np.array_equal(got.cpu().numpy(), want) and np.array_equal(next_.cpu().numpy(), after)
    return segments, want


@pytest.mark.parametrize("kw", [dict(), dict(merge=2), dict(time_step=3), dict(restart=True, merge=2), dict(time_step=0)], ids=str)
@pytest.mark.parametrize("rows", [
    [], [(0, 0, 0, 0)], [(1, 0, 0, 0)], [(5, 0, 0, 0), (1, 4, 6, 0), (3, 0, 0, 0)],
    [(2, 4, 4, 0), (1, 0, 0, 0), (0, 5, 5, 0), (4, 2, 2, 0), (1, 3, 5, 1), (2, 0, 7, 1), (1, 1, 1, 3)],
    [(-3, 0, 0, 0), (2, -1, 4, 0), (7, 8, 2, 2), (-1, 4, 4, 2), (1, 2, 2, 2)],
], ids=lambda r: str(len(r)))
def test_positions_small(rows, kw):
    check_positions(rows, 4, **kw)


@pytest.mark.parametrize("n", [1, 1023, 1024, 1025, 5000, 20011])
def test_positions_many_segments(n):
    rng = np.random.default_rng(n)
    seq = np.cumsum(rng.random(n) < 0.05)
    rows = [(int(rng.integers(0, 9)), 0, 0, int(s)) if rng.random() < 0.5 else (int(rng.integers(0, 3)), int(rng.integers(1, 6)), int(rng.integers(1, 6)), int(s)) for s in seq]
    check_positions(rows, int(seq[-1]) + 1)
    check_positions(rows, int(seq[-1]) + 1, restart=True, time_step=2)


def test_positions_asked_for_by_several_threads():
    """Calls of different sizes side by side: the kernel's limit of shared memory is the same for all."""
    def work(n):
        rng = np.random.default_rng(n)
        rows = [(int(t), 0, 0, i // 7) for i, t in enumerate(rng.integers(0, 4, n))]
        segments = torch.tensor(rows, dtype=torch.int32, device="cuda")
        want, after = positions_of(rows, n // 7 + 1)
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        got = [P.token_positions(segments, want.shape[1], n // 7 + 1, stream=stream) for _ in range(50)]
        stream.synchronize()
        return all(np.array_equal(g.cpu().numpy(), want) and np.array_equal(e.cpu().numpy(), after) for g, e in got)

    with ThreadPoolExecutor(4) as pool:
        assert all(pool.map(work, [16384, 5200, 9000, 700]))


def test_positions_long_segments():
    check_positions([(70000, 0, 0, 0), (3, 150, 201, 0), (100001, 0, 0, 1)], 2)


def test_positions_sizes_past_32_bits():
    # more tokens than any output holds: those that are asked for
    side = 2 ** 31 - 1
    segments = torch.tensor([(2, side, side, 0), (5, 0, 0, 0)], dtype=torch.int32, device="cuda")
    got, _ = P.token_positions(segments, 1000, 1)
    want = np.stack([np.zeros(1000), np.zeros(1000), np.arange(1000)])
    assert np.array_equal(got.cpu().numpy(), want)


def test_positions_behind_the_last_token_and_beyond_the_output():
    rows = [(3, 0, 0, 0), (1, 2, 3, 0)]
    segments, want = check_positions(rows, 1)
    got, _ = P.token_positions(segments, 12, 1)
    assert np.array_equal(got[:, :9].cpu().numpy(), want) and bool((got[:, 9:] == 0).all())
    room = torch.full((3, 20), 77, dtype=torch.int32, device="cuda")
    P.token_positions(segments, 12, 1, out=room)
    assert np.array_equal(room[:, :9].cpu().numpy(), want) and bool((room[:, 9:] == 77).all())     # left as they were
    room.fill_(77)
    P.token_positions(segments, 5, 1, out=room)
    assert np.array_equal(room[:, :5].cpu().numpy(), want[:, :5]) and bool((room[:, 5:] == 77).all())
    empty = torch.empty(0, 4, dtype=torch.int32, device="cuda")
    got, after = P.token_positions(empty, 4, 2)
    assert bool((got == 0).all()) and bool((after == 0).all())
    assert P.token_positions(empty, 0, 0)[0].shape == (3, 0)


# ---- together -------------------------------------------------------------------------------------------------------------


def test_tokens_of_a_record_equal_the_oracles_batch(rec2_small):
    """A square grid of patches is the training batch of that size, cut up: the oracle's decode and resampling."""
    dec = P.Decoder(rec2_small.bytes)
    try:
        crops = pcr_synth.random_resized_crops([(int(w), int(h)) for w, h in rec2_small.dims], 3)
        plan = dec.patch_plan(8, merge=2, crops=crops, grids=np.full((dec.n_images, 2), 6))
        got = dec.decode_patches(5, plan, MEAN, STD, dtype=torch.float32)
        torch.cuda.synchronize()
        assert dec.status() == (-1, 0)
        got = got.view(dec.n_images, 3, 3, 2, 2, 3, 8, 8).permute(0, 5, 1, 3, 6, 2, 4, 7).reshape(dec.n_images, 3, 48, 48).cpu().numpy()
        for i in range(dec.n_images):
            _, rgb = O.decode_image(rec2_small.bytes, i, 5)
            want = O.training_tensor(rgb, crops[i], 48, MEAN, STD, dtype=np.float32)
            assert np.abs(got[i] - want).max() <= 1e-5
        batch = dec.decode_tensor(5, crops, 48, MEAN, STD, dtype=torch.float32).cpu().numpy()
        assert np.abs(got - batch).max() <= 1e-5
    finally:
        dec.close()


def test_from_a_record_to_gradients(rec1_small):
    """Decode to patch tokens, positions of an image encoder, projection, norms and rotation, attention inside each image, and
    the way back to the weights: against the same step in 64 bits by differentiation."""
    dec = P.Decoder(rec1_small.bytes)
    try:
        n = dec.n_images
        plan = dec.patch_plan(16, merge=2, grids=np.array([(2 + 2 * (i % 3), 4) for i in range(n)]))
        tokens = dec.decode_patches(10, plan, MEAN, STD, dtype=torch.float32)
        positions, after = P.token_positions(plan.segments(), len(tokens), n, merge=2, restart=True)
        assert np.array_equal(after.cpu().numpy(), plan.grids.max(1))
    finally:
        torch.cuda.synchronize()
        dec.close()
    H, D, T = 4, 40, len(tokens)
    gen = torch.Generator(device="cuda").manual_seed(5)
    project = torch.randn(768, 3 * H * D, device="cuda", generator=gen) / 768 ** 0.5
    wq, wk = (1 + 0.2 * torch.randn(D, device="cuda", generator=gen) for _ in range(2))
    weigh = torch.randn(T, H, D, device="cuda", generator=gen)
    inv_freq, axes = P.rotary_axes(D, sections=(0, 10, 10), per_axis=True)
    image = plan.index[:, 0]
    apart = image[:, None] != image[None]

    def attend(q, k, v):
        score = torch.einsum("qhd,khd->hqk", q, k) / D ** 0.5
        return (torch.einsum("hqk,khd->qhd", score.masked_fill(apart, float("-inf")).softmax(-1), v) * weigh.to(q.dtype)).sum()

    torch.backends.cuda.matmul.allow_tf32 = False
    qkv = (tokens @ project).view(T, 3 * H, D)
    q, k, v = qkv.split(H, 1)
    yq, yk = P.norm_rotate(q, k, wq, wk, positions, inv_freq, axes)
    yq.requires_grad_(), yk.requires_grad_()
    value = v.clone().requires_grad_()
    loss = attend(yq, yk, value)
    gq, gk, gv = torch.autograd.grad(loss, (yq, yk, value))
    dq, dk, dwq, dwk = P.norm_rotate_backward(gq, gk, q, k, wq, wk, positions, inv_freq, axes)
    got = {"project": tokens.T @ torch.cat([dq, dk, gv], 1).view(T, -1), "wq": dwq, "wk": dwk}

    leaves = {"project": project.double().requires_grad_(), "wq": wq.double().requires_grad_(), "wk": wk.double().requires_grad_()}
    q, k, v = (tokens.double() @ leaves["project"]).view(T, 3 * H, D).split(H, 1)
    angle = (positions[axes.long()].double().T * inv_freq)[:, None]
    heads = []
    for x, w in ((q, leaves["wq"]), (k, leaves["wk"])):
        x = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w
        a, b = x[..., :20], x[..., 20:]
        heads.append(torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1))
    exact = attend(*heads, v)
    want = dict(zip(leaves, torch.autograd.grad(exact, list(leaves.values()))))
    # single-precision products of length 768 and T between well-scaled factors: 1e-5 of the norm leaves them an order of magnitude
    assert abs(loss.item() - exact.item()) <= 1e-4 * float(weigh.abs().sum())
    for name in want:
        assert float((got[name].double() - want[name]).norm()) <= 1e-4 * float(want[name].norm()), name
