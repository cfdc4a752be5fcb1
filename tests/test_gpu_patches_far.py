"""Patch tokens of buffers, rectangles and outputs whose bytes are not counted in 32 bits.  Tolerances as in the tests of patches."""
import pytest
import torch

import paper_1911_00472_b200 as P
from test_gpu_patches import DTYPES, MEAN, STD, U, Info

pytestmark = pytest.mark.gpu


def taps(out, side, flip):
    """(left, right, weight of the right one) of every sample: whole numbers over 2 out, by the definition."""
    num = [min(max((2 * o + 1) * side - out, 0), (side - 1) * 2 * out) for o in range(out)]
    lo = [n // (2 * out) for n in num]
    f = [(n % (2 * out)) / (2 * out) for n in num]
    if flip:
        lo, f = lo[::-1], f[::-1]
    lo = torch.tensor(lo, device="cuda")
    return lo, (lo + 1).clamp(max=side - 1), torch.tensor(f, dtype=torch.float64, device="cuda")


def want_of(rgb, info, crop, grid, patch):
    """Only the pixels that count are taken: the image itself would be too large in 64 bits."""
    x0, y0, w, h, flip = crop
    rows, cols = grid
    ya, yb, fy = taps(rows * patch, h, 0)
    xa, xb, fx = taps(cols * patch, w, flip)

    def pixels(y, x):
        at = info.out_offset + ((y0 + y)[:, None] * info.width + (x0 + x)[None]) * 3
        return torch.stack([rgb[at + c] for c in range(3)]).double()

    fx, fy = fx[None, None], fy[None, :, None]
    v = (pixels(ya, xa) * (1 - fx) + pixels(ya, xb) * fx) * (1 - fy) + (pixels(yb, xa) * (1 - fx) + pixels(yb, xb) * fx) * fy
    mean, std = (torch.tensor(t, dtype=torch.float64, device="cuda")[:, None, None] for t in (MEAN, STD))
    v = (v / 255 - mean) / std
    return v.view(3, rows, patch, cols, patch).permute(1, 3, 0, 2, 4).reshape(rows * cols, 3 * patch * patch)


def check(got, want):
    per = torch.tensor([(1 + abs(m)) / s for m, s in zip(MEAN, STD)], dtype=torch.float64, device="cuda").repeat_interleave(got.shape[1] // 3)
    off, allowed = (got.double() - want).abs(), torch.finfo(got.dtype).eps / 2 * want.abs() + 16 * U * per
    assert got.shape == want.shape and bool((off <= allowed).all()), float((off / allowed).max())


def test_rectangles_and_offsets_past_32_bits():
    """An image of more than 2^31 bytes that begins behind 2^31, and a small one behind 2^32 that ends with the buffer."""
    big, small = Info((1 << 31) + 128, 30000, 24000), Info(0, 61, 43)
    small.out_offset = (big.out_offset + 3 * big.width * big.height + 131) // 4 * 4
    assert 3 * big.width * big.height > 1 << 31 and small.out_offset > 1 << 32
    rgb = torch.randint(0, 256, (small.out_offset + 3 * 61 * 43,), dtype=torch.uint8, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    for patch in (14, 16, 9):
        for flip in (0, 1):
            crops, grids = [(0, 0, 30000, 24000, flip), (0, 0, 61, 43, flip)], [(3, 2), (3, 4)]
            plan = P.patch_plan([big, small], patch, crops=crops, grids=grids)
            want = torch.cat([want_of(rgb, i, c, g, patch) for i, c, g in zip((big, small), crops, grids)])
            for dtype in DTYPES:
                check(P.patch_tokens(rgb, plan.images, plan.index, patch, MEAN, STD, dtype=dtype), want)
    # a rectangle that is counted in 32 bits, at the far corner of the image
    crop = (30000 - 211, 24000 - 97, 211, 97, 0)
    plan = P.patch_plan([big], 14, crops=[crop], grids=[(7, 15)])
    check(P.patch_tokens(rgb, plan.images, plan.index, 14, MEAN, STD), want_of(rgb, big, crop, (7, 15), 14))


@pytest.mark.parametrize("patch,dtype", [(32, torch.float32), (31, torch.float32), (14, torch.bfloat16)], ids=str)
def test_outputs_past_32_bits(patch, dtype):
    info = Info(0, 320, 256)
    rgb = torch.randint(0, 256, (3 * 320 * 256,), dtype=torch.uint8, device="cuda", generator=torch.Generator(device="cuda").manual_seed(patch))
    plan = P.patch_plan([info], patch)
    few = P.patch_tokens(rgb, plan.images, plan.index, patch, MEAN, STD, dtype=dtype)
    check(few, want_of(rgb, info, (0, 0, 320, 256, 0), plan.grids[0].tolist(), patch))
    n, bytes_ = len(few), few.shape[1] * few.element_size()
    times = (1 << 32) // (bytes_ * n) + 2                       # the last repetitions lie beyond 2^32 bytes
    got = P.patch_tokens(rgb, plan.images, plan.index.repeat(times, 1), patch, MEAN, STD, dtype=dtype)
    assert got.numel() * got.element_size() > 1 << 32
    at = got.view(times, n, -1)
    for i in range(0, times, 64):
        assert bool((at[i:i + 64] == few).all())
