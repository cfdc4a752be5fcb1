"""Queries and keys turned by positions (rotate, norm_rotate, norm_rotate_backward) against plain forms in 64 bits.

Tolerances, per element.  The kernels work in single precision, u = 2^-24, and round once to the output type, which is off
by at most eps / 2 of the value.
* cosine and sine, 32-bit operands: what is left of the angle after whole turns is rounded to single precision (at most pi u)
  and the function is off by at most 2 units in the last place, so each is off by at most 8 u.  16-bit operands: the angle,
  at most pi, carries two roundings and that of pi itself (2.5 u of it), the hardware's functions are off by at most
  2^-21.41 = 6.0 u (sine) and 2^-21.19 = 7.0 u (cosine): the sine by 2.5 pi u + 6.0 u = 13.9 u at most, the cosine by 2.5 u times
  the largest x sin x up to pi, 1.82, + 7.0 u = 11.6 u.  A turned element is a sum of two products, a cos - b sin, whose
  roundings are 2 u more: (|a| + |b|) times 16 u is taken.
* the norm: a sum of up to 512 squares in at most 16 additions a lane and 5 between lanes (or 32 and 5 where the lanes go
  over a head value by value), so 1 / sqrt is off by (37 + 6) / 2 u, and the products by 3 u more: 32 u in all.
* backward: dx = r (d w - v m), m = mean(d w v) with v = x r; d w and v by the figures above, m by at most 37 + 16 + 32 + 8
  units u of mean |d w v|: 128 u of r (|d w| + |v| mean |d w v|) is taken, with |a| + |b| in the place of |d|.
* dw: a sum over n rows, added in some order: (n + 64) u of the sum of magnitudes.
"""
import math

import pytest
import torch

import paper_1911_00472_b200 as P

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = [torch.bfloat16, torch.float16, torch.float32]
# batch, tokens, heads of queries and keys, head size, turned
SHAPES = [
    (1, 1, 1, 1, 2, 2), (1, 1, 32, 8, 128, 128), (2, 7, 3, 1, 72, 72), (3, 5, 4, 4, 80, 40), (1, 33, 2, 2, 96, 96), (1, 130, 5, 1, 64, 32),
    (2, 3, 1, 1, 256, 256), (1, 9, 2, 1, 512, 512), (1, 5, 3, 2, 6, 2), (1, 4, 2, 1, 7, 4), (2, 2, 1, 1, 33, 0), (1, 700, 16, 16, 48, 24),
    (5, 61, 7, 0, 112, 112), (1, 300, 0, 3, 192, 128), (64, 1, 9, 3, 24, 24), (1, 1, 1, 1, 1, 0), (1, 40, 2, 1, 66, 66), (1, 3, 2, 2, 510, 34),
]


def turned(x, angle, interleaved):
    """(turned x, |a| + |b| of every element) for x (B, S, H, D) and angle (B, S, rot / 2), all in 64 bits."""
    half = angle.shape[-1]
    rot, y, size = 2 * half, x.clone(), x.abs()
    one, two = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, half), slice(half, rot))
    c, s = angle.cos()[:, :, None], angle.sin()[:, :, None]
    y[..., one], y[..., two] = x[..., one] * c - x[..., two] * s, x[..., one] * s + x[..., two] * c
    size[..., one] = size[..., two] = x[..., one].abs() + x[..., two].abs()
    return y, size


def make(shape, dtype, layout="plain", axes_kind="runs", seed=0, far=1 << 20, weight_dtype=None):
    B, S, Hq, Hk, D, rot = shape
    g = torch.Generator(device="cuda").manual_seed(seed + 17 * D + S)

    def block(H):
        if H == 0:
            return None
        if layout == "plain":
            return torch.randn(B, S, H, D, device="cuda", generator=g).to(dtype)
        if layout == "heads_first":                                   # (batch, heads, tokens, size) seen the other way
            return torch.randn(B, H, S, D, device="cuda", generator=g).to(dtype).transpose(1, 2)
        if layout == "shifted":                                       # rows that start at odd elements, odd strides
            return torch.randn(B, S, H * D + 3, device="cuda", generator=g).to(dtype)[:, :, 1:1 + H * D].unflatten(-1, (H, D))
        return torch.randn(B, S, H + 2, D, device="cuda", generator=g).to(dtype)[:, :, 1:1 + H]        # packed

    half = rot // 2
    sections = {"one": [half], "runs": [half // 4, (half - half // 4) // 2, half - half // 4 - (half - half // 4) // 2], "two": [half - half // 2, half // 2]}[axes_kind]
    inv_freq, axes = P.rotary_axes(rot, sections=sections, interleaved_axes=seed % 2 == 1, per_axis=axes_kind == "two")
    positions = torch.randint(-far, far, (len(sections), B, S), device="cuda", generator=g, dtype=torch.int32)
    wt = weight_dtype or dtype
    wq, wk = ((1 + 0.3 * torch.randn(D, device="cuda", generator=g)).to(wt) for _ in range(2))
    return block(Hq), block(Hk), positions, inv_freq, axes, wq, wk


def angle_of(positions, inv_freq, axes):
    return positions[axes.long()].double().permute(1, 2, 0) * inv_freq.double()


def check(got, want, slack, what=""):
    assert got.shape == want.shape, what
    off = (got.double() - want).abs()
    allowed = torch.finfo(got.dtype).eps / 2 * want.abs() + slack + torch.finfo(got.dtype).smallest_normal * torch.finfo(got.dtype).eps
    assert bool((off <= allowed).all()), (what, float((off / allowed).max()))


def check_forward(x, y, angle, interleaved, weight=None, eps=None, what=""):
    x = x.double()
    if eps is None:
        want, size = turned(x, angle, interleaved)
        check(y, want, 16 * U * size, what)
    else:
        w = torch.ones(x.shape[-1], device="cuda", dtype=torch.float64) if weight is None else weight.double()
        want, size = turned(x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w, angle, interleaved)
        check(y, want, (16 + 32) * U * size, what)


def check_backward(x, g, dx, dw, angle, interleaved, weight, eps, what=""):
    x, g = x.double(), g.double()
    w = torch.ones(x.shape[-1], device="cuda", dtype=torch.float64) if weight is None else weight.double()
    d, size = turned(g, -angle, interleaved)
    r = 1 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    v = x * r
    want = r * (d * w - v * (d * w * v).mean(-1, keepdim=True))
    check(dx, want, 128 * U * r * ((size * w).abs() + v.abs() * (size * w * v).abs().mean(-1, keepdim=True)), what + " dx")
    if weight is not None:
        rows = x.shape[0] * x.shape[1] * x.shape[2]
        check(dw, (d * v).sum((0, 1, 2)), (rows + 64) * U * (size * v).abs().sum((0, 1, 2)), what + " dw")


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_shapes(shape, interleaved, dtype):
    for n, (layout, kind) in enumerate([("plain", "runs"), ("packed", "two"), ("heads_first", "one"), ("shifted", "runs")]):
        q, k, positions, inv_freq, axes, wq, wk = make(shape, dtype, layout, kind, seed=n)
        if q is None:
            q, k, wq, wk = k, None, wk, None
        if k is None:
            wk = None
        angle, eps = angle_of(positions, inv_freq, axes), 1e-6
        y = P.rotate(q, k, positions, inv_freq, axes, interleaved=interleaved)
        z = P.rotate(q, k, positions, inv_freq, axes, interleaved=interleaved, inverse=True)
        m = P.norm_rotate(q, k, wq, wk, positions, inv_freq, axes, eps=eps, interleaved=interleaved)
        gq, gk = (None if t is None else torch.randn(t.shape, device="cuda").to(dtype) for t in (q, k))
        b = P.norm_rotate_backward(gq, gk, q, k, wq, wk, positions, inv_freq, axes, eps=eps, interleaved=interleaved)
        for i, (x, g, w) in enumerate([(q, gq, wq), (k, gk, wk)]):
            if x is None:
                assert y[i] is None and z[i] is None and m[i] is None and b[i] is None and b[2 + i] is None
                continue
            check_forward(x, y[i], angle, interleaved, what=layout)
            check_forward(x, z[i], -angle, interleaved, what=layout + " inverse")
            check_forward(x, m[i], angle, interleaved, w, eps, what=layout + " norm")
            check_backward(x, g, b[i], b[2 + i], angle, interleaved, w, eps, what=layout)


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("short", [False, True])
@pytest.mark.parametrize("vectors", list(range(1, 33)))
def test_rows_of_any_number_of_vectors(vectors, short, dtype):
    """Heads of 1 to 32 pairs of 16-byte vectors (short: of vectors of two elements, as four turned elements ask for), a pair a lane: every way in which the lanes of a row add up, with heads of one
    operand far larger than the other's and tokens that leave lanes without one."""
    size = vectors * (4 if short else 16 if dtype.itemsize == 2 else 8)
    q, k, positions, inv_freq, axes, wq, wk = make((2, 37, 3, 1, size, 4 if short else size), dtype, seed=vectors)
    q[1] *= 100
    angle = angle_of(positions, inv_freq, axes)
    gq, gk = (torch.randn(t.shape, device="cuda").to(dtype) for t in (q, k))
    b = P.norm_rotate_backward(gq, gk, q, k, wq, wk, positions, inv_freq, axes, eps=1e-6, interleaved=vectors % 2 == 1)
    for i, (x, g, w) in enumerate([(q, gq, wq), (k, gk, wk)]):
        check_backward(x, g, b[i], b[2 + i], angle, vectors % 2 == 1, w, 1e-6)


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
def test_many_rows_and_weights_of_single_precision(dtype):
    # more tokens than one round of the grid, so that the sums of the weights' gradients run over several
    q, k, positions, inv_freq, axes, wq, wk = make((2, 4099, 6, 2, 64, 64), dtype, "packed", weight_dtype=torch.float32)
    gq, gk = torch.randn_like(q), torch.randn_like(k)
    angle = angle_of(positions, inv_freq, axes)
    first = None
    for _ in range(2):
        got = P.norm_rotate_backward(gq, gk, q, k, wq, wk, positions, inv_freq, axes)
        assert got[2].dtype == got[3].dtype == torch.float32
        check_backward(q, gq, got[0], got[2], angle, False, wq, 1e-6, "q")
        check_backward(k, gk, got[1], got[3], angle, False, wk, 1e-6, "k")
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))          # always in the same order
    # weights left out on either side
    got = P.norm_rotate_backward(gq, gk, q, k, None, wk, positions, inv_freq, axes)
    assert got[2] is None and torch.equal(got[3], first[3])
    check_backward(q, gq, got[0], None, angle, False, None, 1e-6, "without weights")
    y = P.norm_rotate(q, k, None, wk, positions, inv_freq, axes)
    check_forward(q, y[0], angle, False, None, 1e-6)


def test_three_dimensions_expanded_positions_and_single_frequencies():
    q, k, positions, inv_freq, axes, _, _ = make((3, 50, 4, 2, 64, 64), torch.bfloat16)
    shared = positions[:, :1].expand(-1, 3, -1)
    angle = angle_of(shared, inv_freq.float(), axes)
    y = P.rotate(q, k, shared, inv_freq.float(), axes)
    check_forward(q, y[0], angle, False)
    check_forward(k, y[1], angle, False)
    flat = P.rotate(q.flatten(0, 1), k.flatten(0, 1), shared.flatten(1), inv_freq.float(), axes)
    assert torch.equal(flat[0].view_as(q), y[0]) and torch.equal(flat[1].view_as(k), y[1])
    every_other = P.rotate(q[:, ::2], None, shared[:, :, ::2], inv_freq.float(), axes)
    assert torch.equal(every_other[0], y[0][:, ::2])


def test_farthest_positions_and_axes_that_are_not_there():
    q, k, positions, inv_freq, axes, _, _ = make((1, 64, 2, 1, 32, 32), torch.float32)
    positions.fill_(2 ** 31 - 1)
    positions[:, :, ::2] = -2 ** 31
    # the product position * frequency is exact to 2^-53: 3e8 turns leave 2^-53 * 2^31 of an angle, far below u
    y = P.rotate(q, k, positions, inv_freq, axes)
    check_forward(q, y[0], angle_of(positions, inv_freq, axes), False)
    odd = axes.clone()
    odd[::2], odd[1] = 7, -1
    angle = angle_of(positions, inv_freq, axes)
    angle[..., odd == 7] = 0
    angle[..., odd == -1] = 0
    check_forward(q, P.rotate(q, k, positions, inv_freq, odd)[0], angle, False)


@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place_and_outputs_of_other_strides(interleaved):
    for layout in ("plain", "packed", "heads_first", "shifted"):
        q, k, positions, inv_freq, axes, wq, wk = make((2, 37, 8, 2, 80, 80), torch.bfloat16, layout)
        gq, gk = torch.randn_like(q), torch.randn_like(k)
        angle = angle_of(positions, inv_freq, axes)
        want = P.norm_rotate(q, k, wq, wk, positions, inv_freq, axes, interleaved=interleaved)
        other = torch.full((2, 10, 41, 80), 7.0, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
        P.norm_rotate(q, k, wq, wk, positions, inv_freq, axes, interleaved=interleaved, out=(other[:, 2:39, :8], other[:, 2:39, 8:]))
        check_forward(q, other[:, 2:39, :8], angle, interleaved, wq, 1e-6)       # (other strides may go another way)
        check_forward(k, other[:, 2:39, 8:], angle, interleaved, wk, 1e-6)
        assert bool((other[:, :2] == 7).all()) and bool((other[:, 39:] == 7).all())             # what lies around it is left
        for i in range(2):                        # over the gradients, over the inputs (copies that may stand closer together)
            copies = [t.clone() for t in (gq, gk, q, k)]
            into = tuple(copies[2 * i:2 * i + 2])
            got = P.norm_rotate_backward(*copies, wq, wk, positions, inv_freq, axes, interleaved=interleaved, out=into)
            assert got[0] is into[0] and got[1] is into[1]
            check_backward(q, gq, got[0], got[2], angle, interleaved, wq, 1e-6, layout)
            check_backward(k, gk, got[1], got[3], angle, interleaved, wk, 1e-6, layout)
        before = q.clone()
        P.norm_rotate(q, k, wq, wk, positions, inv_freq, axes, interleaved=interleaved, out=(q, k))
        check_forward(before, q, angle, interleaved, wq, 1e-6)
        check_forward(before, want[0], angle, interleaved, wq, 1e-6)
        before = q.clone()
        turned_again = P.rotate(q, k, positions, inv_freq, axes, interleaved=interleaved, out=(q, k))
        assert turned_again[0] is q
        check_forward(before, q, angle, interleaved)


@pytest.mark.parametrize("size", [128, 72, 80, 50])
def test_values_that_are_not_numbers_stay_in_their_rows(size):
    q, k, positions, inv_freq, axes, wq, wk = make((1, 20, 4, 2, size, size), torch.bfloat16)
    bad = q.clone()
    bad[0, 3, 1, 5] = math.nan
    bad[0, 4, 2, size - 1] = math.inf
    bad[0, 5, 3, size // 2] = torch.finfo(torch.bfloat16).min
    plain, norm = P.rotate(q, k, positions, inv_freq, axes)[0], P.norm_rotate(q, k, wq, wk, positions, inv_freq, axes)[0]
    got, got_norm = P.rotate(bad, k, positions, inv_freq, axes)[0], P.norm_rotate(bad, k, wq, wk, positions, inv_freq, axes)[0]
    hit = torch.zeros(20, 4, dtype=torch.bool, device="cuda")
    hit[3, 1] = hit[4, 2] = hit[5, 3] = True
    assert torch.equal(got[0][~hit], plain[0][~hit]) and torch.equal(got_norm[0][~hit], norm[0][~hit])
    assert bool(got[0, 3, 1, [5, 5 + size // 2]].isnan().all()) and int(got[0, 3, 1].isnan().sum()) == 2
    assert bool(got_norm[0, 3, 1].isnan().all())
    g = torch.randn_like(q)
    dx, dx_bad = (P.norm_rotate_backward(g, None, x, None, wq, None, positions, inv_freq, axes)[0] for x in (q, bad))
    assert torch.equal(dx[0][~hit], dx_bad[0][~hit]) and bool(dx_bad[0, 3, 1].isnan().all())
    # a row of zeros: 1 / sqrt(eps) times nothing
    zero = P.norm_rotate(torch.zeros_like(q), k, wq, wk, positions, inv_freq, axes)[0]
    assert bool((zero == 0).all())
    g = torch.randn_like(q)
    dx = P.norm_rotate_backward(g, None, torch.zeros_like(q), None, wq, None, positions, inv_freq, axes)
    check_backward(torch.zeros_like(q), g, dx[0], dx[2], angle_of(positions, inv_freq, axes), False, wq, 1e-6)


@pytest.mark.parametrize("size", [128, 72])
def test_an_infinite_gradient_in_the_last_token(size):
    """Lanes without a token go along with the last one's data: they add nothing to the weights' gradient, no 0 * inf either."""
    for tokens in (1, 5, 6, 7):
        q, _, positions, inv_freq, axes, w, _ = make((1, tokens, 2, 0, size, size), torch.float32, seed=3)
        g = torch.randn_like(q)
        g[0, -1, 1, 3] = math.inf
        _, _, dw, _ = P.norm_rotate_backward(g, None, q, None, w, None, positions, inv_freq, axes)
        half = size // 2
        assert bool(dw[[3, 3 + half]].isinf().all())
        others = torch.ones(size, dtype=torch.bool, device="cuda")
        others[[3, 3 + half]] = False
        assert bool(dw[others].isfinite().all())


def test_offsets_past_32_bits():
    # two tokens 2^31 + 256 elements apart, and heads as far
    far = (1 << 31) + 256
    buf = torch.zeros(far + 4 * 128, dtype=torch.bfloat16, device="cuda")
    q = torch.as_strided(buf, (1, 2, 2, 128), (0, far, 128, 1))
    q.copy_(torch.randn(1, 2, 2, 128, device="cuda"))
    _, _, positions, inv_freq, axes, wq, _ = make((1, 2, 2, 0, 128, 128), torch.bfloat16)
    angle = angle_of(positions, inv_freq, axes)
    before = q.clone()
    check_forward(q, P.norm_rotate(q, None, wq, None, positions, inv_freq, axes)[0], angle, False, wq, 1e-6)
    y = P.norm_rotate(before, None, wq, None, positions, inv_freq, axes, out=(q, None))[0]
    assert y.data_ptr() == buf.data_ptr()
    check_forward(before, q, angle, False, wq, 1e-6)
    assert bool((buf[256:far] == 0).all())
    heads = torch.as_strided(buf, (1, 2, 2, 128), (0, 128, far, 1))
    check_forward(heads, P.rotate(heads, None, positions, inv_freq, axes)[0], angle, False)
    del buf


def test_shared_heads_and_slices_of_one_buffer():
    """Keys broadcast over heads, and queries and keys turned in place inside one projection's output."""
    q, k, positions, inv_freq, axes, wq, wk = make((2, 19, 8, 1, 64, 64), torch.bfloat16)
    shared = k.expand(-1, -1, 4, -1)
    y = P.norm_rotate(q, shared, wq, wk, positions, inv_freq, axes)
    one = P.norm_rotate(q, k, wq, wk, positions, inv_freq, axes)
    assert y[1].shape == shared.shape and torch.equal(y[1], one[1].expand(-1, -1, 4, -1))
    g = torch.randn_like(y[1])
    dk = P.norm_rotate_backward(torch.randn_like(q), g, q, shared, wq, wk, positions, inv_freq, axes)
    check_backward(shared, g, dk[1], dk[3], angle_of(positions, inv_freq, axes), False, wk, 1e-6)
    qkv = torch.cat([q, k, torch.randn_like(k)], 2)
    value = qkv[:, :, 9:].clone()
    P.norm_rotate(qkv[:, :, :8], qkv[:, :, 8:9], wq, wk, positions, inv_freq, axes, out=(qkv[:, :, :8], qkv[:, :, 8:9]))
    assert torch.equal(qkv[:, :, :8], one[0]) and torch.equal(qkv[:, :, 8:9], one[1]) and torch.equal(qkv[:, :, 9:], value)


@pytest.mark.parametrize("heads", [(1, 1), (300, 0), (129, 3)])
def test_many_and_few_heads(heads):
    q, k, positions, inv_freq, axes, wq, wk = make((1, 37, *heads, 64, 64), torch.float16, "packed")
    angle = angle_of(positions, inv_freq, axes)
    wk = wk if heads[1] else None
    y = P.norm_rotate(q, k, wq, wk, positions, inv_freq, axes)
    gq, gk = torch.randn_like(q), None if k is None else torch.randn_like(k)
    b = P.norm_rotate_backward(gq, gk, q, k, wq, wk, positions, inv_freq, axes)
    for i, (x, g, w) in enumerate([(q, gq, wq), (k, gk, wk)]):
        if x is not None:
            check_forward(x, y[i], angle, False, w, 1e-6)
            check_backward(x, g, b[i], b[2 + i], angle, False, w, 1e-6)


def test_nothing_to_do():
    _, _, positions, inv_freq, axes, wq, wk = make((1, 4, 1, 1, 64, 64), torch.bfloat16)
    for shape in ((0, 4), (64, 0)):
        q = torch.empty(*shape, 64, dtype=torch.bfloat16, device="cuda")
        p = positions[:, 0, :0] if shape[0] == 0 else torch.zeros(3, 64, dtype=torch.int32, device="cuda")
        y = P.rotate(q, q, p, inv_freq, axes)
        assert y[0].shape == q.shape
        got = P.norm_rotate_backward(q, q, q, q, wq, wk, p, inv_freq, axes)
        assert bool((got[2] == 0).all()) and bool((got[3] == 0).all())
    # keys without heads beside queries that have some
    q, none = torch.randn(4, 2, 64, device="cuda"), torch.empty(4, 0, 64, device="cuda")
    got = P.norm_rotate_backward(torch.randn_like(q), none, q, none, wq.float(), wk.float(), positions[:, 0], inv_freq, axes)
    assert bool((got[3] == 0).all()) and not bool((got[2] == 0).all())


def test_graphs_and_streams():
    """Two captured graphs of the same call replayed in turn and at once, and a call on another stream."""
    sets = [make((1, 513, 8, 2, 128, 128), torch.bfloat16, seed=s) for s in (0, 2)]
    grads = [(torch.randn_like(s[0]), torch.randn_like(s[1])) for s in sets]

    def step(s, g):
        y = P.norm_rotate(s[0], s[1], s[5], s[6], *s[2:5])
        return (*y, *P.norm_rotate_backward(*g, s[0], s[1], s[5], s[6], *s[2:5]))

    want = [step(s, g) for s, g in zip(sets, grads)]
    side = torch.cuda.Stream()
    graphs, outs = [], []
    for s, g in zip(sets, grads):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step(s, g))
        graphs.append(graph)
    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graphs[1].replay()
        graphs[0].replay()
        torch.cuda.current_stream().wait_stream(side)
        for got, w in zip(outs, want):
            assert all(torch.equal(a, b) for a, b in zip(got, w))
    side.wait_stream(torch.cuda.current_stream())
    s, g = sets[0], grads[0]
    got = P.norm_rotate_backward(*g, s[0], s[1], s[5], s[6], *s[2:5], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want[0][2:]))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("size,rot", [(72, 72), (10, 4), (33, 32)])
def test_gradients_against_differences(size, rot, interleaved):
    """sum(g * f(x)) moves as the gradients say: the formula's gradient against differences of the formula in 64 bits, and the
    kernel's against the formula's (check_backward)."""
    q, k, positions, inv_freq, axes, wq, wk = make((1, 5, 2, 1, size, rot), torch.float32, far=100)
    g = torch.randn_like(q)
    angle, eps = angle_of(positions, inv_freq, axes), 1e-6

    def f(x, w):
        return (turned(x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w, angle, interleaved)[0] * g.double()).sum()

    dx, _, dw, _ = P.norm_rotate_backward(g, None, q, None, wq, None, positions, inv_freq, axes, eps=eps, interleaved=interleaved)
    check_backward(q, g, dx, dw, angle, interleaved, wq, eps)
    step = 1e-5
    for direction in (torch.randn_like(q).double(), None):
        if direction is not None:
            moved = (f(q.double() + step * direction, wq.double()) - f(q.double() - step * direction, wq.double())) / (2 * step)
            said, scale = (dx.double() * direction).sum(), (dx.double() * direction).abs().sum()
        else:
            turn = torch.randn_like(wq).double()
            moved = (f(q.double(), wq.double() + step * turn) - f(q.double(), wq.double() - step * turn)) / (2 * step)
            said, scale = (dw.double() * turn).sum(), (dw.double() * turn).abs().sum()
        # the difference is off by third derivatives times step^2 (1e-10) and by 64-bit rounding over the step (1e-11); the kernel
        # by what check_backward allows, 128 u of terms that can cancel
        assert abs(float(moved - said)) <= 1e-4 * float(scale) + 1e-6
    # the rotation alone: its gradient is the inverse rotation
    gz = P.rotate(g, None, positions, inv_freq, axes, interleaved=interleaved, inverse=True)[0]
    check_forward(g, gz, -angle, interleaved)


def test_heads_whose_elements_do_not_stand_side_by_side():
    # as gradients come out of a product of matrices
    q, k, positions, inv_freq, axes, wq, wk = make((2, 9, 4, 2, 64, 64), torch.bfloat16)
    gq, gk = torch.randn_like(q), torch.randn_like(k)
    want = P.norm_rotate_backward(gq, gk, q, k, wq, wk, positions, inv_freq, axes)
    apart = [t.permute(3, 0, 2, 1).contiguous().permute(1, 3, 2, 0) for t in (gq, gk, q, k)]
    assert all(t.stride(-1) != 1 for t in apart)
    got = P.norm_rotate_backward(*apart, wq, wk, positions, inv_freq, axes)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(ValueError):
        P.rotate(q, k, positions, inv_freq, axes, out=(apart[2], k))


def test_refusals():
    q, k, positions, inv_freq, axes, wq, wk = make((2, 5, 4, 2, 64, 64), torch.bfloat16)
    ok = lambda **kw: P.norm_rotate(kw.get("q", q), kw.get("k", k), kw.get("wq", wq), kw.get("wk", wk), kw.get("positions", positions),  # noqa: E731
                                    kw.get("inv_freq", inv_freq), kw.get("axes", axes), **{n: v for n, v in kw.items() if n in ("eps", "out", "stream")})
    ok()
    for bad in (dict(q=q[0, 0]), dict(k=k[:1]), dict(k=k.float()), dict(k=k[..., :32]), dict(q=q.double(), k=None), dict(positions=positions.long()),
                dict(positions=positions[:, :1]), dict(inv_freq=inv_freq[:5]), dict(axes=axes.long()), dict(wq=wq[:5]), dict(wq=wq.half()),
                dict(wq=wq.float()), dict(inv_freq=inv_freq.half()), dict(q=q.transpose(2, 3)), dict(positions=positions.cpu()), dict(q=q.cpu(), k=k.cpu()),
                dict(out=(q, q)), dict(out=(q,)), dict(out=(q.float(), k)), dict(q=q.clone().requires_grad_())):
        with pytest.raises((ValueError, P.PcrError)):
            ok(**bad)
    shared = torch.zeros(2, 5, 1, 64, dtype=torch.bfloat16, device="cuda").expand(-1, -1, 4, -1)
    for bad in (dict(eps=-1.0), dict(eps=math.nan), dict(positions=positions.repeat(2, 1, 1)), dict(out=(shared, torch.empty_like(k))),
                dict(inv_freq=inv_freq.repeat(2), axes=axes.repeat(2))):
        with pytest.raises(P.PcrError) as e:
            ok(**bad)
        assert e.value.code == -1
    with pytest.raises(ValueError):
        P.norm_rotate_backward(q, k, q, k[:, :, :1], wq, wk, positions, inv_freq, axes)
    with pytest.raises(ValueError):
        P.norm_rotate_backward(q, None, q, None, wq, wk, positions, inv_freq, axes)
    big = torch.zeros(1, 1, 520, device="cuda")
    with pytest.raises(P.PcrError):
        P.rotate(big, None, positions[:, 0, :1], inv_freq, axes)
    torch.cuda.synchronize()
