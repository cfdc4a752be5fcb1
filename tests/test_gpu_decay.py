"""Linear attention with a decay for each head (decay_attention, its backward pass, decay_step) against its definition in 64 bits.

Tolerances, per element; u = 2^-24.  An output is a sum of terms w (q . k) v with w = f^n, a memory one of w k v.
* w: its exponent n log2 f carries two roundings, so w is off by at most 2 |ln w| u, and by 4 u of exp2 and the products it is put
  together from within a chunk.  A memory that goes over c chunks is multiplied c times by such a factor: 4 c u more.
* sums: up to `size` products and the tokens of a chunk (128 at most) and one addition a chunk, in any order: (size + 128 + c) u.
  Together at most (size + 160 + 5 c) u times E = the sum over |w| (1 + 2 |ln w|) |q| . |k| |v|; gradients likewise.
* 16-bit operands, eps / 2 the largest relative error of a rounding: products of queries and keys and the memory are rounded once for
  the tensor cores, both of magnitude E at most, the output once: eps E + eps / 2 |out|.  Keys that go into a memory are kept in two
  parts, off by eps^2 / 4, and in three where the memory is given out.  fp16 parts have no bits below 2^-25: that much of |q| . 1 |v|.
* gradients of shared heads: each head's sum as above, added up in 32 bits, rounded once.
"""
import math

import pytest
import torch

import paper_1911_00472_b200 as P

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = [torch.bfloat16, torch.float16, torch.float32]
DEV = "cuda:0"


def weights(rate, n):
    """(f^(t-j), its logarithm) for j <= t, 0 above."""
    d = torch.arange(n, device=DEV, dtype=torch.float64)
    d = d[:, None] - d
    ln = torch.where(d > 0, rate * d.clamp(min=0), torch.zeros_like(d))
    return torch.where(d >= 0, ln.exp(), torch.zeros_like(d)), ln.abs().nan_to_num(0, 0, 0)


def walk(a, b, c, rate, first, reverse=False, aged=True):
    """(sums, magnitudes, memory behind the last token, its magnitude) of one head, (tokens, size) each, in 64 bits."""
    if reverse:
        a, b, c = a.flip(0), b.flip(0), c.flip(0)
    n = a.shape[0]
    w, ln = weights(rate, n)
    y = ((a @ b.T) * w) @ c
    E = ((a.abs() @ b.abs().T) * w * (1 + 2 * ln)) @ c.abs()
    step = torch.arange(n, device=DEV, dtype=torch.float64)
    shift = 1 if aged else 0                                     # forward: what was there before ages on its way to the first token
    age = torch.where(step + shift > 0, rate * (step + shift), torch.zeros_like(step))
    y = y + (a @ first) * age.exp()[:, None]
    E = E + (a.abs() @ first.abs()) * (age.exp() * (1 + 2 * age.abs().nan_to_num(0, 0, 0)))[:, None]
    back = torch.where(step.flip(0) > 0, rate * step.flip(0), torch.zeros_like(step))
    fade = back.exp()
    times = n if aged else max(n - 1, 0)
    total = rate * times if times else 0.0
    kept = math.exp(total)
    last = (b * fade[:, None]).T @ c + first * kept
    M = (b.abs() * (fade * (1 + 2 * back.abs().nan_to_num(0, 0, 0)))[:, None]).T @ c.abs() + first.abs() * (kept * (1 + 2 * abs(total)) if kept else 0.0)
    if reverse:
        y, E = y.flip(0), E.flip(0)
    return y, E, last, M


def near(got, want, E, dtype, size, tokens, what, memory=False, extra=0.0):
    eps = 0.0 if dtype == torch.float32 else torch.finfo(dtype).eps
    c = tokens // 32 + 1
    tol = (size + 160 + 5 * c) * U * E + extra
    if memory:
        tol = tol + (eps / 2) ** (2 if dtype == torch.float16 else 3) * E
    else:
        tol = tol + eps * E + eps / 2 * want.abs() + torch.finfo(got.dtype).tiny
    off = (got.double() - want).abs()
    assert torch.isfinite(got).all(), what
    worst = (off / tol.clamp(min=1e-300)).max() if off.numel() else 0.0
    assert worst <= 1.0, (what, float(worst), float(off.max()))


def make(lengths, hq, hk, kd, vd, dtype, layout="plain", packed=True, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed + 31 * kd + hq)
    n = sum(lengths) if packed else lengths[0]
    shape = (n,) if packed else (len(lengths), n)

    def block(h, d, scale=1.0):
        if layout == "slices":                                       # of one projection's output
            x = torch.randn(*shape, h + 2, d, device=DEV, generator=g)[..., 1:1 + h, :]
        elif layout == "shifted":                                    # rows at odd elements, odd strides
            x = torch.randn(*shape, h * d + 3, device=DEV, generator=g)[..., 1:1 + h * d].unflatten(-1, (h, d))
        elif layout == "heads_first":
            x = torch.randn(h, *shape, d, device=DEV, generator=g).movedim(0, -2)
        else:
            x = torch.randn(*shape, h, d, device=DEV, generator=g)
        return x.mul_(scale).to(dtype)                               # (to() keeps strides; a slice in 32 bits stays one)

    def kept(x):                                                     # conversions make slices dense: lay the 16-bit ones out again
        if layout == "plain" or layout == "heads_first" or dtype == torch.float32:
            return x
        h, d = x.shape[-2:]
        if layout == "slices":
            y = torch.zeros(*shape, h + 2, d, device=DEV, dtype=dtype)[..., 1:1 + h, :]
        else:
            y = torch.zeros(*shape, h * d + 3, device=DEV, dtype=dtype)[..., 1:1 + h * d].unflatten(-1, (h, d))
        return y.copy_(x)

    q, k, v, gr = kept(block(hq, kd, kd ** -0.5)), kept(block(hk, kd)), kept(block(hk, vd)), kept(block(hq, vd))
    starts = None
    if packed:
        starts = torch.tensor([0, *torch.tensor(lengths).cumsum(0).tolist()], dtype=torch.int32, device=DEV)
    log_decay = -torch.exp2(-6.0 * torch.arange(hq, device=DEV, dtype=torch.float32) / hq)
    mem = lambda: torch.randn(len(lengths), hq, kd, vd, device=DEV, generator=g)
    return q, k, v, gr, starts, log_decay, mem(), mem()


def rows_of(x, i, lengths, packed, head):
    if packed:
        at = sum(lengths[:i])
        return x[at:at + lengths[i], head].double()
    return x[i, :, head].double()


def check_forward(args, lengths, packed, out, after, first):
    q, k, v, _, _, log_decay, _, _ = args
    group, kd = q.shape[-2] // k.shape[-2], q.shape[-1]
    for i, n in enumerate(lengths):
        for h in range(q.shape[-2]):
            a, b, c = (rows_of(x, i, lengths, packed, j) for x, j in ((q, h), (k, h // group), (v, h // group)))
            before = first[i, h].double() if first is not None else torch.zeros(kd, v.shape[-1], device=DEV, dtype=torch.float64)
            y, E, last, M = walk(a, b, c, float(log_decay[h]), before)
            extra = 2.0 ** -25 * n * a.abs().sum(-1, keepdim=True) * c.abs().max() if q.dtype == torch.float16 and n else 0.0
            near(rows_of(out, i, lengths, packed, h).to(out.dtype), y, E, q.dtype, kd, n, ("out", i, h), extra=extra)
            if after is not None:
                near(after[i, h], last, M, q.dtype, 0, n, ("memory", i, h), memory=True, extra=2.0 ** -25 * n * 4 if q.dtype == torch.float16 else 0.0)


def check_backward(args, lengths, packed, got, first, dafter):
    q, k, v, g, _, log_decay, _, _ = args
    hq, group, kd, vd = q.shape[-2], q.shape[-2] // k.shape[-2], q.shape[-1], v.shape[-1]
    dq, dk, dv, before = got
    zero = torch.zeros(kd, vd, device=DEV, dtype=torch.float64)
    for i, n in enumerate(lengths):
        sums = {}
        for h in range(hq):
            rate = float(log_decay[h])
            a, b, c, o = (rows_of(x, i, lengths, packed, j) for x, j in ((q, h), (k, h // group), (v, h // group), (g, h)))
            s0 = zero if first is None else first[i, h].double()
            s1 = zero if dafter is None else dafter[i, h].double()
            extra = 2.0 ** -22 * n if q.dtype == torch.float16 and n else 0.0
            y, E, _, _ = walk(o, c, b, rate, s0.T)
            near(rows_of(dq, i, lengths, packed, h).to(dq.dtype), y, E, q.dtype, vd, n, ("dq", i, h), extra=extra)
            for name, x in (("dk", walk(c, o, a, rate, s1.T, True, False)), ("dv", walk(b, a, o, rate, s1, True, False))):
                old = sums.get((name, h // group))
                sums[name, h // group] = x[:2] if old is None else (old[0] + x[0], old[1] + x[1])
                if name == "dv" and before is not None:
                    f = math.exp(rate) if n else 1.0
                    near(before[i, h], x[2] * f, x[3] * f, q.dtype, 0, n, ("dstate", i, h), memory=True, extra=extra)
        for (name, h), (y, E) in sums.items():
            near(rows_of(dk if name == "dk" else dv, i, lengths, packed, h).to(dk.dtype), y, E, q.dtype, max(kd, vd), n, (name, i, h), extra=extra * group)


# lengths, heads of queries, of keys, sizes
SHAPES = [
    ([1], 1, 1, 1, 1), ([1], 3, 1, 64, 64), ([2, 0, 1], 2, 2, 16, 32), ([127], 2, 1, 64, 64), ([128], 2, 2, 128, 128), ([129, 1, 64], 2, 1, 128, 128),
    ([257], 4, 2, 72, 72), ([300, 5, 0, 0, 131], 3, 3, 80, 48), ([700], 1, 1, 64, 128), ([65, 66], 2, 2, 128, 32), ([33], 2, 1, 20, 12), ([40, 90], 2, 2, 33, 7),
    ([70], 2, 1, 200, 256), ([1500], 2, 1, 64, 64), ([100, 1300, 3], 1, 1, 96, 96), ([190], 1, 1, 136, 64),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(shape, dtype):
    lengths, hq, hk, kd, vd = shape
    args = make(lengths, hq, hk, kd, vd, dtype)
    q, k, v, _, starts, log_decay, first, _ = args
    out, after = P.decay_attention(q, k, v, log_decay, starts=starts, state=first, final=True)
    check_forward(args, lengths, True, out, after, first)
    again, none = P.decay_attention(q, k, v, log_decay, starts=starts, state=first)
    assert none is None
    check_forward(args, lengths, True, again, None, first)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_backward(shape, dtype):
    lengths, hq, hk, kd, vd = shape
    args = make(lengths, hq, hk, kd, vd, dtype, seed=3)
    q, k, v, g, starts, log_decay, first, dafter = args
    got = P.decay_attention_backward(g, q, k, v, log_decay, starts=starts, state=first, grad_final=dafter, grad_state=True)
    check_backward(args, lengths, True, got, first, dafter)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", ["slices", "shifted", "heads_first"])
@pytest.mark.parametrize("shape", [(3, 150, 2, 1, 64, 64), (2, 400, 3, 3, 128, 72), (5, 1, 2, 2, 32, 32), (1, 260, 2, 2, 24, 40)], ids=str)
def test_batches_and_layouts(shape, layout, dtype):
    b, s, hq, hk, kd, vd = shape
    lengths = [s] * b
    args = make(lengths, hq, hk, kd, vd, dtype, layout, packed=False, seed=5)
    q, k, v, g, _, log_decay, first, _ = args
    out, after = P.decay_attention(q, k, v, log_decay, final=True)
    check_forward(args, lengths, False, out, after, None)
    check_backward(args, lengths, False, P.decay_attention_backward(g, q, k, v, log_decay), None, None)


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_segments(dtype):
    """Sequences long enough for several segments, one of them ending in the middle of everything."""
    lengths = [5000, 1, 2049, 0, 700]
    args = make(lengths, 2, 1, 64, 64, dtype, seed=7)
    q, k, v, g, starts, _, first, dafter = args
    log_decay = torch.tensor([-0.001, -0.03], device=DEV)
    args = (*args[:5], log_decay, *args[6:])
    out, after = P.decay_attention(q, k, v, log_decay, starts=starts, state=first, final=True)
    check_forward(args, lengths, True, out, after, first)
    got = P.decay_attention_backward(g, q, k, v, log_decay, starts=starts, state=first, grad_final=dafter, grad_state=True)
    check_backward(args, lengths, True, got, first, dafter)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rate", [0.0, -math.inf, -40.0, -1e-6])
def test_ends_of_the_decays(rate, dtype):
    lengths = [300, 20]
    args = make(lengths, 2, 2, 64, 64, dtype, seed=9)
    q, k, v, g, starts, _, first, dafter = args
    log_decay = torch.full((2,), rate, device=DEV)
    args = (*args[:5], log_decay, *args[6:])
    out, after = P.decay_attention(q, k, v, log_decay, starts=starts, state=first, final=True)
    check_forward(args, lengths, True, out, after, first)
    got = P.decay_attention_backward(g, q, k, v, log_decay, starts=starts, state=first, grad_final=dafter, grad_state=True)
    check_backward(args, lengths, True, got, first, dafter)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [64, 128, 36])
def test_rows_of_no_sequence(size, dtype):
    q, k, v, g, _, log_decay, _, _ = args = make([500], 2, 1, size, size, dtype, seed=11)
    starts = torch.tensor([7, 200, 200, 431], dtype=torch.int32, device=DEV)
    out, _ = P.decay_attention(q, k, v, log_decay, starts=starts)
    assert not out[:7].any() and not out[431:].any() and out[7:431].any(-1).all()
    given = torch.full_like(out, 3.0)
    P.decay_attention(q, k, v, log_decay, starts=starts, out=given)
    assert (given[:7] == 3).all() and (given[431:] == 3).all() and torch.equal(given[7:431], out[7:431])
    cut = tuple(x[7:431] for x in args[:4])
    check_forward((*cut, None, log_decay, None, None), [193, 0, 231], True, out[7:431], None, None)
    grads = P.decay_attention_backward(g, q, k, v, log_decay, starts=starts)
    kept = [torch.full_like(x, 3.0) for x in (q, k, v)]
    P.decay_attention_backward(g, q, k, v, log_decay, starts=starts, out=kept)
    for x, y in zip(grads, kept):
        assert not x[:7].any() and not x[431:].any() and (y[:7] == 3).all() and (y[431:] == 3).all() and torch.equal(x[7:431], y[7:431])
    check_backward((*cut, None, log_decay, None, None), [193, 0, 231], True, (*(x[7:431] for x in grads[:3]), None), None, None)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("size", [64, 128, 36])
def test_a_token_that_is_not_finite_reaches_none_that_do_not_see_it(size, value, dtype):
    lengths = [150, 200, 130]
    q, k, v, g, starts, log_decay, _, _ = make(lengths, 2, 1, size, size, dtype, seed=13)
    clean, _ = P.decay_attention(q, k, v, log_decay, starts=starts)
    grads = P.decay_attention_backward(g, q, k, v, log_decay, starts=starts)
    bad = 150 + 77
    eps = torch.finfo(dtype).eps
    for which in range(3):
        x = [t.clone() for t in (q, k, v)]
        x[which][bad] = value
        out, _ = P.decay_attention(*x, log_decay, starts=starts)
        for part in (slice(0, bad), slice(350, None)):
            assert torch.isfinite(out[part]).all()
            assert torch.allclose(out[part].double(), clean[part].double(), rtol=4 * eps, atol=8 * eps * float(clean.abs().max()))
    dirty = g.clone()
    dirty[bad] = value
    got = P.decay_attention_backward(dirty, q, k, v, log_decay, starts=starts)
    for x, y, seen in zip(got, grads, (slice(bad, bad + 1), slice(150, bad + 1), slice(150, bad + 1))):
        fine = torch.ones(len(q), dtype=torch.bool, device=DEV)
        fine[seen] = False
        assert torch.isfinite(x[fine]).all()
        assert torch.allclose(x[fine].double(), y[fine].double(), rtol=4 * eps, atol=8 * eps * float(y.abs().max()))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads", [(2, 1), (4, 4)])
def test_gradients_against_differences(heads, dtype):
    """The backward pass is that of the forward pass: the change of a weighted sum of outputs and memories along a direction, from the
    definition in 64 bits at both ends of a step of 2^-10, off by the step's square."""
    lengths = [50, 90]
    q, k, v, g, starts, log_decay, first, dafter = make(lengths, *heads, 24, 40, dtype, seed=15)
    got = P.decay_attention_backward(g, q, k, v, log_decay, starts=starts, state=first, grad_final=dafter, grad_state=True)
    gen = torch.Generator(device=DEV).manual_seed(1)
    group = heads[0] // heads[1]

    def loss(x):
        total = 0.0
        for i, n in enumerate(lengths):
            at = sum(lengths[:i])
            for h in range(heads[0]):
                y, _, last, _ = walk(x[0][at:at + n, h], x[1][at:at + n, h // group], x[2][at:at + n, h // group], float(log_decay[h]), x[3][i, h])
                total += float((y * g[at:at + n, h].double()).sum() + (last * dafter[i, h].double()).sum())
        return total

    at = [t.double() for t in (q, k, v, first)]
    for which in range(4):
        d = torch.randn(at[which].shape, device=DEV, generator=gen, dtype=torch.float64)
        step = 2.0 ** -10
        up, down = list(at), list(at)
        up[which], down[which] = at[which] + step * d, at[which] - step * d
        want = (loss(up) - loss(down)) / (2 * step)              # the sum is linear in each operand: exact but for 64-bit rounding
        have = float((got[which].double() * d).sum())
        size = float((got[which].double() * d).norm())           # independent roundings of elements, each eps at most of about its size
        eps = torch.finfo(dtype).eps
        assert abs(have - want) <= 8 * max(eps, 2.0 ** -16) * size + 1e-9 * abs(want), which


# ---- one token at a time ----------------------------------------------------------------------------------------------------


def step_oracle(q, k, v, log_decay, state, slots):
    state, out = state.double(), torch.zeros(*q.shape[:2], v.shape[-1], device=DEV, dtype=torch.float64)
    size, E = out.clone(), state.abs()
    group = q.shape[1] // k.shape[1]
    f = log_decay.double().exp()[:, None, None]
    for i, s in enumerate(slots):
        if 0 <= s < len(state):
            kk, vv = k[i].double().repeat_interleave(group, 0), v[i].double().repeat_interleave(group, 0)
            state[s] = f * state[s] + kk[:, :, None] * vv[:, None, :]
            E[s] = f * E[s] + (kk[:, :, None] * vv[:, None, :]).abs()
            out[i] = (q[i].double()[:, :, None] * state[s]).sum(1)
            size[i] = (q[i].double().abs()[:, :, None] * E[s]).sum(1)
    return out, size, state, E


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(1, 1, 1, 1, 1), (1, 32, 8, 128, 128), (5, 4, 2, 64, 128), (3, 2, 1, 33, 7), (70, 3, 3, 72, 72), (2, 1, 1, 256, 256), (9, 2, 2, 200, 30)], ids=str)
def test_step(shape, dtype):
    """Factor, product and sum: (4 + size + 8) u of the magnitudes, a rounding to the output's type; several tokens add up."""
    rows, hq, hk, kd, vd = shape
    g = torch.Generator(device=DEV).manual_seed(rows + kd)
    q, k, v = (torch.randn(rows, h, d, device=DEV, generator=g).to(dtype) for h, d in ((hq, kd), (hk, kd), (hk, vd)))
    log_decay = -torch.rand(hq, device=DEV, generator=g)
    state = torch.randn(rows + 3, hq, kd, vd, device=DEV, generator=g)
    slots = torch.randperm(rows + 3, device=DEV, generator=g)[:rows].to(torch.int32)
    if rows > 3:
        slots[1], slots[2], slots[3] = -1, slots[0], slots[0]     # a row of no request, three tokens of one request
    want, size, after, E = step_oracle(q, k, v, log_decay, state, slots.tolist())
    mine = state.clone()
    out = P.decay_step(q, k, v, log_decay, mine, slots=slots)
    assert ((out.double() - want).abs() <= (kd + 24) * U * size + torch.finfo(dtype).eps / 2 * want.abs() + 1e-30).all()
    assert ((mine.double() - after).abs() <= 24 * U * E).all()
    untouched = torch.ones(rows + 3, dtype=torch.bool, device=DEV)
    untouched[slots[(slots >= 0)].long()] = False
    assert torch.equal(mine[untouched], state[untouched])
    plain = state.clone()
    out = P.decay_step(q, k, v, log_decay, plain)                  # row i has memory i
    want, size, after, E = step_oracle(q, k, v, log_decay, state, range(rows))
    assert ((out.double() - want).abs() <= (kd + 24) * U * size + torch.finfo(dtype).eps / 2 * want.abs() + 1e-30).all()
    assert ((plain.double() - after).abs() <= 24 * U * E).all() and torch.equal(plain[rows:], state[rows:])


def test_a_prompt_and_its_continuation():
    """Patch tokens of a record, turned and normed, through a prompt; then token by token from the memory it left: what the whole
    sequence gives in one go."""
    import pcr_synth
    rec = pcr_synth.make_record(0)
    dec = P.Decoder(rec.bytes, device=DEV)
    plan = dec.patch_plan(8, merge=2)
    tokens = dec.decode_patches(10, plan, (0.5,) * 3, (0.25,) * 3, dtype=torch.float32)
    positions, _ = P.token_positions(plan.segments(), len(tokens), dec.n_images, merge=2, restart=True)
    inv_freq, axes = P.rotary_axes(48, sections=(0, 12, 12), per_axis=True)
    q, k = tokens.view(-1, 4, 48).split([3, 1], 1)
    weight = torch.ones(48, device=DEV)
    yq, yk = P.norm_rotate(q, k, weight, weight, positions, inv_freq, axes)
    v = tokens.view(-1, 4, 48)[:, 3:].contiguous()
    n = min(700, len(tokens))
    log_decay = torch.tensor([-0.5, -0.05, -0.005], device=DEV)
    whole, last = P.decay_attention(yq[:n], yk[:n], v[:n], log_decay, final=True)
    prompt = n - 20
    out, memory = P.decay_attention(yq[:prompt], yk[:prompt], v[:prompt], log_decay, final=True)
    for t in range(prompt, n):
        y = P.decay_step(yq[t:t + 1], yk[t:t + 1], v[t:t + 1], log_decay, memory)
        assert torch.allclose(y[0], whole[t], rtol=1e-4, atol=1e-4 * float(whole.abs().max()))
    assert torch.equal(out, whole[:prompt]) or torch.allclose(out, whole[:prompt], rtol=1e-4, atol=1e-4 * float(whole.abs().max()))
    assert torch.allclose(memory, last, rtol=1e-4, atol=1e-4 * float(last.abs().max()))
    dec.close()


# ---- streams, graphs ----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lengths", [[300, 41], [6000]])
def test_captured_and_on_another_stream(lengths, dtype):
    q, k, v, g, starts, log_decay, first, dafter = make(lengths, 4, 2, 64, 64, dtype, seed=17)

    def both():
        return (*P.decay_attention(q, k, v, log_decay, starts=starts, state=first, final=True),
                *P.decay_attention_backward(g, q, k, v, log_decay, starts=starts, state=first, grad_final=dafter, grad_state=True))

    want = [x.clone() for x in both()]
    assert all(torch.equal(x, y) for x, y in zip(want, both()))       # the same call gives the same bits
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    outs = []
    for graph in graphs:
        with torch.cuda.graph(graph):
            outs.append(both())
    for graph in graphs:
        graph.replay()
    torch.cuda.synchronize()
    for got in outs:
        assert all(torch.equal(x, y) for x, y in zip(want, got))
    q.mul_(2.0)                                                       # other values, other sequences in the same memory
    graphs[0].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(both()[:2], outs[0][:2]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, _ = P.decay_attention(q, k, v, log_decay, starts=starts, state=first, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    check = P.decay_attention(q, k, v, log_decay, starts=starts, state=first)[0]
    assert torch.equal(got, check)
    state = first.clone()
    rows = len(lengths)
    graph = torch.cuda.CUDAGraph()
    P.decay_step(q[:rows], k[:rows], v[:rows], log_decay, state)
    with torch.cuda.graph(graph):
        y = P.decay_step(q[:rows], k[:rows], v[:rows], log_decay, state)
    state.copy_(first)
    graph.replay()
    graph.replay()
    again = first.clone()
    P.decay_step(q[:rows], k[:rows], v[:rows], log_decay, again)
    assert torch.equal(P.decay_step(q[:rows], k[:rows], v[:rows], log_decay, again), y) and torch.equal(state, again)
