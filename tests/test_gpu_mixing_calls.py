"""Linear attention with a decay and the bias of distances, called in ways that are allowed and easily forgotten: nothing to do, operands
of odd strides or far apart, several streams and graphs at once.  Every answer is known bit for bit from a plainer call."""
import pytest
import torch

import paper_1911_00472_b200 as P

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DTYPES = [torch.bfloat16, torch.float16, torch.float32]


def operands(shape, hq, hk, kd, vd, dtype, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    new = lambda h, d, s=1.0: (torch.randn(*shape, h, d, device=DEV, generator=g) * s).to(dtype)
    return new(hq, kd, kd ** -0.5), new(hk, kd), new(hk, vd), new(hq, vd), -torch.exp2(-5.0 * torch.arange(hq, device=DEV, dtype=torch.float32) / hq)


def same(got, want):
    for a, b in zip(got, want, strict=True):
        assert (a is None and b is None) or torch.equal(a, b)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hk", [4, 2])
def test_no_sequences(hk, dtype):
    q, k, v, gr, ld = operands((300,), 4, hk, 64, 64, dtype)
    for first in (0, 7, 300):
        starts = torch.full((1,), first, dtype=torch.int32, device=DEV)
        y, last = P.decay_attention(q, k, v, ld, starts=starts, final=True)
        assert last.shape == (0, 4, 64, 64) and not y.any()
        assert not any(x.any() for x in P.decay_attention_backward(gr, q, k, v, ld, starts=starts)[:3])
        out, grads = torch.full_like(y, 3), [torch.full_like(x, 3) for x in (q, k, v)]
        P.decay_attention(q, k, v, ld, starts=starts, out=out)
        P.decay_attention_backward(gr, q, k, v, ld, starts=starts, out=grads)
        assert all((x == 3).all() for x in (out, *grads))


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_tokens(dtype):
    for shape, starts, n in (((3, 0), None, 3), ((0,), torch.zeros(4, dtype=torch.int32, device=DEV), 3), ((0,), None, 1), ((0, 5), None, 0)):
        q, k, v, gr, ld = operands(shape, 4, 2, 32, 16, dtype)
        state = torch.randn(n, 4, 32, 16, device=DEV)
        y, last = P.decay_attention(q, k, v, ld, starts=starts, state=state, final=True)
        assert y.shape == gr.shape and torch.equal(last, state)
        *grads, before = P.decay_attention_backward(gr, q, k, v, ld, starts=starts, grad_final=state, grad_state=True)
        assert [g.shape for g in grads] == [q.shape, k.shape, v.shape] and torch.equal(before, state)
    q, k, v, _, ld = operands((0,), 4, 2, 32, 16, dtype)
    assert P.decay_step(q, k, v, ld, torch.zeros(0, 4, 32, 16, device=DEV)).shape == (0, 4, 16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_heads_and_batches_that_are_one_and_the_same(dtype):
    """Strides of 0: operands that stand for many rows.  They are taken in single precision, as operands of 32 bits are."""
    q, k, v, gr, ld = operands((2, 190), 4, 1, 48, 24, dtype)
    for a, b in ((k[:1].expand(2, -1, -1, -1), v), (k.expand(-1, -1, 4, -1), v.expand(-1, -1, 4, -1)), (k, v[:, :1].expand(-1, 190, -1, -1))):
        y, last = P.decay_attention(q, a, b, ld, final=True)
        y32, last32 = P.decay_attention(q.float(), a.float(), b.float(), ld, final=True)
        same((y, last), (y32.to(dtype), last32))
    one = torch.ones((), device=DEV, dtype=dtype).expand(2, 190, 4, 24)                    # the gradient of a sum
    got = P.decay_attention_backward(one, q, k, v, ld)
    want = P.decay_attention_backward(torch.ones_like(gr), q, k, v, ld)
    same(got, want)


@pytest.mark.parametrize("dtype", DTYPES)
def test_signs_that_are_taken_on_reading(dtype):
    q, k, v, gr, ld = operands((150,), 2, 2, 32, 32, dtype)
    minus = torch._neg_view
    s = torch.cuda.Stream(DEV)
    want, grads = P.decay_attention(-q, k, -v, ld), P.decay_attention_backward(-gr, q, k, -v, ld)
    for stream in (None, s):
        if stream:
            s.wait_stream(torch.cuda.current_stream())
        got = P.decay_attention(minus(q), k, minus(v), ld, stream=stream), P.decay_attention_backward(minus(gr), q, k, minus(v), ld, stream=stream)
        torch.cuda.synchronize()
        same(got[0], want)
        same(got[1], grads)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_far_apart(dtype):
    """Batches 2^32 elements apart, operands and outputs: offsets beyond 32 bits."""
    far, n = 1 << 32, 200
    if torch.cuda.mem_get_info(DEV)[0] < 60 << 30:
        pytest.skip("not enough memory")
    q, k, v, gr, ld = operands((2, n), 2, 1, 64, 64, dtype)
    wide = 2 * 64 * n
    room = torch.empty(far + 8 * wide, device=DEV, dtype=dtype)
    spots = iter(range(8))

    def apart(x, fill=True):
        y = room[next(spots) * wide:].as_strided(x.shape, (far, *x.stride()[1:]))
        return y.copy_(x) if fill else y.zero_()

    a = [apart(x) for x in (q, k, v, gr)]
    out = apart(gr, False)
    want = P.decay_attention(q, k, v, ld)[0]
    assert torch.equal(P.decay_attention(*a[:3], ld, out=out)[0], want)
    grads = [apart(x, False) for x in (q, k, v)]
    same(P.decay_attention_backward(a[3], *a[:3], ld, out=grads)[:3], P.decay_attention_backward(gr, q, k, v, ld)[:3])
    del a, out, grads
    table = torch.randn(1, 8, 3, device=DEV).to(dtype)
    buckets, pos = P.relative_buckets(8, 6, device=DEV), torch.arange(50, device=DEV, dtype=torch.int32).expand(1, 2, 50)
    bias = room.as_strided((2, 3, 50, 50), (far, 2500, 50, 1))
    assert torch.equal(P.relative_bias(table, buckets, pos, out=bias), P.relative_bias(table, buckets, pos))
    assert torch.equal(P.relative_bias_backward(bias, 8, buckets, pos), P.relative_bias_backward(bias.contiguous(), 8, buckets, pos))


def test_memories_far_apart():
    """A memory that begins behind 2^31 elements."""
    if torch.cuda.mem_get_info(DEV)[0] < 30 << 30:
        pytest.skip("not enough memory")
    q, k, v, _, ld = operands((2,), 16, 4, 256, 256, torch.bfloat16)
    state = torch.empty(2200, 16, 256, 256, device=DEV)
    few = torch.randn(2, 16, 256, 256, device=DEV)
    state[0], state[2199] = few[0], few[1]
    got = P.decay_step(q, k, v, ld, state, slots=torch.tensor([2199, 0], dtype=torch.int32, device=DEV))
    want = P.decay_step(q, k, v, ld, few, slots=torch.tensor([1, 0], dtype=torch.int32, device=DEV))
    assert torch.equal(got, want) and torch.equal(state[0], few[0]) and torch.equal(state[2199], few[1])


@pytest.mark.parametrize("dtype", DTYPES)
def test_two_streams_at_once(dtype):
    calls = []
    for seed, shape in ((1, (3000,)), (2, (2, 700))):
        q, k, v, gr, ld = operands(shape, 8, 4, 128, 128, dtype, seed)
        calls.append(lambda q=q, k=k, v=v, gr=gr, ld=ld: (P.decay_attention(q, k, v, ld, final=True), P.decay_attention_backward(gr, q, k, v, ld)))
    want = [c() for c in calls]
    streams = [torch.cuda.Stream(DEV) for _ in calls]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(4):
        for i, (s, c) in enumerate(zip(streams, calls)):
            with torch.cuda.stream(s):
                got.append((i, c()))
    torch.cuda.synchronize()
    for i, (forward, back) in got:
        same(forward, want[i][0])
        same(back, want[i][1])


@pytest.mark.parametrize("dtype", DTYPES)
def test_two_graphs_at_once(dtype):
    """Graphs that were captured one after the other, replayed side by side: neither has workspace of the other's."""
    table = torch.randn(2, 32, 8, device=DEV).to(dtype)
    buckets = P.relative_buckets(32, 60, device=DEV)
    pos = torch.randint(0, 100, (2, 333), device=DEV, dtype=torch.int32)
    rows = torch.randn(8, 333, 333, device=DEV).to(dtype)
    graphs = []
    for seed, shape in ((3, (5000,)), (4, (2, 900))):
        q, k, v, gr, ld = operands(shape, 8, 2, 64, 64, dtype, seed)

        def run(q=q, k=k, v=v, gr=gr, ld=ld):
            return (*P.decay_attention(q, k, v, ld, final=True), *P.decay_attention_backward(gr, q, k, v, ld), P.relative_bias(table, buckets, pos), P.relative_bias_backward(rows, 32, buckets, pos))

        want = run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = run()
        graphs.append((g, got, want, run))                        # (run: what it reads has to stay where it is)
    streams = [torch.cuda.Stream(DEV) for _ in graphs]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for s, (g, got, _, _) in zip(streams, graphs):
            with torch.cuda.stream(s):
                for x in got:
                    if x is not None:
                        x.fill_(5)
                g.replay()
    torch.cuda.synchronize()
    for _, got, want, _ in graphs:
        same(got, want)


def test_positions_of_many_batches():
    """One set of positions for 40000 batches of 32 heads."""
    g = torch.Generator(device=DEV).manual_seed(5)
    rows = torch.randint(-8, 9, (40000, 32, 4, 4), device=DEV, generator=g).float()          # (sums of small whole numbers are exact)
    pos = torch.tensor([[0, 0, 1, 1], [0, 1, 0, 1]], dtype=torch.int32, device=DEV)
    buckets = P.relative_buckets(8, 3, device=DEV)
    got = P.relative_bias_backward(rows, 8, buckets, pos)
    want = torch.zeros(2, 8, 32, dtype=torch.float64, device=DEV)
    total = rows.double().sum(0)
    for a in range(2):
        n = buckets.long()[(pos[a][None, :] - pos[a][:, None]).long() + 3]
        want[a].index_add_(0, n.flatten(), total.flatten(1).T)
    assert torch.equal(got.double(), want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_memory_that_is_no_number(dtype):
    """From a token that is no number on, all that follows in its column is none, over many chunks."""
    q, k, v, gr, ld = operands((2, 2000), 2, 2, 128, 128, dtype)
    clean = P.decay_attention(q, k, v, ld)[0]
    v[0, 3, 1, 5] = float("nan")
    y = P.decay_attention(q, k, v, ld)[0]
    where = torch.zeros_like(y, dtype=torch.bool)
    where[0, 3:, 1, 5] = True
    assert torch.equal(y.isnan(), where)
    # The tokens before it, in that column, are added up once more, with products of queries and keys in 32 bits, which the tensor cores take
    # in 16: off by eps / 2 of E, the sum of magnitudes, and both results are rounded, each by eps / 2 of itself (at most E).  (The sums' own
    # errors are below eps / 2 E in all, 128 + 3 roundings of 2^-24 each.)
    E = torch.tril(q[0, :3, 1].double().abs() @ k[0, :3, 1].double().abs().T) @ v[0, :3, 1, 5].double().abs()
    assert ((y[0, :3, 1, 5].double() - clean[0, :3, 1, 5].double()).abs() <= 2 * torch.finfo(dtype).eps * E).all()
    where[0, :3, 1, 5] = True
    assert torch.equal(y[~where], clean[~where])


@pytest.mark.parametrize("n,dtype", [(4096, torch.float32), (16384, torch.bfloat16), (16384, torch.float16)], ids=str)
def test_long_sums_of_one_sign(n, dtype):
    """Gradients that are all positive, so that nothing hides what a sum loses.  u = 2^-24; every error is relative to the sum itself.
    A sum in the tensor cores goes over 64 columns (32 bits: 12 products, 3 parts of 4) or a row's 1024 (16 bits: 64 products), each of
    which may cut off 2 u.  Those sums are added up by warps, rounded: at most (n rows, n / 1024 blocks of columns, 400 CTAs of 8 warps at
    the least, and one row more) rows times 16 or 1; then 8 warps, then 64 bits, one rounding."""
    g = torch.Generator(device=DEV).manual_seed(6)
    grad = torch.rand(4, n, n, device=DEV, generator=g, dtype=torch.float32).to(dtype)
    pos = torch.arange(n, device=DEV, dtype=torch.int32)[None]
    buckets = P.relative_buckets(32, 128, device=DEV)
    got = P.relative_bias_backward(grad, 32, buckets, pos)[0].double()
    want = torch.zeros(32, 4, dtype=torch.float64, device=DEV)
    for r in range(0, n, 512):
        at = buckets.long()[(pos[0][None, :] - pos[0][r:r + 512][:, None]).long().clamp(-128, 128) + 128]
        want.index_add_(0, at.flatten(), grad[:, r:r + 512].double().flatten(1).T)
    rows = n * (n // 1024) // (400 * 8) + 1
    cut, added = (24, 16 * rows) if dtype == torch.float32 else (128, rows)
    assert ((got - want).abs() <= (cut + added + 8 + 1) * 2.0 ** -24 * want).all()
