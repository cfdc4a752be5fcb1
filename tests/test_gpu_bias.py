"""The learned bias of distances (relative_bias) and its table's gradient against plain forms in 64 bits.

Tolerances, per element; u = 2^-24.  A bias is a sum of at most four values in single precision, 3 u of their magnitudes, and one
rounding to the output's type, eps / 2 of the value.  A table's gradient is a sum over pairs: lanes add up at most 256 values each at
these sizes, lanes and warps another 8 times, slabs in 64 bits: 264 u of the sum of magnitudes, and one rounding.
"""
import math

import pytest
import torch

import paper_1911_00472_b200 as P

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = [torch.bfloat16, torch.float16, torch.float32]
DEV = "cuda:0"
# batch, rows, columns, heads, axes, buckets, reach
SHAPES = [
    (None, 1, 1, 1, 1, 2, 1), (None, 1, 4096, 32, 1, 32, 128), (2, 77, 77, 12, 2, 32, 20), (3, 1, 300, 4, 3, 16, 9), (1, 64, 256, 8, 1, 64, 1000), (2, 130, 8, 5, 2, 7, 3),
    (None, 200, 264, 3, 4, 31, 15), (4, 33, 65, 1, 1, 512, 255), (1, 3, 1000, 16, 2, 48, 0), (None, 50, 50, 40, 4, 512, 300), (2, 16, 512, 9, 1, 16, 64),
]


def make(shape, dtype, seed=0, spread=40, packed=False):
    b, nq, nk, heads, axes, buckets, reach = shape
    g = torch.Generator(device=DEV).manual_seed(seed + nk + heads)
    lead = (axes,) if b is None else (axes, b)
    q = torch.randint(-spread, spread, (*lead, nq), device=DEV, generator=g, dtype=torch.int32)
    k = torch.randint(-spread, spread, (*lead, nk), device=DEV, generator=g, dtype=torch.int32)
    table = torch.randn(axes, buckets, heads, device=DEV, generator=g).to(dtype)
    bucket_of = torch.randint(0, buckets, (2 * reach + 1,), device=DEV, generator=g, dtype=torch.int32)
    qi = ki = None
    if packed:
        qi = torch.randint(0, 3, (*lead[1:], nq), device=DEV, generator=g, dtype=torch.int32)
        ki = torch.randint(0, 3, (*lead[1:], nk), device=DEV, generator=g, dtype=torch.int32)
    return table, bucket_of, q, k, qi, ki, g


def buckets_of(bucket_of, q, k, n):
    """(axes, [batch,] rows, columns), -1 where the table has none."""
    reach = bucket_of.shape[0] // 2
    d = (k.long()[..., None, :] - q.long()[..., :, None]).clamp(-reach, reach) + reach
    got = bucket_of.long()[d]
    return torch.where((got >= 0) & (got < n), got, torch.full_like(got, -1))


def oracle(table, bucket_of, q, k, qi, ki):
    t = torch.cat([table.double(), torch.zeros_like(table[:, :1], dtype=torch.float64)], 1)          # -1: the zeros at the end
    n = buckets_of(bucket_of, q, k, table.shape[1])
    parts = [t[a][n[a]].movedim(-1, -3) for a in range(len(t))]
    y, size = sum(parts), sum(p.abs() for p in parts)
    if qi is not None:
        y = y.masked_fill((qi[..., :, None] != ki[..., None, :]).unsqueeze(-3), -math.inf)
    return y, size


def check(got, want, size, dtype):
    assert got.shape == want.shape and got.dtype == dtype
    inf = torch.isinf(want)
    assert torch.equal(inf, torch.isinf(got)) and (got[inf] < 0).all()
    off = (got.double() - want)[~inf].abs()
    assert (off <= 3 * U * size[~inf] + torch.finfo(dtype).eps / 2 * want[~inf].abs() + 1e-12).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_bias(shape, packed, dtype):
    table, bucket_of, q, k, qi, ki, _ = make(shape, dtype, packed=packed)
    want, size = oracle(table, bucket_of, q, k, qi, ki)
    check(P.relative_bias(table, bucket_of, q, k, q_ids=qi, k_ids=ki), want, size, dtype)
    if dtype != torch.float32:
        wide = table.float() * 1.001
        want, size = oracle(wide, bucket_of, q, k, qi, ki)
        check(P.relative_bias(wide, bucket_of, q, k, q_ids=qi, k_ids=ki, dtype=dtype), want, size, dtype)


def grad_oracle(grad, bucket_of, q, k, qi, ki, n):
    g = grad.double()
    if qi is not None:
        g = torch.where((qi[..., :, None] == ki[..., None, :]).unsqueeze(-3), g, torch.zeros_like(g))
    b = buckets_of(bucket_of, q, k, n)
    if g.dim() == 4 and b.dim() == 3:
        b = b[:, None].expand(-1, g.shape[0], -1, -1)
    heads = g.shape[-3]
    got = torch.zeros(len(b), n + 1, heads, device=DEV, dtype=torch.float64)
    size = got.clone()
    for a in range(len(b)):
        at = b[a].flatten()
        at = torch.where(at < 0, torch.full_like(at, n), at)
        flat = g.movedim(-3, -1).reshape(-1, heads)
        got[a].index_add_(0, at, flat)
        size[a].index_add_(0, at, flat.abs())
    return got[:, :n], size[:, :n]


def check_grad(got, want, size):
    assert got.shape == want.shape
    eps = torch.finfo(got.dtype).eps
    assert ((got.double() - want).abs() <= 264 * U * size + eps / 2 * want.abs() + torch.finfo(got.dtype).tiny).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_gradient(shape, packed, dtype):
    table, bucket_of, q, k, qi, ki, gen = make(shape, dtype, seed=1, packed=packed)
    want, _ = oracle(table, bucket_of, q, k, qi, ki)
    grad = torch.randn(want.shape, device=DEV, generator=gen).to(dtype)
    n = table.shape[1]
    args = (bucket_of, q, k)
    check_grad(P.relative_bias_backward(grad, n, *args, q_ids=qi, k_ids=ki), *grad_oracle(grad, *args, qi, ki, n))
    check_grad(P.relative_bias_backward(grad, n, *args, q_ids=qi, k_ids=ki, dtype=dtype), *grad_oracle(grad, *args, qi, ki, n))
    if q.dim() == 2:                                              # all batches have the same positions
        grad = torch.randn(3, *want.shape, device=DEV, generator=gen).to(dtype)
        check_grad(P.relative_bias_backward(grad, n, *args, q_ids=qi, k_ids=ki), *grad_oracle(grad, *args, qi, ki, n))
        one = grad[:1].expand(3, -1, -1, -1)                      # one gradient for all of them
        check_grad(P.relative_bias_backward(one, n, *args, q_ids=qi, k_ids=ki), *grad_oracle(one, *args, qi, ki, n))


@pytest.mark.parametrize("dtype", DTYPES)
def test_layouts(dtype):
    """Slices, transposed heads, positions that are expanded or interleaved, rows that begin anywhere."""
    table, bucket_of, q, k, _, _, gen = make((2, 40, 72, 6, 2, 16, 30), dtype, seed=2)
    want, size = oracle(table, bucket_of, q, k, None, None)
    for out in (torch.zeros(2, 40, 6, 72, device=DEV, dtype=dtype).transpose(1, 2), torch.zeros(2, 6, 40, 80, device=DEV, dtype=dtype)[..., 3:75],
                torch.zeros(2, 6, 41, 73, device=DEV, dtype=dtype)[..., 1:, :72]):
        P.relative_bias(table, bucket_of, q, k, out=out)
        check(out, want, size, dtype)
        grad = torch.randn(out.shape, device=DEV, generator=gen).to(dtype)
        out.copy_(grad)
        check_grad(P.relative_bias_backward(out, 16, bucket_of, q, k), *grad_oracle(grad, bucket_of, q, k, None, None, 16))
    turned = torch.randn(2, 6, 72, 40, device=DEV, generator=gen).to(dtype).transpose(2, 3)
    check_grad(P.relative_bias_backward(turned, 16, bucket_of, q, k), *grad_oracle(turned, bucket_of, q, k, None, None, 16))
    pos = torch.randint(-20, 20, (72, 3), device=DEV, generator=gen, dtype=torch.int32).T[1:]         # an axis's elements lie apart
    shared = pos[:, None].expand(-1, 2, -1)                                                           # both batches' positions
    want, size = oracle(table, bucket_of, shared, shared, None, None)
    check(P.relative_bias(table, bucket_of, shared), want, size, dtype)
    ids = torch.arange(72, device=DEV, dtype=torch.int32) // 30
    want, size = oracle(table, bucket_of, pos, pos, ids, ids)
    check(P.relative_bias(table, bucket_of, pos, q_ids=ids), want, size, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads", [1, 8, 20])
def test_values_that_are_not_finite(heads, dtype):
    """Masked places may hold anything; elsewhere such a value reaches its own bucket and head, no other."""
    table, bucket_of, q, k, qi, ki, gen = make((2, 50, 88, heads, 2, 32, 12), dtype, seed=3, packed=True)
    want, _ = oracle(table, bucket_of, q, k, qi, ki)
    grad = torch.randn(want.shape, device=DEV, generator=gen).to(dtype)
    mask = (qi[..., :, None] != ki[..., None, :]).unsqueeze(1).expand_as(grad)
    clean = P.relative_bias_backward(grad, 32, bucket_of, q, k, q_ids=qi, k_ids=ki)
    dirty = grad.masked_fill(mask, math.nan)
    assert torch.equal(P.relative_bias_backward(dirty, 32, bucket_of, q, k, q_ids=qi, k_ids=ki), clean)
    at = torch.nonzero(~mask[0, 0])[7].tolist()
    for value in (math.inf, -math.inf, math.nan):
        dirty = grad.clone()
        dirty[0, heads - 1, at[0], at[1]] = value
        got = P.relative_bias_backward(dirty, 32, bucket_of, q, k, q_ids=qi, k_ids=ki)
        hit = torch.zeros_like(got, dtype=torch.bool)
        n = buckets_of(bucket_of, q, k, 32)[:, 0, at[0], at[1]]
        for a in range(2):
            hit[a, n[a], heads - 1] = True
        want, size = grad_oracle(grad, bucket_of, q, k, qi, ki, 32)
        assert ((got.double() - want).abs() <= 264 * U * size)[~hit].all()
        assert (torch.isnan(got[hit]) if math.isnan(value) else got[hit] == value).all()
    table[1, 3, 0] = math.inf
    want, size = oracle(table, bucket_of, q, k, qi, ki)
    check_inf = P.relative_bias(table, bucket_of, q, k, q_ids=qi, k_ids=ki)
    assert torch.equal(torch.isinf(check_inf), torch.isinf(want)) and not torch.isnan(check_inf).any()


def test_far_positions_and_buckets_of_no_table():
    table = torch.randn(1, 4, 2, device=DEV)
    pos = torch.tensor([[-2 ** 31, -5, 0, 7, 2 ** 31 - 1]], dtype=torch.int32, device=DEV)
    bucket_of = torch.tensor([0, 1, 2, 3, 4, -1, 2 ** 30], dtype=torch.int32, device=DEV)                # reach 3; three buckets that are none
    want, size = oracle(table, bucket_of, pos, pos, None, None)
    got = P.relative_bias(table, bucket_of, pos)
    check(got, want, size, torch.float32)
    grad = torch.randn(2, 5, 5, device=DEV)
    check_grad(P.relative_bias_backward(grad, 4, bucket_of, pos), *grad_oracle(grad, bucket_of, pos, pos, None, None, 4))


def test_gradient_against_differences():
    table, bucket_of, q, k, qi, ki, gen = make((2, 30, 45, 3, 2, 16, 20), torch.float32, seed=4, packed=True)
    grad = torch.randn(2, 3, 30, 45, device=DEV, generator=gen)
    got = P.relative_bias_backward(grad, 16, bucket_of, q, k, q_ids=qi, k_ids=ki).double()
    d = torch.randn(table.shape, device=DEV, generator=gen, dtype=torch.float64)
    up, down = (oracle(table.double() + s * d, bucket_of, q, k, qi, ki)[0] for s in (0.5, -0.5))
    want = float(((up - down).nan_to_num(0.0, 0.0, 0.0) * grad.double()).sum())                         # (inf - inf where masked)
    assert abs(float((got * d).sum()) - want) <= 1e-4 * float((got * d).norm())


def test_positions_of_packed_images_and_captured():
    """Positions of a batch of images and clips, each a sequence, into a bias and back; captured, replayed with other positions."""
    rows = [(1, 6, 9, 0), (1, 4, 4, 1), (2, 3, 5, 2), (30, 0, 0, 3)]
    segments = torch.tensor(rows, dtype=torch.int32, device=DEV)
    n = 54 + 16 + 30 + 30
    pos, _ = P.token_positions(segments, n, 4, restart=True)
    ids = torch.repeat_interleave(torch.arange(4, device=DEV, dtype=torch.int32), torch.tensor([54, 16, 30, 30], device=DEV))
    bucket_of = P.relative_buckets(32, 16)
    table = torch.randn(3, 32, 8, device=DEV).bfloat16()
    want, size = oracle(table, bucket_of, pos, pos, ids, ids)
    bias = P.relative_bias(table, bucket_of, pos, q_ids=ids)
    check(bias, want, size, torch.bfloat16)
    assert (bias.float().amax(-1) > -1e30).all()                                                       # every token sees itself
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = P.relative_bias(table, bucket_of, pos, q_ids=ids)
        d = P.relative_bias_backward(y.masked_fill(torch.isinf(y), 0.0), 32, bucket_of, pos, q_ids=ids)
    pos.mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    want, size = oracle(table, bucket_of, pos, pos, ids, ids)
    check(y, want, size, torch.bfloat16)
    check_grad(d, *grad_oracle(y.masked_fill(torch.isinf(y), 0.0), bucket_of, pos, pos, ids, ids, 32))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    z = P.relative_bias(table, bucket_of, pos, q_ids=ids, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(z, y)


def test_gradient_of_nearly_as_many_rows_as_31_bits_hold():
    """Shares of the rows whose ends lie beyond 31 bits: no row is left out.  Operands whose strides are 0 stand for 2 147 483 646 rows of a column; all
    sums are whole numbers below 2^24 up to the slabs' in 64 bits."""
    rows = 715827882
    grad = torch.ones(1, 1, 1, 1, device=DEV, dtype=torch.bfloat16).expand(3, 4, rows, 1)
    q = torch.zeros(1, 1, 1, dtype=torch.int32, device=DEV).expand(1, 3, rows)
    k = torch.zeros(1, 3, 1, dtype=torch.int32, device=DEV)
    got = P.relative_bias_backward(grad, 2, torch.tensor([0, 1, 0], dtype=torch.int32, device=DEV), q, k)
    assert not got[0, 0].any() and (got[0, 1] == 3.0 * rows).all()


def test_columns_of_positions_of_their_own_take_the_ids_of_the_rows():
    table, bucket_of, q, k, ids, _, _ = make((2, 60, 60, 4, 2, 32, 20), torch.float32, packed=True)
    bias = P.relative_bias(table, bucket_of, q, k, q_ids=ids)
    assert torch.equal(bias, P.relative_bias(table, bucket_of, q, k, q_ids=ids, k_ids=ids)) and bias.isinf().any()
    grad = torch.randn_like(bias)
    assert torch.equal(P.relative_bias_backward(grad, 32, bucket_of, q, k, q_ids=ids), P.relative_bias_backward(grad, 32, bucket_of, q, k, q_ids=ids, k_ids=ids))
