"""Outputs of the token operators that the caller gives: what autograd and other operands may still need of that memory."""
import pytest
import torch

import paper_1911_00472_b200 as P

pytestmark = pytest.mark.gpu


def heads(hq=2, hk=2):
    q, k = torch.randn(5, hq, 16, device="cuda"), torch.randn(5, hk, 16, device="cuda")
    inv_freq, axes = P.rotary_axes(16)
    return q, k, torch.arange(5, device="cuda", dtype=torch.int32)[None], inv_freq, axes


def test_autograd_notices_that_a_saved_tensor_was_written_to():
    q, k, positions, inv_freq, axes = heads()
    w = torch.randn(16, device="cuda", requires_grad=True)
    ones = torch.ones(16, device="cuda")
    gq, gk = torch.randn_like(q), torch.randn_like(k)
    for call in (lambda: P.rotate(q, k, positions, inv_freq, axes, out=(q, k)),
                 lambda: P.rotate(q, k, positions, inv_freq, axes, out=(q, k), stream=torch.cuda.Stream()),
                 lambda: P.norm_rotate(q, None, ones, None, positions, inv_freq, axes, out=(q, None)),
                 lambda: P.norm_rotate_backward(gq, gk, q, k, ones, ones, positions, inv_freq, axes, out=(q, k))):
        loss = (q * w).sum()                       # keeps q for w's gradient
        call()
        torch.cuda.synchronize()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    rgb = torch.zeros(192, dtype=torch.uint8, device="cuda")
    plan = P.patch_plan([type("Info", (), dict(out_offset=0, width=8, height=8))], 4)
    tokens, scale = torch.zeros(4, 48, device="cuda"), torch.ones(48, device="cuda", requires_grad=True)
    loss = (tokens * scale).sum()
    P.patch_tokens(rgb, plan.images, plan.index, 4, (0.5,) * 3, (0.5,) * 3, dtype=torch.float32, out=tokens)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    at = torch.zeros(3, 4, dtype=torch.int32, device="cuda")
    table = torch.randn(100, 2, device="cuda", requires_grad=True)
    loss = table[at].sum()
    P.token_positions(plan.segments(), 4, 1, out=at)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    # without an output given nothing that is there is written to
    version = q._version
    P.rotate(q, k, positions, inv_freq, axes)
    assert q._version == version
    with torch.inference_mode():
        inner = torch.randn_like(q)
        P.rotate(inner, None, positions, inv_freq, axes, out=(inner, None))


def test_operands_that_are_stored_negated():
    """A view whose sign is taken on reading (the imaginary part of a conjugate) is turned as what it stands for."""
    q, k, positions, inv_freq, axes = heads()
    wq, wk, gq, gk = torch.randn(16, device="cuda"), torch.randn(16, device="cuda"), torch.randn_like(q), torch.randn_like(k)

    def stored(t):
        n = torch._neg_view(-t)
        assert n.is_neg() and torch.equal(n, t)
        return n

    at = (positions, inv_freq, axes)
    for want, got in ((P.rotate(q, k, *at), P.rotate(stored(q), stored(k), positions, stored(inv_freq), axes)),
                      (P.norm_rotate(q, k, wq, wk, *at), P.norm_rotate(stored(q), stored(k), stored(wq), stored(wk), *at)),
                      (P.norm_rotate_backward(gq, gk, q, k, wq, wk, *at),
                       P.norm_rotate_backward(stored(gq), stored(gk), stored(q), stored(k), stored(wq), stored(wk), *at))):
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    part = torch.view_as_complex(torch.stack([torch.zeros_like(q), -q], -1)).conj().imag          # elements two apart
    assert torch.equal(P.rotate(part, None, *at)[0], P.rotate(q, None, *at)[0])
    with pytest.raises(ValueError):                  # (an output would be read back with the other sign)
        P.rotate(q, None, *at, out=(stored(torch.zeros_like(q)), None))
    rgb = torch.zeros(192, dtype=torch.uint8, device="cuda")
    plan = P.patch_plan([type("Info", (), dict(out_offset=0, width=8, height=8))], 4)
    with pytest.raises(ValueError):
        P.patch_tokens(rgb, plan.images, plan.index, 4, (0.5,) * 3, (0.5,) * 3, dtype=torch.float32, out=stored(torch.zeros(4, 48, device="cuda")))


def test_outputs_that_share_memory_are_refused_and_others_are_not():
    q, k, positions, inv_freq, axes = heads()
    wq, wk, gq, gk = torch.randn(16, device="cuda"), torch.randn(16, device="cuda"), torch.randn_like(q), torch.randn_like(k)
    t, kept = torch.full_like(q, 7.0), (q.clone(), k.clone())
    long = torch.zeros(6, 2, 16, device="cuda")
    long[:5] = q
    calls = [lambda q, k, out: P.rotate(q, k, positions, inv_freq, axes, out=out),
             lambda q, k, out: P.norm_rotate(q, k, wq, wk, positions, inv_freq, axes, out=out),
             lambda q, k, out: P.norm_rotate_backward(gq, gk, q, k, wq, wk, positions, inv_freq, axes, out=out)]
    for call in calls:
        for a, b, out in ((q, k, (k, q)), (q, k, (t, t)), (q, q, (q, t)), (q, k, (t, q)), (q, k, (wq.expand(5, 2, 16), t)),
                          (long[:5], k, (long[1:], t)), (q, k, (t, t.view(-1).as_strided((5, 2, 16), (16, 80, 1))))):
            with pytest.raises(P.PcrError) as e:
                call(a, b, out)
            assert e.value.code == -1
    for out in ((gk, gq), (gk, t), (t, gq)):
        with pytest.raises(P.PcrError):
            calls[2](q, k, out)
    assert torch.equal(q, kept[0]) and torch.equal(k, kept[1]) and bool((t == 7).all())
    for call in calls:
        want = call(q, k, None)
        # queries, keys and their outputs as slices of one buffer, heads between one another
        room = torch.zeros(5, 8, 16, device="cuda")
        room[:, 0::4], room[:, 1::4] = q, k
        got = call(room[:, 0::4], room[:, 1::4], (room[:, 2::4], room[:, 3::4]))
        assert all(torch.equal(a, b) for a, b in zip(want, got)) and torch.equal(room[:, 0::4], q) and torch.equal(room[:, 1::4], k)
        got = call(room[:, 0::4], room[:, 1::4], (room[:, 0::4], room[:, 1::4]))            # in place
        assert all(torch.equal(a, b) for a, b in zip(want, got))
