"""What autograd would lose at the token operators is refused; checked before any device is needed."""
import pytest
import torch
from torch.autograd import forward_ad

import paper_1911_00472_b200 as P
from paper_1911_00472_b200 import tokens as T


def operands():
    q, k = torch.randn(4, 2, 8), torch.randn(4, 1, 8)
    inv_freq, axes = P.rotary_axes(8, device="cpu")
    return {"q": q, "k": k, "positions": torch.zeros(1, 4, dtype=torch.int32), "inv_freq": inv_freq, "axes": axes, "q_weight": torch.ones(8),
            "k_weight": torch.ones(8), "grads": (torch.randn_like(q), torch.randn_like(k))}


NAMES = ["q", "k", "inv_freq", "q_weight", "k_weight", "grad_q", "grad_k"]


def with_one(name, change):
    a = operands()
    if name.startswith("grad_"):
        i = ("q", "k").index(name[-1])
        a["grads"] = tuple(change(g) if j == i else g for j, g in enumerate(a["grads"]))
    else:
        a[name] = change(a[name])
    return a


def test_operands_without_derivatives_pass():
    assert T._check(**operands())[:3] == (1, 4, 8)
    with forward_ad.dual_level():                      # (a level alone is nothing to refuse)
        assert T._check(**operands())[:3] == (1, 4, 8)


@pytest.mark.parametrize("name", NAMES)
def test_operands_with_tangents_are_refused(name):
    with forward_ad.dual_level():
        with pytest.raises(ValueError, match="autograd"):
            T._check(**with_one(name, lambda t: forward_ad.make_dual(t, torch.ones_like(t))))
        with torch.no_grad(), pytest.raises(ValueError, match="autograd"):          # no_grad leaves tangents as they are
            T._check(**with_one(name, lambda t: forward_ad.make_dual(t, torch.ones_like(t))))


@pytest.mark.parametrize("name", NAMES)
def test_operands_that_require_gradients_are_refused(name):
    """Frequencies among them: a model that learns them would get no gradient."""
    a = with_one(name, lambda t: t.clone().requires_grad_())
    with pytest.raises(ValueError, match="autograd"):
        T._check(**a)
    with torch.no_grad():
        assert T._check(**a)[:3] == (1, 4, 8)


def test_outputs_that_autograd_follows_are_refused():
    """Values written into a tensor that requires a gradient, or has a tangent, would keep a derivative that is not theirs."""
    a = operands()
    q, k = a["q"], a["k"]
    leaf, plain = torch.empty_like(q, requires_grad=True), torch.empty_like(k)
    for out in ((leaf, plain), (leaf * 1, plain), (leaf.detach().clone().requires_grad_().view_as(q), plain)):
        with pytest.raises(ValueError, match="autograd"):
            T._outputs(q, k, out)
        with torch.no_grad():
            assert T._outputs(q, k, out) is out
    with forward_ad.dual_level(), pytest.raises(ValueError, match="autograd"):
        T._outputs(q, k, (torch.empty_like(q), forward_ad.make_dual(plain, torch.ones_like(plain))))
    rgb, images, index = torch.zeros(8, dtype=torch.uint8), torch.zeros(1, 10, dtype=torch.int64), torch.zeros(1, 2, dtype=torch.int32)
    tokens = torch.empty(1, 48, requires_grad=True)
    with pytest.raises(ValueError, match="autograd"):
        P.patch_tokens(rgb, images, index, 4, (0,) * 3, (1,) * 3, dtype=torch.float32, out=tokens)
    with pytest.raises(ValueError, match="CUDA"), torch.no_grad():
        P.patch_tokens(rgb, images, index, 4, (0,) * 3, (1,) * 3, dtype=torch.float32, out=tokens)
