"""Losses where the logits are large and the loss is not: what is lost in them shows in the difference."""
import pytest
import torch

import head_reference as R
from test_gpu_head import make, run

pytestmark = pytest.mark.gpu


def alike(T, d, V, high, K=0, masked=0.0, seed=41):
    """Logits of about `high`, about 1 apart: x along what all rows of W have in common."""
    a = make(T, 64, 400, K, masked, seed)
    g = torch.Generator().manual_seed(seed)
    w = 0.05 * torch.randn(d, generator=g)
    x = w * high / float(w.square().sum()) * (1 + 0.02 * torch.rand(T, 1, generator=g))
    a["x"] = x.bfloat16()
    a["W"] = (w + torch.randn(V, d, generator=g) / float(x[0].norm())).bfloat16()
    return a


def losses(a, got):
    """(the losses' errors, and what they may be in the mean square: the other columns' logits err independently and count with their p; the logarithm of
    a sum, that sum in 32 bits and a few roundings of the loss)."""
    z = a["x"].double() @ a["W"].double().t()
    on = a["target"] >= 0
    want = torch.logsumexp(z, 1) - z.gather(1, a["target"].clamp(min=0)[:, None].long())[:, 0]
    d = a["x"].shape[1]
    one = (d / 32 + 16) ** 0.5 * R.HALF32 * 2 ** torch.log2(z.abs().amax()).ceil()       # a chain's roundings, each of up to half a step of the largest
    mean_square = float(torch.softmax(z, 1).square().sum(1).sqrt().amax() * one) + 16 * R.HALF32 + 8 * R.HALF32 * float(want[on].abs().amax())
    return (got["loss"].cpu().double() - want)[on], mean_square


@pytest.mark.parametrize("T,masked,K", [(16, 0.0, 0), (17, 0.0, 0), (17, 0.9, 0), (300, 0.0, 0), (300, 0.95, 0), (130, 0.0, 3), (300, 0.9, 3)])
def test_the_targets_own_logit(T, masked, K):
    """However many tokens there are, and however many of them have a loss."""
    a = alike(T, 8192, 8000, 100.0, K, masked)
    if K:
        a["ids"] = torch.where(a["ids"] >= 0, a["ids"] + 400, -1)                     # (no targets among them)
    off, bound = losses(a, run(a, train=False))
    assert float(off.square().mean().sqrt()) <= bound, (float(off.mean()), float(off.square().mean().sqrt()), bound)


@pytest.mark.parametrize("high", [2000.0, -2000.0])
def test_the_unit_of_the_exponents(high):
    """log2(e) has a rounding of its own, which logits of 2000 make visible; one common to all is not part of a loss."""
    a = alike(16, 64, 60000, high)
    off, bound = losses(a, run(a, train=False))
    assert float(off.square().mean().sqrt()) <= bound, (float(off.mean()), float(off.square().mean().sqrt()), bound)
