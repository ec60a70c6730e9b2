"""The example that trains a model of one layer: its gradients against automatic differentiation in 64 bits, and that it learns."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import one_layer_lm as L  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def reference(model, tokens, target, weight, ids, teacher, tau):
    """The same losses and gradients in 64 bits, with the experts that the library has chosen."""
    p = {k: v.detach().cpu().double().requires_grad_() for k, v in model.p.items()}
    idx = model.moe.topk_idx.cpu().long()
    norm = lambda h, w: h * torch.rsqrt(h.square().mean(1, keepdim=True) + L.EPS) * w  # noqa: E731
    h0 = p["embedding"][tokens.cpu()]
    n1 = norm(h0, p["w1"])
    gates = torch.softmax((n1 @ p["Wr"].t()).gather(1, idx), 1)              # renormalised over the chosen ones
    out = []
    for i in range(idx.shape[1]):
        e = idx[:, i]
        g, u = torch.einsum("td,tfd->tf", n1, p["Wg"][e]), torch.einsum("td,tfd->tf", n1, p["Wu"][e])
        out.append(gates[:, i:i + 1] * torch.einsum("tf,tdf->td", torch.nn.functional.silu(g) * u, p["Wd"][e]))
    z = norm(h0 + sum(out), p["w2"]) @ p["W"].t()
    loss = torch.nn.functional.cross_entropy(z, target.cpu().long(), reduction="none", ignore_index=-100)
    total = (loss * weight.cpu().double()).sum()
    kd = None
    if ids is not None:
        on, at = ids.cpu() >= 0, ids.cpu().clamp(min=0).long()
        l = torch.where(on, teacher.cpu().double() / tau, -1e300)
        q = torch.where(on, torch.softmax(l, 1), 0.0)
        kd = (torch.special.xlogy(q, q) - q * torch.log_softmax(z / tau, 1).gather(1, at)).sum(1)
        total = total + (kd * weight.cpu().double() * tau ** 2).sum()
    total.backward()
    return loss.detach(), None if kd is None else kd.detach(), {k: v.grad for k, v in p.items()}


@pytest.mark.parametrize("entries", [0, 5])
def test_gradients(entries):
    T, V, tau = 96, 131, 1.5
    model = L.OneLayerLM(T, V, d=128, f=64, E=4, entries=entries)
    model.p["w1"] += 0.3 * torch.rand(128, device=DEV)
    tokens, target = L.language(V)(T, 3)
    weight = (target >= 0).float() / (target >= 0).sum()
    more = ()
    if entries:
        g = torch.Generator().manual_seed(5)
        ids = torch.stack([torch.randperm(V, generator=g)[:entries] for _ in range(T)]).int().to(DEV)
        ids[target < 0] = -1
        more = (ids, torch.randn(T, entries, generator=g).to(DEV), tau)
    grads = model.train_step(tokens, target, weight, *more)
    loss, kd, want = reference(model, tokens, target, weight, *(more or (None, None, 1.0)))
    # activations pass through about ten roundings to bf16 (2^-8 each at most) on the way to the head and back, and every gradient is
    # the sum of many terms rounded independently: 2 % of its size bounds that
    on = target.cpu() >= 0
    assert float((model.head.loss.cpu().double() - loss)[on].abs().max()) < 0.02 * float(loss.abs().max())
    if entries:
        assert float((model.head.kd.cpu().double() - kd).abs().max()) < 0.02 * float(kd.abs().max())
    for k, w in want.items():
        off = float((grads[k].cpu().double() - w).norm() / w.norm())
        assert off < 0.02, (k, off)


def test_it_learns_and_teaches():
    V, T = 259, 512
    walk = L.language(V)
    teacher = L.OneLayerLM(T, V)
    curve = L.train(teacher, walk, 50)
    assert curve[0] > 5.0 and curve[-1] < 0.5 * curve[0], curve
    student = L.OneLayerLM(T, V, f=64, E=4, entries=8, seed=1)
    kd = L.train(student, walk, 50, teacher=teacher, entries=8, temperature=1.5)
    assert kd[-1] < 0.5 * kd[0], kd
    tokens, target = walk(T, 7)
    fresh = L.OneLayerLM(T, V, seed=2)
    score = lambda m: float(m.log_probabilities(tokens, target)[target >= 0].mean())  # noqa: E731
    assert score(teacher) > score(fresh) + 1.0 and score(student) > score(fresh) + 1.0
    # activations in 8 bits: an error of 2^-4 at most in each of 256, with signs that come and go
    near = teacher.log_probabilities(tokens, target) - teacher.log_probabilities(tokens, target, eight_bit=True)
    assert float(near.abs().mean()) < 0.1, float(near.abs().mean())
