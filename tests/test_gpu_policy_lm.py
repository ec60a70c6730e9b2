"""The example that is fine-tuned by reinforcement: its gradients against automatic differentiation in 64 bits, its teacher's logits, the limit of the gradients'
norm, and that it runs."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import one_layer_lm as L  # noqa: E402
import policy_lm as P  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def reference(model, tokens, chosen, dlogp, dentropy):
    """The same in 64 bits, with the experts that the library has chosen."""
    p = {k: v.detach().cpu().double().requires_grad_() for k, v in model.p.items()}
    idx, tau, D = model.moe.topk_idx.cpu().long(), model.temperature, model.D
    norm = lambda h, w: h * torch.rsqrt(h.square().mean(-1, keepdim=True) + L.EPS) * w  # noqa: E731
    h0 = p["embedding"][tokens.cpu()]
    q, k, v = model._heads_of(norm(h0, p["w0"]) @ p["Wqkv"].t())
    angle = (model.pos.cpu().double()[:, None] * model.freq.cpu().double())[:, None, :]

    def turned(x, w):
        x = norm(x, w)
        a, b = x[..., :D // 2], x[..., D // 2:]
        return torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1)
    h = h0 + model._attend(turned(q, p["wq"]), turned(k, p["wk"]), v) @ p["Wo"].t()
    n1 = norm(h, p["w1"])
    gates = torch.softmax((n1 @ p["Wr"].t()).gather(1, idx), 1)
    out = []
    for i in range(idx.shape[1]):
        e = idx[:, i]
        g, u = torch.einsum("td,tfd->tf", n1, p["Wg"][e]), torch.einsum("td,tfd->tf", n1, p["Wu"][e])
        out.append(gates[:, i:i + 1] * torch.einsum("tf,tdf->td", torch.nn.functional.silu(g) * u, p["Wd"][e]))
    lp = torch.log_softmax(norm(h + sum(out), p["w2"]) @ p["W"].t() / tau, 1)
    has = chosen.cpu() >= 0
    logp = lp.gather(1, chosen.cpu().long().clamp(min=0)[:, None])[:, 0] * has
    entropy = -(lp.exp() * lp).sum(1) * has
    ((logp * dlogp.cpu().double()).sum() + (entropy * dentropy.cpu().double()).sum()).backward()
    return logp.detach(), entropy.detach(), {k: v.grad for k, v in p.items()}


def test_gradients():
    T, V = 96, 131
    model = P.PolicyLM(T, V, 24, d=128, heads=4, kv_heads=2, D=32, temperature=0.8, f=64, E=4)
    for n in ("w0", "w1", "wq", "wk"):
        model.p[n] += 0.3 * torch.rand(model.p[n].shape, device=DEV)
    g = torch.Generator().manual_seed(3)
    tokens, chosen = torch.randint(0, V, (T,), generator=g).to(DEV), torch.randint(0, V, (T,), generator=g).int()
    chosen[::5] = -100
    chosen = chosen.to(DEV)
    dlogp, dentropy = torch.randn(T, generator=g).to(DEV), 0.3 * torch.randn(T, generator=g).to(DEV)
    grads = model.policy_step(tokens, chosen, dlogp, dentropy)
    logp, entropy, want = reference(model, tokens, chosen, dlogp, dentropy)
    # activations pass through about fifteen roundings to bf16 (2^-8 each at most) on the way to the head and back, and every gradient is the sum of many
    # terms rounded independently: 3 % of its size bounds that
    assert float((model.score.logp.cpu().double() - logp).abs().max()) < 0.03 * float(logp.abs().max())
    assert float((model.score.entropy.cpu().double() - entropy).abs().max()) < 0.03 * float(entropy.abs().max())
    assert set(grads) == set(want)
    for k, w in want.items():
        off = float((grads[k].cpu().double() - w).norm() / w.norm())
        assert off < 0.03, (k, off)


def test_teachers_logits_and_limited_gradients():
    T, V = 300, 515
    model = L.OneLayerLM(T, V)
    tokens, target = L.language(V)(T, 3)
    ids, logits = model.top_logits(tokens, 16)
    z = model.n2.double() @ model.p["W"].double().t()
    order = (z * 2.0 ** 36).round().sort(dim=1, descending=True, stable=True).indices[:, :16]
    assert torch.equal(ids.long(), order)
    assert float((logits.double() - z.gather(1, order)).abs().max()) < 1e-5 * float(z.abs().max())
    ids, logits = model.top_logits(tokens, 100)                          # more than the scores have
    assert ids.shape == logits.shape == (T, 100) and float((logits.double() - z.gather(1, ids.long())).abs().max()) < 1e-5 * float(z.abs().max())
    grads = model.train_step(tokens, target, torch.ones(T, device=DEV) / T)
    before = {k: v.double() for k, v in grads.items()}
    size = math.sqrt(sum(float(v.square().sum()) for v in before.values()))
    norm = L.limited(grads, size / 3)
    assert abs(float(norm) - size) < 1e-6 * size
    for k, v in grads.items():
        # scaled by the formula, rounded to the gradient's type
        want = before[k] * (size / 3 / (size + 1e-6))
        off = (v.double() - want).abs() - want.abs() * (2.0 ** -8 if v.dtype == torch.bfloat16 else 2.0 ** -21) - 1e-38
        assert float(off.max()) <= 0, k


def test_it_runs():
    model = P.PolicyLM(256, 64, 32)
    follows = torch.randperm(64, generator=torch.Generator().manual_seed(0)).to(DEV)
    curve = P.reinforce(model, lambda tokens, chosen: (chosen == follows[tokens]).float(), 3)
    assert len(curve) == 3 and all(math.isfinite(c) for c in curve)
    teacher, student = L.OneLayerLM(256, 64), L.OneLayerLM(256, 64, f=64, E=4, entries=8, seed=1)
    kd = L.train(student, L.language(64), 3, teacher=teacher, entries=8, largest=0.5)
    assert all(math.isfinite(c) for c in kd)
