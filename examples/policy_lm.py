"""A language model of one attention and one MoE layer, fine-tuned by reinforcement: what it samples is scored, and rewarded where it follows a rule.

    python examples/policy_lm.py

Beside one_layer_lm.py's parts the library norms and rotates the queries and keys, gives the samples' log probabilities and entropies with their
gradients, and limits the gradients' norm; torch multiplies the projections and the attention, in 32 bits.
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from one_layer_lm import EPS, Adam, B, OneLayerLM, limited  # noqa: E402


class PolicyLM(OneLayerLM):
    """h0 = embedding; h = h0 + attention(norm(h0)); h1 = h + moe(norm(h)); logits = norm(h1) W^T.  Sequences of `length` tokens side by side."""

    def __init__(self, T, V, length, d=256, heads=4, kv_heads=2, D=64, temperature=1.0, seed=0, device="cuda:0", **kw):
        super().__init__(T, V, d, seed=seed, device=device, **kw)
        g = torch.Generator().manual_seed(seed + 1)
        bf = lambda scale, *s: (scale * torch.randn(*s, generator=g)).bfloat16().to(device)  # noqa: E731
        f32 = lambda *s: torch.zeros(*s, dtype=torch.float32, device=device)  # noqa: E731
        self.length, self.heads, self.kv_heads, self.D, self.temperature = length, heads, kv_heads, D, temperature
        wide = (heads + 2 * kv_heads) * D
        self.p.update(w0=f32(d) + 1.0, Wqkv=bf(d ** -0.5, wide, d), wq=f32(D) + 1.0, wk=f32(D) + 1.0, Wo=bf((heads * D) ** -0.5, d, heads * D))
        self.pos = (torch.arange(T, device=device) % length).int()
        self.freq = (10000.0 ** (-torch.arange(0, D, 2, device=device, dtype=torch.float64) / D)).float()
        self.score = B.ScoreBuffers(T, d, V, device=device)
        row = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device=device)  # noqa: E731
        self.n0, self.h, self.rstd0, self.dw0 = row(T, d), row(T, d), f32(T), f32(d)
        self.q, self.k, self.dwq, self.dwk = row(T, heads, D), row(T, kv_heads, D), f32(D), f32(D)
        self.dqkv = row(T, wide)
        self.qk_ws = torch.empty(B.moe_qk_norm_rope_bwd_workspace_bytes(T, heads, kv_heads, D), dtype=torch.uint8, device=device)
        self.dh, self.de = row(T, d), row(T, d)

    def _heads_of(self, rows):
        """Queries, keys and values as the columns of one matrix that they are."""
        a, b = self.heads * self.D, (self.heads + self.kv_heads) * self.D
        return [part.unflatten(1, (-1, self.D)) for part in (rows[:, :a], rows[:, a:b], rows[:, b:])]

    def _attend(self, q, k, v):
        """Causal attention inside the sequences, in 32 bits."""
        n, L, G = self.T // self.length, self.length, self.heads // self.kv_heads
        q, k, v = (t.view(n, L, -1, self.D).transpose(1, 2) for t in (q, k, v))
        k, v = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
        s = q @ k.transpose(2, 3).contiguous() / math.sqrt(self.D)
        s = s.masked_fill(torch.ones(L, L, dtype=torch.bool, device=q.device).triu(1), -math.inf)
        return (torch.softmax(s, 3) @ v).transpose(1, 2).reshape(self.T, -1)

    def forward(self, tokens):
        p = self.p
        self.tokens, self.h0 = tokens, p["embedding"][tokens]
        B.moe_add_rms_norm(self.h0, None, p["w0"], EPS, None, self.n0, self.rstd0)
        self.qkv = self.n0 @ p["Wqkv"].t()
        q, k, v = self._heads_of(self.qkv)
        B.moe_qk_norm_rope(q, k, p["wq"], p["wk"], self.pos, self.freq, False, EPS, self.q, self.k)
        self.leaves = [t.float().requires_grad_() for t in (self.q, self.k, v)]
        self.mixed = self._attend(*self.leaves)
        B.moe_add_rms_norm(self.mixed.detach().bfloat16() @ p["Wo"].t(), self.h0, p["w1"], EPS, self.h, self.n1, self.rstd1)
        B.moe_router_fwd(self.n1, p["Wr"], self.logits)
        self.moe.run_fwd(self.n1, self.logits, p["Wg"], p["Wu"], p["Wd"])
        B.moe_add_rms_norm(self.moe.out, self.h, p["w2"], EPS, self.h1, self.n2, self.rstd2)

    def policy_step(self, tokens, chosen, dlogp, dentropy=None):
        """Log probabilities and entropies of chosen tokens, and every gradient for given gradients of them; -100: nothing was chosen."""
        self.forward(tokens)
        self.score.run_fwd(self.n2, self.p["W"], chosen, self.temperature)
        self.score.run_bwd(self.n2, self.p["W"], chosen, dlogp, dentropy, self.temperature)
        p, m = self.p, self.moe
        B.moe_add_rms_norm_bwd(self.score.dx, None, self.h1, p["w2"], self.rstd2, self.dh1, self.dw2, self.ws)
        m.run_bwd(self.dh1, p["Wg"], p["Wu"], p["Wd"])
        B.moe_route_bwd(self.logits, m.topk_idx, m.dgate, m.renormalize, self.dlogits)
        B.moe_router_bwd(self.n1, p["Wr"], self.dlogits, m.dx, self.dWr, self.ws)
        B.moe_add_rms_norm_bwd(m.dx, self.dh1, self.h, p["w1"], self.rstd1, self.dh, self.dw1, self.ws)
        dq, dk, dv = (t.bfloat16() for t in torch.autograd.grad(self.mixed, self.leaves, (self.dh @ p["Wo"]).float()))
        qv, kv, _ = self._heads_of(self.qkv)
        to_q, to_k, to_v = self._heads_of(self.dqkv)
        to_v.copy_(dv)
        B.moe_qk_norm_rope_bwd(dq, dk, qv, kv, p["wq"], p["wk"], self.pos, self.freq, False, EPS, to_q, to_k, self.dwq, self.dwk, self.qk_ws)
        B.moe_add_rms_norm_bwd(self.dqkv @ p["Wqkv"], self.dh, self.h0, p["w0"], self.rstd0, self.de, self.dw0, self.ws)
        embedding = torch.zeros(self.V, self.d, device=self.device).index_add_(0, self.tokens, self.de.float())
        return {"embedding": embedding, "w0": self.dw0, "Wqkv": self.dqkv.t() @ self.n0, "wq": self.dwq, "wk": self.dwk,
                "Wo": self.dh.t() @ self.mixed.detach().bfloat16(), "w1": self.dw1, "Wr": self.dWr, "Wg": m.dWg, "Wu": m.dWu, "Wd": m.dWd, "w2": self.dw2,
                "W": self.score.dW}

    def sample(self, tokens, generator):
        """A token behind each of these, drawn at the temperature."""
        self.forward(tokens)
        z = (self.n2.float() @ self.p["W"].float().t()) / self.temperature
        return torch.multinomial(torch.softmax(z, 1), 1, generator=generator)[:, 0].int()


def reinforce(model, reward, steps, lr=2e-3, entropy_weight=0.01, largest=1.0, seed=0):
    """The mean reward of every step, on the host.  reward(tokens, chosen): of each token."""
    g = torch.Generator(device=model.device).manual_seed(seed)
    adam, curve = Adam(model.p, lr), []
    for _ in range(steps):
        tokens = torch.randint(0, model.V, (model.T,), generator=g, device=model.device)
        chosen = model.sample(tokens, g)
        r = reward(tokens, chosen)
        # a step towards what earned more than the mean, away from what earned less, and towards more entropy
        grads = model.policy_step(tokens, chosen, -(r - r.mean()) / model.T, torch.full_like(r, -entropy_weight / model.T))
        limited(grads, largest)
        adam.step(model.p, grads)
        curve.append(float(r.mean()))
    return curve


def main():
    V = 64
    model = PolicyLM(1024, V, 64)
    follows = torch.randperm(V, generator=torch.Generator().manual_seed(0)).to(model.device)
    curve = reinforce(model, lambda tokens, chosen: ((chosen - follows[tokens]) % V < 4).float(), 120)
    print("share of samples that follow the rule: %.3f -> %.3f" % (curve[0], curve[-1]))


if __name__ == "__main__":
    main()
