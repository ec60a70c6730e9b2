"""A language model of one MoE layer, trained by hand: norm, router and experts, residual and norm, vocabulary head.

    python examples/one_layer_lm.py            # trains a teacher on a made-up language, then a student from its top logits

Everything between the embedding and the losses runs in the library; torch holds the memory, looks the embedding up and applies the
updates.  A sentence of the language is a walk: which token follows a token is fixed, but for one in ten that may be any.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2604_00785_amd import binding as B  # noqa: E402

EPS = 1e-5


class OneLayerLM:
    """h0 = embedding; h1 = h0 + moe(norm(h0)); logits = norm(h1) W^T.  T tokens at a time."""

    def __init__(self, T, V, d=256, f=128, E=8, k=2, entries=0, seed=0, device="cuda:0"):
        g = torch.Generator().manual_seed(seed)
        bf = lambda scale, *s: (scale * torch.randn(*s, generator=g)).bfloat16().to(device)  # noqa: E731
        f32 = lambda *s: torch.zeros(*s, dtype=torch.float32, device=device)  # noqa: E731
        self.T, self.V, self.d, self.device = T, V, d, device
        # weights; the norms' and the router's are kept in 32 bits
        self.p = {"embedding": bf(1.0, V, d), "w1": f32(d) + 1.0, "Wr": bf(0.05, E, d).float(), "Wg": bf(d ** -0.5, E, f, d),
                  "Wu": bf(d ** -0.5, E, f, d), "Wd": bf(f ** -0.5, E, d, f), "w2": f32(d) + 1.0, "W": bf(0.02, V, d)}
        self.moe = B.MoELayerBuffers(T, d, E, k, f, device=device, fold=True)
        self.head = B.HeadBuffers(T, d, V, entries, device=device)
        self.scores = B.HeadBuffers(T, d, V, train=False, device=device)
        self.logits, self.dlogits, self.dWr = f32(T, E), f32(T, E), f32(E, d)
        self.rstd1, self.rstd2, self.dw1, self.dw2 = f32(T), f32(T), f32(d), f32(d)
        row = lambda: torch.empty(T, d, dtype=torch.bfloat16, device=device)  # noqa: E731
        self.n1, self.h1, self.n2, self.dh1, self.dh0 = row(), row(), row(), row(), row()
        self.ws = torch.empty(max(B.moe_add_rms_norm_bwd_workspace_bytes(T, d), B.moe_router_bwd_workspace_bytes(T, d, E)), dtype=torch.uint8,
                              device=device)

    def forward(self, tokens):
        p = self.p
        self.tokens, self.h0 = tokens, p["embedding"][tokens]
        B.moe_add_rms_norm(self.h0, None, p["w1"], EPS, None, self.n1, self.rstd1)
        B.moe_router_fwd(self.n1, p["Wr"], self.logits)
        self.moe.run_fwd(self.n1, self.logits, p["Wg"], p["Wu"], p["Wd"])
        B.moe_add_rms_norm(self.moe.out, self.h0, p["w2"], EPS, self.h1, self.n2, self.rstd2)

    def backward(self):
        """From the head's dx to every weight's gradient."""
        p, m = self.p, self.moe
        B.moe_add_rms_norm_bwd(self.head.dx, None, self.h1, p["w2"], self.rstd2, self.dh1, self.dw2, self.ws)
        m.run_bwd(self.dh1, p["Wg"], p["Wu"], p["Wd"])                     # the residual's sum passes its gradient on to both
        B.moe_route_bwd(self.logits, m.topk_idx, m.dgate, m.renormalize, self.dlogits)
        B.moe_router_bwd(self.n1, p["Wr"], self.dlogits, m.dx, self.dWr, self.ws)
        B.moe_add_rms_norm_bwd(m.dx, self.dh1, self.h0, p["w1"], self.rstd1, self.dh0, self.dw1, self.ws)
        embedding = torch.zeros(self.V, self.d, device=self.device).index_add_(0, self.tokens, self.dh0.float())
        return {"embedding": embedding, "w1": self.dw1, "Wr": self.dWr, "Wg": m.dWg, "Wu": m.dWu, "Wd": m.dWd, "w2": self.dw2, "W": self.head.dW}

    def train_step(self, tokens, target, weight, ids=None, teacher=None, temperature=1.0):
        """Losses token by token and every gradient; weight: what a token counts, the division by their number in it."""
        self.forward(tokens)
        more = () if ids is None else (ids, teacher, temperature)
        self.head.run_fwd(self.n2, self.p["W"], target, *more)
        # a temperature divides the distillation's gradients by its square
        dkd = None if ids is None else weight * temperature ** 2
        self.head.run_bwd(self.n2, self.p["W"], target, weight, *more, dkd=dkd)
        return self.backward()

    def log_probabilities(self, tokens, target, eight_bit=False):
        """eight_bit: with the head's input as e4m3 codes and a scale per 64 columns, the form in which an 8-bit product would read it."""
        self.forward(tokens)
        n2 = self.n2
        if eight_bit:
            codes = torch.empty(self.T, self.d, dtype=torch.float8_e4m3fn, device=self.device)
            scale = torch.empty(self.T, self.d // 64, dtype=torch.float32, device=self.device)
            B.moe_add_rms_norm_8bit(self.moe.out, self.h0, self.p["w2"], EPS, 64, self.h1, codes, scale)
            n2 = (codes.float().view(self.T, -1, 64) * scale[:, :, None]).view(self.T, self.d).bfloat16()
        self.scores.run_fwd(n2, self.p["W"], target)
        return -self.scores.loss

    def top_logits(self, tokens, entries):
        self.forward(tokens)
        top = (self.n2.float() @ self.p["W"].float().t()).topk(entries, 1)
        return top.indices.int(), top.values.contiguous()


class Adam:
    """Adam with 32-bit copies of the weights."""

    def __init__(self, p, lr):
        self.lr, self.n = lr, 0
        self.state = {k: (v.float().clone(), torch.zeros_like(v, dtype=torch.float32), torch.zeros_like(v, dtype=torch.float32)) for k, v in p.items()}

    def step(self, p, grads):
        self.n += 1
        for k, (full, m, v) in self.state.items():
            g = grads[k].float()
            m.lerp_(g, 0.1)
            v.lerp_(g * g, 0.01)
            full -= self.lr * (m / (1 - 0.9 ** self.n)) / ((v / (1 - 0.99 ** self.n)).sqrt() + 1e-8)
            p[k].copy_(full)


def language(V, seed=0, device="cuda:0"):
    """walk(T, seed): tokens and their targets, the first quarter without any (a prompt)."""
    follows = torch.randperm(V, generator=torch.Generator().manual_seed(seed))

    def walk(T, seed):
        g = torch.Generator().manual_seed(seed)
        tokens = torch.randint(0, V, (T,), generator=g)
        target = torch.where(torch.rand(T, generator=g) < 0.9, follows[tokens], torch.randint(0, V, (T,), generator=g)).int()
        target[:T // 4] = -100
        return tokens.to(device), target.to(device)
    return walk


def train(model, walk, steps, lr=3e-3, teacher=None, entries=0, temperature=1.0):
    """The mean loss (with a teacher: divergence) of every step, on the host."""
    adam, curve = Adam(model.p, lr), []
    for n in range(steps):
        tokens, target = walk(model.T, 100 + n)
        weight = (target >= 0).float() / (target >= 0).sum()
        more = ()
        if teacher is not None:
            ids, logits = teacher.top_logits(tokens, entries)
            ids[target < 0] = -1                                   # nothing is learnt from prompts
            target = torch.full_like(target, -100)                 # the teacher alone is learnt from
            more = (ids, logits, temperature)
        adam.step(model.p, model.train_step(tokens, target, weight, *more))
        curve.append(float(((model.head.loss if teacher is None else model.head.kd) * weight).sum()))
    return curve


def main():
    V, T, entries = 515, 1024, 16
    walk = language(V)
    teacher = OneLayerLM(T, V)
    curve = train(teacher, walk, 60)
    print("teacher: loss %.3f -> %.3f" % (curve[0], curve[-1]))
    student = OneLayerLM(T, V, f=64, E=4, entries=entries, seed=1)
    curve = train(student, walk, 60, teacher=teacher, entries=entries, temperature=1.5)
    print("student: divergence %.3f -> %.3f" % (curve[0], curve[-1]))
    tokens, target = walk(T, 7)
    for name, m in (("teacher", teacher), ("student", student)):
        print("%s: log probability of a token it has not seen %.3f" % (name, float(m.log_probabilities(tokens, target)[target >= 0].mean())))


if __name__ == "__main__":
    main()
