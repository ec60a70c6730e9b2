"""Distillation from teachers whose logits spread widely: entries that are next to nothing to the teacher, padding by a very low
logit, low temperatures; and targets that only the distillation trains."""
import math

import pytest
import torch

import head_reference as R
from test_gpu_head import make, run

pytestmark = pytest.mark.gpu
LOWEST = float(torch.finfo(torch.float32).min)


def wide(T, d, V, K, gap, seed):
    """Every other token's last entry lies `gap` below its others and is what the student takes for the likeliest column; the tokens between have
    from one to all of their entries at the type's lowest value, as padding."""
    a = make(T, d, V, K, seed=seed)
    z = a["x"].float() @ a["W"].float().t()
    g = torch.Generator().manual_seed(seed)
    for t in range(T):
        if t % 2 == 0:
            best = int(z[t].argmax())
            others = [v for v in a["ids"][t].tolist() if v >= 0 and v != best]
            fresh = [v for v in torch.randperm(V, generator=g)[:2 * K].tolist() if v != best and v not in others]
            a["ids"][t] = torch.tensor((others + fresh)[:K - 1] + [best])
            a["teacher"][t, :K - 1] = torch.linspace(4, 0, K - 1)
            a["teacher"][t, K - 1] = max(0.0 - gap, LOWEST)
        else:
            n = int((a["ids"][t] >= 0).sum())
            low = t // 2 % n + 1                          # (n: all of them, which leaves all alike)
            a["teacher"][t, n - low:n] = LOWEST
    return a


def reference(a, tau):
    """R.head, with bounds on kd and lse_t in which an entry counts as much as the teacher makes of it: log q_j is the result of a subtraction, a division, a logarithm
    and another subtraction, a rounding of at most |l_j - top| / tau + log q_j each, and stands in kd with the factor q_j (1 + |u_j|), u_j = log p_j - log q_j + kd."""
    want, bound = R.head(a["x"], a["W"], a["target"], a["ids"], a["teacher"], tau, a["dloss"], a["dkd"])
    T, K = a["ids"].shape
    there = (a["ids"] >= 0) & (a["teacher"] > -math.inf)
    l = torch.where(there, a["teacher"].to(R.F64) / tau, -math.inf)
    top = l.amax(1, keepdim=True)
    z = a["x"].to(R.F64) @ a["W"].to(R.F64).t() / tau
    log_p = torch.log_softmax(z, 1).gather(1, torch.where(there, a["ids"], 0).long())
    log_q = torch.log_softmax(l, 1)
    q = torch.where(there, log_q.exp(), 0.0)              # (rows without entries are zeros)
    far = torch.where(q > 0, (1 + (log_p - log_q).abs() + want["kd"][:, None]) * (8 * (l - top).abs() + 8 * log_q.abs() + 16), 0.0)
    # as in R.head: the logits' errors and the sums over the columns, then sums over K entries
    Wd, xd = a["W"].to(R.F64), a["x"].to(R.F64)
    spread = (xd.square() @ Wd.square().t()).sqrt()
    off = ((a["x"].shape[1] / 32 + 16) * 2 * R.HALF32 * ((z * tau).abs() + 4 * spread)).amax(1)
    high = (z * tau).abs().amax(1) / min(1.0, tau)
    tol = 2 * off / min(1.0, tau) + (64 + a["W"].shape[0] / 64 / 16 + 8 * high) * R.HALF32
    bound["kd"] = bound["lse_t"] = 2 * tol + (4 * K ** 0.5 + (q * far).sum(1) + 8 * want["kd"]) * R.HALF32
    assert bool(torch.isfinite(bound["kd"]).all())
    return want, bound


GAPS = [30.0, 90.0, 110.0, 1e4, 3.4e38]
SHAPES = [(20, 64, 1000, 4), (40, 128, 777, 70), (21, 64, 600, 200), (300, 64, 1500, 16)]


@pytest.mark.parametrize("T,d,V,K", SHAPES)
@pytest.mark.parametrize("tau", [0.1, 0.5, 1.0, 4.0])
@pytest.mark.parametrize("gap", GAPS)
def test_losses_of_a_teacher_that_spreads_widely(T, d, V, K, tau, gap):
    print("wide teacher", T, d, V, K, tau, gap, flush=True)
    a = wide(T, d, V, K, gap, seed=21)
    got = run(a, tau, train=False)
    want, bound = reference(a, tau)
    for k in ("loss", "lse", "kd", "lse_t"):
        R.check(got[k], want[k], bound[k], k)


@pytest.mark.parametrize("spread", [20.0, 28.0, 60.0])
@pytest.mark.parametrize("tau", [0.05, 0.25, 1.0])
def test_losses_of_logits_that_fall_evenly(spread, tau):
    """Ordinary top logits at a low temperature: from an entry that is all to the teacher to one that is nothing, in even steps."""
    T, d, V, K = 48, 64, 900, 16
    a = make(T, d, V, K, seed=22)
    a["ids"] = torch.stack([torch.randperm(V, generator=torch.Generator().manual_seed(t))[:K] for t in range(T)]).int()
    a["teacher"] = torch.linspace(spread / 2, -spread / 2, K).repeat(T, 1) + 0.01 * torch.arange(T)[:, None]
    got = run(a, tau, train=False)
    want, bound = reference(a, tau)
    for k in ("loss", "lse", "kd", "lse_t"):
        R.check(got[k], want[k], bound[k], k)


@pytest.mark.parametrize("T,d,V,K", SHAPES)
@pytest.mark.parametrize("tau", [0.1, 0.5, 1.0, 4.0])
@pytest.mark.parametrize("gap", [15.0, 19.0, 21.0, 60.0, 86.0, 90.0, 1e4, 3.4e38])
def test_gradients_of_a_teacher_that_spreads_widely(T, d, V, K, tau, gap):
    """What the student gives to an entry that is nothing to the teacher is what it has to unlearn: the whole of p is left of p - q."""
    print("gradient of a wide teacher", T, d, V, K, tau, gap, flush=True)
    a = wide(T, d, V, K, gap, seed=23)
    for v_piece in (0, 256):
        got = run(a, tau, v_piece=v_piece)
        want, bound = reference(a, tau)
        for k in got:
            R.check(got[k], want[k], bound[k], k)


@pytest.mark.parametrize("tau", [0.25, 1.0, 2.0])
@pytest.mark.parametrize("target", ["all", "half", "none"])
def test_gradients_on_either_side_of_the_least_q(tau, target):
    """Entries with log q from 0 to -40 in small steps, the student's p near q, far above and far below; with and without a target, which is an entry in some rows."""
    T, d, V, K = 60, 64, 400, 60
    a = make(T, d, V, K, seed=24)
    a["ids"] = torch.stack([torch.randperm(V, generator=torch.Generator().manual_seed(t))[:K] for t in range(T)]).int()
    z = (a["x"].float() @ a["W"].float().t()).gather(1, a["ids"].long())
    fall = torch.linspace(0, -40 * tau, K)
    a["teacher"] = torch.where(torch.arange(T)[:, None] % 3 == 0, z + fall, fall.expand(T, K)).contiguous()
    a["target"][::4] = a["ids"][::4, 7]
    a["target"][1::4] = a["ids"][1::4, K - 3]
    if target != "all":
        a["target"][(torch.arange(T) % 2 == 1) | (target == "none")] = -100
    got = run(a, tau)
    want, bound = reference(a, tau)
    for k in got:
        R.check(got[k], want[k], bound[k], k)


@pytest.mark.parametrize("T", [1, 200])
@pytest.mark.parametrize("tau", [0.7, 1.0, 3.0])
@pytest.mark.parametrize("weight", [0.0, 1e-9])
@pytest.mark.parametrize("far", [2.0, 4.0, 8.0])
def test_gradient_at_a_target_that_only_the_distillation_trains(T, tau, weight, far):
    """A target that is no entry and counts (next to) nothing by itself has dkd / temperature p, however small p is.  One token has a loss, so
    that nothing else stands in its target's row of dW."""
    d, V, K = 128, 2000, 8
    a = make(T, d, V, K, seed=25, known=0.0)
    for t in range(T):                                    # an entry is likely, the target unlikely
        a["ids"][t] = (int(a["target"][t]) + 1 + torch.arange(K) * 3) % V
    lift = far / (0.05 ** 2 * d)
    a["x"] = (a["x"].float() + lift * (a["W"][a["ids"][:, 0].long()].float() - a["W"][a["target"].long()].float())).bfloat16()
    a["dloss"] *= weight
    a["target"][:T - 1] = -100
    a["ids"][:T - 1] = -1
    got = run(a, tau)
    want, bound = reference(a, tau)
    for k in got:
        R.check(got[k], want[k], bound[k], k)
