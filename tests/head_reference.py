"""The norm in front of a layer and the vocabulary head's losses in 64 bits, with the bounds that the tests hold the kernels to."""
import math

import torch

F64 = torch.float64
HALF16 = torch.finfo(torch.bfloat16).eps / 2        # a rounding to bf16, relative
HALF32 = torch.finfo(torch.float32).eps / 2
HALF8 = torch.finfo(torch.float8_e4m3fn).eps / 2


def norm(x, r, w, eps):
    """(sum, y, 1 / root) in 64 bits; the sum is what the residual stream holds, in bf16."""
    total = x if r is None else (x.float() + r.float()).bfloat16()
    s = total.to(F64)
    q = 1.0 / (s.square().mean(1, keepdim=True) + eps).sqrt()
    return total, s * q * w.to(F64), q[:, 0]


def norm_bwd(dy, dsum, total, w, eps):
    """(dx, dw) and bounds on their errors: sums of d and T terms in fp32 (each of at most n roundings), dx rounded to bf16."""
    s, g, wd = total.to(F64), dy.to(F64), w.to(F64)
    T, d = s.shape
    q = 1.0 / (s.square().mean(1, keepdim=True) + eps).sqrt()
    c = (g * wd * s).mean(1, keepdim=True) * q * q
    add = 0.0 if dsum is None else dsum.to(F64)
    dx = add + q * (g * wd - s * c)
    big = (0.0 if dsum is None else add.abs()) + q * ((g * wd).abs() + s.abs() * (g * wd * s).abs().mean(1, keepdim=True) * q * q)
    terms = g * s * q
    return dx, terms.sum(0), HALF16 * dx.abs() + (2 * d + 16) * HALF32 * big, (2 * T + 2 * d + 16) * HALF32 * terms.abs().sum(0)


def head(x, W, target, ids=None, teacher=None, tau=1.0, dloss=None, dkd=None):
    """Losses and gradients in 64 bits, straight from their definitions, and for each output a bound on the kernel's error."""
    T, d = x.shape
    V = W.shape[0]
    xd, Wd = x.to(F64), W.to(F64)
    z = xd @ Wd.t()
    # a logit is a chain of d / 32 additions of sums of 32 products
    spread = (xd.square() @ Wd.square().t()).sqrt()
    off = ((d / 32 + 16) * 2 * HALF32 * (z.abs() + 4 * spread)).amax(1)
    has = (target >= 0) & (target < V)
    y = torch.where(has, target, 0).long()
    lse = torch.logsumexp(z, 1)
    zy = z.gather(1, y[:, None])[:, 0]
    zero = torch.zeros_like(lse)
    # sums in 32 bits: at most 32 terms in a lane, 2 steps across lanes, the strips of a group and the groups
    chain = 64 + V / 64 / 16
    high = z.abs().amax(1) / min(1.0, tau)
    tol = 2 * off / min(1.0, tau) + (chain + 8 * high) * HALF32
    # (the difference of two numbers of the size of a logit ends at 1e-15: what the other columns weigh against the target does not)
    loss = torch.log1p((z - zy[:, None]).exp().scatter(1, y[:, None], 0.0).sum(1))
    out = {"loss": torch.where(has, loss, zero), "lse": torch.where(has, lse, zero)}
    bound = {"loss": tol, "lse": tol}
    dz = None
    if dloss is not None:
        # (at the target exp(-loss) - 1: the softmax less one ends at 1e-16)
        dz = torch.where(has, dloss.to(F64), zero)[:, None] * torch.softmax(z, 1).scatter(1, y[:, None], torch.expm1(-loss)[:, None])
    if ids is not None:
        K = ids.shape[1]
        there = (ids >= 0) & (ids < V) & (teacher > -math.inf)
        some = there.any(1)
        full = torch.full((T, V + 1), -math.inf, dtype=F64)
        full.scatter_(1, torch.where(there, ids, V).long(), torch.where(there, teacher.to(F64) / tau, -math.inf))
        full = full[:, :V]
        full[~some] = 0.0
        q = torch.softmax(full, 1)
        log_p = torch.log_softmax(z / tau, 1)
        kd = torch.special.xlogy(q, q).sum(1) - (q * log_p).sum(1)
        out["kd"] = torch.where(some, kd, zero)
        out["lse_t"] = torch.where(some, torch.logsumexp(z / tau, 1), zero)
        t_high = torch.where(there, teacher.to(F64).abs() / tau, 0.0).amax(1)
        bound["kd"] = bound["lse_t"] = 2 * tol + (4 * K ** 0.5 + 8 * t_high + 8 * out["kd"]) * HALF32
        if dz is not None:
            dz = dz + torch.where(some, dkd.to(F64) / tau, zero)[:, None] * (log_p.exp() - q)
    if dz is not None:
        # dz is rounded to bf16, its exponentials are off by what the logits and lse are
        rel = (HALF16 + (4 * tol + 64 * HALF32))[:, None] * dz.abs()
        if ids is not None:                                     # p - q at an entry: the error of either
            rel = rel + (8 * tol[:, None] + 64 * HALF32) * torch.where(some, dkd.to(F64).abs() / tau, zero)[:, None] * q
        out["dx"], out["dW"] = dz @ Wd, dz.t() @ xd
        bound["dx"] = HALF16 * out["dx"].abs() + rel @ Wd.abs() + V * HALF32 * (dz.abs() @ Wd.abs()) + 1e-38
        bound["dW"] = HALF16 * out["dW"].abs() + rel.t() @ xd.abs() + T * HALF32 * (dz.abs().t() @ xd.abs()) + 1e-38
    return out, bound


def check(got, want, bound, what):
    got = got.detach().cpu().to(F64)
    assert got.shape == want.shape, what
    assert bool(torch.isfinite(got).all()), what + " is not finite"
    far = (got - want).abs() - bound
    at = int(far.argmax())
    assert float(far.max()) <= 0, (what, "element", at, float(got.flatten()[at]), float(want.flatten()[at]),
                                   float(bound.expand_as(want).flatten()[at]))


def check_norm_rel(got, want, rel, what):
    """The distance as a whole: roundings are independent, so together they are smaller than each could be."""
    size = float(want.norm())
    off = float((got.detach().cpu().to(F64) - want).norm())
    assert off <= rel * size + 1e-37, (what, off / max(size, 1e-300))
