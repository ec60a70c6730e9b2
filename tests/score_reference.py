"""Log probabilities, entropies and alternatives of the vocabulary head in 64 bits, with the bounds that the tests hold the kernels to."""
import torch

F64 = torch.float64
HALF16 = torch.finfo(torch.bfloat16).eps / 2
HALF32 = torch.finfo(torch.float32).eps / 2


def score(x, W, target, K=0, tau=1.0, dlogp=None, dentropy=None, low=False):
    """Results in 64 bits, straight from their definitions, and for each a bound on the kernel's error.  low: dW takes what rounding dz loses, rounded once more."""
    T, d = x.shape
    V = W.shape[0]
    xd, Wd = x.to(F64), W.to(F64)
    z = xd @ Wd.t()
    has = (target >= 0) & (target < V)
    y = torch.where(has, target, 0).long()[:, None]
    top, best = z.max(1, keepdim=True)
    o = (top - z) / tau
    e = (-o).exp().scatter(1, best, 0.0)
    R, Q = e.sum(1), (e * o).sum(1)
    log_top = -torch.log1p(R)
    log_p = log_top[:, None] - o
    logp, entropy = log_p.gather(1, y)[:, 0], Q / (1 + R) - log_top
    # a logit of the product is a chain of d / 32 additions of sums of 32 products; sums in 32 bits: at most 31 terms of a lane, 2 steps across lanes, the strips of a
    # thread, and the threads; a logit over the temperature in units of log2 is rounded a few times
    spread = (xd.square() @ Wd.square().t()).sqrt()
    off = ((d / 32 + 16) * 2 * HALF32 * (z.abs() + 4 * spread)).amax(1) / tau
    rel = off + (64 + V / 64 / 16 + 8 * z.abs().amax(1) / tau) * HALF32
    near = rel * R / (1 + R)                                # of log(1 + R)
    zero = lambda v: torch.where(has if v.dim() == 1 else has[:, None], v, torch.zeros_like(v))  # noqa: E731
    out = {"logp": zero(logp), "entropy": zero(entropy), "lse": zero(top[:, 0] / tau - log_top)}
    bound = {"logp": near + 4 * HALF32 * logp.abs(), "entropy": 2 * rel * (2 * R + Q) / (1 + R) + 16 * HALF32 * entropy,
             "lse": near + 2 * HALF32 * out["lse"].abs()}
    if K:
        # logits that are equal but for the last of 64 bits are equal: of those the lower column comes first
        step = 2.0 ** 40 / z.abs().amax(1, keepdim=True).clamp(min=1e-300)
        order = (z * step).round().sort(dim=1, descending=True, stable=True).indices[:, :K]
        out["ids"] = torch.where(has[:, None], order, -1).int()
        of_top = log_p.gather(1, order)
        out["top"] = zero(of_top)
        bound["top"] = near[:, None] + 4 * HALF32 * of_top.abs()
    if dlogp is not None:
        u, v = zero(dlogp.to(F64)) / tau, zero(torch.zeros(T) if dentropy is None else dentropy.to(F64)) / tau
        p = log_p.exp()
        inner = log_p + entropy[:, None]
        dz = -p * (u[:, None] + v[:, None] * inner)
        dz.scatter_(1, y, (-torch.expm1(logp) * u - p.gather(1, y)[:, 0] * v * inner.gather(1, y)[:, 0])[:, None])
        # dz is rounded to bf16; its exponentials are off by what logits and lse are, and so is log p + entropy, at the size of the logits
        tol = (off + bound["lse"] + bound["entropy"] + (16 + 8 * z.abs().amax(1) / tau) * HALF32)[:, None]
        big = p * (u.abs()[:, None] + v.abs()[:, None] * (inner.abs() + 1))
        err = HALF16 * dz.abs() + 8 * (tol + 8 * HALF32) * big
        out["dx"], out["dW"] = dz @ Wd, dz.t() @ xd
        bound["dx"] = HALF16 * out["dx"].abs() + err @ Wd.abs() + V * HALF32 * (dz.abs() @ Wd.abs()) + 1e-38
        if low:
            err = err - (HALF16 - HALF16 ** 2) * dz.abs()
        bound["dW"] = HALF16 * out["dW"].abs() + err.t() @ xd.abs() + T * HALF32 * (dz.abs().t() @ xd.abs()) + 1e-38
    return out, bound


def check(got, want, bound, what):
    got = got.detach().cpu().to(F64)
    assert got.shape == want.shape, what
    assert bool(torch.isfinite(got).all()), what + " is not finite"
    far = (got - want).abs() - bound
    at = int(far.argmax())
    assert float(far.max()) <= 0, (what, "element", at, float(got.flatten()[at]), float(want.flatten()[at]), float(bound.expand_as(want).flatten()[at]))


def check_all(got, want, bound):
    for n, w in want.items():
        if n == "ids":
            same = got[n].cpu() == w
            assert bool(same.all()), ("ids", torch.nonzero(~same)[0].tolist(), got[n].cpu()[~same][0], w[~same][0])
        else:
            check(got[n], w, bound[n], n)
