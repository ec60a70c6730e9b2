"""Norms of queries and keys with the rotation, and gradients' norm and clipping, in 64 bits, with the bounds that the tests hold the kernels to."""
import math

import torch

F64 = torch.float64
HALF16 = torch.finfo(torch.bfloat16).eps / 2
HALF32 = torch.finfo(torch.float32).eps / 2
LEAST16 = 2.0 ** -133                                # the smallest bf16 number above zero, in absolute terms what a rounding next to zero can lose


def turn(v, pos, freq, pairs, back=False):
    """(result, |a| + |b| of each pair) on [T, H, D]; a frequency for each pair of the first columns."""
    n = 0 if freq is None else freq.numel()
    out, size = v.clone(), v.abs()
    if n:
        angle = (pos.to(F64)[:, None] * freq.to(F64))[:, None, :]
        c, s = angle.cos(), -angle.sin() if back else angle.sin()
        at = torch.arange(n)
        one, two = (2 * at, 2 * at + 1) if pairs else (at, at + n)
        a, b = v[:, :, one], v[:, :, two]
        out[:, :, one], out[:, :, two] = a * c - b * s, a * s + b * c
        size[:, :, one] = size[:, :, two] = a.abs() + b.abs()
    return out, size


def qk_norm(x, w, pos, freq, pairs, eps):
    """One side's result and the bound on its error.

    A root is off by half of its sum's 24 roundings, and two of its own; angles of up to a turn in 32 bits are off by 7 halves of a step, sine and
    cosine by 8; four products and a difference: 44 in all, of the pair's size."""
    x, w = x.to(F64), w.to(F64)
    v = x / (x.square().mean(2, keepdim=True) + eps).sqrt() * w
    y, size = turn(v, pos, freq, pairs)
    return y, HALF16 * y.abs() + 44 * HALF32 * size + LEAST16


def qk_norm_bwd(dy, x, w, pos, freq, pairs, eps):
    """(dx, bound, dw, bound)."""
    x, w, dy = x.to(F64), w.to(F64), dy.to(F64)
    T, H, _ = x.shape
    r = 1.0 / (x.square().mean(2, keepdim=True) + eps).sqrt()
    dv, size = turn(dy, pos, freq, pairs, back=True)
    g, big = dv * w, size * w.abs()
    dx = r * (g - x * (g * x).mean(2, keepdim=True) * r * r)
    # 18 for the turned gradient, 24 for a sum, three roots of 16 each, and some products
    high = r * (big + x.abs() * (big * x.abs()).mean(2, keepdim=True) * r * r)
    terms, tall = dv * x * r, size * x.abs() * r
    return (dx, HALF16 * dx.abs() + 100 * HALF32 * high + LEAST16, terms.sum((0, 1)),
            (44 * tall + (T * H + 64) * terms.abs()).sum((0, 1)) * HALF32 + 1e-38)


def grad_norm(grads):
    return math.sqrt(sum(float(g.to(F64).square().sum()) for g in grads))


def grad_clip(grads, largest):
    """(norm, scaled, bounds): the scale is rounded to 32 bits, the product too, and then to the type."""
    norm = grad_norm(grads)
    scale = min(1.0, largest / (norm + 1e-6))
    outs = [g.to(F64) * scale for g in grads]
    bounds = [o.abs() * ((HALF16 if g.dtype == torch.bfloat16 else 0.0) + 2.01 * HALF32) * (1 + HALF16) + (LEAST16 if g.dtype == torch.bfloat16 else 2.0 ** -149)
              for o, g in zip(outs, grads)]
    return norm, outs, bounds


def check(got, want, bound, what):
    got = got.detach().cpu().to(F64)
    assert got.shape == want.shape, what
    assert bool(torch.isfinite(got).all()), what + " is not finite"
    far = (got - want).abs() - bound
    if far.numel() == 0:
        return
    at = int(far.argmax())
    assert float(far.max()) <= 0, (what, "element", at, float(got.flatten()[at]), float(want.flatten()[at]), float(bound.expand_as(want).flatten()[at]))
