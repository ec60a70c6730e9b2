"""The gradient of the entropy where the model is sure of a column that is not the target: log p and the entropy are next to zero there, and their sum with them."""
import pytest
import torch

import score_reference as R
from paper_2604_00785_amd import binding as B
from test_gpu_head_score import DEV, backward, forward

pytestmark = pytest.mark.gpu
F64 = torch.float64


def inputs(T, d, V, tau, least, most, seed=0, masked=0.1):
    """Tokens whose likeliest column leads by `least` to `most` over the temperature; targets anywhere, one in ten the likeliest."""
    g = torch.Generator().manual_seed(seed)
    W = (0.05 * torch.randn(V, d, generator=g)).bfloat16()
    best = torch.randint(0, V, (T,), generator=g)
    lead = torch.linspace(least, most, T)[:, None] * tau
    x = (0.3 * tau * torch.randn(T, d, generator=g) + lead / (0.05 ** 2 * d) * W[best].float()).bfloat16()
    y = torch.where(torch.rand(T, generator=g) < 0.1, best, (best + 1 + torch.randint(0, max(V - 1, 1), (T,), generator=g)) % V)
    target = torch.where(torch.rand(T, generator=g) < masked, torch.tensor(-100), y).int()
    dlogp, dentropy = torch.randn(T, generator=g), torch.randn(T, generator=g)
    target[T // 2], dlogp[T // 2], dentropy[T // 2] = (best[T // 2] + 1) % V, 0.0, 1.0
    return x, W, target, torch.where(torch.rand(T, generator=g) < 0.7, torch.tensor(0.0), dlogp), dentropy


def gradients(x, W, target, tau, dlogp, dentropy):
    """dx and dW in 64 bits, with bounds of which that of a token is small beside its gradient, however sure it is.

    All columns but the likeliest have a p that is off by what their logit and lse are, `tol` of itself (as in score_reference.score), and a log p of 1 and more.  The likeliest
    one's log p = -log(1 + R) and the entropy are off by a share of themselves, `near` and that of the entropy's bound; some products in 32 bits, and dz in bf16."""
    want, bound = R.score(x, W, target, 0, tau)
    V = W.shape[0]
    xd, Wd = x.to(F64), W.to(F64)
    z = xd @ Wd.t()
    has = (target >= 0) & (target < V)
    y = torch.where(has, target, 0).long()[:, None]
    zero = lambda v: torch.where(has, v.to(F64), torch.zeros(len(has), dtype=F64)) / tau  # noqa: E731
    u, v = zero(dlogp)[:, None], zero(dentropy)[:, None]
    top, best = z.max(1, keepdim=True)
    o = (top - z) / tau
    log_top = -torch.log1p((-o).exp().scatter(1, best, 0.0).sum(1, keepdim=True))
    log_p = log_top - o
    p, H = log_p.exp(), want["entropy"][:, None]
    inner = log_p + H
    dz = -p * (u + v * inner)
    dz.scatter_(1, y, -torch.expm1(log_p.gather(1, y)) * u - p.gather(1, y) * v * inner.gather(1, y))
    near = (bound["lse"] - 2 * R.HALF32 * want["lse"].abs()).clamp(min=0)[:, None]
    of_H = bound["entropy"][:, None]
    spread = (xd.square() @ Wd.square().t()).sqrt()
    off = ((x.shape[1] / 32 + 16) * 2 * R.HALF32 * (z.abs() + 4 * spread)).amax(1, keepdim=True) / tau
    tol = off + bound["lse"][:, None] + of_H + (24 + 8 * z.abs().amax(1, keepdim=True) / tau) * R.HALF32
    err = 4 * tol * p * (u.abs() + v.abs() * (inner.abs() + 1))
    # (where it is the target the gradient of its log p is u (1 - p), 1 - p as near as log p)
    of_u = torch.where(best == y, (near / R.HALF32 / 16) - torch.expm1(log_top), torch.ones_like(H))
    of_top = p * (v.abs() * (near + of_H) + 16 * R.HALF32 * (u.abs() * of_u + v.abs() * (H + log_top.abs())))
    # Where it is another column than the target its gradient may be what the others', of which each is rounded, leave of zero; their sum is one of 32 bits.
    # (An entropy of half of 1/4 at most: the likeliest column is looked after by itself.)
    # (What rounding the target's loses is known, and goes into the sum as it goes into dx.)
    rounded = torch.full_like(dz, R.HALF16).scatter(1, y, 2 * R.HALF16 ** 2)
    others = (err + (rounded + (V / 2048 + 16) * R.HALF32) * dz.abs()).scatter(1, best, 0.0).sum(1, keepdim=True)
    sure = (H < 0.125) | (best == y)
    err.scatter_(1, best, torch.where(sure, of_top + torch.where(best == y, 0.0, others), err).gather(1, best))
    err = err + R.HALF16 * dz.abs()
    dx, dW = dz @ Wd, dz.t() @ xd
    return ({"dx": dx, "dW": dW}, {"dx": R.HALF16 * dx.abs() + err @ Wd.abs() + V * R.HALF32 * (dz.abs() @ Wd.abs()) + 1e-37,
                                   "dW": R.HALF16 * dW.abs() + err.t() @ xd.abs() + len(has) * R.HALF32 * (dz.abs().t() @ xd.abs()) + 1e-37}, has & (v[:, 0] != 0))


def check(got, want, bound, counts, what):
    # the bound tells a gradient from none at all, for every token
    assert bool((bound["dx"].norm(dim=1) < want["dx"].norm(dim=1) / 4)[counts].all()), what
    for n in ("dx", "dW"):
        R.check(got[n], want[n], bound[n], (n, what))


CASES = [(1, 64, 200, 1.0, 12, 12), (3, 128, 700, 1.0, 4, 40), (40, 128, 515, 1.0, 8, 60), (40, 128, 515, 0.1, 8, 30), (130, 64, 2049, 0.7, 3, 30), (256, 128, 1031, 1.0, 3, 25),
         (300, 192, 999, 1.0, 6, 16), (700, 64, 515, 1.5, 3, 60), (4200, 64, 300, 1.0, 4, 30),
         (2383, 192, 145, 1.0, 2, 20), (1400, 64, 3, 1.0, 2, 9), (1030, 128, 6, 0.5, 2, 12), (400, 64, 47, 0.9, 3, 9)]


@pytest.mark.parametrize("edge", [128, 256, 0])
@pytest.mark.parametrize("T,d,V,tau,least,most", CASES)
def test_sure_of_another_column(T, d, V, tau, least, most, edge):
    x, W, target, dlogp, dentropy = inputs(T, d, V, tau, least, most, seed=T)
    f = forward(x, W, target, 0, tau)
    for dl in (dlogp, torch.zeros(T), 3.0 * dentropy.roll(1)):
        want, bound, counts = gradients(x, W, target, tau, dl, dentropy)
        got = backward(x, W, target, tau, f, dl, dentropy, edge=edge)
        check(got, want, bound, counts, (T, edge))
        again = backward(x, W, target, tau, f, dl, dentropy, edge=edge)
        assert all(torch.equal(got[n], again[n]) for n in got)


@pytest.mark.parametrize("T,d,V,piece", [(40, 128, 515, 256), (300, 64, 1500, 512), (130, 64, 70001, 256), (700, 64, 300, 256)])
def test_in_pieces_of_the_vocabulary(T, d, V, piece):
    """The likeliest column in another piece than the one in hand."""
    x, W, target, dlogp, dentropy = inputs(T, d, V, 1.0, 6, 30, seed=T + 1)
    f = forward(x, W, target)
    want, bound, counts = gradients(x, W, target, 1.0, dlogp, dentropy)
    check(backward(x, W, target, 1.0, f, dlogp, dentropy, piece), want, bound, counts, piece)


@pytest.mark.parametrize("T,d,V,parts", [(3, 512, 300, 8), (40, 320, 257, 5), (130, 256, 2049, 4), (600, 1024, 515, 3), (7, 2112, 610, 0), (300, 1024, 1031, 0), (2, 256, 16384, 2)])
def test_with_the_logits_in_parts(T, d, V, parts):
    x, W, target, dlogp, dentropy = inputs(T, d, V, 1.0, 4, 30, seed=T + 2)
    f = forward(x, W, target)
    want, bound, counts = gradients(x, W, target, 1.0, dlogp, dentropy)
    check(backward(x, W, target, 1.0, f, dlogp, dentropy, parts=parts), want, bound, counts, parts)


def test_a_few_sure_tokens_among_others():
    """All the others as they are without them, and the same with the sure ones masked."""
    T, d, V = 520, 128, 515
    x, W, target, dlogp, dentropy = inputs(T, d, V, 1.0, 0.0, 0.0, seed=5, masked=0.2)
    sure = torch.zeros(T, dtype=torch.bool)
    sure[[1, 2, 77, 300, 519]] = True
    a = inputs(T, d, V, 1.0, 10, 20, seed=5)
    x[sure], target[sure], dlogp[sure] = a[0][sure], ((target[sure] + 3).clamp(min=0) % V), 0.0
    f = forward(x, W, target)
    got = backward(x, W, target, 1.0, f, dlogp, dentropy)
    want, bound, counts = gradients(x, W, target, 1.0, dlogp, dentropy)
    check(got, want, bound, counts & sure, "few")
    off = torch.where(sure, torch.tensor(-100, dtype=torch.int32), target)
    alone = backward(x, W, off, 1.0, forward(x, W, off), dlogp, dentropy)
    keep = ~sure & (target >= 0)
    err = (alone["dx"].cpu().double() - got["dx"].cpu().double())[keep].norm() / alone["dx"].cpu().double()[keep].norm()
    assert float(err) < R.HALF16 / 2
    # without a gradient of the entropy nothing depends on which column is the likeliest
    R.check(backward(x, W, target, 1.0, f, dlogp, None)["dx"], *(w["dx"] for w in R.score(x, W, target, 0, 1.0, dlogp, None)), "no entropy")


def test_in_a_graph_with_other_sure_tokens():
    T, d, V, tau = 300, 128, 515, 0.9
    x, W, target, dlogp, dentropy = inputs(T, d, V, tau, 4, 25, seed=9)
    s = B.ScoreBuffers(T, d, V, device=DEV)
    xg, Wg, yg, dl, de = (t.to(DEV) for t in (x, W, target, dlogp, dentropy))
    s.run_fwd(xg, Wg, yg, tau)
    s.run_bwd(xg, Wg, yg, dl, de, tau)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run_fwd(xg, Wg, yg, tau)
        s.run_bwd(xg, Wg, yg, dl, de, tau)
    for shift in (0, 1, 7):
        y2 = torch.where(torch.arange(T) % 3 == shift % 3, target.roll(shift), torch.tensor(-100, dtype=torch.int32))
        yg.copy_(y2)
        s.ws.fill_(255)
        graph.replay()
        f = forward(x, W, y2, 0, tau)
        back = backward(x, W, y2, tau, f, dlogp, dentropy)
        torch.cuda.synchronize()
        assert all(torch.equal(getattr(s, n), t) for n, t in {**f, **back}.items()), shift
