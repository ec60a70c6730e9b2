"""Log probabilities, entropies, alternatives and their gradients against 64 bits: sizes, masks, both tile edges, equal logits, sure tokens, and where what."""
import ctypes
import math

import pytest
import torch

import score_reference as R
from paper_2604_00785_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def inputs(T, d, V, masked=0.3, sure=6.0, seed=0):
    """Tokens that the model is more or less sure of."""
    g = torch.Generator().manual_seed(seed)
    W = (0.05 * torch.randn(V, d, generator=g)).bfloat16()
    y = torch.randint(0, V, (T,), generator=g)
    x = (torch.randn(T, d, generator=g) + torch.rand(T, 1, generator=g) * sure / (0.05 ** 2 * d) * W[y].float()).bfloat16()
    y = torch.where(torch.rand(T, generator=g) < 0.3, torch.randint(0, V, (T,), generator=g), y)
    target = torch.where(torch.rand(T, generator=g) < masked, torch.tensor([-100, V, -1, 1 << 30])[torch.randint(0, 4, (T,), generator=g)], y).int()
    target[T // 2] = y[T // 2]
    return x, W, target, torch.randn(T, generator=g), torch.randn(T, generator=g)


def junk(*shape, dtype=torch.float32):
    return torch.full(shape, -77, dtype=dtype, device=DEV) if dtype == torch.int32 else torch.full(shape, float("nan"), dtype=dtype, device=DEV)


def forward(x, W, target, K=0, tau=1.0, edge=0, path=0):
    """path 1: alternatives from the logits, 2: from strips of them, 100 + p: from logits in p parts of the reduction, 0: as the rule has it."""
    x, W, target = x.to(DEV), W.to(DEV), target.to(DEV)
    (T, d), V = x.shape, W.shape[0]
    out = {"logp": junk(T), "entropy": junk(T), "lse": junk(T)}
    ids, top = (junk(T, K, dtype=torch.int32), junk(T, K)) if K else (None, None)
    n = B.moe_head_score_fwd_workspace_bytes(T, d, V, K)
    ws = torch.full((n if path == 0 else n + max(1, path - 100) * (T + 15) * (V + 64) * 4,), 255, dtype=torch.uint8, device=DEV)
    if edge == 0 and path == 0:
        B.moe_head_score_fwd(x, W, target, tau, out["logp"], out["entropy"], out["lse"], ids, top, ws)
    else:
        p = lambda t: None if t is None else ctypes.c_void_p(t.data_ptr())  # noqa: E731
        edges = (ctypes.c_int * 2)(edge, path)
        rc = B.load().moe_head_score_fwd_edges(p(x), p(W), p(target), ctypes.c_float(tau), T, d, V, K, p(out["logp"]), p(out["entropy"]), p(out["lse"]), p(ids), p(top),
                                               p(ws), ctypes.c_size_t(ws.numel()), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream), edges)
        assert rc == 0 and edge in (0, edges[0])
    if K:
        out.update(ids=ids, top=top)
    return out


def backward(x, W, target, tau, f, dlogp, dentropy, v_piece=0, edge=0, parts=0):
    x, W, target = x.to(DEV), W.to(DEV), target.to(DEV)
    (T, d), V = x.shape, W.shape[0]
    dx, dW = junk(T, d, dtype=torch.bfloat16), junk(V, d, dtype=torch.bfloat16)
    ws = torch.full((B.moe_head_score_bwd_workspace_bytes(T, d, V, v_piece) + parts * (T + 15) * (V + 64) * 4,), 255, dtype=torch.uint8, device=DEV)
    dlogp, dentropy = dlogp.to(DEV), None if dentropy is None else dentropy.to(DEV)
    if edge == 0 and parts == 0:
        B.moe_head_score_bwd(x, W, target, tau, f["logp"], f["entropy"], f["lse"], dlogp, dentropy, v_piece, dx, dW, ws)
    else:
        p = lambda t: None if t is None else ctypes.c_void_p(t.data_ptr())  # noqa: E731
        edges = (ctypes.c_int * 2)(edge + 1000 * parts, 0)
        rc = B.load().moe_head_score_bwd_edges(p(x), p(W), p(target), ctypes.c_float(tau), p(f["logp"]), p(f["entropy"]), p(f["lse"]), p(dlogp), p(dentropy), T, d, V,
                                               v_piece, p(dx), p(dW), p(ws), ctypes.c_size_t(ws.numel()), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream), edges)
        assert rc == 0 and edge in (0, edges[0])
    return {"dx": dx, "dW": dW}


SHAPES = [(1, 64, 1, 1, 1.0), (2, 64, 7, 7, 1.0), (1, 64, 200, 64, 1.3), (1, 2048, 5000, 20, 1.0), (17, 128, 131, 5, 0.7), (40, 64, 70001, 8, 1.0), (129, 704, 3001, 1, 2.5),
          (256, 64, 257, 0, 1.0), (257, 64, 300, 20, 0.5), (300, 192, 1031, 64, 1.0), (1000, 128, 515, 16, 1.0), (4200, 64, 999, 3, 1.0)]


@pytest.mark.parametrize("edge", [128, 256, 0])
@pytest.mark.parametrize("T,d,V,K,tau", SHAPES)
def test_forward(T, d, V, K, tau, edge):
    x, W, target, _, _ = inputs(T, d, V, seed=T)
    want, bound = R.score(x, W, target, K, tau)
    for path in (0, 1, 2) if 0 < K and V <= 16384 else (0,):
        R.check_all(forward(x, W, target, K, tau, edge, path), want, bound)


@pytest.mark.parametrize("path", [1, 2])
@pytest.mark.parametrize("T,V,K", [(3, 16384, 64), (300, 16384, 64), (260, 2049, 60), (260, 2048, 61), (260, 2048, 60), (300, 4097, 20), (300, 8193, 3), (300, 70, 64), (3, 70, 64), (3, 1087, 64),
                                   (257, 543, 64), (257, 255, 60), (3, 8192, 64), (200, 2049, 64), (256, 5000, 60)])
def test_both_ways_to_the_alternatives(T, V, K, path):
    """At the borders of what a workgroup, a thread and a list of candidates hold."""
    x, W, target, _, _ = inputs(T, 64, V, seed=V)
    want, bound = R.score(x, W, target, K)
    R.check_all(forward(x, W, target, K, path=path), want, bound)


@pytest.mark.parametrize("edge", [128, 256, 0])
@pytest.mark.parametrize("T,d,V,tau", [(1, 64, 1, 1.0), (1, 64, 130, 1.0), (5, 128, 1000, 0.7), (64, 192, 333, 1.0), (129, 64, 2000, 1.5), (300, 128, 515, 1.0), (700, 64, 1031, 0.9)])
def test_backward(T, d, V, tau, edge):
    x, W, target, dlogp, dentropy = inputs(T, d, V, seed=T + 1)
    f = forward(x, W, target, 0, tau)
    for de in (dentropy, None):
        want, bound = R.score(x, W, target, 0, tau, dlogp, de)
        got = backward(x, W, target, tau, f, dlogp, de, edge=edge)
        for n in ("dx", "dW"):
            R.check(got[n], want[n], bound[n], n)
    off = target.cpu() < 0
    assert bool((got["dx"].cpu()[off] == 0).all())


@pytest.mark.parametrize("T,d,V,K,tau,parts", [(1, 512, 300, 5, 1.0, 8), (1, 512, 1, 0, 1.0, 8), (7, 2112, 610, 0, 0.7, 8), (7, 2112, 610, 20, 0.7, 0), (40, 320, 257, 64, 1.0, 5),
                                               (65, 576, 130, 2, 1.0, 2), (100, 704, 3001, 20, 1.0, 3), (129, 192, 515, 64, 1.0, 2), (130, 256, 2049, 0, 1.3, 4), (200, 1024, 999, 0, 1.0, 0),
                                               (257, 512, 70, 64, 1.0, 2), (300, 1024, 1031, 0, 1.0, 4), (300, 1024, 1031, 7, 1.0, 0), (2000, 512, 257, 3, 1.0, 2), (3, 256, 16384, 64, 1.0, 2),
                                               (1, 4096, 256, 1, 1.0, 0), (1030, 2048, 256, 0, 1.0, 0)])
def test_parts_of_the_reduction(T, d, V, K, tau, parts):
    """Few tiles with long reductions: the logits' summands apart, forward and backward."""
    x, W, target, dlogp, dentropy = inputs(T, d, V, seed=T + d)
    want, bound = R.score(x, W, target, K, tau, dlogp, dentropy)
    f = forward(x, W, target, K, tau, path=100 + parts if parts else 0)
    R.check_all(f, {n: want[n] for n in f}, bound)
    again = forward(x, W, target, K, tau, path=100 + parts if parts else 0)
    got = backward(x, W, target, tau, f, dlogp, dentropy, parts=parts)
    for n in f:
        assert torch.equal(f[n], again[n]), n
    for n in ("dx", "dW"):
        R.check(got[n], want[n], bound[n], n)


@pytest.mark.parametrize("K", [0, 3])
@pytest.mark.parametrize("T", [3, 1030])
@pytest.mark.parametrize("V", [3, 511, 513, 2048, 2050, 4096, 4099, 8192, 8193, 16384])
def test_logits_themselves_at_the_borders_of_a_workgroup(T, V, K):
    x, W, target, _, _ = inputs(T, 128, V, masked=0.9 if T > 100 else 0.0, seed=V + 1)
    x[0], W[V - 1] = 0, W[0]                             # equal logits
    want, bound = R.score(x, W, target, K)
    R.check_all(forward(x, W, target, K, path=102), want, bound)


@pytest.mark.parametrize("T", [20, 400])
def test_what_is_not_a_number_in_parts(T):
    x, W, target, dlogp, dentropy = inputs(T, 256, 300, masked=0.0, seed=17)
    target[3] = -100
    x[3] = float("nan")                                  # a masked token: leaves no trace
    for K in (0, 4):
        want = forward(x, W, target, K, path=103)
        grads = backward(x, W, target, 1.0, want, dlogp, dentropy, parts=3)
        assert all(bool(torch.isfinite(t).all()) for t in (*want.values(), *grads.values()))
        assert all(bool((want[n][3] == (-1 if n == "ids" else 0)).all()) for n in want) and bool((grads["dx"][3] == 0).all())
        x2 = x.clone()
        x2[5, 200], x2[9], W2 = float("nan"), float("inf"), W.clone()
        got = forward(x2, W, target, K, path=103)
        keep = torch.ones(T, dtype=torch.bool)
        keep[[5, 9]] = False
        for n in want:
            assert torch.equal(got[n].cpu()[keep], want[n].cpu()[keep]), n
            assert n == "ids" or bool(torch.isnan(got[n].cpu()[~keep]).all()), n
        back = backward(x2, W, target, 1.0, got, dlogp, dentropy, parts=3)
        assert torch.equal(back["dx"].cpu()[keep], grads["dx"].cpu()[keep]) and bool(torch.isnan(back["dx"].cpu()[~keep]).any(1).all())
        W2[100, 3] = float("nan")
        got = forward(x, W2, target, K, path=103)
        assert all(bool(torch.isnan(got[n].cpu()[target >= 0]).all()) for n in ("logp", "entropy", "lse"))


def test_parts_in_a_graph():
    """The rule's own choice for a few tokens of long rows, masks that change between the replays, a workspace that others write to."""
    for T, K in ((7, 5), (300, 0)):
        d, V = 2048, 610
        x, W, target, dlogp, dentropy = inputs(T, d, V, seed=18)
        assert B.moe_head_score_fwd_workspace_bytes(T, d, V, K) > B.moe_head_score_fwd_workspace_bytes(T, 64, V, K) + T * V * 4
        s = B.ScoreBuffers(T, d, V, K, device=DEV)
        xg, Wg, yg, dl, de = (t.to(DEV) for t in (x, W, target, dlogp, dentropy))
        s.run_fwd(xg, Wg, yg, 0.9)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.run_fwd(xg, Wg, yg, 0.9)
            s.run_bwd(xg, Wg, yg, dl, de, 0.9)
        for shift in (0, 1, 2):
            y2 = target.roll(shift)
            yg.copy_(y2)
            s.ws.fill_(255)
            graph.replay()
            want = forward(x, W, y2, K, 0.9)
            want.update(backward(x, W, y2, 0.9, want, dlogp, dentropy))
            torch.cuda.synchronize()
            assert all(torch.equal(getattr(s, n), want[n]) for n in want), shift


@pytest.mark.parametrize("T,d,V,masked,piece,parts", [(17, 64, 300, 0.3, 0, 0), (129, 64, 515, 0.0, 0, 0), (200, 704, 2000, 0.2, 0, 0), (256, 128, 1031, 0.0, 0, 0), (256, 192, 700, 0.0, 256, 0),
                                                      (300, 64, 515, 0.3, 0, 0), (250, 512, 515, 0.0, 0, 2), (600, 1024, 515, 0.6, 0, 3)])
def test_what_rounding_loses_is_in_dw_for_few_tokens(T, d, V, masked, piece, parts):
    x, W, target, dlogp, dentropy = inputs(T, d, V, masked=masked, sure=1.0, seed=T + 5)
    assert int(((target >= 0) & (target < V)).sum()) <= 256
    f = forward(x, W, target)
    want, bound = R.score(x, W, target, 0, 1.0, dlogp, dentropy, low=True)
    got = backward(x, W, target, 1.0, f, dlogp, dentropy, piece, parts=parts)
    for n in ("dx", "dW"):
        R.check(got[n], want[n], bound[n], n)
    # the error is that of dW's own rounding, some 0.0017 of it, where dz's would add as much
    assert float((got["dW"].cpu().double() - want["dW"]).norm() / want["dW"].norm()) < 2.0 ** -8 / 3 ** 0.5


def test_backward_in_pieces_of_the_vocabulary():
    x, W, target, dlogp, dentropy = inputs(200, 128, 1500, seed=3)
    f = forward(x, W, target)
    want, bound = R.score(x, W, target, 0, 1.0, dlogp, dentropy)
    for piece in (256, 512, 1536):
        got = backward(x, W, target, 1.0, f, dlogp, dentropy, piece)
        for n in ("dx", "dW"):
            R.check(got[n], want[n], bound[n], (n, piece))


def test_log_probability_alone_is_minus_the_loss():
    """dlogp = -dloss and no entropy: the gradients of the cross entropy."""
    x, W, target, w, _ = inputs(300, 128, 515, seed=4)
    f = forward(x, W, target)
    got = backward(x, W, target, 1.0, f, -w, None)
    T, d, V = 300, 128, 515
    h = B.HeadBuffers(T, d, V)
    h.run_fwd(x.to(DEV), W.to(DEV), target.to(DEV))
    h.run_bwd(x.to(DEV), W.to(DEV), target.to(DEV), w.to(DEV))
    assert float((f["logp"] + h.loss).abs().max()) < 1e-5 and float((f["lse"] - h.lse).abs().max()) < 1e-5
    for a, b in ((got["dx"], h.dx), (got["dW"], h.dW)):
        # either is rounded once on its way and once at the end
        assert float((a.double() - b.double()).norm() / b.double().norm()) < 4 * R.HALF16


def test_reference_gradients_against_differentiation():
    x, W, target, dlogp, dentropy = inputs(9, 64, 31, seed=5)
    xd, Wd = x.double().requires_grad_(), W.double().requires_grad_()
    tau = 0.8
    lp = torch.log_softmax(xd @ Wd.t() / tau, 1)
    has = (target >= 0) & (target < 31)
    y = torch.where(has, target, 0).long()[:, None]
    total = (lp.gather(1, y)[:, 0] * dlogp.double() - (lp.exp() * lp).sum(1) * dentropy.double()) * has
    total.sum().backward()
    want, _ = R.score(x, W, target, 0, tau, dlogp, dentropy)
    assert torch.allclose(want["dx"], xd.grad, rtol=1e-9, atol=1e-11) and torch.allclose(want["dW"], Wd.grad, rtol=1e-9, atol=1e-11)
    # and against differences
    g = torch.Generator().manual_seed(6)
    dx, dW, h = torch.randn(x.shape, generator=g, dtype=torch.float64), torch.randn(W.shape, generator=g, dtype=torch.float64), 1e-5
    value = lambda s: sum(float((R.score(x.double() + s * dx, W.double() + s * dW, target, 0, tau)[0][n] * w.double()).sum())  # noqa: E731
                          for n, w in (("logp", dlogp), ("entropy", dentropy)))
    slope, along = (value(h) - value(-h)) / (2 * h), float((want["dx"] * dx).sum() + (want["dW"] * dW).sum())
    assert abs(slope - along) < 1e-6 * (abs(along) + 1)


@pytest.mark.parametrize("T", [3, 300])
def test_sure_tokens_keep_their_digits(T):
    """Log probabilities and entropies down to e^-80: relative, not absolute, accuracy."""
    d, V, K = 128, 700, 5
    x, W, target, _, _ = inputs(T, d, V, masked=0.0, seed=7)
    scale = torch.linspace(10.0, 90.0, T)[:, None]
    y = target.long()
    x = (x.float() * 0.1 + scale / (0.05 ** 2 * d) * W[y].float()).bfloat16()
    want, bound = R.score(x, W, target, K)
    got = forward(x, W, target, K)
    R.check_all(got, want, bound)
    assert float(want["logp"].max()) > -1e-20 and bool((got["entropy"] > 0).all())
    # at this size of logits a probability is off by some 1e-4 of itself, however small it is
    assert float(((got["logp"].cpu().double() - want["logp"]) / want["logp"]).abs().max()) < 1e-3
    assert float(((got["entropy"].cpu().double() - want["entropy"]) / want["entropy"]).abs().max()) < 1e-3


@pytest.mark.parametrize("path", [1, 2])
@pytest.mark.parametrize("edge", [128, 256])
def test_equal_logits(edge, path):
    """All equal, some equal, and the lower column first."""
    T, d, V, K = 6, 64, 3001, 64
    x, W, target, _, _ = inputs(T, d, V, masked=0.0, seed=8)
    x[0] = 0
    x[1] = 0
    x[1, 0] = 1.0
    W[:, 0] = torch.tensor([0.5, 0.25, 0.125])[torch.arange(V) % 3].bfloat16()
    W[2000:2100] = W[100:200]                            # rows twice
    W[2900:] = W[100:201]
    want, bound = R.score(x, W, target, K)
    got = forward(x, W, target, K, 1.0, edge, path)
    assert want["ids"][0].tolist() == list(range(K)) and want["ids"][1].tolist() == list(range(0, 3 * K, 3))
    R.check_all(got, want, bound)
    assert abs(float(got["entropy"][0]) - math.log(V)) < 1e-5


@pytest.mark.parametrize("path", [1, 2])
@pytest.mark.parametrize("edge", [128, 256])
def test_the_largest_side_by_side(edge, path):
    """Alternatives that all lie in the columns of one lane, of neighbouring lanes, of one strip, and at the ends of the vocabulary."""
    d, V, K = 64, 5003, 40
    g = torch.Generator().manual_seed(9)
    for columns in (torch.arange(4)[None, :] + 16 * torch.arange(8)[:, None] + 1280, torch.arange(4)[None, :] + 16 * torch.arange(4)[:, None] + 1284,
                    torch.arange(1280, 1408), torch.arange(V - 30, V), torch.arange(0, 50), torch.arange(0, V, 128)):
        columns = columns.flatten()
        W = (0.05 * torch.randn(V, d, generator=g)).bfloat16()
        x = torch.randn(4, d, generator=g).bfloat16()
        W[columns] = (W[columns].float() + 0.02 * torch.rand(len(columns), 1, generator=g) * x[:1].float() + 0.2 * x[:1].float()).bfloat16()
        target = torch.tensor([int(columns[0]), 0, V - 1, 17]).int()
        want, bound = R.score(x, W, target, K)
        R.check_all(forward(x, W, target, K, 1.0, edge, path), want, bound)


def test_more_candidates_than_there_is_room_for():
    """Large logits in strips that few threads look through: they are taken one after the other."""
    d, V, K = 64, 1 << 18, 64
    g = torch.Generator().manual_seed(10)
    W = (0.02 * torch.randn(V, d, generator=g)).bfloat16()
    x = torch.randn(3, d, generator=g).bfloat16()
    column = torch.arange(V)
    for edge, few in ((128, column // 64 % 64 < 3), (256, column // 128 % 64 < 6)):
        W2 = W.clone()
        W2[few] = (W[few].float() + 0.1 * x[1:2].float()).bfloat16()
        target = torch.tensor([5, 17, V - 1]).int()
        want, bound = R.score(x, W2, target, K)
        R.check_all(forward(x, W2, target, K, 1.0, edge), want, bound)


@pytest.mark.parametrize("T,V,few", [(2, 16384, lambda c: c // 16 % 256 < 2), (2, 8000, lambda c: c // 16 % 256 < 10), (2, 8192, lambda c: c // 16 % 256 < 20), (300, 2000, lambda c: c // 4 % 64 < 3), (300, 4000, lambda c: c // 4 % 128 < 3),
                                     (300, 8000, lambda c: c // 8 % 128 < 2), (300, 16384, lambda c: c // 16 % 128 < 2)])
def test_more_candidates_among_the_logits_themselves(T, V, few):
    """The same where all logits are looked at: large ones in the columns of few threads, and all equal."""
    d, K = 64, 60
    x, W, target, _, _ = inputs(T, d, V, masked=0.0, seed=16)
    W[few(torch.arange(V))] += (0.05 * x[1].float()).bfloat16()
    x[0] = 0
    want, bound = R.score(x, W, target, K)
    R.check_all(forward(x, W, target, K, path=1), want, bound)


def test_nothing_but_masked_tokens():
    for T in (5, 300):
        x, W, target, dlogp, dentropy = inputs(T, 64, 100, seed=11)
        target[:] = -100
        f = forward(x, W, target, 4)
        assert all(bool((f[n] == 0).all()) for n in ("logp", "entropy", "lse", "top")) and bool((f["ids"] == -1).all())
        g = backward(x, W, target, 1.0, f, dlogp, dentropy)
        assert bool((g["dx"] == 0).all()) and bool((g["dW"] == 0).all())


@pytest.mark.parametrize("path", [0, 2])
@pytest.mark.parametrize("T", [20, 400])
def test_what_is_not_a_number_stays_where_it_is(T, path):
    x, W, target, dlogp, dentropy = inputs(T, 64, 300, masked=0.0, seed=12)
    clean = forward(x, W, target, 4, path=path)
    target[3] = -100
    x2, dl2, de2 = x.clone(), dlogp.clone(), dentropy.clone()
    x2[3], dl2[3], de2[3] = float("nan"), float("nan"), float("inf")              # a masked token: leaves no trace
    want = forward(x, W, target, 4, path=path)
    got = forward(x2, W, target, 4, path=path)
    assert all(torch.equal(got[n], want[n]) for n in got)
    a, b = backward(x, W, target, 1.0, want, dlogp, dentropy), backward(x2, W, target, 1.0, got, dl2, de2)
    assert all(torch.equal(a[n], b[n]) for n in a)
    x2[5, 7], x2[9] = float("nan"), float("inf")                                  # tokens that count: NaN for themselves alone
    got = forward(x2, W, target, 4, path=path)
    keep = torch.ones(T, dtype=torch.bool)
    keep[[5, 9]] = False
    for n in ("logp", "entropy", "lse", "top"):
        assert bool(torch.isnan(got[n].cpu()[~keep]).all()), n
        assert torch.equal(got[n].cpu()[keep], want[n].cpu()[keep]), n
    assert torch.equal(got["ids"].cpu()[keep], want["ids"].cpu()[keep]) and int(got["ids"].max()) < 300 and int(got["ids"].min()) >= -1
    W2 = W.clone()
    W2[100, 3] = float("nan")                                                     # a column: NaN for every token
    got = forward(x, W2, target, 4, path=path)
    on = target >= 0
    assert all(bool(torch.isnan(got[n].cpu()[on]).all()) for n in ("logp", "entropy", "lse"))
    assert all(torch.equal(clean[n].cpu()[keep & on], want[n].cpu()[keep & on]) for n in clean)


def test_logits_past_the_range_of_the_sums():
    x, W, target, _, _ = inputs(4, 64, 300, masked=0.0, seed=13)
    big = x.clone()
    big[1] = (x[1].float() * 1e12).bfloat16()
    for t in (forward(big, W, target, 3), forward(x, W, target, 3, 1e-12)):
        assert bool(torch.isnan(t["logp"][1])) and bool(torch.isnan(t["entropy"][1]))


def test_the_same_bits_again_in_a_graph_and_on_another_stream():
    for T, K in ((7, 5), (300, 20)):
        x, W, target, dlogp, dentropy = inputs(T, 128, 1031, seed=14)
        first = forward(x, W, target, K, 0.9)
        first.update(backward(x, W, target, 0.9, first, dlogp, dentropy))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = forward(x, W, target, K, 0.9)
            again.update(backward(x, W, target, 0.9, again, dlogp, dentropy))
        side.synchronize()
        assert all(torch.equal(first[n], again[n]) for n in first)
        d, V = 128, 1031
        g = {n: junk(*v.shape, dtype=v.dtype) for n, v in first.items()}
        ws = torch.empty(max(B.moe_head_score_fwd_workspace_bytes(T, d, V, K), B.moe_head_score_bwd_workspace_bytes(T, d, V)), dtype=torch.uint8, device=DEV)
        xg, Wg, yg, dl, de = (t.to(DEV) for t in (x, W, target, dlogp, dentropy))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.moe_head_score_fwd(xg, Wg, yg, 0.9, g["logp"], g["entropy"], g["lse"], g["ids"], g["top"], ws)
            B.moe_head_score_bwd(xg, Wg, yg, 0.9, g["logp"], g["entropy"], g["lse"], dl, de, 0, g["dx"], g["dW"], ws)
        for shift in (0, 1, 2):                                                   # other masks between the replays
            y2 = target.roll(shift)
            yg.copy_(y2)
            ws.fill_(255)
            graph.replay()
            want = forward(x, W, y2, K, 0.9)
            want.update(backward(x, W, y2, 0.9, want, dlogp, dentropy))
            torch.cuda.synchronize()
            assert all(torch.equal(g[n], want[n]) for n in g), shift


def test_offsets_past_32_bits():
    """Weights of more than 2^32 bytes; the largest logits at their end."""
    T, d, V, K = 2, 4096, 1 << 20, 3
    W = torch.zeros(V, d, dtype=torch.bfloat16, device=DEV)
    at = [V - 1, V - 70000, V // 2 + 5, 12345]
    W[at, 0] = torch.tensor([3.0, 2.0, 1.0, 2.5], device=DEV).bfloat16()
    x = torch.zeros(T, d, dtype=torch.bfloat16, device=DEV)
    x[0, 0], x[1, 0] = 4.0, -4.0
    got = forward(x, W, torch.tensor([V - 1, V - 1]).int(), K)
    assert got["ids"].tolist() == [[V - 1, 12345, V - 70000], [0, 1, 2]]
    lse = [math.log(V - 4 + sum(math.exp(s * 4 * v) for v in (3.0, 2.0, 1.0, 2.5))) for s in (1, -1)]
    for t, s in ((0, 1), (1, -1)):
        assert abs(float(got["lse"][t]) - lse[t]) < 1e-4 and abs(float(got["logp"][t]) - (s * 12.0 - lse[t])) < 1e-4


def test_more_tokens_than_a_row_of_the_grid_has_workgroups():
    T, d, V = (1 << 20) + 3, 64, 3
    g = torch.Generator(device=DEV).manual_seed(15)
    x, W = torch.randn(T, d, generator=g, device=DEV).bfloat16(), (0.1 * torch.randn(V, d, generator=g, device=DEV)).bfloat16()
    target = (torch.arange(T, device=DEV) % 4 - 1).int()
    got = forward(x, W, target, 2)
    for at in (slice(0, 400), slice(T - 400, T)):
        want, bound = R.score(x[at].cpu(), W.cpu(), target[at].cpu(), 2)
        R.check_all({n: v[at] for n, v in got.items()}, want, bound)
