"""Norms of queries and keys with the rotation, forward and backward, against 64 bits; odd sizes, strides, positions, in place, in a graph, on another stream."""
import pytest
import torch

import qk_reference as R
from paper_2604_00785_amd import binding as B

pytestmark = pytest.mark.gpu
DEV, EPS = "cuda:0", 1e-5


def inputs(T, Hq, Hk, D, rotated, packed=False, far=5000, seed=0):
    g = torch.Generator().manual_seed(seed)
    rows = lambda H: (torch.randn(T, H, D, generator=g) * torch.exp(torch.randn(H, D, generator=g))).bfloat16()  # noqa: E731
    q, k = rows(Hq), rows(Hk)
    wq, wk = torch.rand(D, generator=g) + 0.5, torch.randn(D, generator=g)
    pos = torch.randint(0, far, (T,), generator=g).int()
    freq = (10000.0 ** (-torch.arange(0, rotated, 2) / rotated)).float() if rotated else None
    dqo, dko = torch.randn(T, Hq, D, generator=g).bfloat16(), torch.randn(T, Hk, D, generator=g).bfloat16()
    return q, k, wq, wk, pos, freq, dqo, dko


def dev(t):
    return None if t is None else t.to(DEV)


def packed_of(q, k, extra=24):
    """Queries and keys as columns of one matrix, with columns of something else beside them."""
    T, D = q.shape[0], q.shape[2]
    wide = torch.full((T, q.shape[1] * D + k.shape[1] * D + extra), 7.0, dtype=torch.bfloat16, device=DEV)
    a, b = q.shape[1] * D, (q.shape[1] + k.shape[1]) * D
    views = wide[:, :a].unflatten(1, (-1, D)), wide[:, a:b].unflatten(1, (-1, D))
    views[0].copy_(q)
    views[1].copy_(k)
    return wide, views


def new(t):
    return torch.full(t.shape, float("nan"), dtype=torch.bfloat16, device=DEV)


def run(q, k, wq, wk, pos, freq, pairs, eps=EPS):
    qo, ko = new(q), new(k)
    B.moe_qk_norm_rope(q, k, wq, wk, pos, freq, pairs, eps, qo, ko)
    return qo, ko


def run_bwd(dqo, dko, q, k, wq, wk, pos, freq, pairs, eps=EPS, dq=None, dk=None):
    T, Hq, D = q.shape
    dq, dk = new(q) if dq is None else dq, new(k) if dk is None else dk
    dwq, dwk = torch.full((D,), float("nan"), device=DEV), torch.full((D,), float("nan"), device=DEV)
    ws = torch.full((B.moe_qk_norm_rope_bwd_workspace_bytes(T, Hq, k.shape[1], D),), 255, dtype=torch.uint8, device=DEV)
    B.moe_qk_norm_rope_bwd(dqo, dko, q, k, wq, wk, pos, freq, pairs, eps, dq, dk, dwq, dwk, ws)
    return dq, dk, dwq, dwk


SHAPES = [(1, 1, 1, 8, 0), (1, 2, 1, 16, 16), (3, 1, 2, 24, 16), (1, 16, 16, 128, 128), (5, 3, 1, 64, 64), (7, 8, 2, 80, 80), (33, 5, 5, 96, 48), (19, 17, 3, 72, 64),
          (9, 6, 2, 128, 64), (11, 33, 1, 192, 96), (6, 4, 4, 256, 256), (4, 3, 2, 512, 512), (3, 2, 1, 264, 16), (130, 40, 8, 128, 128), (2049, 3, 1, 64, 32),
          (2051, 2, 2, 136, 128), (2048, 1, 1, 512, 256), (4098, 9, 4, 16, 16)]


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("T,Hq,Hk,D,rotated", SHAPES)
def test_against_64_bits(T, Hq, Hk, D, rotated, pairs):
    q, k, wq, wk, pos, freq, dqo, dko = inputs(T, Hq, Hk, D, rotated)
    args = [dev(t) for t in (q, k, wq, wk, pos, freq)]
    qo, ko = run(*args, pairs)
    R.check(qo, *R.qk_norm(q, wq, pos, freq, pairs, EPS), "q")
    R.check(ko, *R.qk_norm(k, wk, pos, freq, pairs, EPS), "k")
    dq, dk, dwq, dwk = run_bwd(dev(dqo), dev(dko), *args, pairs)
    for n, dx, dw, dy, x, w in (("q", dq, dwq, dqo, q, wq), ("k", dk, dwk, dko, k, wk)):
        want, off, want_w, off_w = R.qk_norm_bwd(dy, x, w, pos, freq, pairs, EPS)
        R.check(dx, want, off, "d" + n)
        R.check(dw, want_w, off_w, "dw" + n)


@pytest.mark.parametrize("T", [37, 2050])
def test_columns_of_a_wider_matrix_in_place(T):
    q, k, wq, wk, pos, freq, dqo, dko = inputs(T, 6, 2, 96, 48, seed=1)
    w = [dev(t) for t in (wq, wk, pos, freq)]
    qo, ko = run(dev(q), dev(k), *w, True)
    wide, (qv, kv) = packed_of(q, k)
    B.moe_qk_norm_rope(qv, kv, *w, True, EPS, qv, kv)
    assert torch.equal(qv, qo) and torch.equal(kv, ko)
    assert bool((wide[:, 8 * 96:] == 7.0).all())                             # what lies beside them stays
    # backward, from strided rows, over the gradients and over the inputs
    plain = run_bwd(dev(dqo), dev(dko), dev(q), dev(k), *w, True)
    for over in ("dy", "x"):
        wide, (qv, kv) = packed_of(q, k)
        grads, (dqv, dkv) = packed_of(dqo, dko, extra=8)
        to = (dqv, dkv) if over == "dy" else (qv, kv)
        again = run_bwd(dqv, dkv, qv, kv, *w, True, dq=to[0], dk=to[1])
        for a, b in zip(plain, again):
            assert torch.equal(a, b), over
        assert bool((wide[:, 8 * 96:] == 7.0).all()) and bool((grads[:, 8 * 96:] == 7.0).all())


def test_far_and_negative_positions():
    q, k, wq, wk, _, freq, dqo, dko = inputs(9, 2, 1, 64, 64, seed=2)
    pos = torch.tensor([0, -1, 1, 2 ** 31 - 1, -2 ** 31, 1 << 20, 999983, -4096, 123456789]).int()
    for pairs in (False, True):
        qo, ko = run(*[dev(t) for t in (q, k, wq, wk, pos, freq)], pairs)
        # (2^31 turns in 64 bits are off by 2^31 2^-52: nothing beside the bound)
        R.check(qo, *R.qk_norm(q, wq, pos, freq, pairs, EPS), "q")
        R.check(ko, *R.qk_norm(k, wk, pos, freq, pairs, EPS), "k")


def test_turning_back_and_the_same_bits_again():
    T = 300
    q, k, wq, wk, pos, freq, dqo, dko = inputs(T, 4, 4, 128, 128, seed=3)
    args = [dev(t) for t in (q, k, wq, wk, pos, freq)]
    first = run(*args, False) + run_bwd(dev(dqo), dev(dko), *args, False)
    again = run(*args, False) + run_bwd(dev(dqo), dev(dko), *args, False)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    # a token's rows depend on nothing but the token
    part = run(*[dev(t[10:20]) for t in (q, k)], *args[2:4], dev(pos[10:20]), args[5], False)
    assert torch.equal(part[0], first[0][10:20]) and torch.equal(part[1], first[1][10:20])


def test_rows_of_zeros_and_what_is_not_a_number():
    q, k, wq, wk, pos, freq, dqo, dko = inputs(5, 3, 2, 64, 32, seed=4)
    q[1] = 0
    q[2, 1, 5], k[3, 0, 0] = float("nan"), float("inf")
    args = [dev(t) for t in (q, k, wq, wk, pos, freq)]
    qo, ko = run(*args, False)
    assert bool((qo[1] == 0).all())
    assert bool(torch.isnan(qo[2, 1]).all()) and bool(torch.isnan(ko[3, 0]).any())
    keep_q, keep_k = torch.ones(5, 3, dtype=torch.bool), torch.ones(5, 2, dtype=torch.bool)
    keep_q[2, 1], keep_k[3, 0] = False, False
    assert bool(torch.isfinite(qo[keep_q.to(DEV)]).all()) and bool(torch.isfinite(ko[keep_k.to(DEV)]).all())
    dq, dk, dwq, dwk = run_bwd(dev(dqo), dev(dko), *args, False)
    assert bool(torch.isfinite(dq[keep_q.to(DEV)]).all()) and bool(torch.isfinite(dk[keep_k.to(DEV)]).all())
    assert bool(torch.isnan(dwq).any()) and bool(torch.isnan(dwk).any())


def test_no_epsilon_and_the_largest_numbers():
    """Squares past what 32 bits hold count as infinite; without an epsilon a head of zeros has no norm, and its neighbours are what they are."""
    q, k, wq, wk, pos, freq, dqo, dko = inputs(4, 3, 2, 64, 64, seed=6)
    q[1, 1], k[2, 0] = 0, 0
    q[3, 2] = 3e19
    args = [dev(t) for t in (q, k, wq, wk, pos, freq)]
    qo, ko = run(*args, True, eps=0.0)
    assert bool(torch.isnan(qo[1, 1]).all()) and bool(torch.isnan(ko[2, 0]).all()) and bool((qo[3, 2] == 0).all())
    dq, dk, _, _ = run_bwd(dev(dqo), dev(dko), *args, True, eps=0.0)
    assert bool((dq[3, 2] == 0).all())
    keep_q, keep_k = torch.ones(4, 3, dtype=torch.bool), torch.ones(4, 2, dtype=torch.bool)
    keep_q[1, 1], keep_q[3, 2], keep_k[2, 0] = False, False, False
    alone = [t.clone() for t in (q, k)]
    alone[0][~keep_q], alone[1][~keep_k] = 1, 1
    args[:2] = [dev(t) for t in alone]
    for got, want, keep in zip((qo, ko, dq, dk), (*run(*args, True, eps=0.0), *run_bwd(dev(dqo), dev(dko), *args, True, eps=0.0)[:2]), (keep_q, keep_k) * 2):
        assert bool(torch.isfinite(got[keep.to(DEV)]).all()) and torch.equal(got[keep.to(DEV)], want[keep.to(DEV)])


def test_gradients_against_differences():
    """The 64-bit derivative against differences of the 64-bit result, along random directions."""
    q, _, wq, _, pos, freq, dqo, _ = inputs(6, 3, 1, 32, 16, seed=5)
    g = torch.Generator().manual_seed(6)
    x, w, dy = q.double(), wq.double(), dqo.double()
    dx, _, dw, _ = R.qk_norm_bwd(dy, x, w, pos, freq, True, EPS)
    dir_x, dir_w, h = torch.randn(x.shape, generator=g, dtype=torch.float64), torch.randn(w.shape, generator=g, dtype=torch.float64), 1e-5
    value = lambda s: float((R.qk_norm(x + s * dir_x, w + s * dir_w, pos, freq, True, EPS)[0] * dy).sum())  # noqa: E731
    slope = (value(h) - value(-h)) / (2 * h)
    want = float((dx * dir_x).sum() + (dw * dir_w).sum())
    assert abs(slope - want) < 1e-6 * (abs(want) + float(dy.abs().sum()))


def test_offsets_past_32_bits():
    """Tokens so far apart that the last one begins behind 2^32 bytes and 2^31 elements."""
    T, ld = 5, 1 << 29
    q, k, wq, wk, pos, freq, _, _ = inputs(T, 2, 1, 64, 64, seed=7)
    big = torch.empty(T * ld, dtype=torch.bfloat16, device=DEV).view(T, ld)
    qv, kv = big[:, :128].unflatten(1, (2, 64)), big[:, 128:192].unflatten(1, (1, 64))
    qv.copy_(q)
    kv.copy_(k)
    B.moe_qk_norm_rope(qv, kv, dev(wq), dev(wk), dev(pos), dev(freq), False, EPS, qv, kv)
    R.check(qv, *R.qk_norm(q, wq, pos, freq, False, EPS), "q")
    R.check(kv, *R.qk_norm(k, wk, pos, freq, False, EPS), "k")


def test_more_tokens_than_a_launch_has_workgroups_for():
    """A token's rows are those of the token alone: the last of 2^22 and some are the same in a small call."""
    T, D = (4 << 20) + 37, 8
    g = torch.Generator(device=DEV).manual_seed(9)
    q, k = (torch.randn(T, 1, D, generator=g, device=DEV).bfloat16() for _ in range(2))
    w, pos = torch.rand(D, generator=g, device=DEV), torch.arange(T, dtype=torch.int32, device=DEV)
    # (no rotated columns, so that a large call and a small one differ in nothing but their workgroups)
    qo, ko = run(q, k, w, w, pos, None, False)
    for at in (slice(T - 50, T), slice(0, 50), slice(T // 2, T // 2 + 50)):
        a, b = run(q[at].clone(), k[at].clone(), w, w, pos[at].clone(), None, False)
        assert torch.equal(a, qo[at]) and torch.equal(b, ko[at])
    dq, dk, dwq, dwk = run_bwd(qo, ko, q, k, w, w, pos, None, False)
    da, db, _, _ = run_bwd(qo[-50:].clone(), ko[-50:].clone(), q[-50:].clone(), k[-50:].clone(), w, w, pos[-50:].clone(), None, False)
    assert torch.equal(da, dq[-50:]) and torch.equal(db, dk[-50:])


@pytest.mark.parametrize("T", [50, 2500])
def test_in_a_graph_and_on_another_stream(T):
    q, k, wq, wk, pos, freq, dqo, dko = inputs(T, 4, 2, 128, 128, seed=8)
    args = [dev(t) for t in (q, k, wq, wk, pos, freq)]
    g = [dev(dqo), dev(dko)]
    eager = run(*args, False) + run_bwd(*g, *args, False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = run(*args, False) + run_bwd(*g, *args, False)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, there))
    outs = [new(q), new(k), new(q), new(k), torch.empty(128, device=DEV), torch.empty(128, device=DEV)]
    ws = torch.empty(B.moe_qk_norm_rope_bwd_workspace_bytes(T, 4, 2, 128), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.moe_qk_norm_rope(*args, False, EPS, *outs[:2])
        B.moe_qk_norm_rope_bwd(*g, *args, False, EPS, *outs[2:], ws)
    for shift in (0, 3, 0):                                                   # other positions between the replays
        args[4].copy_(pos + shift)
        for o in outs:
            o.fill_(float("nan"))
        graph.replay()
        want = run(*args, False) + run_bwd(*g, *args, False)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), shift
