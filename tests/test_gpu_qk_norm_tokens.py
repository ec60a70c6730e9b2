"""Gradients of the norms' weights over many tokens, to what the depth of the kernel's additions can lose: a token or a share that is left out is past it."""
import pytest
import torch

import qk_reference as R
from test_gpu_qk_norm import EPS, dev, inputs, run, run_bwd

pytestmark = pytest.mark.gpu
F64 = torch.float64


def weights_gradient(dy, x, pos, freq, pairs, T, H):
    """(dw, bound, the last token's share of dw).

    A summand is off by 44 halves of a step of its size, as in qk_reference.  A thread adds a chain of its own, then the groups of a workgroup are added up, then the
    workgroups' shares (512 at most) by 32 threads, then theirs."""
    x, dy = x.to(F64), dy.to(F64)
    D = x.shape[2]
    r = 1.0 / (x.square().mean(2, keepdim=True) + EPS).sqrt()
    dv, size = R.turn(dy, pos, freq, pairs, back=True)
    terms, tall = dv * x * r, size * x.abs() * r
    groups = 256 // (4 if D <= 64 else 8 if D <= 128 else 16 if D <= 256 else 32)
    tokens = 4 if T >= 2048 else 1
    blocks = -(-T // tokens)
    depth = -(-blocks // 512) * -(-H // (groups // tokens)) + groups + 16 + 32
    return terms.sum((0, 1)), (44 * tall + depth * terms.abs()).sum((0, 1)) * R.HALF32 + 1e-38, terms[-1].sum(0)


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("T,Hq,Hk,D,Rot", [(4098, 9, 4, 16, 16), (2049, 3, 1, 64, 32), (6001, 4, 2, 128, 128), (3000, 2, 2, 256, 64), (515, 5, 1, 96, 32), (2047, 8, 8, 64, 64)])
def test_many_tokens(T, Hq, Hk, D, Rot, pairs):
    q, k, wq, wk, pos, freq, dqo, dko = inputs(T, Hq, Hk, D, Rot, seed=T)
    dq, dk, dwq, dwk = run_bwd(dev(dqo), dev(dko), *[dev(t) for t in (q, k, wq, wk, pos, freq)], pairs)
    for dy, x, got, H, what in ((dqo, q, dwq, Hq, "dwq"), (dko, k, dwk, Hk, "dwk")):
        want, bound, last = weights_gradient(dy, x, pos, freq, pairs, T, H)
        R.check(got, want, bound, what)
        assert float((last.abs() / bound).max()) > 4, what


def test_no_epsilon_and_small_numbers():
    """Without an epsilon a head has to have a mean square of 2^-126: values of 1e-17 have all their digits."""
    q, k, wq, wk, pos, freq, dqo, dko = inputs(5, 3, 2, 64, 32, seed=7)
    q, k = (q.float() * 1e-17).bfloat16(), (k.float() * 1e-18).bfloat16()
    args = [dev(t) for t in (q, k, wq, wk, pos, freq)]
    qo, ko = run(*args, False, eps=0.0)
    dq, dk, _, _ = run_bwd(dev(dqo), dev(dko), *args, False, eps=0.0)
    for y, dx, x, w, dy, n in ((qo, dq, q, wq, dqo, "q"), (ko, dk, k, wk, dko, "k")):
        R.check(y, *R.qk_norm(x, w, pos, freq, False, 0.0), n)
        want, bound, _, _ = R.qk_norm_bwd(dy, x, w, pos, freq, False, 0.0)
        R.check(dx, want, bound, "d" + n)
