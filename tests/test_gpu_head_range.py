"""Logits that are not finite: what is not a number is not a loss of nothing."""
import pytest
import torch

import head_reference as R
from test_gpu_head import make, run

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("T", [5, 40, 300])              # all tokens are rows; the same with more than one block; rows found first (with a teacher)
@pytest.mark.parametrize("K,tau", [(0, 1.0), (6, 1.0), (6, 1.5), (300, 1.0), (300, 1.5)])
@pytest.mark.parametrize("value", [NAN, INF, -INF])
def test_a_token_that_is_not_finite(T, K, tau, value):
    """One number of a token's x makes its logits NaN or infinite, of either sign: its losses and gradient are NaN, as is dW, and the other tokens' are what they were."""
    a = make(T, 64, 400, K, seed=31)
    clean = run(a, tau)
    t = 3 if T < 20 else T - 2
    a["x"][t, 17] = value
    got = run(a, tau)
    for k in clean:
        if k == "dW":
            assert bool(torch.isnan(got[k]).any(1).all())
            continue
        one = torch.arange(T, device=got[k].device) == t
        assert bool(torch.isnan(got[k][one]).all()), (k, got[k][one])
        assert torch.equal(got[k][~one], clean[k][~one]), k


@pytest.mark.parametrize("T", [5, 300])
@pytest.mark.parametrize("K,row", [(0, "target"), (0, "other"), (6, "target"), (6, "entry"), (6, "other")])
@pytest.mark.parametrize("value", [NAN, INF])
def test_a_column_that_is_not_finite(T, K, row, value):
    """A row of W that makes one logit of every token NaN or +infinity: the target's, an entry's or one that does not count by itself."""
    a = make(T, 64, 400, K, seed=32)
    a["x"][:, 5] = 1.0                                   # (an infinity of its own sign)
    v = {"target": 7, "entry": 8, "other": 9}[row]
    a["target"][:] = 7
    if K:
        a["ids"] = torch.where((a["ids"] >= 7) & (a["ids"] < 10), 0 * a["ids"] - 1, a["ids"])
        a["ids"][:, 0] = 8
    a["W"][v, 5] = value
    got = run(a, 1.5, train=False)
    for k, x in got.items():
        assert bool(torch.isnan(x).all()), (k, x)


def test_nothing_but_the_target_and_entries():
    """Every column is an item, so that no sum over the others is there to carry a NaN."""
    a = make(3, 64, 4, 3, seed=33)
    a["target"][:] = torch.tensor([3, 3, 0])
    a["ids"] = torch.tensor([[0, 1, 2], [0, 1, 2], [1, 2, 3]]).int()
    a["x"][0, 0] = NAN
    a["x"][1, 0] = INF
    got = run(a, 1.5, train=False)
    for k, x in got.items():
        assert bool(torch.isnan(x[:2]).all()) and bool(torch.isfinite(x[2])), (k, x)
    one = make(2, 64, 1, 0, seed=34)
    one["x"][0, 0] = NAN
    got = run(one, train=False)
    assert bool(torch.isnan(got["loss"][0])) and float(got["loss"][1]) == 0.0


@pytest.mark.parametrize("T,K", [(5, 0), (40, 0), (300, 0), (40, 6)])
def test_logits_past_the_range(T, K):
    """Losses are right for logits up to 2^29 of either sign, and NaN from 2^30 on: never a number that says nothing."""
    a = make(T, 64, 400, K, seed=35)
    x = a["x"].float()
    high = float((x @ a["W"].float().t()).abs().max())
    for bits in (20, 27, 29):
        a["x"] = (x * (0.95 * 2.0 ** bits / high)).bfloat16()
        got = run(a, train=False)
        want, bound = R.head(a["x"], a["W"], a["target"], a.get("ids"), a.get("teacher"))
        # (that loss, log(1 + sum exp), is made for those near zero and overflows from 709 on; the difference does not, and has 64 bits enough here)
        z = a["x"].to(R.F64) @ a["W"].to(R.F64).t()
        want["loss"] = torch.logsumexp(z, 1) - z.gather(1, a["target"][:, None].long())[:, 0]
        for k in got:
            R.check(got[k], want[k], bound[k], k)
    # all columns nearly alike: each token's logits are nearly one number, of either sign
    g = torch.Generator().manual_seed(1)
    w = torch.randn(64, generator=g)
    a["W"] = (w + 0.01 * torch.randn(400, 64, generator=g)).bfloat16()
    sign = torch.where(torch.arange(T)[:, None] % 2 == 0, 1.0, -1.0)
    for bits in (30, 31, 33, 40, 100):
        a["x"] = (sign * w * (1.1 * 2.0 ** bits / float(w.square().sum()))).bfloat16()
        assert float((a["x"].float() @ a["W"].float().t()).abs().amin()) > 2.0 ** bits
        for k, v in run(a, train=False).items():
            assert bool(torch.isnan(v).all()), (bits, k)


@pytest.mark.parametrize("T", [5, 40, 300])
def test_temperatures_past_the_range(T):
    """The same with the logits over the temperature: the divergence alone is lost."""
    a = make(T, 64, 400, 6, seed=36)
    clean = run(a, train=False)
    got = run(a, 1e-12, train=False)
    assert torch.equal(got["loss"], clean["loss"]) and torch.equal(got["lse"], clean["lse"])
    assert bool(torch.isnan(got["kd"]).all()) and bool(torch.isnan(got["lse_t"]).all())


@pytest.mark.parametrize("T,K", [(60, 0), (60, 7), (200, 7), (500, 0), (500, 7), (4500, 0)])
def test_what_stands_in_masked_places_leaves_no_trace(T, K):
    """NaN, infinities and huge numbers wherever a token without a loss or an entry that does not count has one: the same bits as with ordinary numbers there."""
    a = make(T, 64, 300, K, masked=0.4, seed=37)
    out = a["target"] < 0
    clean = run(a, 1.5)
    for value in (NAN, INF, 3e38):
        b = dict(a)
        b["x"], b["dloss"] = a["x"].clone(), a["dloss"].clone()
        b["x"][out], b["dloss"][out] = value, value
        if K:
            b["dkd"], b["teacher"] = a["dkd"].clone(), a["teacher"].clone()
            b["dkd"][out] = value
            b["teacher"][a["ids"] < 0] = value
        for k, v in run(b, 1.5).items():
            assert torch.equal(v, clean[k]), (value, k)
