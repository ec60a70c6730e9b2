"""Logits of -infinity in the head's scores: columns that are not there."""
import pytest
import torch

import score_reference as R
from test_gpu_head_score import forward, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K,path", [(0, 0), (0, 102)] + [(K, path) for K in (5, 64) for path in (0, 1, 2, 102)])
@pytest.mark.parametrize("T,V", [(3, 200), (300, 200), (2, 3001), (300, 700)])
def test_columns_that_are_not_there(T, V, K, path):
    x, W, target, _, _ = inputs(T, 256, V, masked=0.1, seed=T + V)
    x[:, 3] = 1.0
    W[:, 3] = 0
    gone = torch.arange(V) % 7 == 3
    gone[64:130] = True
    gone[V - 40:] = True
    kept = torch.nonzero(~gone)[:, 0]
    number = torch.cumsum((~gone).int(), 0) - 1
    target = torch.where((target >= 0) & (target < V), kept[target.long() % len(kept)].int(), target)
    want, bound = R.score(x, W[kept], torch.where((target >= 0) & (target < V), number[target.long().clamp(0, V - 1)].int(), torch.tensor(-100, dtype=torch.int32)), K)
    W = W.clone()
    W[gone, 3] = -float("inf")
    got = forward(x, W, target, K, path=path)
    if K:
        want["ids"] = torch.where(want["ids"] >= 0, kept[want["ids"].long().clamp(min=0)].int(), want["ids"])
    R.check_all(got, want, bound)


@pytest.mark.parametrize("path", [1, 2, 102])
def test_fewer_columns_than_alternatives_and_a_target_that_is_not_there(path):
    x, W, target, _, _ = inputs(4, 256, 90, masked=0.0, seed=3)
    x[:, 3], W[:, 3] = 1.0, 0
    W[5:, 3] = -float("inf")
    target[:] = torch.tensor([0, 4, 2, 60])
    got = {n: t.cpu() for n, t in forward(x, W, target, 9, path=path).items()}
    want, bound = R.score(x[:3], W[:5], target[:3], 5)
    for n, w in want.items():
        part = got[n][:3] if w.dim() == 1 else got[n][:3, :5]
        assert torch.equal(part, w) if n == "ids" else True
        if n != "ids":
            R.check(part, w, bound[n], n)
    assert bool((got["ids"][:, 5:] == -1).all()) and bool(torch.isnan(got["top"][:, 5:]).all())
    assert float(got["logp"][3]) == -float("inf") and bool(torch.isfinite(got["entropy"]).all()) and bool(torch.isfinite(got["lse"]).all())
