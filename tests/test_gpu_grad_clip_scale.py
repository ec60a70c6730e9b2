"""Clipping next to a scale of 1 and far below the 1e-6 of its formula: out = g min(1, largest / (norm + 1e-6)) whatever the norm is."""
import pytest
import torch

import qk_reference as R
from test_gpu_grad_clip import BF, DEV, F32, clip, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("norm,largest,written", [(1.0, 1.0, True), (1.0, 1.0 + 0.9e-6, True), (1.0, 1.0 + 1.1e-6, False), (1e-7, 5e-7, True), (1e-7, 1.2e-6, False), (2.0 ** -20, 2.0 ** -20, True)])
def test_the_formula_next_to_its_border(norm, largest, written, inplace):
    n = 6000
    grads = [torch.zeros(n, device=DEV), torch.zeros(77, dtype=BF, device=DEV)]
    grads[0][[5, 4096, n - 1]] = norm * torch.tensor([0.5, -0.5, 0.5], device=DEV)
    grads[1][76] = norm * 0.5
    host = [g.cpu() for g in grads]
    want, scaled, bounds = R.grad_clip(host, largest)
    assert (largest < want + 1e-6) == written
    got, outs = clip(grads, largest, None if inplace else "new")
    close(got, want)
    for o, s, b, t in zip(outs, scaled, bounds, (F32, BF)):
        assert o.dtype == t
        R.check(o, s, b, (norm, largest))
    # (a difference that 32 bits tell from 1)
    assert torch.equal(outs[0].cpu(), host[0]) == (not written)
