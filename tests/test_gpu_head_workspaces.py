"""Workspaces: one for the largest batch serves smaller ones, and whatever a call accepts it keeps to."""
import pytest
import torch

import score_reference as R
from paper_2604_00785_amd import binding as B
from test_gpu_head_score import DEV, inputs, junk

pytestmark = pytest.mark.gpu
GUARD = 1 << 16


class Calls:
    """Both calls of one shape, on the first n bytes of a workspace; what lies behind them has to stay."""

    def __init__(self, T, d, V, K, most):
        self.host = inputs(T, d, V, seed=T + V)
        self.x, self.W, self.y, self.dl, self.de = (t.to(DEV) for t in self.host)
        self.T, self.d, self.V, self.K = T, d, V, K
        self.want, self.bound = R.score(*self.host[:3], K, 1.0, *self.host[3:])
        self.ws = torch.full((most + GUARD,), 255, dtype=torch.uint8, device=DEV)

    def run(self, n, bwd, f=None):
        T, d, V, K = self.T, self.d, self.V, self.K
        self.ws.fill_(255)
        if not bwd:
            f = {"logp": junk(T), "entropy": junk(T), "lse": junk(T)}
            if K:
                f.update(ids=junk(T, K, dtype=torch.int32), top=junk(T, K))
            B.moe_head_score_fwd(self.x, self.W, self.y, 1.0, f["logp"], f["entropy"], f["lse"], f.get("ids"), f.get("top"), self.ws[:n])
            out = f
        else:
            out = {"dx": junk(T, d, dtype=torch.bfloat16), "dW": junk(V, d, dtype=torch.bfloat16)}
            B.moe_head_score_bwd(self.x, self.W, self.y, 1.0, f["logp"], f["entropy"], f["lse"], self.dl, self.de, 0, out["dx"], out["dW"], self.ws[:n])
        assert bool((self.ws[n:] == 255).all())
        R.check_all(out, {k: self.want[k] for k in out}, self.bound)
        return out


@pytest.mark.parametrize("d,V,K,most,fewer", [(2048, 5000, 0, 513, [1, 16, 160, 200, 512]), (512, 16000, 20, 200, [1, 96, 128, 129]), (512, 1031, 0, 1024, [4, 6, 200, 256, 700]),
                                              (512, 1031, 7, 700, [5, 129, 513]), (64, 12000, 64, 700, [40, 129, 300]), (4096, 256, 3, 300, [1, 17, 257])])
def test_the_largest_batch_serves_smaller_ones(d, V, K, most, fewer):
    fwd, bwd = B.moe_head_score_fwd_workspace_bytes(most, d, V, K), B.moe_head_score_bwd_workspace_bytes(most, d, V)
    for T in (*fewer, most):
        c = Calls(T, d, V, K, max(fwd, bwd))
        c.run(bwd, True, c.run(fwd, False))


@pytest.mark.parametrize("T,d,V,K", [(16, 2048, 5000, 20), (160, 2048, 5000, 0), (96, 512, 16000, 20), (200, 512, 1031, 0), (256, 2048, 1031, 3), (700, 64, 515, 2)])
def test_less_and_less_room_until_it_is_refused(T, d, V, K):
    fwd, bwd = B.moe_head_score_fwd_workspace_bytes(T, d, V, K), B.moe_head_score_bwd_workspace_bytes(T, d, V)
    c = Calls(T, d, V, K, max(fwd, bwd))
    f = None
    for size, back in ((fwd, False), (bwd, True)):
        n, ran = size, 0
        while n > 0:
            try:
                out = c.run(n // 16 * 16, back, f)
            except B.MoeError as e:
                assert "WORKSPACE" in str(e)
                break
            ran, n = ran + 1, int(n * 0.8)
        assert ran > 0 and n > 0
        f = f or out
    torch.cuda.synchronize()


@pytest.mark.parametrize("most,fewer", [(257, [16, 160, 200]), (2048, [64, 256, 513])])
def test_cross_entropy(most, fewer):
    d, V = 2048, 5000
    ws = torch.full((B.moe_head_bwd_workspace_bytes(most, d, V) + GUARD,), 255, dtype=torch.uint8, device=DEV)
    n = ws.numel() - GUARD
    for T in fewer:
        x, W, y, dl, _ = (t.to(DEV) for t in inputs(T, d, V, seed=T))
        h = B.HeadBuffers(T, d, V)
        h.run_fwd(x, W, y)
        h.run_bwd(x, W, y, dl)
        dx, dW = junk(T, d, dtype=torch.bfloat16), junk(V, d, dtype=torch.bfloat16)
        B.moe_head_ce_bwd(x, W, y, h.loss, h.lse, dl, 0, dx, dW, ws[:n])
        assert bool((ws[n:] == 255).all())
        # the same sums, perhaps in another order: what differs is rounded the other way
        for a, b in ((dx, h.dx), (dW, h.dW)):
            assert float((a.double() - b.double()).norm() / b.double().norm()) < R.HALF16 / 8


@pytest.mark.parametrize("T,d,V", [(500, 2048, 1031), (256, 1024, 8000), (500, 2048, 3000), (16, 4096, 5000), (200, 704, 5001)])
def test_a_call_takes_the_same_way_in_its_own_size_as_in_more(T, d, V):
    """The same bits: its size is all that its rule wants."""
    fwd, bwd = B.moe_head_score_fwd_workspace_bytes(T, d, V, 3), B.moe_head_score_bwd_workspace_bytes(T, d, V)
    more = 2 * max(fwd, bwd) + (1 << 28)
    c = Calls(T, d, V, 3, more)
    f, g = c.run(fwd, False), c.run(more, False)
    assert all(torch.equal(f[n], g[n]) for n in f)
    a, b = c.run(bwd, True, f), c.run(more, True, f)
    assert all(torch.equal(a[n], b[n]) for n in a)
    h = B.HeadBuffers(T, d, V)
    h.run_fwd(c.x, c.W, c.y)
    for n in (B.moe_head_bwd_workspace_bytes(T, d, V), more):
        dx, dW = junk(T, d, dtype=torch.bfloat16), junk(V, d, dtype=torch.bfloat16)
        B.moe_head_ce_bwd(c.x, c.W, c.y, h.loss, h.lse, c.dl, 0, dx, dW, c.ws[:n])
        a = (dx, dW) if n < more else a
    assert torch.equal(a[0], dx) and torch.equal(a[1], dW)
