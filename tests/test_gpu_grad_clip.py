"""The norm of many gradients together and their clipping, against 64 bits: sizes and places of all kinds, ends of the range, in place, in a graph."""
import math

import pytest
import torch

import qk_reference as R
from paper_2604_00785_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def tensors(sizes, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(scale * torch.randn(n, generator=g)).to(t).to(DEV) for n, t in sizes]


def space(n):
    return torch.full((B.moe_grad_norm_workspace_bytes(n),), 255, dtype=torch.uint8, device=DEV)


def norm_of(grads):
    norm = torch.full((1,), float("nan"), device=DEV)
    B.moe_grad_norm(grads, norm, space(len(grads)))
    return norm


def clip(grads, largest, outs="new"):
    norm = torch.full((1,), float("nan"), device=DEV)
    if outs == "new":
        outs = [torch.full_like(g, float("nan")) for g in grads]
    B.moe_grad_clip(grads, largest, norm, outs, space(len(grads)))
    return norm, grads if outs is None else outs


def close(norm, want):
    # summed in 64 bits, rounded once
    assert abs(float(norm) - want) <= want * (R.HALF32 + 1e-12) + 2.0 ** -149, (float(norm), want)


SETS = {
    "one": [(1, BF)], "one32": [(1, F32)], "few": [(7, BF), (3, F32)], "pieces": [(8, BF), (4, F32), (9, BF), (5, F32), (2047, BF), (2048, BF), (2049, BF)],
    "empty among them": [(0, BF), (1000, F32), (0, F32), (77, BF), (0, BF)],
    "chunk borders": [(2048 * 256, BF), (1024 * 256 + 1, F32), (2048 * 255 + 7, BF), (4095, F32)],
    "a table full": [(65 + i, BF if i % 3 else F32) for i in range(120)],
    "a table and one": [(300 + 7 * i, F32 if i % 2 else BF) for i in range(121)],
    "many tables": [(1 + 13 * i % 999, BF if i % 2 else F32) for i in range(700)],
    "large": [(30_000_001, BF), (5, F32), (9_999_999, F32), (12345, BF)],
    "more sums than a workgroup adds up": [(150_001, BF if i % 2 else F32) for i in range(500)],
    "large and many": [(400_003, BF if i % 2 else F32) for i in range(130)],
}


@pytest.mark.parametrize("name", SETS)
def test_against_64_bits(name):
    grads = tensors(SETS[name], seed=len(name))
    host = [g.cpu() for g in grads]
    want = R.grad_norm(host)
    close(norm_of(grads), want)
    for largest in (0.37 * want, 2.0 * want, 1e-3):
        norm, outs = clip(grads, largest)
        close(norm, want)
        _, scaled, bounds = R.grad_clip(host, largest)
        for i, (o, s, b) in enumerate(zip(outs, scaled, bounds)):
            R.check(o, s, b, (name, i))
        if largest > want + 1e-6:
            assert all(torch.equal(o, g) for o, g in zip(outs, grads))
        inplace = [g.clone() for g in grads]
        again, _ = clip(inplace, largest, None)
        assert torch.equal(again, norm) and all(torch.equal(a, b) for a, b in zip(inplace, outs))
    assert all(torch.equal(g.cpu(), h) for g, h in zip(grads, host))


def test_slices_at_any_place():
    """Tensors that begin and end in the middle of 16 bytes, side by side; their neighbours stay."""
    g = torch.Generator().manual_seed(3)
    flat = {t: torch.randn(60_000, generator=g).to(t).to(DEV) for t in (BF, F32)}
    outs = {t: torch.full((60_003,), 7.0, dtype=t, device=DEV) for t in (BF, F32)}
    grads, to, at = [], [], 0
    for i, n in enumerate([1, 2, 3, 5, 8, 13, 21, 1000, 4097, 9999, 16384, 20001]):
        t = BF if i % 2 else F32
        grads.append(flat[t][at:at + n])
        to.append(outs[t][at + 2:at + 2 + n])                                 # not at the same place of 16 bytes as what is read
        at += n
    host = [x.cpu() for x in grads]
    norm, _ = clip(grads, 1.5, to)
    want, scaled, bounds = R.grad_clip(host, 1.5)
    close(norm, want)
    covered = {t: torch.zeros(60_003, dtype=torch.bool) for t in (BF, F32)}
    at = 0
    for i, (o, s, b) in enumerate(zip(to, scaled, bounds)):
        R.check(o, s, b, i)
        covered[BF if i % 2 else F32][at + 2:at + 2 + o.numel()] = True
        at += o.numel()
    for t in (BF, F32):
        assert bool((outs[t].cpu()[~covered[t]] == 7.0).all())


def test_large_slices_at_any_place():
    """The same where a thread takes several pieces: slices of 20 million elements that begin at odd places."""
    g = torch.Generator(device=DEV).manual_seed(4)
    flat = torch.randn(20_000_011, generator=g, device=DEV).to(BF)
    out = torch.full((20_000_020,), 7.0, dtype=BF, device=DEV)
    cuts = [1, 3, 4_000_002, 4_000_003, 11_111_112, 20_000_008]
    grads, to = [flat[a:b] for a, b in zip(cuts, cuts[1:])], [out[a + 5:b + 5] for a, b in zip(cuts, cuts[1:])]
    norm, _ = clip(grads, 0.25, to)
    want = R.grad_norm([flat[1:20_000_008].cpu()])
    close(norm, want)
    scaled = flat[1:20_000_008].double() * (0.25 / (want + 1e-6))
    assert float(((out[6:20_000_013].double() - scaled).abs() - scaled.abs() * (R.HALF16 + 3 * R.HALF32) - R.LEAST16).max()) <= 0
    assert bool((out[:6] == 7.0).all()) and bool((out[20_000_013:] == 7.0).all())


def test_ends_of_the_range():
    # squares that 32 bits do not hold, large and small
    for size in (1e30, 1e-30):
        grads = tensors([(5000, BF), (333, F32)], seed=1, scale=size)
        host = [g.cpu() for g in grads]
        norm, outs = clip(grads, 2e-31)
        want, scaled, bounds = R.grad_clip(host, 2e-31)
        close(norm, want)
        for o, s, b in zip(outs, scaled, bounds):
            R.check(o, s, b, size)
    # a norm that 32 bits do not hold: infinity to the caller, but the scale is right
    grads = [torch.full((100,), 3e38, device=DEV), torch.full((50,), 3e38, device=DEV).to(BF)]
    norm, outs = clip(grads, 1.0)
    assert float(norm) == math.inf
    _, scaled, bounds = R.grad_clip([g.cpu() for g in grads], 1.0)
    for o, s, b in zip(outs, scaled, bounds):
        R.check(o, s, b, "large norm")
    # nothing but zeros; nothing at all
    norm, outs = clip([torch.zeros(100, device=DEV), torch.zeros(9, dtype=BF, device=DEV)], 1.0)
    assert float(norm) == 0.0 and all(bool((o == 0).all()) for o in outs)
    norm, _ = clip([torch.zeros(0, device=DEV)], 1.0)
    assert float(norm) == 0.0
    # infinity: finite gradients become 0; NaN: all become NaN
    grads = [torch.tensor([1.0, math.inf, -2.0], device=DEV), torch.ones(100, dtype=BF, device=DEV)]
    norm, outs = clip(grads, 1.0)
    assert float(norm) == math.inf and outs[0][0] == 0 and outs[0][2] == 0 and bool(torch.isnan(outs[0][1])) and bool((outs[1] == 0).all())
    grads[0][1] = math.nan
    norm, outs = clip(grads, 1.0)
    assert bool(torch.isnan(norm).all()) and all(bool(torch.isnan(o).all()) for o in outs)
    norm, outs = clip(grads, 1.0, None)
    assert all(bool(torch.isnan(o).all()) for o in outs)


def test_nothing_is_written_in_place_below_the_largest_norm():
    odd = torch.tensor([0x7FA0, 0x3F80, 0x0001], dtype=torch.int16).view(BF).to(DEV)      # a NaN with a payload would make the norm NaN: keep it out
    grads = [odd[1:], torch.ones(1000, device=DEV)]
    before = [g.clone() for g in grads]
    clip(grads, 1e9, None)
    assert all(torch.equal(a.view(torch.int16) if a.dtype == BF else a, b.view(torch.int16) if b.dtype == BF else b) for a, b in zip(grads, before))


def test_more_than_32_bits_of_elements():
    n = (1 << 32) + 5
    g = torch.ones(n, dtype=BF, device=DEV)
    g[-1] = 2.0
    norm, _ = clip([g], 65536.0 / 2, None)
    close(norm, math.sqrt(n + 3))
    scale = min(1.0, 32768.0 / (math.sqrt(n + 3) + 1e-6))
    for at, v in ((0, 1.0), (n // 2, 1.0), (n - 2, 1.0), (n - 1, 2.0), (n - 5, 1.0)):
        assert abs(float(g[at]) - v * scale) <= v * scale * 1.01 * R.HALF16, at
    assert int((g[:1 << 30] != g[0]).sum()) == 0 and int((g[-(1 << 30):-1] != g[0]).sum()) == 0


@pytest.mark.parametrize("name", ["few", "a table and one", "large"])
def test_in_a_graph_and_on_another_stream(name):
    grads = tensors(SETS[name], seed=5)
    norm, outs = clip(grads, 0.5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there, others = clip(grads, 0.5)
    side.synchronize()
    assert torch.equal(norm, there) and all(torch.equal(a, b) for a, b in zip(outs, others))
    ws, n, to = space(len(grads)), torch.empty(1, device=DEV), [torch.empty_like(g) for g in grads]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.moe_grad_clip(grads, 0.5, n, to, ws)
        B.moe_grad_norm(to, n, ws)                                            # the same workspace again: what was clipped
    for factor in (1.0, 3.0, 1.0):
        for g in grads:
            g.mul_(factor)
        ws.fill_(255)
        graph.replay()
        _, want = clip(grads, 0.5)
        close(norm_of(want), R.grad_norm([w.cpu() for w in want]))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(to, want)) and torch.equal(n, norm_of(want))
