"""moe_add_rms_norm, its form in 8 bits and its derivative against 64 bits."""
import pytest
import torch

import head_reference as R
from paper_2604_00785_amd import binding as B

pytestmark = pytest.mark.gpu
DEV, EPS = "cuda:0", 1e-5
BF = torch.bfloat16


def make(T, d, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed * 1000003 + T * 131 + d)
    n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    return {"x": (scale * n(T, d)).bfloat16(), "r": (2 * scale * n(T, d) * torch.exp(n(d))).bfloat16(), "w": 0.5 + torch.rand(d, generator=g),
            "dy": n(T, d).bfloat16(), "dsum": n(T, d).bfloat16()}


def dev(t):
    return None if t is None else t.to(DEV)


SIZES = [(1, 8), (1, 2048), (3, 64), (5, 520), (2, 2056), (7, 1024), (130, 1536), (33, 4104), (9, 8192), (4, 8200), (2, 32768), (2051, 136)]


@pytest.mark.parametrize("T,d", SIZES)
@pytest.mark.parametrize("residual", [True, False])
def test_forward(T, d, residual):
    print("add_rms_norm", T, d, residual, flush=True)
    a = make(T, d)
    r = a["r"] if residual else None
    want_sum, want, q = R.norm(a["x"], r, a["w"], EPS)
    total = torch.full((T, d), 7.0, dtype=BF, device=DEV) if residual else None
    y, rstd = torch.full((T + 1, d), 7.0, dtype=BF, device=DEV), torch.full((T,), 7.0, device=DEV)
    B.moe_add_rms_norm(dev(a["x"]), dev(r), dev(a["w"]), EPS, total, y[:T], rstd)
    if residual:
        assert torch.equal(total.cpu(), want_sum)
    R.check(y[:T], want, (R.HALF16 + (d + 16) * R.HALF32) * want.abs(), "y")
    R.check(rstd, q, (d + 16) * R.HALF32 * q, "rstd")
    assert bool((y[T] == 7).all())                       # nothing behind the last row


@pytest.mark.parametrize("T,d,group", [(1, 64, 0), (1, 2048, 128), (3, 64, 8), (5, 512, 512), (130, 1536, 64), (17, 4096, 32), (3, 8192, 128), (3, 2056, 0),
                                       (2, 8200, 0), (65, 1024, 16), (2, 16384, 256), (4, 12, 0)])
def test_8bit(T, d, group):
    print("add_rms_norm_8bit", T, d, group, flush=True)
    if d % 8:
        with pytest.raises(B.MoeError):
            z = torch.zeros(T, d, dtype=BF, device=DEV)
            B.moe_add_rms_norm_8bit(z, z, torch.zeros(d, device=DEV), EPS, 0, z, z.to(torch.float8_e4m3fn), torch.zeros(T, 1, device=DEV))
        return
    a = make(T, d, 1)
    a["x"][0, :] = 0                                     # a row of zeros in all groups, and one with a single value
    a["r"][0, :] = 0
    if T > 1:
        a["x"][1, 1:] = 0
        a["r"][1, :] = 0
    want_sum, y, _ = R.norm(a["x"], a["r"], a["w"], EPS)
    n = d // (group or d)
    total, codes = torch.empty(T, d, dtype=BF, device=DEV), torch.empty(T, d, dtype=torch.float8_e4m3fn, device=DEV)
    scale = torch.full((T, n), 7.0, device=DEV)
    B.moe_add_rms_norm_8bit(dev(a["x"]), dev(a["r"]), dev(a["w"]), EPS, group, total, codes, scale)
    assert torch.equal(total.cpu(), want_sum)
    rel = (d + 16) * R.HALF32
    want_scale = y.view(T, n, -1).abs().amax(2) / 448.0
    R.check(scale, want_scale, rel * want_scale, "scale")
    got = codes.float().cpu().to(R.F64).view(T, n, -1) * scale.cpu().to(R.F64)[:, :, None]
    # half a step of e4m3, 2^-10 of the scale below its smallest normal number (2^-6)
    bound = (R.HALF8 + 4 * rel) * y.view(T, n, -1).abs() + (2.0 ** -10 + rel) * want_scale[:, :, None]
    R.check(got, y.view(T, n, -1), bound, "codes")
    assert bool((codes[0].float() == 0).all()) and bool((scale[0] == 0).all())
    if T > 1:
        assert bool((codes.float().abs().cpu().view(T, n, -1)[2:].amax(2) == 448).all())   # the largest of a group is the type's


@pytest.mark.parametrize("T,d", SIZES + [(4100, 256), (2049, 2048)])
@pytest.mark.parametrize("with_dsum", [True, False])
def test_backward(T, d, with_dsum):
    print("add_rms_norm_bwd", T, d, with_dsum, flush=True)
    a = make(T, d, 2)
    total, y, rstd = torch.empty(T, d, dtype=BF, device=DEV), torch.empty(T, d, dtype=BF, device=DEV), torch.empty(T, device=DEV)
    w = dev(a["w"])
    B.moe_add_rms_norm(dev(a["x"]), dev(a["r"]), w, EPS, total, y, rstd)
    dx, dw = torch.empty(T, d, dtype=BF, device=DEV), torch.full((d,), 7.0, device=DEV)
    ws = torch.empty(B.moe_add_rms_norm_bwd_workspace_bytes(T, d), dtype=torch.uint8, device=DEV)
    dsum = a["dsum"] if with_dsum else None
    B.moe_add_rms_norm_bwd(dev(a["dy"]), dev(dsum), total, w, rstd, dx, dw, ws)
    wx, ww, bx, bw = R.norm_bwd(a["dy"], dsum, total.cpu(), a["w"], EPS)
    R.check(dx, wx, bx, "dx")
    R.check(dw, ww, bw, "dw")
    # the same bits again, and with dx in the place of dy
    dy, dw2 = dev(a["dy"]), torch.empty_like(dw)
    B.moe_add_rms_norm_bwd(dy, dev(dsum), total, w, rstd, dy, dw2, ws)
    assert torch.equal(dy, dx) and torch.equal(dw2, dw)


def test_gradient_is_the_difference_of_forward_passes():
    T, d, h = 3, 256, 2.0 ** -6
    a = make(T, d, 3)
    x = a["x"].to(R.F64)
    zero = torch.zeros(T, d, dtype=BF)
    total, y, rstd = torch.empty(T, d, dtype=BF, device=DEV), torch.empty(T, d, dtype=BF, device=DEV), torch.empty(T, device=DEV)
    w = dev(a["w"])
    B.moe_add_rms_norm(dev(a["x"]), dev(zero), w, EPS, total, y, rstd)
    dx, dw = torch.empty(T, d, dtype=BF, device=DEV), torch.empty(d, device=DEV)
    ws = torch.empty(B.moe_add_rms_norm_bwd_workspace_bytes(T, d), dtype=torch.uint8, device=DEV)
    B.moe_add_rms_norm_bwd(dev(a["dy"]), None, total, w, rstd, dx, dw, ws)

    def f(v):
        q = 1.0 / (v.square().mean(1, keepdim=True) + EPS).sqrt()
        return float((v * q * a["w"].to(R.F64) * a["dy"].to(R.F64)).sum())
    for i in range(0, d, 17):
        e = torch.zeros(T, d, dtype=R.F64)
        e[1, i] = h
        slope = (f(x + e) - f(x - e)) / (2 * h)
        assert abs(slope - float(dx[1, i])) <= R.HALF16 * abs(slope) + 1e-3 * h     # h^2 times a third derivative of order one


def test_sum_in_place_and_other_stream():
    a = make(40, 1024, 4)
    want_sum, want, _ = R.norm(a["x"], a["r"], a["w"], EPS)
    x, r, w = dev(a["x"]), dev(a["r"]), dev(a["w"])
    y = torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.moe_add_rms_norm(x, r, w, EPS, r, y)           # the residual stream is updated where it lies
    side.synchronize()
    assert torch.equal(r.cpu(), want_sum)
    R.check(y, want, (R.HALF16 + 1040 * R.HALF32) * want.abs(), "y")


def test_values_that_are_not_finite():
    """A NaN or infinity stays in its row."""
    a = make(4, 512, 5)
    a["x"][1, 3] = float("nan")
    a["x"][2, 5] = float("inf")
    total, y = torch.empty(4, 512, dtype=BF, device=DEV), torch.empty(4, 512, dtype=BF, device=DEV)
    B.moe_add_rms_norm(dev(a["x"]), dev(a["r"]), dev(a["w"]), EPS, total, y)
    assert bool(torch.isnan(y[1]).all()) and bool(torch.isnan(y[2, 5])) and bool((torch.cat([y[2, :5], y[2, 6:]]) == 0).all())
    assert bool(torch.isfinite(y[0]).all()) and bool(torch.isfinite(y[3]).all())
    codes, scale = torch.empty(4, 512, dtype=torch.float8_e4m3fn, device=DEV), torch.empty(4, 4, device=DEV)
    B.moe_add_rms_norm_8bit(dev(a["x"]), dev(a["r"]), dev(a["w"]), EPS, 128, total, codes, scale)
    assert bool(torch.isnan(scale[1]).all()) and bool(torch.isnan(codes[1].float()).all()) and bool(torch.isfinite(scale[0]).all())


@pytest.mark.parametrize("d,group", [(1024, 64), (512, 0), (4096, 128)])
def test_codes_are_those_of_64_bits(d, group):
    """Every code is the nearest to the quotient in 64 bits, borders included but for the last bit of a 32-bit number."""
    T = 500
    a = make(T, d, 6)
    _, y, _ = R.norm(a["x"], a["r"], a["w"], EPS)
    total, codes = torch.empty(T, d, dtype=BF, device=DEV), torch.empty(T, d, dtype=torch.float8_e4m3fn, device=DEV)
    scale = torch.empty(T, d // (group or d), device=DEV)
    B.moe_add_rms_norm_8bit(dev(a["x"]), dev(a["r"]), dev(a["w"]), EPS, group, total, codes, scale)
    q = y.view(T, d // (group or d), -1)
    q = (q / (q.abs().amax(2, keepdim=True) / 448.0)).view(T, d)
    got = codes.float().cpu().to(R.F64)
    # the codes of the quotient one 32-bit rounding to either side
    low, high = ((q * (1 + sign * 2 * R.HALF32)).float().to(torch.float8_e4m3fn).to(R.F64) for sign in (-1, 1))
    assert bool(((got == low) | (got == high)).all())
