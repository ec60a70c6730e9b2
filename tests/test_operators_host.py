"""What the norm and the vocabulary head refuse before anything reaches a device, and the sizes of their workspaces."""
import ctypes

import pytest
import torch

from paper_2604_00785_amd import binding as B

INVALID, WORKSPACE = -1, -2
P, Q = ctypes.c_void_p(4096), ctypes.c_void_p(4104)      # never followed: a call that is refused reads nothing
N = None


def test_norm_refusals():
    lib = B.load()
    ok = [P, P, P, 4, 64, 1e-5, P, P, P, N]
    bad = [(0, N), (2, N), (6, N), (7, N), (0, Q), (1, Q), (2, Q), (6, Q), (7, Q), (8, Q), (3, 0), (3, -1), (4, 0), (4, 60), (4, 32776), (5, -1.0),
           (5, float("nan"))]
    for at, value in bad:
        args = list(ok)
        args[at] = value
        assert lib.moe_add_rms_norm(*args) == INVALID, (at, value)
    ok = [P, P, P, 4, 512, 1e-5, 64, P, P, P, N, N]
    for at, value in [(0, N), (8, N), (9, N), (8, Q), (9, Q), (10, Q), (4, 60), (6, -1), (6, 4), (6, 48), (6, 1024), (6, 7)]:
        args = list(ok)
        args[at] = value
        assert lib.moe_add_rms_norm_8bit(*args) == INVALID, (at, value)
    assert lib.moe_add_rms_norm_8bit(P, P, P, 4, 96, 1e-5, 64, P, P, P, N, N) == INVALID       # 64 does not divide 96


def test_norm_backward_refusals():
    lib = B.load()
    n = B.moe_add_rms_norm_bwd_workspace_bytes(4, 64)
    ok = [P, P, P, P, P, 4, 64, P, P, P, n, N]
    for at in (0, 2, 3, 4, 7, 8, 9):
        for value in (N, Q):
            args = list(ok)
            args[at] = value
            assert lib.moe_add_rms_norm_bwd(*args) == INVALID, at
    assert lib.moe_add_rms_norm_bwd(*ok[:10], n - 1, N) == WORKSPACE
    assert B.moe_add_rms_norm_bwd_workspace_bytes(0, 64) == 0 and B.moe_add_rms_norm_bwd_workspace_bytes(4, 63) == 0
    assert B.moe_add_rms_norm_bwd_workspace_bytes(1 << 20, 64) == 512 * 64 * 4                 # shares do not grow with the rows


DIMS = [("T", 0), ("T", -5), ("d", 0), ("d", 32), ("d", 100), ("V", 0), ("V", (1 << 20) + 1)]


@pytest.mark.parametrize("name,value", DIMS + [("K", 0), ("K", 1025)])
def test_head_refuses_sizes(name, value):
    lib = B.load()
    s = dict(T=4, d=64, V=100, K=3)
    s[name] = value
    T, d, V, K = (s[k] for k in "TdVK")
    big = 1 << 40
    if name != "K":
        assert lib.moe_head_ce_fwd(P, P, P, T, d, V, P, P, P, big, N) == INVALID
        assert lib.moe_head_ce_bwd(P, P, P, P, P, P, T, d, V, 0, P, P, P, big, N) == INVALID
        assert B.moe_head_fwd_workspace_bytes(T, d, V) == 0 and B.moe_head_bwd_workspace_bytes(T, d, V) == 0
    assert lib.moe_head_distill_fwd(P, P, P, P, P, 1.0, T, d, V, K, P, P, P, P, P, big, N) == INVALID
    assert lib.moe_head_distill_bwd(P, P, P, P, P, 1.0, P, P, P, P, P, T, d, V, K, 0, P, P, P, big, N) == INVALID


def test_head_refuses_pointers_pieces_and_temperatures():
    lib = B.load()
    big = 1 << 40
    fwd, bwd = [P, P, P, 4, 64, 100, P, P, P, big, N], [P, P, P, P, P, P, 4, 64, 100, 0, P, P, P, big, N]
    dfwd, dbwd = [P] * 5 + [1.0, 4, 64, 100, 3, P, P, P, P, P, big, N], [P] * 5 + [1.0] + [P] * 5 + [4, 64, 100, 3, 0, P, P, P, big, N]
    for fn, ok in (("moe_head_ce_fwd", fwd), ("moe_head_ce_bwd", bwd), ("moe_head_distill_fwd", dfwd), ("moe_head_distill_bwd", dbwd)):
        for at, x in enumerate(ok[:-1]):
            if x is P:
                for value in (N, Q):
                    args = list(ok)
                    args[at] = value
                    assert getattr(lib, fn)(*args) == INVALID, (fn, at)
        args = list(ok)
        args[-2] = 100
        assert getattr(lib, fn)(*args) == WORKSPACE, fn
    for piece in (-256, 1, 64, 300):
        assert lib.moe_head_ce_bwd(*bwd[:9], piece, *bwd[10:]) == INVALID
        assert lib.moe_head_distill_bwd(*dbwd[:15], piece, *dbwd[16:]) == INVALID
        assert B.moe_head_bwd_workspace_bytes(4, 64, 100, 0, piece) == 0
    for tau in (0.0, -1.0, float("inf"), float("nan")):
        assert lib.moe_head_distill_fwd(*dfwd[:5], tau, *dfwd[6:]) == INVALID
        assert lib.moe_head_distill_bwd(*dbwd[:5], tau, *dbwd[6:]) == INVALID


def test_head_workspaces():
    T, d, V = 8192, 2048, 50304
    assert B.moe_head_fwd_workspace_bytes(T, d, V) < T * V                                     # far from the logits (2 bytes each)
    whole, piece = B.moe_head_bwd_workspace_bytes(T, d, V), B.moe_head_bwd_workspace_bytes(T, d, V, 0, 4096)
    assert whole - piece >= T * (V - 4096) * 2 - 64 * T * d * 4                                # the gradient of a piece only
    assert B.moe_head_bwd_workspace_bytes(T, d, V, 64) > whole
    assert B.moe_head_bwd_workspace_bytes(1 << 20, 64, 1 << 20) < 1 << 35                      # 2 GiB of pieces, not 2 TiB


def test_binding_refuses_types_shapes_and_host_tensors():
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    f32, i32 = lambda *s: torch.zeros(*s), lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    codes = torch.zeros(4, 64, dtype=torch.float8_e4m3fn)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    x, W = bf(4, 64), bf(100, 64)
    calls = [
        lambda: B.moe_add_rms_norm(x, x, f32(64), 1e-5, x, x),                                 # on the host
        lambda: B.moe_add_rms_norm(f32(4, 64), x, f32(64), 1e-5, x, x),
        lambda: B.moe_add_rms_norm(x, bf(4, 32), f32(64), 1e-5, x, x),
        lambda: B.moe_add_rms_norm(x, x, bf(64), 1e-5, x, x),
        lambda: B.moe_add_rms_norm(x, x, f32(64), 1e-5, x, x, f32(5)),
        lambda: B.moe_add_rms_norm_8bit(x, x, f32(64), 1e-5, 32, x, codes, f32(4, 1)),
        lambda: B.moe_add_rms_norm_8bit(x, x, f32(64), 1e-5, 48, x, codes, f32(4, 1)),
        lambda: B.moe_add_rms_norm_8bit(x, x, f32(64), 1e-5, 32, x, codes.view(torch.uint8), f32(4, 2)),
        lambda: B.moe_add_rms_norm_bwd(x, x, x, f32(64), f32(3), x, f32(64), ws),
        lambda: B.moe_head_ce_fwd(x, W, i32(4), f32(4), f32(4), ws),                           # on the host
        lambda: B.moe_head_ce_fwd(x, bf(100, 32), i32(4), f32(4), f32(4), ws),
        lambda: B.moe_head_ce_fwd(x, W, i32(4).long(), f32(4), f32(4), ws),
        lambda: B.moe_head_ce_bwd(x, W, i32(4), f32(4), f32(4), f32(4), 0, x, bf(99, 64), ws),
        lambda: B.moe_head_distill_fwd(x, W, i32(4), i32(4, 3), f32(4, 2), 1.0, f32(4), f32(4), f32(4), f32(4), ws),
        lambda: B.moe_head_distill_fwd(x, W, i32(4), i32(3, 3), f32(3, 3), 1.0, f32(4), f32(4), f32(4), f32(4), ws),
        lambda: B.moe_head_distill_bwd(x, W, i32(4), i32(4, 3), f32(4, 3), 1.0, f32(4), f32(4), f32(4), f32(4), f32(3), 0, x, W, ws),
    ]
    for n, call in enumerate(calls):
        with pytest.raises(B.MoeError):
            call()
            raise AssertionError(n)


@pytest.mark.parametrize("tau", [1.0, 1.7])
def test_the_reference_itself(tau):
    """The 64-bit formulas of head_reference against automatic differentiation of the losses as they are usually written."""
    import head_reference as R
    g = torch.Generator().manual_seed(1)
    T, d, V, K = 6, 64, 11, 4
    x, W = torch.randn(T, d, generator=g).bfloat16(), (0.2 * torch.randn(V, d, generator=g)).bfloat16()
    target = torch.tensor([0, 3, -100, 10, 2, -100]).int()
    ids = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(T)]).int()
    ids[1, 2], ids[4] = -1, -1
    teacher, a, b = torch.randn(T, K, generator=g), torch.rand(T, generator=g), torch.rand(T, generator=g)
    out, _ = R.head(x, W, target, ids, teacher, tau, a, b)
    xd, Wd = x.double().requires_grad_(), W.double().requires_grad_()
    z = xd @ Wd.t()
    loss = torch.nn.functional.cross_entropy(z, target.long(), reduction="none", ignore_index=-100)
    kd = []
    for t in range(T):
        on = ids[t] >= 0
        q = torch.softmax(teacher[t, on].double() / tau, 0)
        kd.append((q * (q.log() - torch.log_softmax(z[t] / tau, 0)[ids[t, on].long()])).sum())
    kd = torch.stack(kd)
    ((loss * a.double()).sum() + (kd * b.double()).sum()).backward()
    for got, want in ((out["loss"], loss), (out["kd"], kd), (out["dx"], xd.grad), (out["dW"], Wd.grad)):
        assert torch.allclose(got, want.detach(), rtol=1e-9, atol=1e-12)
