"""What the head's scores, the norms of queries and keys and the gradients' norm refuse before anything reaches a device."""
import ctypes

import pytest
import torch

from paper_2604_00785_amd import binding as B

INVALID, WORKSPACE = -1, -2
N, P, Q = None, ctypes.c_void_p(4096), ctypes.c_void_p(4104)      # never followed: a call that is refused reads nothing
BIG = 1 << 40


def qk_args(bwd):
    """Names and values of a call that would go through."""
    d = {}
    if bwd:
        d.update(dqo=P, dqo_ld=128, dko=P, dko_ld=64)
    d.update(q=P, q_ld=128, k=P, k_ld=64, wq=P, wk=P, pos=P, freq=P, pairs=0, eps=1e-5, T=4, Hq=2, Hk=1, D=64, R=32)
    d.update(dict(dq=P, dq_ld=128, dk=P, dk_ld=64, dwq=P, dwk=P, ws=P, n=BIG) if bwd else dict(qo=P, qo_ld=128, ko=P, ko_ld=64))
    return d


@pytest.mark.parametrize("bwd", [False, True])
def test_qk_refusals(bwd):
    lib = B.load()
    fn = lib.moe_qk_norm_rope_bwd if bwd else lib.moe_qk_norm_rope
    ok = qk_args(bwd)
    bad = [(n, v) for n, p in ok.items() if p is P for v in (N, Q)]
    bad += [(n, v) for n in ok if n.endswith("_ld") for v in (56, 0, -128, 132, (1 << 32) + 8)]
    bad += [("T", 0), ("T", -1), ("T", (1 << 30) + 1), ("Hq", 0), ("Hk", 0), ("Hq", 4097), ("Hk", -1), ("D", 0), ("D", 60), ("D", 520), ("R", -16), ("R", 8),
            ("R", 80), ("eps", -1e-5), ("eps", float("nan"))]
    for name, value in bad:
        assert fn(*dict(ok, **{name: value}).values(), N) == INVALID, (name, value)
    # in place only with the rows where they are (here all tensors have one address)
    for name in ("dq_ld", "dk_ld") if bwd else ("qo_ld", "ko_ld"):
        assert fn(*dict(ok, **{name: 256}).values(), N) == INVALID, name
    if bwd:
        n = B.moe_qk_norm_rope_bwd_workspace_bytes(4, 2, 1, 64)
        assert n > 0 and fn(*dict(ok, n=n - 1).values(), N) == WORKSPACE
        for T, Hq, Hk, D in ((0, 2, 1, 64), (4, 0, 1, 64), (4, 2, 0, 64), (4, 2, 1, 60), (4, 2, 1, 1024)):
            assert B.moe_qk_norm_rope_bwd_workspace_bytes(T, Hq, Hk, D) == 0
        assert B.moe_qk_norm_rope_bwd_workspace_bytes(1 << 20, 32, 8, 128) <= 1 << 20           # shares do not grow with the tokens


class Grad(ctypes.Structure):
    _fields_ = [("in_", ctypes.c_void_p), ("out", ctypes.c_void_p), ("count", ctypes.c_int64), ("type", ctypes.c_int64)]


def table(*rows):
    return (Grad * len(rows))(*[Grad(*r) for r in rows])


def test_grad_refusals():
    lib = B.load()
    ok = table((1 << 20, 1 << 20, 10, 0), (2 << 20, 3 << 20, 10, 1))
    for call in (lambda g, n, norm, ws, b: lib.moe_grad_norm(g, n, norm, ws, b, N), lambda g, n, norm, ws, b: lib.moe_grad_clip(g, n, 1.0, norm, ws, b, N)):
        for args in ((N, 2, P, P, BIG), (ok, 0, P, P, BIG), (ok, -1, P, P, BIG), (ok, (1 << 20) + 1, P, P, BIG), (ok, 2, N, P, BIG), (ok, 2, Q, P, BIG), (ok, 2, P, N, BIG),
                     (ok, 2, P, Q, BIG)):
            assert call(*args) == INVALID, args
        assert call(ok, 2, P, P, B.moe_grad_norm_workspace_bytes(2) - 1) == WORKSPACE
        for row in ((4096, 4096, 10, 2), (4096, 4096, 10, -1), (4096, 4096, -1, 0), (4096, 4096, (1 << 40) + 1, 0), (0, 4096, 10, 0), (4097, 4096, 10, 0),
                    (4098, 4096, 10, 1)):
            assert call(table((1 << 20, 1 << 20, 5, 0), row), 2, P, P, BIG) == INVALID, row
    for largest in (0.0, -1.0, float("inf"), float("nan")):
        assert lib.moe_grad_clip(ok, 2, largest, P, P, BIG, N) == INVALID
    for row in ((4096, 0, 10, 0), (4096, 4097, 10, 0), (4096, 4098, 10, 1)):
        assert lib.moe_grad_clip(table(row), 1, 1.0, P, P, BIG, N) == INVALID, row
    assert B.moe_grad_norm_workspace_bytes(0) == 0 and B.moe_grad_norm_workspace_bytes(-3) == 0 and B.moe_grad_norm_workspace_bytes((1 << 20) + 1) == 0


@pytest.mark.parametrize("more", [0, 300])
def test_clipping_refuses_outputs_over_other_tensors(more):
    """The same tensor twice, an output over another's input, over another's output, over its own input at another place."""
    lib = B.load()
    rest = [((1 << 30) + 4096 * i, (1 << 31) + 4096 * i, 100, 0) for i in range(more)]
    far, further = ctypes.c_void_p(1 << 40), ctypes.c_void_p(1 << 41)
    for rows in ([(4096, 4096, 10, 0), (4096, 4096, 10, 0)], [(4096, 8192, 10, 0), (4112, 8200, 2, 1)], [(4096, 8192, 10, 0), (8210, 16384, 3, 0)],
                 [(4096, 4100, 10, 0)], [(4096, 4092, 10, 1)], [(4096, 8192, 1000, 0), (4100, 4100, 1, 0)], [(4100, 4100, 1, 1), (4096, 16384, 8, 0)]):
        assert lib.moe_grad_clip(table(*rest, *rows), more + len(rows), 1.0, far, further, BIG, N) == INVALID, rows
    # the norm or the workspace over a tensor, or over each other
    for norm, ws, rows in ((4096, 8192, [(4090, 4090, 10, 0)]), (4096, 8192, [(4096, 1 << 20, 1, 1)]), (1 << 40, 4096, [(1 << 20, 4096 + 1024 * 8 - 2, 1, 0)]),
                           (1 << 40, 4096, [(4096, 1 << 20, 1, 0)]), (4096 + 16, 4096, [(1 << 20, 1 << 21, 1, 0)])):
        assert lib.moe_grad_clip(table(*rest, *rows), more + len(rows), 1.0, ctypes.c_void_p(norm), ctypes.c_void_p(ws), BIG, N) == INVALID, (norm, ws, rows)


def test_binding_refuses_types_shapes_and_host_tensors():
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    q, k, w, pos, freq, ws = bf(4, 2, 64), bf(4, 1, 64), torch.zeros(64), torch.zeros(4, dtype=torch.int32), torch.zeros(16), torch.zeros(1 << 20, dtype=torch.uint8)
    one = torch.zeros(1)
    calls = [
        ("device", lambda: B.moe_qk_norm_rope(q, k, w, w, pos, freq, False, 1e-5, q, k)),               # on the host
        ("device", lambda: B.moe_qk_norm_rope_bwd(q, k, q, k, w, w, pos, freq, False, 1e-5, q, k, w, w, ws)),
        ("q", lambda: B.moe_qk_norm_rope(q[0], k, w, w, pos, freq, False, 1e-5, q, k)),
        ("k", lambda: B.moe_qk_norm_rope(q, None, w, w, pos, freq, False, 1e-5, q, k)),
        ("freq", lambda: B.moe_qk_norm_rope(q, k, w, w, pos, freq.double(), False, 1e-5, q, k)),
        ("freq", lambda: B.moe_qk_norm_rope(q, k, w, w, pos, freq.view(2, 8), False, 1e-5, q, k)),
        ("grads", lambda: B.moe_grad_norm([q], one, ws)),                                                # on the host
        ("outs", lambda: B.moe_grad_clip([q, k], 1.0, one, [q], ws)),
        ("no tensors", lambda: B.moe_grad_norm([], one, ws)),
    ]
    for n, (what, call) in enumerate(calls):
        with pytest.raises(B.MoeError, match=what):
            call()
            raise AssertionError(n)


def score_args(bwd):
    d = dict(x=P, W=P, target=P, temperature=1.0)
    if bwd:
        d.update(logp=P, entropy=P, lse=P, dlogp=P, dentropy=P, T=4, d=64, V=100, v_piece=0, dx=P, dW=P, ws=P, n=BIG)
    else:
        d.update(T=4, d=64, V=100, K=5, logp=P, entropy=P, lse=P, ids=P, top=P, ws=P, n=BIG)
    return d


@pytest.mark.parametrize("bwd", [False, True])
def test_score_refusals(bwd):
    lib = B.load()
    fn = lib.moe_head_score_bwd if bwd else lib.moe_head_score_fwd
    ok = score_args(bwd)
    bad = [(n, v) for n, p in ok.items() if p is P for v in (N, Q) if (n, v) != ("dentropy", N)]
    bad += [("T", 0), ("T", -2), ("T", (1 << 26) + 1), ("d", 0), ("d", 32), ("d", 100), ("V", 0), ("V", (1 << 20) + 1)]
    bad += [("temperature", v) for v in (0.0, -1.0, float("inf"), float("nan"))]
    bad += [("v_piece", v) for v in (-256, 1, 300)] if bwd else [("K", -1), ("K", 65), ("V", 4)]
    for name, value in bad:
        assert fn(*dict(ok, **{name: value}).values(), N) == INVALID, (name, value)
    assert fn(*dict(ok, n=100).values(), N) == WORKSPACE
    if bwd:
        assert B.moe_head_score_bwd_workspace_bytes(4, 64, 100, 300) == 0 and B.moe_head_score_bwd_workspace_bytes(4, 60, 100) == 0
    else:
        for T, d, V, K in ((0, 64, 100, 5), (4, 60, 100, 5), (4, 64, 0, 0), (4, 64, 100, 65), (4, 64, 4, 5), (4, 64, 100, -1)):
            assert B.moe_head_score_fwd_workspace_bytes(T, d, V, K) == 0
        assert B.moe_head_score_fwd_workspace_bytes(8192, 2048, 50304, 20) < 8192 * 50304           # far from the logits (2 bytes each)


def test_scores_in_the_binding():
    bf, f32 = lambda *s: torch.zeros(*s, dtype=torch.bfloat16), lambda *s: torch.zeros(*s)  # noqa: E731
    x, W, y, r, ids, ws = bf(4, 64), bf(100, 64), torch.zeros(4, dtype=torch.int32), f32(4), torch.zeros(4, 5, dtype=torch.int32), torch.zeros(1 << 20, dtype=torch.uint8)
    for what, call in [
        ("device", lambda: B.moe_head_score_fwd(x, W, y, 1.0, r, r, r, ids, f32(4, 5), ws)),             # on the host
        ("x, W", lambda: B.moe_head_score_fwd(None, W, y, 1.0, r, r, r, ids, f32(4, 5), ws)),
        ("x, W", lambda: B.moe_head_score_bwd(x, W[0], y, 1.0, r, r, r, r, r, 0, x, W, ws)),
    ]:
        with pytest.raises(B.MoeError, match=what):
            call()


def test_score_buffers():
    x, W, y, r = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(100, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    for kw in (dict(K=65), dict(K=101), dict(K=-1), dict(v_piece=100)):
        with pytest.raises(B.MoeError, match="no scores"):
            B.ScoreBuffers(4, 64, 100, device="cpu", **kw)
    with pytest.raises(B.MoeError, match="train"):
        B.ScoreBuffers(4, 64, 100, train=False, device="cpu").run_bwd(x, W, y, r)
    for call in (lambda b: b.run_fwd(x, W, y), lambda b: b.run_bwd(x, W, y, r)):
        with pytest.raises(B.MoeError, match="device"):
            call(B.ScoreBuffers(4, 64, 100, 5, device="cpu"))
    assert B.ScoreBuffers(4, 64, 100, 0, train=False, device="cpu").ids is None
