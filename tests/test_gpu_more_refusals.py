"""What the head's scores, the norms of queries and keys and the gradients' norm refuse by name, on tensors that are on the device otherwise."""
import pytest
import torch

from paper_2604_00785_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def bf(*s):
    return torch.zeros(*s, dtype=torch.bfloat16, device=DEV)


def f32(*s):
    return torch.zeros(*s, device=DEV)


def i32(*s):
    return torch.zeros(*s, dtype=torch.int32, device=DEV)


def refused(args, call, changes):
    call(*args.values())                                                          # goes through as it is
    for name, value, what in changes:
        with pytest.raises(B.MoeError, match=what):
            call(*dict(args, **{name: value}).values())
            raise AssertionError((name, what))
    torch.cuda.synchronize()


def test_norms_of_queries_and_keys():
    T, D = 4, 64
    args = dict(q=bf(T, 2, D), k=bf(T, 1, D), wq=f32(D), wk=f32(D), pos=i32(T), freq=f32(16), pairs=False, eps=1e-5, qo=bf(T, 2, D), ko=bf(T, 1, D))
    refused(args, B.moe_qk_norm_rope, [
        ("q", f32(T, 2, D), "q"), ("k", bf(T + 1, 1, D), "k"), ("k", bf(T, 1, D // 2), "k"), ("wq", bf(D), "wq"), ("wk", f32(D + 1), "wk"), ("wk", None, "wk"),
        ("wq", f32(2 * D)[::2], "wq"), ("pos", i32(T).long(), "pos"), ("pos", i32(T + 1), "pos"), ("freq", f32(16).double(), "freq"), ("freq", f32(33), "INVALID"),
        ("freq", f32(7), "INVALID"), ("qo", bf(T, 3, D), "qo"), ("ko", bf(T, 1, D).cpu(), "ko"), ("qo", bf(T, D, 2).transpose(1, 2), "qo"), ("q", bf(T, 4, D)[:, ::2], "q"),
        ("eps", -1.0, "INVALID")])
    args = dict(dqo=bf(T, 2, D), dko=bf(T, 1, D), q=bf(T, 2, D), k=bf(T, 1, D), wq=f32(D), wk=f32(D), pos=i32(T), freq=None, pairs=True, eps=1e-5, dq=bf(T, 2, D),
                dk=bf(T, 1, D), dwq=f32(D), dwk=f32(D), ws=torch.zeros(B.moe_qk_norm_rope_bwd_workspace_bytes(T, 2, 1, D), dtype=torch.uint8, device=DEV))
    refused(args, B.moe_qk_norm_rope_bwd, [
        ("dqo", bf(T, 1, D), "dqo"), ("dk", f32(T, 1, D), "dk"), ("dwq", bf(D), "dwq"), ("dwk", None, "dwk"), ("ws", None, "ws"), ("ws", args["ws"].cpu(), "ws"),
        ("ws", args["ws"][:-1], "WORKSPACE")])


def test_gradients():
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)
    g, h = bf(10), f32(4, 4)
    refused(dict(grads=[g, h], norm=f32(1), ws=ws), B.moe_grad_norm, [
        ("grads", [g, h.double()], r"grads.1."), ("grads", [g, h.t()[1:]], "grads"), ("grads", [g, h.cpu()], "grads"), ("norm", f32(2), "norm"), ("norm", None, "norm"),
        ("ws", None, "ws"), ("ws", ws[:8], "WORKSPACE"), ("grads", [g, None], "grads"), ("grads", [None, g], "grads")])
    refused(dict(grads=[g, h], largest=1.0, norm=f32(1), outs=[bf(10), f32(4, 4)], ws=ws), B.moe_grad_clip, [
        ("grads", [g, g], "outs"), ("outs", [g], "outs"), ("outs", [g, None], "outs"), ("outs", [bf(9), h], r"outs.0."), ("outs", [bf(10), bf(4, 4)], r"outs.1."), ("largest", 0.0, "INVALID"),
        ("outs", [bf(10), f32(4, 8)[:, ::2]], "outs")])
    both = bf(20)
    refused(dict(grads=[g, h], largest=1.0, norm=f32(1), outs=None, ws=ws), B.moe_grad_clip, [("grads", [g, g], "INVALID"), ("grads", [both[:12], both[11:]], "INVALID")])


def test_scores():
    T, d, V, K = 4, 64, 100, 5
    ws = torch.zeros(max(B.moe_head_score_fwd_workspace_bytes(T, d, V, K), B.moe_head_score_bwd_workspace_bytes(T, d, V)), dtype=torch.uint8, device=DEV)
    args = dict(x=bf(T, d), W=bf(V, d), target=i32(T), temperature=1.0, logp=f32(T), entropy=f32(T), lse=f32(T), ids=i32(T, K), top=f32(T, K), ws=ws)
    refused(args, B.moe_head_score_fwd, [
        ("x", f32(T, d), "x"), ("W", bf(V, d + 64), "W"), ("W", bf(V, 2 * d)[:, :d], "W"), ("target", i32(T).long(), "target"), ("logp", f32(T + 1), "logp"),
        ("entropy", None, "entropy"), ("lse", bf(T), "lse"), ("ids", None, "ids"), ("top", None, "top"), ("top", f32(T, K + 1), "top"), ("ids", i32(T, K).long(), "ids"),
        ("temperature", 0.0, "INVALID"), ("ws", ws[:256], "WORKSPACE"), ("ws", None, "ws"), ("x", None, "x")])
    for n in (65, 0):
        with pytest.raises(B.MoeError):
            B.moe_head_score_fwd(*dict(args, W=bf(200, d), ids=i32(T, n), top=f32(T, 65)).values())
    args = dict(x=bf(T, d), W=bf(V, d), target=i32(T), temperature=1.0, logp=f32(T), entropy=f32(T), lse=f32(T), dlogp=f32(T), dentropy=f32(T), v_piece=0, dx=bf(T, d),
                dW=bf(V, d), ws=ws)
    refused(args, B.moe_head_score_bwd, [
        ("dlogp", None, "dlogp"), ("dentropy", f32(T + 1), "dentropy"), ("dx", f32(T, d), "dx"), ("dW", bf(V + 1, d), "dW"), ("v_piece", 100, "INVALID"),
        ("ws", ws[:256], "WORKSPACE")])
