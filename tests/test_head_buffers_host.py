"""What HeadBuffers and the head's calls refuse by name before anything reaches a device: teachers and gradients that the buffers were not made for, or that are missing."""
import pytest
import torch

from paper_2604_00785_amd import binding as B

T, d, V, K = 4, 64, 100, 3


def inputs():
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    return bf(T, d), bf(V, d), torch.zeros(T, dtype=torch.int32), torch.zeros(T, K, dtype=torch.int32), torch.zeros(T, K), torch.zeros(T)


def buffers(**kw):
    return B.HeadBuffers(T, d, V, device="cpu", **kw)


@pytest.mark.parametrize("what,call", [
    ("teacher", lambda x, W, y, ids, l, w: buffers().run_fwd(x, W, y, ids, l)),
    ("teacher", lambda x, W, y, ids, l, w: buffers().run_bwd(x, W, y, w, ids, l, 1.0, w)),
    ("train", lambda x, W, y, ids, l, w: buffers(train=False).run_bwd(x, W, y, w)),
    ("train", lambda x, W, y, ids, l, w: buffers(K=K, train=False).run_bwd(x, W, y, w, ids, l, 1.0, w)),
    ("teacher", lambda x, W, y, ids, l, w: buffers(K=K).run_fwd(x, W, y, ids)),
    ("dkd", lambda x, W, y, ids, l, w: buffers(K=K).run_bwd(x, W, y, w, ids, l)),
    ("dloss", lambda x, W, y, ids, l, w: buffers().run_bwd(x, W, y, None)),
    ("lse_t", lambda x, W, y, ids, l, w: B.moe_head_distill_fwd(x, W, y, ids, l, 1.0, w, w, w, None, torch.zeros(1 << 20, dtype=torch.uint8))),
    ("ids", lambda x, W, y, ids, l, w: B.moe_head_distill_fwd(x, W, y, None, l, 1.0, w, w, w, w, torch.zeros(1 << 20, dtype=torch.uint8))),
])
def test_refusals_name_what_is_wrong(what, call):
    with pytest.raises(B.MoeError, match=what):
        call(*inputs())


def test_the_rest_gets_as_far_as_the_device():
    x, W, y, ids, l, w = inputs()
    for call in (lambda: buffers().run_fwd(x, W, y), lambda: buffers(K=K).run_fwd(x, W, y, ids, l), lambda: buffers(K=K + 1).run_fwd(x, W, y, ids, l),
                 lambda: buffers(K=K).run_fwd(x, W, y), lambda: buffers().run_bwd(x, W, y, w), lambda: buffers(K=K).run_bwd(x, W, y, w, ids, l, 1.0, w)):
        with pytest.raises(B.MoeError, match="device tensors"):
            call()
