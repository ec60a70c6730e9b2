"""The norm of gradients refuses a norm or a workspace that lies over what it reads, before anything reaches a device."""
import ctypes

import pytest
import torch

from paper_2604_00785_amd import binding as B
from test_more_operators_host import INVALID, WORKSPACE, N, table

BF16, F32 = 0, 1


@pytest.mark.parametrize("more", [0, 300])
def test_norm_refuses_a_workspace_over_its_inputs(more):
    lib = B.load()
    rest = [((1 << 30) + 4096 * i, 0, 100, BF16) for i in range(more)]
    n = B.moe_grad_norm_workspace_bytes(more + 1)
    call = lambda row, norm, ws, size: lib.moe_grad_norm(table(*rest, row), more + 1, ctypes.c_void_p(norm), ctypes.c_void_p(ws), size, N)  # noqa: E731
    far, ws = 1 << 40, 1 << 20
    for row in ((ws, 0, 1, F32), (ws + n - 2, 0, 1, BF16), (ws - 18, 0, 10, BF16), (ws + 64, 0, 8, F32), (ws - 4096, 0, n + 8192, BF16)):
        assert call(row, far, ws, n) == INVALID, row
    for row in ((far, 0, 1, F32), (far - 18, 0, 10, BF16), (far + 2, 0, 5, BF16), (far - 400, 0, 1000, F32)):
        assert call(row, far, ws, n) == INVALID, row
    for norm in (ws, ws + 16, ws + n - 16):
        assert call((1 << 50, 0, 10, BF16), norm, ws, n) == INVALID, norm
    # side by side they do not overlap, and what lies behind the bytes that it uses is not the call's: nothing of this is refused before the workspace's size is
    assert call((ws, 0, 10, BF16), far, ws, n - 1) == WORKSPACE


def test_first_entry_that_is_no_tensor_is_refused_by_name():
    g, one, ws = torch.zeros(10), torch.zeros(1), torch.zeros(1 << 20, dtype=torch.uint8)
    for call in (lambda grads: B.moe_grad_norm(grads, one, ws), lambda grads: B.moe_grad_clip(grads, 1.0, one, None, ws), lambda grads: B.moe_grad_clip(grads, 1.0, one, [g, g], ws)):
        for grads in ([1.0, g], [None, g], ["g", g], [[1.0], g], [g, 1.0]):
            with pytest.raises(B.MoeError, match="grads"):
                call(grads)
