"""A workspace for the largest batch is laid out for smaller ones too."""
import pytest

from paper_2604_00785_amd import binding as B

TOKENS = sorted({*range(1, 600, 16), *(1 << k for k in range(17))})


@pytest.mark.parametrize("d", [64, 512, 2048, 4096])
@pytest.mark.parametrize("V", [70, 1031, 5000, 16000, 16384, 50304])
def test_sizes_of_the_scores_grow_with_the_tokens(d, V):
    for K in (0, 1, 20, 64):
        sizes = [B.moe_head_score_fwd_workspace_bytes(T, d, V, K) for T in TOKENS]
        assert sizes[0] > 0 and sizes == sorted(sizes), K
    for piece in (0, 256):
        # (with many tokens, which serve any fewer in whatever room there is, the parts of a reduction may take less than some tokens before)
        sizes = [B.moe_head_score_bwd_workspace_bytes(T, d, V, piece) for T in TOKENS if T <= 512]
        assert sizes[0] > 0 and sizes == sorted(sizes), piece


def test_scores_without_alternatives_ask_for_what_they_leave():
    """16 bytes for each 64 columns of a token beside its row (tokens by sixteens)."""
    for T, d, V in ((8192, 2048, 50304), (1000, 64, 131072), (16384, 128, 40000)):
        n = B.moe_head_score_fwd_workspace_bytes(T, d, V, 0)
        assert T * (2 * d + 16 * (V // 64)) <= n <= (T + 15) * (2 * d + 16 * (V // 64 + 1) + 32) + 4096


def test_no_kernel_that_nothing_launches():
    """1024 threads to a token's logits are for alternatives alone; each other number of threads is there with and without them."""
    names = open(B.LIB_PATH, "rb").read()
    kernel = lambda threads, pieces, lists: b"head_score_whole_kernelILi%dELi%dELb%dE" % (threads, pieces, lists) in names  # noqa: E731
    assert kernel(1024, 2, 1) and not kernel(1024, 2, 0)
    assert all(kernel(t, p, k) for t, p in ((64, 2), (64, 8), (128, 8), (256, 2), (256, 8), (512, 8)) for k in (0, 1))
