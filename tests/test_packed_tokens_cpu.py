"""Packed rows that the binding takes and refuses, by the strides alone (no kernel runs)."""
import pytest
import torch

from paper_2403_08058_b200 import chai

N, H, D = 6, 4, 64
SHAPE = (N, H, D)


def tokens(x, shape=SHAPE):
    return chai._tokens(x, "q", shape, torch.float32, -1)     # (-1: where get_device says a CPU tensor is)


def test_distances_that_are_taken():
    x = torch.zeros(N, 3, H, D)
    assert tokens(x[:, 0]) == 3 * H * D and tokens(x[:, 2]) == 3 * H * D
    assert tokens(torch.zeros(SHAPE)) == H * D
    assert tokens(torch.zeros(N, H * D + 8)[:, : H * D].view(SHAPE)) == H * D + 8
    for one in (torch.zeros(1, H, D), torch.zeros(H, D).expand(1, H, D), torch.zeros(9, H, D)[::3][:1]):
        assert tokens(one, (1, H, D)) == 0                    # (a single token: its own row, whatever the stride)
    assert tokens(torch.zeros(N, 1, D), (N, 1, D)) == D


@pytest.mark.parametrize("apart", [0, 1, 4, D, H * D - 4, H * D - 1])
@pytest.mark.parametrize("n", [2, N])
def test_rows_that_tokens_share_are_refused(apart, n):
    x = torch.zeros(N * H * D).as_strided((n, H, D), (apart, D, 1))
    with pytest.raises(ValueError, match="rows of its own"):
        tokens(x, (n, H, D))


def test_an_expanded_row_is_refused():
    with pytest.raises(ValueError, match="token stride of 0"):
        tokens(torch.zeros(1, H, D).expand(SHAPE))
    with pytest.raises(ValueError, match="token stride of 0"):
        tokens(torch.zeros(1, 1, D).expand(N, 1, D), (N, 1, D))
    with pytest.raises(ValueError, match="side by side"):
        tokens(torch.zeros(1, 1, D).expand(SHAPE))
