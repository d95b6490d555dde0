"""Arrays that rotary positions make and refuse, without a kernel."""
import pytest
import torch

from paper_2403_08058_b200 import chai


def rows_of(x):
    """Storage offsets of all elements."""
    offsets = torch.zeros(x.shape, dtype=torch.int64)
    for d, (n, s) in enumerate(zip(x.shape, x.stride())):
        offsets += (torch.arange(n) * s).view([-1 if i == d else 1 for i in range(4)])
    return offsets.flatten()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,H,N,D", [(1, 1, 1, 64), (2, 3, 5, 64), (1, 4, 1, 128), (3, 1, 7, 64), (2, 1, 1, 64)])
def test_new_arrays_are_dense(B, H, N, D, dtype):
    z = lambda *shape: torch.zeros(*shape, dtype=dtype)
    fused = z(B, N, 3, H, D)
    arrays = {
        "dense": z(B, H, N, D), "tokens first": z(B, N, H, D).transpose(1, 2), "heads first": z(H, B, N, D).transpose(0, 1),
        "requests last": z(H, N, B, D).permute(2, 0, 1, 3),
        "part": fused[:, :, 1].transpose(1, 2), "slice": z(B, H + 2, N + 3, D)[:, 1:-1, 2:-1], "every second": z(2 * B, H, 2 * N, D)[::2, :, ::2],
        "shared": z(1, H, 1, D).expand(B, H, N, D), "shared heads": z(B, 1, N, D).expand(B, H, N, D),
        "windows": z(B, H, (N - 1) * 16 + D).unfold(2, D, 16), "overlapping heads": z(B * 4096).as_strided((B, H, N, D), (4096, 16, 256, 1)),
    }
    for name, x in arrays.items():
        y = chai._rotated_like(x)
        assert y.shape == x.shape and y.dtype is x.dtype and y.stride(3) == 1, name
        assert sorted(rows_of(y).tolist()) == list(range(x.numel())), name        # every element once, no gap
        assert y.untyped_storage().nbytes() == x.numel() * x.element_size(), name
    for name in ("dense", "tokens first", "heads first", "requests last"):
        assert torch.equal(rows_of(chai._rotated_like(arrays[name])), rows_of(arrays[name])), name
    assert chai._rotated_like(arrays["part"]).transpose(1, 2).is_contiguous()
