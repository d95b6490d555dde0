"""Paged caches at the edges of their contract: softmax rows that nothing is left of, row scales of every size, rounding of
what is read back, tables wider than the requests, appends of more than one pass."""
import numpy as np
import pytest
import torch

from paged_cases import tables
from paper_2403_08058_b200 import chai
from test_gpu_paged import DEV, decode, make

pytestmark = pytest.mark.gpu


def status_workspace(c):
    return chai.new_workspace(chai.chai_decode_paged_workspace_bytes(c["B"], c["H"], c["D"]), DEV)


# ---- lengths that another stream writes --------------------------------------------------------------------------

@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("B", [5, 32, 33, 200])
def test_decode_ends_and_stays_in_bounds_while_another_stream_writes_the_lengths(cache, B):
    """Results are anyone's then, but every row that is read is one that the table names, every barrier is met by all, and
    the next call is right.  (All entries of the tables are pages of the pool, so any length may be read.)"""
    rng = np.random.default_rng(B)
    lens = [int(x) for x in rng.integers(0, 6000 // B, B)]
    lens[-1] = 900
    c = make(cache, "bf16", B, 12, 4, 64, 8, lens, seed=B)
    ws, out = status_workspace(c), torch.empty_like(c["q"])
    want = decode(c, workspace=ws).clone()
    right = c["seq"].clone()
    top = c["table"].shape[1] * 8
    other = [torch.from_numpy(rng.integers(-5, top + 1, B).astype(np.int32)).to(DEV) for _ in range(6)]
    other += [torch.zeros_like(right), torch.full_like(right, 1 << 30), right]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(150):
        with torch.cuda.stream(side):
            for j in range(4):
                c["seq"].copy_(other[(4 * i + j) % len(other)])
        decode(c, out=out, workspace=ws)
    torch.cuda.synchronize()
    assert chai.chai_device_status(ws) != chai.CHAI_ERR_TIMEOUT
    c["seq"].copy_(right)
    for _ in range(2):
        assert torch.equal(decode(c, workspace=ws).view(torch.uint8), want.view(torch.uint8))
        assert chai.chai_device_status(ws) == chai.CHAI_OK
