"""Paged caches at the edges of their contract: softmax rows that nothing is left of, row scales of every size, rounding of
what is read back, tables wider than the requests, appends of more than one pass."""
import numpy as np
import pytest
import torch

from paged_cases import partition, tables
from paper_2403_08058_b200 import chai
from test_gpu_paged import DEV, KINDS, decode, make, random_pool

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


@pytest.mark.parametrize("N", [1, 40])
@pytest.mark.parametrize("fp8", [False, True])
def test_append_ends_and_stays_in_bounds_while_another_stream_writes_the_lengths(fp8, N):
    """Tokens may go to any row that the tables name, and to no other page; the next call is right."""
    B, H, k, D, page = 40, 8, 3, 64, 8
    rng = np.random.default_rng(N)
    table_np, n_pages = tables([100] * B, page, N, extra_pages=30, room=N)
    table, top = torch.from_numpy(table_np).to(DEV), table_np.shape[1] * page
    _, reps = partition(B, H, k, N)
    reps = torch.from_numpy(reps).to(DEV)
    dt = torch.uint8 if fp8 else torch.bfloat16
    k_new, v_new = (torch.randn(B, H, N, D, device=DEV).to(torch.bfloat16) for _ in range(2))
    pages = [random_pool(n_pages, p, page, D, dt, p) for p in (k, H)]
    pages += [torch.rand(n_pages, p, page, device=DEV) for p in (k, H)] if fp8 else []
    before = [x.clone() for x in pages]
    put = chai.chai_append_kv_paged_fp8 if fp8 else chai.chai_append_kv_paged
    seq, count = torch.full((B,), 20, dtype=torch.int32, device=DEV), torch.full((B,), N, dtype=torch.int32, device=DEV)
    other = [torch.from_numpy(rng.integers(-5, top + 3, B).astype(np.int32)).to(DEV) for _ in range(5)] + [torch.full_like(seq, 1 << 30)]
    some = [torch.from_numpy(rng.integers(-3, N + 3, B).astype(np.int32)).to(DEV) for _ in range(5)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(100):
        with torch.cuda.stream(side):
            for j in range(3):
                seq.copy_(other[(3 * i + j) % len(other)])
                count.copy_(some[(3 * i + j) % len(some)])
        put(k_new, v_new, *pages, reps, table, seq, new_lens=count)
    torch.cuda.synchronize()
    unnamed = torch.ones(n_pages, dtype=torch.bool)
    unnamed[torch.from_numpy(table_np.ravel().astype(np.int64))] = False
    assert unnamed.sum() == 30
    for x, old in zip(pages, before):
        assert torch.equal(x[unnamed.to(DEV)].view(torch.uint8), old[unnamed.to(DEV)].view(torch.uint8))
    seq.fill_(20)
    for x, old in zip(pages, before):
        x.copy_(old)
    put(k_new, v_new, *pages, reps, table, seq)
    assert seq.tolist() == [20 + N] * B
    if not fp8:
        for b in (0, B - 1):
            assert torch.equal(pages[1][table[b, 20 // page].long(), :, 20 % page], v_new[b, :, 0])


# ---- softmax rows that nothing is left of ------------------------------------------------------------------------

@pytest.mark.parametrize("cache,io", KINDS)
@pytest.mark.parametrize("lens", [[1], [900, 1, 30], [2500], [7] * 200], ids=["one token", "joined and whole", "chunks", "many"])
def test_decode_a_cluster_whose_scores_are_all_minus_infinity_is_zero(cache, io, lens):
    """Keys of -inf along a positive query in every row of cluster 0 (e4m3: -1 with an infinite scale); one request in one
    piece and requests that are joined.  The other clusters keep their results bit for bit."""
    B, H, k, page = len(lens), 6, 2, 16
    c = make(cache, io, B, H, k, 64, page, lens, seed=101)
    c["q"].abs_().add_(0.125)
    ws = status_workspace(c)
    want = decode(c, workspace=ws).clone()
    assert torch.isfinite(want).all()
    if cache == "e4m3":
        c["k_pages"][:, 0] = 0xB8                  # -1
        c["k_scales"][:, 0] = float("inf")
    else:
        c["k_pages"][:, 0] = float("-inf")
    got = decode(c, workspace=ws)
    assert chai.chai_device_status(ws) == chai.CHAI_OK
    mine = (c["membership"] == 0)
    assert not got[mine].any() and not torch.isnan(got[mine]).any()
    assert torch.equal(got[~mine], want[~mine])
    # a row that is left counts alone; one that is NaN is not hidden
    last = lens[0] - 1
    at = (int(c["table_np"][0, last // page]), 0, last % page)
    if cache == "e4m3":
        c["k_pages"][at], c["k_scales"][at] = 0x30, 1.0
    else:
        c["k_pages"][at] = 0.5
    row = c["v_rows"][0][:, last]
    got = decode(c, workspace=ws)
    first = [h for h in range(H) if c["mem"][0, h] == 0]
    assert np.array_equal(got[0, first].double().cpu().numpy(), row[first])     # p = 1, values of the output's type
    if cache == "e4m3":
        c["k_scales"][at] = float("nan")
    else:
        c["k_pages"][at] = float("nan")
    got = decode(c, workspace=ws)
    assert torch.isnan(got[0, first]).all()
