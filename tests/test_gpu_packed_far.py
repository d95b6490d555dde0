"""Attention over pages with scores of ten thousands and more: what counts is their difference to the row's largest."""
import numpy as np
import pytest
import torch

from far_scores import OFFSETS, SCALE, check_rows, fill
from packed_cases import DEV, HALF_STEP, attend, batch, rows
from paper_2403_08058_b200 import chai

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache,io", [("f32", "f32"), ("bf16", "bf16"), ("e4m3", "bf16"), ("e4m3", "f32")])
@pytest.mark.parametrize("offset", list(OFFSETS))
@pytest.mark.parametrize("D,kv,new,step,causal", [
    (64, [300, 1, 129], [150, 1, 129], 0, True),
    (128, [300, 40], [300, 9], 0, False),
    (128, [9000, 700], [2, 3], 0, True),             # divided among CTAs
    (64, [860, 860], [200, 2], 1, True),             # the reference moves with every tile
    (128, [860, 5000], [3, 40], -1, True),
])
def test_attention_far_scores(cache, io, offset, D, kv, new, step, causal):
    H, k, page = 5, 2, 16
    c = batch(cache, io, H, k, D, page, kv, new, seed=D + len(kv))
    c["scale"] = SCALE
    g = torch.Generator(device=DEV).manual_seed(17)
    q = torch.empty(c["n_tokens"], H, D, device=DEV)
    for b, n in enumerate(kv):
        x = torch.empty(k, n, D, device=DEV)
        fill(q, x, offset, step, g)
        t = torch.arange(n, device=DEV)
        at = c["table"][b].long()[t // page]
        if cache == "e4m3":
            c["k_pages"][at, :, t % page] = x.transpose(0, 1).to(torch.float8_e4m3fn).view(torch.uint8)
            c["k_scales"][at, :, t % page] = 1.0
        else:
            c["k_pages"][at, :, t % page] = x.transpose(0, 1).to(c["k_pages"].dtype)
        assert torch.equal(rows(c, "k", b), x.double())
    c["q"] = q.to(c["q"].dtype)
    ws = chai.new_workspace(chai.chai_prefill_paged_workspace_bytes(c["B"], H, c["n_tokens"]), DEV)
    out = attend(c, causal, workspace=ws)
    assert chai.chai_device_status(ws) == chai.CHAI_OK
    start = np.concatenate([[0], np.cumsum(new)])
    for b, (L, n) in enumerate(zip(kv, new)):
        K, V = rows(c, "k", b), rows(c, "v", b)
        last = L - n + torch.arange(n, device=DEV)[:, None] if causal else torch.full((n, 1), L, device=DEV)
        see = torch.arange(L, device=DEV)[None] <= last
        for h in range(H):
            cl = int(c["mem"][b][h])
            mine = slice(int(start[b]), int(start[b]) + n)
            check_rows(out[mine, h], c["q"][mine, int(c["reps_np"][b][cl])], K[cl], V[h], see, HALF_STEP[io], io == "bf16",
                       f"{cache} {io} request {b} head {h}")
