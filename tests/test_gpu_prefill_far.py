"""Prefill of dense arrays with scores of ten thousands and more: what counts is their difference to the row's largest."""
import pytest
import torch

from far_scores import OFFSETS, SCALE, check_rows, fill
from packed_cases import DEV, HALF_STEP, i32
from paged_cases import TORCH, partition
from paper_2403_08058_b200 import chai

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("offset", list(OFFSETS))
@pytest.mark.parametrize("D,T,step,causal", [(64, 300, 0, True), (128, 300, 0, False), (128, 860, 1, True), (64, 860, -1, False),
                                             (128, 860, -1, True)])
@pytest.mark.parametrize("qkv", [False, True])
def test_prefill_far_scores(io, offset, D, T, step, causal, qkv):
    B, H, k = 2, 5, 2
    g = torch.Generator(device=DEV).manual_seed(D + T)
    mem, reps = partition(B, H, k, T)
    q, x = torch.empty(B, H, T, D, device=DEV), torch.empty(B, k, T, D, device=DEV)
    fill(q, x, offset, step, g)
    v = torch.randn(B, k if qkv else H, T, D, generator=g, device=DEV).to(TORCH[io])
    q, K = q.to(TORCH[io]), x.to(TORCH[io])
    assert torch.equal(K.float(), x)
    fn = chai.chai_prefill_attention_qkv if qkv else chai.chai_prefill_attention
    out = fn(q, K, v, i32(mem), i32(reps), SCALE, causal=causal)
    t = torch.arange(T, device=DEV)
    see = t[None] <= (t[:, None] if causal else T)
    for b in range(B):
        for h in range(H):
            cl = int(mem[b][h])
            check_rows(out[b, h], q[b, int(reps[b][cl])], K[b, cl], v[b, cl if qkv else h], see, HALF_STEP[io], io == "bf16",
                       f"{io} request {b} head {h}")
