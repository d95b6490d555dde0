"""Rotary positions of rows that lie on one another, between other rows, and in place."""
import numpy as np
import pytest
import torch

from packed_cases import DEV, i32
from paged_cases import TORCH
from paper_2403_08058_b200 import chai

pytestmark = pytest.mark.gpu


def given(B, N, seed):
    turns, m = chai.chai_rope_frequencies(32, scaling="ramp", factor=2.0, context=512, device=DEV)
    return i32(np.random.default_rng(seed).integers(0, 9000, (B, N))), turns, m


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_rows_that_overlap(io):
    """Sliding windows as input: outputs have rows of their own."""
    B, H, N, D = 2, 3, 700, 64
    g = torch.Generator(device=DEV).manual_seed(4)
    base = torch.randn(B, H, (N - 1) * 16 + D, generator=g, device=DEV).to(TORCH[io])
    x = base.unfold(2, D, 16)
    assert x.shape == (B, H, N, D) and x.stride(2) == 16
    pos, turns, m = given(B, N, 1)
    want = chai.chai_rope(x.contiguous(), None, pos, turns, m)[0]
    for _ in range(4):
        got = chai.chai_rope(x, None, pos, turns, m)[0]
        assert torch.equal(got, want)
    assert got.untyped_storage().nbytes() == got.numel() * got.element_size()
    again = chai.chai_rope(x[:1], x[:1, :2], pos[:1], turns, m)
    assert torch.equal(again[0], want[:1]) and torch.equal(again[1], want[:1, :2])


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_parts_of_one_projection(io):
    """New arrays hold the rows alone; in place, and into other rows of the same array, nothing else is written."""
    B, Hq, Hk, N, D = 2, 4, 2, 50, 64
    g = torch.Generator(device=DEV).manual_seed(5)
    wide = torch.randn(B, N, Hq + 2 * Hk + Hq, D, generator=g, device=DEV).to(TORCH[io])
    part = lambda x, h0, h1: x[:, :, h0:h1].transpose(1, 2)
    q, k = part(wide, 0, Hq), part(wide, Hq, Hq + Hk)
    pos, turns, m = given(B, N, 2)
    want = chai.chai_rope(q.contiguous(), k.contiguous(), pos, turns, m)
    got = chai.chai_rope(q, k, pos, turns, m)
    for a, b in zip(got, want):
        assert torch.equal(a, b) and a.untyped_storage().nbytes() == a.numel() * a.element_size()
        assert a.transpose(1, 2).is_contiguous()                    # (the order of the input's rows)
    one = wide.clone()
    chai.chai_rope(part(one, 0, Hq), part(one, Hq, Hq + Hk), pos, turns, m, q_out=part(one, 0, Hq), k_out=part(one, Hq, Hq + Hk))
    assert torch.equal(part(one, 0, Hq), want[0]) and torch.equal(part(one, Hq, Hq + Hk), want[1])
    assert torch.equal(one[:, :, Hq + Hk:], wide[:, :, Hq + Hk:])
    one = wide.clone()
    chai.chai_rope(part(one, 0, Hq), None, pos, turns, m, q_out=part(one, Hq + 2 * Hk, 2 * Hq + 2 * Hk))
    assert torch.equal(part(one, Hq + 2 * Hk, 2 * Hq + 2 * Hk), want[0])
    assert torch.equal(one[:, :, : Hq + 2 * Hk], wide[:, :, : Hq + 2 * Hk])


def test_refusals_of_arrays_that_overlap():
    pos, turns, m = given(1, 8, 3)
    raw = torch.randn(20000, device=DEV)
    view = lambda at, H=2, strides=(1024, 512, 64, 1): raw.as_strided((1, H, 8, 64), strides, at)
    before = raw.clone()
    with pytest.raises(chai.ChaiError, match="overlap"):
        chai.chai_rope(view(0), None, pos, turns, m, q_out=view(64))
    with pytest.raises(chai.ChaiError, match="overlap"):
        chai.chai_rope(view(0), view(4096), pos, turns, m, q_out=view(8192), k_out=view(8192 + 512))
    with pytest.raises(chai.ChaiError, match="overlap"):
        chai.chai_rope(view(0), None, pos, turns, m, q_out=view(4096, strides=(1024, 512, 32, 1)))
    assert torch.equal(raw, before)
    out = chai.chai_rope(view(0), view(4096), pos, turns, m, q_out=view(8192), k_out=view(8192 + 1024))
    assert torch.equal(out[0], chai.chai_rope(view(0).contiguous(), None, pos, turns, m)[0])
    assert torch.equal(out[1], chai.chai_rope(view(4096).contiguous(), None, pos, turns, m)[0])
