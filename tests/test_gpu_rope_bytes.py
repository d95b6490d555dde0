"""Rotated keys in e4m3 pages: bytes and scales are those of the exact numbers."""
import numpy as np
import pytest
import torch

from oracle import chai_oracle as orc
from packed_cases import DEV, i32, rotate
from paged_cases import TORCH
from paper_2403_08058_b200 import chai

pytestmark = pytest.mark.gpu


def enter(x, pos, turns, m, interleaved):
    """x [n,planes,D] -> (bytes, scales) of the rotated keys."""
    n, planes, D = x.shape
    page = 8
    kp, vp = (torch.zeros(n // page, planes, page, D, dtype=torch.uint8, device=DEV) for _ in range(2))
    ks, vs = (torch.zeros(n // page, planes, page, device=DEV) for _ in range(2))
    chai.chai_append_rope_paged_fp8(x, x, x, kp, vp, ks, vs, i32([list(range(planes))]), i32(np.zeros(n)), pos,
                                    torch.arange(n, device=DEV), turns, m, interleaved)
    return kp.transpose(1, 2).reshape(n, planes, D).cpu().numpy(), ks.transpose(1, 2).reshape(n, planes).cpu().numpy()


def pairs(y, rot, interleaved):
    """The two numbers of every pair."""
    return (y[..., 0:rot:2], y[..., 1:rot:2]) if interleaved else (y[..., : rot // 2], y[..., rot // 2:rot])


def turned_back(y, pos, turns, m, interleaved):
    return rotate(y, -pos[:, None], turns, 1.0, interleaved)[0] / m


def check(x, pos, turns, m, interleaved, decides):
    ref, _ = rotate(x, pos[:, None], turns, m, interleaved)
    want_q, want_s = orc.quantize_rows_fp8(ref.cpu().numpy())
    got_q, got_s = enter(x, pos, turns, m, interleaved)
    assert np.array_equal(got_s, want_s), int((got_s != want_s).sum())
    # 0x00 and 0x80 are one number, 0: its sign is that of what rounds to it, which fp32 cannot tell of a number smaller than its error
    differ = (got_q != want_q) & ((got_q | want_q) & 0x7F != 0)
    assert not differ.any(), int(differ.sum())
    if decides:   # rotated in fp32 alone, some of these are not
        rot = 2 * turns.numel()
        angle = torch.remainder(pos.double()[:, None, None] * turns.double(), 1.0) * (2 * np.pi)
        c, s = (angle.cos() * m).float(), (angle.sin() * m).float()
        a, b = pairs(x.float(), rot, interleaved)
        y = x.float().clone()
        u, v = pairs(y, rot, interleaved)
        u.copy_(a * c - b * s), v.copy_(b * c + a * s)
        other_q, other_s = orc.quantize_rows_fp8(y.double().cpu().numpy())
        assert ((other_q != want_q) & ((other_q | want_q) & 0x7F != 0)).any() or (other_s != want_s).any()


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("D,rot,interleaved", [(64, 64, False), (128, 128, True), (128, 96, False)])
def test_bytes_of_random_rows(io, D, rot, interleaved):
    g = torch.Generator(device=DEV).manual_seed(rot)
    turns, m = chai.chai_rope_frequencies(rot, scaling="ramp", factor=4.0, context=2048, device=DEV)
    x = torch.randn(4096, 4, D, generator=g, device=DEV).to(TORCH[io])
    pos = torch.randint(-5000, 130000, (4096,), generator=g, device=DEV).to(torch.int32)
    check(x, pos, turns, m, interleaved, decides=False)


@pytest.mark.parametrize("D,interleaved", [(64, False), (64, True), (128, False)])
@pytest.mark.parametrize("m", [1.0, 1.1386294361119891])
def test_bytes_next_to_the_middle_of_two(D, interleaved, m):
    """Rows of the middles between neighbouring e4m3 numbers, turned back and rounded to fp32."""
    n, planes = 2048, 3
    g = torch.Generator(device=DEV).manual_seed(D)
    turns, _ = chai.chai_rope_frequencies(D, device=DEV)
    codes = torch.as_tensor(orc.e4m3_values()[:127].copy(), device=DEV, dtype=torch.float64)
    middles = (codes[1:] + codes[:-1]) / 2
    y = middles[torch.randint(0, 118, (n, planes, D), generator=g, device=DEV)]
    y = y * (torch.randint(0, 2, y.shape, generator=g, device=DEV) * 2 - 1)
    y[..., 0] = 400.0                                              # (the scale is 1 whatever the last bits are)
    pos = torch.randint(0, 60000, (n,), generator=g, device=DEV).to(torch.int32)
    x = turned_back(y * 2.0 ** -7, pos, turns, m, interleaved).float()
    check(x, pos, turns, m, interleaved, decides=True)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("io_bits", [0, -40])
def test_bytes_where_the_scale_is_next_to_a_border(interleaved, io_bits):
    """The largest is 1.75 * 2^i but for its last bits, and every pair's other number is one of the smallest that a byte
    holds: where these round depends on which side the largest falls on."""
    n, planes, D = 8192, 2, 64
    g = torch.Generator(device=DEV).manual_seed(5)
    turns, m = chai.chai_rope_frequencies(D, device=DEV)
    pos = torch.randint(1, 60000, (n,), generator=g, device=DEV).to(torch.int32)
    y = torch.empty(n, planes, D, dtype=torch.float64, device=DEV)
    a, b = pairs(y, D, interleaved)
    a.copy_(1.75 * (0.5 + 0.5 * torch.rand(a.shape, generator=g, device=DEV, dtype=torch.float64)))
    b.copy_(torch.rand(b.shape, generator=g, device=DEV, dtype=torch.float64) * 2.0 ** -13)        # (in steps: up to 2^-5)
    x = turned_back(y, pos, turns, m, interleaved).float()
    ref, _ = rotate(x, pos[:, None], turns, m, interleaved)
    x = (x.double() * (1.75 / ref.abs().amax(-1, keepdim=True))).float() * 2.0 ** io_bits
    ref, _ = rotate(x, pos[:, None], turns, m, interleaved)
    assert len(set(orc.quantize_rows_fp8(ref.cpu().numpy())[1].flatten().tolist())) == 2            # both sides occur
    check(x, pos, turns, m, interleaved, decides=True)


@pytest.mark.parametrize("bits", [-111, -113, -117, -118, -119, -121])
def test_scales_of_tiny_rows_next_to_a_border(bits):
    """Down to 2^-118, below which every row has the smallest scale there is."""
    n, D = 4096, 64
    g = torch.Generator(device=DEV).manual_seed(-bits)
    turns, m = chai.chai_rope_frequencies(D, device=DEV)
    pos = torch.randint(1, 3000, (n,), generator=g, device=DEV).to(torch.int32)
    x = torch.randn(n, 1, D, generator=g, device=DEV)
    ref, _ = rotate(x, pos[:, None], turns, m, False)
    x = (x.double() * (1.75 / ref.abs().amax(-1, keepdim=True))).float() * 2.0 ** bits
    check(x, pos, turns, m, False, decides=bits >= -118)
