"""Keys and queries whose scores are a large number and a small difference, both exact, and the definition for them."""
import math

import torch

from packed_cases import DEV

SCALE = 0.125
# What every score has in common before the scale, as two products of the query's and the key's numbers.  The bf16 number above
# it is 2^10 - 8 (2^12) away: after the scale, 183 and 738 binary orders.
OFFSETS = {"2^17+8": (512.0, 256.0, 8.0, 1.0), "-2^17-1000": (-512.0, 256.0, -1000.0, 1.0), "2^20+2^12": (4096.0, 256.0, 4096.0, 1.0),
           "-2^20-2^12": (-4096.0, 256.0, -4096.0, 1.0)}


def fill(q, k, offset, step, g):
    """q [..., D] and k [..., positions, D] (fp32): scores offset + t, t in -4 .. 4 by halves, and, with a step, the first product's
    key grows (or falls) with the position's tile of 128.  Sums of three products of at most 22 bits between their first
    and last: exact in fp32 in any order."""
    a, A, b, B = OFFSETS[offset]
    q.zero_()
    q[..., 0], q[..., 1], q[..., 2] = a, 1.0, b
    k.zero_()
    n = k.shape[-2]
    tile = torch.arange(n, device=DEV) // 128 % 7
    if step < 0:
        tile = 6 - tile
    k[..., 0] = A + (32.0 * tile if step else 0.0)                 # (256 .. 448 by 32: e4m3 numbers)
    k[..., 1] = torch.randint(-8, 9, k.shape[:-1], generator=g, device=DEV) * 0.5
    k[..., 2] = B


def check_rows(got, q, K, V, see, half_step, bf16, what):
    """got, q [n,D] of one head, K, V [L,D], see [n,L] against the definition in 64 bits.

    Scores are exact.  The exponential's argument is one rounding of an exact difference (to the reference, at most 40 binary
    orders, counted twice, numerator and sum) after a common factor that is good to 2^-24; sums over L positions in fp32
    (tensor cores: 4 u a term) add (2 L + 16) u; bf16 rounds each probability, 2^-8.  The result is rounded once."""
    u = 2.0 ** -24
    L = K.shape[0]
    s = (q.double() @ K.double().T * SCALE).masked_fill(~see, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    ref, spread = p @ V.double(), p @ V.double().abs()
    rel = 2 * 48 * u + (2 * L + 16) * (4 * u if bf16 else u) + (2.0 ** -8 if bf16 else 0.0)
    allowed = rel * spread
    allowed = allowed + half_step * (ref.abs() + allowed) + 1e-37
    assert torch.isfinite(got).all(), what
    worst = float(((got.double() - ref).abs() / allowed).max())
    assert worst <= 1.0, f"{what}: {worst:.3g} of what is allowed"
