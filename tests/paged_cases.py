"""Paged pools for the tests: random page order, unused rows and pages full of NaN, and error bounds from arithmetic."""
import numpy as np
import torch

from oracle import chai_oracle as orc
from paper_2403_08058_b200 import synth

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
U32 = 2.0 ** -24                                 # half a step of fp32, relative
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def bits(t):
    """A numpy view of a tensor for bit-exact comparison."""
    t = t.detach().cpu().contiguous()
    return {1: lambda: t.view(torch.uint8), 2: lambda: t.view(torch.int16), 4: lambda: t.view(torch.int32)}[t.element_size()]().numpy()


def tables(lens, page, seed, extra_pages=3, room=0):
    """block_table [B,max_pages] (a random order of distinct pages) and the pool's page count."""
    rng = np.random.default_rng([seed, page])
    max_pages = max(1, -(-(max(lens) + room) // page)) + 1
    n_pages = len(lens) * max_pages + extra_pages
    return rng.permutation(n_pages)[: len(lens) * max_pages].reshape(len(lens), max_pages).astype(np.int32), n_pages


def partition(B, H, k, seed):
    return synth.batch_partitions(B, H, k, "uneven", seed, H, k)


def pool(values, lens, table, n_pages, page, fill):
    """Dense rows values[b] [planes, len, ...] -> pages [n_pages, planes, page, ...]; every other row holds `fill`."""
    planes, tail = values[0].shape[0], values[0].shape[2:]
    out = np.full((n_pages, planes, page) + tail, fill, dtype=values[0].dtype)
    for b, n in enumerate(lens):
        for t in range(n):
            out[table[b, t // page], :, t % page] = values[b][:, t]
    return out


def decode_bounds(q, kr, vr, mem, reps, scale, io, fp8):
    """|error| allowed per output element of one request (q [H,D], kr [k,n,D], vr [H,n,D] in float64).

    A score is a sum of D products in fp32: off by at most (D + 4) u S, S = scale * sum|q k|, u = 2^-24; with scores of
    size up to M the argument of the exponential is rounded too, (M + 2) u, and exp2 itself is good to 2 u or so.  Each
    probability is then off by twice that, relative (numerator and sum), and the two sums over n rows add 2 n u at
    most.  e4m3 caches: products run on the tensor cores, whose fp32 sums are counted at 4 u a term, and q and p are
    held as two fp16 numbers: off by 2^-22 of the largest |q| in the row, and of p by 2^-23 of its scale.  The result
    is rounded once to its type."""
    D, n = q.shape[1], kr.shape[1]
    qr = q[reps]
    s = scale * np.einsum("cd,ctd->ct", qr, kr)
    top = s.max(1, keepdims=True)
    p = np.exp(s - top)
    total = p.sum(1)
    size = scale * np.einsum("cd,ctd->ct", np.abs(qr), np.abs(kr)).max(1)
    if fp8:
        size = size + scale * D / 4.0 * np.abs(qr).max(1) * np.abs(kr).max((1, 2)) / (D + 4)
    u = 4 * U32 if fp8 else U32
    rel = 2 * ((D + 4) * u * size + (np.abs(s).max(1) + np.abs(top[:, 0]) + 8) * U32) + (2 * n + 16) * u
    spread = np.einsum("ht,htd->hd", (p / total[:, None])[mem], np.abs(vr))
    out = rel[mem][:, None] * spread
    if fp8:
        out = out + 2.0 ** -22 * n / total[mem][:, None] * np.abs(vr).max((1, 2))[:, None]
    return out


def assert_decode(got, q, kr, vr, mem, reps, lens, scale, io, fp8, what=""):
    """got [B,H,D] (float64 numpy) against the definition on dense float64 rows kr[b], vr[b]."""
    for b, n in enumerate(lens):
        if n == 0:
            assert not got[b].any(), f"{what}: request {b} of length 0 must be zero"
            continue
        ref = orc.cha_attention(q[b:b + 1], kr[b][None], vr[b][None], mem[b:b + 1], reps[b:b + 1], scale, False)[0]
        allowed = decode_bounds(q[b], kr[b], vr[b], mem[b], reps[b], scale, io, fp8)
        allowed = allowed + HALF_STEP[io] * (np.abs(ref) + allowed) + 1e-37
        err = np.abs(got[b] - ref)
        assert np.isfinite(got[b]).all(), f"{what}: request {b} has values that are not finite"
        worst = (err / allowed).max()
        assert worst <= 1.0, f"{what}: request {b} of length {n}: error {err.max():.3g}, {worst:.2f} of what is allowed"
