"""Packed batches for the tests: the definitions of the serving step's calls in 64 bits, and error bounds from arithmetic."""
import math

import numpy as np
import torch

from paged_cases import TORCH, partition, tables
from paper_2403_08058_b200 import chai

DEV = "cuda"
U32 = 2.0 ** -24
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def i32(x):
    return torch.as_tensor(np.asarray(x, dtype=np.int32), device=DEV)


# ---- plans ------------------------------------------------------------------------------------------------------

def plan(seq, new, table, free, count, n_tokens, page):
    """The definition, one request after the other.  Returns everything the call writes, and the status."""
    table, free = table.copy(), free.copy()
    B, max_pages = table.shape
    n_pages = len(free)
    status = chai.CHAI_OK
    full = bad = False
    if not 0 <= count <= n_pages:
        bad, count = True, min(max(count, 0), n_pages)
    cap = max_pages * page
    for b in range(B):
        if new[b] >= 0:
            continue
        if not 0 <= seq[b] <= cap:
            full = True
            continue
        mine = table[b, : -(-int(seq[b]) // page)]
        if ((mine < 0) | (mine >= n_pages)).any():
            bad = True
            continue
        for p in mine:
            if count < n_pages:
                free[count] = p
                count += 1
            else:
                bad = True
    kv, start, request, positions, slots = np.zeros(B, int), [0], [], [], []
    need_sum = want_sum = 0
    top = count
    for b in range(B):
        s, n = int(seq[b]), int(new[b])
        got = 0
        if n >= 0:
            if 0 <= s <= cap and n <= cap - s:
                held = -(-s // page)
                need = -(-(s + n) // page) - held
                need_sum += need
                want_sum += n
                if (need == 0 or need_sum <= top) and (n == 0 or want_sum <= n_tokens):
                    got = n
                    for i in range(held, held + need):
                        count -= 1
                        table[b, i] = free[count]
                else:
                    full = True
            else:
                full = True
            kv[b] = s + got
        for t in range(got):
            pos = s + t
            pg = int(table[b, pos // page])
            good = 0 <= pg < n_pages
            bad |= not good
            request.append(b)
            positions.append(pos)
            slots.append(pg * page + pos % page if good else -1)
        start.append(start[-1] + got)
    pad = n_tokens - start[-1]
    status = chai.CHAI_ERR_BAD_PAGE if bad else chai.CHAI_ERR_CACHE_FULL if full else chai.CHAI_OK
    return dict(block_table=table, free_pages=free, free_count=np.array([count]), kv_lens=kv, token_start=np.array(start),
                token_request=np.array(request + [-1] * pad), positions=np.array(positions + [0] * pad),
                slots=np.array(slots + [-1] * pad), status=status)


def pool_state(seq, page, n_pages, max_pages, seed):
    """Lists that hold what the requests have, and the stack of the other pages."""
    order = np.random.default_rng(seed).permutation(n_pages).astype(np.int32)
    table = np.full((len(seq), max_pages), -1, np.int32)
    at = 0
    for b, s in enumerate(seq):
        h = -(-max(int(s), 0) // page)
        table[b, :h] = order[at:at + h]
        at += h
    free = np.full(n_pages, -5, np.int32)
    free[: n_pages - at] = order[at:]
    return table, free, n_pages - at


# ---- rotary positions -------------------------------------------------------------------------------------------

def rotate(x, positions, turns, magnitude, interleaved):
    """x [..., D] (any type) at positions broadcastable to [...]: in 64 bits, and the largest |error| of the fp32 arithmetic.

    Cosine and sine are off by at most 4 u: the angle's remainder is rounded to 2^-26 of a turn at most (1.6 u), sincospi is
    good to 1.5 u of 1, the product with the magnitude to 1 u (all u = 2^-24); a product each and their sum add 2 u: 6 u
    (|x1| + |x2|) magnitude together."""
    x = x.double()
    rot = 2 * turns.numel()
    angle = torch.remainder(positions.double()[..., None] * turns.double(), 1.0) * (2 * math.pi)
    c, s = angle.cos() * magnitude, angle.sin() * magnitude
    y, err = x.clone(), torch.zeros_like(x)
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * c - b * s, b * c + a * s
        err[..., 0:rot:2] = err[..., 1:rot:2] = 6 * U32 * magnitude * (a.abs() + b.abs())
    else:
        h = rot // 2
        a, b = x[..., :h], x[..., h:rot]
        y[..., :h], y[..., h:rot] = a * c - b * s, b * c + a * s
        err[..., :h] = err[..., h:rot] = 6 * U32 * magnitude * (a.abs() + b.abs())
    return y, err


# ---- attention --------------------------------------------------------------------------------------------------

def batch(cache, io, H, k, D, page, kv, new, seed, peaked=3.0, pad=0, scale_rows=True):
    """A pool with random rows (NaN in every row that no request has), a packed batch of queries behind it."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    B = len(kv)
    table, n_pages = tables(kv, page, seed)
    mem, reps = partition(B, H, k, seed)
    n_tokens = sum(new) + pad
    c = dict(cache=cache, io=io, B=B, H=H, k=k, D=D, page=page, kv=list(kv), new=list(new), scale=1.0 / math.sqrt(D),
             n_pages=n_pages, n_tokens=n_tokens, mem=mem, reps_np=reps, table=i32(table), kv_lens=i32(kv),
             token_start=i32(np.concatenate([[0], np.cumsum(new)])), membership=i32(mem), reps=i32(reps))
    for name, planes in (("k", k), ("v", H)):
        x = torch.randn(n_pages, planes, page, D, generator=g, device=DEV) * 0.5
        there = torch.zeros(n_pages, page, dtype=torch.bool, device=DEV)
        for b, n in enumerate(kv):
            t = torch.arange(n, device=DEV)
            there[c["table"][b].long()[t // page], t % page] = True
        if cache == "e4m3":
            e = torch.randint(-9, -2, (n_pages, planes, page), generator=g, device=DEV)
            scales = torch.exp2(e.float())
            q8 = (x * 100).to(torch.float8_e4m3fn).view(torch.uint8)
            q8[~there[:, None].expand(-1, planes, -1)] = 0x7F
            scales[~there[:, None].expand(-1, planes, -1)] = math.nan
            c[name + "_pages"], c[name + "_scales"] = q8, scales
        else:
            x[~there[:, None, :, None].expand_as(x)] = math.nan
            c[name + "_pages"] = x.to(TORCH[cache])
    q = torch.randn(n_tokens, H, D, generator=g, device=DEV) * (0.5 * peaked)
    if pad:
        q[sum(new):] = math.nan
    c["q"] = q.to(TORCH[io])
    return c


def pages_of(c):
    return (c["k_pages"], c["v_pages"]) + ((c["k_scales"], c["v_scales"]) if c["cache"] == "e4m3" else ())


def attend(c, causal=True, **kw):
    fn = chai.chai_prefill_attention_paged_fp8 if c["cache"] == "e4m3" else chai.chai_prefill_attention_paged
    return fn(c["q"], *pages_of(c), c["membership"], c["reps"], c["table"], c["kv_lens"], c["token_start"], c["scale"],
              causal=causal, **kw)


def rows(c, name, b):
    n = c["kv"][b]
    at = c["table"][b, : -(-n // c["page"])].long()
    x = c[name + "_pages"][at]
    x = x.view(torch.float8_e4m3fn).double() * c[name + "_scales"][at].double()[..., None] if c["cache"] == "e4m3" else x.double()
    return x.transpose(0, 1).flatten(1, 2)[:, :n]


def check(c, got, causal=True, what=""):
    """got [n_tokens,H,D] against the definition in 64 bits, element by element.

    Bounds: a score is a sum of D products in fp32 (tensor cores: counted at 4 u a term), off by (D + 4) u S with S = scale
    sum |q k|; its exponential's argument is rounded too, (|s| + |max| + 40) u (the reference may be 2^32 away), and a
    probability is off by twice that, relative (numerator and sum); sums over n positions add 2 n u.  bf16: probabilities are
    rounded to bf16 before the product, 2^-8 each.  The result is rounded once to its type."""
    io, mem, reps, scale = c["io"], c["mem"], c["reps_np"], c["scale"]
    start = np.concatenate([[0], np.cumsum(c["new"])])
    u = U32 if io == "f32" else 4 * U32
    for b, (L, n) in enumerate(zip(c["kv"], c["new"])):
        if n == 0:
            continue
        mine = got[int(start[b]):int(start[b]) + n].double()
        if L == 0:
            assert not mine.any(), f"{what}: request {b} sees nothing"
            continue
        K, V = rows(c, "k", b), rows(c, "v", b)
        q = c["q"][int(start[b]):int(start[b]) + n].double()[:, reps[b].tolist()].transpose(0, 1)     # [k, n, D]
        see = torch.arange(L, device=DEV)[None] <= (L - n + torch.arange(n, device=DEV)[:, None] if causal else L + 0 * torch.arange(n, device=DEV)[:, None])
        s = (q @ K.transpose(1, 2) * scale).masked_fill(~see, -math.inf)
        size = (q.abs() @ K.abs().transpose(1, 2) * scale).masked_fill(~see, 0).amax(-1)            # [k, n]
        top = s.amax(-1)
        p = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top)[..., None])
        total = p.sum(-1)
        p = p / torch.where(total > 0, total, torch.ones_like(total))[..., None]
        largest = s.abs().masked_fill(~see, 0).amax(-1)
        rel = 2 * ((c["D"] + 4) * u * size + (2 * largest + 48) * U32) + (2 * L + 16) * u + (0 if io == "f32" else 2.0 ** -8)
        for cl in range(c["k"]):
            heads = np.nonzero(mem[b] == cl)[0].tolist()
            ref = (p[cl] @ V[heads]).transpose(0, 1)                                                # [n, heads, D]
            spread = (p[cl] @ V[heads].abs()).transpose(0, 1)
            allowed = rel[cl][:, None, None] * spread
            allowed = allowed + HALF_STEP[io] * (ref.abs() + allowed) + 1e-37
            err = (mine[:, heads] - ref).abs()
            assert torch.isfinite(mine[:, heads]).all(), f"{what}: request {b} cluster {cl} has values that are not finite"
            worst = float((err / allowed).max())
            assert worst <= 1.0, f"{what}: request {b} (length {L}, {n} tokens) cluster {cl}: error {float(err.max()):.3g}, {worst:.2f} of what is allowed"
