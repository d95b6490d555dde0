"""The paged serving operators of clustered-head attention as a user calls them, their plain forms, and their inputs.

Three operators on one pool of cache pages.  A page holds `page_size` consecutive positions of one request: the keys
of the layer's k representative heads (k_pages [n_pages,k,page_size,D]) and the values of all H heads
(v_pages [n_pages,H,page_size,D]); block_table [B,max_pages] names each request's pages in order.

  append   new tokens go to the positions seq_lens[b] ... of their request: the representatives' keys and every head's
           values, as they are or quantised to e4m3 with one power-of-two scale a row
  read     the cached rows of each request, page by page, into dense arrays (what the prefill call and a cache that is
           moved elsewhere take), e4m3 rows as the numbers they stand for
  decode   attention of one new token a request over its pages: one softmax a cluster, applied to each member's values

`own` selects the framework's calls; otherwise `run` computes the same with elementary torch operations in 32 bits.
"""
import math

import numpy as np
import torch

own = False

E4M3_MAX = 448.0
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2, "e4m3": 1}


# ---- cases ------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one request early in its answer, 32-bit caches: a call where latency is all that counts
        dict(name="decode f32 B1 T256", op="decode", cache="f32", io="f32", B=1, H=32, k=8, D=128, page=16, T=256, lens="full"),
        # a full batch of a 7B-shaped model at its full context, the ordinary call of a serving loop
        dict(name="decode bf16 B16 T2048", op="decode", cache="bf16", io="bf16", B=16, H=32, k=8, D=128, page=16, T=2048,
             lens="full"),
        # requests at different positions, a 33B-shaped model with uneven clusters, larger pages
        dict(name="decode bf16 B8 T4096 ragged", op="decode", cache="bf16", io="bf16", B=8, H=52, k=13, D=128, page=64,
             T=4096, lens="ragged"),
        # one very long document
        dict(name="decode bf16 B1 T131072", op="decode", cache="bf16", io="bf16", B=1, H=32, k=8, D=128, page=128, T=131072,
             lens="full"),
        # small heads, few of them, pages of an odd count of rows, a request without tokens and one with a single token
        dict(name="decode bf16 B5 T700 D64", op="decode", cache="bf16", io="bf16", B=5, H=12, k=3, D=64, page=24, T=700,
             lens="edges"),
        # the 7B-shaped batch on a one-byte cache, every head its own cluster
        dict(name="decode e4m3 B16 T2048 k32", op="decode", cache="e4m3", io="bf16", B=16, H=32, k=32, D=128, page=16, T=2048,
             lens="full"),
        # a 66B-shaped model, one-byte cache, requests at different positions
        dict(name="decode e4m3 B4 T2048 ragged", op="decode", cache="e4m3", io="bf16", B=4, H=72, k=24, D=128, page=32,
             T=2048, lens="ragged"),
        # the token of one decode step enters the cache: once a layer and step, so latency counts
        dict(name="append bf16 B16 N1", op="append", cache="bf16", io="bf16", B=16, H=32, k=8, D=128, page=16, T=2048, N=1,
             lens="ragged"),
        # whole prompts enter the cache after membership is fixed (the compaction happens on the way in)
        dict(name="append bf16 B4 N2048", op="append", cache="bf16", io="bf16", B=4, H=32, k=8, D=128, page=16, T=2048,
             N=2048, lens="empty"),
        # ragged prompts behind a five-token prefix into a one-byte cache
        dict(name="append e4m3 B4 N2043", op="append", cache="e4m3", io="bf16", B=4, H=52, k=13, D=128, page=32, T=2048,
             N=2043, lens="prefix"),
        # a one-byte cache leaves its pages for a dense bf16 cache
        dict(name="read e4m3 B16 T2048", op="read", cache="e4m3", io="bf16", B=16, H=32, k=8, D=128, page=16, T=2048,
             lens="ragged"),
        # a small 32-bit cache with odd pages and short rows leaves its pages
        dict(name="read f32 B3 T333 D64", op="read", cache="f32", io="f32", B=3, H=12, k=5, D=64, page=40, T=333, lens="edges"),
    ]


def draw(rng):
    op = rng.choice(["decode", "decode", "append", "read"])
    cache = rng.choice(["bf16", "bf16", "e4m3", "f32"])
    io = cache if cache != "e4m3" else rng.choice(["bf16", "bf16", "f32"])
    H = rng.choice([4, 7, 8, 12, 24, 32, 40, 52, 72])
    k = min(H, rng.choice([1, 2, 3, 5, 8, 13, 16, 24, 32, 52]))
    D = rng.choice([64, 128, 128])
    page = rng.choice([8, 16, 16, 24, 32, 40, 64, 128])
    lens = rng.choice(["full", "ragged", "ragged", "edges"])
    B = int(2 ** rng.uniform(0, 6.99))
    # at most half the values of the largest listed case of the operator, and no more bytes than any
    most = (131072 * 32 * 128) // 2 if op == "decode" else 16 * 2048 * 32 * 128
    longest = min(65536 if op == "decode" else 8192, most // (B * H * D), 640_000_000 // (B * (H + k) * D * BYTES[io]))
    case = dict(op=op, cache=cache, io=io, B=B, H=H, k=k, D=D, page=page, T=int(2 ** rng.uniform(0, math.log2(longest + 0.99))),
                lens=lens)
    if op == "append":
        case["N"] = rng.choice([1, int(2 ** rng.uniform(0, math.log2(case["T"] + 0.99)))])
        case["lens"] = "ragged" if case["N"] == 1 else rng.choice(["empty", "prefix"]) if case["T"] > 5 else "empty"
        if case["lens"] == "prefix":
            case["N"] = min(case["N"], case["T"] - 5)
    return case


def lengths(case):
    """Cached positions of each request before the call and, for append, the tokens that arrive: from the case alone."""
    B, T = case["B"], case["T"]
    rng = np.random.default_rng([B, T, case["H"], case["page"]])
    ragged = rng.integers(max(1, T // 4), T + 1, B)
    if case["op"] == "append":
        N = case["N"]
        if case["lens"] == "ragged":      # room for the tokens behind what is there
            return np.minimum(ragged, T) - 1 if N == 1 else np.minimum(ragged, T - N), np.full(B, N)
        new = rng.integers(max(1, N // 2), N + 1, B)
        new[0] = N
        if case["lens"] == "empty":
            return np.zeros(B, dtype=np.int64), np.full(B, N)
        return np.full(B, 5), new
    if case["lens"] == "full":
        return np.full(B, T), None
    if case["lens"] == "edges":
        ragged[0] = T
        if B > 1:
            ragged[1] = 0
        if B > 2:
            ragged[2] = 1
    return ragged, None


def work(case):
    B, H, k, D = case["B"], case["H"], case["k"], case["D"]
    lens, new = lengths(case)
    cached, io = BYTES[case["cache"]], BYTES[case["io"]]
    row = D * cached + (4 if case["cache"] == "e4m3" else 0)   # a cached row and its scale
    if case["op"] == "decode":
        rows = int(lens.sum()) * (k + H)
        pages = int(np.ceil(lens / case["page"]).sum())
        return {"bytes": rows * row + B * (k + H) * D * io + 4 * (B * (H + k + 1) + pages), "flops": 2 * D * rows}
    rows = int((new if case["op"] == "append" else lens).sum()) * (k + H)
    return {"bytes": rows * (row + D * io) + 4 * B * (k + 1), "flops": 0}


# ---- inputs -----------------------------------------------------------------------------------------------------

def clusters(B, H, k, seed):
    """A partition of the heads into k clusters for each request, one cluster larger than the others; clusters are
    numbered by their lowest member, which is the representative."""
    rng = np.random.default_rng([seed, H, k])
    mem, reps = np.empty((B, H), dtype=np.int32), np.empty((B, k), dtype=np.int32)
    for b in range(B):
        label = np.concatenate([np.arange(k), np.where(rng.random(H - k) < 0.25, 0, rng.integers(0, k, H - k))])
        label = label[rng.permutation(H)]
        _, first, inverse = np.unique(label, return_index=True, return_inverse=True)
        order = np.argsort(first)
        place = np.empty(k, dtype=np.int64)
        place[order] = np.arange(k)
        mem[b], reps[b] = place[inverse], first[order]
    return mem, reps


def row_scales(x):
    """One power of two a row: the smallest 2^e (e >= -126) with max|x| <= 448 * 2^e over the row's finite elements, 1
    for a row without any."""
    amax = torch.where(x.isfinite(), x.abs(), torch.zeros_like(x)).amax(-1)
    m, e = torch.frexp(amax)
    e = torch.where(m > 0.875, e - 8, e - 9).clamp_(min=-126)
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e), torch.ones_like(amax))


def to_e4m3(x, scales):
    return (x / scales[..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)


def prepare(case, seed):
    B, H, k, D, page, T = (case[n] for n in ("B", "H", "k", "D", "page", "T"))
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    io = DTYPES[case["io"]]
    sigma = 1.0 if case["io"] == "f32" else 0.5
    lens, new = lengths(case)
    mem, reps = clusters(B, H, k, seed)
    max_pages = -(-T // page) + 1
    n_pages = B * max_pages + 3
    order = torch.randperm(n_pages, generator=g, device=dev)[: B * max_pages]
    s = dict(op=case["op"], cache=case["cache"], io=io, page=page, T=T, scale=1.0 / math.sqrt(D),
             block_table=order.reshape(B, max_pages).to(torch.int32),
             seq_lens=torch.as_tensor(lens.astype(np.int32), device=dev),
             membership=torch.as_tensor(mem, device=dev), reps=torch.as_tensor(reps, device=dev))
    for name, planes in (("k", k), ("v", H)):
        shape = (n_pages, planes, page, D)
        if case["cache"] == "e4m3":
            q8 = torch.empty(shape, device=dev, dtype=torch.float8_e4m3fn)
            scales = torch.empty(shape[:-1], device=dev, dtype=torch.float32)
            for part in torch.arange(n_pages).split(max(1, (1 << 27) // (planes * page * D))):
                x = torch.randn((len(part),) + shape[1:], generator=g, device=dev) * sigma
                at = slice(int(part[0]), int(part[-1]) + 1)
                scales[at] = row_scales(x)
                q8[at] = to_e4m3(x, scales[at])
            s[name + "_pages"], s[name + "_scales"] = q8.view(torch.uint8), scales
        else:
            pages = torch.empty(shape, device=dev, dtype=io)
            for part in pages.split(max(1, (1 << 27) // (planes * page * D))):
                part.copy_(torch.randn(part.shape, generator=g, device=dev) * sigma)
            s[name + "_pages"] = pages
    if case["op"] == "decode":
        s["q"] = (torch.randn((B, H, D), generator=g, device=dev) * (4 * sigma)).to(io)
        s["out"] = torch.empty_like(s["q"])
        s["workspace"] = torch.empty(workspace_bytes(B, H, k, D), device=dev, dtype=torch.uint8)
    elif case["op"] == "append":
        for name in ("k_new", "v_new"):
            s[name] = (torch.randn((B, H, case["N"], D), generator=g, device=dev) * sigma).to(io)
        s["new_lens"] = None if (new == case["N"]).all() else torch.as_tensor(new.astype(np.int32), device=dev)
    else:
        s["k_out"] = torch.zeros((B, k, T, D), device=dev, dtype=io)
        s["v_out"] = torch.zeros((B, H, T, D), device=dev, dtype=io)
    return s


def workspace_bytes(B, H, k, D):
    """Room for the decode call's partial results, as the header states the bound: 64 KiB, and (160 + B) * H * (D + 8)
    32-bit words."""
    return (64 << 10) + 4 * (160 + B) * H * (D + 8)


# ---- the operators ----------------------------------------------------------------------------------------------

def run(state):
    if own:
        return framework(state)
    return {"decode": plain_decode, "append": plain_append, "read": plain_read}[state["op"]](state)


def framework(s):
    from paper_2403_08058_b200 import chai

    fp8 = s["cache"] == "e4m3"
    pages = (s["k_pages"], s["v_pages"]) + ((s["k_scales"], s["v_scales"]) if fp8 else ())
    if s["op"] == "decode":
        call = chai.chai_decode_attention_paged_fp8 if fp8 else chai.chai_decode_attention_paged
        return call(s["q"], *pages, s["membership"], s["reps"], s["block_table"], s["seq_lens"], s["scale"], out=s["out"],
                    workspace=s["workspace"])
    if s["op"] == "append":
        call = chai.chai_append_kv_paged_fp8 if fp8 else chai.chai_append_kv_paged
        call(s["k_new"], s["v_new"], *pages, s["reps"], s["block_table"], s["seq_lens"], new_lens=s["new_lens"], advance=False)
        return pool(s)
    call = chai.chai_read_kv_paged_fp8 if fp8 else chai.chai_read_kv_paged
    call(*pages, s["block_table"], s["seq_lens"], k_out=s["k_out"], v_out=s["v_out"])
    return s["k_out"], s["v_out"]


def pool(s):
    """The pages as they are after an append, e4m3 bytes as e4m3 numbers, with their scales."""
    if s["cache"] != "e4m3":
        return s["k_pages"], s["v_pages"]
    return s["k_pages"].view(torch.float8_e4m3fn), s["v_pages"].view(torch.float8_e4m3fn), s["k_scales"], s["v_scales"]


def dense(s, name):
    """The rows of every request in order, [B, planes, max_pages * page, D] in 32 bits."""
    table = s["block_table"].long()
    x = s[name + "_pages"][table]
    if s["cache"] == "e4m3":
        x = x.view(torch.float8_e4m3fn).float() * s[name + "_scales"][table][..., None]
    x = x.float().transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, x.shape[-1])


def plain_decode(s):
    q, mem, reps = s["q"].float(), s["membership"].long(), s["reps"].long()
    D = q.shape[-1]
    k = dense(s, "k")
    scores = torch.matmul(k, q.gather(1, reps[..., None].expand(-1, -1, D))[..., None])[..., 0] * s["scale"]
    here = (torch.arange(k.shape[2], device=q.device) < s["seq_lens"][:, None])[:, None]
    scores = torch.where(here, scores, torch.full_like(scores, -math.inf))
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    p = p.gather(1, mem[..., None].expand(-1, -1, p.shape[-1]))
    return torch.matmul(p[..., None, :], dense(s, "v"))[..., 0, :].to(s["io"])


def plain_append(s):
    B, H, N, D = s["k_new"].shape
    t = torch.arange(N, device=s["k_new"].device).expand(B, N)
    if s["new_lens"] is not None:       # a token that is not there: the first one once more
        t = torch.where(t < s["new_lens"][:, None], t, torch.zeros_like(t))
    pos = s["seq_lens"].long()[:, None] + t
    at, row = s["block_table"].long().gather(1, pos // s["page"]), pos % s["page"]
    reps = s["reps"].long()
    keys = s["k_new"].gather(1, reps[..., None, None].expand(-1, -1, N, D))
    for name, x in (("k", keys), ("v", s["v_new"])):
        x = x.gather(2, t[:, None, :, None].expand(-1, x.shape[1], -1, D)).transpose(1, 2)
        if s["cache"] == "e4m3":
            x = x.float()
            scales = row_scales(x)
            s[name + "_pages"][at, :, row] = to_e4m3(x, scales).view(torch.uint8)
            s[name + "_scales"][at, :, row] = scales
        else:
            s[name + "_pages"][at, :, row] = x
    return pool(s)


def plain_read(s):
    here = (torch.arange(s["T"], device=s["k_out"].device) < s["seq_lens"][:, None])[:, None, :, None]
    for name in ("k", "v"):
        out = s[name + "_out"]
        torch.where(here, dense(s, name)[:, :, : s["T"]].to(s["io"]), out, out=out)
    return s["k_out"], s["v_out"]


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def e4m3_numbers():
    """The 256 numbers of the format: sign, 4 exponent bits (bias 7, exponent 0 subnormal), 3 mantissa bits."""
    code = np.arange(256)
    e, m = (code >> 3) & 15, code & 7
    x = np.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    x[(code & 127) == 127] = np.nan
    return torch.as_tensor(np.where(code & 128, -x, x), device="cuda")


def nearest_e4m3(y):
    """Each number's nearest e4m3 number, ties to the even mantissa."""
    up = e4m3_numbers()[:127]
    size = y.abs().clamp(max=E4M3_MAX)
    hi = torch.searchsorted(up, size).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    d_hi, d_lo = up[hi] - size, size - up[lo]
    code = torch.where((d_lo < d_hi) | ((d_lo == d_hi) & (lo % 2 == 0)), lo, hi)
    return torch.copysign(up[code], y)


def rows_64(s, name, b, n):
    """Rows 0..n-1 of request b in 64 bits, [planes, n, D]."""
    pages = s["block_table"][b, : -(-n // s["page"])].long()
    x = s[name + "_pages"][pages]
    x = e4m3_numbers()[x.long()] * s[name + "_scales"][pages].double()[..., None] if s["cache"] == "e4m3" else x.double()
    return x.permute(1, 0, 2, 3).flatten(1, 2)[:, :n]


def exact(case, seed):
    s = prepare(case, seed)
    lens, new = lengths(case)
    B, H, k, D, page = (case[n] for n in ("B", "H", "k", "D", "page"))
    if case["op"] == "decode":
        out = torch.zeros((B, H, D), device="cuda", dtype=torch.float64)
        for b in range(B):
            n = int(lens[b])
            if n == 0:
                continue
            keys = rows_64(s, "k", b, n)
            q = s["q"][b].double()[s["reps"][b].long()]
            p = torch.softmax((keys * q[:, None]).sum(-1) * s["scale"], -1)
            del keys
            values = rows_64(s, "v", b, n)
            for h in range(H):
                out[b, h] = p[int(s["membership"][b, h])] @ values[h]
        return out
    if case["op"] == "read":
        outs = []
        for name, planes in (("k", k), ("v", H)):
            x = torch.zeros((B, planes, case["T"], D), device="cuda", dtype=torch.float64)
            for b in range(B):
                x[b, :, : int(lens[b])] = rows_64(s, name, b, int(lens[b]))
            outs.append(x)
        return tuple(outs)
    pages, scales = [], []
    for name, planes in (("k", k), ("v", H)):
        stored = s[name + "_pages"]
        stored = e4m3_numbers()[stored.long()] if s["cache"] == "e4m3" else stored.double()
        if s["cache"] == "e4m3":
            scale = s[name + "_scales"].double()
        for b in range(B):
            x = s[name + "_new"][b, :, : int(new[b])].double()
            x = x[s["reps"][b].long()] if name == "k" else x
            pos = int(lens[b]) + torch.arange(x.shape[1], device="cuda")
            at, row = s["block_table"][b].long()[pos // page], pos % page
            if s["cache"] == "e4m3":
                top = x.abs().amax(-1)
                f = torch.exp2(torch.ceil(torch.log2(top / E4M3_MAX)))
                f = torch.where(top > E4M3_MAX * f, 2 * f, torch.where(top <= E4M3_MAX / 2 * f, f / 2, f))
                f = torch.where(top > 0, f.clamp(min=2.0 ** -126), torch.ones_like(f))
                scale[at, :, row] = f.T
                x = nearest_e4m3(x / f[..., None])
            stored[at, :, row] = x.transpose(0, 1)
        pages.append(stored)
        if s["cache"] == "e4m3":
            scales.append(scale)
    return tuple(pages + scales)
