"""The operators around paged caches that a serving step of many tokens needs, as a user calls them, their plain forms and inputs.

A step takes a packed batch: the new tokens of all requests one behind the other in [n_tokens, ...] arrays, request b's in
rows token_start[b] ... token_start[b+1]-1; rows behind the last request are padding.

  plan    pages for the new tokens: block tables grown from a stack of free pages (pages of ended requests given back), and for
          every token its request, its position and its slot (the row of the pool that it will be cached in)
  rope    queries and keys of whole prompts rotated by their positions: half or interleaved layout, part of the head, scaled
  enter   a packed batch's representatives' queries and keys rotated, keys and values cached in their slots, as they are or as
          e4m3 rows with one power-of-two scale each
  attend  clustered attention of a request's new tokens over its pages: causal behind what is cached, or unmasked over states
          of another length (an encoder's)

`own` selects the framework's calls; otherwise `run` computes the same with elementary torch operations in 32 bits, angles and
what decides about a scale in 64.
"""
import math

import numpy as np
import torch

own = False

E4M3_MAX = 448.0
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2, "e4m3": 1}
ROPE = dict(base=10000.0, kind="plain")
LONG = dict(base=10000.0, kind="ramp", factor=8.0, context=4096)


# ---- cases ------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one decode step of a full batch: a token each, now and then a new page; once a step, so latency is all that counts
        dict(name="plan B16 N1", op="plan", B=16, page=16, T=2048, N=1, mix="decode"),
        # a server's step: chunks of some prompts, single tokens of the others, requests that have ended
        dict(name="plan B300 mixed", op="plan", B=300, page=32, T=8192, N=512, mix="mixed"),
        # long documents arrive
        dict(name="plan B4 N131072", op="plan", B=4, page=16, T=131072, N=131072, mix="prompts"),
        # prompts of a 7B-shaped model before clustering: every head's queries and keys
        dict(name="rope bf16 B4 N2048", op="rope", io="bf16", B=4, H=32, Hk=32, D=128, N=2048, rot=128, layout="half", far=0,
             scaled=False, order="heads"),
        # 32-bit rows as a projection leaves them (tokens before heads), a part of a small head, far positions, scaled
        dict(name="rope f32 B3 N777 D64", op="rope", io="f32", B=3, H=12, Hk=5, D=64, N=777, rot=32, layout="pairs",
             far=100000, scaled=True, order="tokens"),
        # one decode step's tokens enter the cache: once a layer and step
        dict(name="enter bf16 16 tokens", op="enter", cache="bf16", io="bf16", B=16, H=32, k=8, D=128, page=16, T=2048, N=1,
             mix="decode", rot=128, layout="half", scaled=False),
        # ragged prompts enter a one-byte cache of a 33B-shaped model, scaled positions
        dict(name="enter e4m3 B4 N2043", op="enter", cache="e4m3", io="bf16", B=4, H=52, k=13, D=128, page=32, T=2048, N=2043,
             mix="prompts", rot=128, layout="half", scaled=True),
        # four guessed tokens a request are verified at once, 7B shape
        dict(name="attend bf16 B16 N4 T2048", op="attend", cache="bf16", io="bf16", B=16, H=32, k=8, D=128, page=16, T=2048,
             N=4, mix="verify", causal=True),
        # a chunk of a long document behind what is cached of it
        dict(name="attend bf16 B1 N2048 T32768", op="attend", cache="bf16", io="bf16", B=1, H=32, k=8, D=128, page=64, T=32768,
             N=2048, mix="chunk", causal=True),
        # a server's step: chunks of some prompts between single tokens of other requests, 33B shape with uneven clusters
        dict(name="attend bf16 B24 mixed", op="attend", cache="bf16", io="bf16", B=24, H=52, k=13, D=128, page=32, T=4096, N=700,
             mix="mixed", causal=True),
        # an encoder's states of another length, unmasked; small heads, odd pages, a request without any states
        dict(name="attend f32 B5 T700 D64", op="attend", cache="f32", io="f32", B=5, H=12, k=3, D=64, page=24, T=700, N=93,
             mix="cross", causal=False),
        # short chunks behind long one-byte caches of a 66B-shaped model
        dict(name="attend e4m3 B4 N64 T8192", op="attend", cache="e4m3", io="bf16", B=4, H=72, k=24, D=128, page=32, T=8192,
             N=64, mix="verify", causal=True),
    ]


def draw(rng):
    op = rng.choice(["plan", "rope", "enter", "enter", "attend", "attend", "attend"])

    def upto(most):
        return int(2 ** rng.uniform(0, math.log2(most + 0.99)))

    if op == "plan":
        page = rng.choice([8, 16, 16, 24, 32, 64, 128])
        B = upto(512)
        T = max(page, upto(min(131072, 524288 // B)))
        return dict(op=op, B=B, page=page, T=T, N=upto(T), mix=rng.choice(["decode", "mixed", "prompts"]))
    D = rng.choice([64, 128, 128])
    rot = rng.choice([D, D, D // 2, D // 4, D // 4 * 3])
    layout = rng.choice(["half", "half", "pairs"])
    H = rng.choice([4, 7, 8, 12, 24, 32, 40, 52, 72])
    k = min(H, rng.choice([1, 2, 3, 5, 8, 13, 16, 24, 32, 52]))
    cache = rng.choice(["bf16", "bf16", "e4m3", "f32"])
    if op == "rope":
        io = rng.choice(["bf16", "bf16", "f32"])
        tokens = upto(16384 * 64 * 128 // ((H + k) * D * BYTES[io]))
        B = min(tokens, upto(32))
        return dict(op=op, io=io, B=B, H=H, Hk=k, D=D, N=tokens // B, rot=rot, layout=layout, far=rng.choice([0, 4000, 1000000]),
                    scaled=rng.choice([False, True]), order=rng.choice(["heads", "tokens"]))
    io = cache if cache != "e4m3" else "bf16"
    page = rng.choice([8, 16, 16, 24, 32, 40, 64, 128])
    if op == "enter":
        B = upto(64)
        most = 8172 * 52 * 128 * 2 // (H * D * BYTES[io])
        T = upto(max(1, min(8192, most // B)))
        N = upto(T)
        return dict(op=op, cache=cache, io=io, B=B, H=H, k=k, D=D, page=page, T=T, N=N,
                    mix=rng.choice(["decode", "mixed", "prompts"]), rot=rot, layout=layout, scaled=rng.choice([False, True]))
    B = upto(64)
    mix = rng.choice(["verify", "verify", "chunk", "mixed", "cross"])
    # no more cached bytes than the largest caches listed, and no more products than the largest listed case
    T = upto(min(32768, max(64, 700_000_000 // (B * (H + k) * D * BYTES[io]))))
    products = 2048 * 32768 * 40 * 128 // (16 if cache == "f32" else 4 if cache == "e4m3" else 1)
    N = min(T, upto(max(1, min(2048, products // (B * T * (H + k) * D)))))
    return dict(op=op, cache=cache, io=io, B=B, H=H, k=k, D=D, page=page, T=T, N=N, mix=mix, causal=mix != "cross")


def lengths(case):
    """(cached positions before the step, new tokens) of each request, from the case alone; -1 new tokens: it has ended."""
    B, T, N, mix = case["B"], case["T"], case["N"], case["mix"]
    rng = np.random.default_rng([B, T, N, case["page"], len(mix)])
    some = rng.integers(1, N + 1, B)
    if mix == "chunk":
        new = np.full(B, N)
        return np.full(B, T - N), new
    if mix == "prompts":
        new = np.maximum(some, (N + 1) // 2)
        new[0] = N
        return np.minimum(rng.integers(0, 6, B), T - new), new
    if mix == "decode":
        return rng.integers(T // 4, T, B), np.ones(B, dtype=np.int64)
    if mix == "verify":
        new = np.full(B, N)
        return np.minimum(rng.integers(T // 4, T + 1, B), T - N), new
    if mix == "cross":                       # the states are there; nothing is added to them
        total = rng.integers(max(1, T // 4), T + 1, B)
        total[0], some[0] = T, N
        if B > 1:
            total[1] = 0
        if B > 2:
            total[2] = 1
        return total - some, some            # (attend: kv_lens = total; before the step is not looked at)
    chunk = rng.random(B) < 0.15             # mixed
    chunk[0] = True
    new = np.where(chunk, some, 1)
    new[0] = N
    before = np.minimum(rng.integers(0, T + 1, B), T - new)
    if case["op"] == "plan" and B > 8:
        ended = rng.random(B) < 0.05
        ended[0] = False
        new = np.where(ended, -1, new)
    return before, new


def room(case):
    """Rows of the packed arrays: the tokens, and some padding as a program with fixed sizes has it."""
    total = int(np.maximum(lengths(case)[1], 0).sum())
    return total + (0 if case["mix"] in ("decode", "verify", "chunk") else 7)


def work(case):
    if case["op"] == "rope":
        rows = case["B"] * case["N"] * (case["H"] + case["Hk"])
        return {"bytes": 2 * rows * case["D"] * BYTES[case["io"]] + 4 * case["B"] * case["N"] + 8 * case["rot"] // 2,
                "flops": 3 * rows * case["rot"]}
    before, new = lengths(case)
    B, page, got = case["B"], case["page"], np.maximum(new, 0)
    total = int(got.sum())
    if case["op"] == "plan":
        taken = int((-(-(before + got) // page) + (-before // page)).sum())
        given = int((-(-before // page))[new < 0].sum())
        return {"bytes": 8 * taken + 8 * given + 16 * B + 16 * room(case) + 8, "flops": 0}
    H, k, D = case["H"], case["k"], case["D"]
    io, row = BYTES[case["io"]], D * BYTES[case["cache"]] + (4 if case["cache"] == "e4m3" else 0)
    if case["op"] == "enter":
        return {"bytes": total * ((3 * k + H) * D * io + (k + H) * row + 16) + 4 * B * k, "flops": 6 * total * k * case["rot"]}
    kv = before + got
    if case["causal"]:
        pairs = sum(int(n) * int(l) - int(n) * (int(n) - 1) // 2 for n, l in zip(got, kv))
    else:
        pairs = sum(int(n) * int(l) for n, l in zip(got, kv))
    rows, pages = int(kv.sum()) * (k + H), int((-(-kv // page)).sum())
    return {"bytes": rows * row + total * (k + H) * D * io + 4 * (B * (H + k + 2) + pages), "flops": 2 * D * pairs * (k + H)}


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


def frequencies(case):
    """Turns a position of each frequency (64 bits) and the factor of the rotated numbers."""
    rot, p = case["rot"], LONG if case["scaled"] else ROPE
    turns = p["base"] ** (-2.0 * np.arange(rot // 2) / rot) / (2 * math.pi)
    if p["kind"] == "plain":
        return turns, 1.0

    def pair_that_turns(times):              # the pair whose angle turns so often over the context of the training
        return rot * math.log(p["context"] / (times * 2 * math.pi)) / (2 * math.log(p["base"]))

    low, high = max(math.floor(pair_that_turns(32.0)), 0), min(math.ceil(pair_that_turns(1.0)), rot - 1)
    keep = 1 - np.clip((np.arange(rot // 2) - low) / max(high - low, 0.001), 0, 1)
    return turns * keep + turns / p["factor"] * (1 - keep), 0.1 * math.log(p["factor"]) + 1


def row_scales(x):
    """One power of two a row: the smallest 2^e (e >= -126) with max|x| <= 448 * 2^e over the row's finite elements, 1
    for a row without any."""
    amax = torch.where(x.isfinite(), x.abs(), torch.zeros_like(x)).amax(-1)
    m, e = torch.frexp(amax)
    e = torch.where(m > 0.875, e - 8, e - 9).clamp_(min=-126)
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e), torch.ones_like(amax))


def to_e4m3(x, scales):
    return (x / scales[..., None]).clamp(-E4M3_MAX, E4M3_MAX).float().to(torch.float8_e4m3fn)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    s = dict(case)

    def ints(x, dtype=torch.int32):
        return torch.as_tensor(np.ascontiguousarray(x), device=dev).to(dtype)

    if case["op"] == "rope":
        B, N, D, io = case["B"], case["N"], case["D"], DTYPES[case["io"]]
        for name, heads in (("q", case["H"]), ("k", case["Hk"])):
            shape = (B, N, heads, D) if case["order"] == "tokens" else (B, heads, N, D)
            x = torch.randn(shape, generator=g, device=dev).to(io)
            s[name] = x.transpose(1, 2) if case["order"] == "tokens" else x
            s[name + "_out"] = torch.empty_like(x).transpose(1, 2) if case["order"] == "tokens" else torch.empty_like(x)
        begin = torch.randint(0, case["far"] + 1, (B, 1), generator=g, device=dev)
        s["positions"] = (begin + torch.arange(N, device=dev)).to(torch.int32)
        turns, s["magnitude"] = frequencies(case)
        s["turns"] = torch.as_tensor(turns, device=dev)
        return s
    B, page, T = case["B"], case["page"], case["T"]
    before, new = lengths(case)
    kv = before + np.maximum(new, 0)
    max_pages = -(-int(max(T, kv.max())) // page) + 1
    n_pages = B * max_pages + 3
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    s.update(before=before, new=new, n_pages=n_pages, n_tokens=room(case), kv=kv)
    start = np.concatenate([[0], np.cumsum(np.maximum(new, 0))])
    if case["op"] == "plan":
        held = -(-before // page)                       # pages that the requests have, in the order of the shuffle
        table = torch.full((B, max_pages), -1, device=dev, dtype=torch.int32)
        where = torch.arange(max_pages, device=dev)[None] < ints(held)[:, None]
        table[where] = order[: int(held.sum())]
        s["block_table"] = table
        s["free_pages"] = torch.cat([order[int(held.sum()):], torch.zeros(int(held.sum()), device=dev, dtype=torch.int32)])
        s["free_count"] = ints([n_pages - int(held.sum())])
        s["free_after"] = torch.zeros_like(s["free_count"])
        s["seq_lens"], s["new_lens"] = ints(before), ints(new)
        s["kv_lens"], s["token_start"] = ints(np.zeros(B)), ints(np.zeros(B + 1))
        s["token_request"], s["positions"] = ints(np.zeros(s["n_tokens"])), ints(np.zeros(s["n_tokens"]))
        s["slots"] = ints(np.zeros(s["n_tokens"]), torch.int64)
        s["workspace"] = torch.empty(512 + 4 * B, device=dev, dtype=torch.uint8)   # as the header states it
        return s
    H, k, D, n = case["H"], case["k"], case["D"], s["n_tokens"]
    io = DTYPES[case["io"]]
    sigma = 1.0 if case["io"] == "f32" else 0.5
    mem, reps = clusters(B, H, k, seed)
    s["membership"], s["reps"] = ints(mem), ints(reps)
    s["block_table"] = order[: B * max_pages].reshape(B, max_pages).contiguous()
    for name, planes in (("k", k), ("v", H)):
        shape = (n_pages, planes, page, D)
        fp8 = case["cache"] == "e4m3"
        pages = torch.empty(shape, device=dev, dtype=torch.float8_e4m3fn if fp8 else io)
        scales = torch.empty(shape[:-1], device=dev, dtype=torch.float32) if fp8 else None
        for part in torch.arange(n_pages).split(max(1, (1 << 27) // (planes * page * D))):
            at = slice(int(part[0]), int(part[-1]) + 1)
            x = torch.randn((len(part),) + shape[1:], generator=g, device=dev) * sigma
            if fp8:
                scales[at] = row_scales(x)
                pages[at] = to_e4m3(x, scales[at])
            else:
                pages[at] = x
        s[name + "_pages"] = pages.view(torch.uint8) if fp8 else pages
        if fp8:
            s[name + "_scales"] = scales
    if case["op"] == "enter":
        # one projection's output holds the three side by side, as a model leaves them
        qkv = (torch.randn((n, 3, H, D), generator=g, device=dev) * sigma).to(io)
        s["q"], s["k"], s["v"] = qkv[:, 0], qkv[:, 1], qkv[:, 2]
        s["q_out"] = torch.zeros((n, H, D), device=dev, dtype=io)
        request, pos = np.full(n, -1), np.zeros(n, dtype=np.int64)
        total = int(start[-1])
        request[:total] = np.repeat(np.arange(B), new)
        pos[:total] = np.arange(total) - np.repeat(start[:-1], new) + np.repeat(before, new)
        table = s["block_table"].cpu().numpy().astype(np.int64)
        slots = np.where(request >= 0, table[request, pos // page] * page + pos % page, -1)
        s["token_request"], s["positions"], s["slots"] = ints(request), ints(pos), ints(slots, torch.int64)
        turns, s["magnitude"] = frequencies(case)
        s["turns"] = torch.as_tensor(turns, device=dev)
        return s
    s["q"] = (torch.randn((n, H, D), generator=g, device=dev) * (4 * sigma)).to(io)
    s["out"] = torch.zeros_like(s["q"])
    s["workspace"] = torch.empty(workspace_bytes(B, H, n), device=dev, dtype=torch.uint8)
    s["kv_lens"], s["token_start"], s["scale"] = ints(kv), ints(start), 1.0 / math.sqrt(D)
    s["start"] = [int(x) for x in start]
    return s


def workspace_bytes(B, H, n_tokens):
    """Room for the plan and the partial results of an attend call, as the header states the bound."""
    return (1 << 20) + 64 * B + 36 * H * (B + n_tokens // 128 + 1) + 640000 * min(n_tokens, 128)


# ---- the operators ----------------------------------------------------------------------------------------------

def run(state):
    if own:
        return framework(state)
    return {"plan": plain_plan, "rope": plain_rope, "enter": plain_enter, "attend": plain_attend}[state["op"]](state)


def framework(s):
    from paper_2403_08058_b200 import chai

    if s["op"] == "plan":
        chai.chai_plan_paged(s["seq_lens"], s["new_lens"], s["block_table"], s["free_pages"], s["free_count"], s["n_tokens"],
                             s["page"], kv_lens=s["kv_lens"], free_count_out=s["free_after"], token_start=s["token_start"],
                             token_request=s["token_request"], positions=s["positions"], slots=s["slots"],
                             workspace=s["workspace"])
        return planned(s)
    if s["op"] == "rope":
        return chai.chai_rope(s["q"], s["k"], s["positions"], s["turns"], magnitude=s["magnitude"],
                              interleaved=s["layout"] == "pairs", q_out=s["q_out"], k_out=s["k_out"])
    fp8 = s["cache"] == "e4m3"
    pages = (s["k_pages"], s["v_pages"]) + ((s["k_scales"], s["v_scales"]) if fp8 else ())
    if s["op"] == "enter":
        call = chai.chai_append_rope_paged_fp8 if fp8 else chai.chai_append_rope_paged
        call(s["q"], s["k"], s["v"], *pages, s["reps"], s["token_request"], s["positions"], s["slots"], s["turns"],
             magnitude=s["magnitude"], interleaved=s["layout"] == "pairs", q_out=s["q_out"])
        return entered(s)
    call = chai.chai_prefill_attention_paged_fp8 if fp8 else chai.chai_prefill_attention_paged
    return call(s["q"], *pages, s["membership"], s["reps"], s["block_table"], s["kv_lens"], s["token_start"], s["scale"],
                causal=s["causal"], out=s["out"], workspace=s["workspace"])


def planned(s):
    return {n: s[n] for n in ("block_table", "free_pages", "free_after", "kv_lens", "token_start", "token_request", "positions",
                              "slots")}


def entered(s):
    """The pages as they are afterwards, e4m3 bytes as e4m3 numbers, with their scales, and the rotated queries."""
    if s["cache"] != "e4m3":
        return s["q_out"], s["k_pages"], s["v_pages"]
    return (s["q_out"], s["k_pages"].view(torch.float8_e4m3fn), s["v_pages"].view(torch.float8_e4m3fn), s["k_scales"],
            s["v_scales"])


def plain_plan(s):
    """All requests fit here: the pool and the lists are large enough, as a program sees to."""
    page, n, dev = s["page"], s["n_tokens"], s["seq_lens"].device
    before, want = s["seq_lens"].long(), s["new_lens"].long()
    table, free, count = s["block_table"], s["free_pages"], s["free_count"].long()
    col = torch.arange(table.shape[1], device=dev)[None]
    held = (before + page - 1) // page
    gone, new = want < 0, want.clamp(min=0)
    # pages of ended requests onto the stack, request by request
    back = torch.where(gone, held, torch.zeros_like(held))
    behind = back.cumsum(0)
    i = torch.arange(len(free), device=dev) - count
    b = torch.searchsorted(behind, i, right=True).clamp(max=len(before) - 1)
    page_of = table[b, (i - behind[b] + back[b]).clamp(0, table.shape[1] - 1)]
    torch.where((i >= 0) & (i < behind[-1]), page_of, free, out=free)
    top = count + behind[-1]
    # pages for the others from its top, in the order of the requests
    after = torch.where(gone, torch.zeros_like(before), before + new)
    need = torch.where(gone, torch.zeros_like(held), (after + page - 1) // page - held)
    off = need.cumsum(0) - need
    fresh = (col >= held[:, None]) & (col < (held + need)[:, None])
    page_of = free[(top - 1 - off[:, None] - (col - held[:, None])).clamp(0, len(free) - 1)]
    torch.where(fresh, page_of, table, out=table)
    s["free_after"].copy_(top - need.sum())
    s["kv_lens"].copy_(after)
    start = s["token_start"]
    start[0] = 0
    start[1:] = new.cumsum(0)
    t = torch.arange(n, device=dev)
    b = torch.searchsorted(start[1:].long(), t, right=True)
    real = b < len(before)
    b = b.clamp(max=len(before) - 1)
    pos = before[b] + t - start[b].long()
    slot = table[b, torch.where(real, pos // page, torch.zeros_like(pos))].long() * page + pos % page
    s["token_request"].copy_(torch.where(real, b, torch.full_like(b, -1)))
    s["positions"].copy_(torch.where(real, pos, torch.zeros_like(pos)))
    s["slots"].copy_(torch.where(real, slot, torch.full_like(slot, -1)))
    return planned(s)


def rotated(x, positions, turns, magnitude, layout, wide=False):
    """x [..., D] at positions [...]: rotated in 32 bits (wide: in 64), angles in 64; not rounded."""
    calc = torch.float64 if wide else torch.float32
    rot = 2 * turns.numel()
    angle = positions.double()[..., None] * turns
    angle = (angle - angle.round()) * (2 * math.pi)
    c, s = (angle.cos() * magnitude).to(calc), (angle.sin() * magnitude).to(calc)
    x = x.to(calc)
    part, rest = x[..., :rot], x[..., rot:]
    if layout == "half":
        a, b = part[..., : rot // 2], part[..., rot // 2:]
        return torch.cat([a * c - b * s, b * c + a * s, rest], -1)
    a, b = part[..., 0::2], part[..., 1::2]
    return torch.cat([torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2), rest], -1)


def plain_rope(s):
    pos = s["positions"][:, None]
    for name in ("q", "k"):
        s[name + "_out"].copy_(rotated(s[name], pos, s["turns"], s["magnitude"], s["layout"]))
    return s["q_out"], s["k_out"]


def plain_enter(s):
    here = torch.arange(s["n_tokens"], device=s["slots"].device)
    here = torch.where(s["slots"] >= 0, here, torch.zeros_like(here))      # padding: the first token once more
    at, row = (s["slots"] // s["page"])[here], (s["slots"] % s["page"])[here]
    rep = s["reps"].long()[s["token_request"].long()[here]]                    # [tokens, k]
    heads = rep[..., None].expand(-1, -1, s["D"])
    pos = s["positions"][here][:, None]
    fp8 = s["cache"] == "e4m3"
    q = rotated(s["q"][here].gather(1, heads), pos, s["turns"], s["magnitude"], s["layout"])
    k = rotated(s["k"][here].gather(1, heads), pos, s["turns"], s["magnitude"], s["layout"], wide=fp8)
    out = s["q_out"][here]
    s["q_out"][here] = out.scatter(1, heads, q.to(out.dtype))
    for name, x in (("k", k), ("v", s["v"][here])):
        if fp8:
            x = x if name == "k" else x.float()
            scales = row_scales(x)
            s[name + "_pages"][at, :, row] = to_e4m3(x, scales).view(torch.uint8)
            s[name + "_scales"][at, :, row] = scales.float()
        else:
            s[name + "_pages"][at, :, row] = x.to(DTYPES[s["io"]])
    return entered(s)


def rows(s, name, b, calc):
    """The cached rows of request b in order, [planes, length, D]."""
    n, page = int(s["kv"][b]), s["page"]
    at = s["block_table"][b, : -(-n // page)].long()
    x = s[name + "_pages"][at]
    if s["cache"] == "e4m3":
        x = x.view(torch.float8_e4m3fn).to(calc) * s[name + "_scales"][at].to(calc)[..., None]
    return x.to(calc).transpose(0, 1).flatten(1, 2)[:, :n]


def plain_attend(s):
    out, D = s["out"], s["D"]
    for b in range(s["B"]):
        n, length, first = int(s["new"][b]), int(s["kv"][b]), s["start"][b]
        k, v = rows(s, "k", b, torch.float32), rows(s, "v", b, torch.float32)
        q = s["q"][first:first + n].float().transpose(0, 1)[s["reps"][b].long()]          # [k, n, D]
        mem = s["membership"][b].long()
        t = torch.arange(length, device=q.device)
        step = max(1, (1 << 29) // (max(length, 1) * s["H"]))
        for i in range(0, n, step):
            scores = torch.matmul(q[:, i:i + step], k.transpose(1, 2)) * s["scale"]
            rows_here = scores.shape[1]
            if s["causal"]:
                last = length - n + i + torch.arange(rows_here, device=q.device)
                scores = torch.where(t[None, None] <= last[None, :, None], scores, torch.full_like(scores, -math.inf))
            if length == 0:
                out[first + i:first + i + rows_here] = 0
                continue
            top = scores.amax(-1, keepdim=True)
            p = torch.exp(scores - torch.where(top == -math.inf, torch.zeros_like(top), top))
            total = p.sum(-1, keepdim=True)
            p = p / torch.where(total > 0, total, torch.ones_like(total))
            out[first + i:first + i + rows_here] = torch.matmul(p[mem], v).transpose(0, 1).to(out.dtype)
    return out


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
    hi = torch.searchsorted(up, size.contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    d_hi, d_lo = up[hi] - size, size - up[lo]
    code = torch.where((d_lo < d_hi) | ((d_lo == d_hi) & (lo % 2 == 0)), lo, hi)
    return torch.copysign(up[code], y)


def exact(case, seed):
    return {"plan": exact_plan, "rope": exact_rope, "enter": exact_enter, "attend": exact_attend}[case["op"]](case, prepare(case, seed))


def exact_plan(case, s):
    """Page by page and token by token, as a host would do it."""
    table, free = s["block_table"].cpu().numpy(), s["free_pages"].cpu().numpy()
    count, page, B = int(s["free_count"]), case["page"], case["B"]
    for b in range(B):
        if s["new"][b] < 0:
            for i in range(-(-int(s["before"][b]) // page)):
                free[count] = table[b, i]
                count += 1
    kv, start, request, pos, slots = [], [0], [], [], []
    for b in range(B):
        n, at = int(s["new"][b]), int(s["before"][b])
        if n < 0:
            kv.append(0)
            start.append(start[-1])
            continue
        for i in range(-(-at // page), -(-(at + n) // page)):
            count -= 1
            table[b, i] = free[count]
        p = np.arange(at, at + n)
        request.append(np.full(n, b))
        pos.append(p)
        slots.append(table[b, p // page].astype(np.int64) * page + p % page)
        kv.append(at + n)
        start.append(start[-1] + n)
    pad = s["n_tokens"] - start[-1]
    request, pos, slots = (np.concatenate(x + [np.full(pad, fill)]) for x, fill in ((request, -1), (pos, 0), (slots, -1)))
    dev = s["seq_lens"].device
    return {name: torch.as_tensor(np.asarray(x), device=dev) for name, x in
            (("block_table", table), ("free_pages", free), ("free_after", [count]), ("kv_lens", kv), ("token_start", start),
             ("token_request", request), ("positions", pos), ("slots", slots))}


def turn_64(x, positions, case, s):
    """Rotation as complex numbers in 64 bits."""
    rot = case["rot"]
    z = torch.polar(torch.full((), s["magnitude"], dtype=torch.float64, device=x.device),
                    torch.remainder(positions.double()[..., None] * s["turns"], 1.0) * (2 * math.pi))
    x = x.double()
    y = x.clone()
    if case["layout"] == "half":
        w = torch.complex(x[..., : rot // 2], x[..., rot // 2:rot]) * z
        y[..., : rot // 2], y[..., rot // 2:rot] = w.real, w.imag
    else:
        w = torch.view_as_complex(x[..., :rot].reshape(x.shape[:-1] + (rot // 2, 2)).contiguous()) * z
        y[..., :rot] = torch.view_as_real(w).flatten(-2)
    return y


def exact_rope(case, s):
    return tuple(turn_64(s[n], s["positions"][:, None], case, s) for n in ("q", "k"))


def exact_enter(case, s):
    q_out = s["q_out"].double()
    stored, scales = {}, {}
    for name in ("k", "v"):
        pages = s[name + "_pages"]
        stored[name] = e4m3_numbers()[pages.long()] if case["cache"] == "e4m3" else pages.double()
        if case["cache"] == "e4m3":
            scales[name] = s[name + "_scales"].double()
    at = 0
    for b in range(case["B"]):
        n = int(s["new"][b])
        mine = slice(at, at + n)
        at += n
        pos = torch.arange(int(s["before"][b]), int(s["kv"][b]), device="cuda")
        page, row = s["block_table"][b].long()[pos // case["page"]], pos % case["page"]
        rep = s["reps"][b].long()
        q_out[mine, rep] = turn_64(s["q"][mine][:, rep], pos[:, None], case, s)
        for name, x in (("k", turn_64(s["k"][mine][:, rep], pos[:, None], case, s)), ("v", s["v"][mine].double())):
            if case["cache"] == "e4m3":
                top = x.abs().amax(-1)
                f = torch.exp2(torch.ceil(torch.log2(top / E4M3_MAX)))
                f = torch.where(top > E4M3_MAX * f, 2 * f, torch.where(top <= E4M3_MAX / 2 * f, f / 2, f))
                f = torch.where(top > 0, f.clamp(min=2.0 ** -126), torch.ones_like(f))
                scales[name][page, :, row] = f
                x = nearest_e4m3(x / f[..., None])
            stored[name][page, :, row] = x
    more = (scales["k"], scales["v"]) if scales else ()
    return (q_out, stored["k"], stored["v"]) + more


def exact_attend(case, s):
    out = torch.zeros(s["out"].shape, device="cuda", dtype=torch.float64)
    for b in range(case["B"]):
        n, length, first = int(s["new"][b]), int(s["kv"][b]), s["start"][b]
        if length == 0:
            continue
        k = rows(s, "k", b, torch.float64)
        mem = s["membership"][b].cpu().numpy()
        sees = torch.arange(length, device="cuda")[None] < (length if not case["causal"] else
                                                              length - n + 1 + torch.arange(n, device="cuda")[:, None])
        at = s["block_table"][b, : -(-length // case["page"])].long()
        for c in range(case["k"]):
            q = s["q"][first:first + n, int(s["reps"][b, c])].double()
            p = torch.softmax((q @ k[c].T * s["scale"]).masked_fill(~sees, -math.inf), -1)
            for h in np.nonzero(mem == c)[0]:
                v = s["v_pages"][at, int(h)]
                v = (e4m3_numbers()[v.long()] * s["v_scales"][at, int(h)].double()[..., None] if case["cache"] == "e4m3"
                     else v.double()).reshape(-1, case["D"])[:length]
                out[first:first + n, int(h)] = p @ v
    return out
