"""Calls of the packed step that a user may make and that the other tests do not: every e4m3 code and any scale, workspaces that
captured graphs share, replays with other lengths, two calls at once, pages that requests share, lists that are out of order."""
import math

import numpy as np
import pytest
import torch

from packed_cases import DEV, HALF_STEP, attend, batch, check, i32, rotate
from paged_cases import TORCH
from paper_2403_08058_b200 import chai

pytestmark = pytest.mark.gpu
KINDS = [("f32", "f32"), ("bf16", "bf16"), ("e4m3", "bf16"), ("e4m3", "f32")]


def workspace(*batches):
    return chai.new_workspace(max(chai.chai_prefill_paged_workspace_bytes(c["B"], c["H"], c["n_tokens"]) for c in batches), DEV)


def capture(fn):
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        fn()
    torch.cuda.current_stream().wait_stream(s)
    return g


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("low,high", [(-10, -8), (-60, -50), (7, 20)])
def test_every_code_and_any_scale(io, D, low, high):
    """Values: scales of any mantissa, tiny or above one; keys: theirs keep the scores small."""
    c = batch("e4m3", io, 6, 2, D, 16, [500, 64], [70, 3], seed=3)
    g = torch.Generator(device=DEV).manual_seed(D)
    codes = torch.tensor([x for x in range(256) if x not in (0x7F, 0xFF)], dtype=torch.uint8, device=DEV)
    for name, lo, hi in (("k", -10, -8), ("v", low, high)):
        x = c[name + "_pages"]
        order = torch.arange(x.numel(), device=DEV) * 89 % 254                      # (254 and 89 have no common factor)
        x.copy_(codes[order].view(x.shape))
        s = c[name + "_scales"]
        s.copy_(torch.exp2(lo + (hi - lo) * torch.rand(s.shape, generator=g, device=DEV)))
    check(c, attend(c), True, f"{io} {D}")


@pytest.mark.parametrize("cache,io", KINDS)
def test_rows_of_the_smallest_and_largest_codes(cache, io):
    """A cache of zeros, of the largest and of the smallest numbers of its type beside ordinary rows."""
    c = batch(cache, io, 4, 2, 128, 8, [300], [40], seed=8)
    at = c["table"][0].long()
    if cache == "e4m3":
        for i, code in enumerate((0x00, 0x80, 0x01, 0x81, 0x7E, 0xFE, 0x08, 0x07)):
            c["k_pages"][at[i], :, i] = code
            c["v_pages"][at[i], :, i] = code
    else:
        for i, x in enumerate((0.0, -0.0, 1e-38, -1e-38, 2.0, -2.0, 1e-30, 1e-20)):
            c["k_pages"][at[i], :, i] = x
            c["v_pages"][at[i], :, i] = x
    check(c, attend(c), True, cache)


@pytest.mark.parametrize("cache,io", KINDS)
@pytest.mark.parametrize("D", [64, 128])
def test_clusters_of_any_size(cache, io, D):
    """One to nine members: groups of one to 256 / D heads."""
    H, sizes = 45, range(1, 10)
    c = batch(cache, io, H, 9, D, 16, [140, 700], [33, 5], seed=4)
    mem = np.concatenate([[cl] * n for cl, n in enumerate(sizes)])
    for b in range(2):
        order = np.random.default_rng(b).permutation(H)
        c["mem"][b] = mem[order]
        c["reps_np"][b] = [int(np.nonzero(c["mem"][b] == cl)[0][-1]) for cl in range(9)]
    c["membership"], c["reps"] = i32(c["mem"]), i32(c["reps_np"])
    check(c, attend(c), True, f"{cache} {io} {D}")


@pytest.mark.parametrize("cache,io", KINDS)
def test_graphs_that_share_a_workspace(cache, io):
    c = [batch(cache, io, 8, 3, 64, 16, [900, 30], [4, 30], seed=1), batch(cache, io, 32, 8, 128, 32, [64, 1200, 5], [1, 200, 5], seed=2)]
    ws = workspace(*c)
    want = [attend(x) for x in c]
    out = [torch.empty_like(x) for x in want]
    graphs = [capture(lambda x=x, o=o: attend(x, out=o, workspace=ws)) for x, o in zip(c, out)]
    for i in (0, 1, 0, 0, 1, 1, 0):
        out[i].fill_(9.0)
        graphs[i].replay()
        assert chai.chai_device_status(ws) == chai.CHAI_OK
        assert torch.equal(out[i], want[i])
        assert torch.equal(attend(c[1 - i], workspace=ws), want[1 - i])          # an eager call between them


@pytest.mark.parametrize("cache,io", KINDS)
def test_a_replay_with_other_lengths(cache, io):
    """A graph captured for a full step takes any that fits; rows behind the last token stay as they are."""
    H, k, D, page = 6, 3, 64, 16
    c = batch(cache, io, H, k, D, page, [600, 333, 280], [200, 33, 80], seed=12)
    assert not torch.isnan(c["q"]).any()
    ws = workspace(c)
    out = torch.empty(c["n_tokens"], H, D, device=DEV, dtype=TORCH[io])
    graph = capture(lambda: attend(c, out=out, workspace=ws))
    for kv, new in (([600, 333, 280], [200, 33, 80]), ([600, 0, 1], [1, 0, 1]), ([1, 333, 64], [1, 300, 2]), ([0, 0, 0], [0, 0, 0]),
                    ([17, 16, 15], [17, 16, 15]), ([600, 333, 280], [200, 33, 80])):
        c["kv"], c["new"] = kv, new
        c["kv_lens"].copy_(i32(kv))
        c["token_start"].copy_(i32(np.concatenate([[0], np.cumsum(new)])))
        out.fill_(7.0)
        graph.replay()
        assert chai.chai_device_status(ws) == chai.CHAI_OK
        check(c, out, True, f"kv {kv} new {new}")
        assert bool((out[sum(new):] == 7.0).all())


@pytest.mark.parametrize("cache,io", KINDS)
def test_two_calls_at_once_and_other_streams(cache, io):
    c = [batch(cache, io, 12, 4, 128, 16, [1500, 200], [8, 200], seed=s) for s in (3, 4)]
    want = [attend(x) for x in c]
    ws, out = [workspace(x) for x in c], [torch.empty_like(w) for w in want]
    streams = [torch.cuda.Stream() for _ in c]
    torch.cuda.synchronize()
    for _ in range(10):
        for x, o, w, s in zip(c, out, ws, streams):
            with torch.cuda.stream(s):
                o.fill_(3.0)
                attend(x, out=o, workspace=w)
    torch.cuda.synchronize()
    for o, w, x in zip(out, want, ws):
        assert torch.equal(o, w) and chai.chai_device_status(x) == chai.CHAI_OK


@pytest.mark.parametrize("cache,io", KINDS[:3])
def test_pages_that_requests_share(cache, io):
    """A common beginning is cached once: the same pages stand in several lists, and one of them twice in a list."""
    c = batch(cache, io, 8, 3, 128, 16, [200, 200, 200], [3, 40, 200], seed=6)
    c["table"][1, :9] = c["table"][0, :9]
    c["table"][2, :4] = c["table"][0, :4]
    c["table"][2, 5] = c["table"][2, 4]
    check(c, attend(c), True, cache)


@pytest.mark.parametrize("cache,io", KINDS[:3])
def test_starts_and_lengths_out_of_range_are_clamped(cache, io):
    c = batch(cache, io, 4, 2, 64, 16, [90, 96], [10, 30], seed=5)
    c["table"] = c["table"][:, :6].contiguous()                # (no entry behind the longer one's last)
    want = attend(c)
    check(c, want)
    c["token_start"].copy_(i32([-5, 10, 1 << 30]))
    assert torch.equal(attend(c), want)
    c["kv_lens"].copy_(i32([90, 1 << 30]))                     # cut to what a list holds
    assert torch.equal(attend(c), want)
    out = torch.full_like(want, 2.0)
    c["kv_lens"].copy_(i32([-3, 96]))
    c["token_start"].copy_(i32([0, 10, 4]))                    # ends before it begins: no tokens
    attend(c, out=out)
    assert not out[:10].any() and bool((out[10:] == 2.0).all())


@pytest.mark.parametrize("cache,io", KINDS[:3])
def test_one_representative_for_two_clusters(cache, io):
    """A head represents the cluster that it is in: the heads of another that names it get zeros, and the status says so."""
    c = batch(cache, io, 8, 2, 64, 16, [100], [20], seed=15)
    ws = workspace(c)
    good = attend(c, workspace=ws)
    c["reps"][0, 1] = c["reps"][0, 0]
    out = attend(c, workspace=ws)
    assert chai.chai_device_status(ws) == chai.CHAI_ERR_BAD_MEMBERSHIP
    first = torch.as_tensor(c["mem"][0] == 0, device=DEV)
    assert torch.equal(out[:, first], good[:, first]) and not out[:, ~first].any()


@pytest.mark.parametrize("cache,io", KINDS[1:2])
def test_the_most_heads_and_clusters(cache, io):
    c = batch(cache, io, 1024, 319, 64, 8, [17, 0, 140], [3, 0, 9], seed=16)
    check(c, attend(c), True, "1024 heads, 319 clusters")


def test_many_more_requests_than_the_gpu_has_multiprocessors():
    rng = np.random.default_rng(8)
    new = [int(x) for x in rng.integers(0, 3, 5000)]
    kv = [n + int(x) for n, x in zip(new, rng.integers(0, 12, 5000))]
    c = batch("bf16", "bf16", 2, 1, 64, 8, kv, new, seed=71)
    check(c, attend(c), True, "5000 short requests")


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_rope_at_the_ends_of_the_range(io):
    turns, m = chai.chai_rope_frequencies(64)
    t = turns.to(DEV)
    pos = i32([[0, 1, -1, 2**31 - 1, -2**31, 131071, 1 << 30]])
    q = torch.randn(1, 3, 7, 128, device=DEV, generator=torch.Generator(device=DEV).manual_seed(2)).to(TORCH[io])
    got = chai.chai_rope(q, positions=pos, turns=t, magnitude=m)
    got = got[0] if isinstance(got, tuple) else got
    ref, err = rotate(q, pos[:, None].expand(-1, 3, -1), t, m, False)
    assert ((got.double() - ref).abs() <= err + HALF_STEP[io] * (ref.abs() + err)).all()
    assert torch.equal(got[:, :, 0], q[:, :, 0])


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_rope_of_rows_that_many_share(io):
    """Inputs with strides of 0 (one array for all requests, one key head for all): outputs have rows of their own."""
    turns, m = chai.chai_rope_frequencies(32, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(3)
    q = torch.randn(1, 4, 19, 64, device=DEV, generator=g).to(TORCH[io]).expand(3, -1, -1, -1)
    k = torch.randn(3, 1, 19, 64, device=DEV, generator=g).to(TORCH[io]).expand(-1, 2, -1, -1)
    pos = i32(np.random.default_rng(1).integers(0, 9000, (3, 19)))
    got = chai.chai_rope(q, k, pos, turns, m)
    want = chai.chai_rope(q.contiguous(), k.contiguous(), pos, turns, m)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    with pytest.raises(chai.ChaiError, match="output"):
        chai.chai_rope(q.contiguous(), None, pos, turns, m, q_out=torch.empty_like(q[:1]).expand(3, -1, -1, -1))


@pytest.mark.parametrize("cache,io", KINDS)
@pytest.mark.parametrize("n", [1, 3, 5, 130])
def test_append_rope_in_one_graph_with_other_slots(cache, io, n):
    """Slots and positions are read when the graph runs; what has none stays as it was, and a token may be anybody's."""
    H, k, D, page, n_pages, B = 5, 2, 64, 8, 80, 3
    g = torch.Generator(device=DEV).manual_seed(n)
    turns, m = chai.chai_rope_frequencies(32)
    turns = turns.to(DEV)
    q, kk, v = (torch.randn(n, H, D, generator=g, device=DEV).to(TORCH[io]) for _ in range(3))
    reps = i32([[0, 3], [4, 1], [2, 2]])
    request, pos, slots = i32(np.zeros(n)), i32(np.zeros(n)), torch.full((n,), -1, dtype=torch.int64, device=DEV)
    fp8 = cache == "e4m3"
    pages = [torch.zeros(n_pages, p, page, D, device=DEV, dtype=torch.uint8 if fp8 else TORCH[cache]) for p in (k, H)]
    scales = [torch.zeros(n_pages, p, page, device=DEV) for p in (k, H)] if fp8 else []
    fn = chai.chai_append_rope_paged_fp8 if fp8 else chai.chai_append_rope_paged
    out = torch.zeros_like(q)
    graph = capture(lambda: fn(q, kk, v, *pages, *scales, reps, request, pos, slots, turns, m, q_out=out))
    rng = np.random.default_rng(n)
    for _ in range(3):
        request.copy_(i32(rng.integers(0, B, n)))
        pos.copy_(i32(rng.integers(0, 5000, n)))
        where = rng.permutation(n_pages * page)[:n]
        where[rng.random(n) < 0.3] = -1
        slots.copy_(torch.as_tensor(where))
        for x in (*pages, *scales, out):
            x.zero_()
        graph.replay()
        live = torch.as_tensor(where >= 0, device=DEV)
        want_q, want_v = torch.zeros_like(out), torch.zeros_like(pages[1])
        eager = [torch.zeros_like(x) for x in (*pages, *scales)]
        some = live.nonzero()[:, 0]
        if len(some):
            q1 = fn(q[some].contiguous(), kk[some].contiguous(), v[some].contiguous(), *eager, reps, request[some].contiguous(),
                    pos[some].contiguous(), slots[some].contiguous(), turns, m, q_out=torch.zeros(len(some), H, D, device=DEV, dtype=TORCH[io]))
            want_q[some] = q1
        assert torch.equal(out, want_q)
        for x, y in zip((*pages, *scales), eager):
            assert torch.equal(x, y)
        if not fp8:
            want_v[slots[some] // page, :, slots[some] % page] = v[some]
            assert torch.equal(pages[1], want_v)
