"""The paged cache on the GPU: append, read-back and decode against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import chai_oracle as orc
from paged_cases import TORCH, assert_decode, bits, partition, pool, tables
from paper_2403_08058_b200 import chai

pytestmark = pytest.mark.gpu
DEV = "cuda"


def make(cache, io, B, H, k, D, page, lens, seed, peaked=3.0, room=0):
    """A pool holding random rows, NaN everywhere else; dense float64 rows beside it."""
    g = torch.Generator().manual_seed(seed)
    table, n_pages = tables(lens, page, seed, room=room)
    mem, reps = partition(B, H, k, seed)
    c = dict(cache=cache, io=io, B=B, H=H, k=k, D=D, page=page, lens=list(lens), mem=mem, reps=reps, n_pages=n_pages,
             scale=1.0 / np.sqrt(D), table_np=table)
    for name, planes in (("k", k), ("v", H)):
        rows = [(torch.randn(planes, n, D, generator=g) * 0.5) for n in lens]
        if cache == "e4m3":
            # rows of very different sizes: the scales matter
            rows = [r * torch.exp2(torch.randint(-3, 4, r.shape[:2], generator=g).float())[..., None] for r in rows]
            quant = [orc.quantize_rows_fp8(r.to(torch.bfloat16).double().numpy()) for r in rows]
            c[name + "_pages"] = torch.from_numpy(pool([x[0] for x in quant], lens, table, n_pages, page, 0x7F)).to(DEV)
            c[name + "_scales"] = torch.from_numpy(pool([x[1].astype(np.float32) for x in quant], lens, table, n_pages,
                                                        page, np.nan)).to(DEV)
            c[name + "_rows"] = [orc.e4m3_values()[x[0]] * x[1][..., None] for x in quant]
        else:
            rows = [r.to(TORCH[cache]) for r in rows]
            c[name + "_rows"] = [r.double().numpy() for r in rows]
            c[name + "_pages"] = torch.from_numpy(pool([r.float().numpy() for r in rows], lens, table, n_pages, page,
                                                       np.nan)).to(TORCH[cache]).to(DEV)
    q = (torch.randn(B, H, D, generator=g) * 0.5 * peaked).to(TORCH[io])
    c["q_np"] = q.double().numpy()
    c["q"] = q.to(DEV)
    c["table"] = torch.from_numpy(table).to(DEV)
    c["seq"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    c["membership"] = torch.from_numpy(mem).to(DEV)
    c["reps_t"] = torch.from_numpy(reps).to(DEV)
    return c


def pages_of(c):
    return (c["k_pages"], c["v_pages"]) + ((c["k_scales"], c["v_scales"]) if c["cache"] == "e4m3" else ())


def decode(c, **kw):
    fn = chai.chai_decode_attention_paged_fp8 if c["cache"] == "e4m3" else chai.chai_decode_attention_paged
    return fn(c["q"], *pages_of(c), c["membership"], c["reps_t"], c["table"], c["seq"], c["scale"], **kw)


def check(c, got, what=""):
    assert_decode(got.double().cpu().numpy(), c["q_np"], c["k_rows"], c["v_rows"], c["mem"], c["reps"], c["lens"],
                  c["scale"], c["io"], c["cache"] == "e4m3", what)


# ---- decode -----------------------------------------------------------------------------------------------------

KINDS = [("f32", "f32"), ("bf16", "bf16"), ("e4m3", "bf16"), ("e4m3", "f32")]


@pytest.mark.parametrize("cache,io", KINDS)
@pytest.mark.parametrize("D,page", [(128, 16), (64, 24), (128, 8), (64, 64), (128, 40)])
def test_decode_matches_the_definition(cache, io, D, page, guard):
    lens = [page * 3, 0, 1, page - 1, page + 1, 333, 8]
    c = make(cache, io, len(lens), 12, 3, D, page, lens, seed=D + page)
    ws = chai.new_workspace(chai.chai_decode_paged_workspace_bytes(c["B"], c["H"], D), DEV)
    ws.fill_(0xFF)                                # a workspace may hold anything
    out = guard.empty_like(c["q"])
    decode(c, out=out, workspace=ws)
    check(c, out, f"{cache} {io} D {D} page {page}")
    assert chai.chai_device_status(ws) == chai.CHAI_OK


@pytest.mark.parametrize("cache,io", KINDS)
@pytest.mark.parametrize("B,H,k,page,lens", [
    (1, 1, 1, 16, [1]),
    (1, 1, 1, 16, [700]),
    (1, 32, 8, 16, [256]),
    (2, 7, 7, 32, [129, 2047]),
    (3, 40, 1, 128, [500, 513, 96]),
    (1, 72, 24, 32, [1500]),
    (4, 52, 13, 64, [1111, 64, 65, 900]),
    (1, 130, 130, 16, [77]),
    (1, 8, 2, 16, [20011]),
])
def test_decode_heads_and_lengths(cache, io, B, H, k, page, lens):
    c = make(cache, io, B, H, k, 128, page, lens, seed=H + page)
    check(c, decode(c), f"{cache} {io} B {B} H {H} k {k} page {page} lens {lens}")


@pytest.mark.parametrize("cache,io", KINDS)
@pytest.mark.parametrize("H,k,lens", [(52, 13, [3000, 1]), (100, 1, [2500]), (112, 112, [600, 700]), (113, 40, [900, 50]), (39, 1, [4000])])
def test_decode_heads_dealt_to_several_ctas(cache, io, H, k, lens):
    """One cluster, clusters of one head, lists that just fit a CTA and that do not; some heads unknown."""
    c = make(cache, io, len(lens), H, k, 64, 16, lens, seed=H)
    ws = chai.new_workspace(chai.chai_decode_paged_workspace_bytes(len(lens), H, 64), DEV)
    check(c, decode(c, workspace=ws), f"H {H} k {k}")
    assert chai.chai_device_status(ws) == chai.CHAI_OK
    lost = [h for h in range(H) if h not in c["reps"][0]][::3] or [int(c["reps"][0, 5])]
    c["membership"][0, lost] = -1
    got = decode(c, workspace=ws)
    assert chai.chai_device_status(ws) == chai.CHAI_ERR_BAD_MEMBERSHIP
    assert not got[0, lost].any()
    # the others as before: known heads against the definition
    kept = [h for h in range(H) if h not in lost]
    want = got.clone()
    c["membership"].copy_(torch.from_numpy(c["mem"]))
    want[0, lost] = decode(c, workspace=ws)[0, lost]
    check(c, want, f"H {H} k {k}, {len(kept)} known")


def test_the_largest_batch_goes_through_all_three():
    """65535 requests of no, one or two tokens: append, read-back and decode.  Rows of bf16, one head; the softmax of two
    scores in 64 bits.  Scores are below 64 * 9 / 8 and good to 66 * 2^-24 * 72 < 2^-11, a probability to twice that."""
    B, D, page = 65535, 64, 8
    g = torch.Generator().manual_seed(65)
    lens = torch.randint(0, 3, (B,), generator=g, dtype=torch.int32)
    x = {n: torch.randn(B, 1, 2, D, generator=g).clamp_(-3, 3).bfloat16() for n in ("k", "v")}
    q = torch.randn(B, 1, D, generator=g).clamp_(-3, 3).bfloat16()
    table = torch.randperm(B, generator=g).to(torch.int32)[:, None].to(DEV)
    kp, vp = (torch.full((B, 1, page, D), float("nan"), device=DEV, dtype=torch.bfloat16) for _ in range(2))
    seq, zero = torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros(B, 1, dtype=torch.int32, device=DEV)
    chai.chai_append_kv_paged(x["k"].to(DEV), x["v"].to(DEV), kp, vp, zero, table, seq, new_lens=lens.to(DEV))
    assert torch.equal(seq.cpu(), lens)
    held = (torch.arange(2)[None] < lens[:, None])[:, None, :, None]
    for got, name in zip(chai.chai_read_kv_paged(kp, vp, table, seq, T_out=2), ("k", "v")):
        assert torch.equal(got.cpu(), torch.where(held, x[name], torch.zeros(())))
    ws = chai.new_workspace(chai.chai_decode_paged_workspace_bytes(B, 1, D), DEV)
    out = chai.chai_decode_attention_paged(q.to(DEV), kp, vp, zero, zero, table, seq, 0.125, workspace=ws).double().cpu()
    assert chai.chai_device_status(ws) == chai.CHAI_OK
    s = 0.125 * (q.double()[:, :, None] * x["k"].double()).sum(-1, keepdim=True)
    p = torch.where(held, (s - torch.where(held, s, -torch.inf).amax(2, keepdim=True)).exp(), torch.zeros((), dtype=torch.float64))
    ref = (p * x["v"].double()).sum(2) / p.sum(2).clamp_min(1e-300)
    assert ((out - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -9 * 3).all()
    assert not out[lens == 0].any()


@pytest.mark.parametrize("cache,io", KINDS[1:3])
def test_decode_the_largest_page(cache, io):
    c = make(cache, io, 2, 2, 1, 64, 65536, [66001, 40], seed=64)
    check(c, decode(c), "page of 65536")


@pytest.mark.parametrize("cache,io", KINDS)
def test_decode_requests_that_share_pages(cache, io):
    """A prefix in pages that three requests have in their lists, and one page twice in one list."""
    lens, page = [150, 100, 64], 16
    c = make(cache, io, 3, 6, 2, 128, page, lens, seed=91)
    t = c["table"]
    t[0, 3] = t[0, 1]
    t[1, :4], t[2, :4] = t[0, :4], t[0, :4]
    for name in ("k_rows", "v_rows"):
        rows = c[name]
        rows[0][:, 48:64] = rows[0][:, 16:32]
        rows[1][:, :64] = rows[0][:, :64]
        rows[2][:, :64] = rows[0][:, :64]
    check(c, decode(c), f"{cache} {io}")


@pytest.mark.parametrize("cache,io", KINDS[1:3])
def test_decode_many_short_requests(cache, io):
    rng = np.random.default_rng(5)
    lens = [int(x) for x in rng.integers(0, 40, 400)]
    c = make(cache, io, 400, 6, 2, 64, 8, lens, seed=400)
    check(c, decode(c), "400 short requests")


@pytest.mark.parametrize("cache,io", KINDS[1:3])
def test_decode_many_heads(cache, io):
    c = make(cache, io, 2, 1024, 300, 64, 8, [19, 50], seed=3)
    check(c, decode(c), "1024 heads, 300 clusters")


@pytest.mark.parametrize("cache,io", KINDS)
def test_decode_peaked_and_flat_scores(cache, io):
    """Scores of +-100 and more, rising along the context, falling, and all equal: running maxima that move."""
    for kind in ("rising", "falling", "equal"):
        lens = [900, 257]
        c = make(cache, io, 2, 4, 2, 128, 16, lens, seed=11)
        for b, n in enumerate(lens):
            slope = {"rising": np.linspace(-1, 1, n), "falling": np.linspace(1, -1, n), "equal": np.ones(n)}[kind]
            keys = c["q_np"][b][c["reps"][b]][:, None] * slope[None, :, None] * 4.0     # [k, n, D]
            if cache == "e4m3":
                q8, s8 = orc.quantize_rows_fp8(keys)
                c["k_rows"][b] = orc.e4m3_values()[q8] * s8[..., None]
            else:
                keys = torch.from_numpy(keys).to(TORCH[cache])
                c["k_rows"][b] = keys.double().numpy()
            for t in range(n):
                at = (int(c["table_np"][b, t // 16]), slice(None), t % 16)
                if cache == "e4m3":
                    c["k_pages"][at] = torch.from_numpy(q8[:, t]).to(DEV)
                    c["k_scales"][at] = torch.from_numpy(s8[:, t].astype(np.float32)).to(DEV)
                else:
                    c["k_pages"][at] = keys[:, t].to(DEV)
        check(c, decode(c), f"{cache} {io} {kind}")


@pytest.mark.parametrize("cache,io", KINDS[:3])
def test_decode_pages_in_one_pool_and_far_apart(cache, io):
    """Keys and values side by side in one pool, with a gap between pages."""
    c = make(cache, io, 3, 6, 4, 128, 16, [100, 17, 48], seed=9)
    n, k, H, page, D = c["n_pages"], 4, 6, 16, 128
    both = torch.zeros((n, (k + H) * page * D + 64), device=DEV, dtype=c["k_pages"].dtype)
    kp = both[:, : k * page * D].view(n, k, page, D)
    vp = both[:, k * page * D: (k + H) * page * D].view(n, H, page, D)
    kp.copy_(c["k_pages"])
    vp.copy_(c["v_pages"])
    want = decode(c)
    c["k_pages"], c["v_pages"] = kp, vp
    got = decode(c)
    assert torch.equal(got.view(torch.uint8), want.view(torch.uint8))
    check(c, got)


def test_decode_offsets_beyond_32_bits():
    """Pages so far apart that element offsets pass 2^32."""
    page, D, k, H = 16, 128, 2, 3
    c = make("bf16", "bf16", 2, H, k, D, page, [90, 33], seed=7)
    n = c["n_pages"]
    apart = (1 << 32) // (n - 2) // 8 * 8 + 8
    big = torch.zeros(((n - 1) * apart + (k + H) * page * D,), device=DEV, dtype=torch.bfloat16)
    kp = big.as_strided((n, k, page, D), (apart, page * D, D, 1))
    vp = big.as_strided((n, H, page, D), (apart, page * D, D, 1), k * page * D)
    kp.copy_(c["k_pages"])
    vp.copy_(c["v_pages"])
    last, old = n - 1, int(c["table_np"][0, 1])    # request 0's second page becomes the farthest one
    other = c["table_np"] == last
    kp[last], vp[last] = kp[old].clone(), vp[old].clone()
    assert not other[:, :6].any()                  # (with this seed nobody else's rows lie there)
    c["table_np"][0, 1] = last
    c["table"] = torch.from_numpy(c["table_np"]).to(DEV)
    c["k_pages"], c["v_pages"] = kp, vp
    check(c, decode(c), "far pages")
    k_out, v_out = chai.chai_read_kv_paged(kp, vp, c["table"], c["seq"], T_out=90)
    assert np.array_equal(v_out[0].double().cpu().numpy(), c["v_rows"][0])
    k_new = torch.randn(2, H, 1, D, device=DEV).to(torch.bfloat16)
    c["seq"].fill_(page + 3)
    chai.chai_append_kv_paged(k_new, k_new, kp, vp, c["reps_t"], c["table"], c["seq"])
    assert torch.equal(vp[last, :, 3], k_new[0, :, 0])


def test_decode_bad_pages_and_unused_entries():
    lens = [40, 300, 0, 1]
    c = make("bf16", "bf16", 4, 8, 3, 128, 16, lens, seed=21)
    ws = chai.new_workspace(chai.chai_decode_paged_workspace_bytes(4, 8, 128), DEV)
    t = c["table"]
    t[0, 3:] = -7                                  # entries behind a request's length are not looked at
    t[2, :] = 1 << 30
    t[3, 1:] = c["n_pages"]
    check(c, decode(c, workspace=ws), "garbage behind the lengths")
    assert chai.chai_device_status(ws) == chai.CHAI_OK
    for bad in (-1, c["n_pages"], 1 << 30, -(1 << 31)):
        t[1, 7] = bad
        got = decode(c, workspace=ws)
        assert chai.chai_device_status(ws) == chai.CHAI_ERR_BAD_PAGE
        assert not got[1].any()
        c2 = dict(c, lens=[40, 0, 0, 1])           # the others are right, request 1 is zero
        check(c2, got, f"page {bad}")
    t[1, 7] = int(c["table_np"][1, 7])
    check(c, decode(c, workspace=ws), "good again")
    assert chai.chai_device_status(ws) == chai.CHAI_OK


def test_decode_bad_membership():
    c = make("bf16", "bf16", 2, 8, 3, 128, 16, [100, 50], seed=22)
    ws = chai.new_workspace(chai.chai_decode_paged_workspace_bytes(2, 8, 128), DEV)
    want = decode(c, workspace=ws)
    h = next(h for h in range(8) if h not in c["reps"][0])
    for bad in (-1, 3, 1 << 20):
        c["membership"][0, h] = bad
        got = decode(c, workspace=ws)
        assert chai.chai_device_status(ws) == chai.CHAI_ERR_BAD_MEMBERSHIP
        assert not got[0, h].any()
        keep = [x for x in range(8) if x != h]
        assert torch.equal(got[0, keep], want[0, keep]) and torch.equal(got[1], want[1])
    c["membership"][0, h] = int(c["mem"][0, h])
    r = int(c["reps"][0, 2])
    for bad in (-1, 8, -(1 << 31)):
        c["reps_t"][0, 2] = bad
        got = decode(c, workspace=ws)
        assert chai.chai_device_status(ws) == chai.CHAI_ERR_BAD_MEMBERSHIP
        out = [x for x in range(8) if c["mem"][0, x] == 2]
        assert not got[0, out].any() and torch.equal(got[1], want[1])
    c["reps_t"][0, 2] = r
    c["membership"].fill_(-1)                      # no head of any request is known
    assert not decode(c, workspace=ws).any()


def test_decode_unused_cluster_slots():
    """Slots behind k_eff (reps -1) have no keys: whatever their pages hold is not used."""
    c = make("bf16", "bf16", 2, 8, 5, 128, 16, [100, 50], seed=23)
    mem, reps = partition(2, 8, 3, 23)
    c["mem"], c["reps"] = mem, np.concatenate([reps, np.full((2, 2), -1, np.int32)], 1)
    c["membership"].copy_(torch.from_numpy(mem))
    c["reps_t"].copy_(torch.from_numpy(c["reps"]))
    c["k_pages"][:, 3:] = float("nan")
    got = decode(c)
    c["reps"] = reps
    c["k_rows"] = [r[:3] for r in c["k_rows"]]
    check(c, got)


def test_decode_infinite_and_nan_scores_follow_the_formula():
    """A key of -inf along a positive query leaves its token out; a NaN key makes its cluster NaN and no other."""
    c = make("f32", "f32", 1, 4, 2, 128, 16, [200], seed=24)
    c["q"].abs_()
    want = decode(c).clone()
    at = lambda t: (int(c["table_np"][0, t // 16]), 0, t % 16)
    for t in (0, 100, 199):
        c["k_pages"][at(t)] = float("-inf")
    got = decode(c)
    mine = torch.tensor([c["mem"][0, h] == 0 for h in range(4)])
    assert torch.isfinite(got).all() and torch.equal(got[0, ~mine], want[0, ~mine])
    keys = c["k_rows"][0].copy()
    keep = [t for t in range(200) if t not in (0, 100, 199)]
    ref = orc.cha_attention(c["q"].double().cpu().numpy(), keys[None][:, :, keep], c["v_rows"][0][None][:, :, keep], c["mem"],
                            c["reps"], c["scale"], False)
    assert np.abs(got.double().cpu().numpy() - ref)[0, mine.numpy()].max() < 1e-5    # (the other cluster's keys are as they were)
    c["k_pages"][at(7)] = float("nan")
    got = decode(c)
    assert torch.isnan(got[0, mine]).all() and torch.equal(got[0, ~mine], want[0, ~mine])


@pytest.mark.parametrize("cache,io", KINDS[1:3])
def test_decode_repeats_bit_for_bit_on_other_streams_and_in_graphs(cache, io):
    c = make(cache, io, 4, 8, 3, 128, 16, [1000, 3, 0, 700], seed=25)
    ws = chai.new_workspace(chai.chai_decode_paged_workspace_bytes(4, 8, 128), DEV)
    out = torch.empty_like(c["q"])
    want = decode(c).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            decode(c, out=out, workspace=ws)
    side.synchronize()
    assert torch.equal(out.view(torch.uint8), want.view(torch.uint8))
    # two graphs on one workspace, replayed in turn while lengths and queries change under them
    graphs, outs = [], []
    for _ in range(2):
        o, g = torch.empty_like(c["q"]), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            decode(c, out=o, workspace=ws)
        graphs.append(g)
        outs.append(o)
    for lens in ([1000, 3, 0, 700], [5, 0, 900, 1], [0, 0, 0, 0], [1000, 3, 0, 700]):
        c["lens"] = lens
        c["seq"].copy_(torch.tensor([min(n, m) for n, m in zip(lens, [1000, 3, 0, 700])], dtype=torch.int32))
        c["lens"] = [min(n, m) for n, m in zip(lens, [1000, 3, 0, 700])]
        sub = dict(c, k_rows=[r[:, :n] for r, n in zip(c["k_rows"], c["lens"])],
                   v_rows=[r[:, :n] for r, n in zip(c["v_rows"], c["lens"])])
        for g, o in zip(graphs, outs):
            o.fill_(7.0)
            g.replay()
        torch.cuda.synchronize()
        check(sub, outs[0], f"replay, lens {lens}")
        assert torch.equal(outs[0].view(torch.uint8), outs[1].view(torch.uint8))
        assert chai.chai_device_status(ws) == chai.CHAI_OK


def test_decode_into_its_own_queries_is_refused():
    c = make("bf16", "bf16", 2, 4, 2, 64, 16, [31, 20], seed=27)
    with pytest.raises(chai.ChaiError) as e:
        decode(c, out=c["q"])
    assert e.value.status == chai.CHAI_ERR_INVALID_ARG and "overlap" in str(e.value)


def test_two_calls_at_once_on_streams_and_workspaces_of_their_own():
    cases = [make("bf16", "bf16", 3, 16, 4, 128, 16, [3000, 500, 77], seed=71), make("e4m3", "bf16", 2, 24, 7, 128, 32, [900, 4000], seed=72)]
    want = [decode(c).clone() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [torch.empty_like(c["q"]) for c in cases]
    spaces = [chai.new_workspace(chai.chai_decode_paged_workspace_bytes(c["B"], c["H"], 128), DEV) for c in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s, o, ws in zip(cases, streams, outs, spaces):
            with torch.cuda.stream(s):
                decode(c, out=o, workspace=ws)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(outs, want))


@pytest.mark.parametrize("B", [33, 148, 149, 200])
def test_decode_batches_around_the_grid(B):
    """More requests than a warp has lanes, as many as the GPU has SMs, and more; some long enough for several pieces."""
    rng = np.random.default_rng(B)
    lens = [int(x) for x in rng.integers(0, 30, B)]
    lens[B // 2], lens[-1], lens[0] = 700, 900, 0
    c = make("bf16", "bf16", B, 5, 2, 64, 8, lens, seed=B)
    ws = chai.new_workspace(chai.chai_decode_paged_workspace_bytes(B, 5, 64), DEV)
    check(c, decode(c, workspace=ws), f"B {B}")
    assert chai.chai_device_status(ws) == chai.CHAI_OK
    c["table"][B // 2, 3] = -1
    got = decode(c, workspace=ws)
    assert chai.chai_device_status(ws) == chai.CHAI_ERR_BAD_PAGE and not got[B // 2].any()
    check(dict(c, lens=[0 if b == B // 2 else n for b, n in enumerate(lens)]), got, "the others")


def test_decode_lengths_are_clamped_to_the_table():
    c = make("bf16", "bf16", 2, 4, 2, 64, 16, [31, 20], seed=26)      # tables have one page to spare
    full = c["table_np"].shape[1] * 16
    c["seq"].copy_(torch.tensor([-5, 1 << 30], dtype=torch.int32))
    c["k_pages"].nan_to_num_(0.0)
    c["v_pages"].nan_to_num_(0.0)
    got = decode(c)
    assert not got[0].any()
    c["seq"].copy_(torch.tensor([0, full], dtype=torch.int32))
    assert torch.equal(got, decode(c))


# ---- append and read-back ---------------------------------------------------------------------------------------

def random_pool(n_pages, planes, page, D, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    if dtype == torch.uint8:
        return torch.randint(0, 256, (n_pages, planes, page, D), generator=g, dtype=torch.uint8).to(DEV)
    return torch.randn(n_pages, planes, page, D, generator=g).to(dtype).to(DEV)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("D,page,N", [(128, 16, 1), (64, 8, 1), (128, 24, 37), (64, 40, 300), (128, 16, 260)])
@pytest.mark.parametrize("advance", [True, False])
def test_append_bit_for_bit(io, fp8, D, page, N, advance):
    B, H, k = 4, 7, 3
    g = torch.Generator().manual_seed(D + page + N)
    lens = [0, 5, page, 2 * page - 1]
    new = [N, max(0, N - 1), N + 100, -3] if N > 1 else None          # clamped to [0, N]
    table, n_pages = tables(lens, page, N, room=N)
    _, reps = partition(B, H, k, N)
    reps = reps.copy()
    reps[1, 2] = -1                                                   # an unused slot: its row stays as it was
    k_new, v_new = ((torch.randn(B, H, N, D, generator=g) * 3).to(TORCH[io]) for _ in range(2))
    k_new[0, reps[0, 1], 0, :6] = torch.tensor([float("inf"), float("-inf"), float("nan"), 0.0, -0.0, 1e-30])
    v_new[0, 2, 0] = 0.0
    v_new[1, 1, 0] = float("inf")
    v_new[2, 1, 0] = 1e-38
    kp, vp = (random_pool(n_pages, p, page, D, torch.uint8 if fp8 else TORCH[io], 7 + p) for p in (k, H))
    ks, vs = (torch.rand(n_pages, p, page, device=DEV) for p in (k, H))
    before = [x.cpu().clone() for x in (kp, vp, ks, vs)]
    seq = torch.tensor(lens, dtype=torch.int32, device=DEV)
    new_t = None if new is None else torch.tensor(new, dtype=torch.int32, device=DEV)
    ws = chai.new_workspace(256, DEV)
    args = (k_new.to(DEV), v_new.to(DEV)) if N > 1 else (k_new[:, :, 0].contiguous().to(DEV), v_new[:, :, 0].contiguous().to(DEV))
    common = (torch.from_numpy(reps).to(DEV), torch.from_numpy(table).to(DEV), seq)
    kw = dict(new_lens=new_t, advance=advance, workspace=ws)
    if fp8:
        chai.chai_append_kv_paged_fp8(*args, kp, vp, ks, vs, *common, **kw)
    else:
        chai.chai_append_kv_paged(*args, kp, vp, *common, **kw)
    assert chai.chai_device_status(ws) == chai.CHAI_OK
    n = [N] * B if new is None else new
    if fp8:
        (k8, ksc), (v8, vsc) = (orc.quantize_rows_fp8(x.double().numpy()) for x in (k_new, v_new))
        wk, wv, wl = orc.append_kv_paged(k8, v8, before[0].numpy(), before[1].numpy(), reps, table, lens, n)
        wks, wvs, _ = orc.append_kv_paged(ksc.astype(np.float32), vsc.astype(np.float32), before[2].numpy(),
                                          before[3].numpy(), reps, table, lens, n)
        for got, want in ((kp, wk), (vp, wv)):
            got = got.cpu().numpy()
            # the sign of a NaN is not part of the contract
            assert ((got == want) | (((got & 0x7F) == 0x7F) & ((want & 0x7F) == 0x7F))).all()
        assert np.array_equal(ks.cpu().numpy(), wks) and np.array_equal(vs.cpu().numpy(), wvs)
    else:
        wk, wv, wl = orc.append_kv_paged(bits(k_new), bits(v_new), bits(before[0]), bits(before[1]), reps, table, lens, n)
        assert np.array_equal(bits(kp), wk) and np.array_equal(bits(vp), wv)
    assert seq.cpu().tolist() == (wl.tolist() if advance else lens)


@pytest.mark.parametrize("N", [1, 400])
def test_append_that_does_not_fit_or_meets_a_bad_page(N):
    B, H, k, D, page = 4, 16, 3, 128, 16
    g = torch.Generator().manual_seed(N)
    lens = [-1, 3, 20, 0]
    table, n_pages = tables([20] * 4, page, 5, room=N)
    cap = table.shape[1] * page
    lens[2] = cap - N + 1                                              # one position too far
    table = table.copy()
    table[3, 0] = n_pages                                              # a bad page
    _, reps = partition(B, H, k, N)
    k_new, v_new = (torch.randn(B, H, N, D, generator=g).to(torch.bfloat16) for _ in range(2))
    kp, vp = (random_pool(n_pages, p, page, D, torch.bfloat16, p) for p in (k, H))
    before = bits(kp).copy(), bits(vp).copy()
    seq = torch.tensor(lens, dtype=torch.int32, device=DEV)
    ws = chai.new_workspace(256, DEV)
    ws.fill_(0xFF)
    for only, status in ((None, None), ([0, 2], chai.CHAI_ERR_CACHE_FULL), ([3], chai.CHAI_ERR_BAD_PAGE), ([1], chai.CHAI_OK)):
        new = [N if only is None or b in only else 0 for b in range(B)]
        if only is not None and 0 not in only:
            seq[0] = 0                                                  # (a negative length is an error by itself)
        chai.chai_append_kv_paged(k_new.to(DEV), v_new.to(DEV), kp, vp, torch.from_numpy(reps).to(DEV),
                                  torch.from_numpy(table).to(DEV), seq, new_lens=torch.tensor(new, dtype=torch.int32, device=DEV),
                                  workspace=ws)
        got = chai.chai_device_status(ws)
        assert got != chai.CHAI_OK if only is None else got == status, (only, got)
        if only is None:
            wk, wv, wl = orc.append_kv_paged(bits(k_new), bits(v_new), before[0], before[1], reps, table, lens, new)
            assert np.array_equal(bits(kp), wk) and np.array_equal(bits(vp), wv) and seq.cpu().tolist() == wl.tolist()
            assert wl.tolist() == [-1, 3 + N, cap - N + 1, 0]
            seq.copy_(torch.tensor(lens, dtype=torch.int32))


@pytest.mark.parametrize("cache,io", KINDS)
@pytest.mark.parametrize("D,page", [(128, 16), (64, 24)])
def test_read_back(cache, io, D, page, guard):
    lens = [100, 0, 1, page, 333]
    c = make(cache, io, 5, 7, 3, D, page, lens, seed=31)
    fn = chai.chai_read_kv_paged_fp8 if cache == "e4m3" else chai.chai_read_kv_paged
    ws = chai.new_workspace(256, DEV)
    for T_out in (333, 90, 1):
        k_out, v_out = (guard.empty((5, p, T_out, D), TORCH[io]) for p in (3, 7))
        k_out.fill_(-7.0)
        v_out.fill_(-7.0)
        fn(*pages_of(c), c["table"], c["seq"], k_out=k_out, v_out=v_out, workspace=ws)
        assert chai.chai_device_status(ws) == chai.CHAI_OK
        for out, rows in ((k_out, c["k_rows"]), (v_out, c["v_rows"])):
            got = out.double().cpu().numpy()
            for b, n in enumerate(lens):
                m = min(n, T_out)
                # (every number here, e4m3 times a power of two included, is one of the output's type)
                assert np.array_equal(got[b, :, :m], rows[b][:, :m]) and (got[b, :, m:] == -7.0).all()
        alone = torch.full_like(v_out, -7.0)
        fn(*pages_of(c), c["table"], c["seq"], v_out=alone)
        assert torch.equal(alone, v_out)
        alone = torch.full_like(k_out, -7.0)
        fn(*pages_of(c), c["table"], c["seq"], k_out=alone)
        assert torch.equal(alone, k_out)
    c["table"][4, 2] = -1
    k_out, v_out = fn(*pages_of(c), c["table"], c["seq"], T_out=333, workspace=ws, **({"dtype": TORCH[io]} if cache == "e4m3" else {}))
    assert chai.chai_device_status(ws) == chai.CHAI_ERR_BAD_PAGE
    want = c["v_rows"][4].copy()
    want[:, 2 * page:3 * page] = 0.0
    assert np.array_equal(v_out[4].double().cpu().numpy(), want) and not v_out[1].any()


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_arrays_that_start_on_odd_16_byte_boundaries(io):
    B, H, k, D, page, N = 2, 5, 3, 64, 8, 45
    g = torch.Generator().manual_seed(61)
    step = 16 // torch.empty((), dtype=TORCH[io]).element_size()
    table, n_pages = tables([0, 0], page, 61, room=N)
    _, reps = partition(B, H, k, 61)
    reps_t, table_t = torch.from_numpy(reps).to(DEV), torch.from_numpy(table).to(DEV)

    def odd(x):
        flat = torch.zeros(x.numel() + step, dtype=x.dtype, device=DEV)
        view = flat[step:].view(x.shape)
        view.copy_(x)
        assert view.data_ptr() % 32 == 16
        return view

    k_new, v_new = (torch.randn(B, H, N, D, generator=g).to(TORCH[io]).to(DEV) for _ in range(2))
    results = []
    for at in (lambda x: x, odd):
        kp, vp = (torch.zeros(n_pages, p, page, D, device=DEV, dtype=torch.uint8) for p in (k, H))
        ks, vs = (torch.zeros(n_pages, p, page, device=DEV) for p in (k, H))
        for count in (N, 1):       # a prompt's rows and a decode step's
            seq = torch.zeros(B, dtype=torch.int32, device=DEV)
            chai.chai_append_kv_paged_fp8(at(k_new[:, :, :count].contiguous()), at(v_new[:, :, :count].contiguous()), kp, vp, ks,
                                          vs, reps_t, table_t, seq)
        seq.fill_(N)
        k_out, v_out = (at(torch.zeros(B, p, N, D, device=DEV, dtype=TORCH[io])) for p in (k, H))
        chai.chai_read_kv_paged_fp8(kp, vp, ks, vs, table_t, seq, k_out=k_out, v_out=v_out)
        results.append((kp, vp, ks, vs, k_out.clone(), v_out.clone()))
    assert all(torch.equal(x, y) for x, y in zip(*results))


def test_writing_what_was_read_back_gives_the_same_numbers():
    B, H, k, D, page, T = 2, 6, 4, 128, 16, 200
    c = make("e4m3", "bf16", B, H, k, D, page, [T, T], seed=41)
    _, v = chai.chai_read_kv_paged_fp8(*pages_of(c), c["table"], c["seq"], T_out=T)
    kp, vp = torch.zeros_like(c["k_pages"]), torch.zeros_like(c["v_pages"])
    ks, vs = torch.zeros_like(c["k_scales"]), torch.zeros_like(c["v_scales"])
    seq = torch.zeros_like(c["seq"])
    chai.chai_append_kv_paged_fp8(v, v, kp, vp, ks, vs, c["reps_t"], c["table"], seq)
    _, v2 = chai.chai_read_kv_paged_fp8(kp, vp, ks, vs, c["table"], seq, T_out=T)
    assert torch.equal(v, v2)


# ---- the operators together -------------------------------------------------------------------------------------

@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_a_request_from_prompt_to_answer(cache):
    """Features and membership from the prefix, the prompt's tokens into pages, then decode steps that append and attend,
    captured once and replayed; against the definition and (bf16) the dense path on the same tokens."""
    from paper_2403_08058_b200 import synth
    case = synth.prefill_case(seed=6, B=3, H=12, T=150, k=4, peaked=4.0)
    q, kf, v = (case[n].to(DEV) for n in ("q_full", "k_full", "v"))
    B, H, T, D = q.shape
    k, page, steps, scale = case["k"], 16, 5, case["scale"]
    lens = [150, 97, 5]
    mem, reps, _, _ = chai.chai_cluster_heads(chai.chai_prefix_features(q, kf, 5, scale), k, 20, 0)
    table_np, n_pages = tables(lens, page, 8, room=steps)
    table = torch.from_numpy(table_np).to(DEV)
    fp8 = cache == "e4m3"
    dt = torch.float8_e4m3fn if fp8 else torch.bfloat16
    kp = torch.zeros(n_pages, k, page, D, device=DEV, dtype=torch.uint8 if fp8 else dt)
    vp = torch.zeros(n_pages, H, page, D, device=DEV, dtype=kp.dtype)
    scales = tuple(torch.zeros(n_pages, p, page, device=DEV) for p in (k, H)) if fp8 else ()
    if fp8:
        kp, vp = kp.view(dt), vp.view(dt)
    put = chai.chai_append_kv_paged_fp8 if fp8 else chai.chai_append_kv_paged
    attend = chai.chai_decode_attention_paged_fp8 if fp8 else chai.chai_decode_attention_paged
    read = chai.chai_read_kv_paged_fp8 if fp8 else chai.chai_read_kv_paged
    seq = torch.zeros(B, dtype=torch.int32, device=DEV)
    put(kf, v, kp, vp, *scales, reps, table, seq, new_lens=torch.tensor(lens, dtype=torch.int32, device=DEV))
    assert seq.tolist() == lens
    ws = chai.new_workspace(chai.chai_decode_paged_workspace_bytes(B, H, D), DEV)
    k_new, v_new, q_new = (torch.zeros(B, H, D, device=DEV, dtype=torch.bfloat16) for _ in range(3))
    out = torch.empty_like(q_new)

    def step():
        put(k_new, v_new, kp, vp, *scales, reps, table, seq)
        attend(q_new, kp, vp, *scales, mem, reps, table, seq, scale, out=out, workspace=ws)

    g = torch.cuda.CUDAGraph()
    keep = seq.clone()
    step()
    with torch.cuda.graph(g):
        step()
    seq.copy_(keep)
    # the dense path beside it
    T_cap = T + steps
    dk, dv = chai.chai_compact_k_cache(kf, reps), v
    dense_k, dense_v = (torch.zeros(B, p, T_cap, D, device=DEV, dtype=torch.bfloat16) for p in (k, H))
    dense_k[:, :, :T], dense_v[:, :, :T] = dk, dv
    dense_seq = torch.tensor(lens, dtype=torch.int32, device=DEV)
    gen = torch.Generator().manual_seed(3)
    for i in range(steps):
        for x in (k_new, v_new, q_new):
            x.copy_((torch.randn(B, H, D, generator=gen) * (2.0 if x is q_new else 0.5)).to(torch.bfloat16))
        g.replay()
        chai.chai_append_kv(k_new, v_new, dense_k, dense_v, reps, dense_seq)
        n = [x + i + 1 for x in lens]
        assert seq.tolist() == n
        kr, vr = read(kp, vp, *scales, table, seq, T_out=T_cap)
        if not fp8:
            ref = chai.chai_decode_attention_ragged(q_new, dense_k, dense_v, mem, reps, dense_seq, scale, T_cap)
            assert (out.float() - ref.float()).abs().max() < 1e-2
            for b in range(B):
                assert torch.equal(kr[b, :, :n[b]], dense_k[b, :, :n[b]]) and torch.equal(vr[b, :, :n[b]], dense_v[b, :, :n[b]])
        assert_decode(out.double().cpu().numpy(), q_new.double().cpu().numpy(),
                      [kr[b, :, :n[b]].double().cpu().numpy() for b in range(B)],
                      [vr[b, :, :n[b]].double().cpu().numpy() for b in range(B)], mem.cpu().numpy(), reps.cpu().numpy(), n,
                      scale, "bf16", fp8, f"step {i}")
        assert chai.chai_device_status(ws) == chai.CHAI_OK


# ---- waits that run out (bounded, nothing faults: see test_gpu_failure_paths.py) ---------------------------------

@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_decode_wait_that_runs_out_is_reported_and_the_next_launch_is_clean(cache, guard):
    B, H, k, D, page, T = 2, 40, 8, 128, 16, 16000
    gen = torch.Generator(device=DEV).manual_seed(51)
    n_pages = B * T // page
    mem, reps = (torch.from_numpy(x).to(DEV) for x in partition(B, H, k, 51))
    table = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32).view(B, -1).contiguous()
    seq = torch.tensor([T, T - 1000], dtype=torch.int32, device=DEV)
    q = torch.randn(B, H, D, generator=gen, device=DEV).to(torch.bfloat16)
    if cache == "bf16":
        pages = [torch.randn(n_pages, p, page, D, generator=gen, device=DEV).to(torch.bfloat16) for p in (k, H)]
        scales, attend = [], chai.chai_decode_attention_paged
    else:
        pages = [torch.randint(0, 120, (n_pages, p, page, D), generator=gen, device=DEV, dtype=torch.uint8) for p in (k, H)]
        scales, attend = [torch.full((n_pages, p, page), 2.0 ** -8, device=DEV) for p in (k, H)], chai.chai_decode_attention_paged_fp8
    ws = chai.new_workspace(chai.chai_decode_paged_workspace_bytes(B, H, D), DEV)
    out = guard.empty_like(q)
    call = lambda: attend(q, *pages, *scales, mem, reps, table, seq, 0.01, out=out, workspace=ws)
    want = call().clone()
    assert chai.chai_device_status(ws) == chai.CHAI_OK and torch.isfinite(want).all()
    # every warp goes through many times what it holds in flight: somebody has to wait for more than a cycle
    chai.chai_set_decode_wait_limit_cycles(1)
    try:
        for _ in range(2):
            call()
            assert chai.chai_device_status(ws) == chai.CHAI_ERR_TIMEOUT
    finally:
        chai.chai_set_decode_wait_limit_cycles(0)
    for _ in range(2):
        out.zero_()
        call()
        assert chai.chai_device_status(ws) == chai.CHAI_OK and torch.equal(out, want)
