"""Paged caches at the edges of their contract: softmax rows that nothing is left of, row scales of every size, rounding of
what is read back, tables wider than the requests, appends of more than one pass."""
import numpy as np
import pytest
import torch

from oracle import chai_oracle as orc
from paged_cases import TORCH, bits, decode_bounds, partition, tables
from paper_2403_08058_b200 import chai
from test_gpu_paged import DEV, KINDS, check, decode, make, random_pool

pytestmark = pytest.mark.gpu


def status_workspace(c):
    return chai.new_workspace(chai.chai_decode_paged_workspace_bytes(c["B"], c["H"], c["D"]), DEV)


# ---- lengths that another stream writes --------------------------------------------------------------------------

@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("B", [5, 32, 33, 200])
def test_decode_ends_and_stays_in_bounds_while_another_stream_writes_the_lengths(cache, B):
    """Results are anyone's then, but every row that is read is one that the table names, every barrier is met by all, and
    the next call is right.  (All entries of the tables are pages of the pool, so any length may be read.)"""
    rng = np.random.default_rng(B)
    lens = [int(x) for x in rng.integers(0, 6000 // B, B)]
    lens[-1] = 900
    c = make(cache, "bf16", B, 12, 4, 64, 8, lens, seed=B)
    ws, out = status_workspace(c), torch.empty_like(c["q"])
    want = decode(c, workspace=ws).clone()
    right = c["seq"].clone()
    top = c["table"].shape[1] * 8
    other = [torch.from_numpy(rng.integers(-5, top + 1, B).astype(np.int32)).to(DEV) for _ in range(6)]
    other += [torch.zeros_like(right), torch.full_like(right, 1 << 30), right]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(150):
        with torch.cuda.stream(side):
            for j in range(4):
                c["seq"].copy_(other[(4 * i + j) % len(other)])
        decode(c, out=out, workspace=ws)
    torch.cuda.synchronize()
    assert chai.chai_device_status(ws) != chai.CHAI_ERR_TIMEOUT
    c["seq"].copy_(right)
    for _ in range(2):
        assert torch.equal(decode(c, workspace=ws).view(torch.uint8), want.view(torch.uint8))
        assert chai.chai_device_status(ws) == chai.CHAI_OK


@pytest.mark.parametrize("N", [1, 40])
@pytest.mark.parametrize("fp8", [False, True])
def test_append_ends_and_stays_in_bounds_while_another_stream_writes_the_lengths(fp8, N):
    """Tokens may go to any row that the tables name, and to no other page; the next call is right."""
    B, H, k, D, page = 40, 8, 3, 64, 8
    rng = np.random.default_rng(N)
    table_np, n_pages = tables([100] * B, page, N, extra_pages=30, room=N)
    table, top = torch.from_numpy(table_np).to(DEV), table_np.shape[1] * page
    _, reps = partition(B, H, k, N)
    reps = torch.from_numpy(reps).to(DEV)
    dt = torch.uint8 if fp8 else torch.bfloat16
    k_new, v_new = (torch.randn(B, H, N, D, device=DEV).to(torch.bfloat16) for _ in range(2))
    pages = [random_pool(n_pages, p, page, D, dt, p) for p in (k, H)]
    pages += [torch.rand(n_pages, p, page, device=DEV) for p in (k, H)] if fp8 else []
    before = [x.clone() for x in pages]
    put = chai.chai_append_kv_paged_fp8 if fp8 else chai.chai_append_kv_paged
    seq, count = torch.full((B,), 20, dtype=torch.int32, device=DEV), torch.full((B,), N, dtype=torch.int32, device=DEV)
    other = [torch.from_numpy(rng.integers(-5, top + 3, B).astype(np.int32)).to(DEV) for _ in range(5)] + [torch.full_like(seq, 1 << 30)]
    some = [torch.from_numpy(rng.integers(-3, N + 3, B).astype(np.int32)).to(DEV) for _ in range(5)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(100):
        with torch.cuda.stream(side):
            for j in range(3):
                seq.copy_(other[(3 * i + j) % len(other)])
                count.copy_(some[(3 * i + j) % len(some)])
        put(k_new, v_new, *pages, reps, table, seq, new_lens=count)
    torch.cuda.synchronize()
    unnamed = torch.ones(n_pages, dtype=torch.bool)
    unnamed[torch.from_numpy(table_np.ravel().astype(np.int64))] = False
    assert unnamed.sum() == 30
    for x, old in zip(pages, before):
        assert torch.equal(x[unnamed.to(DEV)].view(torch.uint8), old[unnamed.to(DEV)].view(torch.uint8))
    seq.fill_(20)
    for x, old in zip(pages, before):
        x.copy_(old)
    put(k_new, v_new, *pages, reps, table, seq)
    assert seq.tolist() == [20 + N] * B
    if not fp8:
        for b in (0, B - 1):
            assert torch.equal(pages[1][table[b, 20 // page].long(), :, 20 % page], v_new[b, :, 0])


# ---- softmax rows that nothing is left of ------------------------------------------------------------------------

@pytest.mark.parametrize("cache,io", KINDS)
@pytest.mark.parametrize("lens", [[1], [900, 1, 30], [2500], [7] * 200], ids=["one token", "joined and whole", "chunks", "many"])
def test_decode_a_cluster_whose_scores_are_all_minus_infinity_is_zero(cache, io, lens):
    """Keys of -inf along a positive query in every row of cluster 0 (e4m3: -1 with an infinite scale); one request in one
    piece and requests that are joined.  The other clusters keep their results bit for bit."""
    B, H, k, page = len(lens), 6, 2, 16
    c = make(cache, io, B, H, k, 64, page, lens, seed=101)
    c["q"].abs_().add_(0.125)
    ws = status_workspace(c)
    want = decode(c, workspace=ws).clone()
    assert torch.isfinite(want).all()
    if cache == "e4m3":
        c["k_pages"][:, 0] = 0xB8                  # -1
        c["k_scales"][:, 0] = float("inf")
    else:
        c["k_pages"][:, 0] = float("-inf")
    got = decode(c, workspace=ws)
    assert chai.chai_device_status(ws) == chai.CHAI_OK
    mine = (c["membership"] == 0)
    assert not got[mine].any() and not torch.isnan(got[mine]).any()
    assert torch.equal(got[~mine], want[~mine])
    # a row that is left counts alone; one that is NaN is not hidden
    last = lens[0] - 1
    at = (int(c["table_np"][0, last // page]), 0, last % page)
    if cache == "e4m3":
        c["k_pages"][at], c["k_scales"][at] = 0x30, 1.0
    else:
        c["k_pages"][at] = 0.5
    row = c["v_rows"][0][:, last]
    got = decode(c, workspace=ws)
    first = [h for h in range(H) if c["mem"][0, h] == 0]
    assert np.array_equal(got[0, first].double().cpu().numpy(), row[first])     # p = 1, values of the output's type
    if cache == "e4m3":
        c["k_scales"][at] = float("nan")
    else:
        c["k_pages"][at] = float("nan")
    got = decode(c, workspace=ws)
    assert torch.isnan(got[0, first]).all()


# ---- e4m3 rows with scales of every size -------------------------------------------------------------------------

U = 2.0 ** -24


def scaled_case(io, D, n, seed, scales, H=4, k=2, B=1, values=None, spread=1.0):
    """Requests of n tokens whose value rows have the given scales (scales(rng, n) -> [n] exponents) and full mantissas."""
    c = make("e4m3", io, B, H, k, D, 16, [n] * B, seed=seed, peaked=spread)
    rng = np.random.default_rng(seed)
    for b in range(B):
        s8 = np.exp2(np.asarray(scales(rng, n), dtype=np.float64))
        codes = rng.integers(1, 0x7F, (H, n, D)) | (rng.integers(0, 2, (H, n, D)) << 7)
        if values is not None:
            codes, s8 = values(rng, codes, s8)
        at = (torch.from_numpy(c["table_np"][b, np.arange(n) // 16].astype(np.int64)), torch.arange(n) % 16)
        c["v_pages"][at[0], :, at[1]] = torch.from_numpy(codes.astype(np.uint8)).transpose(0, 1).to(DEV)
        c["v_scales"][at[0], :, at[1]] = torch.from_numpy(s8.astype(np.float32))[:, None].expand(-1, H).to(DEV)
        c["v_rows"][b] = orc.e4m3_values()[codes] * s8[:, None]
        c.setdefault("v_codes", {})[b] = orc.e4m3_values()[codes]
        c.setdefault("v_size", {})[b] = s8
    return c


def check_tightly(c, what):
    """Bounds for n rows that leave no room for a floor set by the largest scale.

    Scores: fp32 sums of D products on the tensor cores, 4 u a term (u = 2^-24) of S = scale * sum|q k|; a query element is
    held to 2^-22 of itself or 2^-36 of the largest of its row.  Probabilities: twice the score's error (numerator
    and sum), and 2 |s| + 8 units u for an exponential and its argument, of which a row meets three (its own, from chunk
    to chunk, from piece to piece).  Probability times row scale: 2^-22 of
    itself, or 2^-43 of the largest such product of the head; sums over n rows 4 u a term.  The result is rounded once."""
    got = decode(c).double().cpu().numpy()
    D, scale = c["D"], c["scale"]
    for b, n in enumerate(c["lens"]):
        q, kr, vr = c["q_np"][b][c["reps"][b]], c["k_rows"][b], c["v_rows"][b]
        s = scale * np.einsum("cd,ctd->ct", q, kr)
        top = s.max(1, keepdims=True)
        p = np.exp(s - top)
        total = p.sum(1)
        size = scale * np.einsum("cd,ctd->ct", np.abs(q), np.abs(kr)).max(1)
        low = scale * np.abs(q).max(1) * np.abs(kr).sum(2).max(1)
        ds = (4 * (D + 4) * U + 2.0 ** -22) * size + 2.0 ** -36 * low
        rel = 2 * (ds + (6 * np.abs(s).max(1) + 24) * U) + (2 * n + 16) * 4 * U + 2.0 ** -22
        for h in range(c["H"]):
            cl = c["mem"][b, h]
            w = p[cl] / total[cl]
            ref = w @ vr[h]
            product = (w * c["v_size"][b]).max()
            allowed = rel[cl] * (w @ np.abs(vr[h])) + 2.0 ** -43 * product * np.abs(c["v_codes"][b][h]).sum(0) + n * 2.0 ** -140
            allowed = allowed + {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}[c["io"]] * (np.abs(ref) + allowed)
            err = np.abs(got[b, h] - ref)
            assert (err <= allowed).all(), f"{what}: head {h}: {(err / allowed).max():.3g} of what is allowed"


SCALES = {
    "all tiny": lambda r, n: r.integers(-30, -17, n),
    "all large": lambda r, n: r.integers(2, 30, n),
    "rising through the head": lambda r, n: np.linspace(-28, 9, n).astype(int),
    "falling through the head": lambda r, n: np.linspace(9, -28, n).astype(int),
    "one much larger row late": lambda r, n: np.where(np.arange(n) == n - 3, 24, r.integers(-8, -4, n)),
    "smallest scales": lambda r, n: r.integers(-112, -108, n),
    "largest scales": lambda r, n: r.integers(100, 110, n),
    "smallest, then largest": lambda r, n: np.where(np.arange(n) < n // 2, -120, 100),
    "ends of the range in turn": lambda r, n: np.where(np.arange(n) % 37 < 20, -100, 60),
}


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", list(SCALES))
@pytest.mark.parametrize("n,B", [(1, 1), (31, 1), (190, 1), (75, 160)], ids=["a token", "a tile", "pieces", "many requests"])
def test_decode_row_scales_of_every_size(io, D, kind, n, B):
    """Scales that start below 2^-16, pass 2 in the middle of a head, fall, and lie at the ends of the range; heads shared
    by warps (n = 75 in one piece of many requests), pieces that are joined, several chunks (below)."""
    check_tightly(scaled_case(io, D, n, 7 + n, SCALES[kind], B=B), f"{kind}, n {n}")


@pytest.mark.parametrize("kind", list(SCALES))
def test_decode_row_scales_in_several_chunks(kind):
    """150 requests of 600 tokens: a piece holds more than a chunk of 512, and sums go on from chunk to chunk."""
    check_tightly(scaled_case("f32", 64, 600, 3, SCALES[kind], B=150, H=2, k=1), kind)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("size", [-22, -25, -28])
def test_decode_a_row_of_zeros_among_small_ones(D, size):
    """Such a row's scale is 1, whatever the others' (values of about 1e-4, 1e-5 and 1e-6 here)."""
    def values(rng, codes, s8):
        codes[:, 5] = 0
        s8[5] = 1.0
        return codes, s8
    check_tightly(scaled_case("f32", D, 45, 12, lambda r, n: np.full(n, size), values=values, spread=2.0 ** -6), f"2^{size}")


@pytest.mark.parametrize("D", [64, 128])
def test_decode_a_large_row_that_the_softmax_leaves_out(D):
    """A row 2^30 larger than the others whose probability is below 2^-45 of theirs."""
    c = scaled_case("f32", D, 45, 13, lambda r, n: np.where(np.arange(n) == 9, 30, -4))
    key = -np.sign(c["q_np"][0][c["reps"][0]])                       # [k, D]: far below every other score
    q8, s8 = orc.quantize_rows_fp8(key)
    strength = 2.0 ** np.ceil(np.log2(40.0 / (c["scale"] * np.abs(c["q_np"][0][c["reps"][0]]).sum(1).min())))
    page, row = int(c["table_np"][0, 0]), 9
    c["k_pages"][page, :, row] = torch.from_numpy(q8).to(DEV)
    c["k_scales"][page, :, row] = torch.from_numpy((s8 * strength).astype(np.float32)).to(DEV)
    c["k_rows"][0][:, 9] = key * strength
    s = c["scale"] * np.einsum("cd,ctd->ct", c["q_np"][0][c["reps"][0]], c["k_rows"][0])
    assert (s[:, 9] < s.max(1) - 32).all()
    check_tightly(c, "a large row left out")


@pytest.mark.parametrize("D", [64, 128])
def test_decode_a_token_above_the_others_with_small_values(D):
    """A first token whose score lies 12 above the others' and whose values are near zero."""
    c = scaled_case("f32", D, 45, 14, lambda r, n: np.where(np.arange(n) == 0, -30, -15), spread=0.1)
    q = c["q_np"][0][c["reps"][0]]
    key = np.sign(q) * 2.0 ** np.round(np.log2(12.0 / (c["scale"] * np.abs(q).sum(1))))[:, None]
    q8, s8 = orc.quantize_rows_fp8(key)
    page = int(c["table_np"][0, 0])
    c["k_pages"][page, :, 0] = torch.from_numpy(q8).to(DEV)
    c["k_scales"][page, :, 0] = torch.from_numpy(s8.astype(np.float32)).to(DEV)
    c["k_rows"][0][:, 0] = key
    check_tightly(c, "a token above the others")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("exponent", [128, -130, -140])
def test_decode_queries_at_the_ends_of_the_range(D, exponent):
    """Queries near 2^128 and subnormal ones, with a scale that makes their scores ordinary."""
    c = scaled_case("f32", D, 45, 15, lambda r, n: np.full(n, -4))
    rng = np.random.default_rng(15)
    # whole numbers of nine bits: exact at every exponent here
    q = rng.integers(-511, 512, c["q_np"].shape) * 2.0 ** -9 * 2.0 ** (exponent if exponent > 0 else exponent + 9)
    c["q_np"] = q.astype(np.float32).astype(np.float64)
    c["q"] = torch.from_numpy(q.astype(np.float32)).to(DEV)
    c["scale"] = 2.0 ** -126 if exponent > 0 else 2.0 ** (-exponent - 14)
    if exponent > 0:                                   # (the least scale that is a normal number)
        c["k_scales"] *= 2.0 ** -8
        c["k_rows"][0] = c["k_rows"][0] * 2.0 ** -8
    check_tightly(c, f"2^{exponent}")


@pytest.mark.parametrize("D", [64, 128])
def test_decode_a_query_with_one_large_element(D):
    """Keys are zero where the query is large: the scores come from elements 2^-20 of its size."""
    c = scaled_case("f32", D, 45, 16, lambda r, n: np.full(n, -4))
    c["q_np"] = (c["q_np"] * 2.0 ** -20).astype(np.float32).astype(np.float64)
    c["q_np"][..., 3] = 1.0
    c["q"] = torch.from_numpy(c["q_np"].astype(np.float32)).to(DEV)
    c["k_pages"][..., 3] = 0
    c["k_rows"][0][..., 3] = 0.0
    c["scale"] = 2.0 ** 19 / np.sqrt(D)
    check_tightly(c, "one large element")


# ---- read-back ---------------------------------------------------------------------------------------------------

def nearest_bf16(x):
    """float64 -> the nearest bf16 number, ties to even, as float64 (normal range)."""
    m, e = np.frexp(x)
    return np.ldexp(np.rint(m * 256.0), e - 8)      # (rint: ties to even)


def test_read_back_is_rounded_once_with_any_scale():
    """Scales that are no powers of two: the 28-bit product goes to bf16 (or fp32) in one rounding.  Half the rows have a
    scale near (a tie of bf16) / (one of their numbers): fp32 rounds such products to the tie."""
    B, H, k, D, page, T = 1, 8, 8, 128, 16, 512
    rng = np.random.default_rng(77)
    c = make("e4m3", "bf16", B, H, k, D, page, [T], seed=77)
    codes = rng.integers(0, 0x7F, (H, T, D)) | (rng.integers(0, 2, (H, T, D)) << 7)
    numbers = orc.e4m3_values()[codes]
    # scales whose product with some code of the row is just beside a tie: (odd multiple of 2^-8 + 2^-25) / code
    s8 = (1 + rng.integers(0, 2 ** 23, (H, T)) * 2.0 ** -23).astype(np.float32)
    tie = (1 + (2 * rng.integers(0, 128, (H, T // 2)) + 1) * 2.0 ** -8)
    code = 1 + rng.integers(1, 8, (H, T // 2)) / 8.0
    near = (tie / code).astype(np.float32)
    near = np.where(near < 1, near * 2, near).astype(np.float32)
    s8[:, : T // 2] = near
    codes[:, : T // 2, :8] = 0x38 + np.arange(8)     # 1, 1.125 ... 1.875
    numbers = orc.e4m3_values()[codes]
    for dt in ("bf16", "f32"):
        exact = numbers * s8[..., None].astype(np.float64)
        want = nearest_bf16(exact) if dt == "bf16" else exact.astype(np.float32).astype(np.float64)
        if dt == "bf16":    # the oracle's second rounding would show
            assert (nearest_bf16(exact.astype(np.float32).astype(np.float64)) != want).sum() > 20
        at = (torch.from_numpy(c["table_np"][0, np.arange(T) // page].astype(np.int64)), torch.arange(T) % page)
        c["v_pages"][at[0], :, at[1]] = torch.from_numpy(codes.astype(np.uint8)).transpose(0, 1).to(DEV)
        c["v_scales"][at[0], :, at[1]] = torch.from_numpy(s8).T.contiguous().to(DEV)
        _, v = chai.chai_read_kv_paged_fp8(c["k_pages"], c["v_pages"], c["k_scales"], c["v_scales"], c["table"], c["seq"], T_out=T,
                                           dtype=TORCH[dt])
        assert np.array_equal(v[0].double().cpu().numpy(), want), dt


def test_the_largest_and_the_smallest_rows_go_through_pages():
    """What the header says of the ends of the range: 2^128 reads back as infinity, 2^-135 as a bf16 number of 2^-133 steps."""
    B, H, k, D, page = 1, 4, 1, 64, 16
    x = torch.zeros(B, H, 3, D)
    x[0, 0, :, 0] = torch.tensor([247.0, 248.0, 255.0]) * 2.0 ** 120
    x[0, 0, :, 1] = -(2.0 ** 118)
    x[0, 1, :, 0] = torch.tensor([2.0 ** -126 * 300, 2.0 ** -133, 5 * 2.0 ** -135])
    x[0, 1, :, 1] = torch.tensor([2.0 ** -135, 3 * 2.0 ** -135, 2.0 ** -149])
    kp, vp = (torch.zeros(1, p, page, D, device=DEV, dtype=torch.uint8) for p in (k, H))
    ks, vs = (torch.zeros(1, p, page, device=DEV) for p in (k, H))
    table, seq = torch.zeros(1, 1, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    chai.chai_append_kv_paged_fp8(x.to(DEV), x.to(DEV), kp, vp, ks, vs, torch.zeros(1, 1, dtype=torch.int32, device=DEV), table, seq)
    codes, scales = orc.quantize_rows_fp8(x.double().numpy())
    assert np.array_equal(vp[0, :, :3].cpu().numpy(), codes[0]) and np.array_equal(vs[0, :, :3].cpu().numpy(), scales[0].astype(np.float32))
    exact = orc.e4m3_values()[codes] * scales[..., None]
    assert exact.max() == 2.0 ** 128 and (scales[0, 1] == 2.0 ** -126).all()
    for dt, step in ((torch.float32, 2.0 ** -149), (torch.bfloat16, 2.0 ** -133)):
        _, v = chai.chai_read_kv_paged_fp8(kp, vp, ks, vs, table, seq, T_out=3, dtype=dt)
        want = np.where(np.abs(exact) >= 2.0 ** 128, np.inf, exact)
        small = np.abs(exact) < 2.0 ** -126
        want = np.where(small, np.rint(exact / step) * step, want)
        assert np.array_equal(v.double().cpu().numpy(), want)


# ---- tables wider than the requests ------------------------------------------------------------------------------

@pytest.mark.parametrize("cache,io", [("f32", "f32"), ("bf16", "bf16"), ("e4m3", "f32")])
@pytest.mark.parametrize("lens", [[300], [5000, 700, 3000]])
def test_decode_does_not_depend_on_the_width_of_the_table(cache, io, lens):
    """Sums are taken in an order that follows from lengths and memberships: tables for 16 and for 40000 positions more give
    the same bits."""
    c = make(cache, io, len(lens), 12, 3, 128, 16, lens, seed=55)
    want = decode(c).clone()
    check(c, want)
    for more in (1, 2500):
        wide = torch.full((len(lens), c["table"].shape[1] + more), -1, dtype=torch.int32, device=DEV)
        wide[:, : c["table"].shape[1]] = c["table"]
        got = decode(dict(c, table=wide))
        assert torch.equal(got.view(torch.uint8), want.view(torch.uint8)), more


# ---- appends of one launch and of several ------------------------------------------------------------------------

@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("advance", [True, False])
@pytest.mark.parametrize("H,k,N", [(32, 8, 1), (72, 24, 1), (96, 32, 1), (97, 32, 1), (20, 5, 2), (16, 5, 3), (16, 16, 4),
                                   (32, 32, 4), (33, 32, 4), (128, 128, 1), (130, 128, 1), (128, 128, 2), (500, 12, 1)])
def test_append_around_the_passes_of_a_step(io, fp8, advance, H, k, N):
    """Below, at and above one pass (1024 vectors) and two of the one-block form, N of one to four with requests that have
    fewer tokens; pages that are bad for the last vectors only."""
    B, D, page = 4, 128, 8
    g = torch.Generator().manual_seed(H * 8 + N)
    lens = [0, page - 1, 2 * page - N + 1 if N > 1 else page, 3]
    new = [N, N, max(0, N - 2), N - 1] if N > 1 else [1, 1, 1, 0]
    table, n_pages = tables(lens, page, H, room=N)
    table = table.copy()
    _, reps = partition(B, H, k, H)
    reps = reps.copy()
    reps[2, k - 1] = -1
    k_new, v_new = ((torch.randn(B, H, N, D, generator=g) * 3).to(TORCH[io]) for _ in range(2))
    before = [random_pool(n_pages, p, page, D, torch.uint8 if fp8 else TORCH[io], 7 + p) for p in (k, H)]
    before += [torch.rand(n_pages, p, page, generator=g).to(DEV) for p in (k, H)]
    for spoil in (False, True):
        if spoil:        # request 1's last token lies on its second page
            table[1, 1 if N > 1 else 0] = n_pages + 5
        kp, vp, ks, vs = (x.clone() for x in before)
        host = [x.cpu() for x in before]
        seq = torch.tensor(lens, dtype=torch.int32, device=DEV)
        ws = chai.new_workspace(256, DEV)
        call = (chai.chai_append_kv_paged_fp8, (kp, vp, ks, vs)) if fp8 else (chai.chai_append_kv_paged, (kp, vp))
        call[0](k_new.to(DEV), v_new.to(DEV), *call[1], torch.from_numpy(reps).to(DEV), torch.from_numpy(table).to(DEV), seq,
                new_lens=torch.tensor(new, dtype=torch.int32, device=DEV), advance=advance, workspace=ws)
        assert chai.chai_device_status(ws) == (chai.CHAI_ERR_BAD_PAGE if spoil else chai.CHAI_OK)
        if fp8:
            (k8, ksc), (v8, vsc) = (orc.quantize_rows_fp8(x.double().numpy()) for x in (k_new, v_new))
            wk, wv, wl = orc.append_kv_paged(k8, v8, host[0].numpy(), host[1].numpy(), reps, table, lens, new)
            wks, wvs, _ = orc.append_kv_paged(ksc.astype(np.float32), vsc.astype(np.float32), host[2].numpy(), host[3].numpy(),
                                              reps, table, lens, new)
            assert np.array_equal(kp.cpu().numpy(), wk) and np.array_equal(vp.cpu().numpy(), wv)
            assert np.array_equal(ks.cpu().numpy(), wks) and np.array_equal(vs.cpu().numpy(), wvs)
        else:
            wk, wv, wl = orc.append_kv_paged(bits(k_new), bits(v_new), bits(host[0]), bits(host[1]), reps, table, lens, new)
            assert np.array_equal(bits(kp), wk) and np.array_equal(bits(vp), wv)
        assert seq.cpu().tolist() == (wl.tolist() if advance else lens)


@pytest.mark.parametrize("cache,io", [("bf16", "bf16"), ("e4m3", "bf16"), ("f32", "f32")])
def test_arrays_much_longer_than_the_requests(cache, io):
    """Dense arrays for 5000 tokens and 500 planes: blocks go on from run to run; rows behind the lengths stay as they were."""
    B, H, k, D, page, N = 5, 80, 20, 128 if cache == "e4m3" else 64, 16, 5000      # 79 runs of 64 tokens (fp32: 157 of 32)
    lens = [5000, 0, 1, 4097, 37]
    g = torch.Generator(device=DEV).manual_seed(5)
    table_np, n_pages = tables(lens, page, 9)
    table = torch.from_numpy(table_np).to(DEV)
    _, reps = partition(B, H, k, 9)
    reps = torch.from_numpy(reps).to(DEV)
    k_new, v_new = (torch.randn(B, H, N, D, device=DEV, generator=g).to(TORCH[io]) for _ in range(2))
    fp8 = cache == "e4m3"
    pages = [torch.zeros(n_pages, p, page, D, device=DEV, dtype=torch.uint8 if fp8 else TORCH[cache]) for p in (k, H)]
    pages += [torch.zeros(n_pages, p, page, device=DEV) for p in (k, H)] if fp8 else []
    seq, count = torch.zeros(B, dtype=torch.int32, device=DEV), torch.tensor(lens, dtype=torch.int32, device=DEV)
    ws = chai.new_workspace(256, DEV)
    put, get = (chai.chai_append_kv_paged_fp8, chai.chai_read_kv_paged_fp8) if fp8 else (chai.chai_append_kv_paged, chai.chai_read_kv_paged)
    put(k_new, v_new, *pages, reps, table, seq, new_lens=count, workspace=ws)
    assert chai.chai_device_status(ws) == chai.CHAI_OK and seq.tolist() == lens
    k_out, v_out = (torch.full((B, p, N, D), 9.0, device=DEV, dtype=TORCH[io]) for p in (k, H))
    get(*pages, table, seq, k_out=k_out, v_out=v_out, workspace=ws)
    assert chai.chai_device_status(ws) == chai.CHAI_OK
    for b, n in enumerate(lens):
        keys = k_new[b, reps[b].long(), :n]
        for out, x in ((k_out[b], keys), (v_out[b], v_new[b, :, :n])):
            assert (out[:, n:] == 9.0).all()
            if fp8:      # half a step of three mantissa bits, or of the row's smallest numbers
                top = x.float().abs().amax(-1, keepdim=True) if n else x.float()
                assert ((out[:, :n].float() - x.float()).abs() <= torch.maximum(x.float().abs() * 2.0 ** -4, top * 2.0 ** -17)).all()
            else:
                assert torch.equal(out[:, :n], x)
    table[3, 4090 // page] = -1          # a page that a block's last run meets
    get(*pages, table, seq, k_out=k_out, v_out=v_out, workspace=ws)
    assert chai.chai_device_status(ws) == chai.CHAI_ERR_BAD_PAGE
    assert not v_out[3, :, 4080:4096].any()
    seq.zero_()
    put(k_new, v_new, *pages, reps, table, seq, new_lens=count, workspace=ws)
    assert chai.chai_device_status(ws) == chai.CHAI_ERR_BAD_PAGE and seq.tolist() == [5000, 0, 1, 0, 37]


# ---- decode against the definition on the pages themselves -------------------------------------------------------

@pytest.mark.parametrize("cache", ["f32", "e4m3"])
@pytest.mark.parametrize("page", [8, 24, 64])
def test_decode_of_random_pages_follows_the_block_table(cache, page):
    """Every row of the pool is random, tables name pages in any order and more than once; the oracle goes through them row
    by row."""
    B, H, k, D, n_pages, scale = 5, 7, 3, 64, 20, 0.125
    lens = [page * 5 + 3, 0, 1, page * 9, 2 * page - 1]
    rng = np.random.default_rng(page)
    table = rng.integers(0, n_pages, (B, 10)).astype(np.int32)
    mem, reps = partition(B, H, k, page)
    q = torch.randn(B, H, D, generator=torch.Generator().manual_seed(page))
    stored, scales, exact = [], [], []
    for planes in (k, H):
        shape = (n_pages, planes, page, D)
        if cache == "e4m3":
            codes = (rng.integers(0, 0x7F, shape) | (rng.integers(0, 2, shape) << 7)).astype(np.uint8)
            size = np.exp2(rng.integers(-10, -6, shape[:3]))
            stored.append(torch.from_numpy(codes).to(DEV))
            scales.append(torch.from_numpy(size.astype(np.float32)).to(DEV))
            exact.append(orc.e4m3_values()[codes] * size[..., None])
        else:
            x = rng.standard_normal(shape).astype(np.float32)
            stored.append(torch.from_numpy(x).to(DEV))
            exact.append(x.astype(np.float64))
    fn = chai.chai_decode_attention_paged_fp8 if cache == "e4m3" else chai.chai_decode_attention_paged
    got = fn(q.to(DEV), *stored, *scales, *(torch.from_numpy(x).to(DEV) for x in (mem, reps, table, np.array(lens, np.int32))), scale)
    got, q = got.double().cpu().numpy(), q.double().numpy()
    ref = orc.decode_attention_paged(q, *exact, mem, reps, table, lens, scale)
    for b, n in enumerate(lens):
        if n == 0:
            assert not got[b].any()
            continue
        kr, vr = (orc.paged_rows(x, table[b], n) for x in exact)
        allowed = decode_bounds(q[b], kr, vr, mem[b], reps[b], scale, "f32", cache == "e4m3") + 2.0 ** -24 * np.abs(ref[b])
        assert (np.abs(got[b] - ref[b]) <= allowed).all(), f"request {b}"
