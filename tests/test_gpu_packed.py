"""A serving step of many tokens on the GPU -- pages planned, tokens rotated into them, attention over them -- against the
definitions in 64 bits."""
import math

import numpy as np
import pytest
import torch

from oracle import chai_oracle as orc
from packed_cases import DEV, HALF_STEP, attend, batch, check, i32, pages_of, plan, pool_state, rotate, rows
from paged_cases import TORCH, partition
from paper_2403_08058_b200 import chai

pytestmark = pytest.mark.gpu


# ---- plans ------------------------------------------------------------------------------------------------------

def run_plan(seq, new, table, free, count, n_tokens, page, in_place=False, n_out=None):
    t, f, c = i32(table), i32(free), i32([count])
    s = i32(seq)
    ws = chai.new_workspace(int(chai.load().chai_plan_paged_workspace_bytes(len(seq))), DEV)
    ws.fill_(0xFF)
    kw = dict(kv_lens=s) if in_place else dict(free_count_out=torch.full((1,), -9, dtype=torch.int32, device=DEV))
    kv, start, req, pos, slots = chai.chai_plan_paged(s, i32(new), t, f, c, n_tokens, page, workspace=ws, **kw)
    got = dict(block_table=t, free_pages=f, free_count=c if in_place else kw["free_count_out"], kv_lens=kv, token_start=start,
               token_request=req, positions=pos, slots=slots)
    return {k: v.cpu().numpy() for k, v in got.items()}, chai.chai_device_status(ws)


def check_plan(seq, new, table, free, count, n_tokens, page, **kw):
    want = plan(seq, new, table, free, count, n_tokens, page)
    got, status = run_plan(seq, new, table, free, count, n_tokens, page, **kw)
    for name, x in got.items():
        assert np.array_equal(x, want[name]), name
    assert status == want["status"]
    return want


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("page", [8, 16, 24, 128])
@pytest.mark.parametrize("B,most,pad", [(1, 1, 0), (5, 40, 3), (33, 200, 0), (300, 90, 11), (1500, 7, 1), (3, 6000, 5)])
def test_plan(B, most, pad, page, in_place):
    rng = np.random.default_rng([B, most, page])
    seq = rng.integers(0, 300, B)
    new = rng.integers(0, most + 1, B)
    new[rng.random(B) < 0.1] = -1
    max_pages = -(-(300 + most) // page) + 1
    n_pages = B * max_pages + 1
    table, free, count = pool_state(seq, page, n_pages, max_pages, B)
    want = check_plan(seq, new, table, free, count, int(np.maximum(new, 0).sum()) + pad + (1 if not (new > 0).any() else 0), page,
                      in_place=in_place)
    assert want["status"] == chai.CHAI_OK


@pytest.mark.parametrize("B", [7, 2100])
def test_plan_when_not_everybody_fits(B):
    rng = np.random.default_rng(B)
    page, max_pages = 16, 9
    seq, new = rng.integers(0, 144, B), rng.integers(-1, 60, B)
    seq[3], new[3] = 140, 100               # longer than its list
    seq[4] = -2                             # no length
    seq[5], new[5] = 100000, -1             # ends with no length
    n_pages = int((-(-np.maximum(seq, 0)[seq < 1000] // page)).sum()) + 7 * 9 + B
    table, free, count = pool_state(np.where(seq > 1000, 0, seq), page, n_pages, max_pages, B)
    for stack, tokens in ((count, 10 ** 5), (count // 3, 10 ** 5), (0, 10 ** 5), (count, int(np.maximum(new, 0).sum()) // 2), (count, 1),
                          (-3, 100), (n_pages + 5, 100)):
        want = check_plan(seq, new, table, free, stack, tokens, page)
        assert want["status"] != chai.CHAI_OK


def test_plan_pages_that_are_none():
    page, max_pages = 8, 6
    seq, new = np.array([20, 9, 0, 17, 30]), np.array([1, -1, 10, -1, 3])
    table, free, count = pool_state(seq, page, 60, max_pages, 1)
    table[1, 0] = 60                        # an ended list with a wrong entry is not given back
    free[count - 4] = -1
    assert check_plan(seq, new, table, free, count, 30, page)["status"] == chai.CHAI_ERR_BAD_PAGE
    table, free, count = pool_state(seq, page, 60, max_pages, 1)
    table[0, 2] = 1 << 30                   # the page that the next token of request 0 goes to
    assert check_plan(seq, new, table, free, count, 30, page)["status"] == chai.CHAI_ERR_BAD_PAGE
    table, free, count = pool_state(seq, page, 60, max_pages, 1)
    assert check_plan(seq, new, table, free, 60, 30, page)["status"] == chai.CHAI_ERR_BAD_PAGE   # more given back than there are


def test_plan_the_largest_batch():
    B, page = 65535, 8
    rng = np.random.default_rng(2)
    seq, new = rng.integers(0, 9, B), rng.integers(-1, 3, B)
    table, free, count = pool_state(seq, page, 2 * B, 2, 4)
    check_plan(seq, new, table, free, count, 2 * B + 3, page)


def test_plan_long_requests():
    page, max_pages = 16, 70000
    seq, new = np.array([1000003, 0, 5]), np.array([70001, 100000, -1])
    table, free, count = pool_state(seq, page, 150000, max_pages, 4)
    check_plan(seq, new, table, free, count, 170008, page)


def test_plan_steps_one_after_the_other():
    """Requests come, grow, end and come again, each step from what the one before left."""
    rng = np.random.default_rng(8)
    B, page, max_pages, n_pages = 12, 8, 20, 130
    table, free, count = pool_state(np.zeros(B, int), page, n_pages, max_pages, 3)
    seq = np.zeros(B, int)
    for step in range(30):
        new = np.where(seq == 0, rng.integers(0, 70, B), rng.integers(0, 3, B))
        new[(seq > 0) & (rng.random(B) < 0.15)] = -1
        want = check_plan(seq, new, table, free, count, 150, page, in_place=step % 2 == 0)
        table, free, count, seq = want["block_table"], want["free_pages"], int(want["free_count"][0]), want["kv_lens"]
        held = sorted(int(p) for b in range(B) for p in table[b, : -(-int(seq[b]) // page)])
        assert sorted(held + free[:count].tolist()) == list(range(n_pages))      # every page is somewhere, once


# ---- rotary positions -------------------------------------------------------------------------------------------

def frequencies(rot, scaling="plain", **kw):
    return chai.chai_rope_frequencies(rot, scaling=scaling, device=DEV, **kw)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot", [(128, 128), (128, 96), (128, 32), (64, 64), (64, 16), (64, 48)])
@pytest.mark.parametrize("B,Hq,Hk,N", [(1, 1, 0, 1), (2, 3, 5, 37), (3, 7, 1, 130)])
def test_rope(io, interleaved, D, rot, B, Hq, Hk, N, guard):
    g = torch.Generator(device=DEV).manual_seed(rot + N)
    q, k = (torch.randn(B, h, N, D, generator=g, device=DEV).to(TORCH[io]) for h in (Hq, Hk))
    pos = torch.randint(-2 ** 31, 2 ** 31 - 1, (B, N), generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
    pos[:, ::2] = torch.randint(0, 5000, (B, (N + 1) // 2), generator=g, device=DEV).to(torch.int32)
    turns, m = frequencies(rot, "ramp", factor=4.0, context=2048)
    outs = [guard.empty_like(q), guard.empty_like(k) if Hk else None]
    chai.chai_rope(q, k if Hk else None, pos, turns, m, interleaved, q_out=outs[0], k_out=outs[1])
    for x, out in zip((q, k), outs):
        if out is None:
            continue
        ref, err = rotate(x, pos[:, None], turns, m, interleaved)
        assert ((out.double() - ref).abs() <= err + HALF_STEP[io] * (ref.abs() + err) + 1e-37).all()
    # the same in place, from arrays with tokens before heads, and with the positions that are meant where none are given
    qt, kt = q.transpose(1, 2).contiguous().transpose(1, 2), k.transpose(1, 2).contiguous().transpose(1, 2)
    a, b = chai.chai_rope(qt, kt if Hk else None, pos, turns, m, interleaved)
    assert torch.equal(a, outs[0]) and a.stride() == qt.stride() and (not Hk or torch.equal(b, outs[1]))
    chai.chai_rope(q, k if Hk else None, pos, turns, m, interleaved, q_out=q, k_out=k if Hk else None)
    assert torch.equal(q, outs[0]) and (not Hk or torch.equal(k, outs[1]))
    count = torch.arange(N, device=DEV, dtype=torch.int32).expand(B, N).contiguous()
    assert torch.equal(chai.chai_rope(qt, None, None, turns)[0], chai.chai_rope(qt, None, count, turns)[0])


def test_rope_turns_back_and_is_its_own_gradient():
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(2, 3, 50, 128, generator=g, device=DEV)
    pos = torch.randint(0, 100000, (2, 50), generator=g, device=DEV).to(torch.int32)
    turns, m = frequencies(128)
    y = chai.chai_rope(x, None, pos, turns, m)[0]
    back = chai.chai_rope(y, None, -pos, turns, m)[0]
    # two rotations, each off by 6 u (|x1| + |x2|), the second of numbers that are at most |x1| + |x2|
    pair = x.abs()[..., :64] + x.abs()[..., 64:]
    assert ((back - x).abs() <= 18 * 2.0 ** -24 * torch.cat([pair, pair], -1)).all()
    # d sum(w y) / dx = w turned back; a difference along a direction, which is exact for a linear map
    w, d = torch.randn_like(x), torch.randn_like(x)
    grad = chai.chai_rope(w, None, -pos, turns, m)[0]
    along = (w.double() * (rotate(x + d, pos[:, None], turns, m, False)[0] - rotate(x, pos[:, None], turns, m, False)[0])).sum()
    size = (w.double().abs() * (d.double().abs() + x.double().abs())).sum()
    assert abs(float((grad.double() * d.double()).sum() - along)) <= 16 * 2.0 ** -24 * float(size)


def test_rope_offsets_beyond_32_bits():
    turns, m = frequencies(64)
    N, D = 5, 64
    far = (1 << 32) + 8
    big = torch.zeros(far + N * D + 64, device=DEV, dtype=torch.bfloat16)
    x = big.as_strided((2, 1, N, D), (far, N * D, D, 1))
    x.copy_(torch.randn(2, 1, N, D, device=DEV))
    pos = torch.arange(2 * N, device=DEV, dtype=torch.int32).view(2, N)
    want = chai.chai_rope(x.contiguous(), None, pos, turns, m)[0]
    chai.chai_rope(x, None, pos, turns, m, q_out=x)
    assert torch.equal(x.contiguous(), want)


# ---- into the pages ---------------------------------------------------------------------------------------------

def packed(io, H, k, D, page, lens, new, seed, pad=0, fused=True):
    g = torch.Generator(device=DEV).manual_seed(seed)
    B, n = len(lens), sum(new) + pad
    mem, reps = partition(B, H, k, seed)
    max_pages = -(-max(l + x for l, x in zip(lens, new)) // page) + 1
    n_pages = B * max_pages + 2
    table = np.random.default_rng(seed).permutation(n_pages)[: B * max_pages].reshape(B, max_pages)
    qkv = torch.randn(n, 3, H, D, generator=g, device=DEV)
    qkv = (qkv * torch.exp2(torch.randint(-4, 5, (n, 3, H, 1), generator=g, device=DEV).float())).to(TORCH[io])
    parts = [qkv[:, i] if fused else qkv[:, i].contiguous() for i in range(3)]
    req = np.full(n, -1)
    pos, slots = np.zeros(n, int), np.full(n, -1)
    at = 0
    for b, (l, x) in enumerate(zip(lens, new)):
        p = np.arange(l, l + x)
        req[at:at + x], pos[at:at + x], slots[at:at + x] = b, p, table[b, p // page] * page + p % page
        at += x
    return dict(q=parts[0], k=parts[1], v=parts[2], reps=i32(reps), reps_np=reps, token_request=i32(req), positions=i32(pos),
                slots=torch.as_tensor(slots, device=DEV), n_pages=n_pages, req=req, pos=pos, slots_np=slots, n=n, table=table)


@pytest.mark.parametrize("cache,io", [("f32", "f32"), ("bf16", "bf16"), ("e4m3", "bf16"), ("e4m3", "f32")])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("H,k,D,rot,page,lens,new,pad", [
    (1, 1, 64, 64, 8, [0], [1], 0),
    (8, 3, 128, 128, 16, [5, 0, 40, 7], [1, 20, 0, 33], 3),
    (7, 7, 64, 32, 24, [100, 3], [9, 60], 9),
    (72, 24, 128, 96, 32, [31] * 5, [1] * 5, 0),
    (12, 2, 128, 0, 40, [17, 2], [5, 70], 1),
])
def test_append_rope(cache, io, interleaved, H, k, D, rot, page, lens, new, pad, guard):
    c = packed(io, H, k, D, page, lens, new, seed=H + D, pad=pad, fused=pad != 9)
    turns, m = frequencies(rot, "bands", factor=8.0, context=64) if rot else (None, 1.0)
    fp8 = cache == "e4m3"
    dtype = torch.uint8 if fp8 else TORCH[cache]
    kp = guard.empty((c["n_pages"], k, page, D), dtype)
    vp = guard.empty((c["n_pages"], H, page, D), dtype)
    kp.view(torch.uint8).fill_(0x5A), vp.view(torch.uint8).fill_(0x5A)
    ks, vs = (torch.full((c["n_pages"], p, page), 3.0, device=DEV) for p in (k, H)) if fp8 else (None, None)
    q_out = guard.empty((c["n"], H, D), TORCH[io])
    q_out.fill_(7.0)
    ws = chai.new_workspace(256, DEV)
    pages = (kp, vp) + ((ks, vs) if fp8 else ())
    fn = chai.chai_append_rope_paged_fp8 if fp8 else chai.chai_append_rope_paged
    fn(c["q"], c["k"], c["v"], *pages, c["reps"], c["token_request"], c["positions"], c["slots"], turns, m, interleaved,
       q_out=q_out, workspace=ws)
    assert chai.chai_device_status(ws) == chai.CHAI_OK
    touched = torch.zeros(c["n_pages"], page, dtype=torch.bool, device=DEV)
    q_touched = torch.zeros(c["n"], H, dtype=torch.bool, device=DEV)
    for t in range(c["n"]):
        if c["slots_np"][t] < 0:
            continue
        rep, at, row = c["reps_np"][c["req"][t]].tolist(), int(c["slots_np"][t]) // page, int(c["slots_np"][t]) % page
        touched[at, row] = True
        q_touched[t, rep] = True
        pos = c["positions"][t].expand(k)
        for name in ("q", "k"):
            x = c[name][t, rep]
            ref, err = rotate(x, pos, turns, m, interleaved) if rot else (x.double(), torch.zeros_like(x, dtype=torch.float64))
            if name == "q":
                assert ((q_out[t, rep].double() - ref).abs() <= err + HALF_STEP[io] * (ref.abs() + err)).all()
            elif not fp8:
                assert ((kp[at, :, row].double() - ref).abs() <= err + HALF_STEP[io] * (ref.abs() + err)).all()
            else:   # the exact rotation decides about the scale; an element is at most half a step off, on either side of its error
                want_q, want_s = orc.quantize_rows_fp8(ref.cpu().numpy())
                assert np.array_equal(ks[at, :, row].cpu().numpy(), want_s)
                got = kp[at, :, row].view(torch.float8_e4m3fn).double() * ks[at, :, row].double()[:, None]
                step = torch.maximum((ref.abs() + err) * 2.0 ** -4, ks[at, :, row].double()[:, None] * 2.0 ** -10)
                assert ((got - ref).abs() <= step + err).all()
        if fp8:
            want_q, want_s = orc.quantize_rows_fp8(c["v"][t].double().cpu().numpy())
            assert np.array_equal(vp[at, :, row].cpu().numpy(), want_q) and np.array_equal(vs[at, :, row].cpu().numpy(), want_s)
        else:
            assert torch.equal(vp[at, :, row], c["v"][t])
    # everything else as it was
    for x in (kp, vp):
        rest = x.view(torch.uint8).view(c["n_pages"], x.shape[1], page, -1)[~touched[:, None].expand(-1, x.shape[1], -1)]
        assert bool((rest == 0x5A).all())
    if fp8:
        for x in (ks, vs):
            assert bool((x[~touched[:, None].expand_as(x)] == 3.0).all())
    assert bool((q_out[~q_touched] == 7.0).all())


def test_append_rope_scales_next_to_a_border():
    """Rows whose rotated maximum is 1.75 * 2^i but for the last bits: the scale is what exact arithmetic gives."""
    D, page, n = 64, 8, 4096
    turns, m = frequencies(64)
    g = torch.Generator(device=DEV).manual_seed(3)
    pos = torch.randint(0, 3000, (n,), generator=g, device=DEV).to(torch.int32)
    x = torch.randn(n, 1, D, generator=g, device=DEV) * 0.1
    y, _ = rotate(x[:, 0], pos, turns, m, False)
    # stretch each row until its rotated maximum is at the border, then look which side the fp32 row fell on
    x = (x.double() * (1.75 / y.abs().amax(-1))[:, None, None]).float()
    ref, _ = rotate(x[:, 0], pos, turns, m, False)
    want = orc.quantize_rows_fp8(ref.cpu().numpy())[1]
    assert len(set(want.tolist())) == 2                         # both sides occur
    kp, vp = (torch.zeros(n // page, 1, page, D, dtype=torch.uint8, device=DEV) for _ in range(2))
    ks, vs = (torch.zeros(n // page, 1, page, device=DEV) for _ in range(2))
    chai.chai_append_rope_paged_fp8(x, x, x, kp, vp, ks, vs, i32([[0]]), i32(np.zeros(n)), pos, torch.arange(n, device=DEV), turns, m)
    assert np.array_equal(ks.flatten().cpu().numpy(), want)


def test_append_rope_of_rows_with_infinities_and_nan():
    D, page = 64, 8
    turns, m = frequencies(32)
    x = torch.randn(6, 1, D, device=DEV)
    x[0, 0, 3], x[1, 0, 60], x[2] = math.inf, math.nan, 0.0
    x[3], x[4, 0, 50] = 1e-42, 3e38
    pos, slots = torch.arange(6, device=DEV, dtype=torch.int32), torch.arange(6, device=DEV)
    kp, vp = (torch.zeros(1, 1, page, D, dtype=torch.uint8, device=DEV) for _ in range(2))
    ks, vs = (torch.zeros(1, 1, page, device=DEV) for _ in range(2))
    q = chai.chai_append_rope_paged_fp8(x, x, x, kp, vp, ks, vs, i32([[0]]), i32(np.zeros(6)), pos, slots, turns, m)
    ref, _ = rotate(x[:, 0], pos, turns, m, False)
    assert torch.equal(torch.isnan(q[:, 0]), torch.isnan(ref)) and torch.equal(torch.isinf(q[:, 0]), torch.isinf(ref.float()))
    want_q, want_s = orc.quantize_rows_fp8(x[:, 0].double().cpu().numpy())
    assert np.array_equal(vs[0, 0, :6].cpu().numpy(), want_s) and np.array_equal(vp[0, 0, :6].cpu().numpy() & 0x7F, want_q & 0x7F)
    assert np.array_equal(ks[0, 0, :6].cpu().numpy(), orc.quantize_rows_fp8(ref.cpu().numpy())[1])


def test_append_rope_bad_slots_and_requests():
    c = packed("bf16", 4, 2, 64, 8, [0, 0], [10, 10], seed=5)
    turns, m = frequencies(64)
    ws = chai.new_workspace(256, DEV)

    def go(**kw):
        kp, vp = (torch.zeros(c["n_pages"], p, 8, 64, device=DEV, dtype=torch.bfloat16) for p in (2, 4))
        a = dict(c, **kw)
        q = chai.chai_append_rope_paged(a["q"], a["k"], a["v"], kp, vp, a["reps"], a["token_request"], a["positions"], a["slots"],
                                        turns, m, workspace=ws)
        return q, kp, vp, chai.chai_device_status(ws)

    q, kp, vp, status = go()
    assert status == chai.CHAI_OK
    for change in (dict(slots=c["slots"].clone().index_fill_(0, torch.tensor([3], device=DEV), c["n_pages"] * 8)),
                   dict(slots=c["slots"].clone().index_fill_(0, torch.tensor([3], device=DEV), 1 << 40)),
                   dict(token_request=c["token_request"].clone().index_fill_(0, torch.tensor([3], device=DEV), 2)),
                   dict(token_request=c["token_request"].clone().index_fill_(0, torch.tensor([3], device=DEV), -1))):
        q1, kp1, vp1, status = go(**change)
        assert status == chai.CHAI_ERR_BAD_PAGE
        at, row = int(c["slots_np"][3]) // 8, int(c["slots_np"][3]) % 8
        assert not q1[3].any() and not kp1[at, :, row].any() and not vp1[at, :, row].any()
        kp1[at, :, row], vp1[at, :, row], q1[3] = kp[at, :, row], vp[at, :, row], q[3]
        assert torch.equal(q1, q) and torch.equal(kp1, kp) and torch.equal(vp1, vp)
    reps = c["reps"].clone()
    reps[0, 1], reps[1, 0] = -1, 9            # unused slots: their keys and queries are left alone
    q1, kp1, vp1, status = go(reps=reps)
    mine = torch.as_tensor(c["slots_np"][:10], device=DEV)
    assert not kp1[mine // 8, 1, mine % 8].any() and torch.equal(kp1[mine // 8, 0, mine % 8], kp[mine // 8, 0, mine % 8])
    assert torch.equal(vp1, vp)


# ---- attention --------------------------------------------------------------------------------------------------

KINDS = [("f32", "f32"), ("bf16", "bf16"), ("e4m3", "bf16"), ("e4m3", "f32")]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("cache,io", KINDS)
@pytest.mark.parametrize("D,page", [(128, 16), (64, 24), (128, 8), (64, 128), (128, 200)])
def test_attention(cache, io, D, page, causal, guard):
    new = [1, 7, 0, 130, 33, 1, 128, 4, 20]
    kv = [1, 300, 50, 130, 0, 700, 257, 129, 20]
    if causal:
        kv[4] = 33
    c = batch(cache, io, 9, 4, D, page, kv, new, seed=D + page, pad=5)
    ws = chai.new_workspace(chai.chai_prefill_paged_workspace_bytes(c["B"], c["H"], c["n_tokens"]), DEV)
    ws.fill_(0xFF)
    out = guard.empty((c["n_tokens"], 9, D), TORCH[io])
    out.fill_(5.0)
    attend(c, causal, out=out, workspace=ws)
    check(c, out, causal, f"{cache} {io} D {D} page {page}")
    assert chai.chai_device_status(ws) == chai.CHAI_OK
    assert bool((out[sum(new):] == 5.0).all())                 # padding stays as it was


@pytest.mark.parametrize("cache,io", KINDS)
@pytest.mark.parametrize("H,k,page,kv,new", [
    (1, 1, 16, [1], [1]),
    (32, 8, 16, [2048, 600], [4, 4]),              # few rows: key tiles are divided
    (32, 8, 16, [9000], [1]),
    (5, 2, 64, [20011], [17]),
    (72, 24, 32, [1500, 3, 900], [3, 3, 64]),
    (40, 1, 128, [500, 513], [40, 200]),           # one cluster of many members
    (12, 12, 8, [777], [777]),
    (130, 130, 16, [77], [20]),
    (8, 3, 48, [1300, 1300, 5], [1290, 1, 5]),
])
def test_attention_heads_and_lengths(cache, io, H, k, page, kv, new):
    c = batch(cache, io, H, k, 128, page, kv, new, seed=H + page)
    check(c, attend(c), True, f"{cache} {io} H {H} k {k} page {page} kv {kv}")


@pytest.mark.parametrize("cache,io", KINDS)
def test_attention_tokens_that_see_nothing(cache, io):
    """More tokens than cached positions: the first ones see none of them."""
    c = batch(cache, io, 4, 2, 64, 16, [5, 130], [9, 300], seed=2)
    out = attend(c)
    assert not out[:4].any() and not out[9:9 + 170].any()
    check(c, out)


@pytest.mark.parametrize("cache,io", KINDS[:3])
def test_attention_of_one_token_is_the_decode_step(cache, io):
    kv = [300, 1, 77, 2000]
    c = batch(cache, io, 12, 5, 128, 16, kv, [1] * 4, seed=4)
    fn = chai.chai_decode_attention_paged_fp8 if cache == "e4m3" else chai.chai_decode_attention_paged
    want = fn(c["q"], *pages_of(c), c["membership"], c["reps"], c["table"], c["kv_lens"], c["scale"])
    check(c, want)
    check(c, attend(c))


@pytest.mark.parametrize("cache,io", KINDS[:2])
def test_attention_of_prompts_is_the_dense_prefill(cache, io):
    """The rows of chai_prefill_attention on dense arrays, read back from the same pages."""
    B, T = 2, 200
    c = batch(cache, io, 8, 3, 128, 16, [T] * B, [T] * B, seed=6)
    k, v = chai.chai_read_kv_paged(*pages_of(c), c["table"], c["kv_lens"], T)
    dense = c["q"].view(B, T, 8, 128).transpose(1, 2).contiguous()
    want = chai.chai_prefill_attention(dense, k, v, c["membership"], c["reps"], c["scale"]).transpose(1, 2).reshape(B * T, 8, 128)
    check(c, want)
    check(c, attend(c))


@pytest.mark.parametrize("cache,io", KINDS)
@pytest.mark.parametrize("kind", ["rising", "falling", "one_quadrant", "equal", "far_below"])
def test_attention_scores_far_from_the_reference(cache, io, kind):
    """Scores of hundreds that grow along the context, fall, or grow for some rows only: references that move."""
    H, k, D, page, n, L = 4, 2, 64, 16, 150, 900
    c = batch(cache, io, H, k, D, page, [L], [n], seed=9)
    t = torch.linspace(-1, 1, L, device=DEV)
    slope = {"rising": t, "falling": -t, "one_quadrant": t, "equal": torch.ones_like(t), "far_below": -torch.ones_like(t)}[kind] * 40
    at, row = c["table"][0].long()[torch.arange(L, device=DEV) // page], torch.arange(L, device=DEV) % page
    ones = torch.ones(D, device=DEV)
    key = slope[:, None] * ones
    if cache == "e4m3":
        q8, s8 = orc.quantize_rows_fp8(key.double().cpu().numpy())
        c["k_pages"][at, :, row] = torch.as_tensor(q8, device=DEV)[:, None].expand(-1, k, -1)
        c["k_scales"][at, :, row] = torch.as_tensor(s8.astype(np.float32), device=DEV)[:, None].expand(-1, k)
    else:
        c["k_pages"][at, :, row] = key.to(TORCH[cache])[:, None].expand(-1, k, -1)
    c["q"].fill_(1.0)
    if kind == "one_quadrant":
        c["q"].fill_(0.01)
        c["q"][32:64] = 1.5
    check(c, attend(c), True, kind)


@pytest.mark.parametrize("cache,io", KINDS)
def test_attention_infinite_scores_and_nan(cache, io):
    """Scores of -inf are weights of 0; a row of nothing else is zero; a NaN that a row sees makes it NaN, and only such rows."""
    H, k, D, page, L, n = 2, 1, 64, 16, 200, 100
    c = batch(cache, io, H, k, D, page, [L], [n], seed=12)
    c["q"][:, :, 0], c["q"][:, :, 1:] = 1.0, 0.0
    first = c["table"][0].long()[torch.arange(L, device=DEV) // page]
    row = torch.arange(L, device=DEV) % page
    if cache == "e4m3":
        c["k_pages"][first, 0, row] = 0x38                       # 1.0
        c["k_scales"][first, 0, row] = 1.0
        c["k_scales"][first[50], 0, row[50]] = math.nan
        hit = 50
    else:
        kp = c["k_pages"]
        kp[first, 0, row] = 1.0
        kp[first[:100], 0, row[:100], 0] = -math.inf             # rows 0..  see 101 positions and more: the rest counts
        out = attend(c)
        v = rows(c, "v", 0)
        want = torch.stack([v[:, 100:L - n + i + 1].mean(1) for i in range(n)])
        assert (out.double() - want).abs().max() <= 2.0 ** -7
        kp[first, 0, row, 0] = -math.inf
        assert not attend(c).any()                               # nothing but -inf
        kp[first, 0, row, 0] = 1.0
        kp[first[150], 0, row[150], 0] = math.nan
        hit = 150
    out = attend(c)
    sees = torch.arange(n, device=DEV) + L - n >= hit
    assert torch.isnan(out[sees]).all() and torch.isfinite(out[~sees]).all()


def test_attention_bad_pages_and_unresolved_heads():
    for cache, io in KINDS:
        c = batch(cache, io, 8, 3, 64, 16, [100, 300, 40], [3, 140, 40], seed=21)
        ws = chai.new_workspace(chai.chai_prefill_paged_workspace_bytes(3, 8, c["n_tokens"]), DEV)
        good = attend(c, workspace=ws)
        assert chai.chai_device_status(ws) == chai.CHAI_OK
        t = c["table"].clone()
        c["table"][0, 7:], c["table"][2, 3:] = -7, 1 << 30        # behind the lengths: not looked at
        assert torch.equal(attend(c, workspace=ws), good) and chai.chai_device_status(ws) == chai.CHAI_OK
        for bad in (-1, c["n_pages"], 1 << 30, -(1 << 31)):
            c["table"][1, 5] = bad
            out = attend(c, workspace=ws)
            assert chai.chai_device_status(ws) == chai.CHAI_ERR_BAD_PAGE
            assert not out[3:143].any() and torch.equal(out[:3], good[:3]) and torch.equal(out[143:], good[143:])
        c["table"] = t
        lost = [h for h in range(8) if h not in c["reps_np"][1]][:2]
        c["membership"][1, lost] = 77
        out = attend(c, workspace=ws)
        assert chai.chai_device_status(ws) == chai.CHAI_ERR_BAD_MEMBERSHIP
        kept = [h for h in range(8) if h not in lost]
        assert not out[3:143, lost].any() and torch.equal(out[:3], good[:3])
        out[3:143, lost] = good[3:143, lost]
        check(c, out, True, f"{len(kept)} heads")


@pytest.mark.parametrize("cache,io", KINDS)
def test_attention_strided_queries_and_pages_far_apart(cache, io):
    c = batch(cache, io, 6, 4, 128, 16, [100, 17, 300], [10, 17, 150], seed=9)
    want = attend(c)
    n, k, H, page, D = c["n_pages"], 4, 6, 16, 128
    both = torch.zeros((n, (k + H) * page * D + 64), device=DEV, dtype=c["k_pages"].dtype)
    kp, vp = both[:, : k * page * D].view(n, k, page, D), both[:, k * page * D: (k + H) * page * D].view(n, H, page, D)
    kp.copy_(c["k_pages"]), vp.copy_(c["v_pages"])
    c["k_pages"], c["v_pages"] = kp, vp
    wide = torch.zeros(c["n_tokens"], 3, H, D, device=DEV, dtype=c["q"].dtype)
    wide[:, 1] = c["q"]
    c["q"] = wide[:, 1]
    assert torch.equal(attend(c), want)
    # an output that starts on a 16-byte boundary only
    raw = torch.zeros(c["n_tokens"] * H * D + 16, device=DEV, dtype=want.dtype)
    out = raw[16 // want.element_size():][: c["n_tokens"] * H * D].view(c["n_tokens"], H, D)
    assert torch.equal(attend(c, out=out), want)


@pytest.mark.parametrize("cache,io", KINDS[:3])
def test_attention_pages_beyond_32_bits(cache, io):
    page, D, k, H = 16, 64, 2, 3
    c = batch(cache, io, H, k, D, page, [90, 33], [20, 33], seed=7)
    want = attend(c)
    n = c["n_pages"]
    apart = (1 << 32) // (n - 1) // 16 * 16 + 16
    big = torch.zeros(((n - 1) * apart + (k + H) * page * D,), device=DEV, dtype=c["k_pages"].dtype)
    kp = big.as_strided((n, k, page, D), (apart, page * D, D, 1))
    vp = big.as_strided((n, H, page, D), (apart, page * D, D, 1), k * page * D)
    kp.copy_(c["k_pages"]), vp.copy_(c["v_pages"])
    c["k_pages"], c["v_pages"] = kp, vp
    assert int(c["table"].max()) * apart * big.element_size() > 1 << 31
    assert torch.equal(attend(c), want)


@pytest.mark.parametrize("cache,io", KINDS)
def test_attention_is_repeatable(cache, io):
    c = batch(cache, io, 32, 8, 64, 16, [3000, 64, 1700], [5, 64, 400], seed=31)
    ws = chai.new_workspace(chai.chai_prefill_paged_workspace_bytes(3, 32, c["n_tokens"]), DEV)
    first = attend(c, workspace=ws)
    check(c, first)
    for _ in range(5):
        assert torch.equal(attend(c, workspace=ws).view(torch.uint8), first.view(torch.uint8))


@pytest.mark.parametrize("cache,io", KINDS[:3])
def test_attention_many_requests(cache, io):
    rng = np.random.default_rng(5)
    new = [int(x) for x in rng.integers(0, 4, 700)]
    kv = [n + int(x) for n, x in zip(new, rng.integers(0, 40, 700))]
    c = batch(cache, io, 4, 2, 64, 8, kv, new, seed=70)
    check(c, attend(c), True, "700 short requests")


def test_attention_many_heads():
    c = batch("bf16", "bf16", 1000, 200, 64, 8, [19, 150], [3, 140], seed=3)
    check(c, attend(c), True, "1000 heads, 200 clusters")


# ---- together ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("cache,io", KINDS)
def test_a_served_batch(cache, io):
    """Requests come with prompts in chunks, grow by a token, end, and their pages go to others: plan, append and attention
    on the device alone, every step's outputs against dense float64 copies of what was put in.  The last steps are a captured
    graph, replayed."""
    H, k, D, page, B, max_pages, n_pages, n_tokens = 6, 3, 64, 8, 5, 24, 60, 96
    g = torch.Generator(device=DEV).manual_seed(77)
    fp8 = cache == "e4m3"
    mem, reps = partition(B, H, k, 5)
    table, free = torch.full((B, max_pages), -1, dtype=torch.int32, device=DEV), torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    count, seq = i32([n_pages]), i32(np.zeros(B))
    dt = torch.uint8 if fp8 else TORCH[cache]
    kp, vp = (torch.full((n_pages, p, page, D), 0x7F if fp8 else math.nan, device=DEV, dtype=dt) for p in (k, H))
    ks, vs = (torch.full((n_pages, p, page), math.nan, device=DEV) for p in (k, H)) if fp8 else (None, None)
    pages = (kp, vp) + ((ks, vs) if fp8 else ())
    turns, m = frequencies(64)
    qkv = torch.empty(n_tokens, 3, H, D, device=DEV, dtype=TORCH[io])
    new = i32(np.zeros(B))
    reps_t, mem_t = i32(reps), i32(mem)
    enter = chai.chai_append_rope_paged_fp8 if fp8 else chai.chai_append_rope_paged
    look = chai.chai_prefill_attention_paged_fp8 if fp8 else chai.chai_prefill_attention_paged
    q_rot, out = torch.zeros(n_tokens, H, D, device=DEV, dtype=TORCH[io]), torch.zeros(n_tokens, H, D, device=DEV, dtype=TORCH[io])
    plan_ws = chai.new_workspace(512 + 4 * B, DEV)
    ws = chai.new_workspace(chai.chai_prefill_paged_workspace_bytes(B, H, n_tokens), DEV)
    scale = 1.0 / math.sqrt(D)
    start = torch.zeros(B + 1, dtype=torch.int32, device=DEV)
    req, pos = (torch.zeros(n_tokens, dtype=torch.int32, device=DEV) for _ in range(2))
    slots = torch.zeros(n_tokens, dtype=torch.int64, device=DEV)

    def step():
        chai.chai_plan_paged(seq, new, table, free, count, n_tokens, page, kv_lens=seq, token_start=start, token_request=req,
                             positions=pos, slots=slots, workspace=plan_ws)
        enter(qkv[:, 0], qkv[:, 1], qkv[:, 2], *pages, reps_t, req, pos, slots, turns, m, q_out=q_rot)
        look(q_rot, *pages, mem_t, reps_t, table, seq, start, scale, out=out, workspace=ws)

    plans = [[20, 0, 33, 1, 8], [1, 40, 1, 30, 1], [17, 1, -1, 1, 1], [1, 1, 60, 1, -1], [1, 1, 1, -1, 50], [4, 4, 4, 20, 4],
             [1, 1, 1, 1, 1], [-1, 2, 1, 1, 1]]
    cached = [0] * B
    graph = None
    for i, p in enumerate(plans):
        qkv.copy_(torch.randn(qkv.shape, generator=g, device=DEV))
        new.copy_(i32(p))
        if i == 5:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step()
            torch.cuda.current_stream().wait_stream(side)
        if graph is not None:
            graph.replay()
        else:
            step()
        cached = [0 if x < 0 else c + x for c, x in zip(cached, p)]
        assert chai.chai_device_status(plan_ws) == chai.CHAI_OK and chai.chai_device_status(ws) == chai.CHAI_OK
        assert seq.tolist() == cached
        held = sorted(int(x) for b in range(B) for x in table[b, : -(-cached[b] // page)]) + free[: int(count)].tolist()
        assert sorted(held) == list(range(n_pages))
        c = dict(cache=cache, io=io, B=B, H=H, k=k, D=D, page=page, kv=cached, new=[max(x, 0) for x in p], scale=scale, mem=mem,
                 reps_np=reps, table=table, k_pages=kp, v_pages=vp, k_scales=ks, v_scales=vs, q=q_rot)
        check(c, out, True, f"step {i}")
        # what was cached is what was put in
        at = 0
        for b, x in enumerate(c["new"]):
            if x:
                where = torch.arange(cached[b] - x, cached[b], device=DEV)
                got = vp[table[b].long()[where // page], :, where % page]
                if not fp8:
                    assert torch.equal(got, qkv[at:at + x, 2])
                ref, err = rotate(qkv[at:at + x, 0][:, reps[b].tolist()], where[:, None].expand(-1, k), turns, m, False)
                assert ((q_rot[at:at + x][:, reps[b].tolist()].double() - ref).abs() <= err + HALF_STEP[io] * (ref.abs() + err)).all()
            at += x
