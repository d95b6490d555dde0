"""Refusals of the calls that make a serving step of many tokens, their workspace sizes, and the frequencies of rotary positions
against their formulas."""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

from paper_2403_08058_b200 import chai

INVALID, UNSUPPORTED, WORKSPACE = chai.CHAI_ERR_INVALID_ARG, chai.CHAI_ERR_UNSUPPORTED, chai.CHAI_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(chai.LIB_PATH):
        from paper_2403_08058_b200.build import build_library
        build_library()
    return chai.load()


BUFFER = (ctypes.c_char * 4096)()
AT = (ctypes.addressof(BUFFER) + 15) // 16 * 16


def doubles(*x):
    return (ctypes.c_double * len(x))(*x)


def plan(lib, p=None, B=2, n=4, n_pages=9, page=16, max_pages=3, ws=AT, ws_bytes=1 << 20):
    return lib.chai_plan_paged(*(p or [AT] * 11), B, n, n_pages, page, max_pages, ws, ws_bytes, None)


def rope(lib, p=None, turns=AT, B=2, Hq=4, Hk=2, N=3, D=128, rot=64, magnitude=None, strides=None, dtype=1):
    magnitude = None if magnitude is None else doubles(magnitude)
    strides = None if strides is None else (ctypes.c_int64 * 12)(*strides)
    return lib.chai_rope(*(p or [AT] * 5), turns, B, Hq, Hk, N, D, rot, 0, magnitude, strides, dtype, None)


def enter(lib, fp8, p=None, turns=AT, rot=64, magnitude=None, B=2, H=4, k=2, n=5, n_pages=9, page=16, D=128, q_stride=0, k_stride=0,
          v_stride=0, k_page=0, v_page=0, dtype=1, ws=None):
    fn = lib.chai_append_rope_paged_fp8 if fp8 else lib.chai_append_rope_paged
    magnitude = None if magnitude is None else doubles(magnitude)
    p = p or [AT, AT, AT, AT + 65536] + [AT] * (8 if fp8 else 6)
    return fn(*p, turns, rot, 0, magnitude, B, H, k, n, n_pages, page, D, q_stride, k_stride, v_stride, k_page, v_page, dtype, ws, None)


def attend(lib, fp8, p=None, B=2, H=4, k=2, n=5, n_pages=9, page=16, max_pages=3, D=128, q_stride=0, k_page=0, v_page=0, scale=1.0,
           dtype=1, ws=AT, ws_bytes=1 << 30):
    fn = lib.chai_prefill_attention_paged_fp8 if fp8 else lib.chai_prefill_attention_paged
    p = p or [AT] * (10 if fp8 else 8) + [AT + 65536]
    return fn(*p, B, H, k, n, n_pages, page, max_pages, D, q_stride, k_page, v_page, scale, 1, dtype, ws, ws_bytes, None)


def test_plan_refusals(lib):
    for i in range(11):
        p = [AT] * 11
        p[i] = None
        assert plan(lib, p) == INVALID and b"null" in lib.chai_last_error(), i
        p[i] = AT + 2
        assert plan(lib, p) == INVALID and b"aligned" in lib.chai_last_error(), i
    for i in (8, 9, 10):
        p = [AT] * 11
        p[i] = AT + 4
        assert plan(lib, p) == INVALID and b"16-byte" in lib.chai_last_error(), i
    assert plan(lib, ws=None) == INVALID and plan(lib, ws=AT + 8) == INVALID
    for bad in (dict(B=0), dict(B=-1), dict(n=0), dict(n_pages=0), dict(page=0), dict(page=-8), dict(max_pages=0)):
        assert plan(lib, **bad) == INVALID, bad
    for bad in (dict(B=65536), dict(n=(1 << 30) + 1), dict(page=12), dict(page=65544), dict(page=4), dict(max_pages=1 << 26)):
        assert plan(lib, **bad) == UNSUPPORTED, bad
    need = chai.load().chai_plan_paged_workspace_bytes(2)
    assert plan(lib, ws_bytes=need - 1) == WORKSPACE and str(need).encode() in lib.chai_last_error()


def test_rope_refusals(lib):
    for i in (0, 1, 2, 3):
        p = [AT] * 5
        p[i] = None
        assert rope(lib, p) == INVALID and b"null" in lib.chai_last_error(), i
        p[i] = AT + 8
        assert rope(lib, p) == INVALID and b"aligned" in lib.chai_last_error(), i
    assert rope(lib, [AT] * 4 + [AT + 2]) == INVALID
    assert rope(lib, turns=None) == INVALID and rope(lib, turns=AT + 4) == INVALID
    for bad in (dict(B=0), dict(Hq=0), dict(Hk=-1), dict(N=0), dict(B=-3), dict(magnitude=math.nan), dict(magnitude=math.inf)):
        assert rope(lib, **bad) == INVALID, bad
    for bad in (dict(D=96), dict(D=256), dict(rot=8), dict(rot=-16), dict(rot=144), dict(dtype=2), dict(dtype=-1), dict(Hq=65536),
                dict(B=1 << 30, N=1 << 30)):
        assert rope(lib, **bad) == UNSUPPORTED, bad
    dense = [4 * 3 * 128, 3 * 128, 128] * 4
    for i in range(12):
        for bad in (-128, 4, (1 << 40) + 8):
            strides = list(dense)
            strides[i] = bad
            assert rope(lib, strides=strides) == INVALID and b"strides" in lib.chai_last_error(), (i, bad)
        if i % 6 >= 3:                                           # rows of an output on top of one another
            strides[i] = 0
            assert rope(lib, strides=strides) == INVALID and b"output" in lib.chai_last_error(), i


@pytest.mark.parametrize("fp8", [False, True])
def test_append_rope_refusals(lib, fp8):
    n = 12 if fp8 else 10
    for i in range(n):
        p = [AT, AT, AT, AT + 65536] + [AT] * (n - 4)
        p[i] = None
        assert enter(lib, fp8, p) == INVALID and b"null" in lib.chai_last_error(), i
        p[i] = AT + 8
        assert enter(lib, fp8, p) == INVALID and b"aligned" in lib.chai_last_error(), i
    assert enter(lib, fp8, ws=AT + 8) == INVALID
    assert enter(lib, fp8, turns=None) == INVALID and enter(lib, fp8, turns=AT + 4) == INVALID
    for bad in (dict(B=0), dict(H=0), dict(k=0), dict(k=5), dict(n=0), dict(n=-1), dict(n_pages=0), dict(page=0), dict(magnitude=math.nan),
                dict(k_page=2 * 16 * 128 - 16), dict(v_page=4 * 16 * 128 + 4), dict(q_stride=4 * 128 - 8), dict(k_stride=4 * 128 + 4),
                dict(v_stride=1 << 60), dict(v_stride=(1 << 64) - 16)):
        assert enter(lib, fp8, **bad) == INVALID, bad
    for bad in (dict(D=96), dict(rot=24), dict(rot=144), dict(page=20), dict(page=65544), dict(dtype=2), dict(H=1025), dict(B=65536),
                dict(n=(1 << 30) + 1)):
        assert enter(lib, fp8, **bad) == UNSUPPORTED, bad
    for at in (AT, AT + 16, AT + 5 * 4 * 128 * 2 - 16):          # the queries' output inside, before its end, on its last row
        p = [AT, AT, AT, at] + [AT] * (n - 4)
        assert enter(lib, fp8, p) == INVALID and b"overlap" in lib.chai_last_error()
    for i in (0, 1, 2):                                          # any of the three behind it, but for its last row's end
        p = [AT - 65536] * 3 + [AT] * (n - 3)
        p[i] = AT + 4 * 512 * 2
        assert enter(lib, fp8, p) == INVALID and b"overlap" in lib.chai_last_error(), i
    p = [AT + 4 * 512 * 2, AT, AT, AT] + [AT] * (n - 4)
    assert enter(lib, fp8, p) == INVALID and b"overlap" in lib.chai_last_error()
    p = [AT, AT, AT, AT + 5 * 4 * 128 * 2] + [AT] * (n - 4)      # (the rows of a wider array reach further)
    assert enter(lib, fp8, p, q_stride=4 * 128 + 8) == INVALID and b"overlap" in lib.chai_last_error()


@pytest.mark.parametrize("fp8", [False, True])
def test_attention_refusals(lib, fp8):
    n = 11 if fp8 else 9
    for i in range(n):
        p = [AT] * (n - 1) + [AT + 65536]
        p[i] = None
        assert attend(lib, fp8, p) == INVALID and b"null" in lib.chai_last_error(), i
        p[i] = AT + 8
        assert attend(lib, fp8, p) == INVALID and b"aligned" in lib.chai_last_error(), i
    assert attend(lib, fp8, ws=None) == INVALID and attend(lib, fp8, ws=AT + 8) == INVALID
    for bad in (dict(B=0), dict(H=0), dict(k=0), dict(k=5), dict(n=0), dict(n_pages=0), dict(page=0), dict(max_pages=0), dict(scale=0.0),
                dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(q_stride=4 * 128 - 8), dict(q_stride=4 * 128 + 4),
                dict(q_stride=1 << 39), dict(q_stride=(1 << 64) - 16), dict(k_page=2 * 16 * 128 - 16), dict(v_page=4 * 16 * 128 + 4)):
        assert attend(lib, fp8, **bad) == INVALID, bad
    for bad in (dict(D=96), dict(page=20), dict(page=65544), dict(dtype=2), dict(H=1025), dict(B=65536), dict(max_pages=1 << 26),
                dict(n=(1 << 26) + 1), dict(H=1024, k=1000), dict(H=1024, k=320),                                # the planner's shared memory
                dict(n=1 << 26, max_pages=1 << 16), dict(B=60000, max_pages=1 << 16, H=64),   # the line of tiles
                dict(n=1 << 26, max_pages=1 << 16, dtype=0)):
        assert attend(lib, fp8, [AT] * (n - 1) + [AT + (1 << 46)], **bad) == UNSUPPORTED, bad
    need = chai.chai_prefill_paged_workspace_bytes(2, 4, 5)
    assert attend(lib, fp8, ws_bytes=need - 1) == WORKSPACE and str(need).encode() in lib.chai_last_error()
    for at in (AT, AT + 5 * 512 * 2 - 16):
        assert attend(lib, fp8, [AT] * (n - 1) + [at]) == INVALID and b"overlap" in lib.chai_last_error()


def test_workspace_bytes(lib):
    for B, H, n in ((1, 1, 1), (16, 32, 64), (4, 72, 256), (300, 52, 9000), (65535, 1024, 1 << 26)):
        assert chai.chai_prefill_paged_workspace_bytes(B, H, n) == 2**20 + 64 * B + 36 * H * (B + n // 128 + 1) + 640000 * min(n, 128)
    for B, H, n in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (-1, 4, 4)):
        assert chai.chai_prefill_paged_workspace_bytes(B, H, n) == 0
    assert [lib.chai_plan_paged_workspace_bytes(B) for B in (1, 300, 65535, 0, -1)] == [516, 512 + 1200, 512 + 4 * 65535, 0, 0]


def plain_frequencies(rot, scaling, base, factor, context, low, high):
    i = np.arange(rot // 2, dtype=np.longdouble)
    if scaling == "base":
        base = np.longdouble(base) * np.longdouble(factor) ** (np.longdouble(rot) / (rot - 2))
    tau = 2 * np.longdouble(np.pi) + np.longdouble(2.4492935982947064e-16)   # (what fp64 leaves of 2 pi)
    f = np.longdouble(base) ** (-2 * i / rot) / tau
    if scaling in ("plain", "base"):
        return f, 1.0
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "bands":
        s = np.clip((context * f - low) / (high - low), 0, 1)
        return f * s + f / factor * (1 - s), 1.0
    at = lambda times: rot * math.log(context / (times * 2 * math.pi)) / (2 * math.log(base))
    first, last = max(math.floor(at(high)), 0), min(math.ceil(at(low)), rot - 1)
    g = np.clip((i - first) / max(last - first, 0.001), 0, 1)
    return f * (1 - g) + f / factor * g, 0.1 * math.log(factor) + 1


@pytest.mark.parametrize("scaling", ["plain", "linear", "base", "ramp", "bands"])
@pytest.mark.parametrize("rot,base,factor,context", [(64, 10000.0, 4.0, 4096.0), (128, 500000.0, 8.0, 8192.0), (16, 10000.0, 1.0, 2048.0),
                                                     (32, 1e6, 32.0, 100.0)])
def test_frequencies(lib, scaling, rot, base, factor, context):
    low, high = (1.0, 4.0) if scaling == "bands" else (1.0, 32.0)
    turns, magnitude = chai.chai_rope_frequencies(rot, base, scaling, factor, context, low, high)
    want, m = plain_frequencies(rot, scaling, base, factor, context, low, high)
    # fp64: pow is good to an ulp or two, and so is each of at most six operations behind it
    np.testing.assert_allclose(np.asarray(turns, dtype=np.float64), want.astype(np.float64), rtol=16 * 2.0**-53, atol=0)
    assert abs(magnitude - m) <= 4 * 2.0**-53 * m


def test_frequencies_refusals(lib):
    turns, one = doubles(*[0.0] * 8), doubles(0.0)
    f = lambda t=turns, m=one, rot=16, scaling=0, p=(1e4, 2.0, 4096.0, 1.0, 4.0): lib.chai_rope_frequencies(
        t, m, rot, scaling, None if p is None else doubles(*p))
    assert f() == chai.CHAI_OK
    assert f(t=None) == f(m=None) == f(p=None) == INVALID
    assert f(rot=0) == f(rot=15) == f(rot=-2) == f(rot=1026) == INVALID
    assert f(scaling=5) == f(scaling=-1) == UNSUPPORTED
    for scaling, p in ((0, (1.0, 2, 4096, 1, 4)), (0, (math.nan, 2, 4096, 1, 4)), (1, (1e4, 0.5, 4096, 1, 4)), (2, (1e4, math.inf, 4096, 1, 4)),
                       (3, (1e4, 2, 0, 1, 4)), (4, (1e4, 2, 4096, 4, 4)), (4, (1e4, 2, 4096, 0, 4)), (3, (1e4, 2, math.nan, 1, 4))):
        assert f(scaling=scaling, p=p) == INVALID, (scaling, p)
    assert f(rot=2, scaling=2) == INVALID
    with pytest.raises(ValueError, match="scaling"):
        chai.chai_rope_frequencies(16, scaling="other")


def test_binding_refuses_what_it_can_see(lib):
    ints = lambda *shape: torch.zeros(*shape, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        chai.chai_plan_paged(ints(2), ints(2), ints(2, 3), ints(9), ints(1), 4, 16)
    with pytest.raises(ValueError, match="max_pages"):
        chai.chai_plan_paged(ints(2), ints(2), ints(6), ints(9), ints(1), 4, 16)
    with pytest.raises(ValueError, match="CUDA"):
        chai.chai_rope(torch.zeros(1, 2, 3, 64), turns=torch.zeros(8, dtype=torch.float64))
    with pytest.raises(ValueError, match=r"B,Hq,N,D"):
        chai.chai_rope(torch.zeros(2, 3, 64), turns=torch.zeros(8, dtype=torch.float64))
    q, kp, vp = torch.zeros(5, 4, 64), torch.zeros(9, 2, 16, 64), torch.zeros(9, 4, 16, 64)
    with pytest.raises(ValueError):
        chai.chai_append_rope_paged(q, q, q, kp, vp, ints(2, 2), ints(5), ints(5), torch.zeros(5, dtype=torch.int64),
                                    torch.zeros(8, dtype=torch.float64))
    with pytest.raises(ValueError):
        chai.chai_prefill_attention_paged(q, kp, vp, ints(2, 4), ints(2, 2), ints(2, 3), ints(2), ints(3), 1.0)
    with pytest.raises(ValueError):
        chai.chai_prefill_attention_paged(q, kp, vp, ints(2, 4), ints(2, 2), ints(6), ints(2), ints(3), 1.0)
