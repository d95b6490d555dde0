"""The paged calls' refusals (host checks of the library and of the binding), and the oracle's row quantiser."""
import ctypes
import os

import numpy as np
import pytest
import torch

from oracle import chai_oracle as orc
from paper_2403_08058_b200 import chai


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(chai.LIB_PATH):
        from paper_2403_08058_b200.build import build_library
        build_library()
    return chai.load()


def addresses(n):
    buf = (ctypes.c_char * 4096)()
    addresses.keep = buf
    p = (ctypes.addressof(buf) + 15) // 16 * 16
    return [p] * n


# (name, number of pointers, sizes behind them)
SIZES = dict(B=2, H=4, k=2, n_pages=9, page_size=16, max_pages=3, D=128)


def call(lib, name, pointers=None, ws=None, ws_bytes=1 << 24, dtype=1, k_stride=0, v_stride=0, rows=5, **sizes):
    s = dict(SIZES, **sizes)
    n = {"append": 8, "append_fp8": 10, "read": 6, "read_fp8": 8, "decode": 8, "decode_fp8": 10}[name]
    p = pointers if pointers is not None else addresses(n)
    tail = [s["n_pages"], s["page_size"], s["max_pages"], s["D"], k_stride, v_stride]
    if name.startswith("append"):
        fn = lib.chai_append_kv_paged_fp8 if "fp8" in name else lib.chai_append_kv_paged
        return fn(*p, s["B"], s["H"], s["k"], rows, *tail, dtype, 1, ws, None)
    if name.startswith("read"):
        fn = lib.chai_read_kv_paged_fp8 if "fp8" in name else lib.chai_read_kv_paged
        return fn(*p, s["B"], s["H"], s["k"], rows, *tail, dtype, ws, None)
    fn = lib.chai_decode_attention_paged_fp8 if "fp8" in name else lib.chai_decode_attention_paged
    return fn(*p, s["B"], s["H"], s["k"], *tail, 1.0, dtype, ws if ws is not None else addresses(1)[0], ws_bytes, None)


NAMES = ["append", "append_fp8", "read", "read_fp8", "decode", "decode_fp8"]


@pytest.mark.parametrize("name", NAMES)
def test_refusals(lib, name):
    n = {"append": 8, "append_fp8": 10, "read": 6, "read_fp8": 8, "decode": 8, "decode_fp8": 10}[name]
    may_be_null = {"append": [7], "append_fp8": [9], "read": [4, 5], "read_fp8": [6, 7]}.get(name, [])
    for i in range(n):
        p = addresses(n)
        p[i] = None
        if i in may_be_null:
            continue
        assert call(lib, name, p) == chai.CHAI_ERR_INVALID_ARG and b"null" in lib.chai_last_error(), i
    if name.startswith("read"):
        p = addresses(n)
        p[n - 1] = p[n - 2] = None                     # nothing to read into
        assert call(lib, name, p) == chai.CHAI_ERR_INVALID_ARG
    p = addresses(n)
    p[0] += 8
    assert call(lib, name, p) == chai.CHAI_ERR_INVALID_ARG and b"aligned" in lib.chai_last_error()
    for bad in (dict(B=0), dict(H=0), dict(k=0), dict(k=5), dict(n_pages=0), dict(max_pages=0), dict(page_size=0),
                dict(B=-1), dict(page_size=-8), dict(k_stride=2 * 16 * 128 - 8), dict(v_stride=4 * 16 * 128 - 8),
                dict(k_stride=2 * 16 * 128 + 4 if "fp8" in name else 2 * 16 * 128 + 4)):
        assert call(lib, name, **bad) == chai.CHAI_ERR_INVALID_ARG, bad
    if name.startswith("decode"):
        assert call(lib, name, B=65535, max_pages=1 << 15, page_size=16) == chai.CHAI_ERR_UNSUPPORTED
    for bad in (dict(page_size=4), dict(page_size=20), dict(page_size=65544), dict(D=96), dict(dtype=2), dict(dtype=-1),
                dict(H=1025), dict(B=65536), dict(max_pages=1 << 26, page_size=16)):
        assert call(lib, name, **bad) == chai.CHAI_ERR_UNSUPPORTED, bad
    if name.startswith("decode"):
        need = chai.chai_decode_paged_workspace_bytes(2, 4, 128)
        assert call(lib, name, ws_bytes=need - 1) == chai.CHAI_ERR_WORKSPACE and str(need).encode() in lib.chai_last_error()
        assert call(lib, name, ws_bytes=0) == chai.CHAI_ERR_WORKSPACE
        assert call(lib, name) == chai.CHAI_ERR_INVALID_ARG and b"overlap" in lib.chai_last_error()   # q and out are one address here
    else:
        assert call(lib, name, rows=0) == chai.CHAI_ERR_INVALID_ARG
        assert call(lib, name, rows=(1 << 30) // 4) == chai.CHAI_ERR_UNSUPPORTED


def test_workspace_bytes(lib):
    f = chai.chai_decode_paged_workspace_bytes
    for B, H, D in ((1, 1, 64), (16, 32, 128), (4, 72, 128), (1000, 1024, 64)):
        assert f(B, H, D) == (64 << 10) + 4 * (160 + B) * H * (D + 8)        # what the header says
    assert f(0, 1, 64) == f(1, 0, 64) == f(1, 1, 96) == 0
    assert chai.chai_status_string(chai.CHAI_ERR_BAD_PAGE).startswith("block-table")


def test_binding_refuses_what_it_can_see():
    kp, vp = torch.zeros(4, 2, 16, 64), torch.zeros(4, 3, 16, 64)
    table, seq = torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    reps, mem, new = torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3, 64)
    with pytest.raises(ValueError, match="CUDA"):
        chai.chai_append_kv_paged(new, new, kp, vp, reps, table, seq)
    with pytest.raises(ValueError, match="CUDA"):
        chai.chai_decode_attention_paged(new, kp, vp, mem, reps, table, seq, 1.0)
    with pytest.raises(ValueError, match="CUDA"):
        chai.chai_read_kv_paged(kp, vp, table, seq, 8)
    with pytest.raises(ValueError, match="agree"):
        chai.chai_read_kv_paged(kp, vp[:3], table, seq, 8)
    with pytest.raises(ValueError, match="n_pages"):
        chai.chai_read_kv_paged(kp[0], vp, table, seq, 8)


def test_row_quantiser_by_hand():
    q, s = orc.quantize_rows_fp8(np.array([[448.0, 224.0, 1.0, -0.001], [449.0, 1.0, 0.0, 0.0], [0.0, 0.0, 0.0, 0.0],
                                           [np.inf, 1.0, np.nan, -np.inf], [2.0 ** -149, 0, 0, 0]]))
    assert s.tolist() == [1.0, 2.0, 1.0, 2.0 ** -8, 2.0 ** -126]
    v = orc.e4m3_values()[q] * s[:, None]
    assert v[0].tolist() == [448.0, 224.0, 1.0, -2.0 ** -9] and v[1, :2].tolist() == [448.0, 1.0]
    assert v[3, 0] == 448.0 / 256 and v[3, 1] == 1.0 and np.isnan(v[3, 2]) and v[3, 3] == -448.0 / 256


def test_row_quantiser_error_is_half_a_step():
    x = np.random.default_rng(0).standard_normal((50, 128)) * np.exp2(np.random.default_rng(1).integers(-40, 40, (50, 1)))
    q, s = orc.quantize_rows_fp8(x)
    err = np.abs(orc.e4m3_values()[q] * s[:, None] - x)
    # half a step of a normal number is 2^-4 of it; below the smallest normal number half of the fixed step 2^-9
    assert (err <= np.maximum(np.abs(x) * 2.0 ** -4, s[:, None] * 2.0 ** -10)).all()
    top = np.abs(x).max(1)
    assert ((top <= 448 * s) & (top > 224 * s)).all()
