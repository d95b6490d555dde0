"""Thin ctypes binding of libchai.so: same names as include/chai.h, argument marshalling only.

Torch supplies device memory and the current stream; every step of the path runs in the
library's kernels.  There is no fallback: if the library has not been built (or cannot be
loaded) the first call raises.
"""
from __future__ import annotations

import ctypes
import os
import struct

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libchai.so")

CHAI_OK = 0
CHAI_ERR_INVALID_ARG, CHAI_ERR_UNSUPPORTED, CHAI_ERR_WORKSPACE = 1, 2, 3
CHAI_ERR_BAD_MEMBERSHIP, CHAI_ERR_TIMEOUT, CHAI_ERR_CUDA, CHAI_ERR_CACHE_FULL, CHAI_ERR_BAD_PAGE = 4, 5, 6, 7, 8
CHAI_F32, CHAI_BF16 = 0, 1

# every symbol include/chai.h declares
EXPORTS = [
    "chai_prefix_features", "chai_cluster_heads", "chai_compact_k_cache", "chai_decode_attention",
    "chai_decode_workspace_bytes", "chai_decode_attention_host", "chai_decode_attention_host_async", "chai_decode_attention_host_streams", "chai_prefill_attention",
    "chai_prefill_attention_simt", "chai_prefill_workspace_bytes", "chai_device_status",
    "chai_status_string", "chai_last_error", "chai_version", "chai_decode_attention_static",
    "chai_decode_attention_ragged", "chai_append_kv", "chai_compact_k_cache_inplace",
    "chai_prefill_attention_from", "chai_prefill_attention_simt_from",
    "chai_decode_qkv_workspace_bytes", "chai_decode_attention_qkv", "chai_prefill_qkv_workspace_bytes",
    "chai_prefill_attention_qkv", "chai_broadcast_membership", "chai_select_representatives", "chai_cluster_sweep",
    "chai_quantize_cache_fp8", "chai_decode_fp8_workspace_bytes", "chai_decode_attention_fp8",
    "chai_set_decode_wait_limit_cycles",
    "chai_append_kv_paged", "chai_append_kv_paged_fp8", "chai_read_kv_paged", "chai_read_kv_paged_fp8",
    "chai_decode_paged_workspace_bytes", "chai_decode_attention_paged", "chai_decode_attention_paged_fp8",
    "chai_plan_paged", "chai_plan_paged_workspace_bytes", "chai_rope_frequencies", "chai_rope", "chai_append_rope_paged",
    "chai_append_rope_paged_fp8", "chai_prefill_paged_workspace_bytes", "chai_prefill_attention_paged",
    "chai_prefill_attention_paged_fp8",
]
DECODE_STATIC_SCRATCH_BYTES = 8 << 20   # CHAI_DECODE_STATIC_SCRATCH_BYTES

_lib = None


class ChaiError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__(f"libchai status {status}: {text}")
        self.status = status


def load() -> ctypes.CDLL:
    """Load libchai.so from the package directory (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2403_08058_b200.build` "
                           "(there is no CPU or PyTorch fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, ci, cf, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    lib.chai_prefix_features.argtypes = [vp, vp, ci, ci, ci, ci, ci, cf, ci, vp, vp]
    lib.chai_cluster_heads.argtypes = [vp, ci, ci, ci, ci, ci, ctypes.c_uint64, vp, vp, vp, vp, vp]
    lib.chai_compact_k_cache.argtypes = [vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, vp]
    lib.chai_decode_attention.argtypes = [vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, cf, ci, vp, sz, vp]
    for name in ("chai_decode_attention_host", "chai_decode_attention_host_async"):
        getattr(lib, name).argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, cf, ci, vp, sz, vp]
    lib.chai_decode_attention_host_streams.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, cf, ci, vp,
                                                       sz, vp, vp, vp, vp, vp]
    for name in ("chai_prefill_attention", "chai_prefill_attention_simt"):
        getattr(lib, name).argtypes = [vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, cf, ci, ci, vp, sz, vp]
    lib.chai_decode_attention_qkv.argtypes = [vp, vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, cf, ci, vp, sz, vp]
    lib.chai_prefill_attention_qkv.argtypes = [vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, cf, ci, ci, vp, sz, vp]
    lib.chai_broadcast_membership.argtypes = [vp, vp, vp, vp, ci, ci, ci, vp]
    lib.chai_select_representatives.argtypes = [vp, vp, ci, ci, ci, ci, vp, vp]
    lib.chai_quantize_cache_fp8.argtypes = [vp, vp, vp, ci, ci, ci, ci, vp]
    lib.chai_decode_fp8_workspace_bytes.argtypes = [ci, ci, ci, ci, ci]
    lib.chai_decode_fp8_workspace_bytes.restype = sz
    lib.chai_decode_attention_fp8.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, sz, cf, vp, sz, vp]
    lib.chai_cluster_sweep.argtypes = [vp, ci, ci, ci, ci, ci, ctypes.c_uint64, vp, vp, vp]
    for name in ("chai_decode_workspace_bytes", "chai_prefill_workspace_bytes", "chai_decode_qkv_workspace_bytes",
                 "chai_prefill_qkv_workspace_bytes"):
        getattr(lib, name).argtypes = [ci, ci, ci, ci, ci, ci]
        getattr(lib, name).restype = sz
    lib.chai_decode_attention_ragged.argtypes = [vp, vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, sz, cf, ci, vp, sz, vp]
    lib.chai_append_kv.argtypes = [vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, sz, ci, ci, vp, vp]
    lib.chai_compact_k_cache_inplace.argtypes = [vp, vp, ci, ci, ci, ci, ci, ci, ci, vp, vp]
    for name in ("chai_prefill_attention_from", "chai_prefill_attention_simt_from"):
        getattr(lib, name).argtypes = [vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, cf, ci, ci, vp, sz, vp]
    lib.chai_decode_attention_static.argtypes = [vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, cf, ci, vp]
    lib.chai_device_status.argtypes = [vp, ctypes.POINTER(ci), vp]
    lib.chai_set_decode_wait_limit_cycles.argtypes = [ctypes.c_longlong]
    lib.chai_set_decode_wait_limit_cycles.restype = None
    lib.chai_append_kv_paged.argtypes = [vp] * 8 + [ci] * 8 + [sz, sz, ci, ci, vp, vp]
    lib.chai_append_kv_paged_fp8.argtypes = [vp] * 10 + [ci] * 8 + [sz, sz, ci, ci, vp, vp]
    lib.chai_read_kv_paged.argtypes = [vp] * 6 + [ci] * 8 + [sz, sz, ci, vp, vp]
    lib.chai_read_kv_paged_fp8.argtypes = [vp] * 8 + [ci] * 8 + [sz, sz, ci, vp, vp]
    lib.chai_decode_paged_workspace_bytes.argtypes = [ci, ci, ci]
    lib.chai_decode_paged_workspace_bytes.restype = sz
    lib.chai_decode_attention_paged.argtypes = [vp] * 8 + [ci] * 7 + [sz, sz, cf, ci, vp, sz, vp]
    lib.chai_decode_attention_paged_fp8.argtypes = [vp] * 10 + [ci] * 7 + [sz, sz, cf, ci, vp, sz, vp]
    lib.chai_plan_paged_workspace_bytes.argtypes = [ci]
    lib.chai_plan_paged_workspace_bytes.restype = sz
    lib.chai_plan_paged.argtypes = [vp] * 11 + [ci] * 5 + [vp, sz, vp]
    lib.chai_rope_frequencies.argtypes = [vp, vp, ci, ci, vp]
    lib.chai_rope.argtypes = [vp] * 6 + [ci] * 7 + [vp, vp, ci, vp]
    lib.chai_append_rope_paged.argtypes = [vp] * 11 + [ci, ci, vp] + [ci] * 7 + [sz] * 5 + [ci, vp, vp]
    lib.chai_append_rope_paged_fp8.argtypes = [vp] * 13 + [ci, ci, vp] + [ci] * 7 + [sz] * 5 + [ci, vp, vp]
    lib.chai_prefill_paged_workspace_bytes.argtypes = [ci, ci, ci]
    lib.chai_prefill_paged_workspace_bytes.restype = sz
    lib.chai_prefill_attention_paged.argtypes = [vp] * 9 + [ci] * 8 + [sz] * 3 + [cf, ci, ci, vp, sz, vp]
    lib.chai_prefill_attention_paged_fp8.argtypes = [vp] * 11 + [ci] * 8 + [sz] * 3 + [cf, ci, ci, vp, sz, vp]
    lib.chai_status_string.argtypes = [ci]
    lib.chai_status_string.restype = ctypes.c_char_p
    lib.chai_last_error.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _check(rc: int) -> None:
    if rc != CHAI_OK:
        lib = load()
        text = lib.chai_last_error().decode() or lib.chai_status_string(rc).decode()
        raise ChaiError(rc, text)


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return CHAI_F32
    if t.dtype == torch.bfloat16:
        return CHAI_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _dev(*tensors) -> None:
    for t in tensors:
        if t is None:
            continue
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError("tensors must be contiguous CUDA tensors")


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _ptr(t):
    return None if t is None else t.data_ptr()


def chai_version() -> int:
    return int(load().chai_version())


def chai_status_string(status: int) -> str:
    return load().chai_status_string(int(status)).decode()


def chai_decode_workspace_bytes(B, H, k, T, D, dtype) -> int:
    return int(load().chai_decode_workspace_bytes(B, H, k, T, D, dtype))


def chai_prefill_workspace_bytes(B, H, k, T, D, dtype) -> int:
    return int(load().chai_prefill_workspace_bytes(B, H, k, T, D, dtype))


def chai_prefix_features(q_full, k_full, P: int, scale: float, features=None):
    """q_full, k_full [B,H,T_cap,D] -> features [B,H,P*P] fp32."""
    _dev(q_full, k_full, features)
    B, H, T_cap, D = q_full.shape
    if features is None:
        features = torch.empty((B, H, P * P), device=q_full.device, dtype=torch.float32)
    _check(load().chai_prefix_features(_ptr(q_full), _ptr(k_full), B, H, T_cap, D, P, scale, _dt(q_full),
                                       _ptr(features), _stream()))
    return features


def chai_cluster_heads(features, k: int, max_iter: int = 20, seed: int = 0, want_inertia: bool = True):
    """features [B,H,F] fp32 -> (membership [B,H] i32, reps [B,k] i32, k_eff [B] i32, inertia [B] f64|None)."""
    _dev(features)
    if features.dtype != torch.float32:
        raise TypeError("features must be float32")
    B, H, F = features.shape
    dev = features.device
    membership = torch.empty((B, H), device=dev, dtype=torch.int32)
    reps = torch.empty((B, k), device=dev, dtype=torch.int32)
    k_eff = torch.empty((B,), device=dev, dtype=torch.int32)
    inertia = torch.empty((B,), device=dev, dtype=torch.float64) if want_inertia else None
    _check(load().chai_cluster_heads(_ptr(features), B, H, F, k, max_iter, seed, _ptr(membership), _ptr(reps),
                                     _ptr(k_eff), _ptr(inertia), _stream()))
    return membership, reps, k_eff, inertia


def chai_cluster_sweep(features, k_max: int, max_iter: int = 20, seed: int = 0):
    """features [B,H,F] fp32 -> (inertia curve [B,k_max] f64, knee [B] int32): k-means for every k = 1..k_max."""
    _dev(features)
    if features.dtype != torch.float32:
        raise TypeError("features must be float32")
    B, H, F = features.shape
    curve = torch.empty((B, k_max), device=features.device, dtype=torch.float64)
    pick = torch.empty((B,), device=features.device, dtype=torch.int32)
    _check(load().chai_cluster_sweep(_ptr(features), B, H, F, k_max, max_iter, seed, _ptr(curve), _ptr(pick), _stream()))
    return curve, pick


def chai_select_representatives(features, membership, k: int):
    """features [B,H,F] fp32, membership [B,H] -> reps [B,k]: each cluster's member nearest to the cluster mean."""
    _dev(features, membership)
    B, H, F = features.shape
    reps = torch.empty((B, k), device=features.device, dtype=torch.int32)
    _check(load().chai_select_representatives(_ptr(features), _ptr(membership), B, H, F, k, _ptr(reps), _stream()))
    return reps


def chai_compact_k_cache(k_full, reps, T: int | None = None, k_rep=None):
    """k_full [B,H,T_cap,D], reps [B,k] -> k_rep [B,k,T_cap,D] (rows [0,T) of each slot are written)."""
    _dev(k_full, reps, k_rep)
    B, H, T_cap, D = k_full.shape
    k = reps.shape[1]
    T = T_cap if T is None else T
    if k_rep is None:
        k_rep = torch.empty((B, k, T_cap, D), device=k_full.device, dtype=k_full.dtype)
    _check(load().chai_compact_k_cache(_ptr(k_full), _ptr(k_rep), _ptr(reps), B, H, k, T, T_cap, D, _dt(k_full),
                                       _stream()))
    return k_rep


def new_workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty((max(int(nbytes), 256),), device=device, dtype=torch.uint8)


def chai_decode_attention(q, k_rep, v, membership, reps, scale: float, T: int | None = None, out=None,
                          workspace=None):
    """q [B,H,D], k_rep [B,k,T_cap,D], v [B,H,T_cap,D], membership [B,H], reps [B,k] -> out [B,H,D]."""
    _dev(q, k_rep, v, membership, reps, out, workspace)
    B, H, D = q.shape
    k, T_cap = k_rep.shape[1], k_rep.shape[2]
    T = T_cap if T is None else T
    dt = _dt(q)
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        workspace = new_workspace(chai_decode_workspace_bytes(B, H, k, T, D, dt), q.device)
    _check(load().chai_decode_attention(_ptr(q), _ptr(k_rep), _ptr(v), _ptr(membership), _ptr(reps), _ptr(out), B,
                                        H, k, T, T_cap, D, scale, dt, _ptr(workspace), workspace.numel(),
                                        _stream()))
    return out


def chai_decode_attention_static(q, k_rep, v, membership, reps, scale: float, T: int | None = None, out=None):
    """Decode step that uses the library's built-in 8 MiB scratch array: for callers that cannot pass
    a workspace and must not allocate (all HBM already committed to a cache pool, or no allocation
    allowed on the hot loop).  Problems needing more scratch raise ChaiError(CHAI_ERR_WORKSPACE).
    `out` must be supplied by such callers; it is created here only for convenience in tests."""
    _dev(q, k_rep, v, membership, reps, out)
    B, H, D = q.shape
    k, T_cap = k_rep.shape[1], k_rep.shape[2]
    T = T_cap if T is None else T
    if out is None:
        out = torch.empty_like(q)
    _check(load().chai_decode_attention_static(_ptr(q), _ptr(k_rep), _ptr(v), _ptr(membership), _ptr(reps),
                                               _ptr(out), B, H, k, T, T_cap, D, scale, _dt(q), _stream()))
    return out


def chai_decode_attention_ragged(q, k_rep, v, membership, reps, seq_lens, scale: float, T_max: int, k_planes=None,
                                 out=None, workspace=None):
    """Ragged batch: seq_lens [B] int32 (device) gives each request's cached positions, T_max bounds them.
    k_rep is [B,k,T_cap,D], or (k_planes=k) a full [B,H,T_cap,D] cache whose first k planes hold the
    representatives (after chai_compact_k_cache_inplace)."""
    _dev(q, k_rep, v, membership, reps, seq_lens, out, workspace)
    B, H, D = q.shape
    k = reps.shape[1] if k_planes is None else k_planes
    T_cap = k_rep.shape[2]
    stride = k_rep.shape[1] * T_cap * D
    dt = _dt(q)
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        workspace = new_workspace(chai_decode_workspace_bytes(B, H, k, T_max, D, dt), q.device)
    _check(load().chai_decode_attention_ragged(_ptr(q), _ptr(k_rep), _ptr(v), _ptr(membership), _ptr(reps),
                                               _ptr(seq_lens), _ptr(out), B, H, k, T_max, T_cap, D, stride, scale, dt,
                                               _ptr(workspace), workspace.numel(), _stream()))
    return out


def chai_append_kv(k_new, v_new, k_rep, v, reps, seq_lens, advance: bool = True, workspace=None):
    """One new token per request: k_rep[b][c][seq_lens[b]] = k_new[b][reps[b][c]], v[b][h][seq_lens[b]] = v_new[b][h];
    seq_lens is incremented afterwards when `advance`.  k_rep may be the full cache compacted in place."""
    _dev(k_new, v_new, k_rep, v, reps, seq_lens, workspace)
    B, H, D = k_new.shape
    k, T_cap = reps.shape[1], v.shape[2]
    stride = k_rep.shape[1] * T_cap * D
    _check(load().chai_append_kv(_ptr(k_new), _ptr(v_new), _ptr(k_rep), _ptr(v), _ptr(reps), _ptr(seq_lens), B, H, k,
                                 T_cap, D, stride, _dt(k_new), int(bool(advance)), _ptr(workspace), _stream()))


def chai_compact_k_cache_inplace(k_cache, reps, T: int | None = None, workspace=None):
    """k_cache [B,H,T_cap,D]: planes 0..k-1 of each request receive the representatives' keys (rows [0,T))."""
    _dev(k_cache, reps, workspace)
    B, H, T_cap, D = k_cache.shape
    k = reps.shape[1]
    T = T_cap if T is None else T
    _check(load().chai_compact_k_cache_inplace(_ptr(k_cache), _ptr(reps), B, H, k, T, T_cap, D, _dt(k_cache),
                                               _ptr(workspace), _stream()))
    return k_cache


def _decode_host(fn_name, q_host, out_host, q_stage, out_stage, k_rep, v, membership, reps, scale, workspace, T):
    _dev(q_stage, out_stage, k_rep, v, membership, reps, workspace)
    B, H, D = q_host.shape
    k, T_cap = k_rep.shape[1], k_rep.shape[2]
    T = T_cap if T is None else T
    _check(getattr(load(), fn_name)(q_host.data_ptr(), out_host.data_ptr(), _ptr(q_stage), _ptr(out_stage),
                                    _ptr(k_rep), _ptr(v), _ptr(membership), _ptr(reps), B, H, k, T, T_cap, D, scale,
                                    _dt(q_host), _ptr(workspace), workspace.numel(), _stream()))
    return out_host


def chai_decode_attention_host(q_host, out_host, q_stage, out_stage, k_rep, v, membership, reps, scale: float,
                               workspace, T: int | None = None):
    """Decode step with q / out in (pinned) host memory; returns after the stream has drained."""
    return _decode_host("chai_decode_attention_host", q_host, out_host, q_stage, out_stage, k_rep, v, membership,
                        reps, scale, workspace, T)


def chai_decode_attention_host_async(q_host, out_host, q_stage, out_stage, k_rep, v, membership, reps, scale: float,
                                     workspace, T: int | None = None):
    """As above but only enqueued on the current stream: out_host is valid after the caller synchronises it."""
    return _decode_host("chai_decode_attention_host_async", q_host, out_host, q_stage, out_stage, k_rep, v,
                        membership, reps, scale, workspace, T)


def chai_decode_attention_host_streams(q_host, out_host, q_stage, out_stage, k_rep, v, membership, reps, scale: float,
                                       workspace, stream, upload_stream, download_stream, uploaded_event,
                                       computed_event, T: int | None = None):
    """Host-buffer decode step over three torch streams and two torch events (see the header); nothing is
    synchronised here: out_host is valid once download_stream has drained."""
    _dev(q_stage, out_stage, k_rep, v, membership, reps, workspace)
    B, H, D = q_host.shape
    k, T_cap = k_rep.shape[1], k_rep.shape[2]
    T = T_cap if T is None else T
    # a torch event has no CUDA handle before its first record: record once where it does no harm
    for ev, st in ((uploaded_event, upload_stream), (computed_event, stream)):
        if not ev.cuda_event:
            ev.record(st)
    _check(load().chai_decode_attention_host_streams(
        q_host.data_ptr(), out_host.data_ptr(), _ptr(q_stage), _ptr(out_stage), _ptr(k_rep), _ptr(v), _ptr(membership),
        _ptr(reps), B, H, k, T, T_cap, D, scale, _dt(q_host), _ptr(workspace), workspace.numel(), stream.cuda_stream,
        upload_stream.cuda_stream, download_stream.cuda_stream, uploaded_event.cuda_event, computed_event.cuda_event))
    return out_host


def _prefill(fn_name, q, k_rep, v, membership, reps, scale, causal, out, workspace):
    _dev(q, k_rep, v, membership, reps, out, workspace)
    B, H, T, D = q.shape
    k = k_rep.shape[1]
    dt = _dt(q)
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        workspace = new_workspace(chai_prefill_workspace_bytes(B, H, k, T, D, dt), q.device)
    _check(getattr(load(), fn_name)(_ptr(q), _ptr(k_rep), _ptr(v), _ptr(membership), _ptr(reps), _ptr(out), B, H, k,
                                    T, D, scale, int(bool(causal)), dt, _ptr(workspace), workspace.numel(),
                                    _stream()))
    return out


def _prefill_from(fn_name, q, k_rep, v, membership, reps, scale, q_start, causal, out, workspace):
    _dev(q, k_rep, v, membership, reps, out, workspace)
    B, H, T, D = q.shape
    k = k_rep.shape[1]
    dt = _dt(q)
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        workspace = new_workspace(chai_prefill_workspace_bytes(B, H, k, T, D, dt), q.device)
    _check(getattr(load(), fn_name)(_ptr(q), _ptr(k_rep), _ptr(v), _ptr(membership), _ptr(reps), _ptr(out), B, H, k,
                                    T, int(q_start), D, scale, int(bool(causal)), dt, _ptr(workspace),
                                    workspace.numel(), _stream()))
    return out


def chai_prefill_attention_from(q, k_rep, v, membership, reps, scale: float, q_start: int, causal: bool = True,
                                out=None, workspace=None):
    """Rows [q_start, T) of the clustered prefill; rows before q_start of `out` are left untouched."""
    return _prefill_from("chai_prefill_attention_from", q, k_rep, v, membership, reps, scale, q_start, causal, out,
                         workspace)


def chai_prefill_attention_simt_from(q, k_rep, v, membership, reps, scale: float, q_start: int, causal: bool = True,
                                     out=None, workspace=None):
    return _prefill_from("chai_prefill_attention_simt_from", q, k_rep, v, membership, reps, scale, q_start, causal, out,
                         workspace)


def chai_prefill_attention(q, k_rep, v, membership, reps, scale: float, causal: bool = True, out=None,
                           workspace=None):
    """q [B,H,T,D], k_rep [B,k,T,D], v [B,H,T,D] -> out [B,H,T,D]."""
    return _prefill("chai_prefill_attention", q, k_rep, v, membership, reps, scale, causal, out, workspace)


def chai_prefill_attention_simt(q, k_rep, v, membership, reps, scale: float, causal: bool = True, out=None,
                                workspace=None):
    return _prefill("chai_prefill_attention_simt", q, k_rep, v, membership, reps, scale, causal, out, workspace)


def chai_decode_attention_qkv(q, k_rep, v_rep, membership, reps, scale: float, T: int | None = None, seq_lens=None,
                              out=None, workspace=None):
    """CHAI-QKV decode: q [B,H,D], k_rep / v_rep [B,k,T_cap,D] -> out [B,H,D] (a member's row = its cluster's)."""
    _dev(q, k_rep, v_rep, membership, reps, seq_lens, out, workspace)
    B, H, D = q.shape
    k, T_cap = k_rep.shape[1], k_rep.shape[2]
    T = T_cap if T is None else T
    dt = _dt(q)
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        workspace = new_workspace(int(load().chai_decode_qkv_workspace_bytes(B, H, k, T, D, dt)), q.device)
    _check(load().chai_decode_attention_qkv(_ptr(q), _ptr(k_rep), _ptr(v_rep), _ptr(membership), _ptr(reps),
                                            _ptr(seq_lens), _ptr(out), B, H, k, T, T_cap, D, scale, dt, _ptr(workspace),
                                            workspace.numel(), _stream()))
    return out


def chai_prefill_attention_qkv(q, k_rep, v_rep, membership, reps, scale: float, causal: bool = True, q_start: int = 0,
                               out=None, workspace=None):
    """CHAI-QKV prefill: q [B,H,T,D], k_rep / v_rep [B,k,T,D] -> out [B,H,T,D]."""
    _dev(q, k_rep, v_rep, membership, reps, out, workspace)
    B, H, T, D = q.shape
    k = k_rep.shape[1]
    dt = _dt(q)
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        workspace = new_workspace(int(load().chai_prefill_qkv_workspace_bytes(B, H, k, T, D, dt)), q.device)
    _check(load().chai_prefill_attention_qkv(_ptr(q), _ptr(k_rep), _ptr(v_rep), _ptr(membership), _ptr(reps), _ptr(out),
                                             B, H, k, T, int(q_start), D, scale, int(bool(causal)), dt, _ptr(workspace),
                                             workspace.numel(), _stream()))
    return out


def chai_broadcast_membership(membership_static, reps_static, B: int):
    """One membership [H] / reps [k] for every request -> ([B,H], [B,k]) int32 (CHAI-static)."""
    _dev(membership_static, reps_static)
    H, k = membership_static.numel(), reps_static.numel()
    dev = membership_static.device
    membership = torch.empty((B, H), device=dev, dtype=torch.int32)
    reps = torch.empty((B, k), device=dev, dtype=torch.int32)
    _check(load().chai_broadcast_membership(_ptr(membership_static), _ptr(reps_static), _ptr(membership), _ptr(reps), B,
                                            H, k, _stream()))
    return membership, reps


def chai_quantize_cache_fp8(cache, T: int | None = None):
    """cache [B,P,T_cap,D] bf16 -> (bytes [B,P,T_cap,D] uint8 in e4m3, scales [B,P] fp32); rows [0,T) are converted."""
    _dev(cache)
    if cache.dtype != torch.bfloat16:
        raise TypeError("the cache must be bfloat16")
    B, P, T_cap, D = cache.shape
    T = T_cap if T is None else T
    q8 = torch.zeros((B, P, T_cap, D), device=cache.device, dtype=torch.uint8)
    scales = torch.empty((B, P), device=cache.device, dtype=torch.float32)
    _check(load().chai_quantize_cache_fp8(_ptr(cache), _ptr(q8), _ptr(scales), B * P, T, T_cap, D, _stream()))
    return q8, scales


def chai_decode_attention_fp8(q, k_rep8, v8, k_scale, v_scale, membership, reps, scale: float, T: int | None = None,
                              seq_lens=None, out=None, workspace=None):
    """Decode on e4m3 caches: q [B,H,D] bf16, k_rep8 [B,k|H,T_cap,D] uint8, v8 [B,H,T_cap,D] uint8, scales fp32."""
    _dev(q, k_rep8, v8, k_scale, v_scale, membership, reps, seq_lens, out, workspace)
    B, H, D = q.shape
    k, T_cap = reps.shape[1], v8.shape[2]
    T = T_cap if T is None else T
    stride = k_rep8.shape[1] * T_cap * D
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        workspace = new_workspace(int(load().chai_decode_fp8_workspace_bytes(B, H, k, T, D)), q.device)
    _check(load().chai_decode_attention_fp8(_ptr(q), _ptr(k_rep8), _ptr(v8), _ptr(k_scale), _ptr(v_scale),
                                            _ptr(membership), _ptr(reps), _ptr(seq_lens), _ptr(out), B, H, k, T, T_cap, D,
                                            stride, scale, _ptr(workspace), workspace.numel(), _stream()))
    return out


# ---- paged caches -----------------------------------------------------------------------------------------------

_PAGED_IO = {torch.float32: CHAI_F32, torch.bfloat16: CHAI_BF16}


def _paged_call(fn, dev: int, *args) -> None:
    """Calls fn(*args, stream) on the device that the tensors live on, on that device's current stream."""
    if dev == _current_device():
        rc = fn(*args, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, _raw_stream(dev))
    if rc:
        _check(rc)


# (torch.cuda.current_stream builds a Stream object, which costs as much as a launch)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)


def _want(t, name, shape, dtype, dev) -> None:
    if t.shape == shape and t.dtype is dtype and t.get_device() == dev and t.is_contiguous():
        return
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    raise ValueError(f"{name} must be contiguous and on cuda:{dev}")


_E4M3 = (torch.uint8, torch.float8_e4m3fn)


def _pool_shapes(k_pages, v_pages, k_scales, v_scales):
    """Checks a pool; returns (n_pages, k, H, page_size, D, page strides, device index)."""
    if k_pages.dim() != 4 or v_pages.dim() != 4:
        raise ValueError("k_pages must be [n_pages,k,page_size,D] and v_pages [n_pages,H,page_size,D]")
    n, k, ps, D = k_pages.shape
    n_v, H, ps_v, D_v = v_pages.shape
    if n_v != n or ps_v != ps or D_v != D:
        raise ValueError("k_pages and v_pages must agree in pages, page size and head dimension")
    dev = k_pages.get_device()
    if dev < 0 or v_pages.get_device() != dev:
        raise ValueError("the pages must be CUDA tensors on one device")
    if k_pages.is_contiguous() and v_pages.is_contiguous():
        k_stride = v_stride = 0
    else:
        if n > 0 and not (k_pages[0].is_contiguous() and v_pages[0].is_contiguous()):
            raise ValueError("every page must be contiguous (pages may be any distance apart)")
        k_stride, v_stride = (k_pages.stride(0), v_pages.stride(0)) if n > 1 else (0, 0)
        if n > 1 and (k_stride < k * ps * D or v_stride < H * ps * D):
            raise ValueError("pages must not overlap")
    if k_scales is None:
        dtype = k_pages.dtype
        if v_pages.dtype is not dtype or dtype not in _PAGED_IO:
            raise TypeError("k_pages and v_pages must both be float32 or both bfloat16")
    else:
        if k_pages.dtype not in _E4M3 or v_pages.dtype not in _E4M3:
            raise TypeError(f"e4m3 pages must be uint8 or float8_e4m3fn, got {k_pages.dtype} and {v_pages.dtype}")
        _want(k_scales, "k_scales", (n, k, ps), torch.float32, dev)
        _want(v_scales, "v_scales", (n, H, ps), torch.float32, dev)
    return n, k, H, ps, D, k_stride, v_stride, dev


def _pages(k_pages, v_pages, k_scales, v_scales, block_table, seq_lens):
    """Checks a pool and its tables; returns (n_pages, k, H, page_size, D, page strides, B, max_pages, device index)."""
    n, k, H, ps, D, k_stride, v_stride, dev = _pool_shapes(k_pages, v_pages, k_scales, v_scales)
    if block_table.dim() != 2:
        raise ValueError("block_table must be [B,max_pages]")
    B, max_pages = block_table.shape
    _want(block_table, "block_table", (B, max_pages), torch.int32, dev)
    _want(seq_lens, "seq_lens", (B,), torch.int32, dev)
    return n, k, H, ps, D, k_stride, v_stride, B, max_pages, dev


def _paged_workspace(workspace, dev):
    """(pointer, bytes) of a workspace, which may be None."""
    if workspace is None:
        return None, 0
    if workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace must be contiguous and on cuda:{dev}")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _append_paged(fn_name, k_new, v_new, k_pages, v_pages, k_scales, v_scales, reps, block_table, seq_lens, new_lens,
                  advance, workspace):
    n, k, H, ps, D, k_stride, v_stride, B, max_pages, dev = _pages(k_pages, v_pages, k_scales, v_scales, block_table,
                                                                      seq_lens)
    N = k_new.shape[2] if k_new.dim() == 4 else 1
    io = _PAGED_IO.get(k_new.dtype)
    if io is None or (k_scales is None and k_new.dtype is not k_pages.dtype):
        raise TypeError(f"k_new of type {k_new.dtype} does not go into pages of type {k_pages.dtype}")
    shape = (B, H, N, D) if k_new.dim() == 4 else (B, H, D)
    _want(k_new, "k_new", shape, k_new.dtype, dev)
    _want(v_new, "v_new", shape, k_new.dtype, dev)
    _want(reps, "reps", (B, k), torch.int32, dev)
    if new_lens is not None:
        _want(new_lens, "new_lens", (B,), torch.int32, dev)
    ws, ws_bytes = _paged_workspace(workspace, dev)
    if workspace is not None and ws_bytes < 256:
        raise ValueError("workspace must hold at least 256 bytes")
    scales = () if k_scales is None else (k_scales.data_ptr(), v_scales.data_ptr())
    _paged_call(getattr(load(), fn_name), dev, k_new.data_ptr(), v_new.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
                *scales, reps.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(), _ptr(new_lens), B, H, k, N, n, ps,
                max_pages, D, k_stride, v_stride, io, 1 if advance else 0, ws)


def chai_append_kv_paged(k_new, v_new, k_pages, v_pages, reps, block_table, seq_lens, new_lens=None, advance: bool = True,
                         workspace=None):
    """New tokens into a paged cache: k_new, v_new [B,H,N,D] (or [B,H,D] for one token each) go to the positions
    seq_lens[b] .. of their request's pages, keys of representatives only; new_lens [B] says how many of the N tokens
    each request has.  seq_lens grows by them when `advance`.  k_pages [n_pages,k,page_size,D] and
    v_pages [n_pages,H,page_size,D] may lie side by side in one pool (any distance between pages)."""
    _append_paged("chai_append_kv_paged", k_new, v_new, k_pages, v_pages, None, None, reps, block_table, seq_lens, new_lens,
                  advance, workspace)


def chai_append_kv_paged_fp8(k_new, v_new, k_pages, v_pages, k_scales, v_scales, reps, block_table, seq_lens, new_lens=None,
                             advance: bool = True, workspace=None):
    """The same into e4m3 pages (uint8 or float8_e4m3fn) with one fp32 power-of-two scale per row: k_scales
    [n_pages,k,page_size], v_scales [n_pages,H,page_size]; k_new / v_new float32 or bfloat16."""
    _append_paged("chai_append_kv_paged_fp8", k_new, v_new, k_pages, v_pages, k_scales, v_scales, reps, block_table,
                  seq_lens, new_lens, advance, workspace)


def _read_paged(fn_name, k_pages, v_pages, k_scales, v_scales, block_table, seq_lens, T_out, dtype, k_out, v_out, workspace):
    n, k, H, ps, D, k_stride, v_stride, B, max_pages, dev = _pages(k_pages, v_pages, k_scales, v_scales, block_table,
                                                                      seq_lens)
    given = k_out if k_out is not None else v_out
    if given is None:
        if T_out is None:
            raise ValueError("give T_out, or the arrays to read into")
        k_out = torch.zeros((B, k, T_out, D), device=k_pages.device, dtype=dtype)
        v_out = torch.zeros((B, H, T_out, D), device=k_pages.device, dtype=dtype)
        given = k_out
    if given.dim() != 4:
        raise ValueError("k_out must be [B,k,T_out,D] and v_out [B,H,T_out,D]")
    if T_out is not None and given.shape[2] != T_out:
        raise ValueError("T_out differs from the length of the arrays to read into")
    T_out = given.shape[2]
    io = _PAGED_IO.get(given.dtype)
    if io is None or (k_scales is None and given.dtype is not k_pages.dtype):
        raise TypeError(f"pages of type {k_pages.dtype} are not read into arrays of type {given.dtype}")
    if k_out is not None:
        _want(k_out, "k_out", (B, k, T_out, D), given.dtype, dev)
    if v_out is not None:
        _want(v_out, "v_out", (B, H, T_out, D), given.dtype, dev)
    ws, ws_bytes = _paged_workspace(workspace, dev)
    if workspace is not None and ws_bytes < 256:
        raise ValueError("workspace must hold at least 256 bytes")
    scales = () if k_scales is None else (k_scales.data_ptr(), v_scales.data_ptr())
    _paged_call(getattr(load(), fn_name), dev, k_pages.data_ptr(), v_pages.data_ptr(), *scales, block_table.data_ptr(),
                seq_lens.data_ptr(), _ptr(k_out), _ptr(v_out), B, H, k, T_out, n, ps, max_pages, D, k_stride, v_stride, io,
                ws)
    return k_out, v_out


def chai_read_kv_paged(k_pages, v_pages, block_table, seq_lens, T_out: int | None = None, k_out=None, v_out=None,
                       workspace=None):
    """Rows [0, min(seq_lens[b], T_out)) of a paged cache -> (k_out [B,k,T_out,D], v_out [B,H,T_out,D]).  Rows behind
    them are left as they were (zeros in arrays made here).  With only one of k_out / v_out given only that is read."""
    return _read_paged("chai_read_kv_paged", k_pages, v_pages, None, None, block_table, seq_lens, T_out, k_pages.dtype,
                       k_out, v_out, workspace)


def chai_read_kv_paged_fp8(k_pages, v_pages, k_scales, v_scales, block_table, seq_lens, T_out: int | None = None,
                           dtype=torch.bfloat16, k_out=None, v_out=None, workspace=None):
    """The same from e4m3 pages: each row's numbers times its scale, rounded to `dtype` (the type of arrays given)."""
    return _read_paged("chai_read_kv_paged_fp8", k_pages, v_pages, k_scales, v_scales, block_table, seq_lens, T_out, dtype,
                       k_out, v_out, workspace)


def chai_decode_paged_workspace_bytes(B, H, D) -> int:
    return int(load().chai_decode_paged_workspace_bytes(B, H, D))


def _decode_paged(fn_name, q, k_pages, v_pages, k_scales, v_scales, membership, reps, block_table, seq_lens, scale, out,
                  workspace):
    n, k, H, ps, D, k_stride, v_stride, B, max_pages, dev = _pages(k_pages, v_pages, k_scales, v_scales, block_table,
                                                                      seq_lens)
    io = _PAGED_IO.get(q.dtype)
    if io is None or (k_scales is None and q.dtype is not k_pages.dtype):
        raise TypeError(f"queries of type {q.dtype} do not go with pages of type {k_pages.dtype}")
    _want(q, "q", (B, H, D), q.dtype, dev)
    _want(membership, "membership", (B, H), torch.int32, dev)
    _want(reps, "reps", (B, k), torch.int32, dev)
    if out is None:
        out = torch.empty_like(q)
    else:
        _want(out, "out", (B, H, D), q.dtype, dev)
    if workspace is None:
        workspace = new_workspace(chai_decode_paged_workspace_bytes(B, H, D), q.device)
    ws, ws_bytes = _paged_workspace(workspace, dev)
    scales = () if k_scales is None else (k_scales.data_ptr(), v_scales.data_ptr())
    _paged_call(getattr(load(), fn_name), dev, q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), *scales,
                membership.data_ptr(), reps.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(), out.data_ptr(), B, H, k,
                n, ps, max_pages, D, k_stride, v_stride, scale, io, ws, ws_bytes)
    return out


def chai_decode_attention_paged(q, k_pages, v_pages, membership, reps, block_table, seq_lens, scale: float, out=None,
                                workspace=None):
    """Decode over a paged cache: q [B,H,D], k_pages [n_pages,k,page_size,D], v_pages [n_pages,H,page_size,D] of q's
    type, block_table [B,max_pages] and seq_lens [B] int32 -> out [B,H,D].  A request of length 0 gets zeros."""
    return _decode_paged("chai_decode_attention_paged", q, k_pages, v_pages, None, None, membership, reps, block_table,
                         seq_lens, scale, out, workspace)


def chai_decode_attention_paged_fp8(q, k_pages, v_pages, k_scales, v_scales, membership, reps, block_table, seq_lens,
                                    scale: float, out=None, workspace=None):
    """The same over e4m3 pages with one scale per row, as chai_append_kv_paged_fp8 writes them; q float32 or bfloat16."""
    return _decode_paged("chai_decode_attention_paged_fp8", q, k_pages, v_pages, k_scales, v_scales, membership, reps,
                         block_table, seq_lens, scale, out, workspace)


# ---- a serving step of many tokens ------------------------------------------------------------------------------

def chai_plan_paged(seq_lens, new_lens, block_table, free_pages, free_count, n_tokens: int, page_size: int, kv_lens=None,
                    free_count_out=None, token_start=None, token_request=None, positions=None, slots=None, workspace=None):
    """Pages for a step's tokens, from a stack of free pages: seq_lens [B] (cached positions), new_lens [B] (tokens that each
    request gets; below 0: it ends and its pages go back), block_table [B,max_pages] and free_pages [n_pages] (both written),
    free_count [1], all int32 -> (kv_lens [B], token_start [B+1], token_request [n_tokens], positions [n_tokens], slots
    [n_tokens] int64).  kv_lens may be seq_lens; free_count is updated in place unless free_count_out is given.  Pages that an
    ending request shares with any other must not be given back here: nothing counts who has a page."""
    if block_table.dim() != 2 or free_pages.dim() != 1:
        raise ValueError("block_table must be [B,max_pages] and free_pages [n_pages]")
    (B, max_pages), n_pages, dev = block_table.shape, free_pages.shape[0], block_table.get_device()
    if dev < 0:
        raise ValueError("tensors must be contiguous CUDA tensors")
    i32 = torch.int32
    _want(block_table, "block_table", (B, max_pages), i32, dev)
    _want(free_pages, "free_pages", (n_pages,), i32, dev)
    _want(free_count, "free_count", (1,), i32, dev)
    _want(seq_lens, "seq_lens", (B,), i32, dev)
    _want(new_lens, "new_lens", (B,), i32, dev)
    if free_count_out is None:
        free_count_out = free_count
    else:
        _want(free_count_out, "free_count_out", (1,), i32, dev)
    like = block_table.device
    if kv_lens is None:
        kv_lens = torch.empty((B,), device=like, dtype=i32)
    else:
        _want(kv_lens, "kv_lens", (B,), i32, dev)
    if token_start is None:
        token_start = torch.empty((B + 1,), device=like, dtype=i32)
    else:
        _want(token_start, "token_start", (B + 1,), i32, dev)
    if token_request is None:
        token_request = torch.empty((n_tokens,), device=like, dtype=i32)
    else:
        _want(token_request, "token_request", (n_tokens,), i32, dev)
    if positions is None:
        positions = torch.empty((n_tokens,), device=like, dtype=i32)
    else:
        _want(positions, "positions", (n_tokens,), i32, dev)
    if slots is None:
        slots = torch.empty((n_tokens,), device=like, dtype=torch.int64)
    else:
        _want(slots, "slots", (n_tokens,), torch.int64, dev)
    if workspace is None:
        workspace = new_workspace(512 + 4 * B, like)
    ws, ws_bytes = _paged_workspace(workspace, dev)
    _paged_call(load().chai_plan_paged, dev, seq_lens.data_ptr(), new_lens.data_ptr(), block_table.data_ptr(),
                free_pages.data_ptr(), free_count.data_ptr(), free_count_out.data_ptr(), kv_lens.data_ptr(),
                token_start.data_ptr(), token_request.data_ptr(), positions.data_ptr(), slots.data_ptr(), B, n_tokens, n_pages,
                page_size, max_pages, ws, ws_bytes)
    return kv_lens, token_start, token_request, positions, slots


ROPE_SCALINGS = {"plain": 0, "linear": 1, "base": 2, "ramp": 3, "bands": 4}   # CHAI_ROPE_*


def chai_rope_frequencies(rot: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0, context: float = 0.0,
                          low: float = 1.0, high: float | None = None, device=None):
    """Frequencies of rotary positions: (turns [rot/2] float64 on `device`, the magnitude that goes with them).  scaling:
    "plain", "linear", "base", "ramp" (high 32 unless given) or "bands" (high 4 unless given); see the header."""
    if scaling not in ROPE_SCALINGS:
        raise ValueError(f"scaling must be one of {sorted(ROPE_SCALINGS)}")
    if high is None:
        high = 32.0 if scaling == "ramp" else 4.0
    turns = torch.empty((max(int(rot) // 2, 1),), dtype=torch.float64)
    magnitude = ctypes.c_double(1.0)
    _check(load().chai_rope_frequencies(turns.data_ptr(), ctypes.addressof(magnitude), rot, ROPE_SCALINGS[scaling],
                                        (ctypes.c_double * 5)(base, factor, context, low, high)))
    return (turns if device is None else turns.to(device)), magnitude.value


def _double(x: float):
    return ctypes.byref(ctypes.c_double(x))


def _turns(turns, dev):
    """(pointer, rot) of the frequencies, which may be None."""
    if turns is None:
        return None, 0
    _want(turns, "turns", (turns.numel(),), torch.float64, dev)
    return turns.data_ptr(), 2 * turns.numel()


def _rotated_like(x):
    """A dense array with x's rows in their order in memory; in that of the indexes where one row stands for many."""
    if x.is_contiguous():
        return torch.empty_like(x)
    shape, strides = x.shape, x.stride()
    _, H, N, D = shape
    if 0 in strides:
        return torch.empty(shape, device=x.device, dtype=x.dtype)
    if strides != (N * H * D, D, H * D, 1):   # (tokens before heads: as it is)
        dense, apart = [0, 0, 0, 1], D
        for i in sorted((0, 1, 2), key=lambda i: (strides[i], shape[i])):
            dense[i] = apart
            apart *= shape[i]
        strides = dense
    return torch.empty_strided(shape, strides, device=x.device, dtype=x.dtype)


_STRIDES = struct.Struct("12q")   # (an array of ctypes takes four times as long to fill)


def chai_rope(q, k=None, positions=None, turns=None, magnitude: float = 1.0, interleaved: bool = False, q_out=None, k_out=None):
    """q [B,Hq,N,D] and k [B,Hk,N,D] (or None) rotated by positions [B,N] int32 (None: 0 .. N-1) -> (q_out, k_out), new dense
    arrays with rows in the order of the input's unless given (they may be q and k themselves).  Any strides with contiguous
    rows, e.g. x.transpose(1, 2) of [B,N,H,D], or of a part of one projection's output."""
    if q.dim() != 4:
        raise ValueError("q must be [B,Hq,N,D]")
    B, Hq, N, D = q.shape
    dev = q.get_device()
    if dev < 0:
        raise ValueError("q must be a CUDA tensor")
    dtype = q.dtype
    io = _PAGED_IO.get(dtype)
    if io is None:
        raise TypeError(f"unsupported dtype {dtype}")
    Hk = 0
    if k is not None:
        if k.dim() != 4 or k.shape[0] != B or k.shape[2] != N or k.shape[3] != D:
            raise ValueError(f"k must have shape ({B}, Hk, {N}, {D}), got {tuple(k.shape)}")
        Hk = k.shape[1]
    if q_out is None:
        q_out = _rotated_like(q)
    if k_out is None and k is not None:
        k_out = _rotated_like(k)
    strides = []
    for x, out, name in ((q, q_out, "q"), (k, k_out, "k")):
        if x is None:
            strides += [0] * 6
            continue
        if x.dtype is not dtype or out.dtype is not dtype:
            raise TypeError(f"{name} and its output must be {dtype}")
        if out.shape != x.shape or x.get_device() != dev or out.get_device() != dev or x.stride(3) != 1 or out.stride(3) != 1:
            raise ValueError(f"{name} and its output must have one shape, rows without gaps, and be on cuda:{dev}")
        strides += x.stride()[:3] + out.stride()[:3]
    if positions is not None:
        _want(positions, "positions", (B, N), torch.int32, dev)
    if turns is None:
        raise ValueError("give the frequencies (chai_rope_frequencies)")
    at, rot = _turns(turns, dev)
    _paged_call(load().chai_rope, dev, q.data_ptr(), _ptr(k), q_out.data_ptr(), _ptr(k_out), _ptr(positions), at, B, Hq, Hk, N,
                D, rot, 1 if interleaved else 0, _double(magnitude), _STRIDES.pack(*strides), io)
    return q_out, k_out


def _tokens(t, name, shape, dtype, dev) -> int:
    """Checks a packed [n_tokens,H,D] array whose tokens may lie further apart; returns the distance in elements."""
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    apart, heads, one = t.stride()
    if t.get_device() != dev or one != 1 or (heads != shape[2] and shape[1] > 1):
        raise ValueError(f"{name} must be on cuda:{dev}, the heads of a token side by side")
    if shape[0] <= 1:
        return 0
    if apart < shape[1] * shape[2]:   # (0, one row for many tokens, would be taken for "side by side")
        raise ValueError(f"{name} must have rows of its own for every token, got a token stride of {apart}")
    return apart


def _append_rope(fn_name, q, k, v, k_pages, v_pages, k_scales, v_scales, reps, token_request, positions, slots, turns,
                 magnitude, interleaved, q_out, workspace):
    n, kp, H, ps, D, k_stride, v_stride, dev = _pool_shapes(k_pages, v_pages, k_scales, v_scales)
    io = _PAGED_IO.get(q.dtype)
    if io is None or (k_scales is None and q.dtype is not k_pages.dtype):
        raise TypeError(f"tokens of type {q.dtype} do not go into pages of type {k_pages.dtype}")
    n_tokens = q.shape[0]
    shape = (n_tokens, H, D)
    apart = [_tokens(t, name, shape, q.dtype, dev) for t, name in ((q, "q"), (k, "k"), (v, "v"))]
    if q_out is None:
        q_out = torch.zeros(shape, device=q.device, dtype=q.dtype)
    else:
        _want(q_out, "q_out", shape, q.dtype, dev)
    if reps.dim() != 2:
        raise ValueError("reps must be [B,k]")
    _want(reps, "reps", (reps.shape[0], kp), torch.int32, dev)
    _want(token_request, "token_request", (n_tokens,), torch.int32, dev)
    _want(positions, "positions", (n_tokens,), torch.int32, dev)
    _want(slots, "slots", (n_tokens,), torch.int64, dev)
    at, rot = _turns(turns, dev)
    ws, ws_bytes = _paged_workspace(workspace, dev)
    if workspace is not None and ws_bytes < 256:
        raise ValueError("workspace must hold at least 256 bytes")
    scales = () if k_scales is None else (k_scales.data_ptr(), v_scales.data_ptr())
    _paged_call(getattr(load(), fn_name), dev, q.data_ptr(), k.data_ptr(), v.data_ptr(), q_out.data_ptr(), k_pages.data_ptr(),
                v_pages.data_ptr(), *scales, reps.data_ptr(), token_request.data_ptr(), positions.data_ptr(), slots.data_ptr(),
                at, rot, 1 if interleaved else 0, _double(magnitude), reps.shape[0], H, kp, n_tokens, n, ps, D, *apart, k_stride,
                v_stride, io, ws)
    return q_out


def chai_append_rope_paged(q, k, v, k_pages, v_pages, reps, token_request, positions, slots, turns, magnitude: float = 1.0,
                           interleaved: bool = False, q_out=None, workspace=None):
    """A packed batch enters a paged cache: q, k, v [n_tokens,H,D] (they may be parts of one projection's output), where
    each token goes as chai_plan_paged says, turns from chai_rope_frequencies (None: no rotation).  Writes the rotated keys of
    representatives and all values, and returns q_out [n_tokens,H,D] with the representatives' queries rotated (other rows: as
    they were, zeros in an array made here)."""
    return _append_rope("chai_append_rope_paged", q, k, v, k_pages, v_pages, None, None, reps, token_request, positions, slots,
                        turns, magnitude, interleaved, q_out, workspace)


def chai_append_rope_paged_fp8(q, k, v, k_pages, v_pages, k_scales, v_scales, reps, token_request, positions, slots, turns,
                               magnitude: float = 1.0, interleaved: bool = False, q_out=None, workspace=None):
    """The same into e4m3 pages with one power-of-two scale per row (see chai_append_kv_paged_fp8)."""
    return _append_rope("chai_append_rope_paged_fp8", q, k, v, k_pages, v_pages, k_scales, v_scales, reps, token_request,
                        positions, slots, turns, magnitude, interleaved, q_out, workspace)


def chai_prefill_paged_workspace_bytes(B, H, n_tokens) -> int:
    return int(load().chai_prefill_paged_workspace_bytes(B, H, n_tokens))


def _prefill_paged(fn_name, q, k_pages, v_pages, k_scales, v_scales, membership, reps, block_table, kv_lens, token_start, scale,
                   causal, out, workspace):
    n, k, H, ps, D, k_stride, v_stride, dev = _pool_shapes(k_pages, v_pages, k_scales, v_scales)
    io = _PAGED_IO.get(q.dtype)
    if io is None or (k_scales is None and q.dtype is not k_pages.dtype):
        raise TypeError(f"queries of type {q.dtype} do not go with pages of type {k_pages.dtype}")
    if block_table.dim() != 2:
        raise ValueError("block_table must be [B,max_pages]")
    B, max_pages = block_table.shape
    i32 = torch.int32
    _want(block_table, "block_table", (B, max_pages), i32, dev)
    _want(kv_lens, "kv_lens", (B,), i32, dev)
    _want(token_start, "token_start", (B + 1,), i32, dev)
    _want(membership, "membership", (B, H), i32, dev)
    _want(reps, "reps", (B, k), i32, dev)
    n_tokens = q.shape[0]
    shape = (n_tokens, H, D)
    apart = _tokens(q, "q", shape, q.dtype, dev)
    if out is None:
        out = torch.zeros(shape, device=q.device, dtype=q.dtype)
    else:
        _want(out, "out", shape, q.dtype, dev)
    if workspace is None:
        workspace = new_workspace(chai_prefill_paged_workspace_bytes(B, H, n_tokens), q.device)
    ws, ws_bytes = _paged_workspace(workspace, dev)
    scales = () if k_scales is None else (k_scales.data_ptr(), v_scales.data_ptr())
    _paged_call(getattr(load(), fn_name), dev, q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), *scales,
                membership.data_ptr(), reps.data_ptr(), block_table.data_ptr(), kv_lens.data_ptr(), token_start.data_ptr(),
                out.data_ptr(), B, H, k, n_tokens, n, ps, max_pages, D, apart, k_stride, v_stride, scale, 1 if causal else 0, io,
                ws, ws_bytes)
    return out


def chai_prefill_attention_paged(q, k_pages, v_pages, membership, reps, block_table, kv_lens, token_start, scale: float,
                                 causal: bool = True, out=None, workspace=None):
    """Clustered attention of a packed batch over a paged cache: q [n_tokens,H,D], rows token_start[b] .. token_start[b+1]-1
    of request b, whose cached positions are kv_lens[b] with the new tokens last (causal), or all seen by every token
    -> out [n_tokens,H,D].  Rows behind token_start[B] are left as they were (zeros in an array made here)."""
    return _prefill_paged("chai_prefill_attention_paged", q, k_pages, v_pages, None, None, membership, reps, block_table, kv_lens,
                          token_start, scale, causal, out, workspace)


def chai_prefill_attention_paged_fp8(q, k_pages, v_pages, k_scales, v_scales, membership, reps, block_table, kv_lens,
                                     token_start, scale: float, causal: bool = True, out=None, workspace=None):
    """The same over e4m3 pages with one scale per row; q float32 or bfloat16."""
    return _prefill_paged("chai_prefill_attention_paged_fp8", q, k_pages, v_pages, k_scales, v_scales, membership, reps,
                          block_table, kv_lens, token_start, scale, causal, out, workspace)


def chai_set_decode_wait_limit_cycles(cycles: int) -> None:
    """Test hook: cycle limit of the decode kernel's device-side waits for the launches that follow (<= 0: default)."""
    load().chai_set_decode_wait_limit_cycles(int(cycles))


def chai_device_status(workspace) -> int:
    st = ctypes.c_int(0)
    _check(load().chai_device_status(_ptr(workspace), ctypes.byref(st), _stream()))
    return int(st.value)
