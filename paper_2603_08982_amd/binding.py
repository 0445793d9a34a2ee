"""ctypes binding of libsvgear.so: argument marshalling only.

Each function mirrors one entry point of include/svgear.h, allocates outputs and the
workspace with torch on the inputs' device, and enqueues the call on torch's current
stream. No arithmetic of the method happens here.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import os
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None

PROBE_PLAIN = 1
ROUTE_PER_ROW = 2
USE_GIVEN_SCORES = 4

EXPORTED_SYMBOLS = [
    "svgear_version", "svgear_last_hip_error",
    "svgear_kmeans_workspace", "svgear_kmeans", "svgear_kmeans_stepwise", "svgear_kmeans_list_threshold",
    "svgear_permute_workspace", "svgear_permute", "svgear_permute_rows",
    "svgear_permute_static_capacity", "svgear_permute_static",
    "svgear_probe_route_workspace", "svgear_probe_route", "svgear_probe_route_top_p",
    "svgear_sparse_attn_comp_workspace", "svgear_sparse_attn_comp", "svgear_sparse_attn_comp_token_order",
    "svgear_sparse_attn_two_stage_workspace", "svgear_sparse_attn_two_stage",
    "svgear_unpermute",
    "svgear_linear_workspace", "svgear_linear", "svgear_linear_backward_workspace", "svgear_linear_backward",
    "svgear_rotary", "svgear_rotary_backward_workspace", "svgear_rotary_backward",
    "svgear_layer_norm", "svgear_layer_norm_backward_workspace", "svgear_layer_norm_backward",
    "svgear_attention_workspace", "svgear_attention", "svgear_attention_backward_workspace", "svgear_attention_backward",
]

ACTIVATIONS = {"none": 0, "silu": 1, "gelu": 2, "gelu_tanh": 3}
ROTARY_NORMS = {None: 0, "head": 1, "token": 2}
ROTARY_HALVES = 4
ATTENTION_CAUSAL, ATTENTION_SHARED_DOCUMENTS = 1, 2

_c = ctypes
_vp, _i, _i64, _sz, _f, _u = _c.c_void_p, _c.c_int, _c.c_int64, _c.c_size_t, _c.c_float, _c.c_uint
_I64x2, _I64x3, _Ix3 = _c.c_int64 * 2, _c.c_int64 * 3, _c.c_int * 3


class SvgearError(RuntimeError):
    pass


def lib_path() -> str:
    return os.path.join(_HERE, "libsvgear.so")


def load_library():
    """Loads the built library; builds it first only if no built library exists."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = lib_path()
    if not os.path.exists(path):
        from .build import build

        build()
    lib = ctypes.CDLL(path)
    lib.svgear_version.restype = _i
    lib.svgear_last_hip_error.restype = _i
    lib.svgear_kmeans_workspace.restype = _sz
    lib.svgear_kmeans_workspace.argtypes = [_i, _i, _i64, _i, _i]
    lib.svgear_kmeans.restype = _i
    lib.svgear_kmeans.argtypes = [_vp, _vp, _i, _i, _i, _i64, _i64, _i, _c.POINTER(_c.c_int64), _i, _i,
                                  _vp, _vp, _vp, _vp, _vp, _sz, _vp]
    lib.svgear_kmeans_stepwise.restype = _i
    lib.svgear_kmeans_stepwise.argtypes = lib.svgear_kmeans.argtypes
    lib.svgear_permute_workspace.restype = _sz
    lib.svgear_permute_workspace.argtypes = [_i, _i, _i64, _i]
    lib.svgear_permute.restype = _i
    lib.svgear_permute.argtypes = [_vp, _i, _i, _i64, _i64, _i, _vp, _vp, _i, _c.POINTER(_vp),
                                   _c.POINTER(_I64x3), _c.POINTER(_vp), _i, _i, _vp, _sz, _vp]
    lib.svgear_permute_static_capacity.restype = _sz
    lib.svgear_permute_static_capacity.argtypes = []
    lib.svgear_permute_static.restype = _i
    lib.svgear_permute_static.argtypes = lib.svgear_permute.argtypes[:14] + [_vp]
    lib.svgear_permute_rows.restype = _i
    lib.svgear_permute_rows.argtypes = [_vp, _i, _i, _i64, _i, _c.POINTER(_vp), _c.POINTER(_I64x3), _c.POINTER(_vp),
                                        _i, _i, _vp]
    lib.svgear_probe_route_workspace.restype = _sz
    lib.svgear_probe_route_workspace.argtypes = [_i, _i, _i64, _i, _i, _i]
    lib.svgear_probe_route.restype = _i
    lib.svgear_probe_route.argtypes = [_vp, _vp, _vp, _vp, _vp, _i, _vp, _vp, _i, _i, _i64, _i64, _i, _i, _i,
                                       _i64, _f, _u, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
    lib.svgear_probe_route_top_p.restype = _i
    lib.svgear_probe_route_top_p.argtypes = [_vp, _vp, _vp, _vp, _vp, _i, _vp, _vp, _i, _i, _i64, _i64, _i, _i, _i,
                                             _f, _f, _u, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
    lib.svgear_sparse_attn_comp_workspace.restype = _sz
    lib.svgear_sparse_attn_comp_workspace.argtypes = [_i, _i, _i64, _i64, _i, _i, _i]
    lib.svgear_sparse_attn_comp.restype = _i
    lib.svgear_sparse_attn_comp.argtypes = [_vp, _vp, _vp, _i, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i64,
                                            _i64, _i, _i, _i, _f, _vp, _vp, _vp, _sz, _vp]
    lib.svgear_sparse_attn_comp_token_order.restype = _i
    lib.svgear_sparse_attn_comp_token_order.argtypes = [_vp, _c.POINTER(_c.c_int64), _vp, _vp, _i, _vp, _vp, _vp, _vp,
                                                        _vp, _vp, _vp, _vp, _i, _i, _i64, _i64, _i, _i, _i, _f, _vp,
                                                        _c.POINTER(_c.c_int64), _vp, _vp, _sz, _vp]
    lib.svgear_sparse_attn_two_stage_workspace.restype = _sz
    lib.svgear_sparse_attn_two_stage_workspace.argtypes = lib.svgear_sparse_attn_comp_workspace.argtypes
    lib.svgear_sparse_attn_two_stage.restype = _i
    lib.svgear_sparse_attn_two_stage.argtypes = lib.svgear_sparse_attn_comp.argtypes
    lib.svgear_unpermute.restype = _i
    lib.svgear_unpermute.argtypes = [_vp, _vp, _i, _i, _i, _i64, _i, _vp, _c.POINTER(_c.c_int64), _vp]
    lib.svgear_linear_workspace.restype = _sz
    lib.svgear_linear_workspace.argtypes = [_vp, _vp, _vp, _i64, _i, _i, _i64, _i, _i]
    lib.svgear_linear.restype = _i
    lib.svgear_linear.argtypes = [_vp, _vp, _vp, _i64, _vp, _i, _i, _i64, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                  _sz, _vp]
    lib.svgear_linear_backward_workspace.restype = _sz
    lib.svgear_linear_backward_workspace.argtypes = [_vp, _vp, _vp, _vp, _vp, _i64, _i, _i, _i64, _i, _i]
    lib.svgear_linear_backward.restype = _i
    lib.svgear_linear_backward.argtypes = [_vp, _vp, _vp, _vp, _vp, _i64, _vp, _i, _i, _i64, _i, _i, _i, _vp, _vp, _vp, _vp,
                                           _vp, _vp, _vp, _vp, _sz, _vp]
    # host arrays of pointers, strides, sections and sizes as plain addresses: ctypes checks less of them in each call
    places = [_vp, _vp, _vp, _i64, _vp, _i64, _u, _f]
    lib.svgear_rotary.restype = _i
    lib.svgear_rotary.argtypes = [_i, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i64, _i64, _i, *places, _vp]
    lib.svgear_rotary_backward_workspace.restype = _sz
    lib.svgear_rotary_backward_workspace.argtypes = [_i, _i, _i, _i64, _i]
    lib.svgear_rotary_backward.restype = _i
    lib.svgear_rotary_backward.argtypes = [_i, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i64, _i64, _i, *places, _vp, _sz,
                                           _vp]
    lib.svgear_layer_norm.restype = _i
    lib.svgear_layer_norm.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i64, _i, _f, _vp, _vp, _vp]
    lib.svgear_layer_norm_backward_workspace.restype = _sz
    lib.svgear_layer_norm_backward_workspace.argtypes = [_i, _i, _i64, _i, _i]
    lib.svgear_layer_norm_backward.restype = _i
    lib.svgear_layer_norm_backward.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i64, _i, _f, _vp, _vp, _vp, _vp, _vp,
                                               _vp, _vp, _sz, _vp]
    sizes, mask = [_i, _i, _i, _i, _i64, _i64, _i], [_f, _f, _vp, _u, _i, _vp, _vp, _vp]
    lib.svgear_attention_workspace.restype = _sz
    lib.svgear_attention_workspace.argtypes = [*sizes, _i]
    lib.svgear_attention.restype = _i
    lib.svgear_attention.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, *sizes, *mask, _vp, _vp, _vp, _vp, _sz, _vp]
    lib.svgear_attention_backward_workspace.restype = _sz
    lib.svgear_attention_backward_workspace.argtypes = [*sizes, _i]
    lib.svgear_attention_backward.restype = _i
    lib.svgear_attention_backward.argtypes = [_vp] * 11 + [*sizes, *mask] + [_vp] * 7 + [_sz, _vp]
    _LIB = lib
    return lib


_STATUS = {-1: "invalid argument", -2: "workspace too small", -3: "HIP runtime error", -4: "unsupported"}


def _check(rc: int, what: str):
    if rc != 0:
        extra = f" (hip error {load_library().svgear_last_hip_error()})" if rc == -3 else ""
        raise SvgearError(f"{what} failed: {_STATUS.get(rc, rc)}{extra}")


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return 0
    if t.dtype == torch.bfloat16:
        return 1
    raise SvgearError(f"unsupported dtype {t.dtype}")


def _need_gpu(*ts):
    for t in ts:
        if t is not None and not t.is_cuda:
            raise SvgearError("svgear needs device tensors: there is no CPU path")


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _strides4(t: torch.Tensor):
    assert t.dim() == 4 and t.stride(3) == 1, "expected [B,H,N,d] with contiguous d"
    return _I64x3(t.stride(0), t.stride(1), t.stride(2))


def _ws(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def kmeans_list_threshold(min_centroids: int = 0) -> int:
    """svgear_kmeans_list_threshold: sets (>= 1) or queries (<= 0) the number of centroids from which
    the later k-means iterations use candidate lists; returns the previous value."""
    lib = load_library()
    lib.svgear_kmeans_list_threshold.restype = _i
    lib.svgear_kmeans_list_threshold.argtypes = [_i]
    return int(lib.svgear_kmeans_list_threshold(int(min_centroids)))


def _check_centroids(c: torch.Tensor, B: int, H: int, d: int, device: torch.device):
    """Starting centroids, which are written: those of every head of what is clustered."""
    if not (c.dim() == 4 and c.shape[:2] == (B, H) and c.shape[3] == d and c.dtype == torch.float32 and c.is_contiguous()
            and c.device == device):
        raise SvgearError(f"centroids: expected dense fp32 [{B},{H},C,{d}] on {device}")


def kmeans(x: torch.Tensor, centroids: torch.Tensor, iters: int, n_tail: int = 0,
           x2: Optional[torch.Tensor] = None, one_launch: bool = True):
    """svgear_kmeans (one_launch=False: svgear_kmeans_stepwise, the same results with launches of its own for
    every step of a small call too). x [B,H,N,d]; centroids [B,H,C,d] fp32 (updated in place).
    Returns (labels [B,H,N-n_tail] i32, counts [B,H,C] i32, centroids2 or None)."""
    _need_gpu(x, centroids, x2)
    lib = load_library()
    B, H, N, d = x.shape
    _check_centroids(centroids, B, H, d, x.device)
    C = centroids.shape[2]
    if x2 is not None:
        assert x2.shape == x.shape and x2.stride() == x.stride() and x2.dtype == x.dtype
    labels = torch.empty(B, H, N - n_tail, dtype=torch.int32, device=x.device)
    counts = torch.empty(B, H, C, dtype=torch.int32, device=x.device)
    c2 = torch.zeros(B, H, C, d, dtype=torch.float32, device=x.device) if x2 is not None else None
    ws = _ws(lib.svgear_kmeans_workspace(B, H, N, d, C), x.device)
    st = _strides4(x)
    fn = lib.svgear_kmeans if one_launch else lib.svgear_kmeans_stepwise
    rc = fn(_ptr(x), _ptr(x2), _dt(x), B, H, N, n_tail, d, st, C, iters, _ptr(centroids), _ptr(c2), _ptr(labels),
            _ptr(counts), _ptr(ws), ws.numel(), _stream())
    _check(rc, "svgear_kmeans" if one_launch else "svgear_kmeans_stepwise")
    return labels, counts, c2


def permute(labels: torch.Tensor, C: int, tensors: Sequence[torch.Tensor] = (), n_tail: int = 0,
            static_scratch: bool = False, out=None):
    """svgear_permute (static_scratch=True: svgear_permute_static, whose scratch is an array inside
    the library; with out=(perm, offsets, [dst tensors]) preallocated by the caller that call
    touches no allocator at all). Returns (perm [B,H,N] i32, offsets [B,H,C+2] i32, [permuted tensors])."""
    _need_gpu(labels, *tensors)
    lib = load_library()
    B, H, nv = labels.shape
    N = nv + n_tail
    assert labels.dtype == torch.int32 and labels.is_contiguous()
    n = len(tensors)
    d, dt = 64, 0
    if n:
        d, dt = tensors[0].shape[3], _dt(tensors[0])
        for t in tensors:
            assert t.shape == (B, H, N, d) and _dt(t) == dt
    if out is not None:
        perm, offsets, outs = out
        assert perm.shape == (B, H, N) and perm.dtype == torch.int32 and perm.is_contiguous()
        assert offsets.shape == (B, H, C + 2) and offsets.dtype == torch.int32 and offsets.is_contiguous()
        assert len(outs) == n
        for o, t in zip(outs, tensors):
            assert o.shape == t.shape and o.dtype == t.dtype and o.is_contiguous()
        _need_gpu(perm, offsets, *outs)
    else:
        perm = torch.empty(B, H, N, dtype=torch.int32, device=labels.device)
        offsets = torch.empty(B, H, C + 2, dtype=torch.int32, device=labels.device)
        outs = [torch.empty(B, H, N, d, dtype=t.dtype, device=t.device) for t in tensors]
    src = (_vp * max(n, 1))(*[t.data_ptr() for t in tensors])
    dst = (_vp * max(n, 1))(*[t.data_ptr() for t in outs])
    sst = (_I64x3 * max(n, 1))(*[_strides4(t) for t in tensors])
    if static_scratch:
        rc = lib.svgear_permute_static(_ptr(labels), B, H, N, n_tail, C, _ptr(perm), _ptr(offsets), n, src, sst, dst,
                                       dt, d, _stream())
        _check(rc, "svgear_permute_static")
        return perm, offsets, outs
    ws = _ws(lib.svgear_permute_workspace(B, H, N, C), labels.device)
    rc = lib.svgear_permute(_ptr(labels), B, H, N, n_tail, C, _ptr(perm), _ptr(offsets), n, src, sst, dst, dt, d,
                            _ptr(ws), ws.numel(), _stream())
    _check(rc, "svgear_permute")
    return perm, offsets, outs


def permute_rows(perm: torch.Tensor, tensors: Sequence[torch.Tensor]):
    """svgear_permute_rows: the tensors' rows gathered through an existing permutation."""
    _need_gpu(perm, *tensors)
    lib = load_library()
    B, H, N = perm.shape
    assert perm.dtype == torch.int32 and perm.is_contiguous() and len(tensors) >= 1
    d, dt = tensors[0].shape[3], _dt(tensors[0])
    for t in tensors:
        assert t.shape == (B, H, N, d) and _dt(t) == dt
    outs = [torch.empty(B, H, N, d, dtype=t.dtype, device=t.device) for t in tensors]
    n = len(tensors)
    src = (_vp * n)(*[t.data_ptr() for t in tensors])
    dst = (_vp * n)(*[t.data_ptr() for t in outs])
    sst = (_I64x3 * n)(*[_strides4(t) for t in tensors])
    rc = lib.svgear_permute_rows(_ptr(perm), B, H, N, n, src, sst, dst, dt, d, _stream())
    _check(rc, "svgear_permute_rows")
    return outs


def probe_route(qbar, kbar, vbar, kp, vp, q_offsets, k_offsets, budget_cost: int, scale: float,
                flags: int = 0, scores: Optional[torch.Tensor] = None, Nq: Optional[int] = None,
                top_p: Optional[float] = None):
    """svgear_probe_route, or svgear_probe_route_top_p when top_p is given (budget_cost is then
    ignored). Returns dict(scores, mask_bits, row_ptr, col_idx, routed_cost[, row_budget])."""
    _need_gpu(qbar, kbar, vbar, kp, vp, q_offsets, k_offsets, scores)
    lib = load_library()
    B, H, Cq, d = qbar.shape
    Ck = kbar.shape[2]
    Nk = kp.shape[2]
    Nq = Nk if Nq is None else int(Nq)
    dev = qbar.device
    if scores is None:
        scores = torch.empty(B, H, Cq, Ck, dtype=torch.float32, device=dev)
    assert scores.shape == (B, H, Cq, Ck) and scores.dtype == torch.float32 and scores.is_contiguous()
    W = (Ck + 1 + 31) // 32
    mask_bits = torch.empty(B, H, Cq + 1, W, dtype=torch.int32, device=dev)
    row_ptr = torch.empty(B, H, Cq + 2, dtype=torch.int32, device=dev)
    col_idx = torch.empty(B, H, (Cq + 1) * (Ck + 1), dtype=torch.int32, device=dev)
    routed_cost = torch.empty(B, H, dtype=torch.int64, device=dev)
    ws = _ws(lib.svgear_probe_route_workspace(B, H, Nk, d, Cq, Ck), dev)
    for t in (qbar, kbar, vbar, kp, vp, q_offsets, k_offsets):
        assert t.is_contiguous()
    if top_p is not None:
        row_budget = torch.empty(B, H, Cq, dtype=torch.int64, device=dev)
        rc = lib.svgear_probe_route_top_p(_ptr(qbar), _ptr(kbar), _ptr(vbar), _ptr(kp), _ptr(vp), _dt(kp),
                                          _ptr(q_offsets), _ptr(k_offsets), B, H, Nq, Nk, d, Cq, Ck, float(top_p),
                                          float(scale), int(flags), _ptr(scores), _ptr(mask_bits), _ptr(row_ptr),
                                          _ptr(col_idx), _ptr(routed_cost), _ptr(row_budget), _ptr(ws), ws.numel(),
                                          _stream())
        _check(rc, "svgear_probe_route_top_p")
        return dict(scores=scores, mask_bits=mask_bits, row_ptr=row_ptr, col_idx=col_idx, routed_cost=routed_cost,
                    row_budget=row_budget)
    rc = lib.svgear_probe_route(_ptr(qbar), _ptr(kbar), _ptr(vbar), _ptr(kp), _ptr(vp), _dt(kp), _ptr(q_offsets),
                                _ptr(k_offsets), B, H, Nq, Nk, d, Cq, Ck, int(budget_cost), float(scale),
                                int(flags), _ptr(scores), _ptr(mask_bits), _ptr(row_ptr), _ptr(col_idx),
                                _ptr(routed_cost), _ptr(ws), ws.numel(), _stream())
    _check(rc, "svgear_probe_route")
    return dict(scores=scores, mask_bits=mask_bits, row_ptr=row_ptr, col_idx=col_idx, routed_cost=routed_cost)


def sparse_attn_comp(qp, kp, vp, kbar, vbar, q_offsets, k_offsets, mask_bits, row_ptr, col_idx, scale: float,
                     want_lse: bool = False, ws: Optional[torch.Tensor] = None, two_stage: bool = False,
                     q_perm: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None):
    """svgear_sparse_attn_comp (two_stage=True: svgear_sparse_attn_two_stage, the same result
    through separate routed / compensation passes and a merge).
    With q_perm: svgear_sparse_attn_comp_token_order: the first argument is then the UNPERMUTED
    query tensor [B,H,Nq,d] (any strides with contiguous d), and output and lse come in token
    order, written into `out` if given. Returns (output [B,H,Nq,d], lse or None)."""
    _need_gpu(qp, kp, vp, kbar, vbar, q_offsets, k_offsets, mask_bits, row_ptr, col_idx, q_perm, out)
    lib = load_library()
    assert not (two_stage and q_perm is not None)
    ws_fn = lib.svgear_sparse_attn_two_stage_workspace if two_stage else lib.svgear_sparse_attn_comp_workspace
    B, H, Nq, d = qp.shape
    Nk = kp.shape[2]
    Cq = q_offsets.shape[2] - 2
    Ck = k_offsets.shape[2] - 2
    for t in (kp, vp, kbar, vbar, q_offsets, k_offsets, mask_bits, row_ptr, col_idx):
        assert t.is_contiguous()
    lse = torch.empty(B, H, Nq, dtype=torch.float32, device=qp.device) if want_lse else None
    if ws is None:
        ws = _ws(ws_fn(B, H, Nq, Nk, d, Cq, Ck), qp.device)
    if q_perm is not None:
        assert q_perm.is_contiguous() and q_perm.dtype == torch.int32 and q_perm.shape == (B, H, Nq)
        o = torch.empty(B, H, Nq, d, dtype=qp.dtype, device=qp.device) if out is None else out
        assert o.shape == qp.shape and o.dtype == qp.dtype
        rc = lib.svgear_sparse_attn_comp_token_order(
            _ptr(qp), _strides4(qp), _ptr(kp), _ptr(vp), _dt(qp), _ptr(kbar), _ptr(vbar), _ptr(q_offsets),
            _ptr(k_offsets), _ptr(mask_bits), _ptr(row_ptr), _ptr(col_idx), _ptr(q_perm), B, H, Nq, Nk, d, Cq, Ck,
            float(scale), _ptr(o), _strides4(o), _ptr(lse), _ptr(ws), ws.numel(), _stream())
        _check(rc, "svgear_sparse_attn_comp_token_order")
        return o, lse
    assert qp.is_contiguous()
    fn = lib.svgear_sparse_attn_two_stage if two_stage else lib.svgear_sparse_attn_comp
    op = torch.empty_like(qp)
    rc = fn(_ptr(qp), _ptr(kp), _ptr(vp), _dt(qp), _ptr(kbar), _ptr(vbar), _ptr(q_offsets), _ptr(k_offsets),
            _ptr(mask_bits), _ptr(row_ptr), _ptr(col_idx), B, H, Nq, Nk, d, Cq, Ck, float(scale), _ptr(op), _ptr(lse),
            _ptr(ws), ws.numel(), _stream())
    _check(rc, "svgear_sparse_attn_two_stage" if two_stage else "svgear_sparse_attn_comp")
    return op, lse


def _check_out(out: torch.Tensor, like: torch.Tensor):
    """A caller's output of the layer: of the shape, type and device of the tensor that it belongs to, with contiguous d."""
    _require(out.shape == like.shape and out.dtype == like.dtype and out.device == like.device and out.stride(-1) == 1,
             f"out: expected {tuple(like.shape)}, {like.dtype}, {like.device}, with contiguous d")


def unpermute(op: torch.Tensor, perm: torch.Tensor, out: Optional[torch.Tensor] = None):
    """svgear_unpermute: out[b,h,perm[p]] = op[b,h,p]. out, if given: [B,H,N,d] as op, any strides with contiguous d."""
    _need_gpu(op, perm, out)
    lib = load_library()
    B, H, N, d = op.shape
    assert op.is_contiguous() and perm.is_contiguous()
    _require(perm.shape == (B, H, N) and perm.dtype == torch.int32 and perm.device == op.device,
             "perm: expected int32 [B,H,N] on op's device")
    if out is None:
        out = torch.empty_like(op)
    else:
        _check_out(out, op)
    rc = lib.svgear_unpermute(_ptr(op), _ptr(perm), _dt(op), B, H, N, d, _ptr(out), _strides4(out), _stream())
    _check(rc, "svgear_unpermute")
    return out


def _require(ok, what: str):
    if not ok:
        raise SvgearError(what)


_HERE_ALREADY = contextlib.nullcontext()


def _on_device(device: torch.device):
    """The device as the current one, for calls whose tensors lie on another."""
    return _HERE_ALREADY if torch.cuda.current_device() == device.index else torch.cuda.device(device)


def _stream_of(device: torch.device) -> int:
    """The current stream's handle, without the object that torch.cuda.current_stream makes of it (1 us of a small call's 12)."""
    return torch._C._cuda_getCurrentRawStream(device.index)


def _scratch(nbytes: int, device):
    """Workspace of an entry point that may need none: (tensor or None, its address, its size)."""
    if nbytes == 0:
        return None, None, 0
    t = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return t, t.data_ptr(), nbytes


_DTYPES = {torch.float32: 0, torch.bfloat16: 1}


def _same_place(first: torch.Tensor, *ts) -> int:
    """Every tensor given lies on the first one's GPU and has its type, which is returned as the library's."""
    if not first.is_cuda:
        _need_gpu(first)
    device, dtype = first.device, first.dtype
    for t in ts:
        if t is not None and (t.device != device or t.dtype != dtype):
            _need_gpu(t)
            raise SvgearError("tensors of one call share a device and a type")
    dt = _DTYPES.get(dtype)
    return _dt(first) if dt is None else dt


_NO_ROWS = _I64x2(0, 0)

# The library's limits, looked at here too: ctypes keeps the low bits of what an argument does not hold.
_MOST_ROWS, _WIDEST, _MOST_HEADS, _GRID = 1 << 30, 1 << 21, 128, 1 << 31


def _linear_sizes(B: int, N: int, d_in: int, d_out: int):
    if not (0 < B * N <= _MOST_ROWS and 0 < d_in <= _WIDEST and 0 < d_out <= _WIDEST):
        raise SvgearError(f"{B} x {N} rows of {d_in} to {d_out}: expected 1 to 2^30 rows of 1 to 2^21 each")


def _as_bnd(t: torch.Tensor, what: str):
    """[B,N,c] or [N,c] (one batch entry) as (B, N, c, strides)."""
    shape, st = t.shape, t.stride()
    n = len(st)
    if not ((n == 3 or n == 2) and (st[-1] == 1 or shape[-1] == 1)):
        raise SvgearError(f"{what}: expected [B,N,c] or [N,c] with contiguous c")
    if n == 2:
        return 1, shape[0], shape[1], _I64x2(shape[0] * st[0], st[0])
    return shape[0], shape[1], shape[2], _I64x2(st[0], st[1])


def _gate_strides(gate, lead, d_out: int, what: str = "gate", width: str = "d_out"):
    """Strides of a gate (or another vector for each token) of tokens (lead + (d_out,)) or of batch entries (without the tokens' axis), and whether it is the first."""
    if gate is None:
        return _NO_ROWS, False
    shape, st, batches = gate.shape, gate.stride(), len(lead) == 2
    per_token = len(shape) == len(lead) + 1
    if shape != (*(lead if per_token else lead[:-1]), d_out):
        raise SvgearError(f"{what}: expected [B,N,{width}] or [B,{width}] ([N,{width}] or [{width}] for one batch entry)")
    if d_out != 1 and st[-1] != 1:
        raise SvgearError(f"{what}: expected contiguous {width}")
    return _I64x2(st[0] if batches else 0, st[-2] if per_token else 0), per_token


def linear(x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None, act: str = "none",
           gate: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, want_pre: bool = False,
           out: Optional[torch.Tensor] = None):
    """svgear_linear: residual + gate * act(x w^T + bias). x [B,N,d_in] (or [N,d_in], one batch entry), w [d_out,d_in], bias
    [d_out]; act "none", "silu", "gelu" (erf) or "gelu_tanh"; gate [B,d_out] (one for all tokens of a batch entry) or
    [B,N,d_out]; residual [B,N,d_out], which `out` may be. want_pre: also z = x w^T + bias, which linear_backward needs
    where there is an activation or a gate. Returns (y, z or None). Not a part of torch's graph of gradients: results have none, also where
    inputs require them; linear_backward is called for them."""
    dt = _same_place(x, w, bias, gate, residual, out)
    lib = load_library()
    B, N, d_in, xst = _as_bnd(x, "x")
    lead = x.shape[:-1]
    wst = w.stride()
    if len(wst) != 2 or w.shape[1] != d_in or (wst[1] != 1 and d_in != 1):
        raise SvgearError("w: expected [d_out,d_in] with contiguous d_in")
    d_out = w.shape[0]
    _linear_sizes(B, N, d_in, d_out)
    shape = (*lead, d_out)
    if bias is not None and (bias.shape != (d_out,) or not bias.is_contiguous()):
        raise SvgearError("bias: expected [d_out]")
    act_code = ACTIVATIONS.get(act)
    if act_code is None:
        raise SvgearError(f"act: one of {sorted(ACTIVATIONS)}")
    gst = _gate_strides(gate, lead, d_out)[0]
    if residual is not None and residual.shape != shape:
        raise SvgearError("residual: expected the output's shape")
    if out is not None and out.shape != shape:
        raise SvgearError("out: expected the output's shape")
    rst = _as_bnd(residual, "residual")[3] if residual is not None else _NO_ROWS
    device = x.device
    with _on_device(device):
        y = torch.empty(shape, dtype=x.dtype, device=device) if out is None else out
        pre = torch.empty(shape, dtype=x.dtype, device=device) if want_pre else None
        yst = _as_bnd(y, "out")[3]
        head = (x.data_ptr(), xst, w.data_ptr(), wst[0] if d_out > 1 else max(wst[0], d_in))
        ws, *space = _scratch(lib.svgear_linear_workspace(*head, dt, B, N, d_in, d_out), device)
        rc = lib.svgear_linear(*head, _ptr(bias), dt, B, N, d_in, d_out, act_code, _ptr(gate), gst, _ptr(residual), rst,
                               _ptr(pre), y.data_ptr(), yst, *space, _stream_of(device))
    _check(rc, "svgear_linear")
    return y, pre


def linear_backward(dy: torch.Tensor, x: Optional[torch.Tensor], w: Optional[torch.Tensor], pre: Optional[torch.Tensor] = None,
                    act: str = "none", gate: Optional[torch.Tensor] = None, want: Sequence[str] = ("dx", "dw")):
    """svgear_linear_backward: the gradients named in `want` ("dx", "dw", "dbias", "dgate") of linear() for the output's
    gradient dy; the residual's is dy itself. x is needed for dw, w for dx, pre (linear's second result) for an activation or
    dgate. dgate has the gate's shape. In bf16, dz = dy * gate * act'(pre) is rounded for the products of dx and dw. Returns a dict."""
    dt = _same_place(dy, x, w, pre, gate)
    lib = load_library()
    B, N, d_out, dyst = _as_bnd(dy, "dy")
    lead = tuple(dy.shape[:-1])
    _require(len(want) > 0 and set(want) <= {"dx", "dw", "dbias", "dgate"}, "want: dx, dw, dbias, dgate")
    if act not in ACTIVATIONS:
        raise SvgearError(f"act: one of {sorted(ACTIVATIONS)}")
    x, w = (x if "dw" in want else None), (w if "dx" in want else None)
    _require("dw" not in want or x is not None, "dw needs x")
    _require("dx" not in want or w is not None, "dx needs w")
    _require("dgate" not in want or gate is not None, "dgate needs the gate")
    d_in = w.shape[1] if w is not None else x.shape[-1] if x is not None else 1
    _linear_sizes(B, N, d_in, d_out)
    _require(x is None or tuple(x.shape) == (*lead, d_in), "x: expected dy's leading sizes and d_in")
    _require(w is None or (tuple(w.shape) == (d_out, d_in) and (d_in == 1 or w.stride(1) == 1)), "w: expected [d_out,d_in] with contiguous d_in")
    _require(pre is None or (tuple(pre.shape) == tuple(dy.shape) and pre.is_contiguous()), "pre: expected dy's shape, dense")
    _require(pre is not None or (act == "none" and "dgate" not in want), "an activation or dgate needs pre")
    gst, per_token = _gate_strides(gate, lead, d_out)
    xst = _as_bnd(x, "x")[3] if x is not None else _NO_ROWS
    _require(not per_token or gst[1] != 0 or N == 1 or "dgate" not in want, "gate: one gate for all tokens is given as [B,d_out]")
    with _on_device(dy.device):
        new = lambda *shape: torch.empty(*shape, dtype=dy.dtype, device=dy.device)
        r = {}
        for name in want:
            r[name] = new(*lead, d_in) if name == "dx" else new(d_out, d_in) if name == "dw" else new(d_out) if name == "dbias" else new(*gate.shape)
        dx = r.get("dx")
        dxst = _as_bnd(dx, "dx")[3] if dx is not None else _NO_ROWS
        ldw = 0 if w is None else w.stride(0) if d_out > 1 else max(w.stride(0), d_in)
        head = (_ptr(dy), dyst, _ptr(x), xst, _ptr(w), ldw)
        ws, *space = _scratch(lib.svgear_linear_backward_workspace(*head, dt, B, N, d_in, d_out), dy.device)
        rc = lib.svgear_linear_backward(*head, _ptr(pre), dt, B, N, d_in, d_out, ACTIVATIONS[act], _ptr(gate), gst,
                                        _ptr(dx), dxst, _ptr(r.get("dw")), _ptr(r.get("dbias")), _ptr(r.get("dgate")),
                                        *space, _stream_of(dy.device))
    _check(rc, "svgear_linear_backward")
    return r


def rotary_frequencies(sections: Sequence[int], theta: float = 10000.0, device="cuda") -> torch.Tensor:
    """The frequencies of video transformers, for rotary(): theta^(-i / pairs) for pair i of each axis, fp64."""
    f = [theta ** (-torch.arange(n, dtype=torch.float64) / max(n, 1)) for n in sections]
    return torch.cat(f).to(device)


_PTRS = (None, _vp * 1, _vp * 2)
_STRIDES = (None, _c.c_int64 * 3, _c.c_int64 * 6)  # int64_t[n][3], one behind the other


# (looked at once: what is kept is in range)
@functools.lru_cache(maxsize=64)
def _sections(*s):
    if len(s) != 3 or min(s) < 0 or max(s) > 64:
        raise SvgearError("sections: pairs of the three axes")
    return _Ix3(*s)


@functools.lru_cache(maxsize=64)
def _grid(*g):
    if len(g) != 3 or min(g) < 1 or max(g) >= _GRID:
        raise SvgearError("grid: (time, height, width)")
    return _I64x3(*g)


def _pointers(ts):
    return _PTRS[len(ts)](*[None if t is None else t.data_ptr() for t in ts])


def _strides_of(ts):
    flat = []
    for t in ts:
        st = t.stride()
        if len(st) != 4 or st[3] != 1:
            raise SvgearError("expected [B,H,N,d] with contiguous d")
        flat += st[:3]
    return _STRIDES[len(ts)](*flat)


def _rotary_places(tensors, inv_freq, sections, grid, first, positions, n_tail, norm, weights, halves):
    """The checked arguments that rotary and its backward pass share: (weights, arguments from inv_freq to flags)."""
    t0 = tensors[0]
    if t0.dim() != 4 or len(tensors) > 2 or (len(tensors) == 2 and tensors[1].shape != t0.shape):
        raise SvgearError("one or two tensors of one shape [B,H,N,d]")
    B, H, N, d = t0.shape
    if not (0 < B * N <= _MOST_ROWS and 0 < H <= _MOST_HEADS and (d == 64 or d == 128) and 0 <= n_tail < N):
        raise SvgearError(f"[B,H,N,d] = {tuple(t0.shape)}, {n_tail} text tokens: expected 1 to 2^30 tokens, some of them rotated, of 1 to "
                          "128 heads of 64 or 128")
    sections3 = _sections(*sections)
    if norm not in ROTARY_NORMS:
        raise SvgearError('norm: None, "head" or "token"')
    if (inv_freq.device != t0.device or inv_freq.dtype != torch.float64 or inv_freq.shape != (sum(sections),)
            or not inv_freq.is_contiguous()):
        raise SvgearError("inv_freq: expected fp64 [sum(sections)] on the tensors' device")
    if (positions is None) == (grid is None):
        raise SvgearError("positions or grid, one of them")
    pos_b, size3 = 0, None
    if positions is not None:
        shape = positions.shape
        if (positions.device != t0.device or positions.dtype != torch.int32 or not positions.is_contiguous()
                or (shape != (N - n_tail, 3) and shape != (B, N - n_tail, 3))):
            raise SvgearError("positions: expected int32 [N-n_tail,3] or [B,N-n_tail,3] on the tensors' device")
        if len(shape) == 3:
            pos_b = 3 * shape[1]
    else:
        size3 = _grid(*grid)
        if not 0 <= first < _GRID:
            raise SvgearError("first: a token of the grid")
    if weights is None:
        weights = (None,) * len(tensors)
    else:
        size = d if norm == "head" else H * d
        if norm is None or len(weights) != len(tensors):
            raise SvgearError("weights: one for each tensor, with a norm")
        for w in weights:
            if w is not None and (w.shape != (size,) or not w.is_contiguous()):
                raise SvgearError("weights: expected [d] or [H*d]")
    return weights, (inv_freq.data_ptr(), sections3, size3, 0 if size3 is None else first, _ptr(positions), pos_b,
                     ROTARY_NORMS[norm] | (ROTARY_HALVES if halves else 0))


def rotary(tensors: Sequence[torch.Tensor], inv_freq: torch.Tensor, sections: Sequence[int], grid=None, first: int = 0,
           positions: Optional[torch.Tensor] = None, n_tail: int = 0, norm: Optional[str] = None, weights=None,
           eps: float = 1e-6, halves: bool = False, out=None):
    """svgear_rotary: RMS norm (norm "head" or "token", with `weights`) and rotation of queries and keys [B,H,N,d] (any
    strides) by positions on three axes with `sections` pairs each: token n is element first + n of `grid` = (time, height,
    width), or has positions[n] (int32 [N-n_tail,3] or [B,N-n_tail,3]); the last n_tail tokens, fewer than N, are not rotated. `out` may be
    `tensors`. Returns the list of results, dense unless given. Not a part of torch's graph of gradients: rotary_backward is called
    for them."""
    _require(len(tensors) in (1, 2), "one or two tensors")
    t0 = tensors[0]
    outs = [None] * len(tensors) if out is None else list(out)
    dt = _same_place(t0, *tensors, *(weights or ()), *outs)
    lib = load_library()
    ws, places = _rotary_places(tensors, inv_freq, sections, grid, first, positions, n_tail, norm, weights, halves)
    B, H, N, d = t0.shape
    with _on_device(t0.device):
        if out is None:
            outs = [torch.empty(B, H, N, d, dtype=t0.dtype, device=t0.device) for _ in tensors]
        _require(len(outs) == len(tensors) and all(o.shape == t0.shape for o in outs), "out: one for each tensor, of its shape")
        rc = lib.svgear_rotary(len(tensors), _pointers(tensors), _strides_of(tensors), _pointers(outs), _strides_of(outs),
                               _pointers(ws), dt, B, H, N, n_tail, d, *places, float(eps), _stream_of(t0.device))
    _check(rc, "svgear_rotary")
    return outs


def rotary_backward(grads: Sequence[torch.Tensor], tensors: Optional[Sequence[torch.Tensor]], inv_freq: torch.Tensor,
                    sections: Sequence[int], grid=None, first: int = 0, positions: Optional[torch.Tensor] = None,
                    n_tail: int = 0, norm: Optional[str] = None, weights=None, eps: float = 1e-6, halves: bool = False,
                    want_dweight: bool = True, out=None):
    """svgear_rotary_backward: for the gradients of rotary()'s results, (list of its inputs' gradients, list of its weights'
    gradients or None; without a norm None). `tensors`, rotary's inputs, are needed with a norm. `out` (the inputs' gradients) may be
    `grads`."""
    _require(len(grads) in (1, 2), "one or two tensors")
    g0 = grads[0]
    outs = [None] * len(grads) if out is None else list(out)
    _require(norm is None or (tensors is not None and len(tensors) == len(grads) and all(t.shape == g0.shape for t in tensors)),
             "a norm needs rotary's inputs")
    tensors = list(tensors) if norm is not None else []
    dt = _same_place(g0, *grads, *tensors, *(weights or ()), *outs)
    lib = load_library()
    ws, places = _rotary_places(grads, inv_freq, sections, grid, first, positions, n_tail, norm, weights, halves)
    B, H, N, d = g0.shape
    n = len(grads)
    with _on_device(g0.device):
        if out is None:
            outs = [torch.empty(B, H, N, d, dtype=g0.dtype, device=g0.device) for _ in grads]
        _require(len(outs) == n and all(o.shape == g0.shape for o in outs), "out: one for each tensor, of its shape")
        dweight = None
        if norm is not None and want_dweight:
            dweight = [torch.empty(d if norm == "head" else H * d, dtype=g0.dtype, device=g0.device) for _ in grads]
        scratch, *space = _scratch(lib.svgear_rotary_backward_workspace(n, B, H, N, d) if dweight else 0, g0.device)
        rc = lib.svgear_rotary_backward(n, _pointers(grads), _strides_of(grads), _pointers(tensors) if tensors else None,
                                        _strides_of(tensors) if tensors else None, _pointers(outs), _strides_of(outs),
                                        _pointers(ws), _pointers(dweight) if dweight else None, dt, B, H, N, n_tail, d,
                                        *places, float(eps), *space, _stream_of(g0.device))
    _check(rc, "svgear_rotary_backward")
    return outs, dweight


def _norm_arguments(x, weight, bias, scale, shift, eps: float):
    """The checked arguments that layer_norm and its backward pass share: (B, N, c, x's strides, strides of scale, of shift, whether
    either is one of tokens)."""
    B, N, c, xst = _as_bnd(x, "x")
    if not (0 < B * N <= _MOST_ROWS and 0 < c <= 1 << 15):
        raise SvgearError(f"{B} x {N} tokens of {c}: expected 1 to 2^30 tokens of 1 to 2^15 each")
    for w in (weight, bias):
        if w is not None and (w.shape != (c,) or not w.is_contiguous()):
            raise SvgearError("weight, bias: expected [c]")
    if not 0.0 <= eps < float("inf"):
        raise SvgearError("eps: expected a number from 0 on")
    if scale is None and shift is None:
        return B, N, c, xst, _NO_ROWS, _NO_ROWS, False
    lead = x.shape[:-1]
    sst, of_tokens = _gate_strides(scale, lead, c, "scale", "c")
    hst, shift_of_tokens = _gate_strides(shift, lead, c, "shift", "c")
    if scale is not None and shift is not None and of_tokens != shift_of_tokens:
        raise SvgearError("scale and shift: both of batch entries or both of tokens")
    return B, N, c, xst, sst, hst, of_tokens or shift_of_tokens


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
               scale: Optional[torch.Tensor] = None, shift: Optional[torch.Tensor] = None, eps: float = 1e-6,
               out: Optional[torch.Tensor] = None):
    """svgear_layer_norm: (h * weight + bias) * (1 + scale) + shift for h = (x - mean) / sqrt(var + eps) over the last dimension.
    x [B,N,c] (or [N,c], one batch entry); weight, bias [c]; scale, shift [B,c] (one for all tokens of a batch entry) or
    [B,N,c]. `out` may be x. Not a part of torch's graph of gradients: layer_norm_backward is called for them."""
    dt = _same_place(x, weight, bias, scale, shift, out)
    lib = load_library()
    B, N, c, xst, sst, hst, _ = _norm_arguments(x, weight, bias, scale, shift, eps)
    if out is not None and out.shape != x.shape:
        raise SvgearError("out: expected x's shape")
    with _on_device(x.device):
        y = out if out is not None else torch.empty_like(x) if x.is_contiguous() else x.new_empty(x.shape)
        rc = lib.svgear_layer_norm(x.data_ptr(), xst, _ptr(weight), _ptr(bias), _ptr(scale), sst, _ptr(shift), hst, dt, B, N, c,
                                   float(eps), y.data_ptr(), _as_bnd(y, "out")[3], _stream_of(x.device))
    _check(rc, "svgear_layer_norm")
    return y


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                        scale: Optional[torch.Tensor] = None, eps: float = 1e-6, want: Sequence[str] = ("dx",),
                        shift: Optional[torch.Tensor] = None):
    """svgear_layer_norm_backward: the gradients named in `want` ("dx", "dweight", "dbias", "dscale", "dshift") of layer_norm() for
    the output's gradient dy. bias is needed for dscale; dscale has scale's shape, and dshift too, or where there was no scale that of
    `shift`, which is given for it. Returns a dict."""
    dt = _same_place(dy, x, weight, bias, scale, shift)
    lib = load_library()
    _require(dy.shape == x.shape, "dy: expected x's shape")
    B, N, c, xst, sst, _, per_token = _norm_arguments(x, weight, bias, scale, shift, eps)
    yst = _as_bnd(dy, "dy")[3]
    _require(len(want) > 0 and set(want) <= {"dx", "dweight", "dbias", "dscale", "dshift"}, "want: dx, dweight, dbias, dscale, dshift")
    mod = scale if scale is not None else shift
    _require(scale is not None or "dscale" not in want, "dscale needs the scale")
    _require(mod is not None or "dshift" not in want, "dshift needs the scale, or the shift")
    modulation = 0 if mod is None else 2 if per_token else 1
    with _on_device(x.device):
        r = {n: x.new_empty(x.shape if n == "dx" else c if n in ("dweight", "dbias") else mod.shape) for n in want}
        dx = r.get("dx")
        sums = {"dweight", "dbias"} & set(want) or (modulation == 1 and {"dscale", "dshift"} & set(want))
        ws, *space = _scratch(lib.svgear_layer_norm_backward_workspace(dt, B, N, c, modulation) if sums else 0, x.device)
        rc = lib.svgear_layer_norm_backward(dy.data_ptr(), yst, x.data_ptr(), xst, _ptr(weight), _ptr(bias), _ptr(scale), sst, modulation,
                                            dt, B, N, c, float(eps), _ptr(dx), _as_bnd(dx, "dx")[3] if dx is not None else _NO_ROWS,
                                            _ptr(r.get("dweight")), _ptr(r.get("dbias")), _ptr(r.get("dscale")), _ptr(r.get("dshift")),
                                            *space, _stream_of(x.device))
    _check(rc, "svgear_layer_norm_backward")
    return r


def _strides_bhn(t: torch.Tensor, what: str):
    st = t.stride()
    if len(st) != 4 or st[3] != 1:
        raise SvgearError(f"{what}: expected [B,heads,N,d] with contiguous d")
    return _I64x3(*st[:3])


def _attention_arguments(q, k, v, scale, cap, slopes, causal, prefix, q_offsets, k_offsets):
    """The checked arguments that attention and its backward pass share: (sizes, arguments from scale to prefix)."""
    _require(q.dim() == 4 and k.dim() == 4 and k.shape == v.shape, "expected q [B,H,Nq,d], k and v [B,Hk,Nk,d]")
    B, H, Nq, d = q.shape
    Hk, Nk = k.shape[1], k.shape[2]
    _require(k.shape[0] == B and k.shape[3] == d and (d == 64 or d == 128), "expected q, k and v of one batch with heads of 64 or 128")
    _require(min(B, H, Hk, Nq, Nk) > 0 and H % Hk == 0, "expected tokens, and key heads that divide the queries' heads")
    _require(B * H <= _MOST_ROWS and Nq * (H // Hk) <= _MOST_ROWS and Nk <= _MOST_ROWS, "expected at most 2^30 heads and rows of a head")
    device, flags, n_docs, given = q.device, 0, 0, [o for o in (q_offsets, k_offsets) if o is not None]
    if slopes is not None and (slopes.device != device or slopes.dtype != torch.float32 or slopes.shape != (H,) or not slopes.is_contiguous()):
        raise SvgearError("slopes: expected fp32 [H] on the tensors' device")
    if given:
        n_docs = given[0].shape[-1] - 1 if given[0].dim() else -1
        _require(n_docs >= 1 and (len(given) == 2 or n_docs == 1), "offsets: [B,n+1] of queries and keys; of one of them alone [B,2]")
    for t, n, what in ((q_offsets, n_docs + 1, "q_offsets"), (k_offsets, n_docs + 1, "k_offsets"), (prefix, max(n_docs, 1), "prefix")):
        if t is not None and (t.device != device or t.dtype != torch.int32 or not t.is_contiguous() or tuple(t.shape) not in ((n,), (B, n))):
            raise SvgearError(f"{what}: expected int32 [{n}] or [{B},{n}] on the tensors' device")
    rows = given + ([prefix] if prefix is not None else [])
    if rows and any(t.dim() == 1 for t in rows):
        _require(B == 1 or all(t.dim() == 1 for t in rows), "offsets and prefix: all of them one row for the batch, or one for each entry")
        flags |= ATTENTION_SHARED_DOCUMENTS
    _require(causal or prefix is None, "a prefix needs causal=True")
    cap = 0.0 if cap is None else float(cap)
    _require(cap == 0.0 or 2.0 ** -126 <= cap < float("inf"), "cap: a number above 0 that fp32 has, or None")
    scale = float(d) ** -0.5 if scale is None else float(scale)
    _require(abs(scale) < float("inf"), "scale: a finite number")
    if causal:
        flags |= ATTENTION_CAUSAL
    return (B, H, Hk, Nq, Nk, d), (scale, cap, _ptr(slopes), flags, n_docs, _ptr(q_offsets), _ptr(k_offsets), _ptr(prefix))


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scale: Optional[float] = None, cap: Optional[float] = None,
              slopes: Optional[torch.Tensor] = None, causal: bool = False, prefix: Optional[torch.Tensor] = None,
              q_offsets: Optional[torch.Tensor] = None, k_offsets: Optional[torch.Tensor] = None, want_lse: bool = False,
              out: Optional[torch.Tensor] = None):
    """svgear_attention: dense attention of q [B,H,Nq,d] over k, v [B,Hk,Nk,d] (any strides; Hk divides H). cap: scores become
    cap tanh(score / cap); slopes fp32 [H]: less slopes[h] times the distance; q_offsets, k_offsets int32 [B,n+1] (or [n+1], for all
    batch entries): documents that see only themselves (k_offsets alone, [B,2]: padded keys); causal: the last query of a document
    stands at its last key and sees what is not behind it, and the first prefix[b,t] keys (int32 [B,n]) whatever its place. A query that
    sees no key gives 0, and -inf in lse. Scores are scaled by `scale`, d^-0.5 if none is given. `out` may have any strides. Returns (o,
    lse [B,H,Nq] fp32 or None). Not a part of torch's graph of gradients: attention_backward is called for them."""
    dt = _same_place(q, k, v, out)
    lib = load_library()
    sizes, mask = _attention_arguments(q, k, v, scale, cap, slopes, causal, prefix, q_offsets, k_offsets)
    if out is not None and out.shape != q.shape:
        raise SvgearError("out: expected q's shape")
    with _on_device(q.device):
        o = q.new_empty(q.shape) if out is None else out
        lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device) if want_lse else None
        ws, *space = _scratch(lib.svgear_attention_workspace(dt, *sizes, mask[4]), q.device)
        rc = lib.svgear_attention(q.data_ptr(), _strides_bhn(q, "q"), k.data_ptr(), _strides_bhn(k, "k"), v.data_ptr(), _strides_bhn(v, "v"),
                                  dt, *sizes, *mask, o.data_ptr(), _strides_bhn(o, "out"), _ptr(lse), *space, _stream_of(q.device))
    _check(rc, "svgear_attention")
    return o, lse


def attention_backward(dy: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor, lse: torch.Tensor,
                       scale: Optional[float] = None, cap: Optional[float] = None, slopes: Optional[torch.Tensor] = None,
                       causal: bool = False, prefix: Optional[torch.Tensor] = None, q_offsets: Optional[torch.Tensor] = None,
                       k_offsets: Optional[torch.Tensor] = None, want: Sequence[str] = ("dq", "dk", "dv"), out=None):
    """svgear_attention_backward: the gradients named in `want` ("dq"; "dk" and "dv", both or neither) of attention() for the output's
    gradient dy, from what it returned with want_lse and the arguments that it had. `out`: a dict of tensors of any strides for
    them. The slopes get none. Returns a dict."""
    out = {} if out is None else out
    dt = _same_place(dy, q, k, v, o, *out.values())
    lib = load_library()
    sizes, mask = _attention_arguments(q, k, v, scale, cap, slopes, causal, prefix, q_offsets, k_offsets)
    _require(dy.shape == q.shape and o.shape == q.shape, "dy and o: expected q's shape")
    _require(lse is not None and lse.device == q.device and lse.dtype == torch.float32 and lse.shape == q.shape[:3] and lse.is_contiguous(),
             "lse: expected attention()'s, fp32 [B,H,Nq]")
    _require(len(want) > 0 and set(want) <= {"dq", "dk", "dv"} and ("dk" in want) == ("dv" in want), "want: dq, dk and dv")
    _require(set(out) <= set(want), "out: gradients that are wanted")
    like = {"dq": q, "dk": k, "dv": v}
    with _on_device(q.device):
        r = {n: out[n] if n in out else q.new_empty(like[n].shape) for n in want}
        _require(all(r[n].shape == like[n].shape for n in r), "out: expected the shapes of q, k and v")
        ends = [x for n in ("dq", "dk", "dv") for x in (_ptr(r.get(n)), _strides_bhn(r[n], n) if n in r else None)]
        ws, *space = _scratch(lib.svgear_attention_backward_workspace(dt, *sizes, mask[4]), q.device)
        places = [x for t, n in ((dy, "dy"), (q, "q"), (k, "k"), (v, "v"), (o, "o")) for x in (t.data_ptr(), _strides_bhn(t, n))]
        rc = lib.svgear_attention_backward(*places, lse.data_ptr(), dt, *sizes, *mask, *ends, *space, _stream_of(q.device))
    _check(rc, "svgear_attention_backward")
    return r


_SIDE_STREAMS = {}


def run_pair(fn_side, fn_main):
    """Runs two independent library calls concurrently: fn_side on a second stream of the
    same device (default priority), fn_main on the current stream, and joins them. The
    k-means and permutation calls of Q and of K/V do not depend on each other and their small
    kernels leave CUs idle, so running the two side by side shortens the layer (measured
    14.2 -> 12.9 ms for both k-means and permutations at the Wan shape). Tensors fn_side
    returns are handed over to the current stream. Returns (fn_side(), fn_main())."""
    main = torch.cuda.current_stream()
    key = main.device_index
    side = _SIDE_STREAMS.get(key)
    if side is None:
        side = _SIDE_STREAMS[key] = torch.cuda.Stream(device=main.device)
    side.wait_stream(main)
    with torch.cuda.stream(side):
        a = fn_side()
    b = fn_main()
    main.wait_stream(side)

    def hand_over(x):
        if isinstance(x, torch.Tensor):
            x.record_stream(main)
        elif isinstance(x, (tuple, list)):
            for y in x:
                hand_over(y)

    hand_over(a)
    return a, b


def attention_layer(Q, K, V, init_q, init_k, iters: int, budget_cost: int, n_tail: int = 0, flags: int = 0,
                    scale: Optional[float] = None, overlap: bool = True, top_p: Optional[float] = None, mark=None,
                    token_order: bool = True, out: Optional[torch.Tensor] = None):
    """One pass of the whole hot path over a batch of heads: k-means, permutation, probe + route,
    fused attention, un-permutation.

    token_order=True (default): Q's rows are never moved: only its permutation index is
    computed, and the attention kernel reads the queries and writes the output through it
    (svgear_sparse_attn_comp_token_order), so the "unpermute" stage is empty and the
    intermediates hold neither "Qp" nor "Op". token_order=False materialises Qp, runs
    svgear_sparse_attn_comp and svgear_unpermute.

    overlap=True uses a second stream of default priority for Q's side of the k-means and
    permutation stages (they do not depend on K's and V's; the small kernels of one stream fill
    the gaps of the other), joined before the probe, which needs the queries' offsets. (One fork and
    one join for both stages, since a pair costs the host some 40 us: 2 heads of 667 tokens take 192 us with one pair,
    231 with two; with mark, which tells the stages apart, a pair for each.)

    init_q [B,H,Cq,d], init_k [B,H,Ck,d] fp32 are the starting centroids (updated in place,
    so a caller can carry them to the next denoising step). With top_p the routing budget is
    the adaptive per-query-cluster one and budget_cost is ignored. mark(name), if given, is
    called on the current stream after each stage ("kmeans", "permute", "probe_route",
    "attention", "unpermute"). O is written into `out` if given ([B,H,N,d] as Q, any strides with contiguous d, over none
    of Q, K and V). Returns (O, intermediates)."""
    B, H, N, d = Q.shape
    _need_gpu(Q, K, init_q, init_k, out)
    _check_centroids(init_q, B, H, d, Q.device)
    _check_centroids(init_k, B, H, d, Q.device)  # and K's, which kmeans holds it to
    if out is not None:
        _check_out(out, Q)
    if scale is None:
        scale = float(d) ** -0.5
    Cq, Ck = init_q.shape[2], init_k.shape[2]
    km_q, km_k = lambda: kmeans(Q, init_q, iters, n_tail), lambda: kmeans(K, init_k, iters, n_tail, x2=V)
    pm_q = lambda lab: permute(lab, Cq, [] if token_order else [Q], n_tail)
    pm_k = lambda lab: permute(lab, Ck, [K, V], n_tail)

    def q_side():
        r = km_q()
        return r, pm_q(r[0])

    def k_side():
        r = km_k()
        return r, pm_k(r[0])

    one_pair = overlap and mark is None
    mark = mark or (lambda name: None)
    if one_pair:
        (q, q_rows), (k, k_rows) = run_pair(q_side, k_side)
    else:
        pair = run_pair if overlap else (lambda f, g: (f(), g()))
        q, k = pair(km_q, km_k)
        mark("kmeans")
        q_rows, k_rows = pair(lambda: pm_q(q[0]), lambda: pm_k(k[0]))
    (lab_q, qcnt, _), (lab_k, kcnt, vbar) = q, k
    (perm_q, qoff, q_rows), (perm_k, koff, (Kp, Vp)) = q_rows, k_rows
    mark("permute")
    r = probe_route(init_q, init_k, vbar, Kp, Vp, qoff, koff, budget_cost, scale, flags, top_p=top_p)
    mark("probe_route")
    if token_order:
        O, _ = sparse_attn_comp(Q, Kp, Vp, init_k, vbar, qoff, koff, r["mask_bits"], r["row_ptr"], r["col_idx"], scale,
                                q_perm=perm_q, out=out)
        mark("attention")
    else:
        (Qp,) = q_rows
        Op, _ = sparse_attn_comp(Qp, Kp, Vp, init_k, vbar, qoff, koff, r["mask_bits"], r["row_ptr"], r["col_idx"],
                                 scale)
        mark("attention")
        O = unpermute(Op, perm_q, out)
        r.update(Qp=Qp, Op=Op)
    mark("unpermute")
    r.update(lab_q=lab_q, lab_k=lab_k, qcnt=qcnt, kcnt=kcnt, qbar=init_q, kbar=init_k, vbar=vbar, perm_q=perm_q,
             perm_k=perm_k, qoff=qoff, koff=koff, Kp=Kp, Vp=Vp, O=O)
    return O, r


def attention_block(x: torch.Tensor, w_qkv: torch.Tensor, w_out: torch.Tensor, init_q: torch.Tensor, init_k: torch.Tensor,
                    iters: int, budget_cost: int, inv_freq: torch.Tensor, sections: Sequence[int], grid=None, first: int = 0,
                    positions: Optional[torch.Tensor] = None, b_qkv: Optional[torch.Tensor] = None,
                    b_out: Optional[torch.Tensor] = None, norm: Optional[str] = None, norm_weights=None, eps: float = 1e-6,
                    halves: bool = False, gate: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None,
                    n_tail: int = 0, **layer):
    """An attention block of a video transformer from its input to its output: linear() into queries, keys and values, rotary()
    on queries and keys where they lie, attention_layer() on the three as strided views, and linear() back with gate and
    residual.

    x [B,N,c]; w_qkv [3*H*d,c] (rows: queries of all heads, keys, values), b_qkv [3*H*d]; w_out [c_out,H*d], b_out [c_out];
    gate [B,c_out] or [B,N,c_out] and residual [B,N,c_out] as in linear(); norm, norm_weights (of queries and keys), inv_freq,
    sections, and grid and first, or positions, as in rotary(); init_q, init_k [B,H,C,d] (H and d are theirs), iters,
    budget_cost, n_tail and what `layer` holds as in attention_layer(). Returns (y [B,N,c_out], intermediates of the layer). The forward
    pass alone: the layer has no backward pass, so the gradients of linear() and rotary() end at it, and torch's graph of gradients knows
    none of them."""
    _require(x.dim() == 3 and init_q.dim() == 4, "x: expected [B,N,c], init_q: [B,H,C,d]")
    B, N, _ = x.shape
    H, d = init_q.shape[1], init_q.shape[3]
    _require(w_qkv.shape[0] == 3 * H * d and w_out.shape[1] == H * d, "w_qkv: expected [3*H*d,c], w_out: [c_out,H*d]")
    _require("out" not in layer, "the layer's output is the block's own")
    _need_gpu(x)
    for c in (init_q, init_k):
        _check_centroids(c, B, H, d, x.device)
    with _on_device(x.device):
        qkv, _ = linear(x, w_qkv, b_qkv)
        q, k, v = qkv.view(B, N, 3, H, d).permute(2, 0, 3, 1, 4)
        rotary([q, k], inv_freq, sections, grid=grid, first=first, positions=positions, n_tail=n_tail, norm=norm,
               weights=norm_weights, eps=eps, halves=halves, out=[q, k])
        o = torch.empty(B, N, H, d, dtype=x.dtype, device=x.device)
        _, r = attention_layer(q, k, v, init_q, init_k, iters, budget_cost, n_tail, out=o.transpose(1, 2), **layer)
        y, _ = linear(o.view(B, N, H * d), w_out, b_out, gate=gate, residual=residual)
        return y, r


def cross_attention_block(x: torch.Tensor, context: torch.Tensor, w_q: torch.Tensor, w_kv: torch.Tensor, w_out: torch.Tensor, heads: int,
                          lengths: Optional[torch.Tensor] = None, norm_weight: Optional[torch.Tensor] = None,
                          norm_bias: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                          shift: Optional[torch.Tensor] = None, eps: float = 1e-6, b_q: Optional[torch.Tensor] = None,
                          b_kv: Optional[torch.Tensor] = None, b_out: Optional[torch.Tensor] = None,
                          gate: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, saved: bool = False):
    """The attention of a video transformer's tokens to the text of their prompt, from the block's input to its output: layer_norm()
    of x, linear() into queries and of the context into keys and values, attention() over the context's first `lengths[b]` tokens,
    and linear() back with gate and residual.

    x [B,N,c], context [B,M,c_text], lengths int32 [B] or None; w_q [H*d,c] for H = `heads`, w_kv [2*Hk*d,c_text] (rows: keys of all
    heads, values), w_out [c_out,H*d], their biases; norm_weight, norm_bias, scale, shift, eps as in layer_norm(), gate and residual
    as in linear(). Returns (y [B,N,c_out], what cross_attention_block_backward() needs if `saved`, else None)."""
    _require(x.dim() == 3 and context.dim() == 3 and context.shape[0] == x.shape[0], "x: expected [B,N,c], context [B,M,c_text]")
    B, N, _ = x.shape
    M = context.shape[1]
    _require(heads > 0 and w_q.dim() == 2 and w_kv.dim() == 2 and w_q.shape[0] > 0 and w_q.shape[0] % heads == 0, "w_q: expected [heads*d,c]")
    d = w_q.shape[0] // heads
    _require(w_kv.shape[0] > 0 and w_kv.shape[0] % (2 * d) == 0 and w_out.dim() == 2 and w_out.shape[1] == heads * d,
             "w_kv: expected [2*Hk*d,c_text], w_out: [c_out,heads*d]")
    Hk = w_kv.shape[0] // (2 * d)
    _require(lengths is None or (lengths.dtype == torch.int32 and tuple(lengths.shape) == (B,)), "lengths: expected int32 [B]")
    _need_gpu(x, context, lengths)
    with _on_device(x.device):
        k_offsets = None if lengths is None else torch.stack([torch.zeros_like(lengths), lengths], 1)
        h = layer_norm(x, norm_weight, norm_bias, scale=scale, shift=shift, eps=eps)
        q = linear(h, w_q, b_q)[0].view(B, N, heads, d).transpose(1, 2)
        k, v = linear(context, w_kv, b_kv)[0].view(B, M, 2, Hk, d).permute(2, 0, 3, 1, 4)
        o = torch.empty(B, N, heads, d, dtype=x.dtype, device=x.device)
        _, lse = attention(q, k, v, k_offsets=k_offsets, want_lse=saved, out=o.transpose(1, 2))
        y, pre = linear(o.view(B, N, heads * d), w_out, b_out, gate=gate, residual=residual, want_pre=saved and gate is not None)
    kept = None
    if saved:
        kept = {"x": x, "context": context, "w_q": w_q, "w_kv": w_kv, "w_out": w_out, "norm_weight": norm_weight, "norm_bias": norm_bias,
                "scale": scale, "shift": shift, "eps": eps, "gate": gate, "b_q": b_q, "b_kv": b_kv, "b_out": b_out,
                "k_offsets": k_offsets, "h": h, "q": q, "k": k, "v": v, "o": o, "lse": lse, "pre": pre}
    return y, kept


def cross_attention_block_backward(dy: torch.Tensor, kept: dict):
    """The gradients of cross_attention_block() for its output's gradient dy, from what it kept: a dict of "x", "context", "w_q", "w_kv",
    "w_out" and, of the arguments that were given, "b_q", "b_kv", "b_out", "gate", "norm_weight", "norm_bias", "scale", "shift". The
    residual's is dy itself, and "x" is the norm's input's alone: where x is the residual too, the two are added."""
    f = kept
    B, N, H, d = f["o"].shape
    M, Hk = f["context"].shape[1], f["k"].shape[1]
    given = lambda name, gradient: [gradient] if f[name] is not None else []
    with _on_device(dy.device):
        out = linear_backward(dy, f["o"].view(B, N, H * d), f["w_out"], pre=f["pre"], gate=f["gate"],
                              want=["dx", "dw"] + given("b_out", "dbias") + given("gate", "dgate"))
        dq = torch.empty(B, N, H, d, dtype=dy.dtype, device=dy.device)
        dkv = torch.empty(B, M, 2, Hk, d, dtype=dy.dtype, device=dy.device)
        dk, dv = dkv.permute(2, 0, 3, 1, 4)
        attention_backward(out["dx"].view(B, N, H, d).transpose(1, 2), f["q"], f["k"], f["v"], f["o"].transpose(1, 2), f["lse"],
                           k_offsets=f["k_offsets"], out={"dq": dq.transpose(1, 2), "dk": dk, "dv": dv})
        into = linear_backward(dq.view(B, N, H * d), f["h"], f["w_q"], want=["dx", "dw"] + given("b_q", "dbias"))
        text = linear_backward(dkv.view(B, M, 2 * Hk * d), f["context"], f["w_kv"], want=["dx", "dw"] + given("b_kv", "dbias"))
        norm = layer_norm_backward(into["dx"], f["x"], f["norm_weight"], f["norm_bias"], scale=f["scale"], eps=f["eps"], shift=f["shift"],
                                   want=["dx"] + given("norm_weight", "dweight") + given("norm_bias", "dbias") + given("scale", "dscale")
                                   + given("shift", "dshift"))
    r = {"x": norm["dx"], "context": text["dx"], "w_q": into["dw"], "w_kv": text["dw"], "w_out": out["dw"]}
    for name, source, gradient in (("b_q", into, "dbias"), ("b_kv", text, "dbias"), ("b_out", out, "dbias"), ("gate", out, "dgate"),
                                   ("norm_weight", norm, "dweight"), ("norm_bias", norm, "dbias"), ("scale", norm, "dscale"),
                                   ("shift", norm, "dshift")):
        if gradient in source and f[name] is not None:
            r[name] = source[gradient]
    return r
