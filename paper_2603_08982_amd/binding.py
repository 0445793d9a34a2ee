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
]

ACTIVATIONS = {"none": 0, "silu": 1, "gelu": 2, "gelu_tanh": 3}
ROTARY_NORMS = {None: 0, "head": 1, "token": 2}
ROTARY_HALVES = 4

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


def _gate_strides(gate, lead, d_out: int):
    """Strides of a gate of tokens (lead + (d_out,)) or of batch entries (without the tokens' axis), and whether it is the first."""
    if gate is None:
        return _NO_ROWS, False
    per_token = gate.dim() == len(lead) + 1
    _require(tuple(gate.shape) == (*lead, d_out) or tuple(gate.shape) == (*lead[:-1], d_out), "gate: expected [B,N,d_out] or [B,d_out] ([N,d_out] or [d_out] for one batch entry)")
    _require(d_out == 1 or gate.stride(-1) == 1, "gate: expected contiguous d_out")
    if per_token:
        return _I64x2(gate.stride(0) if len(lead) == 2 else 0, gate.stride(-2)), True
    return _I64x2(gate.stride(0) if len(lead) == 2 else 0, 0), False


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
