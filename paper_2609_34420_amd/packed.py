"""Packed batches of graphs of unlike sizes: attention with capped scores, a
prefix mask and dropout of the probabilities (C ABI gt_attn_pack_*, whose
header states the definitions).

    pack = gt_attn_pack([37, 12, 405], H=8)                  # graphs of 37, 12 and 405 nodes
    o, lse = gt_attn_pack_fwd(q, k, v, spd, table, pack, cap=30.0, dropout=GTDropout(0.1, seed, step))
    dq, dk, dv, dtable = gt_attn_pack_bwd(q, k, v, spd, table, pack, o, lse, d_o, cap=30.0,
                                          dropout=GTDropout(0.1, seed, step))
    pack = gt_attn_pack([1, 1], H=8, n_k=[900, 4000], backward=False)    # one new node against each graph's keys
    pack = gt_attn_pack(sizes, H=8, prefix=[0] * len(sizes)) # causal; prefix[g] first keys are seen by all

q, k, v [H, T, d] hold the graphs' rows one behind the other (T may be larger
than their total: the rows behind it are left alone); any strides whose last is
1 and whose others are multiples of 16 bytes, so a [T, H, d] tensor is passed as
x.transpose(0, 1), and one that heads share as an expanded one (its gradient
comes per head). spd holds the graphs' [n_q, n_k] uint8 distances one behind
the other.

Graphs of one size that take no cap, prefix or dropout run faster through
gt_attn_fwd_batch and gt_attn_bwd_batch.
"""
from __future__ import annotations

import ctypes
import math
from typing import NamedTuple

import numpy as np
import torch

from . import (_F, _I32, _I64, _P, _check, _dt, _need, _ptr, _qdims, _raw_stream, _shape, _table, _workspace, lib)

__all__ = ["GTDropout", "GTPack", "gt_attn_pack", "gt_attn_pack_bwd", "gt_attn_pack_bwd_workspace_size",
           "gt_attn_pack_fwd", "gt_attn_pack_fwd_workspace_size"]


class GTDropout(NamedTuple):
    """Dropout of the attention probabilities: rate p, 64-bit seed, and a 32-bit
    offset (a layer and step number, say). offset_dev: an int32 device tensor of
    one element that is added to offset when the kernels run, so that replays of
    a captured graph can draw anew. The backward takes what the forward took."""
    p: float
    seed: int
    offset: int = 0
    offset_dev: torch.Tensor | None = None


class _Rows(ctypes.Structure):
    _fields_ = [("p", _P), ("head_stride", _I64), ("row_stride", _I64)]


# A call's rows arguments are one array of their fields, passed by address (a
# structure object for each takes half a microsecond of a small call's ten).
_ROWS_BYTES = ctypes.sizeof(_Rows)
_Rows4, _Rows8 = _I64 * 12, _I64 * 24


class _Info(ctypes.Structure):
    _fields_ = [("total_q", _I64), ("total_k", _I64), ("spd_bytes", _I64), ("plan_bytes", _I64),
                ("n_graphs", _I32), ("H", _I32), ("backward", _I32), ("jobs", _I32 * 3), ("merges", _I32), ("parts", _I32),
                ("slots", _I32), ("slots3", _I32), ("short_jobs", _I32), ("short_slots", _I32), ("short_blocks", _I32), ("job_off", _I64 * 3),
                ("merge_off", _I64), ("short_off", _I64)]


class _Dropout(ctypes.Structure):
    _fields_ = [("p", ctypes.c_double), ("seed", ctypes.c_uint64), ("offset", ctypes.c_uint32), ("offset_dev", _P)]


def _register(L: ctypes.CDLL) -> None:
    R, Z, info, drop = _P, ctypes.c_size_t, _P, _P
    L.gt_attn_pack_plan.restype = _I32
    L.gt_attn_pack_plan.argtypes = [_I32, _I32, _P, _P, _P, _P, _P, _I32, _P, Z, info]
    L.gt_attn_pack_fwd_workspace_size.restype = Z
    L.gt_attn_pack_fwd_workspace_size.argtypes = [info, _I32]
    L.gt_attn_pack_bwd_workspace_size.restype = Z
    L.gt_attn_pack_bwd_workspace_size.argtypes = [info, _I32]
    L.gt_attn_pack_fwd.restype = _I32
    L.gt_attn_pack_fwd.argtypes = [info, _P, R, R, R, _P, _P, _I32, R, _P, _I64, _P, Z, _I32, _I32, _F, _F, drop, _P]
    L.gt_attn_pack_bwd.restype = _I32
    L.gt_attn_pack_bwd.argtypes = [info, _P, R, R, R, _P, _P, _I32, R, _P, _I64, R, R, R, R, _P, _P, Z, _I32, _I32,
                                   _F, _F, drop, _P]


class GTPack:
    """A packed batch's sizes and its plan on the device (from gt_attn_pack).
    total_q, total_k: packed rows; spd_bytes: bytes of distances; H: heads."""

    def __init__(self, info: _Info, plan: torch.Tensor):
        self._info = info
        self._at = ctypes.addressof(info)
        self._plan = plan
        self._plan_at = plan.data_ptr()
        self._device_index = plan.get_device()
        # the stream whose order the plan's memory goes by
        self._stream = torch.cuda.current_stream(plan.device).cuda_stream if plan.is_cuda else 0
        self._ws = {}                                   # workspace sizes by what they depend on beside the plan
        self.total_q, self.total_k = info.total_q, info.total_k
        self.spd_bytes, self.H, self.n_graphs = info.spd_bytes, info.H, info.n_graphs
        self.backward = bool(info.backward)
        self.device = plan.device

    # (a plan holds addresses: a copy of its attributes would keep those of the original)
    def __copy__(self):
        return self

    def __reduce__(self):
        return _copied_pack, (bytes(self._info), self._plan)


def _copied_pack(info: bytes, plan: torch.Tensor) -> GTPack:
    return GTPack(_Info.from_buffer_copy(info), plan)


def _sizes(x, name: str, n: int | None, dtype=np.int32) -> np.ndarray:
    a = np.asarray(x)
    _need(a.ndim == 1 and (a.size == 0 or a.dtype.kind in "iu"), f"{name} must be a sequence of whole numbers")
    _need(n is None or a.size == n, f"{name} must have one entry per graph")
    _need(a.size > 0, f"{name} must not be empty")
    lim = np.iinfo(dtype).max
    _need(int(a.min()) >= 0 and int(a.max()) <= lim, f"{name} must lie in 0..{lim}")
    return np.ascontiguousarray(a, dtype=dtype)


def gt_attn_pack(n_q, H: int, n_k=None, prefix=None, spd_off=None, spd_ld=None, device="cuda",
                 backward: bool = True) -> GTPack:
    """The plan of a packed batch (C ABI gt_attn_pack_plan) for graphs of n_q[g]
    query rows and n_k[g] keys (n_q by default) and H heads. prefix: None, or the
    number of leading keys that every row of a graph sees beside those up to its own
    position (0: causal). spd_off, spd_ld: where a graph's distances lie in spd (by
    default one matrix of n_q[g] rows of the stride behind the other) and their row
    stride (n_k[g]).
    backward=False: a plan for the forward alone, sooner made where a few rows meet
    many keys (the new nodes of 16 graphs of 1000 to 16000: 40 us for 65). Made
    once per batch of sizes, it serves every layer's and step's calls; a captured
    graph reads it at each replay, so it has to live as long, and keeps to its sizes.
    The copy to the device waits for what the current stream still has to do, and is
    complete on return: a plan made under a stream of its own does not wait for the
    queue of another, and may be used on any."""
    nq = _sizes(n_q, "n_q", None)
    nk = nq if n_k is None else _sizes(n_k, "n_k", nq.size)
    opt = [None if x is None else _sizes(x, name, nq.size, t)
           for x, name, t in ((prefix, "prefix", np.int32), (spd_off, "spd_off", np.int64), (spd_ld, "spd_ld", np.int64))]
    _need(isinstance(H, int) and 1 <= H <= 65535, "H must lie in 1..65535")
    info = _Info()

    def call(buf):
        return lib().gt_attn_pack_plan(nq.size, H, nq.ctypes.data, nk.ctypes.data,
                                       *(None if x is None else x.ctypes.data for x in opt), int(bool(backward)),
                                       None if buf is None else buf.ctypes.data,
                                       0 if buf is None else buf.nbytes, ctypes.byref(info))

    # (64 bytes per 32 rows and list in most plans; a second call where it is more)
    blocks = int((nq.astype(np.int64) + 31).sum() + ((nk.astype(np.int64) + 31).sum() if backward else 0)) // 32
    buf = np.empty(8192 + 192 * blocks + 512 * min(nq.size, 64), dtype=np.uint8)
    st = call(buf)
    if st == 3 and info.plan_bytes > buf.nbytes:
        buf = np.empty(info.plan_bytes, dtype=np.uint8)
        st = call(buf)
    _check(st, "gt_attn_pack_plan")
    return GTPack(info, torch.from_numpy(buf[:max(1, info.plan_bytes)]).to(device))


def gt_attn_pack_fwd_workspace_size(pack: GTPack, d: int) -> int:
    n = pack._ws.get(("fwd", d))
    if n is None:
        n = pack._ws["fwd", d] = int(lib().gt_attn_pack_fwd_workspace_size(pack._at, d))
    return n


def gt_attn_pack_bwd_workspace_size(pack: GTPack, n_buckets: int) -> int:
    n = pack._ws.get(("bwd", n_buckets))
    if n is None:
        n = pack._ws["bwd", n_buckets] = int(lib().gt_attn_pack_bwd_workspace_size(pack._at, n_buckets))
    return n


def _rows(t, name: str, H: int, rows: int, d: int, dtype, dev: int, written: bool = False) -> tuple:
    """A [H, >= rows, d] tensor as the fields of the C ABI's rows."""
    if not isinstance(t, torch.Tensor) or t.dim() != 3:
        raise ValueError(f"{name} must be a 3-D tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    h, n, w = t.shape
    if h != H or w != d or n < rows:
        raise ValueError(f"{name} must have shape ({H}, >= {rows}, {d}), got ({h}, {n}, {w})")
    p = t.data_ptr()
    if p % 16:
        raise ValueError(f"{name} must be 16-byte aligned")
    if t.is_contiguous():
        hs, rs = n * d, d
    else:
        hs, rs, one = t.stride()
        unit = 8 if dtype == torch.bfloat16 else 4
        if one != 1 or (rows > 1 and (rs % unit or not d <= rs <= 1 << 23)) or (H > 1 and (hs % unit or hs < 0)):
            raise ValueError(f"{name} must have unit feature stride, and row and head strides that are multiples of "
                             f"16 bytes, the row stride in {d}..{1 << 23}; got {t.stride()}")
        if written and H > 1 and rows > 0 and not (hs >= (rows - 1) * rs + d or (rs >= (H - 1) * hs + d and hs >= d)):
            raise ValueError(f"{name} is written: its rows must not overlap")
        # (a stride that no element is reached by may be anything in torch)
        hs, rs = hs if H > 1 else 0, rs if rows > 1 else d
    if dev >= 0 and t.get_device() != dev:
        raise ValueError("tensors must be device tensors on one device")
    return p, hs, rs


def _dropout(dropout, dev: int):
    _need(isinstance(dropout, GTDropout), "dropout must be a GTDropout or None")
    if dropout.p == 0:
        return None
    p, seed, offset, dyn = dropout
    _need(0.0 <= p < 1.0 and round(p * 65536) <= 65535, f"dropout must lie in 0 <= p < 1 - 2^-17, got {p}")
    _need(0 <= seed < 1 << 64, "seed must be a 64-bit unsigned number")
    _need(0 <= offset < 1 << 32, "offset must be a 32-bit unsigned number")
    if dyn is not None:
        _need(isinstance(dyn, torch.Tensor) and dyn.dtype == torch.int32 and dyn.numel() == 1 and dyn.is_cuda
              and dyn.get_device() == dev, "offset_dev must be an int32 tensor of one element on q's device")
    return ctypes.byref(_Dropout(p, seed, offset, _ptr(dyn)))


def _common(q, k, v, spd, table, pack, scale, cap):
    """Checks of both calls; returns what they pass on."""
    if not isinstance(pack, GTPack):
        raise ValueError("pack must come from gt_attn_pack")
    if isinstance(q, torch.Tensor) and q.dim() == 3 and q.shape[1] == 0:
        dt = q.dtype                                   # a batch without query rows
    else:
        dt = _qdims(q, "q", 3)
    H, _, d = q.shape
    if H != pack.H:
        raise ValueError(f"the plan is for {pack.H} heads, q has {H}")
    rows = (*_rows(q, "q", H, pack.total_q, d, dt, -1), *_rows(k, "k", H, pack.total_k, d, dt, -1),
            *_rows(v, "v", H, pack.total_k, d, dt, -1))
    if k.shape != v.shape:
        raise ValueError("k and v must have one shape")
    if not (isinstance(spd, torch.Tensor) and spd.dtype == torch.uint8 and spd.is_contiguous()
            and spd.numel() >= pack.spd_bytes):
        raise ValueError(f"spd must be a contiguous uint8 tensor of at least {pack.spd_bytes} bytes")
    _table(table, H)
    if not table.is_contiguous():
        raise ValueError("table must be contiguous")
    dev = q.get_device()
    if dev < 0:
        raise ValueError("tensors must be device tensors")
    if pack._device_index != dev:
        raise ValueError("the plan must be on q's device")
    _same_device(dev, k, v, spd, table)
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    cap = 0.0 if cap is None else float(cap)
    if cap != 0.0 and not 2.0 ** -10 <= cap <= 1024.0:
        raise ValueError(f"cap must lie in 2^-10..2^10, or be None, got {cap}")
    return dt, H, d, dev, rows, scale, cap


def _same_device(dev: int, *ts):
    for t in ts:
        if t is not None and t.get_device() != dev:
            raise ValueError("tensors must be device tensors on one device")


def _lse(lse, H: int, T: int):
    if not (isinstance(lse, torch.Tensor) and lse.dtype == torch.float32 and lse.shape == (H, T)
            and lse.is_contiguous()):
        raise ValueError(f"lse must be a contiguous float32 tensor of shape ({H}, {T})")


def _on_stream(stream, q, given, call):
    """call() with `stream` as the current one, so that what it allocates (the results
    whose place in `given` is None, and a workspace) is that stream's memory: a block of
    another's may have work pending there. The results are kept from reuse until the
    caller's current stream, where they go next, has passed them too."""
    if isinstance(q, torch.Tensor) and stream.device_index != q.get_device():
        raise ValueError("stream must be of the tensors' device")
    cur = torch.cuda.current_stream(stream.device)
    with torch.cuda.stream(stream):
        got = call()
    for t, g in zip(got, given):
        if g is None and t.numel():
            t.record_stream(cur)
    return got


def _current(dev: int, pack: GTPack) -> int:
    """The raw current stream. The plan, which the caller does not see, is kept from
    reuse until a stream other than its own has passed the call."""
    raw = _raw_stream(dev) if _raw_stream is not None else torch.cuda.current_stream(dev).cuda_stream
    if raw != pack._stream:
        pack._plan.record_stream(torch.cuda.current_stream(dev))
    return raw


def _like(x):
    # (half the time of torch.empty with a shape; of another layout it would keep that)
    return torch.empty_like(x) if x.is_contiguous() else torch.empty(x.shape, device=x.device, dtype=x.dtype)


def _launch(dev: int, fn, *args) -> int:
    # kernels are launched on the current device, which must be the tensors'
    if torch.cuda.current_device() == dev:
        return fn(*args)
    with torch.cuda.device(dev):
        return fn(*args)


def gt_attn_pack_fwd(q, k, v, spd, table, pack: GTPack, scale: float | None = None, cap: float | None = None,
                     dropout: GTDropout | None = None, out=None, lse=None, workspace=None, stream=None):
    """O [H, T, d] (q's type) and LSE [H, T] fp32 of the packed batch (C ABI
    gt_attn_pack_fwd). cap: bound of the scores before the bias, None for none;
    dropout: GTDropout or None. Rows behind the batch's total stay as they are
    (uninitialised where the call allocates). stream: as if it were the current one; the
    caller orders it with the streams of what is passed in."""
    if stream is not None:
        return _on_stream(stream, q, (out, lse), lambda: gt_attn_pack_fwd(
            q, k, v, spd, table, pack, scale, cap, dropout, out, lse, workspace))
    dt, H, d, dev, rows, scale, cap = _common(q, k, v, spd, table, pack, scale, cap)
    T = q.shape[1]
    drop = None if dropout is None else _dropout(dropout, dev)
    if out is None:
        out = _like(q)
    if lse is None:
        lse = torch.empty((H, T), device=q.device, dtype=torch.float32)
    else:
        _lse(lse, H, T)
        _same_device(dev, lse)
    r = _Rows4(*rows, *_rows(out, "out", H, pack.total_q, d, dt, dev, written=True))
    at = ctypes.addressof(r)
    need = gt_attn_pack_fwd_workspace_size(pack, d)
    if workspace is not None:
        _workspace(workspace, need, q)
    elif need:
        workspace = torch.empty(need, device=q.device, dtype=torch.uint8)
    s = _current(dev, pack)
    st = _launch(dev, lib().gt_attn_pack_fwd, pack._at, pack._plan_at, at, at + _ROWS_BYTES, at + 2 * _ROWS_BYTES,
                 spd.data_ptr(), table.data_ptr(), table.shape[1], at + 3 * _ROWS_BYTES, lse.data_ptr(), T,
                 _ptr(workspace), 0 if workspace is None else workspace.numel(), d, _dt(q), scale, cap, drop, s)
    _check(st, "gt_attn_pack_fwd")
    return out, lse


def gt_attn_pack_bwd(q, k, v, spd, table, pack: GTPack, o, lse, d_o, scale: float | None = None,
                     cap: float | None = None, dropout: GTDropout | None = None, workspace=None, grads=None,
                     stream=None):
    """dQ, dK, dV and dTable of the packed batch (C ABI gt_attn_pack_bwd), with
    the forward's arguments and results. `grads` may hold preallocated (dq, dk,
    dv, dtable); rows behind the batch's totals stay as they are. stream: as the
    forward's."""
    if stream is not None:
        return _on_stream(stream, q, (None,) * 4 if grads is None else grads, lambda: gt_attn_pack_bwd(
            q, k, v, spd, table, pack, o, lse, d_o, scale, cap, dropout, workspace, grads))
    dt, H, d, dev, rows, scale, cap = _common(q, k, v, spd, table, pack, scale, cap)
    T, nb = q.shape[1], table.shape[1]
    drop = None if dropout is None else _dropout(dropout, dev)
    _lse(lse, H, T)
    if grads is None:
        grads = [_like(x) for x in (q, k, v, table)]
    elif len(grads) != 4:
        raise ValueError("grads must be (dq, dk, dv, dtable)")
    dq, dk, dv, dtable = grads
    tq, tk = pack.total_q, pack.total_k
    if not pack.backward:
        raise ValueError("the plan was made without the backward")
    r = _Rows8(*rows, *_rows(o, "o", H, tq, d, dt, dev), *_rows(d_o, "d_o", H, tq, d, dt, dev),
               *_rows(dq, "dq", H, tq, d, dt, dev, written=True), *_rows(dk, "dk", H, tk, d, dt, dev, written=True),
               *_rows(dv, "dv", H, tk, d, dt, dev, written=True))
    at = [ctypes.addressof(r) + i * _ROWS_BYTES for i in range(8)]
    _shape(dtable, "dtable", table.shape, torch.float32)
    if not dtable.is_contiguous():
        raise ValueError("dtable must be contiguous")
    _same_device(dev, lse, dtable)
    need = gt_attn_pack_bwd_workspace_size(pack, nb)
    if workspace is not None:
        _workspace(workspace, need, q)
    else:
        workspace = torch.empty(need, device=q.device, dtype=torch.uint8)
    s = _current(dev, pack)
    st = _launch(dev, lib().gt_attn_pack_bwd, pack._at, pack._plan_at, at[0], at[1], at[2], spd.data_ptr(),
                 table.data_ptr(), nb, at[3], lse.data_ptr(), T, at[4], at[5], at[6], at[7], dtable.data_ptr(),
                 workspace.data_ptr(), workspace.numel(), d, _dt(q), scale, cap, drop, s)
    _check(st, "gt_attn_pack_bwd")
    return dq, dk, dv, dtable
