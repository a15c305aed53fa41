"""ctypes binding of include/bitstack_f8.h (argument marshalling only): products in 8-bit floating point with a scale for each block
of 128, the same grouped by expert, and the routing around them.

8-bit values are torch.float8_e4m3fn; power-of-two scales are torch.float8_e8m0fnu, others torch.float32.  A weight is a pair (q, scales) of
tensors, [out, in] and [ceil(out / 128), ceil(in / 128)], with a leading dimension for the weights of a layer of experts; the rows of q lie
a multiple of 16 bytes apart.  Without `stream` everything runs on the current stream of the tensors' device; with it, what a call allocates belongs
to that stream, and the caller orders it with the streams that made the inputs and use the outputs."""
from __future__ import annotations

import ctypes as C
import threading
from typing import NamedTuple

import torch

from . import binding
from .binding import BitStackError, _check

T_F16, T_F32, T_BF16, T_F8 = 0, 1, 2, 3
S_E8M0, S_F32 = 0, 1
_TYPES = {torch.float16: T_F16, torch.float32: T_F32, torch.bfloat16: T_BF16}
_SCALES = {torch.float8_e8m0fnu: S_E8M0, torch.float32: S_F32}
_lib = None


class _Weight(C.Structure):
    _fields_ = [("q", C.c_void_p), ("ld", C.c_size_t), ("scales", C.c_void_p), ("scale_type", C.c_int), ("out", C.c_int),
                ("inn", C.c_int), ("experts", C.c_int)]


class _Rows(C.Structure):
    _fields_ = [("x", C.c_void_p), ("scales", C.c_void_p), ("ld", C.c_size_t), ("dtype", C.c_int), ("rows", C.c_int), ("gated", C.c_int)]


class _Args(threading.local):
    """argument blocks of one thread, filled anew for every call"""

    def __init__(self):
        self.w, self.x = _Weight(), _Rows()
        self.wp, self.xp = C.byref(self.w), C.byref(self.x)


_args = _Args()


def _f8_lib():
    global _lib
    if _lib is None:
        L = binding.lib()
        vp, i32, sz = C.c_void_p, C.c_int, C.c_size_t
        for name, res, args in (
            ("bitstack_f8_row_bytes", sz, [i32]),
            ("bitstack_f8_row_scales", sz, [i32]),
            ("bitstack_f8_quantise", i32, [vp, i32, sz, i32, i32, i32, vp, vp, vp]),
            ("bitstack_f8_quantise_weight", i32, [vp, i32, sz, i32, i32, vp, sz, vp, vp]),
            ("bitstack_f8_workspace_bytes", sz, [i32] * 5),
            ("bitstack_f8_call_workspace_bytes", sz, [vp, vp, i32, i32, i32]),
            ("bitstack_f8_linear", i32, [vp, vp, vp, i32, sz, vp, sz, vp]),
            ("bitstack_f8_grouped_linear", i32, [vp, vp, vp, vp, i32, vp, i32, sz, vp, sz, vp]),
            ("bitstack_route_workspace_bytes", sz, [i32] * 3),
            ("bitstack_route", i32, [vp, i32, sz, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]),
            ("bitstack_combine", i32, [vp, i32, sz, i32, i32, vp, vp, i32, i32, vp, sz, vp]),
        ):
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        _lib = L
    return _lib


class F8Rows(NamedTuple):
    """Activations in 8 bits, as quantise_f8 makes them: several products may read them.  q [rows, in rounded up to 128], scales
    [blocks / 4, rows, 4] (blocks: ceil(in / 128), rounded up to 4), `width` = in."""
    q: torch.Tensor
    scales: torch.Tensor
    width: int

    def values(self) -> torch.Tensor:
        """the numbers they stand for, fp32 [rows, width]"""
        n, kb = self.q.shape[0], self.q.shape[1] // 128
        s = self.scales.transpose(0, 1).reshape(n, -1)[:, :kb].contiguous().view(torch.float8_e8m0fnu).float()
        return (self.q.float().view(n, kb, 128) * s[:, :, None]).view(n, -1)[:, : self.width]


class Routing(NamedTuple):
    """What `route` returns; see bitstack_route."""
    experts: torch.Tensor   # int32 [tokens, top_k], -1 where there is none
    weights: torch.Tensor   # fp32 [tokens, top_k]
    slots: torch.Tensor     # int32 [tokens, top_k]: the row of (token, j), -1 where there is none
    rows: torch.Tensor      # int32 [tokens * top_k]: the token of a row, -1 past the last one
    offsets: torch.Tensor   # int32 [experts + 1]


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _type(t: torch.Tensor, what: str) -> int:
    code = _TYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"{what}: float16, bfloat16 or float32, not {t.dtype}")
    return code


class _On:
    """A stream that is not the current one of the tensors' device: its handle, and the context in which a call allocates, so that what it
    allocates belongs to that stream.  Inputs are kept from reuse until the stream has passed the call."""

    def __init__(self, device, stream, inputs):
        if stream is None:
            stream = torch.cuda.current_stream(device)
        else:
            _need(stream.device == device, "the stream is another device's")
            if stream != torch.cuda.current_stream(device):
                for t in inputs:
                    if t is not None:
                        t.record_stream(stream)
        self.handle = stream.cuda_stream
        self._ctx = torch.cuda.stream(stream)   # its device too

    def __enter__(self):
        self._ctx.__enter__()
        return self.handle

    def __exit__(self, *exc):
        return self._ctx.__exit__(*exc)


class _Current:
    """The current stream of the current device: nothing to enter (entering costs as much as a small launch)."""

    def __init__(self, index):
        self.index = index

    def __enter__(self):
        return _raw_stream(self.index)

    def __exit__(self, *exc):
        return None


_raw_stream = torch._C._cuda_getCurrentRawStream
_current: dict = {}


def _on(device, stream, inputs):
    if device.type != "cuda":
        raise ValueError(f"tensors on a GPU are needed, not on {device}")
    index = device.index
    if stream is None and index == torch._C._cuda_getDevice():
        on = _current.get(index)
        if on is None:
            on = _current[index] = _Current(index)
        return on
    return _On(device, stream, inputs)


def _same_device(device, *tensors):
    for t in tensors:
        if t is not None and t.device != device:
            raise ValueError(f"all tensors have to be on {device}: one is on {t.device}")


def _matrix(t: torch.Tensor, what: str):
    """elements from row to row"""
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or (stride[1] != 1 and shape[1] > 1):
        raise ValueError(f"{what}: a matrix whose rows are contiguous is needed")
    return stride[0] if shape[0] > 1 else shape[1]


def _fill_weight(q, scales, grouped):
    if q.dtype is not torch.float8_e4m3fn:
        raise ValueError(f"q: float8_e4m3fn, not {q.dtype}")
    kind = _SCALES.get(scales.dtype)
    if kind is None:
        raise ValueError(f"scales: float8_e8m0fnu or float32, not {scales.dtype}")
    shape, stride = q.shape, q.stride()
    _need(len(shape) == (3 if grouped else 2) and (stride[-1] == 1 or shape[-1] == 1), "q: rows of e4m3, [out, in] or [experts, out, in]")
    out, inn = shape[-2], shape[-1]
    e = shape[0] if grouped else 1
    # experts of one row each: their distance is the rows'
    ld = stride[-2] if out > 1 else stride[0] if e > 1 else -(-inn // 16) * 16
    _need(e == 1 or stride[0] == out * ld, "q: the experts' weights have to follow one another")
    want = (-(-out // 128), -(-inn // 128))
    if scales.shape != ((e, *want) if grouped else want) or not scales.is_contiguous():
        raise ValueError(f"scales: one for each 128 x 128 block of q, {want}, contiguous")
    w = _args.w
    w.q, w.ld, w.scales, w.scale_type, w.out, w.inn, w.experts = q.data_ptr(), ld, scales.data_ptr(), kind, out, inn, e
    return out, inn, e


def _fill_rows(x, inn, gated):
    a = _args.x
    if isinstance(x, F8Rows):
        _need(not gated, "gated: apply it in quantise_f8")
        L = _f8_lib()
        if x.width != inn:
            raise ValueError(f"x has {x.width} columns, the weight {inn}")
        _need(x.q.dtype is torch.float8_e4m3fn and x.q.is_contiguous() and x.scales.is_contiguous() and x.scales.element_size() == 1
              and tuple(x.q.shape[1:]) == (L.bitstack_f8_row_bytes(inn),) and tuple(x.scales.shape) == (L.bitstack_f8_row_scales(inn) // 4, x.q.shape[0], 4),
              "x: as quantise_f8 makes it")
        a.x, a.scales, a.ld, a.dtype, a.rows, a.gated = x.q.data_ptr(), x.scales.data_ptr(), 0, T_F8, x.q.shape[0], 0
        return x.q.shape[0], torch.float16, x[:2]
    t = _type(x, "x")
    ld = _matrix(x, "x")
    rows, width = x.shape
    if width != (2 * inn if gated else inn):
        raise ValueError(f"x has {width} columns, the weight {inn}{' (gated: twice as many are needed)' if gated else ''}")
    a.x, a.scales, a.ld, a.dtype, a.rows, a.gated = x.data_ptr(), None, ld, t, rows, 1 if gated else 0
    return rows, x.dtype, (x,)


def _product(x, q, scales, offsets, index, gated, y, out_dtype, workspace, stream, grouped):
    L = _f8_lib()
    out, inn, experts = _fill_weight(q, scales, grouped)
    rows, dtype, held = _fill_rows(x, inn, gated)
    device = q.device
    _same_device(device, scales, offsets, index, y, workspace, *held)
    if grouped:
        _need(offsets.dtype is torch.int32 and offsets.is_contiguous() and offsets.shape == (experts + 1,), "offsets: int32 [experts + 1]")
        if index is not None:
            _need(index.dtype is torch.int32 and index.dim() == 1 and index.is_contiguous(), "rows: int32 [rows of y]")
            rows = index.shape[0]
    args = _args
    with _on(device, stream, (*held, q, scales, offsets, index, y, workspace)) as handle:
        if y is None:
            y = q.new_empty((rows, out), dtype=out_dtype or dtype)
            ld_y = out
        else:
            if y.shape != (rows, out) or (out_dtype is not None and y.dtype is not out_dtype):
                raise ValueError(f"y: [{rows}, {out}] is needed")
            ld_y = _matrix(y, "y")
        t = _type(y, "y")
        if workspace is None:
            nbytes = L.bitstack_f8_call_workspace_bytes(args.xp, args.wp, rows, t, grouped)
            if nbytes:
                workspace = q.new_empty(nbytes, dtype=torch.uint8)
        else:
            _need(workspace.is_contiguous(), "workspace: contiguous")
            nbytes = workspace.numel() * workspace.element_size()
        ws = None if workspace is None else workspace.data_ptr()
        if grouped:
            rc = L.bitstack_f8_grouped_linear(args.xp, args.wp, offsets.data_ptr(), None if index is None else index.data_ptr(), rows, y.data_ptr(), t, ld_y, ws,
                                              nbytes, handle)
        else:
            rc = L.bitstack_f8_linear(args.xp, args.wp, y.data_ptr(), t, ld_y, ws, nbytes, handle)
        if rc:
            raise BitStackError(rc, "bitstack_f8_grouped_linear" if grouped else "bitstack_f8_linear")
    return y


def f8_workspace_bytes(x_rows: int, inn: int, y_rows: int, out: int, experts: int = 1) -> int:
    """bitstack_f8_workspace_bytes: of a `workspace` for products with up to so many rows.  One that a call allocates for itself may be larger and then
    makes it faster."""
    n = int(_f8_lib().bitstack_f8_workspace_bytes(x_rows, inn, y_rows, out, experts))
    if n == 0:
        raise BitStackError(-2, "bitstack_f8_workspace_bytes")
    return n


def linear_f8(x, q, scales, *, gated: bool = False, y=None, out_dtype=None, workspace=None, stream=None):
    """bitstack_f8_linear: y = x8 w^T.  x [tokens, in] (gated: [tokens, 2 in], gate and value side by side) or an F8Rows; q [out, in] and its
    scales.  y has the type of x (fp16 for F8Rows) unless given.  workspace: a uint8 tensor of f8_workspace_bytes, else one is allocated."""
    return _product(x, q, scales, None, None, gated, y, out_dtype, workspace, stream, False)


def grouped_linear_f8(x, q, scales, offsets, rows=None, *, gated: bool = False, y=None, out_dtype=None, workspace=None, stream=None):
    """bitstack_f8_grouped_linear: the rows [offsets[e], offsets[e + 1]) of y are products with expert e's weight, of x's rows of the same
    number, or of x[rows] where `rows` is given (Routing.rows).  q [experts, out, in].  Rows past the last group are zero."""
    return _product(x, q, scales, offsets, rows, gated, y, out_dtype, workspace, stream, True)


def quantise_f8(x, *, gated: bool = False, stream=None) -> F8Rows:
    """bitstack_f8_quantise: x [rows, in] (gated: [rows, 2 in]) -> F8Rows."""
    L = _f8_lib()
    t, ld = _type(x, "x"), _matrix(x, "x")
    _need(not gated or x.shape[1] % 2 == 0, "gated: gate and value side by side are needed")
    n, inn = x.shape[0], x.shape[1] // (2 if gated else 1)
    with _on(x.device, stream, (x,)) as handle:
        q = torch.empty((n, L.bitstack_f8_row_bytes(inn)), dtype=torch.float8_e4m3fn, device=x.device)
        s = torch.empty((L.bitstack_f8_row_scales(inn) // 4, n, 4), dtype=torch.uint8, device=x.device)
        _check(L.bitstack_f8_quantise(x.data_ptr(), t, ld, n, inn, int(gated), q.data_ptr(), s.data_ptr(), handle), "bitstack_f8_quantise")
    return F8Rows(q, s, inn)


def _f8_output(out, shape, device):
    """(q, scales) that the caller gives to be written, as quantise_weight_f8 makes them or with rows closer together"""
    q, s = out
    e, rows, inn = shape
    q3, s3 = (q, s) if q.dim() == 3 else (q[None], s[None])
    _need(q.dtype is torch.float8_e4m3fn and tuple(q3.shape) == shape and (q3.stride(2) == 1 or inn == 1), f"out: q, float8_e4m3fn {list(shape[3 - q.dim():])}")
    _need(s.dtype is torch.float8_e8m0fnu and tuple(s3.shape) == (e, -(-rows // 128), -(-inn // 128)) and s.is_contiguous(), "out: scales, float8_e8m0fnu, one for each 128 x 128 block, contiguous")
    _same_device(device, q, s)
    ld = q3.stride(1) if rows > 1 else -(-inn // 16) * 16
    _need(e == 1 or (q3.stride(0) >= rows * ld and q3.stride(0) % 16 == 0), "out: q, experts a multiple of 16 bytes apart")
    written = (e - 1) * q3.stride(0) + (rows - 1) * ld + min(ld, -(-inn // 128) * 128)
    _need(q.storage_offset() + written <= q.untyped_storage().nbytes(), "out: q's last row ends with its last column: it is written up to a multiple of 16")
    return q3, s3, ld


def quantise_weight_f8(w, *, out=None, stream=None):
    """bitstack_f8_quantise_weight for w [out, in] or [experts, out, in] -> (q, scales), q's rows a multiple of 128 bytes apart and zero
    past `in`; or into `out`, such a pair whose rows may be any multiple of 16 bytes apart (zeroed past `in` up to there or to a multiple of 128)."""
    L = _f8_lib()
    _need(w.dim() in (2, 3), "w: [out, in] or [experts, out, in]")
    t = _type(w, "w")
    each = w if w.dim() == 3 else w[None]
    e, rows, inn = each.shape
    with _on(w.device, stream, (w, *(out or ()))) as handle:
        if out is None:
            ld_q = int(L.bitstack_f8_row_bytes(inn))
            q = torch.empty((e, rows, ld_q), dtype=torch.float8_e4m3fn, device=w.device)
            s = torch.empty((e, -(-rows // 128), -(-inn // 128)), dtype=torch.float8_e8m0fnu, device=w.device)
        else:
            _need(out[0].dim() == w.dim() and out[1].dim() == w.dim(), "out: q and scales of as many dimensions as w")
            q, s, ld_q = _f8_output(out, (e, rows, inn), w.device)
        for i in range(e):
            _check(L.bitstack_f8_quantise_weight(each[i].data_ptr(), t, _matrix(each[i], "w"), rows, inn, q[i].data_ptr(), ld_q, s[i].data_ptr(),
                                                 handle), "bitstack_f8_quantise_weight")
    if out is not None:
        return out
    q = q[:, :, :inn]
    return (q, s) if w.dim() == 3 else (q[0], s[0])


def route(logits, top_k: int, *, renormalise: bool = True, stream=None) -> Routing:
    """bitstack_route: logits [tokens, experts] -> Routing."""
    L = _f8_lib()
    t, ld = _type(logits, "logits"), _matrix(logits, "logits")
    n, e = logits.shape
    with _on(logits.device, stream, (logits,)) as handle:
        nbytes = L.bitstack_route_workspace_bytes(n, e, top_k)
        if nbytes == 0:
            raise BitStackError(-2, "bitstack_route_workspace_bytes")
        # one allocation: experts, weights, slots, rows (each nk words), the offsets, then (256-byte aligned) the workspace where it is a small part; a
        # larger one is not kept with the tables (300 tokens, 6 of 64 experts: 15.7 us, with an allocation more 16.9)
        nk = n * top_k
        at = -(-(4 * nk + e + 1) // 64) * 64
        apart = nbytes > max(256, at // 2)
        words = torch.empty(at if apart else at + nbytes // 4, dtype=torch.int32, device=logits.device)
        experts, weights, slots, rows, offsets, _ = words.split_with_sizes((nk, nk, nk, nk, e + 1, words.shape[0] - 4 * nk - e - 1))
        r = Routing(experts.view(n, top_k), weights.view(torch.float32).view(n, top_k), slots.view(n, top_k), rows, offsets)
        p, step = words.data_ptr(), 4 * nk
        counts = torch.empty(nbytes, dtype=torch.uint8, device=logits.device) if apart else words
        ws = counts.data_ptr() if apart else p + 4 * at
        _check(L.bitstack_route(logits.data_ptr(), t, ld, n, e, top_k, renormalise, p, p + step, p + 2 * step, p + 3 * step, p + 4 * step, ws, nbytes,
                                handle), "bitstack_route")
    return r


def combine(h, slots, weights, *, y=None, stream=None):
    """bitstack_combine: y[t] = sum_j weights[t, j] h[slots[t, j]], a slot of -1 adds nothing.  h [rows, width]; y has its type."""
    L = _f8_lib()
    t, ld = _type(h, "h"), _matrix(h, "h")
    _need(slots.dtype is torch.int32 and weights.dtype is torch.float32 and slots.dim() == 2 and slots.shape == weights.shape
          and slots.is_contiguous() and weights.is_contiguous(), "slots: int32, weights: float32, both [tokens, top_k] and contiguous")
    _same_device(h.device, slots, weights, y)
    n, k = slots.shape
    with _on(h.device, stream, (h, slots, weights, y)) as handle:
        if y is None:
            y = h.new_empty((n, h.shape[1]))
        else:
            _need(tuple(y.shape) == (n, h.shape[1]) and y.dtype is h.dtype, "y: [tokens, width] of h's type")
        _check(L.bitstack_combine(h.data_ptr(), t, ld, h.shape[0], h.shape[1], slots.data_ptr(), weights.data_ptr(), n, k, y.data_ptr(), _matrix(y, "y"),
                                  handle), "bitstack_combine")
    return y
