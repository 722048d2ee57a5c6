"""Torch-facing wrapper of the C ABI's operators on rows: lookup by id,
linear maps of rows grouped by type, group norm with an activation, and the
gradients of each.

Each function turns tensors into pointers and makes one call of the library;
outputs and workspaces are torch's, taken on the stream the call runs on, so
that a call can be captured into a graph.  Names follow the C ABI
(``lookup_rows`` = taurus_lookup_rows, ...).
"""
from __future__ import annotations

from typing import Optional

import torch

from . import _native as N

_CODE = {torch.float32: N.F32, torch.bfloat16: N.BF16, torch.float16: N.F16}
_ACT = {"none": N.ACT_NONE, "relu": N.ACT_RELU, "silu": N.ACT_SILU}


def _code(dtype, what: str) -> int:
    if dtype not in _CODE:
        raise ValueError(f"{what} must be float32, bfloat16 or float16, got {dtype}")
    return _CODE[dtype]


# the current stream's handle without a Stream object (4 us a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


class _Call:
    """The device and stream of one call.  Tensors made inside belong to the
    stream; when it is not the current one, tensors that come from elsewhere
    are marked as used on it."""
    __slots__ = ("device", "ptr", "ctx", "stream", "used")

    def __init__(self, first: torch.Tensor, stream, what: str):
        if not first.is_cuda:
            raise ValueError(f"{what} must be a device tensor")
        self.device = first.device
        self.ctx = self.stream = self.used = None
        index = self.device.index
        self.ptr = _raw_stream(index)
        if stream is not None:
            if stream.device != self.device:
                raise ValueError(f"the stream is on {stream.device}, {what} on {self.device}")
            if stream.cuda_stream != self.ptr:
                self.ptr, self.stream, self.used = stream.cuda_stream, stream, []
                self.ctx = torch.cuda.stream(stream)
        if self.ctx is None and torch.cuda.current_device() != index:
            self.ctx = torch.cuda.device(index)

    def __enter__(self):
        if self.ctx is not None:
            self.ctx.__enter__()
        return self

    def __exit__(self, *exc):
        if self.ctx is not None:
            self.ctx.__exit__(*exc)
        if self.used is not None:
            for t in self.used:
                t.record_stream(self.stream)

    def _mine(self, t: torch.Tensor, what: str):
        if t.device != self.device:
            raise ValueError(f"{what} must be on {self.device}, got {t.device}")
        if self.used is not None:
            self.used.append(t)

    def rows(self, t: torch.Tensor, shape, what: str, dtype=None):
        """(pointer, stride) of a row array: [rows][cols], values of a row next
        to one another, rows that do not overlap."""
        self._mine(t, what)
        if t.dim() != 2 or (shape is not None and t.shape != shape):
            want = "two dimensions" if shape is None else f"shape {tuple(shape)}"
            raise ValueError(f"{what} must have {want}, got shape {tuple(t.shape)}")
        if dtype is not None and t.dtype != dtype:
            raise ValueError(f"{what} must be {dtype}, got {t.dtype}")
        m, d = t.shape
        stride = t.stride(0) if m > 1 else d
        if (d > 1 and m > 0 and t.stride(1) != 1) or stride < d:
            raise ValueError(f"{what}: the values of a row must lie next to one another and rows must not overlap")
        return t.data_ptr(), max(stride, 1)

    def dense(self, t: Optional[torch.Tensor], shape, dtype, what: str):
        """Pointer of a contiguous array (None: a null pointer)."""
        if t is None:
            return None
        self._mine(t, what)
        if t.dtype != dtype:
            raise ValueError(f"{what} must be {dtype}, got {t.dtype}")
        if t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{what} must be contiguous with shape {tuple(shape)}, got shape {tuple(t.shape)}")
        return t.data_ptr()

    def offsets(self, off: torch.Tensor, what: str = "off"):
        """(pointer, ranges) of int64 offsets."""
        if off.dim() != 1 or off.numel() < 1:
            raise ValueError(f"{what} must hold the ranges' offsets, one more than ranges")
        return self.dense(off, off.shape, torch.int64, what), off.numel() - 1

    def out(self, given: Optional[torch.Tensor], shape, dtype, what: str, *inputs):
        """An output row array, checked against the inputs or made."""
        if given is None:
            t = torch.empty(shape, dtype=dtype, device=self.device)
            return t, t.data_ptr(), max(shape[1], 1)
        p, stride = self.rows(given, shape, what, dtype)
        for other in inputs:
            if other is not None and _overlap(given, other):
                raise ValueError(f"{what} overlaps an input")
        return given, p, stride

    def work(self, nbytes: int, call: str):
        if nbytes < 0:
            raise N.TaurusError(int(nbytes), call, N.last_error())
        if nbytes == 0:
            return None, None
        t = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        return t, t.data_ptr()


def _overlap(a: torch.Tensor, b: torch.Tensor) -> bool:
    """Whether two arrays share memory: their address ranges meet, and they
    are not different columns of one wider array."""
    def span(t):
        n = sum((s - 1) * st for s, st in zip(t.shape, t.stride())) + 1 if t.numel() else 0
        return t.data_ptr(), t.data_ptr() + n * t.element_size()
    (a0, a1), (b0, b1) = span(a), span(b)
    if a0 >= b1 or b0 >= a1:
        return False
    if a.dim() == 2 and b.dim() == 2 and a.shape[0] > 1 and b.shape[0] > 1:
        pitch = a.stride(0) * a.element_size()
        if pitch == b.stride(0) * b.element_size() and pitch > 0:
            at = (b0 - a0) % pitch
            return not (at >= a.shape[1] * a.element_size() and at + b.shape[1] * b.element_size() <= pitch)
    return True


# ----------------------------------------------------------------- lookup --

def lookup_rows(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, *, out: Optional[torch.Tensor] = None,
                out_dtype=None, stream=None) -> torch.Tensor:
    """taurus_lookup_rows: out[i] = scale * table[ids[i]], zeros where ids[i]
    is outside the table.  table [n][d], ids int32[m]; returns [m][d] of
    out_dtype (default: out's or the table's)."""
    with _Call(table, stream, "table") as c:
        tp, ts = c.rows(table, None, "table")
        n, d = table.shape
        m = ids.numel()
        ip = c.dense(ids, (m,), torch.int32, "ids")
        dtype = out_dtype or (out.dtype if out is not None else table.dtype)
        code, out_code = _code(table.dtype, "table"), _code(dtype, "out")
        out, op, os = c.out(out, (m, d), dtype, "out", table, ids)
        N.check(N.lib().taurus_lookup_rows(tp, code, n, d, ts, ip, m, scale, op, out_code, os, c.ptr),
                "taurus_lookup_rows")
        return out


def lookup_rows_grad(grad: torch.Tensor, ids: torch.Tensor, n: int, scale: float = 1.0, *,
                     out: Optional[torch.Tensor] = None, out_dtype=None, accumulate: bool = False,
                     stream=None) -> torch.Tensor:
    """taurus_lookup_rows_grad: gradient [n][d] of the table of lookup_rows
    from grad [m][d] (out_dtype: default out's or float32).  accumulate: add
    to the rows of out that ids names instead of writing every row."""
    if accumulate and out is None:
        raise ValueError("accumulate adds to out, which must be given")
    with _Call(grad, stream, "grad") as c:
        gp, gs = c.rows(grad, None, "grad")
        m, d = grad.shape
        ip = c.dense(ids, (m,), torch.int32, "ids")
        dtype = out_dtype or (out.dtype if out is not None else torch.float32)
        code, out_code = _code(grad.dtype, "grad"), _code(dtype, "out")
        out, op, os = c.out(out, (n, d), dtype, "out", grad, ids)
        L = N.lib()
        nbytes = L.taurus_lookup_rows_grad_bytes(m, d)
        work, wp = c.work(nbytes, "taurus_lookup_rows_grad_bytes")
        N.check(L.taurus_lookup_rows_grad(gp, code, gs, ip, m, n, d, scale, int(accumulate), op, out_code, os, wp,
                                          nbytes, c.ptr), "taurus_lookup_rows_grad")
        return out


# ---------------------------------------------------------- grouped linear --

def grouped_linear(x: torch.Tensor, off: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, *,
                   out: Optional[torch.Tensor] = None, out_dtype=None, stream=None) -> torch.Tensor:
    """taurus_grouped_linear: rows off[g] <= r < off[g + 1] of x [m][d_in]
    times weight[g] (weight [groups][d_in][d_out], x's type) plus bias[g]
    (float32 [groups][d_out]).  Rows no type holds are left as they were (in
    a new out: unspecified)."""
    with _Call(x, stream, "x") as c:
        xp, xs = c.rows(x, None, "x")
        m, d_in = x.shape
        fp, groups = c.offsets(off)
        if weight.dim() != 3:
            raise ValueError(f"weight must have shape [types][d_in][d_out], got {tuple(weight.shape)}")
        d_out = weight.shape[2]
        code = _code(x.dtype, "x")
        wp = c.dense(weight, (groups, d_in, d_out), x.dtype, "weight")
        bp = c.dense(bias, (groups, d_out), torch.float32, "bias")
        dtype = out_dtype or (out.dtype if out is not None else x.dtype)
        out_code = _code(dtype, "out")
        out, op, os = c.out(out, (m, d_out), dtype, "out", x, off, weight, bias)
        N.check(N.lib().taurus_grouped_linear(xp, code, m, d_in, xs, fp, groups, wp, d_out, bp, op, out_code, os,
                                              c.ptr), "taurus_grouped_linear")
        return out


def grouped_linear_grad(grad: torch.Tensor, x: torch.Tensor, off: torch.Tensor, weight: torch.Tensor, *,
                        need=("x", "weight", "bias"), weight_dtype=torch.float32, stream=None):
    """taurus_grouped_linear_grad: (dx of x's type, dweight of weight_dtype,
    dbias float32) from grad [m][d_out], x's type; None in the place of those
    that `need` does not name.  Rows of dx no type holds are unspecified."""
    for name in need:
        if name not in ("x", "weight", "bias"):
            raise ValueError(f"need names x, weight and bias, got {name!r}")
    with _Call(x, stream, "x") as c:
        xp, xs = c.rows(x, None, "x")
        m, d_in = x.shape
        fp, groups = c.offsets(off)
        if weight.dim() != 3:
            raise ValueError(f"weight must have shape [types][d_in][d_out], got {tuple(weight.shape)}")
        d_out = weight.shape[2]
        code = _code(x.dtype, "x")
        gp, gs = c.rows(grad, (m, d_out), "grad", x.dtype)
        wp = c.dense(weight, (groups, d_in, d_out), x.dtype, "weight")
        dx = torch.empty((m, d_in), dtype=x.dtype, device=c.device) if "x" in need else None
        dw = db = None
        w_code = _code(weight_dtype, "dweight")
        if "weight" in need:
            dw = torch.empty((groups, d_in, d_out), dtype=weight_dtype, device=c.device)
        if "bias" in need:
            db = torch.empty((groups, d_out), dtype=torch.float32, device=c.device)
        L = N.lib()
        work, kp, nbytes = None, None, 0
        if dw is not None or db is not None:
            nbytes = L.taurus_grouped_linear_grad_bytes(code, m, groups, d_in, d_out)
            work, kp = c.work(nbytes, "taurus_grouped_linear_grad_bytes")
        N.check(L.taurus_grouped_linear_grad(
            gp, gs, xp, xs, code, m, d_in, d_out, fp, groups, wp, None if dx is None else dx.data_ptr(), d_in,
            None if dw is None else dw.data_ptr(), w_code, None if db is None else db.data_ptr(), kp, nbytes, c.ptr),
            "taurus_grouped_linear_grad")
        return dx, dw, db


# -------------------------------------------------------------- group norm --

def _act(act) -> int:
    if act not in _ACT:
        raise ValueError(f"act must be one of {', '.join(_ACT)}, got {act!r}")
    return _ACT[act]


def group_norm(x: torch.Tensor, groups: int = 1, weight: Optional[torch.Tensor] = None,
               bias: Optional[torch.Tensor] = None, *, off: Optional[torch.Tensor] = None, eps: float = 1e-5,
               act: str = "none", out: Optional[torch.Tensor] = None, out_dtype=None, stats: bool = False, stream=None):
    """taurus_group_norm: act((x - mean) * rstd * weight + bias) over groups
    of consecutive channels of x [m][d], row by row, or over the rows of each
    segment off[s] <= r < off[s + 1].  weight, bias: float32 [d] or None.
    stats: return (out, mean, rstd), both float32 [rows or segments][groups],
    for group_norm_grad.  Rows no segment holds are left as they were (in a
    new out: unspecified)."""
    with _Call(x, stream, "x") as c:
        xp, xs = c.rows(x, None, "x")
        m, d = x.shape
        fp, segs = (None, 0) if off is None else c.offsets(off)
        wp = c.dense(weight, (d,), torch.float32, "weight")
        bp = c.dense(bias, (d,), torch.float32, "bias")
        dtype = out_dtype or (out.dtype if out is not None else x.dtype)
        code, out_code, act_code = _code(x.dtype, "x"), _code(dtype, "out"), _act(act)
        out, op, os = c.out(out, (m, d), dtype, "out", x, off, weight, bias)
        mean = rstd = None
        if stats:
            mean = torch.empty((m if off is None else segs, groups), dtype=torch.float32, device=c.device)
            rstd = torch.empty_like(mean)
        L = N.lib()
        nbytes, work, kp = 0, None, None
        if off is not None:  # row by row needs no workspace
            nbytes = L.taurus_group_norm_bytes(code, m, d, groups, segs, 1, 0)
            work, kp = c.work(nbytes, "taurus_group_norm_bytes")
        N.check(L.taurus_group_norm(xp, code, m, d, xs, groups, fp, segs, wp, bp, eps, act_code, op, out_code, os,
                                    None if mean is None else mean.data_ptr(),
                                    None if rstd is None else rstd.data_ptr(), kp, nbytes, c.ptr), "taurus_group_norm")
        return (out, mean, rstd) if stats else out


def group_norm_grad(grad: torch.Tensor, x: torch.Tensor, groups: int, weight: Optional[torch.Tensor],
                    bias: Optional[torch.Tensor], mean: torch.Tensor, rstd: torch.Tensor, *,
                    off: Optional[torch.Tensor] = None, act: str = "none", need=("x", "weight", "bias"), stream=None):
    """taurus_group_norm_grad: (dx of x's type, dweight, dbias float32 [d])
    from grad [m][d], x's type, and the mean and rstd that group_norm gave;
    None in the place of those that `need` does not name.  Rows of dx no
    segment holds are unspecified."""
    for name in need:
        if name not in ("x", "weight", "bias"):
            raise ValueError(f"need names x, weight and bias, got {name!r}")
    with _Call(x, stream, "x") as c:
        xp, xs = c.rows(x, None, "x")
        m, d = x.shape
        fp, segs = (None, 0) if off is None else c.offsets(off)
        code, act_code = _code(x.dtype, "x"), _act(act)
        gp, gs = c.rows(grad, (m, d), "grad", x.dtype)
        wp = c.dense(weight, (d,), torch.float32, "weight")
        bp = c.dense(bias, (d,), torch.float32, "bias")
        stat_shape = (m if off is None else segs, groups)
        mp = c.dense(mean, stat_shape, torch.float32, "mean")
        rp = c.dense(rstd, stat_shape, torch.float32, "rstd")
        dx = torch.empty((m, d), dtype=x.dtype, device=c.device) if "x" in need else None
        dw = torch.empty(d, dtype=torch.float32, device=c.device) if "weight" in need else None
        db = torch.empty(d, dtype=torch.float32, device=c.device) if "bias" in need else None
        L = N.lib()
        nbytes = L.taurus_group_norm_bytes(code, m, d, groups, segs, int(off is not None), 1)
        work, kp = c.work(nbytes, "taurus_group_norm_bytes")
        N.check(L.taurus_group_norm_grad(
            gp, gs, xp, xs, code, m, d, groups, fp, segs, wp, bp, mp, rp, act_code,
            None if dx is None else dx.data_ptr(), d, None if dw is None else dw.data_ptr(),
            None if db is None else db.data_ptr(), kp, nbytes, c.ptr), "taurus_group_norm_grad")
        return dx, dw, db
