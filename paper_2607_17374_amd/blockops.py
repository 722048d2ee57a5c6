"""Torch-facing wrapper of the C ABI's operators that make residual blocks and
a classifier out of layers: linear maps with an activation and a residual,
norms around a gated residual sum, log probabilities of labels, and the
gradients of each.

As in ``rowops``, each function turns tensors into pointers and makes one call
of the library; outputs and workspaces are torch's, taken on the stream the
call runs on.  Names follow the C ABI (``linear`` = taurus_linear, ...).
"""
from __future__ import annotations

import functools
from typing import NamedTuple, Optional

import torch

from . import _native as N
from .rowops import _Call, _code

_ACT = {"none": N.ACT_NONE, "relu": N.ACT_RELU, "silu": N.ACT_SILU, "gelu": N.ACT_GELU,
        "gelu_tanh": N.ACT_GELU_TANH}
_NORM = {"layer": N.NORM_LAYER, "rms": N.NORM_RMS}


def check_act(act) -> None:
    if act not in _ACT:
        raise ValueError(f"act must be one of {', '.join(_ACT)}, got {act!r}")


def _act(act) -> int:
    check_act(act)
    return _ACT[act]


@functools.lru_cache(maxsize=4096)
def _bytes(call: str, *sizes) -> int:
    """A call's workspace: follows from the sizes alone (refused ones are not
    remembered)."""
    nbytes = getattr(N.lib(), call)(*sizes)
    if nbytes < 0:
        raise N.TaurusError(int(nbytes), call, N.last_error())
    return nbytes


def _needed(need, names) -> None:
    for name in need:
        if name not in names:
            raise ValueError(f"need names {', '.join(names)}, got {name!r}")


# ------------------------------------------------------------------ linear --

def linear(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None,
           residual: Optional[torch.Tensor] = None, *, act: str = "none", out: Optional[torch.Tensor] = None,
           out_dtype=None, pre: bool = False, stream=None):
    """taurus_linear: act(x weight + bias) + residual.  x [m][d_in], weight
    [d_in][d_out] of x's type, bias float32 [d_out], residual [m][d_out] of
    out's type; act: none, relu, silu, gelu or gelu_tanh.  pre: return (out, z)
    with z = x weight + bias in x's type, for linear_grad."""
    with _Call(x, stream, "x") as c:
        xp, xs = c.rows(x, None, "x")
        m, d_in = x.shape
        if weight.dim() != 2:
            raise ValueError(f"weight must have shape [d_in][d_out], got {tuple(weight.shape)}")
        d_out = weight.shape[1]
        code, act_code = _code(x.dtype, "x"), _act(act)
        wp = c.dense(weight, (d_in, d_out), x.dtype, "weight")
        bp = c.dense(bias, (d_out,), torch.float32, "bias")
        dtype = out_dtype or (out.dtype if out is not None else x.dtype)
        out_code = _code(dtype, "out")
        rp, rs = (None, d_out) if residual is None else c.rows(residual, (m, d_out), "residual", dtype)
        out, op, os = c.out(out, (m, d_out), dtype, "out", x, weight, bias, residual)
        z = torch.empty((m, d_out), dtype=x.dtype, device=c.device) if pre else None
        L = N.lib()
        nbytes = _bytes("taurus_linear_bytes", code, m, d_in, d_out)
        work, kp = c.work(nbytes, "taurus_linear_bytes")
        N.check(L.taurus_linear(xp, code, m, d_in, xs, wp, d_out, bp, rp, rs, act_code, op, out_code, os,
                                None if z is None else z.data_ptr(), d_out, kp, nbytes, c.ptr), "taurus_linear")
        return (out, z) if pre else out


def linear_grad(grad: torch.Tensor, x: torch.Tensor, weight: torch.Tensor, pre: Optional[torch.Tensor] = None, *,
                act: str = "none", need=("x", "weight", "bias"), weight_dtype=torch.float32, stream=None):
    """taurus_linear_grad: (dx of x's type, dweight of weight_dtype, dbias
    float32) from grad [m][d_out], x's type, and the z that linear gave (pre;
    not needed without an activation); None in the place of those that `need`
    does not name.  The residual's gradient is grad.  Behind an activation,
    grad act'(z) of 16-bit arrays is rounded to their type before dx and dweight
    are formed; fp32 arrays avoid that."""
    _needed(need, ("x", "weight", "bias"))
    with _Call(x, stream, "x") as c:
        xp, xs = c.rows(x, None, "x")
        m, d_in = x.shape
        if weight.dim() != 2:
            raise ValueError(f"weight must have shape [d_in][d_out], got {tuple(weight.shape)}")
        d_out = weight.shape[1]
        code, act_code = _code(x.dtype, "x"), _act(act)
        gp, gs = c.rows(grad, (m, d_out), "grad", x.dtype)
        wp = c.dense(weight, (d_in, d_out), x.dtype, "weight")
        if pre is None and act != "none":
            raise ValueError("the gradient of an activation needs pre")
        zp, zs = (None, d_out) if pre is None else c.rows(pre, (m, d_out), "pre", x.dtype)
        dx = torch.empty((m, d_in), dtype=x.dtype, device=c.device) if "x" in need else None
        w_code = _code(weight_dtype, "dweight")
        dw = torch.empty((d_in, d_out), dtype=weight_dtype, device=c.device) if "weight" in need else None
        db = torch.empty(d_out, dtype=torch.float32, device=c.device) if "bias" in need else None
        L = N.lib()
        nbytes = _bytes("taurus_linear_grad_bytes", code, m, d_in, d_out, act_code)
        work, kp = c.work(nbytes, "taurus_linear_grad_bytes")
        N.check(L.taurus_linear_grad(gp, gs, xp, xs, code, m, d_in, d_out, wp, zp, zs, act_code,
                                     None if dx is None else dx.data_ptr(), d_in,
                                     None if dw is None else dw.data_ptr(), w_code,
                                     None if db is None else db.data_ptr(), kp, nbytes, c.ptr), "taurus_linear_grad")
        return dx, dw, db


# ----------------------------------------------------------- residual norm --

_NORM_KEYS = {"kind", "weight", "bias", "eps"}


def check_norm_args(norm: Optional[dict], what: str) -> None:
    if norm is None:
        return
    if not norm.keys() <= _NORM_KEYS:
        raise ValueError(f"{what} does not know {', '.join(sorted(norm.keys() - _NORM_KEYS))}")
    if norm.get("kind", "layer") not in _NORM:
        raise ValueError(f"{what}'s kind must be one of {', '.join(_NORM)}, got {norm['kind']!r}")


class _Norm:
    """A norm's arguments: dict of kind (layer or rms), weight, bias, eps."""
    __slots__ = ("kind", "weight", "bias", "wp", "bp", "eps")

    def __init__(self, c: _Call, norm: Optional[dict], d: int, what: str):
        self.kind, self.eps = N.NORM_NONE, 1e-5
        self.weight = self.bias = self.wp = self.bp = None
        if norm is None:
            return
        check_norm_args(norm, what)
        self.kind, self.eps = _NORM[norm.get("kind", "layer")], norm.get("eps", 1e-5)
        self.weight, self.bias = norm.get("weight"), norm.get("bias")
        if self.weight is not None:
            self.wp = c.dense(self.weight, (d,), torch.float32, f"{what}'s weight")
        if self.bias is not None:
            self.bp = c.dense(self.bias, (d,), torch.float32, f"{what}'s bias")


def _gate(c: _Call, gate: Optional[torch.Tensor], off: Optional[torch.Tensor], d: int):
    """(gate pointer, offsets pointer, segments, gate's shape)."""
    fp, segs = (None, 0) if off is None else c.offsets(off)
    shape = (d,) if off is None else (segs, d)
    return c.dense(gate, shape, torch.float32, "gate"), fp, segs, shape


def residual_norm(x: torch.Tensor, f: torch.Tensor, *, scale: float = 1.0, gate: Optional[torch.Tensor] = None,
                  off: Optional[torch.Tensor] = None, post: Optional[dict] = None, pre: Optional[dict] = None,
                  out: Optional[torch.Tensor] = None, out_h: Optional[torch.Tensor] = None, stats: bool = False,
                  stream=None):
    """taurus_residual_norm: y = x + scale * gate * post(f) and h = pre(y), row
    by row; returns (y, h), h None without pre.  f [m][d], x and y of f's type
    or float32, h of f's type.  post, pre: dicts of kind (layer, the default,
    or rms), weight, bias (float32 [d] or None) and eps (1e-5).  gate: float32
    [d], or with offsets [segments][d], one row for each segment off[s] <= r <
    off[s + 1].  stats: return (y, h, stats), float32 [m][4], for
    residual_norm_grad.  Rows no segment holds are left as they were (in new
    outputs: unspecified)."""
    with _Call(f, stream, "f") as c:
        fp, fs = c.rows(f, None, "f")
        m, d = f.shape
        xp, xs = c.rows(x, (m, d), "x")
        code, x_code = _code(f.dtype, "f"), _code(x.dtype, "x")
        gp, op, segs, _ = _gate(c, gate, off, d)
        a, b = _Norm(c, post, d, "post"), _Norm(c, pre, d, "pre")
        inputs = (x, f, gate, off, a.weight, a.bias, b.weight, b.bias)
        y, yp, ys = c.out(out, (m, d), x.dtype, "out", *inputs)
        h, hp, hs = None, None, d
        if pre is not None:
            h, hp, hs = c.out(out_h, (m, d), f.dtype, "out_h", *inputs, out)
        elif out_h is not None:
            raise ValueError("out_h is the norm's output, and there is no pre")
        st = torch.empty((m, 4), dtype=torch.float32, device=c.device) if stats else None
        N.check(N.lib().taurus_residual_norm(
            xp, x_code, xs, fp, code, fs, m, d, scale, gp, op, segs, a.kind, a.wp, a.bp, a.eps, b.kind, b.wp, b.bp,
            b.eps, yp, ys, hp, hs, None if st is None else st.data_ptr(), c.ptr), "taurus_residual_norm")
        return (y, h, st) if stats else (y, h)


class ResidualNormGrad(NamedTuple):
    """residual_norm_grad's outputs; None where there is nothing or it was not
    asked for."""
    x: Optional[torch.Tensor]            # of y's type
    f: Optional[torch.Tensor]            # of f's type
    gate: Optional[torch.Tensor]         # float32, gate's shape
    post_weight: Optional[torch.Tensor]  # float32 [d], as those below
    post_bias: Optional[torch.Tensor]
    pre_weight: Optional[torch.Tensor]
    pre_bias: Optional[torch.Tensor]


def residual_norm_grad(grad_y: Optional[torch.Tensor], grad_h: Optional[torch.Tensor], y: torch.Tensor,
                       f: torch.Tensor, stats: Optional[torch.Tensor], *, scale: float = 1.0,
                       gate: Optional[torch.Tensor] = None, off: Optional[torch.Tensor] = None,
                       post: Optional[dict] = None, pre: Optional[dict] = None,
                       need=("x", "f", "gate", "post", "pre"), stream=None) -> ResidualNormGrad:
    """taurus_residual_norm_grad: the gradients of residual_norm's arguments
    (those that were given) from grad_y, y's type (None: y is used by h alone)
    and grad_h, f's type (None without pre), at the y and stats that
    residual_norm gave (stats None without norms).  Rows no segment holds are
    unspecified in x and f."""
    _needed(need, ("x", "f", "gate", "post", "pre"))
    with _Call(f, stream, "f") as c:
        fp, fs = c.rows(f, None, "f")
        m, d = f.shape
        yp, ys = c.rows(y, (m, d), "y")
        code, y_code = _code(f.dtype, "f"), _code(y.dtype, "y")
        gyp, gys = (None, d) if grad_y is None else c.rows(grad_y, (m, d), "grad_y", y.dtype)
        if (grad_h is None) != (pre is None):
            raise ValueError("grad_h is needed with pre, and only then")
        ghp, ghs = (None, d) if grad_h is None else c.rows(grad_h, (m, d), "grad_h", f.dtype)
        gp, op, segs, gate_shape = _gate(c, gate, off, d)
        a, b = _Norm(c, post, d, "post"), _Norm(c, pre, d, "pre")
        if stats is None and (post is not None or pre is not None):
            raise ValueError("the gradient of a norm needs stats")
        sp = c.dense(stats, (m, 4), torch.float32, "stats")

        def new(wanted, shape, dtype=torch.float32):
            return torch.empty(shape, dtype=dtype, device=c.device) if wanted else None

        g = ResidualNormGrad(new("x" in need, (m, d), y.dtype), new("f" in need, (m, d), f.dtype),
                             new("gate" in need and gate is not None, gate_shape),
                             new("post" in need and a.weight is not None, d),
                             new("post" in need and a.bias is not None, d),
                             new("pre" in need and b.weight is not None, d),
                             new("pre" in need and b.bias is not None, d))
        p = [None if t is None else t.data_ptr() for t in g]
        L = N.lib()
        nbytes = _bytes("taurus_residual_norm_grad_bytes", code, m, d, segs, int(off is not None))
        work, kp = c.work(nbytes, "taurus_residual_norm_grad_bytes")
        N.check(L.taurus_residual_norm_grad(
            gyp, gys, ghp, ghs, yp, y_code, ys, fp, code, fs, m, d, scale, gp, op, segs, a.kind, a.wp, a.bp, b.kind,
            b.wp, sp, p[0], d, p[1], d, p[2], p[3], p[4], p[5], p[6], kp, nbytes, c.ptr), "taurus_residual_norm_grad")
        return g


# --------------------------------------------------------- label log probs --

class LabelLogProbs(NamedTuple):
    """label_log_probs' outputs; None where it was not asked for."""
    logp: Optional[torch.Tensor]      # float32 [m], of the labels
    stats: torch.Tensor               # float32 [m][2]: largest scaled logit, log of the sum above it
    entropy: Optional[torch.Tensor]   # float32 [m]
    top_logp: Optional[torch.Tensor]  # float32 [m][top], largest first
    top_ids: Optional[torch.Tensor]   # int32 [m][top]


def label_log_probs(x: torch.Tensor, labels: Optional[torch.Tensor] = None, scale: float = 1.0, *, top: int = 0,
                    entropy: bool = False, stream=None) -> LabelLogProbs:
    """taurus_label_log_probs: log probabilities of labels (int32 [m]; outside
    the classes: 0) under the softmax of scale * x, rows of logits [m][c],
    its entropy, and its `top` likeliest classes.  Masked classes have logits
    of -inf.  The two values of stats add up to the log of the sum of
    exponentials."""
    with _Call(x, stream, "x") as c:
        xp, xs = c.rows(x, None, "x")
        m, classes = x.shape
        code = _code(x.dtype, "x")
        lp = c.dense(labels, (m,), torch.int32, "labels")

        def new(wanted, shape, dtype=torch.float32):
            return torch.empty(shape, dtype=dtype, device=c.device) if wanted else None

        L = N.lib()
        nbytes = _bytes("taurus_label_log_probs_bytes", code, m, classes, top)
        work, kp = c.work(nbytes, "taurus_label_log_probs_bytes")
        r = LabelLogProbs(new(labels is not None, m), new(True, (m, 2)), new(entropy, m), new(top > 0, (m, top)),
                          new(top > 0, (m, top), torch.int32))
        p = [None if t is None else t.data_ptr() for t in r]
        N.check(L.taurus_label_log_probs(xp, code, m, classes, xs, lp, scale, top, *p, kp, nbytes, c.ptr),
                "taurus_label_log_probs")
        return r


def label_log_probs_grad(x: torch.Tensor, labels: Optional[torch.Tensor], stats: torch.Tensor,
                         grad_logp: Optional[torch.Tensor], scale: float = 1.0, *,
                         entropy: Optional[torch.Tensor] = None, grad_entropy: Optional[torch.Tensor] = None,
                         out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """taurus_label_log_probs_grad: gradient [m][c], x's type, of the logits
    from grad_logp (with labels; float32 [m]) and grad_entropy (with the
    entropy; float32 [m]), at the stats and entropy that label_log_probs
    gave."""
    if (labels is None) != (grad_logp is None):
        raise ValueError("labels and grad_logp go together")
    if (entropy is None) != (grad_entropy is None):
        raise ValueError("entropy and grad_entropy go together")
    with _Call(x, stream, "x") as c:
        xp, xs = c.rows(x, None, "x")
        m, classes = x.shape
        code = _code(x.dtype, "x")
        lp = c.dense(labels, (m,), torch.int32, "labels")
        sp = c.dense(stats, (m, 2), torch.float32, "stats")
        ep = c.dense(entropy, (m,), torch.float32, "entropy")
        gp = c.dense(grad_logp, (m,), torch.float32, "grad_logp")
        gep = c.dense(grad_entropy, (m,), torch.float32, "grad_entropy")
        out, op, os = c.out(out, (m, classes), x.dtype, "out", x, labels, stats, entropy, grad_logp, grad_entropy)
        N.check(N.lib().taurus_label_log_probs_grad(xp, code, m, classes, xs, lp, scale, sp, ep, gp, gep, op, os,
                                                    c.ptr), "taurus_label_log_probs_grad")
        return out
