"""Layer norm and rms norm, with the residual stream's sum before them in the same pass (include/smat.h, "norms").

    y, h, stats = norm(x, w, b, residual=r, save=True)     h = x + r, y = (h - mu) s w + b, stats: the rows' mu and s
    dx, dw, db  = norm_grad(dy, h, stats, w, dh=dh)        dh: the gradient that reaches h otherwise

`Norm` is the layer: torch.nn.LayerNorm or torch.nn.RMSNorm over the last dimension, with a residual. Its backward pass
reads h and eight bytes a row.

Tensors are CUDA tensors of one dtype per call (float32 or bfloat16) with any number of leading dimensions and a row stride;
w and b are vectors of the same dtype, or of float32 beside bfloat16. Argument marshalling only; the operators build no
autograd graph and refuse tensors whose gradient or tangent that would lose, as those of `linear`.
"""

import struct
from typing import Optional

import torch

from . import linear as L
from . import smat as S

KINDS = {"layer": 0, "rms": 1}

_NORM = struct.Struct("@7P6q3if")
_NORM_GRAD = struct.Struct("@8P6q4i")


def _kind(kind: str) -> int:
    k = KINDS.get(kind)
    if k is None:
        raise ValueError(f"kind: {kind!r} is none of {', '.join(KINDS)}")
    return k


def _weights(cols: int, dtype, device, w: Optional[torch.Tensor], b: Optional[torch.Tensor]):
    """(address of w, of b, their dtype code); 0 for one that is not there."""
    t = w if w is not None else b
    if t is None:
        return 0, 0, S.dtype_code(dtype)
    wt = t.dtype
    if wt is not dtype and wt is not torch.float32:
        raise ValueError(f"{'w' if t is w else 'b'}: must be {dtype} or torch.float32")
    pw = L._vector("w", w, wt, device, cols) if w is not None else 0
    pb = L._vector("b", b, wt, device, cols) if b is not None else 0
    return pw, pb, S.dtype_code(wt)


def _place(name: str, t: Optional[torch.Tensor], like: torch.Tensor, rows: int, cols: int):
    """(t or a new tensor of like's shape, address, row stride)"""
    if t is None:  # (the first takes 0.3 us less)
        t = torch.empty_like(like) if like.is_contiguous() else torch.empty(like.shape, dtype=like.dtype, device=like.device)
        return t, t.data_ptr(), cols
    return (t, *L._like(name, t, like.dtype, like.device, rows, cols))


def norm(x: torch.Tensor, w: Optional[torch.Tensor] = None, b: Optional[torch.Tensor] = None,
         residual: Optional[torch.Tensor] = None, kind: str = "layer", eps: float = 1e-5, save: bool = False,
         out: Optional[torch.Tensor] = None, sum_out: Optional[torch.Tensor] = None,
         stream: Optional[torch.cuda.Stream] = None):
    """y, or a tuple of y, with a residual h = x + residual, and with save the statistics that norm_grad reads.

    x, residual, out (for y) and sum_out (for h) [..., cols]; sum_out may be the residual. w, b [cols] or None. The
    statistics are [2, rows] in float32, mu and s of every row ([1, rows], s, with kind "rms")."""
    if stream is not None:
        return L._on(stream, norm, x, w, b, residual, kind, eps, save, out, sum_out)
    L._no_graph(x, w, b, residual)
    k = _kind(kind)
    if sum_out is not None and residual is None:
        raise ValueError("sum_out: without a residual")
    rows, cols, ldx = L._rows("x", x)
    code = S.dtype_code(x.dtype)
    dtype, device = x.dtype, x.device
    pw, pb, wcode = _weights(cols, dtype, device, w, b)
    pr = ph = 0
    ldr = ldh = cols
    h = None
    if residual is not None:
        pr, ldr = L._like("residual", residual, dtype, device, rows, cols)
        h, ph, ldh = _place("sum_out", sum_out, x, rows, cols)
    y, py, ldy = _place("out", out, x, rows, cols)
    stats, ps = None, 0
    if save:
        stats = torch.empty((1 if k else 2, rows), dtype=torch.float32, device=device)
        ps = stats.data_ptr()
    args = _NORM.pack(x.data_ptr(), pr, pw, pb, ph, py, ps, rows, cols, ldx, ldr, ldh, ldy, code, wcode, k, eps)
    L._call("smat_norm", device, args)
    if h is None:
        return (y, stats) if save else y
    return (y, h, stats) if save else (y, h)


def norm_grad(dy: torch.Tensor, h: torch.Tensor, stats: torch.Tensor, w: Optional[torch.Tensor] = None,
              bias: bool = False, kind: str = "layer", dh: Optional[torch.Tensor] = None,
              out: Optional[torch.Tensor] = None, weight_out: Optional[torch.Tensor] = None,
              bias_out: Optional[torch.Tensor] = None, accumulate: bool = False, need_x: bool = True,
              need_w: bool = True, stream: Optional[torch.cuda.Stream] = None):
    """(dx, dw, db) of norm: h is what it normalised (x, or the sum it returned), stats what it saved, dh the gradient that
    reaches h otherwise and is added to dx. dx is the gradient of x and of the residual alike; None for need_x, need_w or bias
    False. dw and db have the type of w (that of weight_out or bias_out, or of h, where there is no w). out may be dh. With
    accumulate, dw and db are added to weight_out and bias_out, which then are needed."""
    if stream is not None:
        return L._on(stream, norm_grad, dy, h, stats, w, bias, kind, dh, out, weight_out, bias_out, accumulate, need_x, need_w)
    L._no_graph(dy, h, w, dh)
    k = _kind(kind)
    if (weight_out is not None and not need_w) or (bias_out is not None and not bias) or (out is not None and not need_x):
        raise ValueError("an output is given for a gradient that is not asked for")
    if accumulate and ((need_w and weight_out is None) or (bias and bias_out is None)):
        raise ValueError("accumulate: needs weight_out and bias_out")
    rows, cols, lddy = L._rows("dy", dy)
    code = S.dtype_code(dy.dtype)
    dtype, device = dy.dtype, dy.device
    ph, ldh = L._like("h", h, dtype, device, rows, cols)
    if tuple(stats.shape) != (1 if k else 2, rows):
        raise ValueError(f"stats: must be {1 if k else 2} x {rows}, as norm saved them")
    if stats.dtype is not torch.float32 or stats.device != device or not stats.is_contiguous():
        raise ValueError(f"stats: must be contiguous torch.float32 on {device}")
    like = next((t for t in (w, weight_out, bias_out) if t is not None), None)
    wt = like.dtype if like is not None else dtype
    pw, _, wcode = _weights(cols, dtype, device, w if w is not None else like, None)
    pdh, lddh = L._like("dh", dh, dtype, device, rows, cols) if dh is not None else (0, cols)
    dx, px, lddx = _place("out", out, dy, rows, cols) if need_x else (None, 0, cols)
    dw = db = None
    pdw = pdb = 0
    if need_w:
        dw = weight_out if weight_out is not None else torch.empty(cols, dtype=wt, device=device)
        pdw = L._vector("weight_out", dw, wt, device, cols)
    if bias:
        db = bias_out if bias_out is not None else torch.empty(cols, dtype=wt, device=device)
        pdb = L._vector("bias_out", db, wt, device, cols)
    args = _NORM_GRAD.pack(dy.data_ptr(), ph, stats.data_ptr(), pw if w is not None else 0, pdh, px, pdw, pdb, rows, cols, lddy,
                           ldh, lddh, lddx, code, wcode, k, 1 if accumulate else 0)
    L._run("smat_norm_grad", args, device)
    return dx, dw, db


# -------------------------------------------------------------------- layer ---
class _Norm(torch.autograd.Function):
    """(y, h, anchor): h is x without a residual, and not returned then; `anchor` as in linear._Linear8."""

    @staticmethod
    def forward(ctx, x, w, b, residual, kind, eps):
        ctx.kind, ctx.bias = kind, b is not None
        ctx.set_materialize_grads(False)
        x, residual = L._rows_like(x), L._rows_like(residual)
        need = any(ctx.needs_input_grad[:4])
        got = norm(x, w, b, residual, kind, eps, save=need)
        got = got if isinstance(got, tuple) else (got,)
        h = got[1] if residual is not None else x
        anchor = x.new_empty(0)
        ctx.save_for_backward(h, got[-1] if need else None, w, anchor)
        return got[0], h if residual is not None else None, anchor

    @staticmethod
    def backward(ctx, dy, dh, _):
        if dy is None and dh is None:
            return (None,) * 6
        return L._first_only(ctx, dy if dy is not None else dh, lambda ctx, _: _Norm._gradients(ctx, dy, dh))

    @staticmethod
    def _gradients(ctx, dy, dh):
        h, stats, w, _ = ctx.saved_tensors
        need_x, need_w, need_b, need_r = ctx.needs_input_grad[:4]
        if dy is None:  # y led nowhere: the sum's gradient alone
            zero = None if w is None else torch.zeros_like(w)
            return (dh if need_x else None, zero if need_w else None, torch.zeros_like(zero) if need_b else None,
                    dh if need_r else None, None, None)
        dy, dh = L._rows_like(dy), L._rows_like(dh)
        need_x = need_x or need_r
        dx, dw, db = norm_grad(dy, h, stats, w, bias=need_b, kind=ctx.kind, dh=dh if need_x else None, need_x=need_x, need_w=need_w)
        return dx if ctx.needs_input_grad[0] else None, dw, db, dx if need_r else None, None, None


class Norm(torch.nn.Module):
    """Layer norm (kind "layer", as torch.nn.LayerNorm) or rms norm ("rms", as torch.nn.RMSNorm) over the last dimension.
    norm(x) is y; norm(x, residual) is (y, h) with h = x + residual, the residual stream that goes on. First derivatives only:
    one taken of its gradients raises RuntimeError. Inputs may have any strides. Under torch.autocast it runs in its input's
    type, with fp32 weights beside bf16 inputs as they are."""

    def __init__(self, features: int, kind: str = "layer", eps: float = 1e-5, bias: bool = True, device=None, dtype=None):
        super().__init__()
        _kind(kind)
        self.kind, self.eps = kind, float(eps)
        self.weight = torch.nn.Parameter(torch.ones(features, device=device, dtype=dtype))
        self.bias = torch.nn.Parameter(torch.zeros(features, device=device, dtype=dtype)) if bias and kind == "layer" else None

    def extra_repr(self) -> str:
        return f"{self.weight.shape[0]}, kind={self.kind!r}, eps={self.eps}, bias={self.bias is not None}"

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None):
        if not torch.is_grad_enabled():
            return norm(L._rows_like(x), self.weight, self.bias, L._rows_like(residual), self.kind, self.eps)
        y, h, _ = _Norm.apply(x, self.weight, self.bias, residual, self.kind, self.eps)
        return y if residual is None else (y, h)
