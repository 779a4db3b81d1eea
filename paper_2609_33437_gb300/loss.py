"""The loss behind a language model's last layer: softmax cross entropy of the logits x W^T over a vocabulary, without keeping
the logits, and its gradient, which makes them again a piece of the vocabulary at a time (include/smat.h, "loss over a
vocabulary").

    loss, lse = token_loss(x, w, targets)                     one loss a row, 0 where the target is `ignore`
    dx, dw    = token_loss_grad(g, x, w, targets, lse)        g: the gradient that reaches the losses
    cross_entropy(x, w, targets)                              the differentiable form, reduced

Tensors are CUDA tensors of one dtype per call (float32 or bfloat16); x may have any number of leading dimensions and a row
stride. Argument marshalling only; the operators build no autograd graph and refuse tensors whose gradient or tangent that would
lose, as those of `linear`. `linear.poll_errors` tells of these products too.
"""

import struct
from typing import Optional

import torch

from . import linear as L
from . import smat as S

_TOKEN_LOSS = struct.Struct("@5P6q2i")
_TOKEN_LOSS_GRAD = struct.Struct("@7P8q2i")


def _targets(targets: torch.Tensor, shape, device) -> int:
    if targets.dtype is not torch.int64 or targets.device != device or targets.shape != shape or not targets.is_contiguous():
        raise ValueError(f"targets: must be contiguous torch.int64 of shape {tuple(shape)} on {device}")
    return targets.data_ptr()


def _row_values(name: str, t: torch.Tensor, shape, device) -> int:
    if t.dtype is not torch.float32 or t.device != device or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous torch.float32 of shape {tuple(shape)} on {device}")
    return t.data_ptr()


def token_loss(x: torch.Tensor, w: torch.Tensor, targets: torch.Tensor, ignore: int = -100,
               stream: Optional[torch.cuda.Stream] = None):
    """(loss, lse), float32 of x's leading dimensions: lse = log sum exp of the logits x W^T, loss = lse - logit[target], 0
    where the target is `ignore`, NaN where it is no row of w. x [..., k], w [n, k], targets int64 [...]."""
    if stream is not None:
        return L._on(stream, token_loss, x, w, targets, ignore)
    L._no_graph(x, w)
    rows, k, ldx = L._rows("x", x)
    code = S.dtype_code(x.dtype)
    device, shape = x.device, x.shape[:-1]
    if w.dim() != 2:
        raise ValueError("w: must be a matrix")
    n = w.shape[0]
    pw, ldw = L._like("w", w, x.dtype, device, n, k)
    pt = _targets(targets, shape, device)
    loss, lse = torch.empty(shape, dtype=torch.float32, device=device), torch.empty(shape, dtype=torch.float32, device=device)
    args = _TOKEN_LOSS.pack(x.data_ptr(), pw, pt, loss.data_ptr(), lse.data_ptr(), rows, k, n, ldx, ldw, ignore, code, 0)
    L._run("smat_token_loss", args, device)
    return loss, lse


def token_loss_grad(g: torch.Tensor, x: torch.Tensor, w: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor,
                    ignore: int = -100, out: Optional[torch.Tensor] = None, weight_out: Optional[torch.Tensor] = None,
                    accumulate: bool = False, need_x: bool = True, need_w: bool = True,
                    stream: Optional[torch.cuda.Stream] = None):
    """(dx, dW) of token_loss, for the losses' gradients g and its lse; None for need_x or need_w False. With accumulate, dW is
    added to `weight_out`. Rows whose target is `ignore` are left out, and their dx is 0."""
    if stream is not None:
        return L._on(stream, token_loss_grad, g, x, w, targets, lse, ignore, out, weight_out, accumulate, need_x, need_w)
    L._no_graph(x, w, g)
    if (out is not None and not need_x) or (weight_out is not None and not need_w):
        raise ValueError("an output is given for a gradient that is not asked for")
    if accumulate and weight_out is None:
        raise ValueError("accumulate: needs weight_out")
    rows, k, ldx = L._rows("x", x)
    code = S.dtype_code(x.dtype)
    dtype, device, shape = x.dtype, x.device, x.shape[:-1]
    if w.dim() != 2:
        raise ValueError("w: must be a matrix")
    n = w.shape[0]
    pw, ldw = L._like("w", w, dtype, device, n, k)
    pt, pg, pl = _targets(targets, shape, device), _row_values("g", g, shape, device), _row_values("lse", lse, shape, device)
    dx, px, lddx = None, 0, k
    if need_x:
        dx = out
        if dx is None:
            dx = torch.empty(x.shape, dtype=dtype, device=device)
            px = dx.data_ptr()
        else:
            px, lddx = L._like("out", dx, dtype, device, rows, k)
    dw, pdw, lddw = None, 0, k
    if need_w:
        dw = weight_out
        if dw is None:
            dw = torch.empty((n, k), dtype=dtype, device=device)
            pdw = dw.data_ptr()
        else:
            pdw, lddw = L._like("weight_out", dw, dtype, device, n, k)
    args = _TOKEN_LOSS_GRAD.pack(pg, x.data_ptr(), pw, pt, pl, px, pdw, rows, k, n, ldx, ldw, lddx, lddw, ignore, code,
                                 1 if accumulate else 0)
    L._run("smat_token_loss_grad", args, device)
    return dx, dw


class _TokenLoss(torch.autograd.Function):
    """(loss, anchor): `anchor` as in linear._Linear8."""

    @staticmethod
    def forward(ctx, x, w, targets, ignore):
        ctx.ignore = ignore
        ctx.set_materialize_grads(False)
        x, w = L._rows_like(x), L._rows_like(w)
        loss, lse = token_loss(x, w, targets, ignore)
        anchor = x.new_empty(0)
        ctx.save_for_backward(x, w, targets, lse, anchor)
        return loss, anchor

    @staticmethod
    def backward(ctx, g, _):
        if g is None:
            return None, None, None, None
        return L._first_only(ctx, g, _TokenLoss._gradients)

    @staticmethod
    def _gradients(ctx, g):
        x, w, targets, lse, _ = ctx.saved_tensors
        need_x, need_w = ctx.needs_input_grad[:2]
        dx, dw = token_loss_grad(g.contiguous(), x, w, targets, lse, ctx.ignore, need_x=need_x, need_w=need_w)
        return dx, dw, None, None


def cross_entropy(x: torch.Tensor, w: torch.Tensor, targets: torch.Tensor, ignore: int = -100,
                  reduction: str = "mean") -> torch.Tensor:
    """torch.nn.functional.cross_entropy of the logits x W^T, which are not kept, in fp32: reduction "mean" (over the targets
    that are not `ignore`), "sum" or "none". First derivatives only, of x and w. Under torch.autocast x and w are cast as for
    torch.nn.functional.linear."""
    if reduction not in ("mean", "sum", "none"):
        raise ValueError(f"reduction: {reduction!r} is none of mean, sum, none")
    if torch.is_autocast_enabled("cuda"):
        dtype = torch.get_autocast_dtype("cuda")
        x, w = x.to(dtype), w.to(dtype)
    targets = targets.contiguous()
    if torch.is_grad_enabled():
        loss, _ = _TokenLoss.apply(x, w, targets, ignore)
    else:
        loss, _ = token_loss(L._rows_like(x), L._rows_like(w), targets, ignore)
    if reduction == "none":
        return loss
    return loss.sum() if reduction == "sum" else loss.sum() / (targets != ignore).sum()
