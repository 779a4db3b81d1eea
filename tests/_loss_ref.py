"""The loss over a vocabulary from its definition in 64 bits (torch float64 on the GPU: sizes that a CPU would take long for),
and how far what the kernels make may be off."""

import math

import torch

import _linear_ref as R

U = 2.0 ** -24


def forward(x, w, targets, ignore):
    """logits, lse, loss and the bounds of lse and loss."""
    xd, wd = x.double(), w.double()
    l = xd @ wd.T
    mag = xd.abs() @ wd.abs().T
    err = R.sum_error(mag, x.dtype, x.shape[-1])  # of every logit
    lse = torch.logsumexp(l, 1)
    p = torch.exp(l - lse[:, None])
    # lse moves by the logits' errors weighted with p. An exponential: its argument is rounded (the logit's, the largest one's and
    # their difference's size in units of log2(e)) and it is off by 2 to 4 units; a sum of n positive terms, some of them in
    # turn, loses 8 sqrt(n) u at most with near certainty, see _linear_ref.sum_error; joins of parts and the logarithm as much again
    n = l.shape[1]
    top = l.amax(1)
    size = (p * (l.abs() + top.abs()[:, None] + (l - top[:, None]).abs())).sum(1)
    e_lse = (p * err).sum(1) + U * (3 * size + 8 * math.sqrt(n) + 40 + 4 * lse.abs())
    counts = targets != ignore
    at = torch.where(counts, targets, 0)[:, None]
    loss = torch.where(counts, lse - l.gather(1, at)[:, 0], 0.0)
    e_loss = torch.where(counts, e_lse + err.gather(1, at)[:, 0] + U * (loss.abs() + l.gather(1, at)[:, 0].abs()), 0.0)
    return l, err, lse, e_lse, loss, e_loss


def gradient(g, x, w, targets, lse, ignore):
    """dx, dw and their bounds, from the lse that is given (fp32)."""
    l, err, *_ = forward(x, w, targets, ignore)
    counts = targets != ignore
    p = torch.exp(l - lse.double()[:, None])
    hot = torch.zeros_like(p).scatter_(1, torch.where(counts, targets, 0)[:, None], 1.0)
    if x.dtype == torch.bfloat16:  # the target's own logit is made in fp32
        mag = (x.double().abs() * w.double()[torch.where(counts, targets, 0)].abs()).sum(1, keepdim=True)
        err = torch.where(hot > 0, R.sum_error(mag, torch.float32, x.shape[-1]), err)
    gd = torch.where(counts, g.double(), 0.0)[:, None]
    d = torch.where(counts[:, None], gd * (p - hot), 0.0)
    # p: the logit's error, the roundings of its argument, the exponential's units; then the difference and the product; bf16
    # rounds d once more
    e_p = p * (err * 1.01 + U * (3 * (l.abs() + lse.double().abs()[:, None]) + 8))
    e_d = torch.where(counts[:, None], gd.abs() * (e_p + 3 * U * (p + hot)), 0.0)
    if x.dtype == torch.bfloat16:
        e_d = e_d + R.rounding(x.dtype) * (d.abs() + e_d)
    xd = torch.where(counts[:, None], x.double(), 0.0)
    wd = w.double()
    out = []
    for a, ea, b, terms in ((d, e_d, wd, l.shape[1]), (d.T, e_d.T, xd, l.shape[0])):
        ref = a @ b
        # in bf16 the errors of single d are independent of one another: their sum is at most 8 times its standard deviation, with
        # near certainty, and never more than the sum of their bounds
        most = ea @ b.abs()
        spread = 8 * torch.sqrt((ea * ea) @ (b * b))
        off = torch.minimum(most, spread) if x.dtype == torch.bfloat16 else most
        # the part of e_d that all entries of a row share (lse's rounding) is no random one: in full
        off = off + R.sum_error((a.abs() + ea) @ b.abs(), x.dtype, terms)
        if x.dtype == torch.bfloat16:
            shared = (gd.abs() * p * (err * 1.01 + U * 8 + 3 * U * (l.abs() + lse.double().abs()[:, None])))
            off = off + (shared if a is d else shared.T) @ b.abs()
        out.append((ref, off + R.rounding(x.dtype) * 1.01 * (ref.abs() + off) + 1e-37))
    return out
