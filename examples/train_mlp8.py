"""Merge-aware training of a small residual MLP whose layers run on the library's linear operators and keep their
activations in 8 bits.

A few blocks x + MLP(x) and a classifier are trained on a synthetic task with the periodic schedule (three ordinary
steps, one simulated-loss step per period): on a simulated-loss step the parameters' storage holds theta~, so forward and
backward products read theta~; the weight gradients are then mapped and theta is updated. Run on one GPU:

    python examples/train_mlp8.py [--steps 200] [--width 256] [--hidden 1024] [--blocks 4] [--batch 2056]
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_33437_gb300 import linear as L  # noqa: E402
from paper_2609_33437_gb300 import smat as S  # noqa: E402
from paper_2609_33437_gb300.schedule import PeriodicSmat  # noqa: E402


class Net(torch.nn.Module):
    """Blocks x + MLP(x), then a linear classifier with a GELU before it."""

    def __init__(self, width, hidden, blocks, classes, dtype):
        super().__init__()
        kw = dict(device="cuda", dtype=dtype)
        self.blocks = torch.nn.ModuleList(L.Mlp8(width, hidden, act="quick_gelu", **kw) for _ in range(blocks))
        self.neck = L.Linear8(width, width, act="gelu", **kw)
        self.head = L.Linear8(width, classes, **kw)

    def forward(self, x):
        for b in self.blocks:
            x = b(x, residual=x)
        return self.head(self.neck(x))


def train(steps=200, width=256, hidden=1024, blocks=4, batch=2056, classes=10, dtype=torch.float32, lr=1e-3, seed=0,
          period=4):
    """The losses of every step."""
    torch.manual_seed(seed)
    net = Net(width, hidden, blocks, classes, dtype)
    teacher = torch.randn(width, classes, device="cuda")
    params = list(net.parameters())
    theta0 = [p.detach().clone() for p in params]
    # weights are masked and perturbed, biases perturbed only (the mask set of the paper's linear weights)
    keep = [0.9 if p.dim() == 2 else 1.0 for p in params]
    sched = PeriodicSmat(params, keep, [1e-4] * len(params), theta0=theta0, period=period, seed=seed, alpha_min=0.8,
                         alpha_max=1.0, alpha_mode=S.SMAT_ALPHA_GLOBAL, noise=S.SMAT_NOISE_UNIFORM)
    opt = torch.optim.AdamW(params, lr=lr)
    losses = []
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    for step in range(steps):
        x = torch.randn(batch, width, device="cuda", generator=gen)
        target = (x @ teacher).argmax(1)
        sched.before_forward(step)
        loss = torch.nn.functional.cross_entropy(net(x.to(dtype)).float(), target)
        loss.backward()
        sched.optimizer_step(step, opt)
        opt.zero_grad()
        losses.append(loss.detach())
    sched.close()
    losses = torch.stack(losses).tolist()
    # the losses have been waited for: a look at what no call returns. Before a checkpoint is written is the place for it in
    # a longer run.
    if L.poll_errors():
        raise RuntimeError("a wait inside a product ran out: some step's gradients are unfinished")
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    for name, value in (("steps", 200), ("width", 256), ("hidden", 1024), ("blocks", 4), ("batch", 2056)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--bf16", action="store_true", help="bf16 parameters and activations")
    a = ap.parse_args()
    losses = train(a.steps, a.width, a.hidden, a.blocks, a.batch, dtype=torch.bfloat16 if a.bf16 else torch.float32)
    for i in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"step {i:5d}  loss {losses[i]:.4f}")
    print(f"step {len(losses) - 1:5d}  loss {losses[-1]:.4f}")
