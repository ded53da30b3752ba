"""A block of a graph network made of the sparse product and the layers beside it, and a small training run of it.

    s = h + dropout(A h);   y = layer norm of s;   h' = s + dropout(feed-forward block of y)

The product runs in float32 (``autograd.SparseOperator``), the layers in the type of ``h``; parameters are held in float32.  Each
block has a seed of its own for its two dropouts; the step counts as their offset.

    python -m paper_2106_16064_amd.graph_block --scale 14 --width 64 --hidden 128 --steps 50
"""
from __future__ import annotations

import argparse

import torch

from .layers import add_layer_norm, dropout, gated_ff


class GraphBlock(torch.nn.Module):
    """``width`` features per vertex in and out, ``hidden`` in the feed-forward block."""

    def __init__(self, width, hidden, p=0.1, activation="silu", seed=0, device="cuda:0"):
        super().__init__()
        at = {"device": device}
        self.p, self.activation, self.seed = p, activation, seed
        self.weight = torch.nn.Parameter(torch.ones(width, **at))
        self.bias = torch.nn.Parameter(torch.zeros(width, **at))
        self.w_gate = torch.nn.Parameter(torch.randn(hidden, width, **at) * width ** -0.5)
        self.w_up = torch.nn.Parameter(torch.randn(hidden, width, **at) * width ** -0.5)
        self.w_down = torch.nn.Parameter(torch.randn(width, hidden, **at) * hidden ** -0.5)

    def forward(self, op, h, step=0):
        """``op``: the matrix, as ``SparseOperator``; ``step``: an int, or an int64 GPU tensor of one element."""
        p = self.p if self.training else 0.0
        met = op(h.float()).to(h.dtype)
        y, s = add_layer_norm(met, h, self.weight, self.bias, p=p, seed=2 * self.seed, offset=step)
        weights = (w.to(h.dtype) for w in (self.w_gate, self.w_up, self.w_down))
        return dropout(gated_ff(y, *weights, self.activation), p, 2 * self.seed + 1, step, residual=s)


def train(op, features, target, blocks=2, hidden=128, p=0.1, steps=50, rate=0.01, seed=0):
    """Fits ``blocks`` of them to ``target`` (least squares); returns the blocks and the loss of each step."""
    torch.manual_seed(seed)
    layers = torch.nn.ModuleList(GraphBlock(features.shape[1], hidden, p, seed=i, device=features.device)
                                 for i in range(blocks))
    optimiser = torch.optim.Adam(layers.parameters(), rate)
    losses = []
    for step in range(steps):
        h = features
        for block in layers:
            h = block(op, h, step)
        loss = (h.float() - target.float()).square().mean()
        optimiser.zero_grad()
        loss.backward()
        optimiser.step()
        losses.append(loss.detach())
    return layers, torch.stack(losses).tolist()


def main(argv=None):
    from .autograd import SparseOperator
    from .workloads import rmat_csr
    parser = argparse.ArgumentParser(description="Trains graph blocks on an R-MAT graph to repeat another network of random weights.")
    parser.add_argument("--scale", type=int, default=14, help="2^scale vertices")
    parser.add_argument("--width", type=int, default=64)
    parser.add_argument("--hidden", type=int, default=128)
    parser.add_argument("--blocks", type=int, default=2)
    parser.add_argument("--steps", type=int, default=50)
    parser.add_argument("--p", type=float, default=0.1, help="rate of dropout")
    parser.add_argument("--dtype", choices=("float32", "bfloat16"), default="bfloat16")
    args = parser.parse_args(argv)
    dtype = getattr(torch, args.dtype)
    op = SparseOperator(rmat_csr(args.scale, 16, seed=0, values="rownorm"))
    torch.manual_seed(1)
    features = torch.randn(op.fwd.K, args.width, device="cuda:0", dtype=dtype)
    teacher = GraphBlock(args.width, args.hidden, 0.0, seed=9)
    with torch.no_grad():
        target = teacher.eval()(op, features)
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    _, losses = train(op, features, target, args.blocks, args.hidden, args.p, args.steps)
    end.record()
    end.synchronize()
    print(f"{op.fwd.M} vertices, {args.blocks} blocks of {args.width} x {args.hidden}, {args.dtype}: "
          f"loss {losses[0]:.4f} -> {losses[-1]:.4f} in {args.steps} steps, {start.elapsed_time(end) / args.steps:.2f} ms a step")
    return losses


if __name__ == "__main__":
    main()
