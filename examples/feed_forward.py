"""A feed-forward block in FP32 accuracy, trained and then served:

    h = layer_norm(x),  (u, z) = linear(h, W1, b1, gelu),  y = x + linear(u, W2, b2)

`python examples/feed_forward.py` trains the block to reproduce another one with
random weights, prints the loss as it falls and the time of a training step, and
then runs single tokens through it.  Everything after the inputs are made is a
kernel of libsgemmcube.so, but for the loss and its gradient.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2507_23387_amd as sgc  # noqa: E402

NAMES = ("norm.weight", "norm.bias", "w1", "b1", "w2", "b2")


class FeedForward:
    """The block's parameters (weights K x N) and its forward and backward pass."""

    def __init__(self, hidden: int, inner: int, generator: torch.Generator, activation="gelu"):
        def normal(*shape, std):
            return torch.randn(shape, generator=generator).mul_(std).cuda()

        self.activation = activation
        self.parameters = {
            "norm.weight": torch.ones(hidden, device="cuda"),
            "norm.bias": torch.zeros(hidden, device="cuda"),
            "w1": normal(hidden, inner, std=hidden**-0.5), "b1": normal(inner, std=0.1),
            "w2": normal(inner, hidden, std=inner**-0.5), "b2": normal(hidden, std=0.1),
        }

    def __call__(self, x, keep=False):
        """y, or (y, what backward needs) with keep=True."""
        p = self.parameters
        h = sgc.layer_norm(x, p["norm.weight"], p["norm.bias"], keep_stats=keep)
        h, *stats = h if keep else (h,)
        u = sgc.linear(h, p["w1"], p["b1"], activation=self.activation, keep_preact=keep)
        u, *z = u if keep else (u,)
        y = sgc.linear(u, p["w2"], p["b2"], residual=x)
        return (y, (x, *stats, h, *z, u)) if keep else y

    def backward(self, dy, kept):
        """(gradient of x, the parameters' gradients in NAMES' order)."""
        p = self.parameters
        x, mean, rstd, h, z, u = kept
        du, dw2, db2 = sgc.linear_backward(dy, u, p["w2"])
        dh, dw1, db1 = sgc.linear_backward(du, h, p["w1"], z, activation=self.activation)
        dx, dweight, dbias = sgc.layer_norm_backward(dh, x, p["norm.weight"], mean, rstd, out=dh)
        return dx.add_(dy), (dweight, dbias, dw1, db1, dw2, db2)


def optimizer(block, lr: float, state_bits: int):
    """AdamW that decays the matrices alone."""
    tensors = [block.parameters[name] for name in NAMES]
    return sgc.AdamW(tensors, lr=lr, weight_decay=[0.01 if t.dim() == 2 else 0.0 for t in tensors],
                     state_bits=state_bits)


def train_step(block, opt, x, target):
    """One step on the mean squared error; returns the loss, still on the device."""
    y, kept = block(x, keep=True)
    error = y.sub_(target)
    loss = error.square().mean()
    _, grads = block.backward(error.mul_(2.0 / error.numel()), kept)
    opt.step(grads)
    return loss


def main(argv=None):
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--rows", type=int, default=4096)
    parser.add_argument("--hidden", type=int, default=1024)
    parser.add_argument("--inner", type=int, default=4096)
    parser.add_argument("--steps", type=int, default=50)
    parser.add_argument("--lr", type=float, default=1e-3)
    parser.add_argument("--state-bits", type=int, default=8, choices=(8, 32))
    args = parser.parse_args(argv)

    generator = torch.Generator().manual_seed(0)
    teacher = FeedForward(args.hidden, args.inner, generator)
    block = FeedForward(args.hidden, args.inner, generator)
    opt = optimizer(block, args.lr, args.state_bits)
    x = torch.randn((args.rows, args.hidden), generator=generator).cuda()
    target = teacher(x)

    losses = [train_step(block, opt, x, target)]  # also the first use of every kernel
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(args.steps - 1):
        losses.append(train_step(block, opt, x, target))
    end.record()
    losses = torch.stack(losses).tolist()
    for step in range(0, args.steps, max(1, args.steps // 10)):
        print(f"step {step + 1:4d}  loss {losses[step]:.6f}")
    if args.steps > 1:
        ms = begin.elapsed_time(end) / (args.steps - 1)
        print(f"{ms:.3f} ms a step of {args.rows} rows, {args.hidden} to {args.inner} and back")

    token = x[:1]
    block(token)
    begin.record()
    for _ in range(100):
        y = block(token)
    end.record()
    end.synchronize()
    print(f"{10 * begin.elapsed_time(end):.1f} us a token; "
          f"off the teacher by {(y - target[:1]).square().mean().item():.6f}")
    return losses


if __name__ == "__main__":
    main()
