"""A language model without attention, trained and then asked, in FP32 accuracy: each token
predicts the next by

    x = embedding(ids) sqrt(hidden);  per block x += down(gated_linear(layer_norm(x)));
    loss = linear_cross_entropy(layer_norm(x), table)

with one table at both ends (its gradient is the loss's, to which the lookup's is added).
`python examples/language_model.py` trains it on text drawn from a random table of which
token follows which, and prints the loss as it falls, the time of a training step and of
the score of a single token.  Everything after the inputs are made is a kernel of
libsgemmcube.so, but for the residual sums of the gradients and the mean of the losses.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2507_23387_amd as sgc  # noqa: E402


class LanguageModel:
    """Parameters, forward and backward pass.  Weights are K x N, the table vocabulary x
    hidden."""

    def __init__(self, vocab: int, hidden: int, inner: int, blocks: int,
                 generator: torch.Generator, activation="silu"):
        def normal(*shape, std):
            return torch.randn(shape, generator=generator).mul_(std).cuda()

        self.activation, self.blocks, self.scale = activation, blocks, hidden**0.5
        p = self.parameters = {"table": normal(vocab, hidden, std=hidden**-0.5)}
        for b in range(blocks):
            p[f"{b}.norm.weight"] = torch.ones(hidden, device="cuda")
            p[f"{b}.norm.bias"] = torch.zeros(hidden, device="cuda")
            p[f"{b}.gate"] = normal(hidden, inner, std=hidden**-0.5)
            p[f"{b}.up"] = normal(hidden, inner, std=hidden**-0.5)
            p[f"{b}.down"] = normal(inner, hidden, std=inner**-0.5)
        p["norm.weight"] = torch.ones(hidden, device="cuda")
        p["norm.bias"] = torch.zeros(hidden, device="cuda")

    def features(self, ids, keep=False):
        """The output layer's input, or (that, what backward needs) with keep=True."""
        p, kept = self.parameters, []
        x = sgc.embedding(ids, p["table"], scale=self.scale)
        for b in range(self.blocks):
            h = sgc.layer_norm(x, p[f"{b}.norm.weight"], p[f"{b}.norm.bias"], keep_stats=keep)
            h, *stats = h if keep else (h,)
            u = sgc.gated_linear(h, p[f"{b}.gate"], p[f"{b}.up"], activation=self.activation,
                                 keep_preact=keep)
            u, *z = u if keep else (u,)
            kept.append((x, stats, h, z, u))
            x = sgc.linear(u, p[f"{b}.down"], residual=x)
        f = sgc.layer_norm(x, p["norm.weight"], p["norm.bias"], keep_stats=keep)
        f, *stats = f if keep else (f,)
        return (f, (kept, x, stats)) if keep else f

    def losses(self, ids, targets):
        """The losses of the targets, one for each token."""
        return sgc.linear_cross_entropy(self.features(ids), self.parameters["table"], targets,
                                        transpose_w=True)[0]

    def gradients(self, ids, targets, dloss):
        """(losses, the parameters' gradients in their order) for the losses' gradients."""
        p, grads = self.parameters, {}
        f, (kept, x, stats) = self.features(ids, keep=True)
        loss, lse = sgc.linear_cross_entropy(f, p["table"], targets, transpose_w=True)
        df, table, _ = sgc.linear_cross_entropy_backward(
            dloss, f, p["table"], targets, lse, transpose_w=True, need=("dX", "dW"))
        dx, grads["norm.weight"], grads["norm.bias"] = sgc.layer_norm_backward(
            df, x, p["norm.weight"], *stats, out=df)
        for b in reversed(range(self.blocks)):
            x, stats, h, z, u = kept[b]
            du, grads[f"{b}.down"], _ = sgc.linear_backward(dx, u, p[f"{b}.down"],
                                                            need=("dX", "dW"))
            dh, grads[f"{b}.gate"], grads[f"{b}.up"], _, _ = sgc.gated_linear_backward(
                du, h, p[f"{b}.gate"], p[f"{b}.up"], *z, activation=self.activation,
                need=("dX", "dW_gate", "dW_up"))
            dh, grads[f"{b}.norm.weight"], grads[f"{b}.norm.bias"] = sgc.layer_norm_backward(
                dh, x, p[f"{b}.norm.weight"], *stats, out=dh)
            dx.add_(dh)
        grads["table"] = sgc.embedding_backward(dx, ids, len(table), scale=self.scale,
                                                add_to=table)
        return loss, [grads[name] for name in p]


def optimizer(model, lr: float, state_bits: int = 32):
    """AdamW that decays the matrices alone."""
    tensors = list(model.parameters.values())
    return sgc.AdamW(tensors, lr=lr, weight_decay=[0.01 if t.dim() == 2 else 0.0 for t in tensors],
                     state_bits=state_bits)


def train_step(model, opt, ids, targets, dloss):
    """One step on sum(dloss * losses); returns the losses, still on the device."""
    losses, grads = model.gradients(ids, targets, dloss)
    opt.step(grads)
    return losses


def main(argv=None):
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--tokens", type=int, default=8192)
    parser.add_argument("--vocab", type=int, default=32000)
    parser.add_argument("--hidden", type=int, default=1024)
    parser.add_argument("--inner", type=int, default=2816)
    parser.add_argument("--blocks", type=int, default=2)
    parser.add_argument("--steps", type=int, default=50)
    parser.add_argument("--lr", type=float, default=1e-3)
    parser.add_argument("--state-bits", type=int, default=32, choices=(8, 32))
    args = parser.parse_args(argv)

    generator = torch.Generator().manual_seed(0)
    model = LanguageModel(args.vocab, args.hidden, args.inner, args.blocks, generator)
    opt = optimizer(model, args.lr, args.state_bits)
    # Each token is followed by one of four; an end of text now and then, of which nothing
    # is to be learnt.
    follows = torch.randint(args.vocab, (args.vocab, 4), generator=generator)
    ids = [0]
    for choice in torch.randint(4, (args.tokens,), generator=generator).tolist():
        ids.append(int(follows[ids[-1], choice]))
    ids = torch.tensor(ids)
    targets = ids[1:].clone()
    targets[torch.rand(args.tokens, generator=generator) < 0.02] = -1
    ids, targets = ids[:-1].cuda(), targets.cuda()
    dloss = torch.full((args.tokens,), 1.0 / int((targets >= 0).sum()), device="cuda")

    means = [train_step(model, opt, ids, targets, dloss).dot(dloss)]  # first use of every kernel
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(args.steps - 1):
        means.append(train_step(model, opt, ids, targets, dloss).dot(dloss))
    end.record()
    means = torch.stack(means).tolist()
    for step in range(0, args.steps, max(1, args.steps // 10)):
        print(f"step {step + 1:4d}  loss {means[step]:.6f}")
    if args.steps > 1:
        ms = begin.elapsed_time(end) / (args.steps - 1)
        print(f"{ms:.3f} ms a step of {args.tokens} tokens, {args.vocab} x {args.hidden}, "
              f"{args.blocks} blocks of {args.inner}")

    model.losses(ids[:1], targets[:1])
    begin.record()
    for _ in range(100):
        model.losses(ids[:1], targets[:1])
    end.record()
    end.synchronize()
    print(f"{10 * begin.elapsed_time(end):.1f} us for the score of a token")
    return means


if __name__ == "__main__":
    main()
