"""The embedding, the gated block and the cross entropy as a program uses them together
(examples/language_model.py): losses and gradients against the same model in 64 bits with
torch's autograd, a training step captured into a graph, the example itself.

The bound on gradients is relative to each tensor's norm: every operator's result is off by
a few 2^-22 of its operands' magnitudes (their own tests), which a chain of 10 operators
with sums of at most 300 terms keeps below 300^(1/2) 10 2^-21, 8e-5."""
import os
import sys

import pytest
import torch

from tests.gpu_util import log

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BOUND = 300**0.5 * 10 * 2.0**-21


@pytest.fixture()
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import language_model

    return language_model


def _losses64(model, p, ids, targets):
    act = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu,
           "relu": torch.relu}[model.activation]
    norm = lambda x, name: torch.nn.functional.layer_norm(  # noqa: E731
        x, x.shape[1:], p[f"{name}.weight"], p[f"{name}.bias"], 1e-5)
    live = (ids >= 0)[:, None]
    x = torch.where(live, p["table"][ids.clamp(min=0)] * model.scale, 0.0)
    for b in range(model.blocks):
        h = norm(x, f"{b}.norm")
        x = x + (act(h @ p[f"{b}.gate"]) * (h @ p[f"{b}.up"])) @ p[f"{b}.down"]
    z = norm(x, "norm") @ p["table"].t()
    loss = torch.logsumexp(z, 1) - z.gather(1, targets.clamp(min=0)[:, None])[:, 0]
    return torch.where(targets >= 0, loss, 0.0)


@pytest.mark.parametrize("tokens", [1, 37, 400])
@pytest.mark.parametrize("activation", ["silu", "gelu"])
def test_against_autograd_in_64_bits(gpu, example, tokens, activation):
    generator = torch.Generator().manual_seed(7)
    model = example.LanguageModel(301, 136, 200, 2, generator, activation)
    ids = torch.randint(301, (tokens,), generator=generator)
    targets = torch.randint(301, (tokens,), generator=generator)
    if tokens > 2:
        ids[tokens // 2], targets[tokens // 2], targets[1] = -1, -1, -1  # a place without a token
    dloss = torch.rand(tokens, generator=generator)
    log(f"language model, {tokens} tokens, {activation}")
    loss, grads = model.gradients(ids.cuda(), targets.cuda(), dloss.cuda())
    assert torch.equal(loss, model.losses(ids.cuda(), targets.cuda()))

    p = {name: t.double().cpu().requires_grad_() for name, t in model.parameters.items()}
    want = _losses64(model, p, ids, targets)
    assert (loss.double().cpu() - want).norm() <= BOUND * want.norm()
    (want * dloss.double()).sum().backward()
    for (name, t), got in zip(p.items(), grads):
        error = (got.double().cpu() - t.grad).norm()
        assert error <= BOUND * t.grad.norm() + 1e-30, (name, (error / t.grad.norm()).item())


def test_a_captured_step(gpu, example):
    """A step in a graph on tokens that change between replays, against the same steps of
    another model without one."""
    generator = torch.Generator().manual_seed(8)
    models = [example.LanguageModel(301, 136, 200, 1, torch.Generator().manual_seed(9))
              for _ in range(2)]
    opts = [example.optimizer(m, 1e-3) for m in models]
    draw = lambda: torch.randint(301, (2, 200), generator=generator).cuda()  # noqa: E731
    ids, targets = draw()
    dloss = torch.full((200,), 1 / 200, device="cuda")

    def step(which, number):
        losses, grads = models[which].gradients(ids, targets, dloss)
        opts[which].step(grads, step=number)
        return losses

    # The captured step's number, and so its corrections, stay on every replay.
    step(0, 1), step(1, 1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(0, 2)
    for _ in range(3):
        new = draw()
        ids.copy_(new[0])
        targets.copy_(new[1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held.clone(), step(1, 2))
        for a, b in zip(models[0].parameters.values(), models[1].parameters.values()):
            assert torch.equal(a, b)


def test_a_graph_refuses_values_that_were_written_over(gpu):
    """autograd is told of what the calls write to; results require no gradient."""
    import paper_2507_23387_amd as sgc

    x, w = torch.randn((4, 8), device="cuda"), torch.randn((8, 8), device="cuda")
    ids = torch.arange(4, device="cuda")
    parameter = torch.nn.Parameter(w)
    for write in (lambda t: sgc.embedding(ids, parameter, out=t),
                  lambda t: sgc.embedding_backward(x, ids, 4, add_to=t),
                  lambda t: sgc.gated_linear(x, parameter, w, out=t)):
        t = torch.randn((4, 8), device="cuda")
        ones = torch.ones((4, 8), device="cuda", requires_grad=True)
        loss, before = (ones * t).sum(), t.clone()
        assert not write(t).requires_grad and not torch.equal(t, before)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    loss, lse = sgc.linear_cross_entropy(x, parameter, ids)
    assert not loss.requires_grad and not lse.requires_grad


def test_the_example_runs(gpu, example, capsys):
    means = example.main(["--tokens", "512", "--vocab", "1000", "--hidden", "128", "--inner",
                          "256", "--steps", "6"])
    assert len(means) == 6 and all(m == m for m in means)
    assert "us for the score of a token" in capsys.readouterr().out
