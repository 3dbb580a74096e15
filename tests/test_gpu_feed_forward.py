"""The layers together, as examples/feed_forward.py runs them: the block and all its
gradients against the same formulas in 64 bits, training, and single tokens."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "feed_forward.py")

# What each product, norm and sum of the block is off by is below 1e-6 of its
# result's norm (22-bit operands and 32-bit sums), and a gradient passes through
# at most eight of them.
REL = 1e-5


@pytest.fixture(scope="module")
def example(gpu):
    spec = importlib.util.spec_from_file_location("feed_forward", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def off(got, want):
    return ((got.double().cpu() - want).norm() / want.norm()).item()


@pytest.mark.parametrize("rows,hidden,inner", [(1, 64, 256), (37, 96, 200), (300, 256, 1024)])
def test_block_and_gradients_in_64_bits(example, rows, hidden, inner):
    gen = torch.Generator().manual_seed(rows)
    block = example.FeedForward(hidden, inner, gen)
    x = torch.randn((rows, hidden), generator=gen)
    dy = torch.randn((rows, hidden), generator=gen) * 1e-6
    y, kept = block(x.cuda(), keep=True)
    dx, grads = block.backward(dy.cuda(), kept)

    p = {n: block.parameters[n].double().cpu().requires_grad_() for n in example.NAMES}
    xd = x.double().requires_grad_()
    mean = xd.mean(1, keepdim=True)
    var = (xd - mean).square().mean(1, keepdim=True)
    h = (xd - mean) / (var + 1e-5).sqrt() * p["norm.weight"] + p["norm.bias"]
    z = h @ p["w1"] + p["b1"]
    u = z * 0.5 * (1 + torch.erf(z / math.sqrt(2)))
    want = xd + u @ p["w2"] + p["b2"]
    assert off(y, want.detach()) < REL
    want.backward(dy.double())
    assert off(dx, xd.grad) < REL
    for name, grad in zip(example.NAMES, grads):
        assert off(grad, p[name].grad) < REL, name
    assert torch.equal(block(x.cuda()), y)  # the same with nothing kept


@pytest.mark.parametrize("state_bits", [8, 32])
def test_training_and_tokens(example, state_bits, capsys):
    losses = example.main(["--rows", "256", "--hidden", "64", "--inner", "256", "--steps", "60",
                           "--lr", "3e-3", "--state-bits", str(state_bits)])
    assert len(losses) == 60 and all(map(math.isfinite, losses))
    # A factor of 29 in plain FP32 with 32-bit states.
    assert losses[-1] < losses[0] / 4
    assert "a token" in capsys.readouterr().out
