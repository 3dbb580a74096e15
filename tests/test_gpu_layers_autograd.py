"""The layers have no autograd of their own, but tell torch's of what they write to: a
graph that has saved a tensor refuses to go back through values it no longer has."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _saved(shape):
    """A tensor, and a loss whose graph has saved its values."""
    t = torch.randn(shape, device="cuda")
    w = torch.ones(shape, device="cuda", requires_grad=True)
    return t, (w * t).sum()


def _writes():
    import paper_2507_23387_amd as sgc

    x, w = torch.randn((4, 8), device="cuda"), torch.randn((8, 8), device="cuda")
    _, mean, rstd = sgc.layer_norm(x, keep_stats=True)
    grad = [torch.ones((4, 8), device="cuda")]
    opt = sgc.AdamW([torch.ones((4, 8), device="cuda")], state_bits=8)
    spare = torch.empty((4, 8), device="cuda")
    return {
        "linear": lambda t: sgc.linear(x, w, out=t),
        "linear, residual in place": lambda t: sgc.linear(x, w, residual=t, out=t),
        "layer_norm": lambda t: sgc.layer_norm(x, out=t),
        "layer_norm in place": lambda t: sgc.layer_norm(t, out=t),
        "layer_norm_backward in place":
            lambda t: sgc.layer_norm_backward(t, x, None, mean, rstd, out=t),
        "AdamW.step, 32 bits": lambda t: sgc.AdamW([t]).step(grad),
        "AdamW.step, 8 bits": lambda t: sgc.AdamW([t], state_bits=8).step(grad),
        "AdamW.state_values": lambda t: opt.state_values(out=([t], [spare])),
    }


def test_a_graph_refuses_values_that_were_written_over(gpu):
    for name, write in _writes().items():
        t, loss = _saved((4, 8))
        before = t.clone()
        write(t)
        assert not torch.equal(t, before), name
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()


def test_results_without_autograd(gpu):
    """Parameters that require gradients are taken, by the optimizer too, and the
    results do not; inference tensors are written to as well."""
    import paper_2507_23387_amd as sgc

    w = torch.nn.Parameter(torch.ones((8, 8), device="cuda"))
    x = torch.randn((4, 8), device="cuda", requires_grad=True)
    y = sgc.linear(x, w)
    assert not y.requires_grad and not sgc.layer_norm(x).requires_grad
    dX, dW, _ = sgc.linear_backward(torch.ones_like(y), x, w)
    assert not dX.requires_grad and not dW.requires_grad
    opt = sgc.AdamW([w])
    opt.step([dW])
    assert w.requires_grad and not torch.equal(w, torch.ones_like(w))
    with torch.inference_mode():
        for write in _writes().values():
            write(torch.randn((4, 8), device="cuda"))
