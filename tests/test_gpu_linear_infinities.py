"""An infinity among a linear layer's gradients: it shows in its row of dX and its
column of dW and dbias, and everything else is what it is without it.

D's largest finite magnitude sets the power of two that D is split with, so the
entry that the infinity takes the place of is 0 in the clean gradient.  dW of
4096 x 4096 is computed by the 256-wide kernels, which leave results that FP16
cannot hold to a second kernel; 300 x 200 by the small tiles."""
import pytest
import torch

from tests.gpu_util import log

pytestmark = pytest.mark.gpu

ORDERS = {"elementwise": 0, "termwise": 1, "elementwise_cross_first": 2}
SHAPES = [(512, 4096, 4096), (130, 200, 300)]


def _operands(m, n, k, layout):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(51)
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    W = randn(*((n, k) if layout == "nk" else (k, n))) / k**0.5
    dY = randn(m, n) * 1e-4
    dY[4, 5] = 0
    return dY, randn(m, n), randn(m, k), W


def _backward(dY, Z, X, W, layout, order, activation=2):
    """Through the C-ABI, into gradients that hold 7."""
    from paper_2507_23387_amd import binding

    m, n, k = dY.shape[0], dY.shape[1], X.shape[1]
    size = binding.sgemm_cube_linear_backward_workspace_size(m, n, k)
    ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
    dX, dW, db = (torch.full(s, 7.0, device="cuda") for s in (X.shape, W.shape, (n,)))
    assert binding.sgemm_cube_linear_backward(
        m, n, k, dY.data_ptr(), n, Z.data_ptr(), n, X.data_ptr(), k, W.data_ptr(), W.shape[1],
        layout == "nk", activation, dX.data_ptr(), k, dW.data_ptr(), W.shape[1], db.data_ptr(),
        2048.0, ORDERS[order], ws.data_ptr(), size, torch.cuda.current_stream().cuda_stream) == 0
    return dX, dW.t() if layout == "nk" else dW, db


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("layout", ["kn", "nk"])
def test_an_infinity_stays_in_its_row_and_column(gpu, layout, order):
    for m, n, k in SHAPES:
        dY, Z, X, W = _operands(m, n, k, layout)
        clean = _backward(dY, Z, X, W, layout, order)
        assert all(torch.isfinite(g).all() for g in clean)
        other = torch.arange(n, device="cuda") != 5
        rows = torch.arange(m, device="cuda") != 4
        # In dY, and from the product with gelu' (1.13 at most, at sqrt 2).
        for value, z in ((float("inf"), 0.5), (-float("inf"), 0.5), (3.2e38, 2**0.5)):
            log(f"linear_backward {layout} {order} {m}x{n}x{k}, {value} in dY")
            dY[4, 5], Z[4, 5] = value, z
            dX, dW, db = _backward(dY, Z, X, W, layout, order)
            assert not torch.isfinite(dX[4]).any() and torch.equal(dX[rows], clean[0][rows])
            assert not torch.isfinite(dW[:, 5]).any()
            assert torch.equal(dW[:, other], clean[1][:, other])
            assert torch.isinf(db[5]) and torch.equal(db[other], clean[2][other])


@pytest.mark.parametrize("order", ORDERS)
def test_replays_after_an_infinity(gpu, order):
    """A captured call keeps what marks its splits, and a caller's workspace keeps what
    an earlier replay left there."""
    import paper_2507_23387_amd as sgc
    from paper_2507_23387_amd import binding

    for m, n, k in SHAPES:
        dY, Z, X, W = _operands(m, n, k, "kn")
        ws = torch.zeros(binding.sgemm_cube_linear_backward_workspace_size(m, n, k),
                         dtype=torch.uint8, device="cuda")

        def step(workspace=None):
            return sgc.linear_backward(dY, X, W, Z, "gelu", order=order, workspace=workspace)

        step(ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = step(ws)
        for value in (0.0, float("inf"), 0.0, 1e-4):
            log(f"linear_backward {order} {m}x{n}x{k}, replay with {value} in dY")
            dY[4, 5] = value
            for h in held:
                h.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            got = [h.clone() for h in held]
            want = step()
            torch.cuda.synchronize()
            for g, w in zip(got, want):
                assert torch.equal(torch.isfinite(g), torch.isfinite(w))
                assert torch.equal(g[torch.isfinite(g)], w[torch.isfinite(w)])
