"""Layer norm where a workgroup takes several turns: more rows than one grid holds, for
each of the kernels (by the row's length), so that rows are on their way while others
are reduced, the sums change places in LDS, and the column sums run on.

The bounds are test_gpu_norm.py's."""
import pytest
import torch

from tests.gpu_util import log
from tests.test_gpu_norm import ROUND, U, _chain, _rows

pytestmark = pytest.mark.gpu

# Rows of a grid: 8192, 5120, 2048, 1280, 512 and 256 forward; 4096, 2048, 1024, 512, 256
# and 256 backward.  Three turns or so, the last of them not full.
FORWARD = [(18001, 500), (11301, 1000), (4501, 2000), (2823, 4000), (1131, 8000), (565, 12000)]
BACKWARD = [(9001, 500), (4501, 1000), (2301, 1531), (1131, 4000), (565, 8000), (564, 12000)]


def _own_type(x, dtype):
    rel, least = ROUND[dtype]
    return (rel + U) * x + least


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
def test_forward(gpu, dtype):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(91)
    for i, (rows, cols) in enumerate(FORWARD):
        log(f"layer_norm {dtype} {rows}x{cols}")
        x = _rows(gen, rows, cols, getattr(torch, dtype), (0, 3)[i % 2])
        w = torch.randn(cols, generator=gen, device="cuda")
        b = torch.randn(cols, generator=gen, device="cuda")
        y, mean, rstd = sgc.layer_norm(x, w, b, keep_stats=True)
        x64 = x.double()
        mu = x64.mean(1)
        r = 1.0 / torch.sqrt(((x64 - mu[:, None])**2).mean(1) + 1e-5)
        c = _chain(cols)
        dmu = c * U * x64.abs().mean(1)
        rel_r = 0.5 * (c + 6) * U + (dmu * r)**2 + dmu * r * 4 * U + 3 * U
        assert torch.all((mean.double() - mu).abs() <= dmu + U * mu.abs())
        assert torch.all((rstd.double() - r).abs() <= rel_r * r)
        hat = (x64 - mu[:, None]) * r[:, None]
        want = hat * w.double() + b.double()
        tol = w.double().abs() * (hat.abs() * (rel_r[:, None] + 4 * U)
                                  + (dmu * r)[:, None] * (1 + 8 * U))
        tol = tol + _own_type(want.abs() + tol, dtype)
        assert torch.all((y.double() - want).abs() <= tol)
        assert sgc.layer_norm(x, w, b, out=x) is x and torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
def test_backward(gpu, dtype):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(92)
    for i, (rows, cols) in enumerate(BACKWARD):
        log(f"layer_norm_backward {dtype} {rows}x{cols}")
        pad = (3, 0)[i % 2]
        x = _rows(gen, rows, cols, getattr(torch, dtype), pad)
        dy = _rows(gen, rows, cols, getattr(torch, dtype), pad)
        w = torch.randn(cols, generator=gen, device="cuda")
        _, mean, rstd = sgc.layer_norm(x, w, keep_stats=True)
        dx, dw, db = sgc.layer_norm_backward(dy, x, w, mean, rstd)
        dy64, r = dy.double(), rstd.double()[:, None]
        h = (x.double() - mean.double()[:, None]) * r
        g = dy64 * w.double()
        m1, m2 = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
        want = r * (g - m1 - h * m2)
        mass = g.abs().mean(1, keepdim=True) + h.abs() * (g * h).abs().mean(1, keepdim=True)
        tol = r * ((_chain(cols) + 8) * U * mass + 4 * U * (g.abs() + mass))
        tol = tol + _own_type(want.abs() + tol, dtype)
        assert torch.all((dx.double() - want).abs() <= tol)
        k = (min(rows, 1024) + 8) * U
        assert torch.all((dw.double() - (dy64 * h).sum(0)).abs() <= k * (dy64 * h).abs().sum(0))
        assert torch.all((db.double() - dy64.sum(0)).abs() <= k * dy64.abs().sum(0))
        again = sgc.layer_norm_backward(dy, x, w, mean, rstd, out=dy)
        assert again[0] is dy
        assert all(torch.equal(a, b) for a, b in zip(again, (dx, dw, db)))
