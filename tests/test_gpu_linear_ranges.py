"""A linear layer's gradients whose rows and columns lie many decades apart.

Each entry of dX sums one row of D = dY act'(Z), each of dW one column, so each is
held to that line's own size.  The bounds are test_gpu_linear.py's, u = 2^-24: 3 2^-21
+ (3 k / 32 + 40) u of |A||B|; W's and X's floor of 2^-36; and D's, whose lines are
brought to 2^3 at least, 2^-39 of the line's largest magnitude (2^-38 with the
residual's own rounding)."""
import pytest
import torch

from tests.gpu_util import log
from tests.test_gpu_linear import ORDERS, U, _act64, _case, _mat

pytestmark = pytest.mark.gpu

# In this order: dW as an outer product, dX by rows with dW on tiles, both on tiles in
# one launch, ragged ones, and the 256-wide kernels.
SHAPES = [(20, 1301, 1303), (100, 1500, 1400), (300, 200, 130), (777, 530, 131),
          (520, 4096, 4090)]


def _bound(A, B, line):
    """|A||B|'s share and the two floors; `line`: the largest magnitudes of D's lines,
    as a column where D is A and as a row where it is B."""
    k = A.shape[1]
    tol = (3 * 2.0**-21 + (3 * k / 32 + 40) * U) * (A.abs() @ B.abs())
    rows, cols = A.abs().sum(1)[:, None], B.abs().sum(0)[None, :]
    if line.shape[1] == 1:
        return tol + 2.0**-38 * line * cols + 2.0**-35 * rows
    return tol + 2.0**-38 * line * rows + 2.0**-35 * cols


def _check(dY, X, Wkn, Z, act, dX, dW, db):
    d, x, w = dY.double(), X.double().contiguous(), Wkn.double().contiguous()
    D = d * (1.0 if act == "none" else _act64(act, Z.double(), grad=True))
    off = 0 * d if act == "none" else 16 * U * (1 + Z.double().abs()) * d.abs()
    wt, xt = w.t().contiguous(), x.t().contiguous()
    for name, got, A, B, line, extra in (
            ("dX", dX, D, wt, D.abs().amax(1, keepdim=True), off @ wt.abs()),
            ("dW", dW, xt, D, D.abs().amax(0, keepdim=True), xt.abs() @ off)):
        want = A @ B
        tol = _bound(A, B, line) + extra + U * want.abs() + 2.0**-126
        worst = ((got.double() - want).abs() / tol).max().item()
        assert worst <= 1, f"{name}: {worst:.3g} of the bound"
    tol = (min(D.shape[0], 1024) + 8) * U * D.abs().sum(0) + off.sum(0) + 2.0**-126
    assert torch.all((db.double() - D.sum(0)).abs() <= tol)


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("layout", ["kn", "nk"])
def test_lines_of_a_gradient_keep_their_digits(gpu, order, layout):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(61)
    for i, (m, n, k) in enumerate(SHAPES):
        X, W, Wkn = _case(gen, m, n, k, layout, (0, 3)[i % 2])
        Z, act = _mat(gen, m, n), ("none", "gelu", "silu")[i % 3]
        for rows, cols in ((0, 14), (14, 0), (6, 8)):
            log(f"linear_backward {layout} {order} {m}x{n}x{k}, rows over {rows} decades, "
                f"columns over {cols}")
            r = 10.0 ** (-rows * torch.rand((m, 1), generator=gen, device="cuda"))
            c = 10.0 ** (-cols * torch.rand((1, n), generator=gen, device="cuda"))
            dY = _mat(gen, m, n) * r * c
            dY[m // 2], dY[:, n // 2] = 0, 0
            got = sgc.linear_backward(dY, X, W, None if act == "none" else Z, act,
                                      transpose_w=layout == "nk", order=order)
            dX, dW, db = got
            _check(dY, X, Wkn, Z, act, dX, dW.t() if layout == "nk" else dW, db)
            assert not dX[m // 2].any() and not db[n // 2].any()
            for which in ("dX", "dW", "db"):
                at = ("dX", "dW", "db").index(which)
                only = sgc.linear_backward(dY, X, W, None if act == "none" else Z, act,
                                           transpose_w=layout == "nk", order=order, need=(which,))
                assert torch.equal(only[at], got[at])


def test_the_largest_and_the_smallest_floats(gpu):
    """Lines of 1e-38 and of 3e38 beside each other."""
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(62)
    for m, n, k in ((40, 50, 60), (300, 200, 130)):
        for layout in ("kn", "nk"):
            X, W, Wkn = _case(gen, m, n, k, layout, 0)
            dY = _mat(gen, m, n).clamp(-2, 2)
            dY[1] *= 1e-38
            dY[:, 3] *= 1e-30
            dY[2] *= 1e34
            dX, dW, db = sgc.linear_backward(dY, X, W, transpose_w=layout == "nk")
            _check(dY, X, Wkn, None, "none", dX, dW.t() if layout == "nk" else dW, db)
