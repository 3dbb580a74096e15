"""The gated linear layer and its gradients against their definitions in 64 bits.

Bounds, u = 2^-24, with the product's of test_gpu_linear.py for G and U (t_g, t_u):
Y       |U| (1.13 t_g + 16 u |G|) + |act(G)| t_u + 1.13 t_g t_u + u |Y|.
dU      its activation's 16 u |G| of |dY| and the product's rounding; dG 16 u (1 + |G|) of
        |dY U| and two roundings.
dX, dW  the products', D's own through the other operand, D's floor of 2^-38 of its line's
        largest magnitude, and for dX u of each of the two products that it adds."""
import math

import pytest
import torch

from tests.gpu_util import log
from tests.test_gpu_linear import ACTS, ORDERS, SHAPES, U, _act64, _case, _mat, _product64

pytestmark = pytest.mark.gpu


def _weights(gen, m, n, k, layout, pad):
    X, Wg, Wgkn = _case(gen, m, n, k, layout, pad)
    _, Wu, Wukn = _case(gen, 1, n, k, layout, 0 if pad == 3 else pad)
    return X, (Wg, Wu), (Wgkn, Wukn)


def _check_forward(X, Wkn, biases, act, Y, G=None, Up=None):
    z, tol = [], []
    for W, b, got in zip(Wkn, biases, (G, Up)):
        P, t = _product64(X, W)
        v = P if b is None else P + b.double()
        t = t + 2 * U * (v.abs() + P.abs())
        if got is not None:
            worst = ((got.double() - v).abs() - t).max().item()
            assert worst <= 0, f"G or U past the bound by {worst:.3e}"
        z.append(v)
        tol.append(t)
    a = _act64(act, z[0])
    y = a * z[1]
    bound = (z[1].abs() * (1.13 * tol[0] + 16 * U * z[0].abs()) + a.abs() * tol[1]
             + 1.13 * tol[0] * tol[1] + U * y.abs() + 2.0**-126)
    worst = ((Y.double() - y).abs() - bound).max().item()
    assert worst <= 0, f"Y past the bound by {worst:.3e}"


def _check_backward(dY, X, Wkn, G, Up, act, nk, grads):
    dX, dWg, dWu, dbg, dbu = grads
    d, g, u = dY.double(), G.double(), Up.double()
    D = (d * u * _act64(act, g, grad=True), d * _act64(act, g))
    off = ((d * u).abs() * 16 * U * (1 + g.abs()) + 3 * U * D[0].abs(),
           d.abs() * 16 * U * g.abs() + 2 * U * D[1].abs())
    Xt = X.double().t().contiguous()
    if dX is not None:
        want, bound = 0.0, 0.0
        top = torch.maximum(*(e.abs().amax(1, keepdim=True) for e in D))
        for e, o, W in zip(D, off, Wkn):
            Wt = W.double().t().contiguous()
            part, t = _product64(e, Wt)
            want = want + part
            bound = (bound + t + (o + 2.0**-38 * top) @ Wt.abs() + 2 * U * (e.abs() @ Wt.abs()))
        worst = ((dX.double() - want).abs() - bound - 2.0**-126).max().item()
        assert worst <= 0, f"dX past the bound by {worst:.3e}"
    for name, got, e, o in (("dW_gate", dWg, D[0], off[0]), ("dW_up", dWu, D[1], off[1])):
        if got is None:
            continue
        want, bound = _product64(Xt, e)
        floor = 2.0**-38 * Xt.abs().sum(1)[:, None] * e.abs().amax(0, keepdim=True)
        bound = bound + Xt.abs() @ o + floor + U * want.abs() + 2.0**-126
        got = got.double().t() if nk else got.double()
        worst = ((got - want).abs() - bound).max().item()
        assert worst <= 0, f"{name} past the bound by {worst:.3e}"
    for got, e, o in ((dbg, D[0], off[0]), (dbu, D[1], off[1])):
        if got is None:
            continue
        bound = (min(e.shape[0], 1024) + 8) * U * e.abs().sum(0) + o.sum(0) + 2.0**-126
        assert torch.all((got.double() - e.sum(0)).abs() <= bound)


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("layout", ["kn", "nk"])
def test_forward(gpu, order, layout):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(91)
    for i, (m, n, k) in enumerate(SHAPES):
        act, pad = ACTS[i % 5], (0, 3, 4)[i % 3]
        log(f"gated_linear {order} {layout} {m}x{n}x{k} {act} pad {pad}")
        X, W, Wkn = _weights(gen, m, n, k, layout, pad)
        b = [_mat(gen, 1, n)[0] if (i + j) % 4 != 1 else None for j in range(2)]
        kw = dict(bias_gate=b[0], bias_up=b[1], activation=act, transpose_w=layout == "nk",
                  order=order)
        Y, G, Up = sgc.gated_linear(X, *W, keep_preact=True, **kw)
        _check_forward(X, Wkn, b, act, Y, G, Up)
        assert torch.equal(sgc.gated_linear(X, *W, **kw), Y)  # the same bits without G and U
        out = _mat(gen, m, n, 5)
        assert sgc.gated_linear(X, *W, out=out, **kw) is out
        wide = out._base if out._base is not None else out
        assert torch.equal(out, Y) and torch.isnan(wide[:, n:]).all()


@pytest.mark.parametrize("act", ACTS)
def test_every_activation(gpu, act):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(92)
    for m, n, k in ((1, 512, 64), (20, 512, 64), (200, 500, 64), (4200, 4300, 64)):
        for layout in ("kn", "nk"):
            X, W, Wkn = _weights(gen, m, n, k, layout, 0)
            X.mul_(torch.logspace(-4, 1.3, m, device="cuda")[:, None])
            b = [_mat(gen, 1, n)[0], None]
            kw = dict(activation=act, transpose_w=layout == "nk")
            Y, G, Up = sgc.gated_linear(X, *W, bias_gate=b[0], keep_preact=True, **kw)
            _check_forward(X, Wkn, b, act, Y, G, Up)
            dY = _mat(gen, m, n)
            grads = sgc.gated_linear_backward(dY, X, *W, G, Up, **kw)
            _check_backward(dY, X, Wkn, G, Up, act, layout == "nk", grads)


def test_halves_of_one_matrix(gpu):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(93)
    for m, n, k in ((1, 300, 130), (40, 520, 260), (300, 260, 130), (2100, 4100, 70)):
        X = _mat(gen, m, k)
        both = _mat(gen, k, 2 * n, 0, 1 / math.sqrt(k))
        Y = sgc.gated_linear(X, both[:, :n], both[:, n:])
        _check_forward(X, (both[:, :n], both[:, n:]), (None, None), "silu", Y)
        rows = both.t().contiguous()
        Y = sgc.gated_linear(X, rows[:n], rows[n:], transpose_w=True)
        _check_forward(X, (both[:, :n], both[:, n:]), (None, None), "silu", Y)
        same = sgc.gated_linear(X, rows[:n], rows[:n], transpose_w=True, activation="none")
        z = sgc.gated_linear(X, rows[:n], rows[:n], transpose_w=True, keep_preact=True)[1]
        assert torch.equal(same, z * z)


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("layout", ["kn", "nk"])
def test_backward(gpu, order, layout):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(94)
    names = ("dX", "dW_gate", "dW_up", "db_gate", "db_up")
    for i, (m, n, k) in enumerate(SHAPES):
        act, pad = ACTS[(i + 1) % 5], (3, 0, 4)[i % 3]
        log(f"gated_linear_backward {order} {layout} {m}x{n}x{k} {act} pad {pad}")
        X, W, Wkn = _weights(gen, m, n, k, layout, pad)
        # Rows that differ by six decades, some masked out.
        rows = torch.logspace(-9, -3, m, device="cuda")[:, None]
        rows[m // 3: m // 2] = 0
        dY, G, Up = _mat(gen, m, n, pad) * rows, _mat(gen, m, n, pad), _mat(gen, m, n, 4 - pad)
        kw = dict(activation=act, transpose_w=layout == "nk", order=order)
        grads = sgc.gated_linear_backward(dY, X, *W, G, Up, **kw)
        _check_backward(dY, X, Wkn, G, Up, act, layout == "nk", grads)
        for need in ((names[i % 5],), (names[(i + 1) % 5], names[(i + 3) % 5])):
            only = sgc.gated_linear_backward(dY, X, *W, G, Up, need=need, **kw)
            for name, a, b in zip(names, only, grads):
                assert (a is None) if name not in need else torch.equal(a, b)


@pytest.mark.parametrize("act", ACTS)
def test_backward_against_differences(gpu, act):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(95)
    m, n, k = 23, 41, 37
    X, W, _ = _weights(gen, m, n, k, "kn", 0)
    b, dY = [_mat(gen, 1, n)[0] for _ in range(2)], _mat(gen, m, n)
    Y, G, Up = sgc.gated_linear(X, *W, *b, activation=act, keep_preact=True)
    if act == "relu":
        dY = dY * (G.abs() > 1e-3)
    grads = sgc.gated_linear_backward(dY, X, *W, G, Up, act)
    h = 1e-6
    for which, grad in enumerate(grads):
        E = torch.randn(grad.shape, generator=gen, device="cuda", dtype=torch.float64)
        ends = []
        for sign in (h, -h):
            x, wg, wu, bg, bu = (t.double() + (sign * E if j == which else 0)
                                 for j, t in enumerate((X, *W, *b)))
            ends.append((_act64(act, x @ wg + bg) * (x @ wu + bu) * dY.double()).sum().item())
        want = (ends[0] - ends[1]) / (2 * h)
        got = (grad.double() * E).sum().item()
        assert abs(got - want) <= 2e-6 * (grad.double() * E).abs().sum().item()


@pytest.mark.parametrize("m,n,k", [(3, 500, 130), (20, 1301, 1303), (100, 1500, 1400),
                                   (300, 200, 130), (777, 530, 131), (520, 4096, 4090)])
def test_lines_far_apart(gpu, m, n, k):
    """Rows and columns of dY 14 decades apart; a gate that closes whole columns."""
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(96)
    for layout in ("kn", "nk"):
        for rows, cols in ((0, 14), (14, 0), (6, 8)):
            X, W, Wkn = _weights(gen, m, n, k, layout, 0)
            dY = _mat(gen, m, n) * torch.logspace(-rows, 0, m, device="cuda")[:, None]
            dY *= torch.logspace(0, -cols, n, device="cuda")
            G, Up = _mat(gen, m, n), _mat(gen, m, n)
            Up[:, n // 2] = 0
            grads = sgc.gated_linear_backward(dY, X, *W, G, Up, "silu", layout == "nk")
            d, g, u = dY.double(), G.double(), Up.double()
            _check_backward(dY, X, Wkn, G, Up, "silu", layout == "nk", grads)
            assert d.shape == g.shape == u.shape


def test_rows_and_columns_are_apart(gpu):
    """A NaN or an infinity in X stays in its row, in a weight in its column; in dY in its
    row of dX and its column of both dW."""
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(97)
    for m, n, k in ((5, 70, 130), (48, 257, 300), (300, 260, 128), (700, 1100, 520)):
        for layout in ("kn", "nk"):
            t = layout == "nk"
            X, W, _ = _weights(gen, m, n, k, layout, 0)
            dY = _mat(gen, m, n)
            clean, G, Up = sgc.gated_linear(X, *W, transpose_w=t, keep_preact=True)
            grads = sgc.gated_linear_backward(dY, X, *W, G, Up, transpose_w=t)
            dY[4, 5] = float("inf")
            bad = sgc.gated_linear_backward(dY, X, *W, G, Up, transpose_w=t)
            rest = [i for i in range(m) if i != 4]
            assert not torch.isfinite(bad[0][4]).any()
            assert torch.equal(bad[0][rest], grads[0][rest])
            for a, b in zip(bad[1:3], grads[1:3]):
                a, b = (a.t(), b.t()) if t else (a, b)
                assert not torch.isfinite(a[:, 5]).any()
                cols = [j for j in range(n) if j != 5]
                assert torch.equal(a[:, cols], b[:, cols])
            X[3, k - 1] = float("nan")
            X[1, 0] = float("inf")
            (W[1][7] if t else W[1][:, 7])[k // 2] = float("nan")
            Y = sgc.gated_linear(X, *W, transpose_w=t)
            off = torch.zeros((m, n), dtype=torch.bool, device="cuda")
            off[3] = off[1] = True
            off[:, 7] = True
            assert not torch.isfinite(Y[:, 7]).any() and not torch.isfinite(Y[3]).any()
            assert torch.equal(Y[~off], clean[~off])


def test_large_weights(gpu):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(98)
    for m, n, k in ((3, 70, 130), (300, 200, 128), (4200, 4300, 64)):
        X, W, Wkn = _weights(gen, m, n, k, "nk", 0)
        W[1][n // 2] *= 1000.0
        for order in ORDERS:
            kw = dict(transpose_w=True, order=order)
            Y, G, Up = sgc.gated_linear(X, *W, keep_preact=True, **kw)
            _check_forward(X, Wkn, (None, None), "silu", Y, G, Up)
            dY = _mat(gen, m, n)
            grads = sgc.gated_linear_backward(dY, X, *W, G, Up, **kw)
            _check_backward(dY, X, Wkn, G, Up, "silu", True, grads)
            # A scale past what the scaled kernels take, on entries that it fits.
            kw["scale"] = 2.0**16
            args, small = (X / 64, *(w / 64 for w in W)), [w / 64 for w in Wkn]
            Y, G, Up = sgc.gated_linear(*args, keep_preact=True, **kw)
            _check_forward(args[0], small, (None, None), "silu", Y, G, Up)
            grads = sgc.gated_linear_backward(dY, *args, G, Up, **kw)
            _check_backward(dY, args[0], small, G, Up, "silu", True, grads)


def test_empty(gpu):
    import paper_2507_23387_amd as sgc

    f = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    gen = torch.Generator(device="cuda")
    gen.manual_seed(99)
    assert sgc.gated_linear(f(0, 8), f(8, 4), f(8, 4)).shape == (0, 4)
    assert sgc.gated_linear(f(4, 8), f(8, 0), f(8, 0)).shape == (4, 0)
    for m in (1, 70, 300):
        b = [_mat(gen, 1, 9)[0], _mat(gen, 1, 9)[0]]
        Y, G, Up = sgc.gated_linear(f(m, 0), f(0, 9), f(0, 9), *b, keep_preact=True)
        assert torch.equal(G, b[0].expand(m, 9)) and torch.equal(Up, b[1].expand(m, 9))
        _check_forward(f(m, 0), (f(0, 9), f(0, 9)), b, "silu", Y, G, Up)
    got = sgc.gated_linear_backward(f(0, 4), f(0, 8), f(8, 4), f(8, 4), f(0, 4), f(0, 4))
    assert got[0].shape == (0, 8) and all(torch.equal(g, f(*g.shape)) for g in got)
    got = sgc.gated_linear_backward(f(5, 0), f(5, 8), f(8, 0), f(8, 0), f(5, 0), f(5, 0))
    assert torch.equal(got[0], f(5, 8))
    one = f(5, 3) + 1
    got = sgc.gated_linear_backward(one, f(5, 0), f(0, 3), f(0, 3), one, one, "none")
    assert got[0].shape == (5, 0) and got[1].shape == (0, 3)
    assert torch.equal(got[3], f(3) + 5) and torch.equal(got[4], f(3) + 5)
    got = sgc.gated_linear_backward(f(70, 30), _mat(gen, 70, 40), _mat(gen, 40, 30),
                                    _mat(gen, 40, 30), _mat(gen, 70, 30), _mat(gen, 70, 30))
    assert all(torch.equal(g, torch.zeros_like(g)) for g in got)


def test_streams_workspace_and_graph(gpu):
    import paper_2507_23387_amd as sgc
    from paper_2507_23387_amd import binding

    gen = torch.Generator(device="cuda")
    gen.manual_seed(100)
    for m, n, k in ((1, 500, 700), (40, 300, 260), (300, 260, 130), (2100, 2050, 66)):
        X, W, _ = _weights(gen, m, n, k, "kn", 0)
        dY = _mat(gen, m, n)
        size = max(binding.sgemm_cube_gated_linear_workspace_size(m, n, k),
                   binding.sgemm_cube_gated_linear_backward_workspace_size(m, n, k))
        ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")

        def step():
            Y, G, Up = sgc.gated_linear(X, *W, keep_preact=True, workspace=ws)
            return (Y, G, Up, *sgc.gated_linear_backward(dY, X, *W, G, Up, workspace=ws))

        want = step()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(want, other))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = step()
        for _ in range(3):
            X.copy_(_mat(gen, m, k))
            dY.copy_(_mat(gen, m, n) * 1e-6)
            graph.replay()
            torch.cuda.synchronize()
            got = [h.clone() for h in held]
            ws.fill_(255)
            assert all(torch.equal(a, c) for a, c in zip(got, step()))


def test_refused(gpu):
    import paper_2507_23387_amd as sgc

    f = lambda *s, **k: torch.zeros(s, device="cuda", **k)  # noqa: E731
    X, W, Y = f(4, 8), f(8, 6), f(4, 6)
    small = f(16, dtype=torch.uint8)
    back = sgc.gated_linear_backward
    for bad in (lambda: sgc.gated_linear(X.half(), W, W), lambda: sgc.gated_linear(X, W, W.cpu()),
                lambda: sgc.gated_linear(X, W, W, f(6).double()),
                lambda: sgc.gated_linear(X, W, W, out=Y.half()),
                lambda: back(Y.half(), X, W, W, Y, Y), lambda: back(Y, X, W, W, Y, None)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: sgc.gated_linear(X, W, f(8, 5)), lambda: sgc.gated_linear(X, f(7, 6), f(7, 6)),
                lambda: sgc.gated_linear(X, W, W, transpose_w=True),
                lambda: sgc.gated_linear(X, W, W, f(5)), lambda: sgc.gated_linear(X, W, W, None, f(7)),
                lambda: sgc.gated_linear(X, W, W, activation="swish"),
                lambda: sgc.gated_linear(X, W, W, out=f(5, 6)),
                lambda: back(f(4, 5), X, W, W, Y, Y), lambda: back(Y, X, W, W, f(4, 5), Y),
                lambda: back(Y, X, W, W, Y, Y, need=("dW",)),
                lambda: back(Y, X, W, W, Y, Y, workspace=small.cpu())):
        with pytest.raises(ValueError):
            bad()
    wide = f(4, 20)
    for bad in (lambda: sgc.gated_linear(X, W, W, scale=3.0),
                lambda: sgc.gated_linear(X, W, W, order=7),
                lambda: sgc.gated_linear(X, W, W, workspace=small),
                lambda: sgc.gated_linear(wide[:, :8], W, W, out=wide[:, 4:10]),
                lambda: back(Y, X, W, W, Y, Y, scale=0.5),
                lambda: back(Y, X, W, W, Y, Y, workspace=small)):
        with pytest.raises(sgc.SgemmCubeError):
            bad()
