"""The linear layer and its gradients against their definitions in 64 bits.

Tolerances, u = 2^-24.  A split operand is off by 2^-22 of each entry, or by 2^-36
where an entry is below FP16's normal range, and the dropped low-low product by
2^-22 of |A||B|; 3 MFMAs per 32 of k add their products to an accumulator, each
rounded once (partial sums of a split contraction fewer, joined in a tree).  So
  |P - AB| <= (3 2^-21 + (3 K / 32 + 40) u) |A||B| + 2^-35 (rows of |A| + columns of |B|).
Activations: |act'| < 1.13, their own arithmetic some 16 u of |z|; derivatives 16 u
(1 + |z|).  The backward pass multiplies D by a power of two that brings its
largest magnitude to 2^3 at least, so D's floor of 2^-36 is 2^-38 of that."""
import math

import pytest
import torch

from tests.gpu_util import log

pytestmark = pytest.mark.gpu

U = 2.0**-24
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
ORDERS = ["elementwise", "termwise", "elementwise_cross_first"]
# Rows from one to several tiles, columns and k that end inside every piece; the
# last ones fill the larger tiles of each order.
SHAPES = [(1, 1, 1), (1, 7, 3), (1, 300, 1000), (2, 129, 64), (3, 64, 65), (5, 1003, 530),
          (16, 256, 256), (17, 33, 31), (31, 4096, 130), (32, 515, 2049), (33, 130, 4100),
          (48, 1024, 777), (64, 200, 300), (65, 65, 65), (127, 96, 4097), (300, 200, 1000),
          (777, 530, 129), (1100, 2100, 70), (2300, 2050, 66), (4200, 4300, 130),
          (4090, 4091, 70), (4096, 4096, 64), (16300, 1000, 128), (16384, 2048, 64),
          (3, 2100, 2049), (16, 4096, 1030), (300, 1, 65), (1000, 16, 130), (4097, 17, 64),
          (700, 100, 2050), (3001, 128, 70), (1500, 200, 40), (270, 256, 1001), (5000, 3, 33),
          (1, 5003, 65), (20, 4100, 130), (128, 3001, 190),
          (24, 1301, 1303), (25, 1301, 1303), (2, 2050, 1030),
          (65, 4101, 200), (96, 4096, 999), (81, 4100, 1030), (2001, 70, 777), (1990, 96, 333)]


def _act64(name, z, grad=False):
    if name == "none":
        return torch.ones_like(z) if grad else z
    if name == "relu":
        return (z > 0).double() if grad else z.clamp(min=0)
    if name == "gelu":
        phi = torch.special.ndtr(z)
        return phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi) if grad else z * phi
    c, k = math.sqrt(2 / math.pi), 0.044715
    x = z if name == "silu" else 2 * c * (z + k * z**3)
    dx = 1.0 if name == "silu" else 2 * c * (1 + 3 * k * z * z)
    s = torch.sigmoid(x)
    return s + z * s * (1 - s) * dx if grad else z * s


def _mat(gen, rows, cols, pad=0, scale=1.0):
    wide = torch.full((rows, cols + pad), float("nan"), device="cuda")
    wide[:, :cols] = torch.randn((rows, cols), generator=gen, device="cuda") * scale
    return wide[:, :cols]


def _product64(A, B):
    """A B and the product's tolerance."""
    A, B = A.double().contiguous(), B.double().contiguous()
    k = A.shape[1]
    mass = A.abs() @ B.abs()
    tol = (3 * 2.0**-21 + (3 * k / 32 + 40) * U) * mass
    return A @ B, tol + 2.0**-35 * (A.abs().sum(1)[:, None] + B.abs().sum(0)[None, :])


def _case(gen, m, n, k, layout, pad):
    X = _mat(gen, m, k, pad)
    W = _mat(gen, *((n, k) if layout == "nk" else (k, n)), pad, 1 / math.sqrt(k))
    return X, W, (W.t() if layout == "nk" else W)


def _check_forward(X, Wkn, b, R, act, Y, Z):
    P, tol = _product64(X, Wkn)
    z = P if b is None else P + b.double()
    tol = tol + 2 * U * (z.abs() + P.abs())
    if Z is not None:
        assert torch.all((Z.double() - z).abs() <= tol)
    y = _act64(act, z)
    tol = 1.13 * tol + 16 * U * z.abs() + U * y.abs() + 2.0**-126
    if R is not None:
        y = y + R.double()
        tol = tol + U * y.abs()
    worst = ((Y.double() - y).abs() - tol).max().item()
    assert worst <= 0, f"past the bound by {worst:.3e}"


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("layout", ["kn", "nk"])
def test_forward(gpu, order, layout):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(31)
    for i, (m, n, k) in enumerate(SHAPES):
        act, pad = ACTS[i % 5], (0, 3, 4)[i % 3]
        log(f"linear {order} {layout} {m}x{n}x{k} {act} pad {pad}")
        X, W, Wkn = _case(gen, m, n, k, layout, pad)
        b = _mat(gen, 1, n)[0] if i % 4 != 1 else None
        R = _mat(gen, m, n, pad) if i % 4 >= 2 else None
        kw = dict(bias=b, residual=R, activation=act, transpose_w=layout == "nk", order=order)
        Y, Z = sgc.linear(X, W, keep_preact=True, **kw)
        _check_forward(X, Wkn, b, R, act, Y, Z)
        assert torch.equal(sgc.linear(X, W, **kw), Y)  # the same bits without Z
        # Into rows apart, the residual in place.
        out = _mat(gen, m, n, 5)
        if R is not None:
            out.copy_(R)
            kw["residual"] = out
        wide = out._base if out._base is not None else out
        assert sgc.linear(X, W, out=out, **kw) is out
        assert torch.equal(out, Y) and torch.isnan(wide[:, n:]).all()


@pytest.mark.parametrize("act", ACTS)
def test_every_activation(gpu, act):
    """Each at every path, over a wide range of Z."""
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(32)
    for m, n, k in ((1, 512, 64), (20, 512, 64), (200, 500, 64), (4200, 4300, 64)):
        X, W, Wkn = _case(gen, m, n, k, "kn", 0)
        X.mul_(torch.logspace(-4, 1.3, m, device="cuda")[:, None])
        b = _mat(gen, 1, n)[0]
        Y, Z = sgc.linear(X, W, bias=b, activation=act, keep_preact=True)
        _check_forward(X, Wkn, b, None, act, Y, Z)


def test_scales_and_large_weights(gpu):
    """Residual scales from 1 to 2^24, and weights past 32, where s B_hi overflows
    FP16 and the scaled kernels hand over to the unscaled ones."""
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(33)
    for m, n, k in ((3, 70, 130), (300, 200, 128), (4200, 4300, 64)):
        X, W, Wkn = _case(gen, m, n, k, "nk", 0)
        W[n // 2] *= 1000.0
        R = _mat(gen, m, n)
        for order in ORDERS:
            for scale in (2.0**11, 2.0**16):
                log(f"linear {order} {m}x{n}x{k} scale {scale}")
                Y, Z = sgc.linear(X, W, residual=R, activation="silu", transpose_w=True,
                                  keep_preact=True, order=order, scale=scale)
                if scale == 2.0**11:  # Rule 2: 2^16 overflows the residuals of these entries
                    _check_forward(X, Wkn, None, R, "silu", Y, Z)
                else:
                    dY = _mat(gen, m, n)
                    dX, dW, _ = sgc.linear_backward(dY, X / 64, W / 64, Z, "silu", True,
                                                    order=order, scale=2.0**12)
                    _check_backward(dY, X / 64, (W / 64).t(), Z, "silu", True, dX, dW, None)


def test_rows_and_columns_are_apart(gpu):
    """A NaN or an infinity in X stays in its row, in W in its column."""
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(34)
    for m, n, k in ((5, 70, 130), (48, 257, 300), (300, 260, 128)):
        for layout in ("kn", "nk"):
            X, W, _ = _case(gen, m, n, k, layout, 0)
            t = layout == "nk"
            clean = sgc.linear(X, W, transpose_w=t)
            X[3, k - 1] = float("nan")
            X[1, 0] = float("inf")
            col = W[7] if t else W[:, 7]
            col[k // 2] = float("nan")
            Y = sgc.linear(X, W, transpose_w=t)
            bad = torch.zeros((m, n), dtype=torch.bool, device="cuda")
            bad[3] = bad[1] = True
            bad[:, 7] = True
            assert torch.equal(~torch.isfinite(Y), bad)
            assert torch.equal(Y[~bad], clean[~bad])


def test_empty_products(gpu):
    import paper_2507_23387_amd as sgc

    f = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    gen = torch.Generator(device="cuda")
    gen.manual_seed(35)
    assert sgc.linear(f(0, 8), f(8, 4)).shape == (0, 4)
    assert sgc.linear(f(4, 8), f(8, 0)).shape == (4, 0)
    for m in (1, 70, 300):
        b, R = _mat(gen, 1, 9)[0], _mat(gen, m, 9)
        Y, Z = sgc.linear(f(m, 0), f(0, 9), bias=b, residual=R, activation="gelu", keep_preact=True)
        assert torch.equal(Z, b.expand(m, 9))
        _check_forward(f(m, 0), f(0, 9), b, R, "gelu", Y, Z)
    dX, dW, db = sgc.linear_backward(f(0, 4), f(0, 8), f(8, 4))
    assert dX.shape == (0, 8) and torch.equal(dW, f(8, 4)) and torch.equal(db, f(4))
    dX, dW, db = sgc.linear_backward(f(5, 0), f(5, 8), f(8, 0))
    assert torch.equal(dX, f(5, 8)) and dW.shape == (8, 0) and db.shape == (0,)
    dX, dW, db = sgc.linear_backward(torch.ones((5, 3), device="cuda"), f(5, 0), f(0, 3))
    assert dX.shape == (5, 0) and dW.shape == (0, 3) and torch.equal(db, f(3) + 5)
    got = sgc.linear_backward(f(70, 30), _mat(gen, 70, 40), _mat(gen, 40, 30))
    assert all(torch.equal(g, torch.zeros_like(g)) for g in got)  # a gradient of zeros


def _check_backward(dY, X, Wkn, Z, act, transpose_w, dX, dW, db):
    dY64, X64, W64 = dY.double(), X.double().contiguous(), Wkn.double().contiguous()
    z = torch.zeros_like(dY64) if act == "none" else Z.double()
    D = dY64 * _act64(act, z, grad=True)
    off = torch.zeros_like(D) if act == "none" else 16 * U * (1 + z.abs()) * dY64.abs()
    floor = 2.0**-38 * D.abs().max()
    if dX is not None:
        Wt = W64.t().contiguous()
        want, tol = _product64(D, Wt)
        tol = tol + (off + floor) @ Wt.abs() + U * want.abs() + 2.0**-126
        worst = ((dX.double() - want).abs() - tol).max().item()
        assert worst <= 0, f"dX past the bound by {worst:.3e}"
    if dW is not None:
        Xt = X64.t().contiguous()
        want, tol = _product64(Xt, D)
        tol = tol + Xt.abs() @ (off + floor) + U * want.abs() + 2.0**-126
        got = dW.double().t() if transpose_w else dW.double()
        worst = ((got - want).abs() - tol).max().item()
        assert worst <= 0, f"dW past the bound by {worst:.3e}"
    if db is not None:
        tol = (min(D.shape[0], 1024) + 8) * U * D.abs().sum(0) + off.sum(0) + 2.0**-126
        assert torch.all((db.double() - D.sum(0)).abs() <= tol)


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("layout", ["kn", "nk"])
def test_backward(gpu, order, layout):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(36)
    for i, (m, n, k) in enumerate(SHAPES):
        act, pad = ACTS[(i + 1) % 5], (3, 0, 4)[i % 3]
        log(f"linear_backward {order} {layout} {m}x{n}x{k} {act} pad {pad}")
        X, W, Wkn = _case(gen, m, n, k, layout, pad)
        # Rows that differ by six decades, some masked out.
        rows = torch.logspace(-9, -3, m, device="cuda")[:, None]
        rows[m // 3: m // 2] = 0
        dY, Z = _mat(gen, m, n, pad) * rows, _mat(gen, m, n, pad)
        kw = dict(preact=Z, activation=act, transpose_w=layout == "nk", order=order)
        dX, dW, db = sgc.linear_backward(dY, X, W, **kw)
        _check_backward(dY, X, Wkn, Z, act, layout == "nk", dX, dW, db)
        only = sgc.linear_backward(dY, X, W, need=("dX",), **kw)
        assert torch.equal(only[0], dX) and only[1] is None and only[2] is None
        only = sgc.linear_backward(dY, X, W, need=("dW",), **kw)
        assert torch.equal(only[1], dW) and only[0] is None and only[2] is None
        only = sgc.linear_backward(dY, X, W, need=("db",), **kw)
        assert torch.equal(only[2], db) and only[0] is None and only[1] is None


def test_backward_sizes_of_gradients(gpu):
    """From 1e-35 to 1e30, where FP16 holds none of them; an infinity in dY."""
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(37)
    m, n, k = 130, 200, 70
    for size in (1e-35, 1e-20, 1e-7, 1.0, 1e10, 1e30):
        X, W, Wkn = _case(gen, m, n, k, "kn", 0)
        dY, Z = _mat(gen, m, n) * size, _mat(gen, m, n)
        for order in ORDERS:
            dX, dW, db = sgc.linear_backward(dY, X, W, Z, "gelu", order=order)
            _check_backward(dY, X, Wkn, Z, "gelu", False, dX, dW, db)
    clean = dX.clone()
    dY[4, 5] = float("inf")
    dX, dW, db = sgc.linear_backward(dY, X, W, Z, "gelu", order=ORDERS[-1])
    assert not torch.isfinite(dX[4]).any()
    assert torch.equal(torch.cat([dX[:4], dX[5:]]), torch.cat([clean[:4], clean[5:]]))
    assert not torch.isfinite(dW[:, 5]).any() and torch.isfinite(dW[:, :5]).all()
    assert torch.isinf(db[5]) and torch.isfinite(db[:5]).all()


@pytest.mark.parametrize("act", ACTS)
def test_backward_against_differences(gpu, act):
    """<dX, E>, <dW, E>, <db, E> against central differences of the forward
    definition in 64 bits.  Z keeps a distance from relu's corner."""
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(38)
    m, n, k = 23, 41, 37
    X, W, _ = _case(gen, m, n, k, "kn", 0)
    b, dY = _mat(gen, 1, n)[0], _mat(gen, m, n)
    Y, Z = sgc.linear(X, W, bias=b, activation=act, keep_preact=True)
    if act == "relu":
        dY = dY * (Z.abs() > 1e-3)
    grads = sgc.linear_backward(dY, X, W, Z, act)
    h = 1e-6
    for which, grad in enumerate(grads):
        E = torch.randn(grad.shape, generator=gen, device="cuda", dtype=torch.float64)
        loss = []
        for sign in (h, -h):
            at = [X.double(), W.double(), b.double()]
            at[which] = at[which] + sign * E
            loss.append((_act64(act, at[0] @ at[1] + at[2]) * dY.double()).sum().item())
        want = (loss[0] - loss[1]) / (2 * h)
        got = (grad.double() * E).sum().item()
        assert abs(got - want) <= 2e-6 * (grad.double() * E).abs().sum().item()


def test_streams_workspace_and_graph(gpu):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(39)
    for m, n, k in ((1, 500, 700), (40, 300, 260), (300, 260, 130)):
        X, W, _ = _case(gen, m, n, k, "kn", 0)
        b, dY = _mat(gen, 1, n)[0], _mat(gen, m, n)
        ws = torch.full((sgc.layers.binding.sgemm_cube_linear_workspace_size(m, n, k) + 256,), 255,
                        dtype=torch.uint8, device="cuda")  # NaN wherever it is read as it was

        def step():
            Y, Z = sgc.linear(X, W, bias=b, activation="silu", keep_preact=True, workspace=ws)
            return (Y, Z, *sgc.linear_backward(dY, X, W, Z, "silu"))

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
            assert all(torch.equal(a, c) for a, c in zip(got, step()))


def test_refused(gpu):
    import paper_2507_23387_amd as sgc

    f = lambda *s, **k: torch.zeros(s, device="cuda", **k)  # noqa: E731
    X, W, dY = f(4, 8), f(8, 6), f(4, 6)
    for bad in (lambda: sgc.linear(X.half(), W), lambda: sgc.linear(X, W.cpu()),
                lambda: sgc.linear(X, W, bias=f(6).double()),
                lambda: sgc.linear(X, W, residual=f(4, 6).half()),
                lambda: sgc.linear_backward(dY.half(), X, W)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: sgc.linear(X, W.t()), lambda: sgc.linear(X, W, transpose_w=True),
                lambda: sgc.linear(X, f(7, 6)), lambda: sgc.linear(X, W, bias=f(5)),
                lambda: sgc.linear(X, W, residual=f(4, 5)), lambda: sgc.linear(X, W, out=f(5, 6)),
                lambda: sgc.linear(X, W, activation="swish"), lambda: sgc.linear(X[0], W),
                lambda: sgc.linear(f(1, 8).expand(4, 8), W),
                lambda: sgc.linear_backward(f(4, 5), X, W),
                lambda: sgc.linear_backward(dY, X, W, activation="gelu"),
                lambda: sgc.linear_backward(dY, X, W, f(4, 5), activation="gelu"),
                lambda: sgc.linear_backward(dY, X, W, need=("dZ",))):
        with pytest.raises(ValueError):
            bad()
    wide = f(4, 20)
    for bad in (lambda: sgc.linear(X, W, scale=3.0), lambda: sgc.linear(X, W, order=7),
                lambda: sgc.linear(X, W, workspace=f(16, dtype=torch.uint8)),
                lambda: sgc.linear(wide[:, :8], W, out=wide[:, 4:10]),
                lambda: sgc.linear(X, W, residual=wide[:, :6], out=wide[:, 2:8]),
                lambda: sgc.linear_backward(dY, X, W, scale=0.5)):
        with pytest.raises(sgc.SgemmCubeError):
            bad()


def test_workspaces_the_device_cannot_reach_are_refused(gpu):
    import paper_2507_23387_amd as sgc
    from paper_2507_23387_amd import binding

    X, W, dY = (torch.zeros(s, device="cuda") for s in ((4, 8), (8, 6), (4, 6)))
    size = binding.sgemm_cube_linear_backward_workspace_size(4, 6, 8)
    for ws in (torch.zeros(size, dtype=torch.uint8),
               torch.zeros(2 * size, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError):
            sgc.linear(X, W, workspace=ws)
        with pytest.raises(ValueError):
            sgc.linear_backward(dY, X, W, workspace=ws)
