"""Layer norm and its gradients against the definition in 64 bits.

Tolerances are worst-case bounds of 32-bit arithmetic, u = 2^-24.  A sum of n
terms whose longest chain of additions is c is off by at most c u times the sum
of magnitudes.  Along a row a thread adds at most n / 64 terms and the rest is a
tree, so c = n / 64 + 32; down a column the kernels' slabs keep c below
min(rows, 1024) + 8.  The result's own type adds half a unit in the last place:
2^-24, 2^-11 or 2^-8 of the value, and 2^-25 where FP16 is subnormal."""
import pytest
import torch

from tests.gpu_util import log

pytestmark = pytest.mark.gpu

U = 2.0**-24
ROUND = {"float32": (2.0**-24, 0.0), "float16": (2.0**-11, 2.0**-25), "bfloat16": (2.0**-8, 0.0)}
SHAPES = [(1, 1), (5, 1), (1, 7), (3, 63), (4, 64), (2, 65), (9, 250), (5, 1000), (130, 1531),
          (48, 4096), (7, 8192), (3, 8200), (2, 16384), (3, 33000), (1030, 130), (5000, 12)]


def _chain(n):
    return n / 64 + 32


def _rows(gen, rows, cols, dtype, pad, offset=0.0):
    wide = torch.full((rows, cols + pad), float("nan"), dtype=dtype, device="cuda")
    x = torch.randn((rows, cols), generator=gen, device="cuda") + offset
    wide[:, :cols] = x.to(dtype)
    return wide[:, :cols]


def _forward64(x, w, b, eps):
    x = x.double().cpu()
    mu = x.mean(1, keepdim=True)
    var = ((x - mu)**2).mean(1, keepdim=True)
    r = 1.0 / torch.sqrt(var + eps)
    y = (x - mu) * r
    if w is not None:
        y = y * w.double().cpu()
    if b is not None:
        y = y + b.double().cpu()
    return y, mu[:, 0], r[:, 0]


def _check_forward(x, w, b, eps, got, mean, rstd):
    n = x.shape[1]
    y64, mu, r = _forward64(x, w, b, eps)
    x64 = x.double().cpu()
    c = _chain(n)
    dmu = c * U * x64.abs().mean(1)
    # Variance: its own sum, and the centred values' error (u of each, and dmu,
    # whose first order vanishes in the sum over the row).
    rel_r = 0.5 * (c + 6) * U + (dmu * r)**2 + dmu * r * 4 * U + 3 * U
    assert torch.all((mean.double().cpu() - mu).abs() <= dmu + U * mu.abs())
    assert torch.all((rstd.double().cpu() - r).abs() <= rel_r * r)
    w64 = torch.ones(n, dtype=torch.float64) if w is None else w.double().cpu()
    hat = ((x64 - mu[:, None]) * r[:, None]).abs()
    tol = w64.abs() * (hat * (rel_r[:, None] + 4 * U) + (dmu * r)[:, None] * (1 + 8 * U))
    rel, least = ROUND[str(x.dtype).removeprefix("torch.")]
    tol = tol + (rel + U) * (y64.abs() + tol) + least
    worst = ((got.double().cpu() - y64).abs() - tol).max().item()
    assert worst <= 0.0, f"past the bound by {worst:.3e}"


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("pad", [0, 3])
def test_forward(gpu, dtype, pad):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(11)
    for rows, cols in SHAPES:
        log(f"layer_norm {dtype} {rows}x{cols} pad {pad}")
        x = _rows(gen, rows, cols, getattr(torch, dtype), pad)
        w = torch.randn(cols, generator=gen, device="cuda")
        b = torch.randn(cols, generator=gen, device="cuda")
        y, mean, rstd = sgc.layer_norm(x, w, b, eps=1e-5, keep_stats=True)
        _check_forward(x, w, b, 1e-5, y, mean, rstd)
        assert torch.equal(sgc.layer_norm(x, w, b), y)
    plain, mean, rstd = sgc.layer_norm(x, keep_stats=True)
    _check_forward(x, None, None, 1e-5, plain, mean, rstd)
    only_b = sgc.layer_norm(x, None, b)
    _check_forward(x, None, b, 1e-5, only_b, mean, rstd)


def test_forward_large_mean_keeps_the_spread(gpu):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(12)
    for cols in (250, 4096, 33000):
        x = _rows(gen, 3, cols, torch.float32, 0, offset=1000.0)
        y, mean, rstd = sgc.layer_norm(x, eps=0.0, keep_stats=True)
        _check_forward(x, None, None, 0.0, y, mean, rstd)


def test_forward_rows_are_apart(gpu):
    """NaN and infinities stay in their rows; constant rows give the bias."""
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(13)
    for cols in (63, 1000, 4096, 40000):
        x = _rows(gen, 6, cols, torch.float32, 0)
        b = torch.randn(cols, generator=gen, device="cuda")
        clean = sgc.layer_norm(x, None, b)
        x[1, cols // 2] = float("nan")
        x[3, cols - 1] = float("inf")
        x[4] = 2.5
        y = sgc.layer_norm(x, None, b)
        assert torch.isnan(y[1]).all() and torch.isnan(y[3]).all()
        assert torch.equal(y[[0, 2, 5]], clean[[0, 2, 5]])
        assert torch.equal(y[4], b)


def test_in_place_and_streams(gpu):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(14)
    for cols in (130, 4096, 40000):
        x = _rows(gen, 37, cols, torch.bfloat16, 5)
        w = torch.randn(cols, generator=gen, device="cuda")
        want, mean, rstd = sgc.layer_norm(x, w, keep_stats=True)
        dy = _rows(gen, 37, cols, torch.bfloat16, 2)
        want_grad = sgc.layer_norm_backward(dy, x, w, mean, rstd)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = sgc.layer_norm_backward(dy, x, w, mean, rstd)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(want_grad, other))
        got = sgc.layer_norm_backward(dy, x, w, mean, rstd, out=dy)
        assert got[0] is dy and all(torch.equal(a, c) for a, c in zip(want_grad, got))
        assert sgc.layer_norm(x, w, out=x) is x
        assert torch.equal(x, want)


def _backward64(dy, x, w, mean, rstd):
    dy, x = dy.double().cpu(), x.double().cpu()
    w = torch.ones(x.shape[1], dtype=torch.float64) if w is None else w.double().cpu()
    r = rstd.double().cpu()[:, None]
    h = (x - mean.double().cpu()[:, None]) * r
    g = dy * w
    m1, m2 = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    return r * (g - m1 - h * m2), (dy * h).sum(0), dy.sum(0), (r, h, g, dy)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("pad", [0, 3])
def test_backward(gpu, dtype, pad):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(15)
    for rows, cols in SHAPES:
        log(f"layer_norm_backward {dtype} {rows}x{cols} pad {pad}")
        x = _rows(gen, rows, cols, getattr(torch, dtype), pad)
        dy = _rows(gen, rows, cols, getattr(torch, dtype), pad)
        w = torch.randn(cols, generator=gen, device="cuda") if rows != 5 else None
        _, mean, rstd = sgc.layer_norm(x, w, keep_stats=True)
        dx, dw, db = sgc.layer_norm_backward(dy, x, w, mean, rstd)
        dx64, dw64, db64, (r, h, g, dy64) = _backward64(dy, x, w, mean, rstd)
        c = (_chain(cols) + 8) * U
        tol = r * (c * (g.abs().mean(1, keepdim=True)
                        + h.abs() * (g * h).abs().mean(1, keepdim=True))
                   + 4 * U * (g.abs() + g.abs().mean(1, keepdim=True)
                              + h.abs() * (g * h).abs().mean(1, keepdim=True)))
        rel, least = ROUND[dtype]
        tol = tol + (rel + U) * (dx64.abs() + tol) + least
        assert torch.all((dx.double().cpu() - dx64).abs() <= tol)
        k = (min(rows, 1024) + 8) * U
        assert torch.all((dw.double().cpu() - dw64).abs() <= k * (dy64 * h).abs().sum(0))
        assert torch.all((db.double().cpu() - db64).abs() <= k * dy64.abs().sum(0))


def test_backward_against_differences(gpu):
    """<dX, D> and the weight's and bias's against central differences of the
    forward definition in 64 bits along random directions: the differences' own
    error is about (1e-5)^2 of the third derivative, the gradients' some 1e-6."""
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(16)
    rows, cols = 17, 333
    x = _rows(gen, rows, cols, torch.float32, 0)
    w = torch.randn(cols, generator=gen, device="cuda")
    b = torch.randn(cols, generator=gen, device="cuda")
    dy = _rows(gen, rows, cols, torch.float32, 0)
    _, mean, rstd = sgc.layer_norm(x, w, b, keep_stats=True)
    dx, dw, db = sgc.layer_norm_backward(dy, x, w, mean, rstd)
    rng = torch.Generator()
    rng.manual_seed(17)
    h = 1e-5
    for grad, which in ((dx, 0), (dw, 1), (db, 2)):
        D = torch.randn(grad.shape, generator=rng, dtype=torch.float64)
        loss = []
        for sign in (h, -h):
            at = [x.double().cpu(), w.double().cpu(), b.double().cpu()]
            at[which] = at[which] + sign * D
            loss.append((_forward64(*at, 1e-5)[0] * dy.double().cpu()).sum().item())
        want = (loss[0] - loss[1]) / (2 * h)
        got = (grad.double().cpu() * D).sum().item()
        assert abs(got - want) <= 1e-5 * (grad.double().cpu() * D).abs().sum().item()


def test_empty_and_refused(gpu):
    import paper_2507_23387_amd as sgc

    f = lambda *s, **k: torch.zeros(s, device="cuda", **k)  # noqa: E731
    assert sgc.layer_norm(f(0, 8)).shape == (0, 8)
    y, mean, rstd = sgc.layer_norm(f(3, 0), keep_stats=True)
    assert y.shape == (3, 0) and torch.isnan(mean).all()
    dx, dw, db = sgc.layer_norm_backward(f(0, 8), f(0, 8), None, f(0), f(0))
    assert dx.shape == (0, 8) and torch.equal(dw, f(8)) and torch.equal(db, f(8))
    x = f(4, 8)
    for bad in (lambda: sgc.layer_norm(x.double()), lambda: sgc.layer_norm(x.cpu()),
                lambda: sgc.layer_norm(x, weight=f(8, dtype=torch.float16)),
                lambda: sgc.layer_norm(x, out=f(4, 8, dtype=torch.float16)),
                lambda: sgc.layer_norm_backward(f(4, 8, dtype=torch.float16), x, None, f(4), f(4))):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: sgc.layer_norm(f(8)), lambda: sgc.layer_norm(f(8, 4).t()),
                lambda: sgc.layer_norm(f(1, 8).expand(4, 8)), lambda: sgc.layer_norm(x, f(7)),
                lambda: sgc.layer_norm(x, f(16)[::2]), lambda: sgc.layer_norm(x, out=f(4, 9)),
                lambda: sgc.layer_norm_backward(f(4, 9), x, None, f(4), f(4)),
                lambda: sgc.layer_norm_backward(x, x, None, f(5), f(4))):
        with pytest.raises(ValueError):
            bad()
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(sgc.SgemmCubeError):
            sgc.layer_norm(x, eps=eps)
    wide = f(5, 8)
    with pytest.raises(sgc.SgemmCubeError):  # rows that overlap the input's
        sgc.layer_norm(wide[:4], out=wide[1:])


def test_graph(gpu):
    """Captured calls replay with the eager bits, new inputs in the same memory."""
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(18)
    x, dy = _rows(gen, 300, 2050, torch.float32, 0), _rows(gen, 300, 2050, torch.float32, 0)
    w = torch.randn(2050, generator=gen, device="cuda")

    def step():
        y, mean, rstd = sgc.layer_norm(x, w, keep_stats=True)
        return (y, *sgc.layer_norm_backward(dy, x, w, mean, rstd))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(3):
        x.copy_(torch.randn(x.shape, generator=gen, device="cuda"))
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(held, want))


def test_same_bits_each_time(gpu):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(19)
    x, dy = _rows(gen, 3001, 700, torch.float16, 1), _rows(gen, 3001, 700, torch.float16, 1)
    _, mean, rstd = sgc.layer_norm(x, keep_stats=True)
    first = sgc.layer_norm_backward(dy, x, None, mean, rstd)
    for _ in range(5):
        again = sgc.layer_norm_backward(dy, x, None, mean, rstd)
        assert all(torch.equal(a, c) for a, c in zip(first, again))
