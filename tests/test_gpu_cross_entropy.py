"""The cross entropy over a vocabulary and its gradients against their definitions in 64
bits.

Bounds, u = 2^-24, with the product's of test_gpu_linear.py for the logits (t_ij, and 2 u
of the logit and the product for the bias):
lse     sum p_j t_j from the logits; an exponential exp(z - m) is off by (|z - m| + 2) u for
        its argument's product, |z - m| u for the difference and 2 u for exp2, and where
        sums meet again by as much for the step between their maxima, at most 32 + V / 1024
        meetings and as many additions: u (3 sum p_j |z_j - m| + 8 (32 + V / 1024)); and
        3 u (|lse| + |m|) for the logarithm and the last addition.
loss    lse's, t at the target, and u of the three values.
D       p |c| (t + 3 |z - lse| u + 8 u) for c = dloss + dlse (whose sum is off by u), and
        u (|D| + |dloss|) at the target.
dX, dW  the product's, D's own through |W| or |X|, D's floor of 2^-38 of its line's largest
        magnitude, and 2 u a piece of the vocabulary that dX is added from."""
import math

import pytest
import torch

from tests.gpu_util import log
from tests.test_gpu_linear import ORDERS, U, _case, _mat, _product64

pytestmark = pytest.mark.gpu

IDS = [torch.int64, torch.int32]
# (rows, vocabulary, features)
SHAPES = [(1, 1, 1), (1, 2, 5), (1, 3001, 130), (2, 5000, 64), (3, 257, 65), (5, 1003, 530),
          (16, 4096, 70), (17, 33, 31), (48, 9000, 100), (64, 200, 300), (65, 1030, 65),
          (128, 2500, 190), (129, 255, 64), (300, 130, 70), (300, 200, 1000), (777, 1003, 530),
          (1100, 2100, 70), (2001, 70, 77), (257, 10000, 33), (4100, 4300, 66), (700, 30000, 65),
          (5000, 70, 40), (4, 70000, 33)]
# Several pieces of the vocabulary: 512 MiB of W's planes, or of few rows' logits, a piece;
# of the gradients 1 GiB of W and D.
MANY = [(130, 40000, 8200), (9000, 40000, 20), (20, 40000, 8200), (128, 1100000, 3)]


def _targets(gen, m, v, dtype, kind="some"):
    t = (torch.rand(m, generator=gen, device="cuda", dtype=torch.float64) * v).long().clamp(max=v - 1)
    if kind == "some":
        t[torch.rand(m, generator=gen, device="cuda") < 0.2] = -1
        t[m // 2] = -100
        t[0] = v - 1
    return t.to(dtype)


def _logits(X, Wkn, b):
    P, tol = _product64(X, Wkn)
    z = P if b is None else P + b.double()
    return z, tol + 2 * U * (z.abs() + P.abs()).nan_to_num(posinf=0.0)


def _check_forward(X, Wkn, b, t, loss, lse):
    z, tol = _logits(X, Wkn, b)
    v = z.shape[1]
    top = z.amax(1)
    want = torch.logsumexp(z, 1)
    p = (z - want[:, None]).exp()
    spread = (p * (z - top[:, None]).abs().nan_to_num(posinf=0.0)).sum(1)
    off = ((p * tol).sum(1) * 1.01 + U * (3 * spread + 8 * (32 + v / 1024))
           + 3 * U * (want.abs() + top.abs()))
    worst = ((lse.double() - want).abs() - off).max().item()
    assert worst <= 0, f"lse past the bound by {worst:.3e}"
    at = t.long().clamp(min=0)[:, None]
    zt = z.gather(1, at)[:, 0]
    loss64 = torch.where(t >= 0, want - zt, 0.0)
    off = off + tol.gather(1, at)[:, 0] + U * (want.abs() + zt.abs() + loss64.abs())
    off = torch.where(t >= 0, off, 0.0)
    infinite = loss64.isinf()  # a target that the bias leaves out
    assert torch.equal(loss.double()[infinite], loss64[infinite])
    worst = ((loss.double() - loss64).abs() - off)[~infinite]
    assert worst.numel() == 0 or worst.max() <= 0, f"loss past the bound by {worst.max():.3e}"


def _check_backward(g, h, X, Wkn, b, t, lse, nk, dX, dW, db):
    z, tol = _logits(X, Wkn, b)
    v = z.shape[1]
    live = torch.where(t >= 0, g, 0.0).double()
    c = live if h is None else live + h.double()
    x = z - lse.double()[:, None]
    p = x.exp()
    off = p * c.abs()[:, None] * (1.01 * tol + U * (3 * x.abs().nan_to_num(posinf=0.0) + 8))
    off = off + p * U * c.abs()[:, None]
    D = p * c[:, None]
    at = t.long().clamp(min=0)[:, None]
    D.scatter_add_(1, at, -live[:, None])
    off = off.scatter_add_(1, at, U * (live.abs()[:, None] + D.gather(1, at).abs()))
    if dX is not None:
        Wt = Wkn.double().t().contiguous()
        want, bound = _product64(D, Wt)
        floor = 2.0**-38 * D.abs().amax(1, keepdim=True) * Wt.abs().sum(0)[None, :]
        pieces = 1 + X.shape[0] * v / 2**25
        bound = bound + off @ Wt.abs() + floor + 2 * U * pieces * (D.abs() @ Wt.abs()) + 2.0**-126
        worst = ((dX.double() - want).abs() - bound).max().item()
        assert worst <= 0, f"dX past the bound by {worst:.3e}"
    if dW is not None:
        Xt = X.double().t().contiguous()
        want, bound = _product64(Xt, D)
        floor = 2.0**-38 * Xt.abs().sum(1)[:, None] * D.abs().amax(0, keepdim=True)
        bound = bound + Xt.abs() @ off + floor + U * want.abs() + 2.0**-126
        got = dW.double().t() if nk else dW.double()
        worst = ((got - want).abs() - bound).max().item()
        assert worst <= 0, f"dW past the bound by {worst:.3e}"
    if db is not None:
        bound = (min(D.shape[0], 1024) + 8) * U * D.abs().sum(0) + 1.01 * off.sum(0) + 2.0**-126
        assert torch.all((db.double() - D.sum(0)).abs() <= bound)


def _problem(gen, i, m, v, k, layout):
    X, W, Wkn = _case(gen, m, v, k, layout, (0, 3, 4)[i % 3])
    X.mul_(0.2 + 3.0 * torch.rand((m, 1), generator=gen, device="cuda"))
    b = _mat(gen, 1, v)[0] if i % 3 != 1 else None
    if b is not None and v > 4 and i % 2:
        b[1] = b[v - 2] = -float("inf")
    return X, W, Wkn, b, _targets(gen, m, v, IDS[i % 2])


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("layout", ["kn", "nk"])
def test_forward(gpu, order, layout):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(81)
    for i, (m, v, k) in enumerate(SHAPES + MANY):
        log(f"linear_cross_entropy {order} {layout} {m}x{v}x{k}")
        X, W, Wkn, b, t = _problem(gen, i, m, v, k, layout)
        kw = dict(bias=b, transpose_w=layout == "nk", order=order)
        loss, lse = sgc.linear_cross_entropy(X, W, t, **kw)
        _check_forward(X, Wkn, b, t, loss, lse)
        again = sgc.linear_cross_entropy(X, W, t, **kw)
        assert torch.equal(again[0], loss) and torch.equal(again[1], lse)


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("layout", ["kn", "nk"])
def test_backward(gpu, order, layout):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(82)
    for i, (m, v, k) in enumerate(SHAPES + (MANY if order == "elementwise" else [])):
        log(f"linear_cross_entropy_backward {order} {layout} {m}x{v}x{k}")
        X, W, Wkn, b, t = _problem(gen, i, m, v, k, layout)
        kw = dict(bias=b, transpose_w=layout == "nk", order=order)
        _, lse = sgc.linear_cross_entropy(X, W, t, **kw)
        g = torch.logspace(-9, -2, m, device="cuda")
        h = _mat(gen, 1, m)[0] * 1e-4 if i % 2 else None
        args = (g, X, W, t, lse)
        dX, dW, db = sgc.linear_cross_entropy_backward(*args, dlse=h, **kw)
        _check_backward(g, h, X, Wkn, b, t, lse, layout == "nk", dX, dW, db)
        for n, name in enumerate(("dX", "dW", "db")):
            only = sgc.linear_cross_entropy_backward(*args, dlse=h, need=(name,), **kw)
            assert torch.equal(only[n], (dX, dW, db)[n])
            assert all(o is None for j, o in enumerate(only) if j != n)


def test_backward_against_differences(gpu):
    """<dX, E>, <dW, E>, <db, E> of sum(g loss + 0.01 lse^2) against central differences
    in 64 bits."""
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(83)
    m, v, k = 23, 41, 37
    X, W, _ = _case(gen, m, v, k, "kn", 0)
    b, g, t = _mat(gen, 1, v)[0], _mat(gen, 1, m)[0], _targets(gen, m, v, torch.int64)
    loss, lse = sgc.linear_cross_entropy(X, W, t, bias=b)
    grads = sgc.linear_cross_entropy_backward(g, X, W, t, lse, dlse=0.02 * lse, bias=b)

    def value(x, w, c):
        z = x @ w + c
        l = torch.logsumexp(z, 1)
        per = torch.where(t >= 0, l - z.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0)
        return (per * g.double() + 0.01 * l * l).sum().item()

    h = 1e-5
    for which, grad in enumerate(grads):
        E = torch.randn(grad.shape, generator=gen, device="cuda", dtype=torch.float64)
        ends = []
        for sign in (h, -h):
            at = [X.double(), W.double(), b.double()]
            at[which] = at[which] + sign * E
            ends.append(value(*at))
        want = (ends[0] - ends[1]) / (2 * h)
        got = (grad.double() * E).sum().item()
        assert abs(got - want) <= 4e-6 * (grad.double() * E).abs().sum().item()


@pytest.mark.parametrize("m", [3, 200, 4200])
def test_large_logits_and_certain_rows(gpu, m):
    """Logits of hundreds, where one entry has all of the probability: losses of 0 and of
    hundreds, no overflow."""
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(84)
    v, k = 4300, 66
    X, W, Wkn = _case(gen, m, v, k, "nk", 0)
    t = _targets(gen, m, v, torch.int64, "all")
    X[0] = W[t[0]] * 300
    X[1] = -W[t[1]] * 300
    X[2] = 0
    loss, lse = sgc.linear_cross_entropy(X, W, t, transpose_w=True)
    _check_forward(X, Wkn, None, t, loss, lse)
    assert loss[0] == 0 and loss[1] > 100
    assert abs(loss[2].item() - math.log(v)) < 1e-5
    g = torch.full((m,), 1.0 / m, device="cuda")
    dX, dW, db = sgc.linear_cross_entropy_backward(g, X, W, t, lse, transpose_w=True)
    _check_backward(g, None, X, Wkn, None, t, lse, True, dX, dW, db)


@pytest.mark.parametrize("m,v", [(3, 2500), (150, 700), (4100, 4300)])
def test_left_out_entries_and_rows(gpu, m, v):
    """A bias of -inf; targets past the vocabulary; NaN and infinities in a row; a row whose
    gradients are 0."""
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(85)
    k = 66
    X, W, Wkn = _case(gen, m, v, k, "kn", 0)
    b = _mat(gen, 1, v)[0]
    t = _targets(gen, m, v, torch.int64, "all").clamp(min=v // 2 + 1)
    clean_loss, clean = sgc.linear_cross_entropy(X, W, t, bias=b)
    # All but one entry left out: the loss is 0 there, infinite elsewhere.
    one = torch.full((v,), -float("inf"), device="cuda")
    one[v - 1] = 0.5
    t1 = t.clone()
    t1[0], t1[1] = v - 1, 0
    loss, lse = sgc.linear_cross_entropy(X, W, t1, bias=one)
    _check_forward(X, Wkn, one, t1, loss, lse)
    assert loss[0] == 0 and loss[1] == float("inf")
    g = torch.ones(m, device="cuda")
    dX, dW, db = sgc.linear_cross_entropy_backward(g, X, W, t1, lse, bias=one)
    _check_backward(g, None, X, Wkn, one, t1, lse, False, dX, dW, db)
    # Every entry left out.
    loss, lse = sgc.linear_cross_entropy(X, W, t, bias=torch.full_like(b, -float("inf")))
    assert loss.isnan().all() and (lse == -float("inf")).all()
    # Rows that are not numbers stay by themselves.
    X2, t2 = X.clone(), t.clone()
    X2[1, 3] = float("nan")
    t2[2] = v
    loss, lse = sgc.linear_cross_entropy(X2, W, t2, bias=b)
    assert loss[1].isnan() and lse[1].isnan() and loss[2].isnan() and lse[2] == clean[2]
    keep = torch.arange(m, device="cuda") > 2
    assert torch.equal(loss[keep], clean_loss[keep]) and torch.equal(lse[keep], clean[keep])
    # A row whose target is past the vocabulary has a gradient of NaN, the others their own.
    dX, _, _ = sgc.linear_cross_entropy_backward(g, X, W, t, clean, bias=b)
    dX2, _, db2 = sgc.linear_cross_entropy_backward(g, X, W, t2, clean, bias=b)
    assert dX2[2].isnan().all() and db2.isnan().all()
    assert torch.equal(dX2[keep], dX[keep])
    # Rows left out: by a target or by gradients of 0, whatever their lse.
    t3, g3, lse3 = t.clone(), g.clone(), clean.clone()
    t3[0], g3[1] = -1, 0
    lse3[0] = lse3[1] = float("nan")
    dX3, dW3, db3 = sgc.linear_cross_entropy_backward(g3, X, W, t3, lse3, bias=b)
    assert torch.equal(dX3[:2], torch.zeros_like(dX3[:2]))
    _check_backward(g3, None, X, Wkn, b, t3, torch.where(g3 * (t3 >= 0) > 0, lse3, clean), False,
                    dX3, dW3, db3)


def test_empty(gpu):
    import paper_2507_23387_amd as sgc

    f = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    ids = lambda n, x=0: torch.full((n,), x, device="cuda")  # noqa: E731
    loss, lse = sgc.linear_cross_entropy(f(0, 8), f(8, 4), ids(0))
    assert loss.shape == lse.shape == (0,)
    loss, lse = sgc.linear_cross_entropy(f(3, 8), f(8, 0), torch.tensor([-1, 0, 5], device="cuda"))
    assert (lse == -float("inf")).all() and loss[0] == 0 and loss[1:].isnan().all()
    for m in (2, 300):  # no features: the bias alone
        b = torch.tensor([0.0, 1.0, 2.0], device="cuda")
        loss, lse = sgc.linear_cross_entropy(f(m, 0), f(0, 3), ids(m, 1), bias=b)
        want = torch.logsumexp(b.double(), 0).item()
        assert (lse.double() - want).abs().max() < 1e-6
        assert (loss.double() - (want - 1)).abs().max() < 1e-6
        dX, dW, db = sgc.linear_cross_entropy_backward(f(m) + 1, f(m, 0), f(0, 3), ids(m, 1), lse,
                                                       bias=b)
        p = torch.softmax(b.double(), 0)
        p[1] -= 1
        assert dX.shape == (m, 0) and dW.shape == (0, 3)
        assert (db.double() / m - p).abs().max() < 1e-6
    dX, dW, db = sgc.linear_cross_entropy_backward(f(0), f(0, 8), f(8, 4), ids(0), f(0))
    assert dX.shape == (0, 8) and torch.equal(dW, f(8, 4)) and torch.equal(db, f(4))
    dX, dW, db = sgc.linear_cross_entropy_backward(f(3), f(3, 8), f(8, 0), ids(3, -1), f(3))
    assert torch.equal(dX, f(3, 8)) and dW.shape == (8, 0) and db.shape == (0,)


def test_streams_workspace_and_graph(gpu):
    import paper_2507_23387_amd as sgc
    from paper_2507_23387_amd import binding

    gen = torch.Generator(device="cuda")
    gen.manual_seed(86)
    for m, v, k in ((1, 900, 70), (40, 3000, 100), (300, 2600, 130), (3000, 4200, 64)):
        X, W, _ = _case(gen, m, v, k, "nk", 0)
        t, g = _targets(gen, m, v, torch.int64), torch.rand(m, generator=gen, device="cuda")
        size = max(binding.sgemm_cube_linear_cross_entropy_workspace_size(m, v, k),
                   binding.sgemm_cube_linear_cross_entropy_backward_workspace_size(m, v, k))
        ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")

        def step():
            loss, lse = sgc.linear_cross_entropy(X, W, t, transpose_w=True, workspace=ws)
            return (loss, lse, *sgc.linear_cross_entropy_backward(
                g, X, W, t, lse, transpose_w=True, workspace=ws))

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
            t.copy_(_targets(gen, m, v, torch.int64))
            graph.replay()
            torch.cuda.synchronize()
            got = [h.clone() for h in held]
            ws.fill_(255)
            assert all(torch.equal(a, c) for a, c in zip(got, step()))


def test_large_weights(gpu):
    """Weights past 32, where s B_hi overflows FP16 and the scaled kernels hand over to the
    unscaled ones."""
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(87)
    for m, v, k in ((3, 700, 130), (300, 900, 128), (4200, 4300, 64)):
        X, W, Wkn = _case(gen, m, v, k, "nk", 0)
        W[v // 2] *= 700.0
        X.mul_(0.01)
        t, g = _targets(gen, m, v, torch.int64), torch.ones(m, device="cuda")
        for order in ORDERS:
            log(f"linear_cross_entropy, large weights, {order} {m}x{v}x{k}")
            kw = dict(transpose_w=True, order=order)
            loss, lse = sgc.linear_cross_entropy(X, W, t, **kw)
            _check_forward(X, Wkn, None, t, loss, lse)
            dX, dW, db = sgc.linear_cross_entropy_backward(g, X, W, t, lse, **kw)
            _check_backward(g, None, X, Wkn, None, t, lse, True, dX, dW, db)


@pytest.mark.parametrize("m,v,k", [(3, 700, 130), (300, 900, 128), (260, 9000, 65),
                                   (4200, 4300, 64)])
def test_large_scale(gpu, m, v, k):
    """A scale past what the scaled kernels take, on entries that it fits."""
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(88)
    X, W, Wkn = _case(gen, m, v, k, "nk", 0)
    t, g = _targets(gen, m, v, torch.int64), torch.ones(m, device="cuda")
    for order in ORDERS:
        log(f"linear_cross_entropy, scale 2^16, {order} {m}x{v}x{k}")
        kw = dict(transpose_w=True, order=order, scale=2.0**16)
        loss, lse = sgc.linear_cross_entropy(X, W, t, **kw)
        _check_forward(X, Wkn, None, t, loss, lse)
        dX, dW, db = sgc.linear_cross_entropy_backward(g, X, W, t, lse, **kw)
        _check_backward(g, None, X, Wkn, None, t, lse, True, dX, dW, db)


def test_refused(gpu):
    import paper_2507_23387_amd as sgc

    f = lambda *s, **k: torch.zeros(s, device="cuda", **k)  # noqa: E731
    X, W, t, e = f(4, 8), f(8, 6), f(4, dtype=torch.int64), f(4)
    small = f(16, dtype=torch.uint8)
    back = sgc.linear_cross_entropy_backward
    for bad in (lambda: sgc.linear_cross_entropy(X.half(), W, t),
                lambda: sgc.linear_cross_entropy(X, W.cpu(), t),
                lambda: sgc.linear_cross_entropy(X, W, t.float()),
                lambda: sgc.linear_cross_entropy(X, W, t, bias=f(6).half()),
                lambda: back(e.double(), X, W, t, e), lambda: back(e, X, W, t, e.half()),
                lambda: back(None, X, W, t, e), lambda: back(e, X, W, t, None)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: sgc.linear_cross_entropy(X, W.t(), t),
                lambda: sgc.linear_cross_entropy(X, W, t, transpose_w=True),
                lambda: sgc.linear_cross_entropy(X, W, t[:3]),
                lambda: sgc.linear_cross_entropy(X, W, t, bias=f(5)),
                lambda: back(f(3), X, W, t, e), lambda: back(e, X, W, t, f(5)),
                lambda: back(e, X, W, t, e, dlse=f(2)), lambda: back(e, X, W, t, e, need=("dZ",)),
                lambda: back(e, X, W, t, e, workspace=small.cpu())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: sgc.linear_cross_entropy(X, W, t, scale=3.0),
                lambda: sgc.linear_cross_entropy(X, W, t, order=7),
                lambda: sgc.linear_cross_entropy(X, W, t, workspace=small),
                lambda: back(e, X, W, t, e, scale=0.5), lambda: back(e, X, W, t, e, workspace=small)):
        with pytest.raises(sgc.SgemmCubeError):
            bad()
