"""AdamW over many tensors, states in 32 and in 8 bits.

The 32-bit step is compared with the formulas in 64 bits.  Every operation is
rounded once, u = 2^-24: m and v are sums of two products (3 u of their terms'
magnitudes), the update a quotient of such (at most 12 u of its magnitude where
m does not cancel, so m's error counts through |terms of m|), and p one product
less another.  The 8-bit step is held to the same definition in 32-bit
operations bit for bit on the CPU, and its codes to half a code of the 64-bit
state they stand for (one where rounding to 32 bits moves a tie)."""
import math

import pytest
import torch

from tests.gpu_util import log

pytestmark = pytest.mark.gpu

U = 2.0**-24
HYPER = dict(lr=1e-3, betas=(0.9, 0.95), eps=1e-8)
SIZES = [1, 3, 4, 5, 63, 255, 256, 257, 1000, 1023, 1024, 1025, 4095, 4097, 20000]


def _inputs(gen, sizes, dtype):
    dev = dict(generator=gen, device="cuda")
    p = [torch.randn(n, **dev) * 0.02 for n in sizes]
    g = [(torch.randn(n, **dev) * 1e-2).to(dtype) for n in sizes]
    m = [torch.randn(n, **dev) * 1e-3 for n in sizes]
    v = [(torch.randn(n, **dev) * 1e-3)**2 for n in sizes]
    return p, g, m, v


def _step64(p, g, m, v, decay, step, scale):
    (b1, b2), lr, eps = HYPER["betas"], HYPER["lr"], HYPER["eps"]
    p, g, m, v = (x.double().cpu() for x in (p, g, m, v))
    g = g * scale
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    den = torch.sqrt(v1) / math.sqrt(1 - b2**step) + eps
    size = lr / (1 - b1**step)
    terms = (b1 * m).abs() + ((1 - b1) * g).abs()
    tol_m, tol_v = 4 * U * terms, 6 * U * v1
    p1 = p * (1 - lr * decay) - size * m1 / den
    tol_p = 3 * U * p.abs() + size * (tol_m + 12 * U * m1.abs()) / den + U * p1.abs()
    return p1, m1, v1, tol_p, tol_m, tol_v


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
def test_step_32_bits(gpu, dtype):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(21)
    sizes = SIZES * 8  # more tensors than one launch takes
    p, g, m, v = _inputs(gen, sizes, getattr(torch, dtype))
    g[4].zero_(), m[4].zero_(), v[4].zero_()
    decay = [0.1 * (i % 3) for i in range(len(sizes))]
    before = [[x.clone() for x in xs] for xs in (p, m, v)]
    log(f"adamw 32 bits, {len(sizes)} tensors, {dtype}")
    opt = sgc.AdamW(p, weight_decay=decay, states={"exp_avgs": m, "exp_avg_sqs": v}, step=6, **HYPER)
    opt.step(g, grad_scale=0.25)
    assert opt.steps == 7
    for i in range(len(sizes)):
        p1, m1, v1, tp, tm, tv = _step64(before[0][i], g[i], before[1][i], before[2][i], decay[i],
                                         7, 0.25)
        # Values below 2^-126 lose bits by their own type: 2^-149 at most.
        tiny = 2.0**-148
        assert torch.all((p[i].double().cpu() - p1).abs() <= tp + tiny), i
        assert torch.all((m[i].double().cpu() - m1).abs() <= tm + tiny), i
        assert torch.all((v[i].double().cpu() - v1).abs() <= tv + tiny), i
    assert torch.equal(p[4].cpu(), (before[0][4] * (1 - 1e-3 * decay[4])).cpu())


def _sqrt(x):
    """Rounded once: torch's own square root on the CPU can be a unit off."""
    return torch.sqrt(x.double()).float()


def _f32(x):
    return torch.tensor(x, dtype=torch.float32)


def _decode(mc, ms, vc, vs):
    x = mc.float() * _f32(1 / 127.0)
    y = vc.float() * _f32(1 / 255.0)
    y = y * y
    return (x * x.abs()) * ms, (y * y) * vs


def _encode(m, v):
    ms, vs = m.abs().amax(1, keepdim=True), v.amax(1, keepdim=True)
    rm = torch.where(ms > 0, m.abs() / ms, 0.0)
    rv = torch.where(vs > 0, v / vs, 0.0)
    mc = torch.sign(m) * torch.round(_sqrt(rm) * 127)
    vc = torch.round(_sqrt(_sqrt(rv)) * 255)
    return mc, ms, torch.where(v > 0, vc.clamp(min=1), vc), vs


def _blocks(x):
    n = x.numel()
    out = torch.zeros(-(-n // 256) * 256, dtype=x.dtype)
    out[:n] = x.cpu()
    return out.view(-1, 256)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_step_8_bits(gpu, dtype):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(22)
    p, g, m, v = _inputs(gen, SIZES, getattr(torch, dtype))
    g[7].zero_(), m[7].zero_(), v[7].zero_()
    g[8][256:512] = 0  # a block that no gradient reaches
    states = {k: [] for k in ("exp_avgs", "exp_avg_sqs", "exp_avg_scales", "exp_avg_sq_scales")}
    for i, n in enumerate(SIZES):
        mb, vb = _blocks(m[i]), _blocks(v[i])
        if i == 8:
            mb[1] = vb[1] = 0
        mc, ms, vc, vs = _encode(mb, vb)
        for key, x, t in (("exp_avgs", mc, torch.int8), ("exp_avg_sqs", vc, torch.uint8)):
            states[key].append(x.view(-1)[:n].to(t).cuda())
        states["exp_avg_scales"].append(ms.view(-1).cuda())
        states["exp_avg_sq_scales"].append(vs.view(-1).cuda())
    before = {k: [x.cpu().clone() for x in xs] for k, xs in states.items()}
    p0 = [x.cpu().clone() for x in p]
    log(f"adamw 8 bits {dtype}")
    opt = sgc.AdamW(p, weight_decay=0.1, state_bits=8, states=states, **HYPER)
    opt.step(g, step=3, grad_scale=0.5)
    values = opt.state_values()
    (b1, b2), lr, eps = HYPER["betas"], HYPER["lr"], HYPER["eps"]
    for i, n in enumerate(SIZES):
        m0, v0 = _decode(_blocks(before["exp_avgs"][i]), before["exp_avg_scales"][i][:, None],
                         _blocks(before["exp_avg_sqs"][i]), before["exp_avg_sq_scales"][i][:, None])
        gs = _blocks(g[i].float()) * _f32(0.5)
        m1 = _f32(b1) * m0 + _f32(1 - b1) * gs
        v1 = _f32(b2) * v0 + _f32(1 - b2) * (gs * gs)
        den = _sqrt(v1) * _f32(1 / math.sqrt(1 - b2**3)) + _f32(eps)
        p1 = _blocks(p0[i]) * _f32(1 - lr * 0.1) - _f32(lr / (1 - b1**3)) * (m1 / den)
        mc, ms, vc, vs = _encode(m1, v1)
        flat = lambda x: x.view(-1)[:n]  # noqa: E731
        assert torch.equal(p[i].cpu(), flat(p1)), i
        assert torch.equal(states["exp_avg_scales"][i].cpu(), ms[:, 0]), i
        assert torch.equal(states["exp_avg_sq_scales"][i].cpu(), vs[:, 0]), i
        assert torch.equal(states["exp_avgs"][i].cpu(), flat(mc).to(torch.int8)), i
        assert torch.equal(states["exp_avg_sqs"][i].cpu(), flat(vc).to(torch.uint8)), i
        mv, vv = _decode(mc, ms, vc, vs)
        assert torch.equal(values[0][i].cpu(), flat(mv)) and torch.equal(values[1][i].cpu(), flat(vv))
        # The codes stand for the 64-bit state to half a code, up to a tie.
        m64 = b1 * m0.double() + (1 - b1) * gs.double()
        root = torch.sqrt(m64.abs() / m64.abs().amax(1, keepdim=True).clamp(min=1e-300)) * 127
        assert torch.all((root - mc.abs().double()).abs() <= 0.5 + 1e-4)
        assert torch.all((flat(vc) > 0) == (flat(v1) > 0))


def test_8_bits_zero_state_then_steps(gpu):
    """From zero states; a value that has been seen never divides by eps alone."""
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(23)
    p = [torch.zeros(1000, device="cuda")]
    opt = sgc.AdamW(p, lr=1e-2, weight_decay=0.0, state_bits=8)
    sizes = 10.0 ** torch.linspace(-7, 0, 1000, device="cuda")  # seven decades in a block
    for _ in range(20):
        opt.step([torch.randn(1000, generator=gen, device="cuda") * sizes])
    assert opt.steps == 20 and torch.isfinite(p[0]).all()
    # |update| <= lr times about 1 a step, and where v's code is rounded up less.
    assert p[0].abs().max().item() <= 20 * 1e-2 * 4


def test_nonfinite_gradients_stay_in_their_place(gpu):
    import paper_2507_23387_amd as sgc

    for bits in (32, 8):
        p = [torch.ones(1000, device="cuda")]
        opt = sgc.AdamW(p, state_bits=bits, weight_decay=0.0)
        g = torch.ones(1000, device="cuda")
        g[300] = float("nan")
        g[600] = float("inf")
        opt.step([g])
        bad = torch.zeros(1000, dtype=torch.bool, device="cuda")
        bad[300] = bad[600] = True
        # inf: m = inf, v = inf, m / sqrt(v) = NaN
        assert torch.equal(torch.isnan(p[0]), bad)
        m, v = opt.state_values()
        if bits == 32:
            assert torch.equal(torch.isfinite(m[0]), ~bad)
        else:
            bad[256:768] = True  # the blocks of both
            assert torch.equal(torch.isnan(m[0]), bad) and torch.equal(torch.isnan(v[0]), bad)


@pytest.mark.parametrize("bits", [32, 8])
def test_views_at_odd_addresses(gpu, bits):
    """Tensors that start anywhere in a buffer, beside others' values."""
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(24)
    n = 3000
    flat = torch.randn(n + 8, generator=gen, device="cuda")
    grad = torch.randn(n + 8, generator=gen, device="cuda").half()
    results = []
    for at in (0, 1, 2, 3, 5):
        p = [torch.full((n + 8,), 7.0, device="cuda")[at:at + n]]
        p[0].copy_(flat[:n])
        base = p[0]._base
        g = torch.zeros(n + 8, dtype=torch.half, device="cuda")[at:at + n]
        g.copy_(grad[:n])
        types = (torch.float32, torch.float32) if bits == 32 else (torch.int8, torch.uint8)
        m, v = (torch.zeros(n + 8, dtype=t, device="cuda") for t in types)
        states = {"exp_avgs": [m[at:at + n]], "exp_avg_sqs": [v[at:at + n]]}
        if bits == 8:
            states["exp_avg_scales"] = [torch.zeros(12, device="cuda")]
            states["exp_avg_sq_scales"] = [torch.zeros(12, device="cuda")]
        opt = sgc.AdamW(p, state_bits=bits, states=states)
        opt.step([g])
        opt.step([g])
        out = tuple([torch.full((n + 8,), 7.0, device="cuda")[at:at + n]] for _ in range(2))
        opt.state_values(out=out)
        results.append((p[0].clone(), *(o[0].clone() for o in out)))
        for whole in (base, out[0][0]._base, out[1][0]._base):
            assert torch.all(whole[:at] == 7.0) and torch.all(whole[at + n:] == 7.0)
        assert not m[:at].any() and not m[at + n:].any() and not v[at + n:].any()
    for r in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], r))


def test_empty_and_refused(gpu):
    import paper_2507_23387_amd as sgc

    f = lambda n, **k: torch.zeros(n, device="cuda", **k)  # noqa: E731
    sgc.AdamW([]).step([])
    opt = sgc.AdamW([f(0), f(5), f(0)])
    opt.step([f(0), torch.ones(5, device="cuda"), f(0)])
    assert (opt.params[1] != 0).all()
    p = [f(8)]
    with pytest.raises(TypeError):
        sgc.AdamW([f(8, dtype=torch.float16)])
    with pytest.raises(TypeError):
        sgc.AdamW([torch.zeros(8)])
    with pytest.raises(TypeError):
        sgc.AdamW(p).step([f(8, dtype=torch.float64)])
    with pytest.raises(TypeError):
        sgc.AdamW([f(8), f(8)]).step([f(8), f(8, dtype=torch.float16)])
    for bad in (lambda: sgc.AdamW(p, state_bits=16), lambda: sgc.AdamW(p, weight_decay=[0.1, 0.2]),
                lambda: sgc.AdamW([f(16)[::2]]), lambda: sgc.AdamW(p).step([]),
                lambda: sgc.AdamW(p).step([f(9)]), lambda: sgc.AdamW(p).step([f(16)[::2]]),
                lambda: sgc.AdamW(p, states={"exp_avgs": [f(8)]}),
                lambda: sgc.AdamW(p, states={"exp_avgs": [f(8)], "exp_avg_sqs": [f(7)]})):
        with pytest.raises(ValueError):
            bad()
    for kw in (dict(lr=float("nan")), dict(eps=-1.0), dict(betas=(1.0, 0.9)),
               dict(betas=(0.9, -0.1)), dict(weight_decay=float("inf"))):
        with pytest.raises(sgc.SgemmCubeError):
            sgc.AdamW(p, **kw).step([f(8)])
    with pytest.raises(sgc.SgemmCubeError):
        sgc.AdamW(p).step([f(8)], step=0)
    with pytest.raises(sgc.SgemmCubeError):  # the gradient is the parameter
        sgc.AdamW(p).step(p)
    shared = f(12)
    with pytest.raises(sgc.SgemmCubeError):
        sgc.AdamW(p, states={"exp_avgs": [shared[:8]], "exp_avg_sqs": [shared[4:]]}).step([f(8)])


def test_exchanged_memory_is_refused(gpu):
    import paper_2507_23387_amd as sgc

    p, g = [torch.zeros(8, device="cuda") for _ in range(2)], [torch.ones(8, device="cuda")] * 2
    opt = sgc.AdamW(p)
    opt.step(g)
    before = p[0].clone()
    p[1].data = torch.zeros(8, device="cuda")
    with pytest.raises(ValueError, match="memory"):
        opt.step(g)
    assert torch.equal(p[0], before) and opt.steps == 1
    with pytest.raises(TypeError):
        opt.states["exp_avgs"] = []


def test_graph(gpu):
    import paper_2507_23387_amd as sgc

    gen = torch.Generator(device="cuda")
    gen.manual_seed(25)
    g = [torch.randn(n, generator=gen, device="cuda") for n in SIZES]
    for bits in (32, 8):
        a, b = ([torch.ones(n, device="cuda") for n in SIZES] for _ in range(2))
        held, eager = sgc.AdamW(a, state_bits=bits), sgc.AdamW(b, state_bits=bits)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held.step(g, step=1)
        for _ in range(3):
            graph.replay()
            eager.step(g, step=1)
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(a, b))
