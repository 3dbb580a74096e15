"""The operators of an FP32 feed-forward block and of its training step, as cases
that can be timed.

    linear       Y = act(X W + b) + R, and Z = X W + b where the training step keeps it
    linear_grad  from dY: dZ = dY * act'(Z); dX = dZ W^T, dW = X^T dZ, db = sums of dZ's columns
    norm         layer norm of rows, with each row's mean and 1 / standard deviation
    norm_grad    from dY: dX, and the gradients of the norm's weight and bias
    adamw        an AdamW step over all tensors of a model, states in 32 or in 8 bits

Each case is one call (adamw in 8 bits: a step, then the states' values as a
checkpoint writes them) of the package's public functions where `own` is true,
and the same mathematics in elementary torch operations, in 32 bits, where it is
false.  The listed sizes are those of this repository's workloads and tests
(workloads.py, cases.py: 1, 48, 777 to 8192 rows, 4096 and 8192 columns, odd and
ragged ones) and ordinary widths of feed-forward blocks; draw() gives others of
the same ranges.

    layout  "kn": W is K x N;  "nk": W is N x K, its rows the outputs
    pad     extra elements between the rows of X (a view of a wider matrix)
    dtype   of a norm's X and Y, or of the gradients that adamw reads
"""
import math

import torch

own = False

ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")
DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
EPS_NORM = 1e-5
ADAMW = {"lr": 1e-3, "beta1": 0.9, "beta2": 0.95, "eps": 1e-8, "weight_decay": 0.1, "step": 7}
GRAD_SCALE = 0.125  # the gradients carry a loss scale of 8
BLOCK = 256         # values that share a scale in 8-bit states


def _linear(name, m, n, k, activation, layout="kn", bias=True, residual=False, keep=False, pad=0):
    return {"name": name, "op": "linear", "m": m, "n": n, "k": k, "activation": activation,
            "layout": layout, "bias": bias, "residual": residual, "keep": keep, "pad": pad}


def _linear_grad(name, m, n, k, activation, layout="kn", pad=0):
    return {"name": name, "op": "linear_grad", "m": m, "n": n, "k": k, "activation": activation,
            "layout": layout, "pad": pad}


def _norm(name, op, m, n, dtype="float32", pad=0):
    return {"name": name, "op": op, "m": m, "n": n, "dtype": dtype, "pad": pad}


def _adamw(name, hidden, inner, layers, bits, dtype="float32"):
    return {"name": name, "op": "adamw", "hidden": hidden, "inner": inner, "layers": layers,
            "bits": bits, "dtype": dtype}


def listed():
    return [
        # One token through the first product of a block: latency, and the weights' bytes.
        _linear("linear_token", 1, 8192, 4096, "silu", layout="nk"),
        # A serving step's rows through the second product, with the block's residual.
        _linear("linear_serve48", 48, 4096, 4096, "none", residual=True),
        # The first product of a training step, which keeps Z for its gradient.
        _linear("linear_train8192", 8192, 8192, 4096, "gelu", keep=True),
        # A ragged small gradient: rows and columns that end inside every tile.
        _linear_grad("linear_grad_ragged777", 777, 1003, 530, "relu", layout="nk", pad=3),
        # The gradient of an ordinary training step.
        _linear_grad("linear_grad_train8192", 8192, 4096, 4096, "gelu_tanh"),
        # A serving step's rows.
        _norm("norm_serve48", "norm", 48, 4096, "float16"),
        # A training step's rows.
        _norm("norm_train16384", "norm", 16384, 4096),
        # Odd rows of odd length, not aligned to anything.
        _norm("norm_grad_ragged3001", "norm_grad", 3001, 1531, pad=2),
        _norm("norm_grad_train16384", "norm_grad", 16384, 4096, "bfloat16"),
        # A small model of odd widths: 48 tensors, where launches count.
        _adamw("adamw_small200", 200, 1000, 8, 32),
        # A training step's update, with states in 32 bits and in 8.
        _adamw("adamw_train4096", 4096, 8192, 3, 32, "bfloat16"),
        _adamw("adamw8_train1024", 1024, 4096, 16, 8),
    ]


def _size(rng, low, high):
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    if v > 96 and rng.random() < 0.5:
        v = max(64, v // 64 * 64)
    return v - 1 if v == 3072 else v


def draw(rng):
    op = rng.choice(["linear", "linear", "linear", "linear_grad", "linear_grad", "norm",
                     "norm_grad", "adamw"])
    pad = rng.choice([0, 0, 0, 4, 1])
    if op in ("linear", "linear_grad"):
        while True:
            m = _size(rng, 1, 16384) if rng.random() < 0.7 else _size(rng, 1, 128)
            n, k = _size(rng, 64, 8192), _size(rng, 64, 8192)
            if m * n * k <= 2 ** (37 if op == "linear" else 36) and n * k >= 2**14:
                break
        case = {"op": op, "m": m, "n": n, "k": k, "activation": rng.choice(ACTIVATIONS),
                "layout": rng.choice(["kn", "nk"]), "pad": pad}
        if op == "linear":
            case.update(bias=rng.random() < 0.7, residual=rng.random() < 0.4,
                        keep=m > 64 and rng.random() < 0.5)
        return case
    if op == "adamw":
        while True:
            hidden, inner = _size(rng, 64, 4096), _size(rng, 128, 16384)
            layers = rng.randint(1, 24)
            if 2**14 <= 2 * hidden * inner * layers <= 2**27:
                break
        return {"op": op, "hidden": hidden, "inner": inner, "layers": layers,
                "bits": rng.choice([8, 32]), "dtype": rng.choice(list(DTYPES))}
    while True:
        m, n = _size(rng, 1, 32768), _size(rng, 64, 16384)
        if 2**12 <= m * n <= 2**26:
            break
    return {"op": op, "m": m, "n": n, "dtype": rng.choice(list(DTYPES)), "pad": pad}


# --- inputs -------------------------------------------------------------------

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1000003 + 29)
    return gen


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _padded(x, pad):
    if not pad:
        return x
    wide = torch.zeros((x.shape[0], x.shape[1] + pad), dtype=x.dtype, device="cuda")
    wide[:, :x.shape[1]].copy_(x)
    return wide[:, :x.shape[1]]


def _activations(gen, m, k):
    """Rows as a norm leaves them, with a few strong features."""
    x = _normal(gen, m, k)
    return x.mul_(1.0 + 7.0 * (torch.rand(k, generator=gen, device="cuda") < 0.01))


def _gradients(gen, m, n):
    """Small gradients whose size differs from row to row; some rows are masked out of the loss."""
    rows = torch.exp(1.5 * _normal(gen, m, 1)).mul_(1e-5)
    rows.mul_(torch.rand((m, 1), generator=gen, device="cuda") > 0.1)
    return _normal(gen, m, n).mul_(rows)


def _prepare_linear(case, gen):
    m, n, k = case["m"], case["n"], case["k"]
    state = {"X": _padded(_activations(gen, m, k), case["pad"]),
             "W": _normal(gen, *((n, k) if case["layout"] == "nk" else (k, n))).div_(math.sqrt(k))}
    if case["op"] == "linear":
        state["bias"] = _normal(gen, n).mul_(0.1) if case["bias"] else None
        state["residual"] = _normal(gen, m, n) if case["residual"] else None
    else:
        state["dY"] = _gradients(gen, m, n)
        state["Z"] = None if case["activation"] == "none" else _normal(gen, m, n)
    return state


def _prepare_norm(case, gen):
    m, n, dtype = case["m"], case["n"], DTYPES[case["dtype"]]
    x = _normal(gen, m, n).mul_(0.5 + torch.rand((m, 1), generator=gen, device="cuda"))
    x.add_(_normal(gen, n).mul_(0.3))
    x = _padded(x.to(dtype), case["pad"])
    state = {"x": x, "weight": 1.0 + 0.1 * _normal(gen, n), "bias": 0.1 * _normal(gen, n)}
    if case["op"] == "norm_grad":
        state["dy"] = _gradients(gen, m, n).mul_(1e3).to(dtype)
        x = x.float()
        state["mean"] = x.mean(dim=1)
        var = (x - state["mean"][:, None]).square_().mean(dim=1)
        state["rstd"] = torch.rsqrt(var + EPS_NORM)
    return state


def _shapes(case):
    h, f = case["hidden"], case["inner"]
    return [(h,), (h,), (h, f), (f,), (f, h), (h,)] * case["layers"]


def _views(flat, shapes):
    """Tensors of these shapes in one buffer, each at the start of a block."""
    got, at = [], 0
    for shape in shapes:
        n = math.prod(shape)
        got.append(flat[at:at + n].view(shape))
        at += -(-n // BLOCK) * BLOCK
    return got


def _prepare_adamw(case, gen):
    shapes = _shapes(case)
    sizes = [math.prod(s) for s in shapes]
    blocks = [-(-n // BLOCK) for n in sizes]
    total = sum(blocks) * BLOCK
    used = torch.zeros(total, device="cuda")
    for view in _views(used, [(n,) for n in sizes]):
        view.fill_(1.0)
    # Every tenth block of gradients and states is zero: rows that no token has reached.
    live = torch.rand((total // BLOCK, 1), generator=gen, device="cuda") > 0.1
    used = used.view(-1, BLOCK).mul_(live).view(-1)
    g = _normal(gen, total).mul_(used).mul_(8e-3).to(DTYPES[case["dtype"]])
    m = _normal(gen, total).mul_(used).mul_(3e-4)
    v = _normal(gen, total).mul_(used).mul_(1e-3).square_()
    p = _normal(gen, total).mul_(0.02)
    # Matrices decay, vectors do not.
    decay = [ADAMW["weight_decay"] if len(s) == 2 else 0.0 for s in shapes]
    kept = torch.tensor([1.0 - ADAMW["lr"] * d for d in decay], device="cuda")
    kept = torch.repeat_interleave(kept, torch.tensor(blocks, device="cuda")).view(-1, 1)
    state = {"p": p, "g": g, "shapes": shapes, "decay": decay, "kept_of_block": kept}
    if case["bits"] == 8:
        state["m"], state["m_scale"] = _encode_m(m.view(-1, BLOCK))
        state["v"], state["v_scale"] = _encode_v(v.view(-1, BLOCK))
        # What the states stand for is written here.
        state["m_values"], state["v_values"] = torch.empty_like(p), torch.empty_like(p)
    else:
        state["m"], state["v"] = m, v
    return state


def prepare(case, seed):
    gen = _generator(seed)
    if case["op"] == "adamw":
        state = _prepare_adamw(case, gen)
    elif case["op"] in ("norm", "norm_grad"):
        state = _prepare_norm(case, gen)
    else:
        state = _prepare_linear(case, gen)
    state["case"] = dict(case)
    return state


# --- the plain forms ----------------------------------------------------------

_TANH_C = math.sqrt(2.0 / math.pi)


def _act(z, activation):
    if activation == "relu":
        return torch.where(z > 0, z, 0.0)
    if activation == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if activation == "gelu_tanh":
        return z / (1.0 + torch.exp(-2.0 * _TANH_C * (z + 0.044715 * z * z * z)))
    if activation == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_grad(z, activation):
    if activation == "relu":
        return torch.where(z > 0, 1.0, 0.0)
    if activation == "gelu":
        density = torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * density
    u2 = z if activation == "silu" else 2.0 * _TANH_C * (z + 0.044715 * z * z * z)
    du2 = 1.0 if activation == "silu" else 2.0 * _TANH_C * (1.0 + 3.0 * 0.044715 * z * z)
    s = 1.0 / (1.0 + torch.exp(-u2))
    return s + z * s * (1.0 - s) * du2


def _plain_linear(state, case):
    W = state["W"].t() if case["layout"] == "nk" else state["W"]
    z = state["X"] @ W
    if state["bias"] is not None:
        z = z + state["bias"]
    y = _act(z, case["activation"])
    if state["residual"] is not None:
        y = y + state["residual"]
    return (y, z) if case["keep"] else y


def _plain_linear_grad(state, case):
    dz = state["dY"]
    if state["Z"] is not None:
        dz = dz * _act_grad(state["Z"], case["activation"])
    if case["layout"] == "nk":
        return dz @ state["W"], dz.t() @ state["X"], dz.sum(dim=0)
    return dz @ state["W"].t(), state["X"].t() @ dz, dz.sum(dim=0)


def _plain_norm(state):
    x = state["x"].float()
    mean = x.mean(dim=1)
    centred = x - mean[:, None]
    rstd = torch.rsqrt((centred * centred).mean(dim=1) + EPS_NORM)
    y = centred * rstd[:, None] * state["weight"] + state["bias"]
    return y.to(state["x"].dtype), mean, rstd


def _plain_norm_grad(state):
    x, dy = state["x"].float(), state["dy"].float()
    rstd = state["rstd"][:, None]
    hat = (x - state["mean"][:, None]) * rstd
    wdy = dy * state["weight"]
    dx = rstd * (wdy - wdy.mean(dim=1, keepdim=True) - hat * (wdy * hat).mean(dim=1, keepdim=True))
    return dx.to(state["x"].dtype), (dy * hat).sum(dim=0), dy.sum(dim=0)


def _ratio(x, scale):
    return torch.where(scale > 0, x / scale, 0.0)


def _encode_m(m):
    """Blocks of m in 8 bits: the block's largest magnitude times (c / 127) |c / 127|."""
    scale = m.abs().amax(dim=1, keepdim=True)
    c = torch.round(torch.sqrt(_ratio(m.abs(), scale)) * 127.0)
    return (torch.sign(m) * c).to(torch.int8), scale


def _encode_v(v):
    """Blocks of v in 8 bits: the block's largest value times (c / 255)^4; no positive value is 0."""
    scale = v.amax(dim=1, keepdim=True)
    c = torch.round(torch.sqrt(torch.sqrt(_ratio(v, scale))) * 255.0)
    return torch.where(v > 0, torch.clamp(c, min=1.0), c).to(torch.uint8), scale


def _decode_m(c, scale):
    x = c.float() * (1.0 / 127.0)
    return (x * x.abs()) * scale


def _decode_v(c, scale):
    x = c.float() * (1.0 / 255.0)
    x = x * x
    return (x * x) * scale


def _plain_adamw(state, case):
    h = ADAMW
    correct1 = 1.0 - h["beta1"] ** h["step"]
    correct2 = 1.0 / math.sqrt(1.0 - h["beta2"] ** h["step"])
    p, g = state["p"].view(-1, BLOCK), state["g"].float().view(-1, BLOCK) * GRAD_SCALE
    if case["bits"] == 8:
        m, v = _decode_m(state["m"], state["m_scale"]), _decode_v(state["v"], state["v_scale"])
    else:
        m, v = state["m"].view(-1, BLOCK), state["v"].view(-1, BLOCK)
    m = h["beta1"] * m + (1.0 - h["beta1"]) * g
    v = h["beta2"] * v + (1.0 - h["beta2"]) * (g * g)
    update = m / (torch.sqrt(v) * correct2 + h["eps"])
    p.copy_(p * state["kept_of_block"] - (h["lr"] / correct1) * update)
    if case["bits"] != 8:
        state["m"].view(-1, BLOCK).copy_(m)
        state["v"].view(-1, BLOCK).copy_(v)
        return state["p"], state["m"], state["v"]
    m_codes, m_scale = _encode_m(m)
    v_codes, v_scale = _encode_v(v)
    state["m"].copy_(m_codes)
    state["m_scale"].copy_(m_scale)
    state["v"].copy_(v_codes)
    state["v_scale"].copy_(v_scale)
    state["m_values"].view(-1, BLOCK).copy_(_decode_m(state["m"], state["m_scale"]))
    state["v_values"].view(-1, BLOCK).copy_(_decode_v(state["v"], state["v_scale"]))
    return state["p"], state["m_values"], state["v_values"]


# --- the framework's operators ------------------------------------------------

def _own_linear(sgc, state, case):
    return sgc.linear(state["X"], state["W"], bias=state["bias"], residual=state["residual"],
                      activation=case["activation"], transpose_w=case["layout"] == "nk",
                      keep_preact=case["keep"])


def _own_linear_grad(sgc, state, case):
    return sgc.linear_backward(state["dY"], state["X"], state["W"], preact=state["Z"],
                               activation=case["activation"],
                               transpose_w=case["layout"] == "nk")


def _own_adamw(sgc, state, case):
    opt = state.get("optimizer")
    if opt is None:
        # A program makes its optimizer once, over the tensors it trains.
        h, shapes = ADAMW, state["shapes"]
        sizes = [(math.prod(s),) for s in shapes]
        states = {"exp_avgs": _views(state["m"].view(-1), sizes),
                  "exp_avg_sqs": _views(state["v"].view(-1), sizes)}
        if case["bits"] == 8:
            blocks = [-(-n // BLOCK) for n, in sizes]
            states["exp_avg_scales"] = list(torch.split(state["m_scale"].view(-1), blocks))
            states["exp_avg_sq_scales"] = list(torch.split(state["v_scale"].view(-1), blocks))
            state["values"] = (_views(state["m_values"], sizes), _views(state["v_values"], sizes))
        opt = sgc.AdamW(_views(state["p"], shapes), lr=h["lr"], betas=(h["beta1"], h["beta2"]),
                        eps=h["eps"], weight_decay=state["decay"], state_bits=case["bits"],
                        states=states)
        state["optimizer"], state["grads"] = opt, _views(state["g"], shapes)
    opt.step(state["grads"], step=ADAMW["step"], grad_scale=GRAD_SCALE)
    if case["bits"] != 8:
        return state["p"], state["m"], state["v"]
    opt.state_values(out=state["values"])
    return state["p"], state["m_values"], state["v_values"]


def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        import paper_2507_23387_amd as sgc

        if op == "linear":
            return _own_linear(sgc, state, case)
        if op == "linear_grad":
            return _own_linear_grad(sgc, state, case)
        if op == "norm":
            return sgc.layer_norm(state["x"], state["weight"], state["bias"], eps=EPS_NORM,
                                  keep_stats=True)
        if op == "norm_grad":
            return sgc.layer_norm_backward(state["dy"], state["x"], state["weight"],
                                           state["mean"], state["rstd"])
        return _own_adamw(sgc, state, case)
    if op == "linear":
        return _plain_linear(state, case)
    if op == "linear_grad":
        return _plain_linear_grad(state, case)
    if op == "norm":
        return _plain_norm(state)
    if op == "norm_grad":
        return _plain_norm_grad(state)
    return _plain_adamw(state, case)


# --- what a pass has to move and compute ---------------------------------------

def work(case):
    op = case["op"]
    if op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        outputs = 1 + case["keep"] + case["residual"]
        return {"bytes": 4.0 * (m * k + k * n + outputs * m * n + case["bias"] * n),
                "flops": 2.0 * m * n * k}
    if op == "linear_grad":
        m, n, k = case["m"], case["n"], case["k"]
        inputs = 1 if case["activation"] == "none" else 2
        return {"bytes": 4.0 * (2 * m * k + 2 * k * n + inputs * m * n + n),
                "flops": 4.0 * m * n * k}
    if op == "adamw":
        n = sum(math.prod(s) for s in _shapes(case))
        grad = DTYPES[case["dtype"]].itemsize
        # 8 bits: both states read and written in a byte, and their values written.
        states = 16.0 if case["bits"] == 32 else 4.0 + 8.0 + 16.0 / BLOCK
        return {"bytes": n * (8.0 + grad + states), "flops": 14.0 * n}
    m, n, size = case["m"], case["n"], DTYPES[case["dtype"]].itemsize
    if op == "norm":
        return {"bytes": 2.0 * size * m * n + 8.0 * (m + n), "flops": 7.0 * m * n}
    return {"bytes": 3.0 * size * m * n + 8.0 * m + 12.0 * n, "flops": 13.0 * m * n}


# --- the definitions in 64 bits -------------------------------------------------

def _exact_act(z, activation, grad):
    if activation == "none":
        return torch.ones_like(z) if grad else z
    if activation == "relu":
        return (z > 0).double() if grad else z.clamp(min=0)
    if activation == "gelu":
        phi = torch.special.ndtr(z)
        return phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi) if grad else z * phi
    if activation == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s)) if grad else z * s
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (z + 0.044715 * z**3))
    if not grad:
        return z * (1 + t) / 2
    return (1 + t) / 2 + z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z) / 2


def _exact_adamw(state, case):
    h, t = ADAMW, ADAMW["step"]
    rows = lambda x: x.double().reshape(-1, BLOCK)  # noqa: E731
    p, g = rows(state["p"]), rows(state["g"]) * GRAD_SCALE
    m, v = rows(state["m"]), rows(state["v"])
    if case["bits"] == 8:
        m = m * m.abs() / 127**2 * state["m_scale"].double()
        v = (v / 255) ** 4 * state["v_scale"].double()
    m += (1 - h["beta1"]) * (g - m)
    v += (1 - h["beta2"]) * (g**2 - v)
    step = h["lr"] / (1 - h["beta1"] ** t) * m / ((v / (1 - h["beta2"] ** t)).sqrt() + h["eps"])
    p = state["kept_of_block"].double() * p - step
    if case["bits"] == 8:
        top = m.abs().amax(1, keepdim=True).clamp(min=1e-300)
        code = ((m.abs() / top) ** 0.5 * 127).round()
        m = m.sign() * (code / 127) ** 2 * top
        top = v.amax(1, keepdim=True).clamp(min=1e-300)
        code = ((v / top) ** 0.25 * 255).round().clamp(min=1)
        v = torch.where(v > 0, (code / 255) ** 4 * top, v)
    return p.reshape(-1), m.reshape(-1), v.reshape(-1)


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "adamw":
        return _exact_adamw(state, case)
    if op in ("linear", "linear_grad"):
        X, W = state["X"].double(), state["W"].double()
        W = W.t().contiguous() if case["layout"] == "nk" else W
        if op == "linear":
            z = torch.mm(X, W)
            z = z if state["bias"] is None else z.add_(state["bias"].double())
            y = _exact_act(z, case["activation"], False)
            y = y if state["residual"] is None else y + state["residual"].double()
            return (y, z) if case["keep"] else y
        dz = state["dY"].double()
        if state["Z"] is not None:
            dz = dz * _exact_act(state["Z"].double(), case["activation"], True)
        dW = torch.mm(X.t().contiguous(), dz)
        return (torch.mm(dz, W.t().contiguous()), dW.t() if case["layout"] == "nk" else dW,
                dz.sum(0))
    x, w = state["x"].double(), state["weight"].double()
    if op == "norm":
        mean, var = x.mean(1), x.var(1, unbiased=False)
        y = (x - mean[:, None]) / (var[:, None] + EPS_NORM).sqrt() * w + state["bias"].double()
        return y, mean, 1 / (var + EPS_NORM).sqrt()
    dy, rstd = state["dy"].double(), state["rstd"].double()[:, None]
    hat = (x - state["mean"].double()[:, None]) * rstd
    share = (dy * w).sum(1, keepdim=True) + hat * (dy * w * hat).sum(1, keepdim=True)
    return rstd * (dy * w - share / x.shape[1]), (dy * hat).sum(0), dy.sum(0)
