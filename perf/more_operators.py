"""The two ends of a language model and the gated form of its feed-forward block,
as cases that can be timed.

    embed       y_i = scale * W[id_i], zeros for a negative id (no token)
    embed_grad  dW_v = scale * sum of dy_i over the i with id_i = v: a new dW, zeros where
                no id is, or (add) added to the dW that a tied output layer's gradient left
    xent        z = X W + b; per row lse = log(sum_j exp z_j), loss = lse - z_t, 0 for a
                negative target (a row that is left out)
    xent_grad   from dloss (and dlse, of a penalty on lse): D = p (dloss + dlse) - [j = t] dloss
                with p = exp(z - lse); dX = D W^T, dW = X^T D, db = sums of D's columns
    gated       G = X Wg + bg, U = X Wu + bu, Y = act(G) U; G and U too where the training
                step keeps them
    gated_grad  from dY: dU = dY act(G), dG = dY U act'(G); dX = dG Wg^T + dU Wu^T,
                dWg = X^T dG, dWu = X^T dU, and the sums of dG's and dU's columns

Each case is one call of the package's public functions where `own` is true, and
the same mathematics in elementary torch operations, in 32 bits, where it is false.
The listed sizes are those of this repository's workloads and tests (1, 48, 777 to
16384 rows, 4096 and 8192 columns, 1003 and 530 as ragged ones) with vocabularies of
ordinary sizes; draw() gives others of the same ranges.

    layout  "kn": W is K x N (K x V);  "nk": N x K (V x K), as an embedding table lies
    pad     extra elements between the rows of X or dy (a view of a wider matrix)
    dtype   of the embedding table and its rows, or of dy
    ids     bits of the ids and targets, 32 or 64
"""
import math

import torch

own = False

ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")
DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
IDS = {32: torch.int32, 64: torch.int64}
Z_PENALTY = 1e-4  # of the mean of lse^2


def _embed(name, op, n, vocab, k, dtype="float32", ids=64, pad=0, add=False):
    case = {"name": name, "op": op, "n": n, "vocab": vocab, "k": k, "dtype": dtype, "ids": ids,
            "pad": pad}
    return case if op == "embed" else {**case, "add": add}


def _xent(name, op, m, vocab, k, layout="nk", bias=False, ids=64, pad=0, penalty=False):
    case = {"name": name, "op": op, "m": m, "vocab": vocab, "k": k, "layout": layout,
            "bias": bias, "ids": ids, "pad": pad}
    return case if op == "xent" else {**case, "penalty": penalty}


def _gated(name, op, m, n, k, activation, layout="kn", bias=False, pad=0, keep=False):
    case = {"name": name, "op": op, "m": m, "n": n, "k": k, "activation": activation,
            "layout": layout, "pad": pad}
    return {**case, "bias": bias, "keep": keep} if op == "gated" else case


def listed():
    return [
        # A serving step's tokens: latency.
        _embed("embed_serve48", "embed", 48, 32768, 4096, "float16", ids=32),
        # A training step's tokens.
        _embed("embed_train16384", "embed", 16384, 32768, 4096),
        # A small model of odd sizes, rows not aligned to anything.
        _embed("embed_grad_ragged777", "embed_grad", 777, 1003, 530, pad=3),
        # A training step's tokens, added to the gradient of the tied output layer.
        _embed("embed_grad_train16384", "embed_grad", 16384, 32768, 4096, "bfloat16", add=True),
        # The score of one token: the bytes of the output layer.
        _xent("xent_token", "xent", 1, 32768, 4096),
        # The loss of an evaluation's rows.
        _xent("xent_train4096", "xent", 4096, 65536, 4096),
        # A small model of odd sizes: a few launches of small grids.
        _xent("xent_grad_ragged777", "xent_grad", 777, 1003, 530, layout="kn", bias=True, pad=3),
        # The gradient of an ordinary training step, with the penalty on lse.
        _xent("xent_grad_train4096", "xent_grad", 4096, 32768, 4096, penalty=True),
        # One token through the first half of a gated block: the bytes of both weights.
        _gated("gated_token", "gated", 1, 8192, 4096, "silu", layout="nk"),
        # The same of a training step, which keeps G and U for the gradient.
        _gated("gated_train4096", "gated", 4096, 8192, 4096, "silu", keep=True),
        # A ragged small gradient: rows and columns that end inside every tile.
        _gated("gated_grad_ragged777", "gated_grad", 777, 1003, 530, "gelu_tanh", layout="nk",
               pad=3),
        # The gradient of an ordinary training step.
        _gated("gated_grad_train4096", "gated_grad", 4096, 8192, 4096, "silu"),
    ]


def _size(rng, low, high):
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    return max(64, v // 64 * 64) if v > 96 and rng.random() < 0.5 else v


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "embed_grad", "xent", "xent", "xent_grad", "xent_grad",
                     "gated", "gated", "gated_grad", "gated_grad"])
    pad = rng.choice([0, 0, 0, 4, 1])
    ids = rng.choice([32, 64])
    if op in ("embed", "embed_grad"):
        while True:
            n, vocab, k = _size(rng, 1, 65536), _size(rng, 256, 131072), _size(rng, 64, 8192)
            if n * k <= 2**26 and vocab * k <= 2**28:
                break
        case = {"op": op, "n": n, "vocab": vocab, "k": k, "dtype": rng.choice(list(DTYPES)),
                "ids": ids, "pad": pad}
        return case if op == "embed" else {**case, "add": rng.random() < 0.5}
    layout = rng.choice(["kn", "nk"])
    if op in ("xent", "xent_grad"):
        while True:
            m = _size(rng, 1, 16384) if rng.random() < 0.7 else _size(rng, 1, 128)
            vocab, k = _size(rng, 512, 131072), _size(rng, 64, 8192)
            if (m * vocab * k <= 2 ** (40 if op == "xent" else 38) and m * vocab <= 2**28
                    and vocab * k <= 2**28):
                break
        case = {"op": op, "m": m, "vocab": vocab, "k": k, "layout": layout,
                "bias": rng.random() < 0.3, "ids": ids, "pad": pad}
        return case if op == "xent" else {**case, "penalty": rng.random() < 0.5}
    while True:
        m = _size(rng, 1, 16384) if rng.random() < 0.7 else _size(rng, 1, 128)
        n, k = _size(rng, 64, 16384), _size(rng, 64, 8192)
        if m * n * k <= 2**37 and 2**14 <= n * k <= 2**26:
            break
    case = {"op": op, "m": m, "n": n, "k": k, "activation": rng.choice(ACTIVATIONS),
            "layout": layout, "pad": pad}
    if op == "gated":
        case.update(bias=rng.random() < 0.4, keep=m > 64 and rng.random() < 0.6)
    return case


# --- inputs -------------------------------------------------------------------

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1000003 + 41)
    return gen


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _uniform(gen, *shape):
    return torch.rand(shape, generator=gen, device="cuda")


def _padded(x, pad):
    if not pad:
        return x
    wide = torch.zeros((x.shape[0], x.shape[1] + pad), dtype=x.dtype, device="cuda")
    wide[:, :x.shape[1]].copy_(x)
    return wide[:, :x.shape[1]]


def _tokens(gen, n, vocab, bits):
    """Ids as text has them, the v-th most frequent about 1 / v as often as the first, in no
    order of frequency; one in 16 is a place without a token."""
    rank = torch.exp(_uniform(gen, n).double() * math.log(vocab + 1.0)).long() - 1
    order = torch.randperm(vocab, generator=gen, device="cuda")
    ids = order[rank.clamp_(0, vocab - 1)]
    return torch.where(_uniform(gen, n) < 1 / 16, -1, ids).to(IDS[bits])


def _prepare_embed(case, gen):
    n, vocab, k, dtype = case["n"], case["vocab"], case["k"], DTYPES[case["dtype"]]
    state = {"ids": _tokens(gen, n, vocab, case["ids"]), "scale": math.sqrt(k)}
    if case["op"] == "embed":
        state["W"] = _padded(_normal(gen, vocab, k).mul_(0.02).to(dtype), case["pad"])
        return state
    rows = torch.exp(1.5 * _normal(gen, n, 1)).mul_(1e-2)
    state["dy"] = _padded(_normal(gen, n, k).mul_(rows).to(dtype), case["pad"])
    state["dW"] = _normal(gen, vocab, k).mul_(0.1) if case["add"] else None
    return state


def _prepare_xent(case, gen):
    m, vocab, k = case["m"], case["vocab"], case["k"]
    W = _normal(gen, vocab, k).div_(math.sqrt(k))
    targets = _tokens(gen, m, vocab, case["ids"])
    # Rows as a norm leaves them; a trained model's rows know more or less of their target.
    X = _normal(gen, m, k)
    X.add_(W[targets.long().clamp(min=0)].mul_(16.0 * _uniform(gen, m, 1)))
    state = {"X": _padded(X, case["pad"]), "W": W if case["layout"] == "nk" else W.t().contiguous(),
             "targets": targets, "bias": _normal(gen, vocab).mul_(0.5) if case["bias"] else None}
    if case["op"] == "xent":
        return state
    z = torch.mm(X, W.t())
    if case["bias"]:
        z.add_(state["bias"])
    top = z.amax(dim=1)
    state["lse"] = z.sub_(top[:, None]).exp_().sum(dim=1).log_().add_(top)
    # The mean over the rows that count.
    state["dloss"] = (targets >= 0).float().div_(max(m - m // 16, 1))
    state["dlse"] = state["lse"].mul(2.0 * Z_PENALTY / m) if case["penalty"] else None
    return state


def _prepare_gated(case, gen):
    m, n, k = case["m"], case["n"], case["k"]
    X = _normal(gen, m, k)
    X.mul_(1.0 + 7.0 * (_uniform(gen, k) < 0.01))  # a few strong features
    shape = (n, k) if case["layout"] == "nk" else (k, n)
    state = {"X": _padded(X, case["pad"]), "Wg": _normal(gen, *shape).div_(math.sqrt(k)),
             "Wu": _normal(gen, *shape).div_(math.sqrt(k))}
    if case["op"] == "gated":
        state["bg"], state["bu"] = ((_normal(gen, n).mul_(0.1), _normal(gen, n).mul_(0.1))
                                    if case["bias"] else (None, None))
        return state
    state["G"], state["U"] = _normal(gen, m, n), _normal(gen, m, n)
    # Small gradients whose size differs from row to row; some rows are left out of the loss.
    rows = torch.exp(1.5 * _normal(gen, m, 1)).mul_(1e-5)
    rows.mul_(_uniform(gen, m, 1) > 0.1)
    state["dY"] = _normal(gen, m, n).mul_(rows)
    return state


def prepare(case, seed):
    gen = _generator(seed)
    if case["op"] in ("embed", "embed_grad"):
        state = _prepare_embed(case, gen)
    elif case["op"] in ("xent", "xent_grad"):
        state = _prepare_xent(case, gen)
    else:
        state = _prepare_gated(case, gen)
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
    if activation == "none":
        return torch.ones_like(z)
    if activation == "relu":
        return torch.where(z > 0, 1.0, 0.0)
    if activation == "gelu":
        density = torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * density
    u2 = z if activation == "silu" else 2.0 * _TANH_C * (z + 0.044715 * z * z * z)
    du2 = 1.0 if activation == "silu" else 2.0 * _TANH_C * (1.0 + 3.0 * 0.044715 * z * z)
    s = 1.0 / (1.0 + torch.exp(-u2))
    return s + z * s * (1.0 - s) * du2


def _plain_embed(state):
    ids = state["ids"].long()
    rows = state["W"][ids.clamp(min=0)].float() * state["scale"]
    return torch.where((ids >= 0)[:, None], rows, 0.0).to(state["W"].dtype)


def _plain_embed_grad(state, case):
    ids, scale = state["ids"].long(), state["scale"]
    live = torch.where((ids >= 0)[:, None], state["dy"].float() * scale, 0.0)
    dW = state["dW"]
    if dW is None:
        dW = torch.zeros((case["vocab"], case["k"]), device="cuda")
    return dW.index_add_(0, ids.clamp(min=0), live)


def _logits(state, case):
    W = state["W"].t() if case["layout"] == "nk" else state["W"]
    z = state["X"] @ W
    return z if state["bias"] is None else z + state["bias"]


def _plain_xent(state, case):
    z, targets = _logits(state, case), state["targets"].long()
    at = z.gather(1, targets.clamp(min=0)[:, None])[:, 0]
    top = z.amax(dim=1)
    lse = torch.log(torch.exp(z - top[:, None]).sum(dim=1)) + top
    return torch.where(targets >= 0, lse - at, 0.0), lse


def _plain_xent_grad(state, case):
    targets = state["targets"].long()
    g = torch.where(targets >= 0, state["dloss"], 0.0)
    h = g if state["dlse"] is None else g + state["dlse"]
    D = torch.exp(_logits(state, case) - state["lse"][:, None]) * h[:, None]
    D.scatter_add_(1, targets.clamp(min=0)[:, None], -g[:, None])
    if case["layout"] == "nk":
        return D @ state["W"], D.t() @ state["X"], D.sum(dim=0)
    return D @ state["W"].t(), state["X"].t() @ D, D.sum(dim=0)


def _plain_gated(state, case):
    nk = case["layout"] == "nk"
    G = state["X"] @ (state["Wg"].t() if nk else state["Wg"])
    U = state["X"] @ (state["Wu"].t() if nk else state["Wu"])
    if state["bg"] is not None:
        G, U = G + state["bg"], U + state["bu"]
    Y = _act(G, case["activation"]) * U
    return (Y, G, U) if case["keep"] else Y


def _plain_gated_grad(state, case):
    dY, G, U = state["dY"], state["G"], state["U"]
    dU = dY * _act(G, case["activation"])
    dG = dY * U * _act_grad(G, case["activation"])
    if case["layout"] == "nk":
        dX = dG @ state["Wg"] + dU @ state["Wu"]
        dWg, dWu = dG.t() @ state["X"], dU.t() @ state["X"]
    else:
        dX = dG @ state["Wg"].t() + dU @ state["Wu"].t()
        dWg, dWu = state["X"].t() @ dG, state["X"].t() @ dU
    return dX, dWg, dWu, dG.sum(dim=0), dU.sum(dim=0)


# --- the framework's operators ------------------------------------------------

def _run_own(state, case):
    import paper_2507_23387_amd as sgc

    op = case["op"]
    if op == "embed":
        return sgc.embedding(state["ids"], state["W"], scale=state["scale"])
    if op == "embed_grad":
        return sgc.embedding_backward(state["dy"], state["ids"], case["vocab"],
                                      scale=state["scale"], add_to=state["dW"])
    nk = case["layout"] == "nk"
    if op == "xent":
        return sgc.linear_cross_entropy(state["X"], state["W"], state["targets"],
                                        bias=state["bias"], transpose_w=nk)
    if op == "xent_grad":
        return sgc.linear_cross_entropy_backward(
            state["dloss"], state["X"], state["W"], state["targets"], state["lse"],
            dlse=state["dlse"], bias=state["bias"], transpose_w=nk)
    if op == "gated":
        return sgc.gated_linear(state["X"], state["Wg"], state["Wu"], bias_gate=state["bg"],
                                bias_up=state["bu"], activation=case["activation"],
                                transpose_w=nk, keep_preact=case["keep"])
    return sgc.gated_linear_backward(state["dY"], state["X"], state["Wg"], state["Wu"],
                                     state["G"], state["U"], activation=case["activation"],
                                     transpose_w=nk)


def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        return _run_own(state, case)
    if op == "embed":
        return _plain_embed(state)
    if op == "embed_grad":
        return _plain_embed_grad(state, case)
    if op == "xent":
        return _plain_xent(state, case)
    if op == "xent_grad":
        return _plain_xent_grad(state, case)
    if op == "gated":
        return _plain_gated(state, case)
    return _plain_gated_grad(state, case)


# --- what a pass has to move and compute ---------------------------------------

def _distinct(n, vocab):
    """How many ids n tokens of _tokens' distribution are expected to have."""
    total = math.log(vocab + 1.0)
    rank = torch.arange(vocab, dtype=torch.float64)
    p = torch.log((rank + 2.0) / (rank + 1.0)) / total * (15.0 / 16.0)
    return float((1.0 - torch.exp(n * torch.log1p(-p))).sum())


def work(case):
    op = case["op"]
    if op in ("embed", "embed_grad"):
        n, vocab, k, size = case["n"], case["vocab"], case["k"], DTYPES[case["dtype"]].itemsize
        ids = case["ids"] / 8 * n
        if op == "embed":
            return {"bytes": ids + size * k * (n + _distinct(n, vocab)), "flops": 1.0 * n * k}
        rows = 2.0 * _distinct(n, vocab) if case["add"] else vocab
        return {"bytes": ids + size * n * k + 4.0 * k * rows, "flops": 2.0 * n * k}
    m, k = case["m"], case["k"]
    if op in ("xent", "xent_grad"):
        v = case["vocab"]
        if op == "xent":
            return {"bytes": 4.0 * (m * k + v * k + 3 * m + case["bias"] * v),
                    "flops": 2.0 * m * v * k}
        return {"bytes": 4.0 * (2 * m * k + 2 * v * k + 4 * m + v), "flops": 6.0 * m * v * k}
    n = case["n"]
    if op == "gated":
        return {"bytes": 4.0 * (m * k + 2 * n * k + (1 + 2 * case["keep"]) * m * n
                                + 2 * case["bias"] * n), "flops": 4.0 * m * n * k}
    return {"bytes": 4.0 * (2 * m * k + 4 * n * k + 3 * m * n + 2 * n), "flops": 8.0 * m * n * k}


# --- the definitions in 64 bits -------------------------------------------------

def _exact_act(z, activation, grad=False):
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


def _exact_embed(state, case):
    ids = state["ids"].long()
    live = ids >= 0
    if case["op"] == "embed":
        y = torch.zeros((case["n"], case["k"]), dtype=torch.float64, device="cuda")
        y[live] = state["W"][ids[live]].double() * state["scale"]
        return y
    dW = torch.zeros((case["vocab"], case["k"]), dtype=torch.float64, device="cuda")
    if case["add"]:
        dW += state["dW"]
    return dW.index_put_((ids[live],), state["dy"][live].double() * state["scale"],
                         accumulate=True)


def _exact_xent(state, case):
    t = state["targets"].long()
    live = t >= 0
    X = state["X"].double().contiguous()
    W = state["W"].double()
    W = W.t().contiguous() if case["layout"] == "nk" else W
    z = torch.mm(X, W)
    if state["bias"] is not None:
        z += state["bias"].double()
    rows = torch.arange(case["m"], device="cuda")
    if case["op"] == "xent":
        lse = torch.logsumexp(z, dim=1)
        loss = torch.zeros_like(lse)
        loss[live] = lse[live] - z[rows[live], t[live]]
        return loss, lse
    D = (z - state["lse"].double()[:, None]).exp()
    g = state["dloss"].double() * live
    D *= (g + (0.0 if state["dlse"] is None else state["dlse"].double()))[:, None]
    D[rows[live], t[live]] -= g[live]
    dX, dW = torch.mm(D, W.t().contiguous()), torch.mm(X.t().contiguous(), D)
    return dX, dW.t() if case["layout"] == "nk" else dW, D.sum(0)


def _exact_gated(state, case):
    nk, act = case["layout"] == "nk", case["activation"]
    X = state["X"].double().contiguous()
    Wg, Wu = ((state[w].double().t().contiguous() if nk else state[w].double())
              for w in ("Wg", "Wu"))
    if case["op"] == "gated":
        G, U = torch.mm(X, Wg), torch.mm(X, Wu)
        if state["bg"] is not None:
            G += state["bg"].double()
            U += state["bu"].double()
        Y = U * _exact_act(G, act)
        return (Y, G, U) if case["keep"] else Y
    G, U, dY = (state[x].double() for x in ("G", "U", "dY"))
    dG, dU = dY * _exact_act(G, act, grad=True) * U, dY * _exact_act(G, act)
    dX = torch.mm(dG, Wg.t().contiguous()) + torch.mm(dU, Wu.t().contiguous())
    dWg, dWu = (torch.mm(X.t().contiguous(), d) for d in (dG, dU))
    if nk:
        dWg, dWu = dWg.t(), dWu.t()
    return dX, dWg, dWu, dG.sum(0), dU.sum(0)


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] in ("embed", "embed_grad"):
        return _exact_embed(state, case)
    if case["op"] in ("xent", "xent_grad"):
        return _exact_xent(state, case)
    return _exact_gated(state, case)
