"""The layers around the FP32-accuracy product (include/sgemm_cube_layers.h) on
torch tensors: marshalling only, like binding.py.  Every call checks its
tensors, takes its results and workspace from torch's allocator, enqueues the
library's kernels on the current torch stream and returns; nothing is kept
between calls, and a non-zero status raises SgemmCubeError.  There is no
autograd here: results require no gradient, whatever the operands do, and the
backward functions are called by the program.
"""
from __future__ import annotations

from types import MappingProxyType

import torch

from . import binding
from .binding import _check, _order

_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_F32 = (torch.float32,)
_current_device = torch.cuda.current_device
_address, _count = torch.Tensor.data_ptr, torch.Tensor.numel
_contiguous, _device_of = torch.Tensor.is_contiguous, torch.Tensor.get_device
# The current stream's handle, without the Stream object that wraps it (2.8 us a
# call, of the 10 to 17 that a small layer takes).
_stream = torch._C._cuda_getCurrentRawStream
# Tells autograd of tensors that the library has written to, as torch's own in-place
# operations do, so that a graph which has saved one refuses its old values.
_written = torch.autograd.graph.increment_version


def _refuse(t, name, dtype):
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype not in dtype:
        raise TypeError(f"{name} must be a CUDA/HIP tensor of type "
                        + " or ".join(str(d).removeprefix("torch.") for d in dtype))
    raise ValueError(f"{name} must be on the current device, with the other operands")


def _matrix(t, name, device, shape=None, dtype=_F32):
    """(address, leading dimension) of a 2-D tensor whose columns are adjacent."""
    if not isinstance(t, torch.Tensor) or t.dtype not in dtype or t.get_device() != device:
        _refuse(t, name, dtype)
    got = t.shape
    if len(got) != 2 or (shape is not None and got != shape):
        raise ValueError(f"{name} must be 2-D" if shape is None else
                         f"{name} must have the shape {tuple(shape)}, not {tuple(got)}")
    rows, cols = got
    ld, step = t.stride()
    if (cols > 1 and step != 1) or (rows > 1 and ld < cols):
        raise ValueError(f"{name} must be row-major: unit column stride, rows apart")
    return t.data_ptr(), max(ld if rows > 1 else cols, 1)


def _vector(t, name, device, n):
    """Address of a contiguous FP32 vector of n values, or None."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.dtype not in _F32 or t.get_device() != device:
        _refuse(t, name, _F32)
    if t.shape != (n,) or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{name} must be a contiguous vector of {n} values")
    return t.data_ptr()


def _new(shape, like, dtype=torch.float32):
    return like.new_empty(shape, dtype=dtype)


def _workspace(t, device, need, like):
    """(tensor, address, bytes) of a caller's workspace, or of a new one of `need`
    bytes, which its tensor keeps until the kernels are enqueued."""
    if t is None:
        t = like.new_empty((max(need, 256),), dtype=torch.uint8)
    elif (not isinstance(t, torch.Tensor) or t.get_device() != device or not t.is_contiguous()):
        raise ValueError("workspace must be a contiguous tensor on the current device")
    return t, t.data_ptr(), t.numel() * t.element_size()


def _weight_shape(W, transpose_w):
    """(K, N) of a weight stored as K x N, or as N x K."""
    if W.dim() != 2:
        raise ValueError("W must be 2-D")
    return (W.size(1), W.size(0)) if transpose_w else (W.size(0), W.size(1))


def _activation(name) -> int:
    if name not in binding.ACTIVATIONS:
        raise ValueError(f"activation must be one of {', '.join(binding.ACTIVATIONS)}")
    return binding.ACTIVATIONS[name]


def linear(X, W, bias=None, residual=None, activation: str = "none", transpose_w: bool = False,
           keep_preact: bool = False, scale: float = 2.0**11, order="elementwise", out=None,
           workspace=None):
    """act(X W + bias) + residual at the accuracy of an FP32 product, the sums and
    the epilogue in one pass.  X is M x K, W K x N, or N x K with transpose_w=True.
    activation: none, relu, gelu, gelu_tanh or silu.  With keep_preact=True returns
    (Y, Z), Z = X W + bias, which linear_backward needs of a layer with an
    activation.  residual may be out.  order: of the three products' sums, as for
    matmul, but for few rows or columns, which are summed termwise (up to 128, or 256
    where there are few entries: a row's last bits can change with the batch there).
    workspace: a byte tensor of sgemm_cube_linear_workspace_size bytes that a program
    keeps between calls.  The results are not part of an autograd graph."""
    device = _current_device()
    px, ldx = _matrix(X, "X", device)
    pw, ldw = _matrix(W, "W", device)
    M, K = X.shape
    K2, N = _weight_shape(W, transpose_w)
    if K != K2:
        raise ValueError(f"shape mismatch: X has {K} columns, W takes {K2}")
    pb = _vector(bias, "bias", device, N)
    pr, ldr = (None, N) if residual is None else _matrix(residual, "residual", device, (M, N))
    if out is None:
        Y = X.new_empty((M, N))
        py, ldy = Y.data_ptr(), max(N, 1)
    else:
        Y = out
        py, ldy = _matrix(Y, "out", device, (M, N))
    Z = X.new_empty((M, N)) if keep_preact else None
    held, ws, size = _workspace(workspace, device,
                                binding.sgemm_cube_linear_workspace_size(M, N, K), X)
    _check(binding.sgemm_cube_linear(
        M, N, K, px, ldx, pw, ldw, int(transpose_w), pb, _activation(activation), pr, ldr, py, ldy,
        Z.data_ptr() if keep_preact else None, max(N, 1), scale, _order(order), ws, size,
        _stream(device)), "sgemm_cube_linear")
    if out is not None:
        _written(out)
    return (Y, Z) if keep_preact else Y


_GRADIENTS = ("dX", "dW", "db")


def linear_backward(dY, X, W, preact=None, activation: str = "none", transpose_w: bool = False,
                    need=_GRADIENTS, scale: float = 2.0**11, order="elementwise",
                    workspace=None):
    """(dX, dW, db) of linear at X and W from its output's gradient; preact: the Z
    that it kept, if it has an activation.  dW has W's layout.  What `need` leaves
    out is None.  (The residual's gradient is dY.)  order, workspace: as for linear,
    sgemm_cube_linear_backward_workspace_size bytes."""
    device = _current_device()
    pdy, lddy = _matrix(dY, "dY", device)
    px, ldx = _matrix(X, "X", device)
    pw, ldw = _matrix(W, "W", device)
    M, K = X.shape
    K2, N = _weight_shape(W, transpose_w)
    if K != K2 or dY.shape != (M, N):
        raise ValueError(f"shape mismatch: dY {tuple(dY.shape)}, X {tuple(X.shape)}, "
                         f"W for {K2} x {N}")
    if activation != "none" and preact is None:
        raise ValueError(f"{activation} needs preact, what linear returned with keep_preact=True")
    if need is not _GRADIENTS and not set(need) <= set(_GRADIENTS):
        raise ValueError("need may hold dX, dW and db")
    pz, ldz = (None, N) if activation == "none" else _matrix(preact, "preact", device,
                                                                 (M, N))
    dX = X.new_empty((M, K)) if "dX" in need else None
    dW = X.new_empty(W.shape) if "dW" in need else None
    db = X.new_empty((N,)) if "db" in need else None
    held, ws, size = _workspace(workspace, device,
                                binding.sgemm_cube_linear_backward_workspace_size(M, N, K), X)
    _check(binding.sgemm_cube_linear_backward(
        M, N, K, pdy, lddy, pz, ldz, px, ldx, pw, ldw, int(transpose_w), _activation(activation),
        None if dX is None else dX.data_ptr(), max(K, 1),
        None if dW is None else dW.data_ptr(), max(W.shape[1], 1),
        None if db is None else db.data_ptr(), scale, _order(order), ws, size, _stream(device)),
        "sgemm_cube_linear_backward")
    return dX, dW, db


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, keep_stats: bool = False, out=None):
    """Layer norm of the rows of x (float32, float16 or bfloat16), rounded once to
    x's type; weight and bias are float32.  With keep_stats=True returns
    (y, mean, rstd), what layer_norm_backward needs.  out may be x.  The results are
    not part of an autograd graph."""
    device = _current_device()
    px, ldx = _matrix(x, "x", device, dtype=_DTYPES)
    rows, cols = x.shape
    pw, pb = _vector(weight, "weight", device, cols), _vector(bias, "bias", device, cols)
    if out is None:
        y = _new((rows, cols), x, x.dtype)
        py, ldy = y.data_ptr(), max(cols, 1)
    else:
        y = out
        py, ldy = _matrix(y, "out", device, x.shape, (x.dtype,))
    mean, rstd = _new((2, rows), x) if keep_stats else (None, None)
    _check(binding.sgemm_cube_layer_norm(
        rows, cols, _DTYPES[x.dtype], px, ldx, pw, pb, eps, py, ldy,
        mean.data_ptr() if keep_stats else None, rstd.data_ptr() if keep_stats else None,
        _stream(device)), "sgemm_cube_layer_norm")
    if out is not None:
        _written(out)
    return (y, mean, rstd) if keep_stats else y


def layer_norm_backward(dy, x, weight, mean, rstd, out=None):
    """(dx, dweight, dbias) of layer_norm at x, with the mean and rstd that it
    kept.  out may be dy; dweight and dbias are float32."""
    device = _current_device()
    px, ldx = _matrix(x, "x", device, dtype=_DTYPES)
    rows, cols = x.shape
    pdy, lddy = _matrix(dy, "dy", device, x.shape, (x.dtype,))
    pw = _vector(weight, "weight", device, cols)
    pm, pr = _vector(mean, "mean", device, rows), _vector(rstd, "rstd", device, rows)
    dx = out if out is not None else _new((rows, cols), x, x.dtype)
    pdx, lddx = _matrix(dx, "out", device, x.shape, (x.dtype,))
    dw, db = _new((2, cols), x)
    held, ws, size = _workspace(
        None, device, binding.sgemm_cube_layer_norm_backward_workspace_size(rows, cols), x)
    _check(binding.sgemm_cube_layer_norm_backward(
        rows, cols, _DTYPES[x.dtype], pdy, lddy, px, ldx, pw, pm, pr, pdx, lddx, dw.data_ptr(),
        db.data_ptr(), ws, size, _stream(device)),
        "sgemm_cube_layer_norm_backward")
    if out is not None:
        _written(out)
    return dx, dw, db


def _flat(t, name, device, n, dtype):
    """Address of a contiguous tensor of n values."""
    if not isinstance(t, torch.Tensor) or t.dtype not in dtype or t.get_device() != device:
        _refuse(t, name, dtype)
    if t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous and hold {n} values")
    return t.data_ptr()


class AdamW:
    """AdamW with decoupled weight decay over a program's tensors, one kernel
    launch for up to 48 of them (sgemm_cube_adamw).

    params        contiguous float32 tensors, updated in place
    weight_decay  one number, or one per tensor
    state_bits    32: float32 states; 8: int8 and uint8 codes with a float32
                  scale per 256 values
    states        dict of lists with one contiguous tensor per parameter, to go
                  on from: "exp_avgs", "exp_avg_sqs" (32 bits: float32; 8 bits:
                  int8 and uint8) and, for 8 bits, "exp_avg_scales" and
                  "exp_avg_sq_scales".  They are used in place.  Without it the
                  states start at zero.  The attribute `states` holds them.

    The object holds the parameters and states themselves; new values are copied
    into them.  Two entries that share memory are refused, and so is a parameter whose
    memory was exchanged since (p.data = ...).  Gradients are given to each step; they
    must not lie in the parameters or states.
    """

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8,
                 weight_decay=0.01, state_bits: int = 32, states=None, step: int = 0):
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        self.params = tuple(params)
        self.lr, self.betas, self.eps = lr, tuple(betas), eps
        self.state_bits, self.steps = state_bits, step
        n = len(self.params)
        decay = list(weight_decay) if hasattr(weight_decay, "__len__") else [weight_decay] * n
        if len(decay) != n:
            raise ValueError(f"weight_decay must be one number or {n}")
        self.states = self._zero_states() if states is None else dict(states)
        kinds = self._kinds()
        if set(self.states) != set(kinds):
            raise ValueError(f"states must hold {', '.join(kinds)}")
        # Aliases of the given states: their memory stays as long as the optimizer.
        self.states = MappingProxyType({key: tuple(t.detach() if isinstance(t, torch.Tensor) else t
                                                   for t in self.states[key]) for key in kinds})
        self._list = (binding.AdamwTensor * n)()
        self._entries = list(self._list)
        self._device = device = _current_device()
        for i, p in enumerate(self.params):
            count = p.numel() if isinstance(p, torch.Tensor) else 0
            entry = self._entries[i]
            entry.count, entry.weight_decay = count, decay[i]
            entry.param = _flat(p, f"params[{i}]", device, count, _F32)
            for key, (field, dtype, scale) in kinds.items():
                if len(self.states[key]) != n:
                    raise ValueError(f"states[{key!r}] must hold {n} tensors")
                size = -(-count // binding.ADAMW_BLOCK) if scale else count
                setattr(entry, field, _flat(self.states[key][i], f"states[{key!r}][{i}]", device,
                                            size, (dtype,)))
        self._check_apart()
        self._counts = [p.numel() for p in self.params]
        self._addresses = list(map(_address, self.params))

    def _kinds(self):
        """states' keys: (field of the list's entries, type, one value per block)."""
        f32 = torch.float32
        if self.state_bits == 32:
            return {"exp_avgs": ("exp_avg", f32, False), "exp_avg_sqs": ("exp_avg_sq", f32, False)}
        return {"exp_avgs": ("exp_avg", torch.int8, False),
                "exp_avg_sqs": ("exp_avg_sq", torch.uint8, False),
                "exp_avg_scales": ("exp_avg_scale", f32, True),
                "exp_avg_sq_scales": ("exp_avg_sq_scale", f32, True)}

    def _zero_states(self):
        block = binding.ADAMW_BLOCK
        return {key: [torch.zeros(-(-p.numel() // block) if scale else p.numel(), dtype=dtype,
                                  device=p.device) for p in self.params]
                for key, (_, dtype, scale) in self._kinds().items()}

    def step(self, grads, step: int | None = None, grad_scale: float = 1.0):
        """One step from grads (contiguous tensors of one type: float32, float16 or
        bfloat16), multiplied by grad_scale first.  step: its number, by default
        one more than the last.  A captured step keeps its number, and with it the bias
        corrections, on every replay."""
        grads = list(grads)
        if len(grads) != len(self._counts):
            raise ValueError(f"grads must hold {len(self._counts)} tensors")
        number = self.steps + 1 if step is None else step
        dtype = grads[0].dtype if grads and isinstance(grads[0], torch.Tensor) else torch.float32
        if dtype not in _DTYPES:
            raise TypeError("grads must be float32, float16 or bfloat16")
        device = self._check_held()
        # _flat's checks over the whole list at a time, two thirds of the time of one
        # tensor after the other; where one fails, _flat finds which.
        if (set(map(type, grads)) != {torch.Tensor} or {g.dtype for g in grads} != {dtype}
                or set(map(_device_of, grads)) != {device} or not all(map(_contiguous, grads))
                or list(map(_count, grads)) != self._counts):
            for i, (g, n) in enumerate(zip(grads, self._counts)):
                _flat(g, f"grads[{i}]", device, n, (dtype,))
        for entry, address in zip(self._entries, map(_address, grads)):
            entry.grad = address
        _check(binding.sgemm_cube_adamw(
            len(grads), self._list, _DTYPES[dtype], self.state_bits, self.lr, self.betas[0],
            self.betas[1], self.eps, grad_scale, number, _stream(device)), "sgemm_cube_adamw")
        _written(self.params)
        self.steps = number

    def state_values(self, out=None):
        """(exp_avgs, exp_avg_sqs) as lists of float32 tensors in the parameters'
        shapes, as a checkpoint holds them; out: a pair of lists to write to.
        With 32-bit states, views of the states themselves (or copies in out)."""
        if out is None and self.state_bits == 32:
            return tuple([state.view(p.shape) for state, p in zip(self.states[key], self.params)]
                         for key in ("exp_avgs", "exp_avg_sqs"))
        if out is None:
            out = tuple([torch.empty_like(p) for p in self.params] for _ in range(2))
        n = len(self._counts)
        if len(out) != 2 or len(out[0]) != n or len(out[1]) != n:
            raise ValueError(f"out must be a pair of lists of {n} tensors")
        device = self._check_held()
        addresses = [(binding.ctypes.c_void_p * n)(*(
            _flat(t, f"out[{k}][{i}]", device, self._counts[i], _F32)
            for i, t in enumerate(out[k]))) for k in range(2)]
        if self.state_bits == 32:
            for k, key in enumerate(("exp_avgs", "exp_avg_sqs")):
                for t, s in zip(out[k], self.states[key]):
                    t.view(-1).copy_(s.view(-1))
            return out
        _check(binding.sgemm_cube_adamw_values(n, self._list, *addresses, _stream(device)),
               "sgemm_cube_adamw_values")
        _written([*out[0], *out[1]])
        return out

    def _check_apart(self):
        """Refuses memory that two entries share (a tied weight given twice, say): one
        launch writes both, in no order.  (An entry's own operands are the library's to
        check.)"""
        held = {"params": self.params, **self.states}
        spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), i, key)
                       for key, tensors in held.items() for i, t in enumerate(tensors)
                       if t.numel())
        # The furthest end so far of any entry, and of any other than that one.
        first, second = (0, -1, ""), (0, -1, "")
        for begin, end, i, key in spans:
            other = first if first[1] != i else second
            if other[0] > begin:
                raise ValueError(f"{key}[{i}] shares memory with {other[2]}[{other[1]}]")
            if end > first[0]:
                if first[1] != i:
                    second = first
                first = (end, i, key)
            elif first[1] != i and end > second[0]:
                second = (end, i, key)

    def _check_held(self):
        """The device; refuses parameters that have moved since their addresses were
        taken."""
        if _current_device() != self._device:
            raise ValueError("the parameters are not on the current device")
        if list(map(_address, self.params)) != self._addresses:
            raise ValueError("a parameter is no longer in the memory it had")
        return self._device
