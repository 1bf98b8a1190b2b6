"""The softmax head's operators on torch tensors: layer norm, the exact softmax
loss with its gradient, AdamW, and a head that trains with them.

Argument marshalling for the calls of ``include/huge.h``, as in ``binding``.
Rows may be any two-dimensional GPU tensors whose columns are adjacent (a slice
of a wider buffer among them).  Work runs on ``stream`` (default: torch's
current stream), and outputs are allocated for that stream.  A stream that is
given keeps the arguments until the call's work on it is done; on the current
one torch's own rule holds, that who uses a tensor of another stream there
records it.  What the classes hold is kept on either.
Errors that only the device can see are kept in a status word until ``check``.
Nothing here is part of torch's autograd: results do not require a gradient,
also where arguments do; the gradients are calls of their own.
"""
from __future__ import annotations

import ctypes

from .binding import (HUGE_DTYPE_BF16, HUGE_DTYPE_F32, HUGE_ERR_INVALID_ARG, HUGE_STATE_F32,
                      HUGE_STATE_Q8, HugeAdamwConfig, HugeAdamwTensor, HugeError,
                      HugeSoftmaxConfig, _arg, _dptr, _ok, load)

_DTYPES = {"f32": HUGE_DTYPE_F32, "bf16": HUGE_DTYPE_BF16}


def _dtype_code(t, what):
    import torch
    if t.dtype is torch.float32:
        return HUGE_DTYPE_F32
    if t.dtype is torch.bfloat16:
        return HUGE_DTYPE_BF16
    raise TypeError(f"{what}: expected float32 or bfloat16, got {t.dtype}")


def _rows(t, what, dim=None, like=None):
    """(pointer, row stride) of a GPU tensor of rows whose columns are adjacent."""
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dim() != 2:
        got = f"shape {tuple(t.shape)} on {t.device}" if isinstance(t, torch.Tensor) \
            else type(t).__name__
        raise TypeError(f"{what}: expected a two-dimensional GPU tensor, got {got}")
    if like is not None and (t.dtype is not like.dtype or t.device != like.device):
        raise TypeError(f"{what}: {t.dtype} on {t.device}, expected {like.dtype} on {like.device}")
    n, cols = t.shape
    if dim is not None and cols != dim:
        raise ValueError(f"{what}: rows of {cols}, expected {dim}")
    ld, step = t.stride()
    if cols > 1 and step != 1:
        raise ValueError(f"{what}: the columns of a row must be adjacent, stride {step}")
    if n <= 1:
        ld = cols
    if ld < cols:
        raise ValueError(f"{what}: rows overlap (stride {ld} of {cols})")
    return t.data_ptr(), ld


def _vector(t, n, dtype, what, device):
    """Pointer of a contiguous GPU vector of n elements (None stays None)."""
    import torch
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.is_cuda and t.is_contiguous()):
        _arg(t, (str(dtype).split(".")[1],), what)
    if t.numel() != n:
        raise ValueError(f"{what}: {t.numel()} elements, expected {n}")
    if t.device != device:
        raise ValueError(f"{what}: on {t.device}, expected {device}")
    return t.data_ptr()


def _current(device):
    """torch's current stream on a device, as a pointer."""
    import torch
    return torch._C._cuda_getCurrentRawStream(device.index)


def _same_device(stream, device):
    if stream.device != device:
        raise ValueError(f"stream: of {stream.device}, expected {device}")


class _on:
    """``with _on(device, stream, tensors) as pointer``: the device is current, and
    the pointer is the stream to launch on.  With a stream of the caller's, what is
    allocated inside belongs to it, and `tensors` are not given to others before its
    work on them is done."""

    __slots__ = ("stream", "tensors", "guards", "device")

    def __init__(self, device, stream, tensors):
        self.device, self.stream, self.tensors = device, stream, tensors

    def __enter__(self):
        import torch
        self.guards = []
        if torch.cuda.current_device() != self.device.index:
            self.guards.append(torch.cuda.device(self.device))
        if self.stream is not None:
            _same_device(self.stream, self.device)
            self.guards.append(torch.cuda.stream(self.stream))
        for g in self.guards:
            g.__enter__()
        return _current(self.device) if self.stream is None else self.stream.cuda_stream

    def __exit__(self, *error):
        for g in reversed(self.guards):
            g.__exit__(*error)
        if self.stream is not None:
            for t in self.tensors:
                if t is not None:
                    t.record_stream(self.stream)


def _capturing(stream):
    """Whether a stream's work is being captured into a graph (the default stream's
    never is)."""
    import torch
    if stream.cuda_stream == 0:
        return False
    with torch.cuda.stream(stream):
        return torch.cuda.is_current_stream_capturing()


class _Status:
    """The sticky status word of an operator, the memory of its own, and the stream
    of its last call: a call on another stream first waits for the work on that one,
    and the memory is not given to others before the work on any of them is done."""

    def __init__(self, device):
        import torch
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._status_ptr = self.status.data_ptr()
        self._own = [self.status]
        self._last = torch.cuda.current_stream(self.device)
        self._last_ptr = self._last.cuda_stream

    def _ordered(self, stream):
        import torch
        now = _current(self.device) if stream is None else stream.cuda_stream
        if now != self._last_ptr:
            stream = torch.cuda.current_stream(self.device) if stream is None else stream
            _same_device(stream, self.device)
            # a graph waits for nothing outside of it: what came before its capture is
            # done when that begins, and its replays are the caller's to order
            if not _capturing(stream) or _capturing(self._last):
                stream.wait_stream(self._last)
            for t in self._own:
                t.record_stream(stream)
            self._last, self._last_ptr = stream, now

    def check(self):
        """Raise HugeError if a call since the last check met a device-side error
        (synchronises); the status is cleared."""
        import torch
        with torch.cuda.stream(self._last):  # the clearing comes before a next call
            st = int(self.status.item())
            if st != 0:
                self.status.zero_()
        if st != 0:
            raise HugeError(st, type(self).__name__ + " (device)")


# --------------------------------------------------------------------------- #
# Layer norm
# --------------------------------------------------------------------------- #
def layer_norm(x, gamma, beta, eps=1e-5, stream=None):
    """(y, mean, rstd) of the rows x, by huge_layer_norm.  gamma, beta: float32."""
    import torch
    px, ld = _rows(x, "layer_norm x")
    code = _dtype_code(x, "layer_norm x")
    n, dim = x.shape
    pg = _vector(gamma, dim, torch.float32, "layer_norm gamma", x.device)
    pb = _vector(beta, dim, torch.float32, "layer_norm beta", x.device)
    if pg is None or pb is None:
        raise TypeError("layer_norm: gamma and beta are required")
    with _on(x.device, stream, (x, gamma, beta,)) as st:
        y = torch.empty((n, dim), dtype=x.dtype, device=x.device)
        mean, rstd = torch.empty((2, n), dtype=torch.float32, device=x.device).unbind()
        _ok(load().huge_layer_norm(px, ld, n, dim, code, pg, pb, float(eps), y.data_ptr(), dim,
                                   mean.data_ptr(), rstd.data_ptr(), st), "huge_layer_norm")
    return y, mean, rstd


def layer_norm_backward(dy, x, gamma, mean, rstd, want_dx=True, want_weights=True, stream=None):
    """(dx, dgamma, dbeta) by huge_layer_norm_backward; None where not wanted."""
    import torch
    px, ldx = _rows(x, "layer_norm_backward x")
    code = _dtype_code(x, "layer_norm_backward x")
    n, dim = x.shape
    pdy, ldy = _rows(dy, "layer_norm_backward dy", dim, x)
    if dy.shape[0] != n:
        raise ValueError(f"layer_norm_backward: {dy.shape[0]} rows of dy, {n} of x")
    pg = _vector(gamma, dim, torch.float32, "layer_norm_backward gamma", x.device)
    pm = _vector(mean, n, torch.float32, "layer_norm_backward mean", x.device)
    pr = _vector(rstd, n, torch.float32, "layer_norm_backward rstd", x.device)
    if pg is None or pm is None or pr is None:
        raise TypeError("layer_norm_backward: gamma, mean and rstd are required")
    L = load()
    with _on(x.device, stream, (dy, x, gamma, mean, rstd,)) as st:
        dx = torch.empty((n, dim), dtype=x.dtype, device=x.device) if want_dx else None
        dgamma = dbeta = ws = None
        bytes_ = 0
        if want_weights:
            bytes_ = L.huge_layer_norm_workspace_bytes(n, dim)
            ws = torch.empty(bytes_, dtype=torch.uint8, device=x.device)
            dgamma, dbeta = torch.empty((2, dim), dtype=torch.float32, device=x.device).unbind()
        _ok(L.huge_layer_norm_backward(pdy, ldy, px, ldx, n, dim, code, pg, pm, pr, _dptr(dx), dim,
                                       _dptr(dgamma), _dptr(dbeta), _dptr(ws), bytes_, st),
            "huge_layer_norm_backward")
    return dx, dgamma, dbeta


# --------------------------------------------------------------------------- #
# Exact softmax loss
# --------------------------------------------------------------------------- #
class SoftmaxLoss(_Status):
    """Workspace of huge_softmax_loss and huge_softmax_grad for tables of
    num_classes x dim and up to max_rows rows a call.  grad=False: the loss only,
    in a smaller workspace."""

    def __init__(self, max_rows, num_classes, dim, dtype="f32", grad=True, device="cuda"):
        import torch
        L = load()
        self.cfg = HugeSoftmaxConfig(int(num_classes), int(max_rows), int(dim), _DTYPES[dtype],
                                     int(bool(grad)))
        self.ws_bytes = L.huge_softmax_workspace_bytes(ctypes.byref(self.cfg))
        if self.ws_bytes == 0:
            raise HugeError(HUGE_ERR_INVALID_ARG, "huge_softmax_workspace_bytes")
        super().__init__(device)
        self._ws = torch.empty(self.ws_bytes + 256, dtype=torch.uint8, device=self.device)
        self._own.append(self._ws)
        self._ws_ptr = self._ws.data_ptr() + ((-self._ws.data_ptr()) % 256)

    def _inputs(self, what, h, w, labels, bias, weights):
        """Pointers in the order of the C calls, checked."""
        import torch
        c = self.cfg
        ph, ldh = _rows(h, what + " h", c.dim)
        if _dtype_code(h, what + " h") != c.dtype:
            raise TypeError(f"{what}: h is {h.dtype}, not the type of this SoftmaxLoss")
        if h.device != self.device:
            raise ValueError(f"{what}: h on {h.device}, expected {self.device}")
        pw, ldw = _rows(w, what + " w", c.dim, h)
        if w.shape[0] != c.num_classes:
            raise ValueError(f"{what}: {w.shape[0]} rows of w, expected {c.num_classes}")
        n = h.shape[0]
        return (ctypes.byref(c), ph, ldh, n, pw, ldw,
                _vector(bias, c.num_classes, torch.float32, what + " bias", h.device),
                _vector(labels, n, torch.int32, what + " labels", h.device),
                _vector(weights, n, torch.float32, what + " weights", h.device))

    def loss(self, h, w, labels, bias=None, weights=None, total=None, stream=None):
        """(loss, lse), float32 per row of h.  total: a float64 tensor of one element
        that receives the sum of the losses."""
        import torch
        a = self._inputs("SoftmaxLoss.loss", h, w, labels, bias, weights)
        pt = _vector(total, 1, torch.float64, "SoftmaxLoss.loss total", h.device)
        self._ordered(stream)
        with _on(self.device, stream, (h, w, labels, bias, weights, total,)) as st:
            loss, lse = torch.empty((2, a[3]), dtype=torch.float32, device=self.device).unbind()
            _ok(load().huge_softmax_loss(*a, loss.data_ptr(), lse.data_ptr(), pt,
                                         self._status_ptr, self._ws_ptr, self.ws_bytes, st),
                "huge_softmax_loss")
        return loss, lse

    def grad(self, h, w, labels, lse, bias=None, weights=None, scale=1.0, want_h=True,
             want_w=True, want_bias=True, stream=None):
        """(dh, dw, dbias) of scale times the sum of the losses, dh and dw in the
        type of h; None where not wanted."""
        import torch
        a = self._inputs("SoftmaxLoss.grad", h, w, labels, bias, weights)
        pl = _vector(lse, a[3], torch.float32, "SoftmaxLoss.grad lse", h.device)
        if pl is None:
            raise TypeError("SoftmaxLoss.grad: lse is required")
        c = self.cfg
        self._ordered(stream)
        with _on(self.device, stream, (h, w, labels, lse, bias, weights,)) as st:
            new = lambda *shape, t=h.dtype: torch.empty(shape, dtype=t, device=self.device)  # noqa: E731
            dh = new(a[3], c.dim) if want_h else None
            dw = new(c.num_classes, c.dim) if want_w else None
            db = new(c.num_classes, t=torch.float32) if want_bias else None
            _ok(load().huge_softmax_grad(*a, pl, float(scale), _dptr(dh), _dptr(dw), _dptr(db),
                                         self._status_ptr, self._ws_ptr, self.ws_bytes, st),
                "huge_softmax_grad")
        return dh, dw, db


# --------------------------------------------------------------------------- #
# AdamW
# --------------------------------------------------------------------------- #
class AdamW(_Status):
    """AdamW over a list of contiguous float32 or bfloat16 GPU tensors of one
    device that share no memory, updated in place by huge_adamw_step.  states:
    "f32", or "q8" for moments in 8 bits.  The parameters' storage must stay where
    it is.  bfloat16 parameters have no copy in 32 bits: a step below half of their
    last bit, 2^-9 to 2^-8 of the value, does not move them."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01,
                 states="f32"):
        import torch
        L = load()
        self.params = list(params)
        if not self.params:
            raise ValueError("AdamW: no parameters")
        self.kind = {"f32": HUGE_STATE_F32, "q8": HUGE_STATE_Q8}[states]
        for k, p in enumerate(self.params):
            _arg(p, ("float32", "bfloat16"), f"AdamW params[{k}]")
            if p.device != self.params[0].device:
                raise ValueError(f"AdamW params[{k}]: on {p.device}, expected "
                                 f"{self.params[0].device}")
        ends = sorted((p.data_ptr(), p.data_ptr() + p.numel() * p.element_size())
                      for p in self.params if p.numel())
        if any(a[1] > b[0] for a, b in zip(ends, ends[1:])):
            raise ValueError("AdamW: parameters that share memory")
        super().__init__(self.params[0].device)
        self.steps = 0
        self.lr = float(lr)
        self.cfg = HugeAdamwConfig(self.lr, float(betas[0]), float(betas[1]), float(eps),
                                   float(weight_decay), 1.0, 1, self.kind)
        count = len(self.params)
        self._tensors = (HugeAdamwTensor * count)()
        # one buffer for all states, each 256-byte aligned in it
        at, self._state_at = 0, []
        for p in self.params:
            self._state_at.append(at)
            at += -(-L.huge_adamw_state_bytes(p.numel(), self.kind) // 256) * 256
        self.states = torch.zeros(at + 256, dtype=torch.uint8, device=self.device)
        self._own += [self.states, *self.params]
        self._skip = (-self.states.data_ptr()) % 256
        for k, p in enumerate(self.params):
            t = self._tensors[k]
            t.d_param, t.n = p.data_ptr(), p.numel()
            t.d_state = self.states.data_ptr() + self._skip + self._state_at[k]
            t.param_dtype = _dtype_code(p, f"AdamW params[{k}]")
        # where values() puts the moments: one array, each 16-byte aligned in it
        self._flat_at, self._flat_split, self._flat = [], [], 0
        for p in 2 * self.params:
            pad = -p.numel() % 4
            self._flat_at.append(self._flat)
            self._flat_split += [p.numel(), pad]
            self._flat += p.numel() + pad
        self._values = (ctypes.c_void_p * (2 * count))()
        if self.kind == HUGE_STATE_F32:  # m, then v, each in whole blocks of 256
            half = [L.huge_adamw_state_bytes(p.numel(), self.kind) // 2 for p in self.params]
            self._views = [[self._view(self._state_at[k] + which * half[k], p)
                            for k, p in enumerate(self.params)] for which in (0, 1)]

    def _view(self, at, p):
        import torch
        at += self._skip
        return self.states[at:at + 4 * p.numel()].view(torch.float32).view(p.shape)

    def _list(self, ts, dtypes, what):
        import torch
        ts = list(ts)
        if len(ts) != len(self.params):
            raise ValueError(f"{what}: {len(ts)} tensors, expected {len(self.params)}")
        types = [getattr(torch, d) for d in dtypes]
        for k, (t, p) in enumerate(zip(ts, self.params)):
            if not (isinstance(t, torch.Tensor) and t.dtype in types and t.is_cuda
                    and t.is_contiguous()):
                _arg(t, dtypes, f"{what}[{k}]")
            if t.numel() != p.numel() or t.device != p.device:
                raise ValueError(f"{what}[{k}]: {t.numel()} elements on {t.device}, expected "
                                 f"{p.numel()} on {p.device}")
        return ts

    def step(self, grads, lr=None, grad_scale=1.0, stream=None):
        """One step with these gradients (float32 or bfloat16, one per parameter).  In
        a graph's capture its learning rate and bias corrections are recorded too."""
        grads = self._list(grads, ("float32", "bfloat16"), "AdamW.step grads")
        c = self.cfg
        c.lr = self.lr if lr is None else float(lr)
        c.grad_scale = float(grad_scale)
        c.step = self.steps + 1
        for t, g in zip(self._tensors, grads):
            t.d_grad = g.data_ptr()
            t.grad_dtype = _dtype_code(g, "AdamW.step grads")
        self._ordered(stream)
        with _on(self.device, stream, (self.states, *self.params, *grads,)) as st:
            _ok(load().huge_adamw_step(ctypes.byref(c), self._tensors, len(grads),
                                       self._status_ptr, st), "huge_adamw_step")
        self.steps += 1

    def _pointers(self, ts):
        return (ctypes.c_void_p * len(ts))(*[t.data_ptr() for t in ts])

    def values(self, stream=None):
        """(m, v): lists of float32 tensors shaped like the parameters, ready on the
        stream.  States "f32": the moments themselves, as views that the next step
        changes (clone what is to stay); "q8": what they stand for, in new tensors."""
        import torch
        self._ordered(stream)
        if self.kind == HUGE_STATE_F32:
            return [list(ts) for ts in self._views]
        with _on(self.device, stream, (self.states,)) as st:
            flat = torch.empty(self._flat, dtype=torch.float32, device=self.device)
            base, count = flat.data_ptr(), len(self.params)
            for k, at in enumerate(self._flat_at):
                self._values[k] = base + 4 * at
            m, v = (ctypes.byref(self._values, 8 * count * which) for which in (0, 1))
            _ok(load().huge_adamw_get_state(self._tensors, count, self.kind,
                                            ctypes.cast(m, ctypes.POINTER(ctypes.c_void_p)),
                                            ctypes.cast(v, ctypes.POINTER(ctypes.c_void_p)), st),
                "huge_adamw_get_state")
        parts = flat.split(self._flat_split)[::2]
        out = [t if p.dim() == 1 else t.view(p.shape) for t, p in zip(parts, 2 * self.params)]
        return out[:count], out[count:]

    def load(self, m, v, steps, stream=None):
        """Set the moments (float32, v >= 0) and the steps that they have seen."""
        m = self._list(m, ("float32",), "AdamW.load m")
        v = self._list(v, ("float32",), "AdamW.load v")
        if int(steps) < 0:
            raise ValueError(f"AdamW.load: {steps} steps")
        self._ordered(stream)
        with _on(self.device, stream, (self.states, *m, *v,)) as st:
            _ok(load().huge_adamw_set_state(self._tensors, len(m), self.kind, self._pointers(m),
                                            self._pointers(v), st), "huge_adamw_set_state")
        self.steps = int(steps)


# --------------------------------------------------------------------------- #
# A head that trains
# --------------------------------------------------------------------------- #
class SoftmaxHead:
    """Layer norm, a linear layer and the softmax loss over num_classes classes on
    rows of embeddings, trained by AdamW: the downstream classifier of Sec. 4.2,
    or the exact softmax over all nodes that negative sampling stands in for.

    step(x, labels) trains the head on rows x (n x dim) and returns the mean loss
    (device) and the gradient of x, for a caller that trains the rows too.  Steps and
    losses on different streams wait for each other; what a call returns is ready
    on its own stream."""

    def __init__(self, num_classes, dim, max_rows, dtype="f32", lr=1e-3, weight_decay=0.01,
                 states="f32", eps=1e-5, seed=0, device="cuda"):
        import torch
        self.op = SoftmaxLoss(max_rows, num_classes, dim, dtype=dtype, device=device)
        dev = self.op.device
        g = torch.Generator(device=dev).manual_seed(int(seed))
        self.eps = float(eps)
        self.gamma = torch.ones(dim, device=dev)
        self.beta = torch.zeros(dim, device=dev)
        w = torch.randn((num_classes, dim), device=dev, generator=g) * dim ** -0.5
        self.w = w.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
        self.bias = torch.zeros(num_classes, device=dev)
        self.opt = AdamW([self.gamma, self.beta, self.w, self.bias], lr=lr,
                         weight_decay=weight_decay, states=states)
        self.total = torch.zeros(1, dtype=torch.float64, device=dev)
        self.op._own.append(self.total)

    def _ordered(self, stream):
        # before the first kernel: layer norm, which waits for nothing, reads parameters
        self.op._ordered(stream)
        self.opt._ordered(stream)

    def loss(self, x, labels, weights=None, stream=None):
        """Loss per row, forward only."""
        self._ordered(stream)
        y, _, _ = layer_norm(x, self.gamma, self.beta, self.eps, stream=stream)
        return self.op.loss(y, self.w, labels, self.bias, weights, stream=stream)[0]

    def step(self, x, labels, weights=None, lr=None, want_dx=True, stream=None):
        """One training step on the mean over the rows of their losses."""
        scale = 1.0 / max(1, x.shape[0])
        self._ordered(stream)
        y, mean, rstd = layer_norm(x, self.gamma, self.beta, self.eps, stream=stream)
        _, lse = self.op.loss(y, self.w, labels, self.bias, weights, total=self.total,
                              stream=stream)
        dy, dw, db = self.op.grad(y, self.w, labels, lse, self.bias, weights, scale=scale,
                                  stream=stream)
        dx, dgamma, dbeta = layer_norm_backward(dy, x, self.gamma, mean, rstd, want_dx=want_dx,
                                                stream=stream)
        self.opt.step([dgamma, dbeta, dw, db], lr=lr, stream=stream)
        with _on(self.op.device, stream, ()):
            return self.total * scale, dx

    def check(self):
        """Raise the first device-side error since the last check."""
        self.op.check()
        self.opt.check()
