"""What a softmax head normalises, answers and clips with, on torch tensors: RMS norm
with the residual's addition, rows in 8 bits, log probabilities with entropy and the
most likely classes, and the norm over a list of gradients.

Argument marshalling for the calls of ``include/huge.h``, with the rules of ``head``:
rows are two-dimensional GPU tensors whose columns are adjacent, work runs on
``stream`` (default: torch's current stream), and nothing here is part of torch's
autograd.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple

import numpy as np

from . import head as _head
from .binding import (HUGE_DTYPE_Q8, HUGE_ERR_INVALID_ARG, HugeError, HugeGradTensor,
                      HugeLogProbsConfig, _arg, _dptr, _ok)
from .head import _DTYPES, _Status, _dtype_code, _on, _rows, _vector

BLOCK = 32  # columns that share a scale of rows in 8 bits


# --------------------------------------------------------------------------- #
# Rows in 8 bits
# --------------------------------------------------------------------------- #
class Q8Rows(NamedTuple):
    """Rows in 8 bits: codes (n x dim, float8_e4m3fn) under scales (n x ceil(dim / 32),
    uint8), each 2^(scale - 127) for 32 columns."""
    codes: "torch.Tensor"   # noqa: F821
    scales: "torch.Tensor"  # noqa: F821


def _q8(q, what, dim=None, device=None):
    """(codes' pointer, stride, scales' pointer, stride, n, dim) of Q8Rows."""
    import torch
    if not (isinstance(q, (tuple, list)) and len(q) == 2):
        raise TypeError(f"{what}: expected Q8Rows, got {type(q).__name__}")
    codes, scales = q
    pc, ldc = _rows(codes, what + " codes", dim)
    n, cols = codes.shape
    ps, lds = _rows(scales, what + " scales", -(-cols // BLOCK))
    if codes.dtype is not torch.float8_e4m3fn or scales.dtype is not torch.uint8:
        raise TypeError(f"{what}: {codes.dtype} and {scales.dtype}, expected float8_e4m3fn and "
                        "uint8")
    if scales.shape[0] != n:
        raise ValueError(f"{what}: {scales.shape[0]} rows of scales, {n} of codes")
    for t in q:
        if t.device != (device or codes.device):
            raise ValueError(f"{what}: on {t.device}, expected {device or codes.device}")
    return pc, ldc, ps, lds, n, cols


def _new_q8(n, dim, device):
    import torch
    return Q8Rows(torch.empty((n, dim), dtype=torch.float8_e4m3fn, device=device),
                  torch.empty((n, -(-dim // BLOCK)), dtype=torch.uint8, device=device))


def q8_rows(x, stream=None):
    """The rows x (float32 or bfloat16) in 8 bits, by huge_quantise_rows."""
    px, ld = _rows(x, "q8_rows x")
    code = _dtype_code(x, "q8_rows x")
    n, dim = x.shape
    with _on(x.device, stream, (x,)) as st:
        q = _new_q8(n, dim, x.device)
        _ok(_head.load().huge_quantise_rows(px, ld, n, dim, code, q.codes.data_ptr(), dim,
                                            q.scales.data_ptr(), q.scales.shape[1], st),
            "huge_quantise_rows")
    return q


def q8_values(q, dtype="f32", stream=None):
    """What rows in 8 bits stand for ("f32" or "bf16"), by huge_dequantise_rows."""
    import torch
    code = _DTYPES[dtype]
    pc, ldc, ps, lds, n, dim = _q8(q, "q8_values")
    device = q[0].device
    with _on(device, stream, q) as st:
        y = torch.empty((n, dim), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32,
                        device=device)
        _ok(_head.load().huge_dequantise_rows(pc, ldc, ps, lds, n, dim, y.data_ptr(), dim, code,
                                              st), "huge_dequantise_rows")
    return y


# --------------------------------------------------------------------------- #
# RMS norm
# --------------------------------------------------------------------------- #
def rms_norm(x, gamma, residual=None, eps=1e-5, q8=False, stream=None):
    """(y, total, rstd) of the rows x, by huge_rms_norm: total = x + residual in their
    type (x itself without a residual), y its norm in their type or, with q8, in 8 bits
    (Q8Rows).  gamma: float32."""
    import torch
    px, ld = _rows(x, "rms_norm x")
    code = _dtype_code(x, "rms_norm x")
    n, dim = x.shape
    pg = _vector(gamma, dim, torch.float32, "rms_norm gamma", x.device)
    if pg is None:
        raise TypeError("rms_norm: gamma is required")
    pr, ldr = None, 0
    if residual is not None:
        pr, ldr = _rows(residual, "rms_norm residual", dim, x)
        if residual.shape[0] != n:
            raise ValueError(f"rms_norm: {residual.shape[0]} rows of residual, {n} of x")
    with _on(x.device, stream, (x, residual, gamma)) as st:
        # dense like x, or where that is a part of wider rows by themselves
        total = x if residual is None else torch.empty_like(x)
        rstd = torch.empty(n, dtype=torch.float32, device=x.device)
        py = pc = ps = None
        ld_scales = 0
        if q8:
            y = _new_q8(n, dim, x.device)
            pc, ps, ld_scales = y.codes.data_ptr(), y.scales.data_ptr(), y.scales.shape[1]
        else:
            y = torch.empty_like(x)
            py = y.data_ptr()
        _ok(_head.load().huge_rms_norm(px, ld, pr, ldr, n, dim, code, pg, float(eps),
                                       None if residual is None else total.data_ptr(), dim, py,
                                       dim, pc, dim, ps, ld_scales, rstd.data_ptr(), st),
            "huge_rms_norm")
    return y, total, rstd


def rms_norm_backward(dy, total, gamma, rstd, dtotal=None, want_dx=True, want_gamma=True,
                      stream=None):
    """(dx, dgamma) by huge_rms_norm_backward; None where not wanted.  dx is the gradient
    of x and of the residual, with dtotal, what reaches their sum past the norm."""
    import torch
    pt, ldt = _rows(total, "rms_norm_backward total")
    code = _dtype_code(total, "rms_norm_backward total")
    n, dim = total.shape
    pdy, ldy = _rows(dy, "rms_norm_backward dy", dim, total)
    pdt, lddt = None, 0
    if dtotal is not None:
        pdt, lddt = _rows(dtotal, "rms_norm_backward dtotal", dim, total)
    for name, t in (("dy", dy), ("dtotal", dtotal)):
        if t is not None and t.shape[0] != n:
            raise ValueError(f"rms_norm_backward: {t.shape[0]} rows of {name}, {n} of total")
    pg = _vector(gamma, dim, torch.float32, "rms_norm_backward gamma", total.device)
    pr = _vector(rstd, n, torch.float32, "rms_norm_backward rstd", total.device)
    if pg is None or pr is None:
        raise TypeError("rms_norm_backward: gamma and rstd are required")
    L = _head.load()
    with _on(total.device, stream, (dy, total, gamma, rstd, dtotal)) as st:
        dx = torch.empty_like(total) if want_dx else None
        dgamma = ws = None
        bytes_ = 0
        if want_gamma:
            bytes_ = L.huge_rms_norm_workspace_bytes(n, dim)
            ws = torch.empty(bytes_, dtype=torch.uint8, device=total.device)
            dgamma = torch.empty(dim, dtype=torch.float32, device=total.device)
        _ok(L.huge_rms_norm_backward(pdy, ldy, pt, ldt, pdt, lddt, n, dim, code, pg, pr, _dptr(dx),
                                     dim, _dptr(dgamma), _dptr(ws), bytes_, st),
            "huge_rms_norm_backward")
    return dx, dgamma


# --------------------------------------------------------------------------- #
# Log probabilities
# --------------------------------------------------------------------------- #
class Answers(NamedTuple):
    """logp (of the labels, or None), entropy, lse: float32 per row.  ids (int32) and
    top_logp: rows x top, the most likely classes first; None with top=0."""
    logp: "torch.Tensor"      # noqa: F821
    entropy: "torch.Tensor"   # noqa: F821
    lse: "torch.Tensor"       # noqa: F821
    ids: "torch.Tensor"       # noqa: F821
    top_logp: "torch.Tensor"  # noqa: F821


class LogProbs(_Status):
    """Workspace of huge_log_probs and, with grad=True, huge_log_probs_grad for tables of
    num_classes x dim and up to max_rows rows a call.  dtype: of the rows and the table;
    "q8": a table in 8 bits (Q8Rows) and rows in bfloat16.  top: how many of the most
    likely classes a call finds, up to 64."""

    def __init__(self, max_rows, num_classes, dim, dtype="f32", top=0, grad=False, device="cuda"):
        import torch
        L = _head.load()
        self.q8 = dtype == "q8"
        code = _DTYPES["bf16" if self.q8 else dtype]
        self.cfg = HugeLogProbsConfig(int(num_classes), int(max_rows), int(dim), code,
                                      HUGE_DTYPE_Q8 if self.q8 else code, int(top),
                                      int(bool(grad)))
        self.ws_bytes = L.huge_log_probs_workspace_bytes(ctypes.byref(self.cfg))
        if self.ws_bytes == 0:
            raise HugeError(HUGE_ERR_INVALID_ARG, "huge_log_probs_workspace_bytes")
        super().__init__(device)
        self._ws = torch.empty(self.ws_bytes + 256, dtype=torch.uint8, device=self.device)
        self._own.append(self._ws)
        self._ws_ptr = self._ws.data_ptr() + ((-self._ws.data_ptr()) % 256)

    def _inputs(self, what, h, w, labels, bias):
        """(rows of h, arguments of h, of w, scales, bias and labels), checked."""
        import torch
        c = self.cfg
        ph, ldh = _rows(h, what + " h", c.dim)
        if _dtype_code(h, what + " h") != c.dtype:
            raise TypeError(f"{what}: h is {h.dtype}, not the type of this LogProbs")
        if h.device != self.device:
            raise ValueError(f"{what}: h on {h.device}, expected {self.device}")
        ps, lds = None, 0
        if self.q8:
            pw, ldw, ps, lds, classes, _ = _q8(w, what + " w", c.dim, self.device)
        else:
            pw, ldw = _rows(w, what + " w", c.dim, h)
            classes = w.shape[0]
        if classes != c.num_classes:
            raise ValueError(f"{what}: {classes} rows of w, expected {c.num_classes}")
        n = h.shape[0]
        return (n, (ctypes.byref(c), ph, ldh, n, pw, ldw), (ps, lds),
                (_vector(bias, c.num_classes, torch.float32, what + " bias", h.device),
                 _vector(labels, n, torch.int32, what + " labels", h.device)))

    def log_probs(self, h, w, labels=None, bias=None, stream=None):
        """Answers of the rows h."""
        import torch
        n, a, scales, more = self._inputs("LogProbs.log_probs", h, w, labels, bias)
        tables = w if self.q8 else (w,)
        self._ordered(stream)
        with _on(self.device, stream, (h, *tables, labels, bias)) as st:
            entropy, lse, *logp = torch.empty((2 + (labels is not None), n), dtype=torch.float32,
                                              device=self.device).unbind()
            logp = logp[0] if logp else None
            ids = top_logp = None
            if self.cfg.top:
                ids = torch.empty((n, self.cfg.top), dtype=torch.int32, device=self.device)
                top_logp = torch.empty((n, self.cfg.top), dtype=torch.float32, device=self.device)
            _ok(_head.load().huge_log_probs(*a, *scales, *more, _dptr(logp), entropy.data_ptr(),
                                            lse.data_ptr(), _dptr(ids), _dptr(top_logp),
                                            self._status_ptr, self._ws_ptr, self.ws_bytes, st),
                "huge_log_probs")
        return Answers(logp, entropy, lse, ids, top_logp)

    def grad(self, h, w, answers, labels=None, dlogp=None, dentropy=None, bias=None, want_h=True,
             want_w=True, want_bias=True, stream=None):
        """(dh, dw, dbias) of the sum over rows of dlogp logp + dentropy entropy (float32
        weights of either sign, None: zeros), dh and dw in the type of h; None where not
        wanted.  answers: what log_probs returned for the same inputs."""
        import torch
        what = "LogProbs.grad"
        if self.q8:
            raise TypeError(f"{what}: a table in 8 bits has no gradient")
        n, a, _, more = self._inputs(what, h, w, labels, bias)
        vec = lambda t, name: _vector(t, n, torch.float32, f"{what} {name}", h.device)  # noqa: E731
        pl, pe = vec(answers.lse, "lse"), vec(answers.entropy, "entropy")
        pdl, pde = vec(dlogp, "dlogp"), vec(dentropy, "dentropy")
        if pl is None:
            raise TypeError(f"{what}: lse is required")
        if dlogp is not None and labels is None:
            raise TypeError(f"{what}: dlogp without labels")
        if dentropy is not None and pe is None:
            raise TypeError(f"{what}: dentropy without entropy")
        c = self.cfg
        self._ordered(stream)
        with _on(self.device, stream, (h, w, labels, bias, answers.lse, answers.entropy, dlogp,
                                       dentropy)) as st:
            new = lambda *shape, t=h.dtype: torch.empty(shape, dtype=t, device=self.device)  # noqa: E731
            dh = new(n, c.dim) if want_h else None
            dw = new(c.num_classes, c.dim) if want_w else None
            db = new(c.num_classes, t=torch.float32) if want_bias else None
            _ok(_head.load().huge_log_probs_grad(*a, *more, pl, pe, pdl, pde, _dptr(dh), _dptr(dw),
                                                 _dptr(db), self._status_ptr, self._ws_ptr,
                                                 self.ws_bytes, st), "huge_log_probs_grad")
        return dh, dw, db


# --------------------------------------------------------------------------- #
# Norms of gradients
# --------------------------------------------------------------------------- #
_TABLE = [("d_grad", "u8"), ("n", "i8"), ("dtype", "i4"), ("fill", "i4")]  # HugeGradTensor


def _grads(grads, what):
    """The list, its device, its table for the C calls and what holds that.  A property of
    all tensors at a time: lists may be hundreds long, and each look costs host time."""
    import torch
    grads = list(grads)
    if not grads:
        raise ValueError(f"{what}: no gradients")
    codes = {torch.float32: _DTYPES["f32"], torch.bfloat16: _DTYPES["bf16"]}
    T = torch.Tensor
    if all(issubclass(c, T) for c in set(map(type, grads))):
        types = list(map(T.dtype.__get__, grads))
        kinds, devices = set(types), set(map(T.get_device, grads))
        if codes.keys() >= kinds and min(devices) >= 0 and all(map(T.is_contiguous, grads)):
            device = grads[0].device
            if len(devices) > 1:
                k = next(k for k, g in enumerate(grads) if g.device != device)
                raise ValueError(f"{what}[{k}]: on {grads[k].device}, expected {device}")
            table = np.empty(len(grads), _TABLE)
            table["d_grad"] = list(map(T.data_ptr, grads))
            table["n"] = list(map(T.numel, grads))
            table["dtype"] = (codes[types[0]] if len(kinds) == 1
                              else list(map(codes.__getitem__, types)))
            return grads, device, table.ctypes.data_as(ctypes.POINTER(HugeGradTensor)), table
    for k, g in enumerate(grads):  # one of them is refused
        _arg(g, ("float32", "bfloat16"), f"{what}[{k}]")
    raise TypeError(f"{what}: expected GPU tensors")


def grad_norm(grads, stream=None):
    """The 2-norm over all elements of a list of contiguous float32 or bfloat16 GPU tensors
    (one float32 element), by huge_grad_norm."""
    import torch
    grads, device, table, _keep = _grads(grads, "grad_norm")
    L = _head.load()
    with _on(device, stream, grads) as st:
        norm = torch.empty(1, dtype=torch.float32, device=device)
        bytes_ = L.huge_grad_norm_workspace_bytes(len(grads))
        ws = torch.empty(bytes_, dtype=torch.uint8, device=device)
        _ok(L.huge_grad_norm(table, len(grads), norm.data_ptr(), ws.data_ptr(), bytes_, st),
            "huge_grad_norm")
    return norm


def clip_grads(grads, max_norm, stream=None):
    """Scales a list of gradients in place so that their norm is at most max_norm, by
    huge_clip_grads, and returns the norm before.  They stay as they are where one of them
    is not finite.  The tensors must share no memory."""
    import torch
    grads, device, table, _keep = _grads(grads, "clip_grads")
    if not float(max_norm) > 0:
        raise ValueError(f"clip_grads: max_norm {max_norm}")
    _head._apart(grads, "clip_grads: gradients")
    L = _head.load()
    with _on(device, stream, grads) as st:
        norm = torch.empty(1, dtype=torch.float32, device=device)
        bytes_ = L.huge_grad_norm_workspace_bytes(len(grads))
        ws = torch.empty(bytes_, dtype=torch.uint8, device=device)
        _ok(L.huge_clip_grads(table, len(grads), float(max_norm), norm.data_ptr(), ws.data_ptr(),
                              bytes_, st), "huge_clip_grads")
    return norm
