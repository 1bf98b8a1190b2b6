"""Plain numpy definitions, in float64, of the softmax head's operators: layer
norm, the exact softmax loss and AdamW.  They share no code with the kernels and
follow the formulas of include/huge.h line by line.
"""
from __future__ import annotations

import numpy as np


def layer_norm(x, gamma, beta, eps):
    """(y, mean, rstd) of the rows x."""
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    return (x - mean[:, None]) * rstd[:, None] * gamma + beta, mean, rstd


def layer_norm_backward(dy, x, gamma, mean, rstd):
    """(dx, dgamma, dbeta)."""
    dy, x = np.asarray(dy, np.float64), np.asarray(x, np.float64)
    xh = (x - mean[:, None]) * rstd[:, None]
    a = dy * gamma
    dx = rstd[:, None] * (a - a.mean(1)[:, None] - xh * (a * xh).mean(1)[:, None])
    return dx, (dy * xh).sum(0), dy.sum(0)


def softmax_loss(h, w, labels, bias=None, weights=None):
    """(loss, lse, counted): counted[i] is the weight of row i, 0 where it has no
    loss.  Classes whose bias is -inf are left out, their rows of w unread."""
    h, w = np.asarray(h, np.float64), np.asarray(w, np.float64)
    n, classes = len(h), len(w)
    b = np.zeros(classes) if bias is None else np.asarray(bias, np.float64)
    c = np.ones(n) if weights is None else np.asarray(weights, np.float64)
    loss, lse, counted = np.zeros(n), np.full(n, -np.inf), np.zeros(n)
    kept = np.flatnonzero(b != -np.inf)
    for i in range(n):
        x = w[kept] @ h[i] + b[kept]
        if kept.size:
            top = x.max()
            lse[i] = top + np.log(np.exp(x - top).sum())
        y = int(labels[i])
        if y < -1 or y >= classes or not (c[i] >= 0 and np.isfinite(c[i])):
            loss[i] = np.nan
        elif y >= 0 and c[i] > 0 and b[y] != -np.inf:
            counted[i] = c[i]
            loss[i] = c[i] * (lse[i] - (w[y] @ h[i] + b[y]))
    return loss, lse, counted


def softmax_grad(h, w, labels, bias=None, weights=None, scale=1.0):
    """(dh, dw, dbias) of scale * sum of the losses, and sums of the absolute
    values of their terms, which bound what rounding does to them."""
    h, w = np.asarray(h, np.float64), np.asarray(w, np.float64)
    _, lse, counted = softmax_loss(np.where(np.isfinite(h), h, 0.0), w, labels, bias, weights)
    b = np.zeros(len(w)) if bias is None else np.asarray(bias, np.float64)
    hc = np.where(counted[:, None] > 0, h, 0.0)      # rows without a loss are not read
    wc = np.where((b != -np.inf)[:, None], w, 0.0)   # nor are classes that are out
    g = np.zeros((len(h), len(w)))
    p = np.zeros_like(g)
    for i in np.flatnonzero(counted):
        p[i] = np.exp(wc @ hc[i] + b - lse[i])
        g[i] = scale * counted[i] * p[i]
        g[i, int(labels[i])] -= scale * counted[i]
    return (g @ wc, g.T @ hc, g.sum(0)), (np.abs(g) @ np.abs(wc), np.abs(g).T @ np.abs(hc),
                                          np.abs(g).sum(0))


def adamw(p, g, m, v, step, lr, beta1, beta2, eps, weight_decay, grad_scale=1.0):
    """(p, m, v) after one step."""
    p, m, v = (np.asarray(t, np.float64) for t in (p, m, v))
    g = np.asarray(g, np.float64) * grad_scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    mh, vh = m / (1 - beta1 ** step), v / (1 - beta2 ** step)
    return p - lr * (mh / (np.sqrt(vh) + eps) + weight_decay * p), m, v


def adamw_f32(p, g, m, v, step, lr, beta1, beta2, eps, weight_decay, grad_scale=1.0,
              largest=np.float32(np.inf)):
    """The same with every product and sum rounded to float32, in the order of
    include/huge.h: the kernels' states are these bit for bit.  An element keeps its
    values where one of the new ones is not finite (the parameter: not below `largest`,
    which a narrower type of parameters rounds to infinity)."""
    f = np.float32
    p, g, m, v = (np.asarray(t, f) for t in (p, g, m, v))
    with np.errstate(over="ignore", invalid="ignore"):
        g = g * f(grad_scale)
        mn = m * f(beta1) + g * f(1 - beta1)
        vn = v * f(beta2) + (g * g) * f(1 - beta2)
        rate, fix = f(lr / (1 - beta1 ** step)), f(1 / np.sqrt(1 - beta2 ** step))
        new = p * f(1 - lr * weight_decay) - (mn * rate) / (np.sqrt(vn) * fix + f(eps))
        ok = np.isfinite(mn) & np.isfinite(vn) & (np.abs(new) < largest)
    return np.where(ok, new, p), np.where(ok, mn, m), np.where(ok, vn, v), ok


def q8_f32(m, v, block=256):
    """The values that moments in 8 bits stand for, in float32 arithmetic."""
    f = np.float32
    m, r = np.asarray(m, f).ravel(), np.sqrt(np.asarray(v, f).ravel())
    mo, vo = np.zeros_like(m), np.zeros_like(m)
    for a in range(0, m.size, block):
        mb, rb = m[a:a + block], r[a:a + block]
        s, t = np.abs(mb).max(), rb.max()
        inv_s, inv_t = (f(1) / s if s > 0 else f(0)), (f(1) / t if t > 0 else f(0))
        q = np.rint(np.sqrt(np.abs(mb) * inv_s) * f(127))
        u = np.rint(np.sqrt(rb * inv_t) * f(255))
        u = np.where(rb > 0, np.maximum(u, f(1)), u)
        k = q * (f(1) / f(127))
        c = u * (f(1) / f(255))
        root = t * (c * c)
        mo[a:a + block] = np.sign(mb) * (s * (k * k))
        vo[a:a + block] = root * root
    return mo, vo
