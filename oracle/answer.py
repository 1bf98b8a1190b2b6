"""Plain numpy definitions, in float64, of what a softmax head normalises, answers and
clips with: RMS norm, rows in 8 bits, log probabilities with entropy and the most
likely classes, and the norm over gradients.  They share no code with the kernels and
follow the formulas of include/huge.h line by line.
"""
from __future__ import annotations

import numpy as np


def rms_norm(total, gamma, eps):
    """(y, rstd) of the rows total."""
    total = np.asarray(total, np.float64)
    rstd = 1.0 / np.sqrt((total ** 2).mean(1) + eps)
    return total * rstd[:, None] * gamma, rstd


def rms_norm_backward(dy, total, gamma, rstd, dtotal=None):
    """(dx, dgamma)."""
    dy, total = np.asarray(dy, np.float64), np.asarray(total, np.float64)
    z, a = total * rstd[:, None], dy * gamma
    dx = rstd[:, None] * (a - z * (a * z).mean(1)[:, None])
    return dx if dtotal is None else dx + dtotal, (dy * z).sum(0)


def e4m3_values():
    """The values of the 128 codes without a sign; the last is NaN."""
    c = np.arange(128)
    e, m = c >> 3, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v[127] = np.nan
    return v


def q8_rows(x, block=32, least=-100):
    """(codes, scales) of the rows x, by search among all codes."""
    x = np.asarray(x, np.float64)
    n, dim = x.shape
    table = e4m3_values()[:127]
    codes = np.zeros((n, dim), np.uint8)
    scales = np.zeros((n, -(-dim // block)), np.uint8)
    for i in range(n):
        for b in range(scales.shape[1]):
            v = x[i, b * block:(b + 1) * block]
            if not np.isfinite(v).all():
                scales[i, b], codes[i, b * block:b * block + v.size] = 255, 127
                continue
            e = least
            while np.abs(v).max() > 448 * 2.0 ** e:
                e += 1
            a = np.abs(v) / 2.0 ** e
            hi = np.clip(np.searchsorted(table, a), 0, 126)
            lo = np.maximum(hi - 1, 0)
            up = (table[hi] - a < a - table[lo]) | ((table[hi] - a == a - table[lo]) & (hi % 2 == 0))
            codes[i, b * block:b * block + v.size] = np.where(up, hi, lo) | (np.signbit(v) << 7)
            scales[i, b] = e + 127
    return codes, scales


def q8_values(codes, scales, block=32):
    codes, scales = np.asarray(codes), np.asarray(scales)
    v = e4m3_values()[codes & 127] * np.where(codes & 128, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(s, block, 1)[:, :codes.shape[1]]


def logits(h, w, bias=None):
    """x, -inf where a class is out; what is in its row of w is not used."""
    h, w = np.asarray(h, np.float64), np.asarray(w, np.float64)
    b = np.zeros(len(w)) if bias is None else np.asarray(bias, np.float64)
    x = np.full((len(h), len(w)), -np.inf)
    kept = np.flatnonzero(~(b < -1e28))
    for i in range(len(h)):
        x[i, kept] = w[kept] @ h[i] + b[kept]
    return x


def log_probs(h, w, labels=None, bias=None, top=0):
    """(logp, entropy, lse, ids, top_logp)."""
    x = logits(h, w, bias)
    n = len(x)
    lse, entropy, logp = np.full(n, -np.inf), np.zeros(n), np.zeros(n)
    ids, best = np.full((n, top), -1), np.full((n, top), -np.inf)
    for i in range(n):
        kept = np.flatnonzero(x[i] != -np.inf)
        v = x[i, kept]
        if kept.size:
            if not np.isfinite(v).all():
                lse[i] = entropy[i] = np.nan
                best[i] = np.nan
            else:
                lse[i] = v.max() + np.log(np.exp(v - v.max()).sum())
                p = np.exp(v - lse[i])
                entropy[i] = -(p * (v - lse[i])).sum()
                order = kept[np.argsort(-v, kind="stable")][:top]
                ids[i, :order.size], best[i, :order.size] = order, x[i, order] - lse[i]
        if labels is not None:
            y = int(labels[i])
            if y < -1 or y >= x.shape[1]:
                logp[i] = np.nan
            elif y >= 0:
                logp[i] = -np.inf if x[i, y] == -np.inf else x[i, y] - lse[i]
    return logp, entropy, lse, ids, best


def log_probs_grad(h, w, labels, dlogp=None, dentropy=None, bias=None):
    """(dh, dw, dbias) of sum dlogp logp + dentropy entropy, and what bounds the rounding of
    an element of G: its terms' absolute values, and |dentropy| p."""
    h, w = np.asarray(h, np.float64), np.asarray(w, np.float64)
    n, classes = len(h), len(w)
    dl = np.zeros(n) if dlogp is None else np.array(dlogp, np.float64)
    de = np.zeros(n) if dentropy is None else np.asarray(dentropy, np.float64)
    b = np.zeros(classes) if bias is None else np.asarray(bias, np.float64)
    g, size, soft = (np.zeros((n, classes)) for _ in range(3))
    wc = np.where((b < -1e28)[:, None], 0.0, w)
    hc = np.zeros_like(h)
    for i in range(n):
        y = -1 if labels is None else int(labels[i])
        if y < 0 or y >= classes or b[y] < -1e28:
            dl[i] = 0.0
        kept = np.flatnonzero(~(b < -1e28))
        if (dl[i] == 0 and de[i] == 0) or not kept.size:
            continue
        hc[i] = h[i]
        x = wc[kept] @ h[i] + b[kept]
        lp = x - (x.max() + np.log(np.exp(x - x.max()).sum()))
        p = np.exp(lp)
        entropy = -(p * lp).sum()
        g[i, kept] = -dl[i] * p - de[i] * p * (lp + entropy)
        size[i, kept] = p * (abs(dl[i]) + abs(de[i]) * (np.abs(lp) + entropy))
        soft[i, kept] = abs(de[i]) * p
        if dl[i]:
            g[i, y] += dl[i]
            size[i, y] += abs(dl[i])
    return (g @ wc, g.T @ hc, g.sum(0)), size, soft, hc, wc


def grad_norm(grads):
    return np.sqrt(sum((np.asarray(g, np.float64) ** 2).sum() for g in grads))
