"""The softmax head's oracle against central differences, closed forms and torch's
autograd in float64 (CPU)."""
import math

import numpy as np
import pytest
import torch

from oracle import head as ref


def _difference(f, x, at, step=1e-6):
    a, b = x.copy(), x.copy()
    a[at] += step
    b[at] -= step
    return (f(a) - f(b)) / (2 * step)


def test_layer_norm_gradient_is_the_difference_quotient():
    rng = np.random.default_rng(1)
    x, g, b = rng.normal(size=(5, 7)) + 0.4, rng.normal(size=7), rng.normal(size=7)
    dy = rng.normal(size=(5, 7))
    _, mean, rstd = ref.layer_norm(x, g, b, 1e-5)
    dx, dg, db = ref.layer_norm_backward(dy, x, g, mean, rstd)
    for at in np.ndindex(5, 7):
        assert abs(dx[at] - _difference(lambda t: (ref.layer_norm(t, g, b, 1e-5)[0] * dy).sum(),
                                        x, at)) < 1e-7
    for k in range(7):
        assert abs(dg[k] - _difference(lambda t: (ref.layer_norm(x, t, b, 1e-5)[0] * dy).sum(),
                                       g, k)) < 1e-7
        assert abs(db[k] - _difference(lambda t: (ref.layer_norm(x, g, t, 1e-5)[0] * dy).sum(),
                                       b, k)) < 1e-7


def test_softmax_gradient_is_the_difference_quotient():
    rng = np.random.default_rng(2)
    h, w, b = rng.normal(size=(6, 4)), rng.normal(size=(9, 4)), rng.normal(size=9)
    b[3] = -np.inf
    labels = np.array([0, 8, -1, 3, 5, 5])
    c = np.array([1.0, 2.5, 1.0, 1.0, 0.0, 0.5])
    (dh, dw, db), _ = ref.softmax_grad(h, w, labels, b, c, scale=0.25)

    def total(h_, w_, b_):
        return 0.25 * ref.softmax_loss(h_, w_, labels, b_, c)[0].sum()

    for at in np.ndindex(6, 4):
        assert abs(dh[at] - _difference(lambda t: total(t, w, b), h, at)) < 1e-7
    for at in np.ndindex(9, 4):
        assert abs(dw[at] - _difference(lambda t: total(h, t, b), w, at)) < 1e-7
    for k in range(9):
        if k != 3:
            assert abs(db[k] - _difference(lambda t: total(h, w, t), b, k)) < 1e-7
    assert db[3] == 0 and not dw[3].any()


def test_softmax_loss_against_autograd():
    rng = np.random.default_rng(3)
    h, w, b = rng.normal(size=(12, 8)), rng.normal(size=(20, 8)), rng.normal(size=20)
    labels = rng.integers(0, 20, 12)
    th, tw, tb = (torch.tensor(t, requires_grad=True) for t in (h, w, b))
    loss = torch.nn.functional.cross_entropy(th @ tw.t() + tb, torch.tensor(labels),
                                             reduction="sum")
    loss.backward()
    got, lse, _ = ref.softmax_loss(h, w, labels, b)
    assert abs(got.sum() - loss.item()) < 1e-10
    np.testing.assert_allclose(lse, torch.logsumexp(th @ tw.t() + tb, 1).detach(), atol=1e-12)
    grads, _ = ref.softmax_grad(h, w, labels, b)
    for g, t in zip(grads, (th, tw, tb)):
        np.testing.assert_allclose(g, t.grad, atol=1e-12)


def test_softmax_closed_forms():
    """Zero rows: log V, and p = 1/V; one class: no loss; nothing left: no loss."""
    h, w = np.zeros((3, 4)), np.random.default_rng(4).normal(size=(7, 4))
    loss, lse, _ = ref.softmax_loss(h, w, [0, 6, -1])
    np.testing.assert_allclose(lse, math.log(7))
    np.testing.assert_allclose(loss, [math.log(7), math.log(7), 0])
    assert ref.softmax_loss(h, w[:1], [0, 0, 0])[0].max() == 0
    loss, lse, counted = ref.softmax_loss(h, w, [0, 1, 2], np.full(7, -np.inf))
    assert not loss.any() and (lse == -np.inf).all() and not counted.any()


def test_adamw_first_step_is_the_sign():
    """From zero moments the first step is lr g / (|g| + eps), whatever the betas."""
    g = np.array([1e-3, -5.0, 0.0, 2.0])
    p, m, v = ref.adamw(np.ones(4), g, np.zeros(4), np.zeros(4), 1, 0.1, 0.9, 0.99, 1e-8, 0.0)
    np.testing.assert_allclose(p, 1 - 0.1 * g / (np.abs(g) + 1e-8), atol=1e-12)


def test_adamw_float32_form_and_float64_form_agree():
    rng = np.random.default_rng(5)
    f = np.float32
    p, g = rng.normal(size=500).astype(f), (rng.normal(size=500) * 1e-2).astype(f)
    m, v = (rng.normal(size=500) * 1e-2).astype(f), (rng.random(500) * 1e-4).astype(f)
    a = ref.adamw(p, g, m, v, 7, 1e-3, 0.9, 0.999, 1e-8, 0.01)
    b = ref.adamw_f32(p, g, m, v, 7, 1e-3, 0.9, 0.999, 1e-8, 0.01)
    # each of the few roundings is 2^-24 of a number no larger than these
    for x, y, big in zip(a, b, (np.abs(p) + 0.1, np.abs(m) + np.abs(g), v + g * g)):
        assert (np.abs(x - y) <= 16 * 2.0 ** -24 * big).all()


def test_adamw_against_torch():
    rng = np.random.default_rng(6)
    p0 = rng.normal(size=50)
    t = torch.nn.Parameter(torch.tensor(p0))
    opt = torch.optim.AdamW([t], lr=1e-2, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    p, m, v = p0, np.zeros(50), np.zeros(50)
    for step in range(1, 5):
        g = rng.normal(size=50)
        t.grad = torch.tensor(g)
        opt.step()
        p, m, v = ref.adamw(p, g, m, v, step, 1e-2, 0.8, 0.95, 1e-6, 0.1)
    np.testing.assert_allclose(p, t.detach().numpy(), rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("size", [1, 255, 256, 257, 1000])
def test_q8_values(size):
    """The largest of a block is kept, every value is within half a code's distance,
    no positive v becomes zero, and values that a code stands for stay."""
    rng = np.random.default_rng(size)
    f = np.float32
    m = (rng.normal(size=size) * np.exp(2 * rng.normal(size=size))).astype(f)
    v = (rng.normal(size=size) * np.exp(3 * rng.normal(size=size))).astype(f) ** 2
    mq, vq = ref.q8_f32(m, v)
    for a in range(0, size, 256):
        s, t = np.abs(m[a:a + 256]).max(), np.sqrt(v[a:a + 256]).max()
        # in the square root of the value, codes are 1/127 (1/255) apart
        em = np.abs(np.sqrt(np.abs(mq[a:a + 256]) / s) - np.sqrt(np.abs(m[a:a + 256]) / s))
        assert em.max() <= 0.5 / 127 + 1e-5
        ev = np.abs((vq[a:a + 256] / t ** 2) ** 0.25 - (v[a:a + 256] / t ** 2) ** 0.25)
        assert ev.max() <= 1.0 / 255 + 1e-5
    assert ((vq > 0) == (v > 0)).all()
    again = ref.q8_f32(mq, vq)
    np.testing.assert_array_equal(again[0], mq)
