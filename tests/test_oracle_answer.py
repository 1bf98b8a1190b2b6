"""Pins of oracle/answer.py: gradients against differences, codes against torch's type,
entropies and orders against closed forms."""
import numpy as np
import pytest

from oracle import answer as ref


def test_rms_norm_gradient_is_the_difference():
    rng = np.random.default_rng(0)
    x, dy, dt = (rng.normal(size=(3, 7)) for _ in range(3))
    g = 1 + 0.3 * rng.normal(size=7)

    def value(x, g):
        return (ref.rms_norm(x, g, 1e-3)[0] * dy).sum() + (x * dt).sum()

    dx, dg = ref.rms_norm_backward(dy, x, g, ref.rms_norm(x, g, 1e-3)[1], dt)
    for i in range(3):
        for j in range(7):
            e = np.zeros_like(x)
            e[i, j] = 1e-6
            assert (value(x + e, g) - value(x - e, g)) / 2e-6 == pytest.approx(dx[i, j], abs=1e-7)
    for j in range(7):
        e = np.zeros(7)
        e[j] = 1e-6
        assert (value(x, g + e) - value(x, g - e)) / 2e-6 == pytest.approx(dg[j], abs=1e-7)


def test_codes_are_those_of_the_type():
    torch = pytest.importorskip("torch")
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    v = ref.q8_values(np.arange(256, dtype=np.uint8)[None], np.full((1, 8), 127, np.uint8))[0]
    np.testing.assert_array_equal(v, t)
    x = np.random.default_rng(1).normal(size=(50, 32)) * 100
    x[:, 0] = 448.0  # scale 1
    codes, scales = ref.q8_rows(x)
    assert (scales == 127).all()
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    x32 = x.astype(np.float32).astype(np.float64)
    np.testing.assert_array_equal(ref.q8_rows(x32)[0], want)
    # an error of half a step, the last scale's that holds the largest
    y = np.random.default_rng(2).normal(size=(40, 70)) * 10.0 ** np.arange(-20, 20)[:, None]
    v = ref.q8_values(*ref.q8_rows(y))
    most = np.stack([np.abs(y[:, k:k + 32]).max(1) for k in (0, 32, 64)], 1)
    assert (np.abs(v - y) <= np.maximum(np.abs(y) * 2.0 ** -4,
                                        np.repeat(most, 32, 1)[:, :70] * 2.0 ** -17)).all()


def test_entropy_and_order():
    h = np.zeros((1, 4))
    w = np.random.default_rng(3).normal(size=(9, 4))
    logp, entropy, lse, ids, best = ref.log_probs(h, w, [5], top=4)
    assert lse[0] == pytest.approx(np.log(9)) and entropy[0] == pytest.approx(np.log(9))
    assert logp[0] == pytest.approx(-np.log(9)) and ids[0].tolist() == [0, 1, 2, 3]
    b = np.full(9, -np.inf)
    logp, entropy, lse, ids, best = ref.log_probs(h, w, [5], b, top=2)
    assert lse[0] == -np.inf and entropy[0] == 0 and logp[0] == -np.inf and (ids == -1).all()
    b[[6, 2]] = [0.0, np.log(3)]
    w[0] = np.nan  # out
    logp, entropy, lse, ids, best = ref.log_probs(h, w, [6], b, top=3)
    assert logp[0] == pytest.approx(np.log(0.25)) and ids[0].tolist() == [2, 6, -1]
    assert entropy[0] == pytest.approx(-0.25 * np.log(0.25) - 0.75 * np.log(0.75))
    assert best[0, 2] == -np.inf


def test_gradient_is_the_difference():
    rng = np.random.default_rng(4)
    n, classes, dim = 4, 6, 3
    h, w, b = rng.normal(size=(n, dim)), rng.normal(size=(classes, dim)), rng.normal(size=classes)
    b[1] = -np.inf
    labels = np.array([0, 5, -1, 1])  # one without, one whose label is out
    dl, de = rng.normal(size=n), rng.normal(size=n)
    de[1] = 0.0

    def value(h, w, b):
        logp, entropy, *_ = ref.log_probs(h, w, labels, b)
        return (dl * np.where((labels >= 0) & (labels != 1), logp, 0.0)).sum() + (de * entropy).sum()

    grads = ref.log_probs_grad(h, w, labels, dl, de, b)[0]
    for k, t in enumerate((h, w, b)):
        for at in np.ndindex(t.shape):
            if not np.isfinite(t[at]):
                continue
            args = [h.copy(), w.copy(), b.copy()]
            args[k][at] += 1e-6
            up = value(*args)
            args[k][at] -= 2e-6
            assert (up - value(*args)) / 2e-6 == pytest.approx(grads[k][at], abs=1e-7)


def test_grad_norm():
    assert ref.grad_norm([np.array([3.0]), np.array([[4.0, 12.0]])]) == 13.0
