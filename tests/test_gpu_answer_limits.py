"""Log probabilities, clipping and norms at the ends of what their calls take: large weights,
factors that no float holds, elements that are small beside their row's bound."""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_2307_14490_amd as P  # noqa: E402
from gpu_common import say  # noqa: E402
from test_gpu_answer import TYPES, _need_gpu  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def normal(*shape, seed=0):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,dim", [(5, 33, 16), (40, 64, 16), (80, 1001, 100),
                                           (70, 300, 400)])
def test_gradients_scale_with_large_weights(n, classes, dim, dtype):
    """Weights times a power of two give gradients times that power, bit for bit: no step
    rounds otherwise.  With classes that are out, and a last tile that is not whole."""
    h = normal(n, dim, seed=n).to(TYPES[dtype])
    w = (normal(classes, dim, seed=classes) * dim ** -0.5).to(TYPES[dtype])
    bias = normal(classes, seed=3)
    bias[[1, classes // 2]] = -math.inf
    labels = torch.arange(n, device="cuda", dtype=torch.int32) * 7 % classes
    op = P.LogProbs(n, classes, dim, dtype=dtype, grad=True)
    dl, de = normal(n, seed=1), normal(n, seed=2)
    for b in (None, bias):
        a = op.log_probs(h, w, labels, b)
        one = op.grad(h, w, a, labels, dl, de, b)
        assert all(t.isfinite().all() for t in one)
        for power in (2.0 ** 30, 2.0 ** 56):
            say(f"weights times {power:.3g}, {n} x {classes} x {dim} {dtype}, bias {b is not None}")
            for got, want in zip(op.grad(h, w, a, labels, dl * power, de * power, b), one):
                assert torch.equal(got.float(), want.float() * power)


# norms beyond the largest float, or so far above the largest wanted that the factor is below
# the smallest: an element of 1000 equal ones becomes max_norm / sqrt(1000)
FAR = [(3e38, 1.0), (3e38, 1e-3), (1e38, 1e-2), (3e38, 1e-6), (3e38, 1e-12), (2e30, 1e-12)]
U = 2.0 ** -24


def equal_gradients(value, dtype, offset):
    return torch.full((1003,), value, device="cuda", dtype=TYPES[dtype])[offset:offset + 1000]


@pytest.mark.parametrize("value,most", FAR)
@pytest.mark.parametrize("dtype,offset", [("f32", 0), ("f32", 3), ("bf16", 0), ("bf16", 1)])
def test_clipping_by_factors_that_no_float_holds(value, most, dtype, offset):
    g = equal_gradients(value, dtype, offset)
    v = g[0].double().item()
    norm = P.clip_grads([g], most)
    full = v * 1000 ** 0.5
    assert norm.item() == (math.inf if full > 3.4028235e38 else pytest.approx(full, rel=2 * U))
    # the factor's rounding, the product's, and half a step of bf16
    want = most / 1000 ** 0.5
    rel = 3 * U + (2.0 ** -8 if dtype == "bf16" else 0.0)
    assert ((g.double() - want).abs() <= rel * want).all(), (g[0].item(), want)


@pytest.mark.parametrize("states", ["f32", "q8"])
@pytest.mark.parametrize("value,most", FAR)
@pytest.mark.parametrize("dtype,offset", [("f32", 0), ("f32", 3), ("bf16", 0)])
def test_clipped_steps_by_factors_that_no_float_holds(value, most, dtype, offset, states):
    """As steps with the scaled gradients themselves, beta1 and beta2 0: the moments are a
    gradient and its square."""
    g = equal_gradients(value, dtype, offset)
    p = normal(1000, seed=4)
    opt = P.AdamW([p], betas=(0.0, 0.0), states=states, weight_decay=0.0, lr=0.25)
    before = p.clone()
    opt.step([g], max_norm=most)
    opt.check()
    m, v = opt.values()
    want = most / 1000 ** 0.5
    # 8 bits: 7 bits of a square root, whose largest (here: every) element is a code itself
    assert ((m[0].double() - want).abs() <= 8 * U * want).all()
    assert ((v[0].double() - want ** 2).abs() <= 16 * U * want ** 2 + 2.0 ** -149).all()
    # m / (sqrt v + eps) = 1 / (1 + eps / want)
    moved = 0.25 / (1 + 1e-8 / want)
    assert ((before - p).double() - moved).abs().max().item() <= 8 * U * (0.25 + 4)


def by_bias(bias):
    """Probabilities, their logarithms and the entropy of logits that are the bias, in fp64."""
    x = bias.double()
    logp = x - torch.logsumexp(x, 0)
    p = logp.exp()
    return p, logp, -(p * logp).sum()


def test_elements_of_the_rows_gradient_are_within_what_is_stated():
    """Elements far below what their row's can be, one in each column of dh: rows whose logits
    are the bias alone, and classes whose rows have a single 1."""
    classes, dim = 64, 32
    bias = torch.full((classes,), -40.0, device="cuda")
    bias[0] = 0.0
    bias[1:32] = -torch.linspace(18, 34, 31, device="cuda")
    w = torch.zeros(classes, dim, device="cuda", dtype=torch.bfloat16)
    w[1:32, :31] = torch.eye(31, device="cuda", dtype=torch.bfloat16)
    h = torch.zeros(40, dim, device="cuda", dtype=torch.bfloat16)
    h[:, 31] = 1.0
    op = P.LogProbs(40, classes, dim, dtype="bf16", grad=True)
    a = op.log_probs(h, w, bias=bias)
    de = torch.linspace(0.5, 2.0, 40, device="cuda")
    dh = op.grad(h, w, a, dentropy=de, bias=bias)[0].double()
    p, logp, entropy = by_bias(bias)
    g = (-p * (logp + entropy) * de.double()[:, None])[:, 1:32]
    most = 0.4 * de.double()[:, None] + (entropy * de.double()[:, None]).abs()
    # the logarithm's and the exponent's roundings, at logits of 40; of fp16, of bf16
    err = (dh[:, :31] - g).abs()
    assert (err <= g.abs() * (2.0 ** -8 + 2.0 ** -11 + 256 * U) + most * 2.0 ** -36).all()
    # and there they show
    assert (err > g.abs() * 2.0 ** -6).any()


def test_elements_of_the_classes_gradient_are_within_what_is_stated():
    """Rows whose weights fall by 2^-31, each in a column of dw of its own."""
    classes, dim, n = 40, 32, 31
    bias = torch.linspace(-3, 0, classes, device="cuda")
    w = torch.zeros(classes, dim, device="cuda", dtype=torch.bfloat16)
    h = torch.eye(dim, device="cuda", dtype=torch.bfloat16)[:n].contiguous()
    op = P.LogProbs(n, classes, dim, dtype="bf16", grad=True)
    a = op.log_probs(h, w, bias=bias)
    de = torch.tensor([2.0 ** -i * (1 + i / 37) for i in range(n)], device="cuda")
    dw = op.grad(h, w, a, dentropy=de, bias=bias)[1].double()
    p, logp, entropy = by_bias(bias)
    at = -p * (logp + entropy)
    g = at[:, None] * de.double()[None, :]
    size = (p * (logp.abs() + entropy))[:, None] * de.double()[None, :]  # terms that cancel
    err = (dw[:, :n] - g).abs()
    assert (err <= g.abs() * (2.0 ** -8 + 2.0 ** -11) + 64 * U * size
            + g.abs().max(1, keepdim=True).values * 2.0 ** -35).all()
    # and there they show: up to 2^-35 of the first of an element 2^-30 (1 + 30 / 37) of it, which is
    # 2^-5.86, where bf16 and fp16 alone round by 2^-7.83 at most
    assert (err > g.abs() * 2.0 ** -7.5).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [5, 40, 80])
def test_a_logit_of_minus_infinity_beside_finite_ones(n, dtype):
    """An infinity in the row of a class that counts: no entropy, and lse and classes either
    those of the others or none."""
    h = normal(n, 16, seed=5).abs().add_(0.1).to(TYPES[dtype])
    w = normal(200, 16, seed=6).to(TYPES[dtype])
    op = P.LogProbs(n, 200, 16, dtype=dtype, top=4)
    out = torch.zeros(200, device="cuda")
    out[7] = -math.inf
    want = op.log_probs(h, w, bias=out)
    w[7, 3] = -math.inf
    a = op.log_probs(h, w)
    assert a.entropy.isnan().all()
    for i in range(n):
        if a.lse[i].isnan():
            assert (a.ids[i] == -1).all() and a.top_logp[i].isnan().all()
        else:
            assert torch.equal(a.ids[i], want.ids[i])
            assert torch.allclose(a.lse[i], want.lse[i], rtol=1e-5, atol=1e-5)
            assert torch.allclose(a.top_logp[i], want.top_logp[i], rtol=1e-5, atol=1e-5)


def test_rows_in_8_bits_beyond_the_largest_float():
    """A norm times gamma that no float holds makes its block NaN, as an infinity does."""
    x = torch.ones(3, 64, device="cuda")
    x[1, 40] = 8.0
    gamma = torch.ones(64, device="cuda")
    gamma[40] = 3e38
    y, _, _ = P.rms_norm(x, gamma, q8=True)
    v = P.q8_values(y)
    # row 1: squares of 63 ones and 64: 8 / sqrt(127 / 64) = 5.7 times 3e38
    assert v[1, 32:].isnan().all() and not v[1, :32].isnan().any()
    assert not v[[0, 2]].isnan().any()
    near = (v[0, 40].double() / 3e38 - 1).abs().item()
    assert near <= 2.0 ** -4 + 1e-5  # half a step of e4m3; eps


@pytest.mark.parametrize("states", ["f32", "q8"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_clipped_steps_leave_the_moments_of_scaled_gradients(states, dtype):
    """Moments, not parameters, which hardly show the factor.  In 8 bits a moment is a code under
    its block's scale: the scales follow the factor, and the codes are the same but where its
    last bit moves one across a border."""
    sizes = [300, 5000, 16385, 1]
    gs = [normal(n, seed=n).mul_(10.0 ** (k - 2)).to(TYPES[dtype]) for k, n in enumerate(sizes)]
    norm = math.sqrt(sum(g.double().square().sum().item() for g in gs))
    for most, scale in ((0.25 * norm, 1.0), (0.03 * norm, -2.0), (10 * norm, 0.5)):
        a, b, c = (P.AdamW([torch.zeros(n, device="cuda") for n in sizes], states=states)
                   for _ in range(3))
        f = scale * min(1.0, most / (abs(scale) * norm))
        a.step(gs, max_norm=most, grad_scale=scale)
        b.step(gs, grad_scale=f)
        c.step(gs, grad_scale=1.01 * f)
        for x, y, z in zip(*([*o.values()[0], *o.values()[1]] for o in (a, b, c))):
            # the factor's rounding, and some each of the moment's and the scale's
            far = ((x - y).abs() > 16 * U * y.abs()).double().mean().item()
            assert far <= (0.0 if states == "f32" else 0.002), far
            if x.numel() > 1:  # a hundredth more does not pass
                assert ((z - y).abs() > 16 * U * y.abs()).double().mean().item() > 0.5


@pytest.mark.parametrize("dtype", ["f32", "bf16", "q8"])
@pytest.mark.parametrize("n", [5, 40, 80])
def test_zeros_of_either_sign_are_equals(n, dtype):
    """Rows of zeros and biases of -0 in the first half: the lowest classes all the same."""
    classes, dim, top = 4000, 32, 20
    h = torch.zeros(n, dim, device="cuda", dtype=TYPES["bf16" if dtype == "q8" else dtype])
    w = normal(classes, dim, seed=8).abs().neg().to(h.dtype)
    bias = torch.zeros(classes, device="cuda")
    bias[: classes // 2] = -0.0
    op = P.LogProbs(n, classes, dim, dtype=dtype, top=top)
    a = op.log_probs(h, P.q8_rows(w) if dtype == "q8" else w, bias=bias)
    assert (a.ids == torch.arange(top, device="cuda", dtype=torch.int32)).all()
