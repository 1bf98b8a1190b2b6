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
