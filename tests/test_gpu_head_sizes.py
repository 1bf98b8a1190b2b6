"""The exact softmax loss at sizes that take more than one launch."""
import pytest

torch = pytest.importorskip("torch")

import paper_2307_14490_amd as P  # noqa: E402
from gpu_common import say  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def test_more_rows_than_threads_of_one_launch():
    """2^28 + 37 rows: 16 threads a row would be more than 2^32 - 1 of them."""
    n, classes, dim = 2 ** 28 + 37, 3, 4
    say(f"softmax loss {n} x {classes} x {dim} bf16")
    g = torch.Generator(device="cuda").manual_seed(5)
    h = torch.empty((n, dim), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    w = torch.randn((classes, dim), device="cuda", generator=g).bfloat16()
    labels = torch.randint(-1, classes, (n,), device="cuda", generator=g, dtype=torch.int32)
    bias = torch.randn(classes, device="cuda", generator=g)
    op = P.SoftmaxLoss(n, classes, dim, dtype="bf16", grad=False)
    loss, lse = op.loss(h, w, labels, bias)
    op.check()
    # a logit's sum of 4 products and the bias, then the sum of 3 exponentials, the
    # logarithm and the difference, each rounded to 2^-24
    u = 2.0 ** -24
    step = 2 ** 24
    for a in range(0, n, step):
        hv, y = h[a:a + step].double(), labels[a:a + step].long()
        x = hv @ w.double().t().contiguous() + bias.double()
        size = (hv.abs() @ w.double().abs().t().contiguous() + bias.double().abs()).amax(1)
        want = torch.logsumexp(x, 1)
        bound = u * (12 * size + 64 + 8 * want.abs())
        assert ((lse[a:a + step].double() - want).abs() <= bound).all(), a
        want = torch.where(y >= 0, want - x.gather(1, y.clamp(min=0)[:, None])[:, 0], 0.0)
        assert ((loss[a:a + step].double() - want).abs() <= 3 * bound).all(), a
