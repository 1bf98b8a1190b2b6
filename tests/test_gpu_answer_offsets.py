"""RMS norm with the residual's addition and its gradient beyond 2^31 elements: rows that
differ, so that an offset that wraps shows, each as a call on a copy of it gives it."""
import pytest

torch = pytest.importorskip("torch")

import paper_2307_14490_amd as P  # noqa: E402
from gpu_common import say  # noqa: E402
from test_gpu_answer import _need_gpu  # noqa: E402,F401

pytestmark = pytest.mark.gpu

N, DIM = 300_000, 8192  # 2^31 elements end at row 262144


@pytest.fixture(scope="module")
def arrays():
    """x, residual, dy and dtotal: a row each, times factors that no two of 251 rows share."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    out = []
    for k in range(4):
        row = torch.randn((1, DIM), device="cuda", generator=gen).to(torch.bfloat16)
        turn = (torch.arange(N, device="cuda") * (k + 1) % 251).float()
        out.append(row * (0.5 + turn / 128).to(torch.bfloat16)[:, None])
        out[-1][-1, 0] = 3.0 + k  # the last row is like no other
    gamma = torch.linspace(0.5, 1.5, DIM, device="cuda")
    yield (*out, gamma)
    del out
    torch.cuda.empty_cache()


PARTS = [slice(0, 3), slice(131_070, 131_075), slice(262_140, 262_150), slice(N - 40, N)]


def test_rms_norm_of_rows_that_differ(arrays):
    x, res, _, _, gamma = arrays
    say(f"rms norm with residual, {N} x {DIM} bf16")
    y, total, rstd = P.rms_norm(x, gamma, residual=res)
    q, total8, rstd8 = P.rms_norm(x, gamma, residual=res, q8=True)
    assert torch.equal(total, total8) and torch.equal(rstd, rstd8)
    v = P.q8_values(q, "bf16")
    again = P.q8_rows(y)
    for part in PARTS:
        one, total1, rstd1 = P.rms_norm(x[part].clone(), gamma, residual=res[part].clone())
        assert torch.equal(y[part], one) and torch.equal(total[part], total1)
        assert torch.equal(rstd[part], rstd1)
        q1 = P.rms_norm(x[part].clone(), gamma, residual=res[part].clone(), q8=True)[0]
        b1 = P.q8_rows(one)
        for got, want in ((q, q1), (again, b1)):
            assert torch.equal(got.codes[part].view(torch.uint8), want.codes.view(torch.uint8))
            assert torch.equal(got.scales[part], want.scales)
        assert torch.equal(v[part], P.q8_values(q1, "bf16"))


def test_gradient_of_rms_norm_of_rows_that_differ(arrays):
    x, _, dy, dtotal, gamma = arrays
    say(f"gradient of rms norm, {N} x {DIM} bf16")
    _, _, rstd = P.rms_norm(x, gamma)
    dx, dgamma = P.rms_norm_backward(dy, x, gamma, rstd, dtotal=dtotal)
    for part in PARTS:
        one, _ = P.rms_norm_backward(dy[part].clone(), x[part].clone(), gamma, rstd[part].clone(),
                                     dtotal=dtotal[part].clone())
        assert torch.equal(dx[part], one)
    want = torch.zeros(DIM, device="cuda", dtype=torch.float64)
    size = torch.zeros_like(want)
    for i in range(0, N, 10_000):
        z = dy[i:i + 10_000].double() * (x[i:i + 10_000].double()
                                         * rstd[i:i + 10_000].double()[:, None])
        want += z.sum(0)
        size += z.abs().sum(0)
    # a product's rounding; the rows of one of 1024 workgroups in sequence, then their sums, 32 and 32
    assert ((dgamma.double() - want).abs() <= (1 + N / 1024 + 1 + 64) * 2.0 ** -24 * size).all()
