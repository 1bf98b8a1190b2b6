"""Log probabilities of more classes and rows than are taken at once, and norms beyond 2^31
elements, against float64 on the GPU."""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_2307_14490_amd as P  # noqa: E402
from gpu_common import say  # noqa: E402
from test_gpu_answer import TYPES, _need_gpu, on_device  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def make(n, classes, dim, dtype, bias, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = TYPES["bf16" if dtype == "q8" else dtype]
    h = torch.randn((n, dim), device="cuda", generator=g).to(kind)
    w = (torch.randn((classes, dim), device="cuda", generator=g) * 1.5 / math.sqrt(dim)).to(kind)
    lab = torch.randint(0, classes, (n,), device="cuda", generator=g).to(torch.int32)
    b = torch.randn(classes, device="cuda", generator=g) if bias else None
    return h, w, lab, b


def close(a, want, rows=slice(None)):
    """ids as they are, the rest within a few fp32 roundings of sums of many terms."""
    assert torch.equal(a.ids[rows].long(), want[3])
    for x, y in ((a.logp, want[0]), (a.entropy, want[1]), (a.lse, want[2]), (a.top_logp, want[4])):
        assert ((x[rows].double() - y).abs().max() / y.abs().max()).item() <= 1e-5


@pytest.mark.parametrize("dtype,bias", [("bf16", False), ("bf16", True), ("f32", True),
                                        ("q8", False)])
def test_more_classes_than_a_piece(dtype, bias):
    """Three pieces of the vocabulary, whose last is a part of one."""
    n, classes, dim, top = 70, 2 * 32768 * 32 + 12_345, 32, 12
    say(f"pieces of {classes} classes, {dtype}, bias {bias}")
    h, w, lab, b = make(n, classes, dim, dtype, bias, 5)
    table = w
    if dtype == "q8":
        table = P.q8_rows(w)
        w = P.q8_values(table)
    op = P.LogProbs(n, classes, dim, dtype=dtype, top=top)
    a = op.log_probs(h, table, lab, b)
    close(a, on_device(h, w, lab, b, top))
    same = op.log_probs(h, table, lab, b)
    assert all(torch.equal(x, y) for x, y in zip(a, same))
    op.check()


@pytest.mark.parametrize("top", [5, 64])
def test_more_classes_than_a_piece_for_one_row(top):
    """More than 2^24 tiles of 16, with offsets past 32 bits."""
    classes, dim = (1 << 24) * 16 + 1_000_003, 8
    say(f"pieces of {classes} classes for one row, best {top}")
    g = torch.Generator(device="cuda").manual_seed(6)
    codes = torch.randint(0, 120, (classes, dim), device="cuda", generator=g, dtype=torch.uint8)
    codes |= torch.randint(0, 2, (classes, dim), device="cuda", generator=g,
                           dtype=torch.uint8) << 7
    scales = torch.randint(118, 121, (classes, 1), device="cuda", generator=g, dtype=torch.uint8)
    table = P.Q8Rows(codes.view(torch.float8_e4m3fn), scales)
    h = torch.randn(1, dim, device="cuda", generator=g).to(torch.bfloat16)
    lab = torch.tensor([classes - 2], dtype=torch.int32, device="cuda")
    op = P.LogProbs(1, classes, dim, dtype="q8", top=top)
    a = op.log_probs(h, table, lab)
    w = P.q8_values(table)
    x = torch.cat([(w[i:i + (1 << 25)].double() * h[0].double()).sum(1)
                   for i in range(0, classes, 1 << 25)])
    del w
    lse = torch.logsumexp(x, 0)
    v, ids = torch.topk(x, top)
    assert a.ids[0].tolist() == ids.tolist()
    assert abs(a.lse.item() - lse.item()) <= 1e-5 * abs(lse.item())
    assert abs(a.logp.item() - (x[lab.long()] - lse).item()) <= 1e-5 * abs(lse.item())
    assert (a.top_logp[0].double() - (v - lse)).abs().max().item() <= 1e-5 * abs(lse.item())
    p = (x - lse).exp_()
    entropy = -(p * (x - lse)).sum().item()
    assert abs(a.entropy.item() - entropy) <= 1e-5 * lse.item()
    op.check()


@pytest.mark.parametrize("dtype,bias", [("bf16", False), ("f32", True)])
def test_more_rows_than_are_taken_at_once(dtype, bias):
    """The tiles' largest logits of all rows would take more than 1 GiB."""
    n, classes, dim, top = 43_111, 200_003, 32, 3
    say(f"pieces of {n} rows, {dtype}")
    h, w, lab, b = make(n, classes, dim, dtype, bias, 7)
    op = P.LogProbs(n, classes, dim, dtype=dtype, top=top)
    a = op.log_probs(h, w, lab, b)
    for rows in (slice(0, 50), slice(42_930, 42_960), slice(n - 60, n)):
        close(a, on_device(h[rows], w, lab[rows], b, top), rows)
    op.check()


def test_norm_of_more_than_2_to_the_32_bytes():
    """Offsets past 32 bits, the last element alone."""
    n = (1 << 31) + 5000
    say(f"norm of {n} elements")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-1] = 3.0
    assert P.grad_norm([g]).item() == 3.0
    g[7] = 4.0
    assert P.clip_grads([g, torch.zeros(3, device="cuda")], 1.0).item() == 5.0
    # bf16 values nearest to 0.6 and 0.8
    assert g[-1].item() == torch.tensor(0.6).bfloat16().item()
    assert g[7].item() == torch.tensor(0.8).bfloat16().item()


def test_rms_norm_of_more_than_2_to_the_31_elements():
    n, dim = 300_000, 8192
    say(f"rms norm of {n} x {dim}")
    x = torch.randn((1, dim), device="cuda").to(torch.bfloat16).expand(n, dim).contiguous()
    g = torch.ones(dim, device="cuda")
    y, _, rstd = P.rms_norm(x, g)
    assert torch.equal(y[0], y[-1]) and (rstd == rstd[0]).all()
    want = P.rms_norm(x[:1].clone(), g)[0]
    assert torch.equal(y[-1:], want)
    q, _, _ = P.rms_norm(x, g, q8=True)
    assert torch.equal(q.codes[-1].view(torch.uint8), q.codes[0].view(torch.uint8))
    assert torch.equal(P.q8_values(q, "bf16")[-1], P.q8_values(P.Q8Rows(q.codes[:1], q.scales[:1]), "bf16")[0])


@pytest.mark.parametrize("dim,dtype,n", [(32, "f32", 270_000), (128, "bf16", 140_001),
                                         (257, "f32", 40_003), (1500, "f32", 9001),
                                         (2000, "bf16", 17_000)])
def test_rms_norm_in_8_bits_of_several_rows_a_workgroup(dim, dtype, n):
    """More rows than workgroups take at once: the same as in parts that are not."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    x = torch.randn((n, dim), device="cuda", generator=gen)
    x = x.to(torch.bfloat16) if dtype == "bf16" else x
    res = x.flip(0)
    gamma = torch.linspace(0.5, 1.5, dim, device="cuda")
    y, total, rstd = P.rms_norm(x, gamma, residual=res, q8=True)
    step = 4000
    for a in range(0, n, step):
        part = slice(a, a + step)
        y1, total1, rstd1 = P.rms_norm(x[part], gamma, residual=res[part], q8=True)
        assert torch.equal(y1.codes.view(torch.uint8), y.codes[part].view(torch.uint8))
        assert torch.equal(y1.scales, y.scales[part])
        assert torch.equal(total1, total[part]) and torch.equal(rstd1, rstd[part])
