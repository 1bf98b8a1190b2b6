"""The softmax head's operators against the float64 oracle (oracle/head.py), through
the package's entry points and, where pointers matter, the C ABI.

Tolerances come from the roundings that the definitions in include/huge.h leave
open: u = 2^-24 per fp32 operation times the sum of the absolute terms, a dot
product of D terms counted as D u (its worst case), and half a bf16 step, 2^-8 of
the value, for each rounding to bf16.
"""
import ctypes
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2307_14490_amd as P  # noqa: E402
from paper_2307_14490_amd import binding as B  # noqa: E402
from oracle import head as ref  # noqa: E402
from gpu_common import say  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF = 2.0 ** -8
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def within(got, want, bound, what):
    g = got.detach().double().cpu().numpy() if isinstance(got, torch.Tensor) else got
    assert g.shape == np.shape(want), what
    same = np.isfinite(want)
    np.testing.assert_array_equal(np.isfinite(g), same, err_msg=what)
    np.testing.assert_array_equal(g[~same], want[~same], err_msg=what)
    err = np.abs(g - want)[same] / np.broadcast_to(bound, g.shape)[same]
    worst = float(err.max()) if err.size else 0.0
    say(f"  {what}: largest error / bound {worst:.3g}")
    assert worst <= 1.0, what


def rows(a, dtype, pad=0, offset=0):
    """a (numpy) on the GPU as rows of a wider buffer that starts `offset` elements
    into an allocation; the rest of it is NaN.  Also its values after rounding."""
    n, d = a.shape
    flat = torch.full((offset + n * (d + pad) + 1,), math.nan, dtype=TYPES[dtype], device="cuda")
    t = flat[offset:offset + n * (d + pad)].view(n, d + pad)[:, :d]
    t.copy_(torch.from_numpy(a).to(TYPES[dtype]))
    return t, t.double().cpu().numpy()


def vec(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()


# --------------------------------------------------------------------------- #
# Layer norm
# --------------------------------------------------------------------------- #
NORM = [(1, 1), (3, 2), (1, 32), (5, 36), (64, 64), (257, 128), (33, 100), (1000, 129), (70, 256),
        (19, 260), (40, 513), (300, 516), (9, 1000), (50, 1024), (6, 1500), (7, 2048), (5, 2049),
        (4, 2052), (3, 5000), (2, 8192), (20_001, 12), (4099, 384)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,dim", NORM)
def test_layer_norm_and_its_gradient(n, dim, dtype):
    rng = np.random.default_rng(n * 10_007 + dim)
    for pad, offset in ((0, 0), (4, 0), (3, 1)):
        say(f"layer norm {n} x {dim} {dtype}, pad {pad}, offset {offset}")
        x, xv = rows(rng.normal(size=(n, dim)) * 0.7 + 0.3, dtype, pad, offset)
        dy, dyv = rows(rng.normal(size=(n, dim)), dtype, pad, offset)
        g, b = vec(1 + 0.2 * rng.normal(size=dim)), vec(rng.normal(size=dim))
        gv, bv = g.double().cpu().numpy(), b.double().cpu().numpy()
        y, mean, rstd = P.layer_norm(x, g, b, 1e-5)
        want, m, r = ref.layer_norm(xv, gv, bv, 1e-5)
        half = BF if dtype == "bf16" else 0.0
        ax = np.abs(xv).max(1)
        # sums of dim terms in registers and over lanes: at most 32 + 8 in sequence
        em = 48 * U * ax
        within(mean, m, em + 1e-30, "mean")
        # d(rstd)/rstd = -(d var) rstd^2 / 2
        er = r * (48 * U + 2 * em * ax * r * r + 4 * U)
        within(rstd, r, er, "rstd")
        xh = np.abs((xv - m[:, None]) * r[:, None])
        ez = em[:, None] * r[:, None] + xh * (er / r)[:, None] + 4 * U * xh
        ey = ez * np.abs(gv) + 4 * U * (xh * np.abs(gv) + np.abs(bv))
        within(y, want, ey + half * np.abs(want) + 1e-30, "y")
        # the backward pass from the oracle's mean and rstd as float32
        m32, r32 = vec(m), vec(r)
        mv, rv = m32.double().cpu().numpy(), r32.double().cpu().numpy()
        dx, dg, db = P.layer_norm_backward(dy, x, g, m32, r32)
        wx, wg, wb = ref.layer_norm_backward(dyv, xv, gv, mv, rv)
        xh = np.abs((xv - mv[:, None]) * rv[:, None])
        ex = 4 * U * (xh + ax[:, None] * rv[:, None])  # of xh
        a = np.abs(dyv * gv)
        s1, s2 = a.mean(1)[:, None], (a * xh).mean(1)[:, None]
        e2 = 48 * U * s2 + (a * ex).mean(1)[:, None]
        edx = rv[:, None] * (48 * U * s1 + xh * e2 + ex * s2 + 8 * U * (a + s1 + xh * s2))
        within(dx, wx, edx + half * np.abs(wx) + 1e-30, "dx")
        depth = 48 + 2 * math.sqrt(n)  # rows summed in sequence by a group, then their sums
        within(dg, wg, depth * U * (np.abs(dyv) * xh).sum(0) + (np.abs(dyv) * ex).sum(0) + 1e-30,
               "dgamma")
        within(db, wb, depth * U * np.abs(dyv).sum(0) + 1e-30, "dbeta")


def test_layer_norm_of_no_rows_and_parts_of_the_gradient():
    g, b = torch.ones(8, device="cuda"), torch.zeros(8, device="cuda")
    none = torch.empty((0, 8), device="cuda")
    y, mean, rstd = P.layer_norm(none, g, b)
    assert y.shape == (0, 8) and mean.numel() == 0
    dx, dg, db = P.layer_norm_backward(none, none, g, mean, rstd)
    assert dx.shape == (0, 8) and not dg.any() and not db.any()
    x = torch.randn(100, 8, device="cuda")
    y, mean, rstd = P.layer_norm(x, g, b)
    full = P.layer_norm_backward(y, x, g, mean, rstd)
    only_x = P.layer_norm_backward(y, x, g, mean, rstd, want_weights=False)
    only_w = P.layer_norm_backward(y, x, g, mean, rstd, want_dx=False)
    assert only_x[1] is None and only_w[0] is None
    assert torch.equal(full[0], only_x[0])
    assert torch.equal(full[1], only_w[1]) and torch.equal(full[2], only_w[2])


def test_layer_norm_constant_and_nan_rows():
    """A constant row has variance 0; a NaN stays in its row (and its column sums)."""
    x = torch.randn(9, 64, device="cuda")
    x[2] = 3.0
    x[5, 7] = math.nan
    g, b = torch.ones(64, device="cuda"), torch.full((64,), 0.25, device="cuda")
    y, mean, rstd = P.layer_norm(x, g, b, 1e-5)
    assert torch.equal(y[2], b) and abs(rstd[2].item() - 1e-5 ** -0.5) < 1e-3
    assert y[5].isnan().all() and not y[[0, 1, 2, 3, 4, 6, 7, 8]].isnan().any()


def test_layer_norm_in_place():
    x = torch.randn(300, 96, device="cuda", dtype=torch.bfloat16)
    g, b = torch.rand(96, device="cuda"), torch.rand(96, device="cuda")
    want = P.layer_norm(x, g, b)[0]
    st = P.load().huge_layer_norm(x.data_ptr(), 96, 300, 96, B.HUGE_DTYPE_BF16, g.data_ptr(),
                                  b.data_ptr(), 1e-5, x.data_ptr(), 96, None, None, None)
    assert st == 0
    torch.cuda.synchronize()
    assert torch.equal(x, want)


# --------------------------------------------------------------------------- #
# Softmax loss
# --------------------------------------------------------------------------- #
def softmax_case(n, classes, dim, dtype, rng, pad=0, offset=0, bias=True, masked=0.0,
                 weights=True, unlabelled=0.2, size=1.5):
    h, hv = rows(rng.normal(size=(n, dim)), dtype, pad, offset)
    w, wv = rows(rng.normal(size=(classes, dim)) * size / math.sqrt(dim), dtype, pad, offset)
    labels = rng.integers(0, classes, n)
    labels[rng.random(n) < unlabelled] = -1
    b = (rng.normal(size=classes)).astype(np.float32) if bias else None
    if bias and masked:
        b[rng.random(classes) < masked] = -np.inf
    c = rng.integers(0, 5, n).astype(np.float32) * np.float32(0.75) if weights else None
    return dict(h=h, w=w, hv=hv, wv=wv, labels=labels, b=b, c=c,
                tl=torch.from_numpy(labels.astype(np.int32)).cuda(),
                tb=None if b is None else vec(b), tc=None if c is None else vec(c))


def check_softmax(k, dtype, scale=0.5, grad=True):
    n, classes, dim = len(k["hv"]), len(k["wv"]), k["hv"].shape[1]
    op = P.SoftmaxLoss(max(1, n), classes, dim, dtype=dtype, grad=grad)
    total = torch.full((1,), 7.0, dtype=torch.float64, device="cuda")
    loss, lse = op.loss(k["h"], k["w"], k["tl"], k["tb"], k["tc"], total=total)
    hs = np.where(np.isfinite(k["hv"]), k["hv"], 0.0)
    want, wlse, counted = ref.softmax_loss(k["hv"], k["wv"], k["labels"], k["b"], k["c"])
    b = np.zeros(classes) if k["b"] is None else np.where(k["b"] == -np.inf, 0, k["b"])
    wk = np.where(np.isfinite(k["wv"]), k["wv"], 0.0)
    # a logit's error: the D products' sum (exact products for bf16), the bias, and
    # the three parts' product that is left out (2^-24 of the whole each)
    e = (dim + 8) * U * (np.abs(hs) @ np.abs(wk).T + np.abs(b))
    el = e.max(1) if classes else 0.0
    mag = np.where(np.isfinite(wlse), np.abs(wlse), 0.0)
    within(lse, wlse, el + 64 * U + 8 * U * mag + 1e-30, "lse")
    c1 = np.ones(n) if k["c"] is None else np.where(np.isfinite(k["c"]), k["c"], 0)
    within(loss, want, c1 * (2 * el + 64 * U + 16 * U * mag) + 8 * U * np.nan_to_num(np.abs(want))
           + 1e-30, "loss")
    if np.isfinite(want).all():
        exact = loss.double().sum().item()
        assert abs(total.item() - exact) <= 1e-12 * max(1.0, loss.double().abs().sum().item())
    if not grad:
        op.check()
        return op
    dh, dw, db = op.grad(k["h"], k["w"], k["tl"], lse, k["tb"], k["tc"], scale=scale)
    wants, sizes = ref.softmax_grad(k["hv"], k["wv"], k["labels"], k["b"], k["c"], scale)
    # a probability is off by the logit's and lse's errors (relatively), the label's
    # element by that of p; each term's rounding, then sums over rows or classes
    rel = 2 * np.max(el) + 128 * U + 32 * U * np.max(mag)
    half = BF if dtype == "bf16" else 0.0
    pmass = scale * counted  # |g| does not bound p's error where p is near 1: p <= 1 does
    ph = pmass[:, None] * np.abs(wk).max(0)
    within(dh, wants[0], (rel + half + (classes ** 0.5 + 64) * U) * sizes[0] + rel * ph
           + half * np.abs(wants[0]) + 1e-30, "dh")
    pw = (pmass[counted > 0, None] * np.abs(hs[counted > 0])).sum(0)
    within(dw, wants[1], (rel + half + (n ** 0.5 + 64) * U) * sizes[1] + rel * pw
           + half * np.abs(wants[1]) + 1e-30, "dw")
    within(db, wants[2], (rel + (n ** 0.5 + 64) * U) * sizes[2] + rel * pmass.sum() + 1e-30, "db")
    again = op.grad(k["h"], k["w"], k["tl"], lse, k["tb"], k["tc"], scale=scale)
    for x, y in zip((dh, dw, db), again):
        assert torch.equal(x, y)
    op.check()
    return op


SOFT = [(1, 1, 4), (1, 2, 8), (2, 33, 4), (5, 31, 36), (33, 32, 32), (32, 65, 64), (100, 257, 100),
        (129, 1000, 128), (300, 10, 128), (64, 511, 160), (70, 300, 224), (31, 999, 256),
        (40, 333, 260), (65, 130, 384), (17, 70, 516), (90, 200, 300), (100, 99, 420),
        (70, 150, 772), (66, 90, 900), (67, 301, 188), (40, 64, 1024), (1000, 5, 32),
        (1, 5000, 64), (7, 3001, 24), (513, 700, 68)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,dim", SOFT)
def test_softmax_loss_and_gradient(n, classes, dim, dtype):
    say(f"softmax {n} x {classes} x {dim} {dtype}")
    rng = np.random.default_rng(n * 7919 + classes * 31 + dim)
    check_softmax(softmax_case(n, classes, dim, dtype, rng), dtype)
    check_softmax(softmax_case(n, classes, dim, dtype, rng, pad=3, offset=1, bias=False,
                               weights=False, unlabelled=0.0), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 160, 192, 256, 320, 384, 512, 640])
def test_softmax_aligned_without_bias(dim, dtype):
    """Rows of whole 16-byte pieces and no bias: the table is used as it lies."""
    rng = np.random.default_rng(dim)
    for n, classes, pad in ((90, 77, 0), (200, 1003, 8), (333, 64, 0)):
        say(f"softmax {n} x {classes} x {dim} {dtype}, pad {pad}")
        check_softmax(softmax_case(n, classes, dim, dtype, rng, pad=pad, bias=False), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,dim", [(16, 500, 1024), (20, 601, 1024), (38, 901, 336),
                                           (33, 1000, 480), (64, 900, 576), (64, 900, 580),
                                           (64, 7, 484)])
def test_softmax_few_wide_rows(n, classes, dim, dtype):
    """Up to 64 rows whose operands fill LDS, or just do not fit."""
    rng = np.random.default_rng(n * 7919 + classes * 31 + dim)
    for pad, offset in ((0, 0), (3, 1)):
        say(f"few rows {n} x {classes} x {dim} {dtype}, pad {pad}")
        check_softmax(softmax_case(n, classes, dim, dtype, rng, pad=pad, offset=offset), dtype,
                      grad=False)


def softmax_on_device(h, w, labels, bias, c, scale):
    """loss, lse, dh, dw, dbias in float64 on the GPU, for sizes beyond the oracle's."""
    h, w, labels = h.double(), w.double(), labels.long()
    x = h @ w.t() + bias.double()
    lse = torch.logsumexp(x, 1)
    live = labels >= 0
    at = x.gather(1, labels.clamp(min=0)[:, None])[:, 0]
    k = torch.where(live, c.double(), torch.zeros_like(at))
    g = torch.exp(x - lse[:, None]) * (k * scale)[:, None]
    g[torch.arange(len(h), device="cuda")[live], labels[live]] -= (k * scale)[live]
    return k * (lse - at), lse, g @ w, g.t().contiguous() @ h, g.sum(0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,dim", [(140_003, 37, 32), (70, 140_003, 32), (110_001, 70, 128),
                                           (96, 150_001, 100), (9_001, 3_001, 256)])
def test_softmax_many_tiles(n, classes, dim, dtype):
    """More tiles than the card takes at once: whole rounds of them and what is left
    over, along the rows and along the classes."""
    say(f"softmax {n} x {classes} x {dim} {dtype}")
    g = torch.Generator(device="cuda").manual_seed(n + dim)
    new = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    h = new(n, dim).to(TYPES[dtype])
    w = (new(classes, dim) * 1.5 / math.sqrt(dim)).to(TYPES[dtype])
    labels = torch.randint(-1, classes, (n,), device="cuda", generator=g).to(torch.int32)
    bias, c = new(classes), torch.rand(n, device="cuda", generator=g) + 0.5
    op = P.SoftmaxLoss(n, classes, dim, dtype=dtype)
    loss, lse = op.loss(h, w, labels, bias, c)
    got = (loss, lse, *op.grad(h, w, labels, lse, bias, c, scale=1.0))
    want = softmax_on_device(h, w, labels, bias, c, 1.0)
    # norms here: fp32 sums of many terms about 1e-6, a rounding to bf16 and one of
    # the probabilities before it 2^-8 each at most
    for name, x, y in zip(("loss", "lse", "dh", "dw", "db"), got, want):
        tol = 2.0 ** -8 if dtype == "bf16" and name in ("dh", "dw") else 2e-6
        err = ((x.double() - y).norm() / y.norm()).item()
        far = ((x.double() - y).abs().max() / y.abs().max()).item()
        say(f"  {name}: {err:.3g} of the norm, {far:.3g} of the largest")
        assert err <= tol and far <= 4 * tol, name
    op.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,dim", [(4_100, 9_001, 384), (9_001, 3_001, 320), (33, 40_001, 288)])
def test_softmax_many_tiles_of_wide_rows(n, classes, dim, dtype):
    """Rows of which LDS takes one record: every tile comes in halves (fp32)."""
    test_softmax_many_tiles(n, classes, dim, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_softmax_many_rows_few_classes_and_few_rows_many_classes(dtype):
    rng = np.random.default_rng(11)
    check_softmax(softmax_case(20_011, 37, 32, dtype, rng), dtype)
    check_softmax(softmax_case(19, 40_003, 32, dtype, rng), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_softmax_confident_rows(dtype):
    """Logits of tens: probabilities near 1 and near 0."""
    rng = np.random.default_rng(12)
    k = softmax_case(200, 90, 64, dtype, rng, size=8.0, unlabelled=0.0)
    best = (k["hv"] @ k["wv"].T + k["b"]).argmax(1)
    k["labels"][::2] = best[::2]
    k["tl"] = torch.from_numpy(k["labels"].astype(np.int32)).cuda()
    check_softmax(k, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_softmax_classes_taken_out(dtype):
    """Classes with bias -inf: their rows of w may hold anything."""
    rng = np.random.default_rng(13)
    for masked in (0.1, 0.9):
        k = softmax_case(150, 200, 48, dtype, rng, masked=masked)
        out = torch.from_numpy(np.flatnonzero(k["b"] == -np.inf)).cuda()
        k["w"][out[::2]] = math.nan
        k["w"][out[1::2]] = math.inf
        k["wv"] = k["w"].double().cpu().numpy()
        op = check_softmax(k, dtype)
        loss, lse = op.loss(k["h"], k["w"], k["tl"], k["tb"], k["tc"])
        dh, dw, db = op.grad(k["h"], k["w"], k["tl"], lse, k["tb"], k["tc"])
        assert not dw[out].any() and not db[out].any() and dh.isfinite().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_softmax_nothing_left(dtype):
    rng = np.random.default_rng(14)
    k = softmax_case(40, 70, 32, dtype, rng)
    k["b"][:] = -np.inf
    k["tb"].fill_(-math.inf)
    op = P.SoftmaxLoss(40, 70, 32, dtype=dtype)
    loss, lse = op.loss(k["h"], k["w"], k["tl"], k["tb"], k["tc"])
    assert not loss.any() and (lse == -math.inf).all()
    for g in op.grad(k["h"], k["w"], k["tl"], lse, k["tb"], k["tc"]):
        assert not g.any()
    op.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_softmax_rows_without_a_loss_are_not_used(dtype):
    """NaN rows without a label, with weight 0 or with a masked label leave the
    gradients of the others alone; a NaN row with a loss shows in its outputs."""
    rng = np.random.default_rng(15)
    k = softmax_case(96, 50, 32, dtype, rng, unlabelled=0.3, masked=0.1)
    dead = (k["labels"] < 0) | (k["c"] == 0)
    dead |= (k["labels"] >= 0) & (k["b"][np.maximum(k["labels"], 0)] == -np.inf)
    assert dead.any() and not dead.all()
    op = P.SoftmaxLoss(96, 50, 32, dtype=dtype)
    args = (k["w"], k["tl"])
    loss, lse = op.loss(k["h"], *args, k["tb"], k["tc"])
    want = op.grad(k["h"], *args, lse, k["tb"], k["tc"])
    h = k["h"].clone()
    h[torch.from_numpy(dead).cuda()] = math.nan
    loss2, lse2 = op.loss(h, *args, k["tb"], k["tc"])
    live = torch.from_numpy(~dead).cuda()
    assert torch.equal(loss2, loss) and torch.equal(lse2[live], lse[live])
    for x, y in zip(want, op.grad(h, *args, lse2, k["tb"], k["tc"])):
        assert torch.equal(x, y)
    row = int(np.flatnonzero(~dead)[0])
    h[row] = math.nan
    loss3, lse3 = op.loss(h, *args, k["tb"], k["tc"])
    assert loss3[row].isnan() and lse3[row].isnan()
    assert int(loss3.isnan().sum()) == 1


def test_softmax_device_errors():
    """Bad labels and weights: NaN loss, no gradient, reported once by check()."""
    rng = np.random.default_rng(16)
    k = softmax_case(60, 40, 32, "f32", rng, unlabelled=0.0, weights=True)
    k["labels"][3], k["labels"][7] = 40, -2
    k["tl"] = torch.from_numpy(k["labels"].astype(np.int32)).cuda()
    op = P.SoftmaxLoss(60, 40, 32)
    loss, lse = op.loss(k["h"], k["w"], k["tl"], k["tb"], k["tc"])
    want, wlse, counted = ref.softmax_loss(k["hv"], k["wv"], k["labels"], k["b"], k["c"])
    np.testing.assert_array_equal(loss.isnan().cpu().numpy(), np.isnan(want))
    with pytest.raises(P.HugeError) as e:
        op.check()
    assert e.value.status == B.HUGE_ERR_ID_OUT_OF_RANGE
    op.check()
    dh, dw, db = op.grad(k["h"], k["w"], k["tl"], lse, k["tb"], k["tc"])
    assert not dh[3].any() and not dh[7].any() and dw.isfinite().all()
    with pytest.raises(P.HugeError):
        op.check()
    for bad in (-1.0, math.nan, math.inf):
        c = k["tc"].clone()
        c[5] = bad
        loss, _ = op.loss(k["h"], k["w"], k["tl"].clamp(0, 39), k["tb"], c)
        assert loss[5].isnan() and int(loss.isnan().sum()) == 1
        with pytest.raises(P.HugeError) as e:
            op.check()
        assert e.value.status == B.HUGE_ERR_BAD_COUNT


def test_softmax_no_rows_and_wanted_parts():
    op = P.SoftmaxLoss(50, 30, 16)
    w = torch.randn(30, 16, device="cuda")
    none = torch.empty((0, 16), device="cuda")
    lab = torch.empty(0, dtype=torch.int32, device="cuda")
    total = torch.full((1,), 3.0, dtype=torch.float64, device="cuda")
    loss, lse = op.loss(none, w, lab, total=total)
    assert loss.numel() == 0 and total.item() == 0
    dh, dw, db = op.grad(none, w, lab, lse)
    assert dh.shape == (0, 16) and not dw.any() and not db.any()
    h = torch.randn(50, 16, device="cuda")
    lab = torch.randint(0, 30, (50,), device="cuda", dtype=torch.int32)
    _, lse = op.loss(h, w, lab)
    full = op.grad(h, w, lab, lse)
    for k, name in enumerate(("want_h", "want_w", "want_bias")):
        part = op.grad(h, w, lab, lse, **{n: n == name for n in ("want_h", "want_w", "want_bias")})
        assert all((t is None) == (j != k) for j, t in enumerate(part))
        assert torch.equal(part[k], full[k])


def test_softmax_fewer_rows_than_planned_and_rows_alone():
    """A call of fewer rows than the workspace's, and each row by itself, give the
    same losses (up to rounding)."""
    op = P.SoftmaxLoss(300, 1000, 64)
    w, h = torch.randn(1000, 64, device="cuda") * 0.2, torch.randn(300, 64, device="cuda")
    lab = torch.randint(0, 1000, (300,), device="cuda", dtype=torch.int32)
    loss, lse = op.loss(h, w, lab)
    for n in (1, 2, 31, 100):
        l2, s2 = op.loss(h[:n], w, lab[:n])
        assert (l2 - loss[:n]).abs().max() < 2e-5 and (s2 - lse[:n]).abs().max() < 2e-5


def test_softmax_gradient_against_differences():
    """fp32 gradients against central differences of the float64 loss."""
    rng = np.random.default_rng(17)
    k = softmax_case(12, 40, 8, "f32", rng)
    op = P.SoftmaxLoss(12, 40, 8)
    _, lse = op.loss(k["h"], k["w"], k["tl"], k["tb"], k["tc"])
    dh, dw, db = (t.double().cpu().numpy() for t in
                  op.grad(k["h"], k["w"], k["tl"], lse, k["tb"], k["tc"]))
    step = 1e-5

    def total(h, w, b):
        return ref.softmax_loss(h, w, k["labels"], b, k["c"])[0].sum()

    b64 = k["b"].astype(np.float64)
    for which, got in ((0, dh), (1, dw), (2, db)):
        base = [k["hv"], k["wv"], b64]
        for at in list(np.ndindex(got.shape))[::7]:
            lo, hi = [t.copy() for t in base], [t.copy() for t in base]
            lo[which][at] -= step
            hi[which][at] += step
            diff = (total(*hi) - total(*lo)) / (2 * step)
            assert abs(got[at] - diff) < 1e-4, (which, at)


def test_softmax_on_another_stream_and_in_a_graph():
    """The same call on a side stream, and recorded once and replayed between the
    program's own work: the same bits each time."""
    op = P.SoftmaxLoss(200, 3000, 64, dtype="bf16")
    g = torch.Generator(device="cuda").manual_seed(3)
    h = torch.randn(200, 64, device="cuda", generator=g).bfloat16()
    w = (torch.randn(3000, 64, device="cuda", generator=g) * 0.2).bfloat16()
    lab = torch.randint(0, 3000, (200,), device="cuda", dtype=torch.int32, generator=g)

    def both(stream=None):
        loss, lse = op.loss(h, w, lab, stream=stream)
        return (loss, *op.grad(h, w, lab, lse, stream=stream))

    want = [t.clone() for t in both()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = both(side)
    torch.cuda.current_stream().wait_stream(side)
    for x, y in zip(want, got):
        assert torch.equal(x, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        both()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        held = both()
    for _ in range(3):
        for t in held:
            t.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(want, held):
            assert torch.equal(x, y)
        torch.randn(100, 100, device="cuda").sum().item()


@pytest.mark.parametrize("dtype,classes", [("f32", 300_001), ("bf16", 560_003)])
def test_softmax_table_in_pieces(dtype, classes):
    """A table whose packed rows exceed what is packed at once: labels, sums and partial
    results across the pieces."""
    n, dim = 90, 1024
    say(f"softmax {n} x {classes} x {dim} {dtype}")
    g = torch.Generator(device="cuda").manual_seed(7)
    new = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    h = new(n, dim).to(TYPES[dtype])
    w = (new(classes, dim) * 1.5 / math.sqrt(dim)).to(TYPES[dtype])
    labels = torch.randint(-1, classes, (n,), device="cuda", generator=g).to(torch.int32)
    labels[:4] = torch.tensor([0, classes - 1, classes // 2, 262_144], dtype=torch.int32)
    bias, c = new(classes), torch.rand(n, device="cuda", generator=g) + 0.5
    op = P.SoftmaxLoss(n, classes, dim, dtype=dtype)
    loss, lse = op.loss(h, w, labels, bias, c)
    got = (loss, lse, *op.grad(h, w, labels, lse, bias, c, scale=1.0))
    for name, x, y in zip(("loss", "lse", "dh", "dw", "db"), got,
                          softmax_on_device(h, w, labels, bias, c, 1.0)):
        tol = 2.0 ** -8 if dtype == "bf16" and name in ("dh", "dw") else 2e-6
        err = ((x.double() - y).norm() / y.norm()).item()
        say(f"  {name}: {err:.3g} of the norm")
        assert err <= tol, name
    op.check()


@pytest.mark.parametrize("hs,ws", [(1e15, 1e-15), (1e-18, 1e18), (1e-30, 1e29), (1e35, 1e-36)])
def test_softmax_fp32_scales(hs, ws):
    """Rows of very large and very small values whose products are ordinary, and
    rows in which few elements are much larger than the others."""
    rng = np.random.default_rng(18)
    n, classes, dim = 80, 150, 64
    k = softmax_case(n, classes, dim, "f32", rng, unlabelled=0.0)
    h = k["hv"] * np.where(rng.random((n, dim)) < 0.05, 30.0, 0.1)
    w = k["wv"] * np.where(rng.random((classes, dim)) < 0.05, 3.0, 1.0)
    k["h"], k["hv"] = rows(h * hs, "f32")
    k["w"], k["wv"] = rows(w * ws, "f32")
    op = P.SoftmaxLoss(n, classes, dim)
    loss, lse = op.loss(k["h"], k["w"], k["tl"], k["tb"], k["tc"])
    dh, dw, db = op.grad(k["h"], k["w"], k["tl"], lse, k["tb"], k["tc"], scale=0.5)
    want, wlse, _ = ref.softmax_loss(k["hv"], k["wv"], k["labels"], k["b"], k["c"])
    (wh, ww, wb), _ = ref.softmax_grad(k["hv"], k["wv"], k["labels"], k["b"], k["c"], 0.5)
    # an element keeps 22 bits, or 2^-40 of its row's largest: logits of at most a few
    # tens are within 1e-5
    for name, x, y in (("loss", loss, want), ("lse", lse, wlse), ("dh", dh, wh), ("dw", dw, ww),
                       ("db", db, wb)):
        d = np.linalg.norm(x.double().cpu().numpy() / np.abs(y).max() - y / np.abs(y).max())
        say(f"  {name}: {d / np.linalg.norm(y / np.abs(y).max()):.3g} of the norm")
        assert d <= 2e-5 * np.linalg.norm(y / np.abs(y).max()), name


# --------------------------------------------------------------------------- #
# AdamW
# --------------------------------------------------------------------------- #
HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-7, weight_decay=0.05)


def adam_values(size, rng):
    f = np.float32
    scale = np.exp(2 * rng.normal(size=size))
    return ((rng.normal(size=size)).astype(f), (rng.normal(size=size) * scale * 1e-2).astype(f),
            (rng.normal(size=size) * scale * 1e-2).astype(f),
            ((rng.normal(size=size) * scale * 1e-2) ** 2).astype(f))


@pytest.mark.parametrize("states", ["f32", "q8"])
@pytest.mark.parametrize("ptype,gtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"),
                                         ("f32", "bf16")])
def test_adamw_steps_bit_for_bit(ptype, gtype, states):
    """Three steps over tensors of many sizes, some not aligned to 16 bytes, against
    the float32 form of the definition: the same bits, moments and parameters."""
    say(f"adamw {ptype} {gtype} {states}")
    rng = np.random.default_rng(21)
    sizes = [1, 2, 3, 255, 256, 257, 1000, 4096, 4097, 20_003]
    vals = [adam_values(s, rng) for s in sizes]
    params, grads, m, v = [], [], [], []
    for j, (p, g, mk, vk) in enumerate(vals):
        shift = j % 2  # every other tensor starts one element into its allocation
        t = torch.zeros(len(p) + shift, dtype=TYPES[ptype], device="cuda")[shift:]
        t.copy_(torch.from_numpy(p))
        params.append(t)
        t = torch.zeros(len(p) + shift, dtype=TYPES[gtype], device="cuda")[shift:]
        t.copy_(torch.from_numpy(g))
        grads.append(t)
        m.append(vec(mk))
        v.append(vec(vk))
    opt = P.AdamW(params, lr=HYPER["lr"], betas=(HYPER["beta1"], HYPER["beta2"]),
                  eps=HYPER["eps"], weight_decay=HYPER["weight_decay"], states=states)
    opt.load(m, v, 4)
    p_ = [t.float().cpu().numpy() for t in params]
    g_ = [t.float().cpu().numpy() for t in grads]
    s_ = [(a[2], a[3]) if states == "f32" else ref.q8_f32(a[2], a[3]) for a in vals]
    for step in (5, 6, 7):
        opt.step(grads, grad_scale=0.5)
        gm, gv = opt.values()
        for j in range(len(sizes)):
            pn, mn, vn, ok = ref.adamw_f32(p_[j], g_[j], *s_[j], step, grad_scale=0.5, **HYPER)
            assert ok.all()
            p_[j] = torch.from_numpy(pn).to(TYPES[ptype]).float().numpy()
            s_[j] = (mn, vn) if states == "f32" else ref.q8_f32(mn, vn)
            np.testing.assert_array_equal(params[j].float().cpu().numpy(), p_[j], f"p {j} {step}")
            np.testing.assert_array_equal(gm[j].cpu().numpy(), s_[j][0], f"m {j} {step}")
            np.testing.assert_array_equal(gv[j].cpu().numpy(), s_[j][1], f"v {j} {step}")
    assert opt.steps == 7
    opt.check()


@pytest.mark.parametrize("states", ["f32", "q8"])
def test_adamw_magnitudes(states):
    """Gradients of 1e-30 to 1e18, whole blocks of zeros, tiny and large moments beside
    each other: the same bits as the float32 form."""
    rng = np.random.default_rng(25)
    f = np.float32
    size = 64 * 256 + 77
    p, _, m, v = adam_values(size, rng)
    g = (rng.normal(size=size) * 10.0 ** rng.uniform(-30, 18, size)).astype(f)
    scale = np.repeat(10.0 ** rng.uniform(-25, 15, 65), 256)[:size]
    m, v = (m * scale).astype(f), (v * scale * scale).astype(f)
    g[:512] = m[:256] = v[:256] = 0
    g[1024:8192] = (g[1024:8192] * 1e-12).astype(f)
    ok = np.abs(g) < 1e18
    g[~ok] = 0
    t = vec(p)
    opt = P.AdamW([t], states=states)
    opt.load([vec(m)], [vec(v)], 3)
    s = (m, v) if states == "f32" else ref.q8_f32(m, v)
    for step in (4, 5):
        opt.step([vec(g)])
        pn, mn, vn, ok = ref.adamw_f32(p, g, *s, step, 1e-3, 0.9, 0.999, 1e-8, 0.01)
        assert ok.all()
        s = (mn, vn) if states == "f32" else ref.q8_f32(mn, vn)
        gm, gv = opt.values()
        np.testing.assert_array_equal(gm[0].cpu().numpy(), s[0])
        np.testing.assert_array_equal(gv[0].cpu().numpy(), s[1])
        np.testing.assert_array_equal(t.cpu().numpy(), pn)
        p = pn
    opt.check()


def test_adamw_against_float64():
    rng = np.random.default_rng(22)
    p, g, m, v = adam_values(5000, rng)
    t = vec(p)
    opt = P.AdamW([t], lr=HYPER["lr"], betas=(HYPER["beta1"], HYPER["beta2"]), eps=HYPER["eps"],
                  weight_decay=HYPER["weight_decay"])
    opt.load([vec(m)], [vec(v)], 0)
    opt.step([vec(g)], lr=1e-2)
    wp, wm, wv = ref.adamw(p, g, m, v, 1, **{**HYPER, "lr": 1e-2})
    gm, gv = opt.values()
    within(gm[0], wm, 4 * U * (np.abs(m) + np.abs(g)), "m")
    within(gv[0], wv, 4 * U * (v + g.astype(np.float64) ** 2) + 1e-44, "v")
    move = np.abs(wp - p * (1 - 1e-2 * HYPER["weight_decay"]))
    within(t, wp, 4 * U * np.abs(p) + 16 * U * move
           + 1e-2 * 10 * 4 * U * (np.abs(m) + np.abs(g)) / (np.sqrt(wv) * 10 + 1e-7), "p")


def test_adamw_more_tensors_than_a_launch_holds_and_empty_ones():
    rng = np.random.default_rng(23)
    sizes = [int(s) for s in rng.integers(0, 400, 150)]
    sizes[0] = sizes[64] = sizes[149] = 0
    params = [torch.randn(s, device="cuda") for s in sizes]
    grads = [torch.randn(s, device="cuda") for s in sizes]
    want = [p.cpu().numpy() for p in params]
    opt = P.AdamW(params, lr=1e-2)
    opt.step(grads)
    for s, p, g, w in zip(sizes, params, grads, want):
        z = np.zeros(s, np.float32)
        new = ref.adamw_f32(w, g.cpu().numpy(), z, z, 1, 1e-2, 0.9, 0.999, 1e-8, 0.01)[0]
        np.testing.assert_array_equal(p.cpu().numpy(), new)


@pytest.mark.parametrize("states", ["f32", "q8"])
def test_adamw_gradients_that_are_not_finite(states):
    """Such elements keep parameter and moments, the others move; check() reports."""
    rng = np.random.default_rng(24)
    p, g, m, v = adam_values(1000, rng)
    g[[3, 300, 999]] = [np.nan, np.inf, 1e30]  # the square of the last overflows
    t = vec(p)
    opt = P.AdamW([t], states=states)
    opt.load([vec(m)], [vec(v)], 1)
    m0, v0 = (x[0].cpu().numpy() for x in opt.values())
    opt.step([vec(g)])
    gm, gv = (x[0].cpu().numpy() for x in opt.values())
    pn, mn, vn, ok = ref.adamw_f32(p, g, m0, v0, 2, 1e-3, 0.9, 0.999, 1e-8, 0.01)
    assert (~ok).sum() == 3
    if states == "q8":
        mn, vn = ref.q8_f32(mn, vn)
    np.testing.assert_array_equal(t.cpu().numpy(), pn)
    np.testing.assert_array_equal(gm, mn)
    np.testing.assert_array_equal(gv, vn)
    with pytest.raises(P.HugeError) as e:
        opt.check()
    assert e.value.status == B.HUGE_ERR_NOT_FINITE
    opt.check()


def test_adamw_zero_gradients_from_zero_moments():
    """0 / (0 + eps): nothing but the decay."""
    for states in ("f32", "q8"):
        t = torch.randn(777, device="cuda")
        was = t.clone()
        opt = P.AdamW([t], lr=1e-2, weight_decay=0.5, states=states)
        opt.step([torch.zeros_like(t)])
        assert torch.equal(t, was * float(np.float32(1 - 1e-2 * 0.5)))
        m, v = opt.values()
        assert not m[0].any() and not v[0].any()


# --------------------------------------------------------------------------- #
# Together
# --------------------------------------------------------------------------- #
@pytest.mark.parametrize("dtype,states", [("f32", "f32"), ("bf16", "q8")])
def test_head_learns_separable_classes(dtype, states):
    g = torch.Generator(device="cuda").manual_seed(5)
    centres = torch.randn(20, 64, device="cuda", generator=g) * 2
    lab = torch.randint(0, 20, (4096,), device="cuda", generator=g)
    x = (centres[lab] + torch.randn(4096, 64, device="cuda", generator=g)).to(TYPES[dtype])
    lab = lab.to(torch.int32)
    head = P.SoftmaxHead(20, 64, 4096, dtype=dtype, lr=2e-2, states=states)
    losses = [head.step(x, lab)[0].item() for _ in range(60)]
    head.check()
    assert losses[0] > 2.0 and losses[-1] < 0.1 * losses[0]
    assert abs(head.loss(x, lab).mean().item() - losses[-1]) < 0.5 * losses[-1]


def test_head_gradient_of_the_rows():
    """dx through layer norm and loss against differences of the oracle's loss."""
    rng = np.random.default_rng(31)
    x = rng.normal(size=(6, 12))
    lab = rng.integers(0, 9, 6)
    head = P.SoftmaxHead(9, 12, 6, seed=1)
    w = head.w.double().cpu().numpy()
    x32 = vec(x)
    x64 = x32.double().cpu().numpy()
    _, dx = head.step(x32, torch.from_numpy(lab.astype(np.int32)).cuda())

    def total(t):
        y, _, _ = ref.layer_norm(t, np.ones(12), np.zeros(12), 1e-5)
        return ref.softmax_loss(y, w, lab)[0].sum() / 6

    for at in np.ndindex(6, 12):
        lo, hi = x64.copy(), x64.copy()
        lo[at] -= 1e-5
        hi[at] += 1e-5
        assert abs(dx[at].item() - (total(hi) - total(lo)) / 2e-5) < 1e-5


@pytest.mark.parametrize("states", ["f32", "q8"])
def test_example_finds_the_blocks(states):
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                    "examples"))
    import classify_blocks
    assert classify_blocks.main(["--epochs", "2", "--states", states], log=say) > 0.9


# --------------------------------------------------------------------------- #
# Refusals that need a device for their arguments
# --------------------------------------------------------------------------- #
def test_refusals():
    x = torch.randn(8, 16, device="cuda")
    g = torch.ones(16, device="cuda")
    with pytest.raises(TypeError):
        P.layer_norm(x.double(), g, g)
    with pytest.raises(TypeError):
        P.layer_norm(x.cpu(), g, g)
    with pytest.raises(TypeError):
        P.layer_norm(x[0], g, g)
    with pytest.raises(ValueError):
        P.layer_norm(x.t().contiguous().t(), g, g)
    with pytest.raises(ValueError):
        P.layer_norm(x, g[:15].contiguous(), g)
    with pytest.raises(ValueError):
        P.layer_norm(x[:1].expand(8, 16), g, g)
    with pytest.raises(P.HugeError):
        P.layer_norm(x, g, g, eps=0.0)
    y, mean, rstd = P.layer_norm(x, g, g)
    with pytest.raises(ValueError):
        P.layer_norm_backward(y[:7], x, g, mean, rstd)
    with pytest.raises(TypeError):
        P.layer_norm_backward(y.bfloat16(), x, g, mean, rstd)
    op = P.SoftmaxLoss(8, 5, 16, grad=False)
    w, lab = torch.randn(5, 16, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda")
    loss, lse = op.loss(x, w, lab)
    with pytest.raises(P.HugeError):
        op.grad(x, w, lab, lse)  # planned without the gradient
    with pytest.raises(P.HugeError):
        op.loss(torch.randn(9, 16, device="cuda"), w, torch.zeros(9, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        op.loss(x, w[:4], lab)
    with pytest.raises(ValueError):
        op.loss(x[:, :12], w, lab)
    with pytest.raises(TypeError):
        op.loss(x, w, lab.long())
    with pytest.raises(TypeError):
        op.loss(x.bfloat16(), w, lab)
    with pytest.raises(ValueError):
        op.loss(x, w, lab[:7])
    p = torch.randn(10, device="cuda")
    with pytest.raises(TypeError):
        P.AdamW([torch.randn(4, 4, device="cuda").t()])
    with pytest.raises(TypeError):
        P.AdamW([p.half()])
    opt = P.AdamW([p])
    was = p.clone()
    with pytest.raises(ValueError):
        opt.step([p, p])
    with pytest.raises(ValueError):
        opt.step([p[:9]])
    for bad in (-1.0, math.nan, math.inf):
        with pytest.raises(P.HugeError):
            opt.step([p], lr=bad)
    with pytest.raises(P.HugeError):
        P.AdamW([p], betas=(1.0, 0.9)).step([p])
    with pytest.raises(P.HugeError):
        P.AdamW([p], eps=0.0).step([p])
    assert opt.steps == 0 and torch.equal(p, was)


def test_softmax_workspace_is_checked():
    L = P.load()
    cfg = B.HugeSoftmaxConfig(5, 8, 16, B.HUGE_DTYPE_F32, 0)
    need = L.huge_softmax_workspace_bytes(ctypes.byref(cfg))
    x, w = torch.randn(8, 16, device="cuda"), torch.randn(5, 16, device="cuda")
    lab = torch.zeros(8, dtype=torch.int32, device="cuda")
    out = torch.full((2, 8), 5.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.zeros(need + 512, dtype=torch.uint8, device="cuda")
    at = ws.data_ptr() + (-ws.data_ptr()) % 256

    def call(ptr, nbytes):
        return L.huge_softmax_loss(ctypes.byref(cfg), x.data_ptr(), 16, 8, w.data_ptr(), 16, None,
                                   lab.data_ptr(), None, out[0].data_ptr(), out[1].data_ptr(), None,
                                   status.data_ptr(), ptr, nbytes, None)

    assert call(at, need - 1) == B.HUGE_ERR_WORKSPACE
    assert call(None, need) == B.HUGE_ERR_WORKSPACE
    assert call(at + 16, need) == B.HUGE_ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert (out == 5.0).all()
    assert call(at, need) == B.HUGE_OK
