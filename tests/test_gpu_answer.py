"""RMS norm, rows in 8 bits, log probabilities and clipped gradients against the float64
oracle (oracle/answer.py), through the package's entry points and, where pointers
matter, the C ABI.

Tolerances are counted as in test_gpu_head: u = 2^-24 per fp32 operation times the sum
of the absolute terms, half a step of the type (bf16 2^-8, e4m3 2^-4) for each
rounding to it.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2307_14490_amd as P  # noqa: E402
from paper_2307_14490_amd import binding as B  # noqa: E402
from oracle import answer as ref  # noqa: E402
from gpu_common import say  # noqa: E402
from test_gpu_head import BF, TYPES, U, _need_gpu, rows, vec, within  # noqa: E402,F401

pytestmark = pytest.mark.gpu


# --------------------------------------------------------------------------- #
# RMS norm and rows in 8 bits
# --------------------------------------------------------------------------- #
RMS = [(1, 1), (3, 2), (1, 32), (5, 36), (64, 64), (257, 128), (33, 100), (1000, 129), (70, 256),
       (19, 260), (40, 513), (300, 516), (9, 1000), (50, 1024), (6, 1500), (7, 2048), (5, 2049),
       (4, 2052), (3, 5000), (2, 8192), (20_001, 12), (4099, 384)]


def check_q8(q, y, ey, what):
    """Rows in 8 bits that hold y up to its error ey: a code is half a step off."""
    v = P.q8_values(q).double().cpu().numpy()
    codes, scales = q.codes.view(torch.uint8).cpu().numpy(), q.scales.cpu().numpy()
    np.testing.assert_array_equal(v, ref.q8_values(codes, scales))
    np.testing.assert_array_equal(P.q8_values(q, "bf16").double().cpu().numpy(), v)
    unit = np.repeat(2.0 ** (scales.astype(np.float64) - 127), 32, 1)[:, :v.shape[1]]
    within(v, y, ey + np.maximum((np.abs(y) + ey) * 2.0 ** -4, unit * 2.0 ** -10), what)
    # the smallest scale: a block's largest is above 224 of it (or the scale is the least)
    n, dim = v.shape
    pad = np.zeros((n, -dim % 32))
    most = (np.abs(np.concatenate([y, pad], 1)) + np.concatenate([ey, pad], 1)) \
        .reshape(n, -1, 32).max(2)
    assert ((most >= 224 * 2.0 ** (scales.astype(np.float64) - 127)) | (scales == 27)).all(), what


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,dim", RMS)
def test_rms_norm_and_its_gradient(n, dim, dtype):
    rng = np.random.default_rng(n * 10_007 + dim)
    for pad, offset, residual in ((0, 0, True), (4, 0, False), (3, 1, True)):
        say(f"rms norm {n} x {dim} {dtype}, pad {pad}, offset {offset}, residual {residual}")
        new = lambda: rows(rng.normal(size=(n, dim)), dtype, pad, offset)  # noqa: E731
        x, xv = new()
        r, rv = new() if residual else (None, 0)
        dy, dyv = new()
        dt, dtv = new() if residual else (None, 0)
        g = vec(1 + 0.2 * rng.normal(size=dim))
        gv = g.double().cpu().numpy()
        y, total, rstd = P.rms_norm(x, g, r, 1e-5)
        # the sum is rounded once to the rows' type: what torch's addition gives
        want = torch.from_numpy(xv + rv).to(TYPES[dtype]).double().numpy()
        tv = total.double().cpu().numpy()
        np.testing.assert_array_equal(tv, want)
        wy, wr = ref.rms_norm(tv, gv, 1e-5)
        # squares: at most 32 + 8 in sequence; d rstd / rstd is half of that of the mean
        er = wr * 32 * U
        within(rstd, wr, er, "rstd")
        half = BF if dtype == "bf16" else 0.0
        ey = np.abs(wy) * 36 * U + 1e-40
        within(y, wy, ey + half * np.abs(wy) + 1e-30, "y")
        q, _, rstd8 = P.rms_norm(x, g, r, 1e-5, q8=True)
        assert torch.equal(rstd, rstd8)
        check_q8(q, wy, np.abs(wy) * 2.0 ** -48, "y in 8 bits")
        codes, scales = ref.q8_rows(wy) if wy.size < 40_000 else (None, None)
        if codes is not None:  # the formula's own codes
            np.testing.assert_array_equal(q.scales.cpu().numpy(), scales)
            np.testing.assert_array_equal(q.codes.view(torch.uint8).cpu().numpy(), codes)
        # the backward pass from the oracle's rstd as float32
        r32 = vec(wr)
        rv32 = r32.double().cpu().numpy()
        dx, dg = P.rms_norm_backward(dy, total, g, r32, dt)
        wx, wg = ref.rms_norm_backward(dyv, tv, gv, rv32, dtv if residual else None)
        z, a = np.abs(tv * rv32[:, None]), np.abs(dyv * gv)
        s = (a * z).mean(1)[:, None]
        ex = rv32[:, None] * (8 * U * (a + z * s) + 52 * U * z * s) + 4 * U * np.abs(dtv)
        within(dx, wx, ex + half * np.abs(wx) + 1e-30, "dx")
        depth = 48 + 2 * math.sqrt(n)  # rows summed in sequence by a group, then their sums
        within(dg, wg, (depth + 4) * U * (np.abs(dyv) * z).sum(0) + 1e-30, "dgamma")


def test_rms_norm_of_no_rows_and_parts_of_the_gradient():
    g = torch.ones(8, device="cuda")
    none = torch.empty((0, 8), device="cuda")
    y, total, rstd = P.rms_norm(none, g, none)
    assert y.shape == (0, 8) and rstd.numel() == 0
    assert P.rms_norm(none, g, q8=True)[0].codes.shape == (0, 8)
    dx, dg = P.rms_norm_backward(none, none, g, rstd)
    assert dx.shape == (0, 8) and not dg.any()
    x = torch.randn(100, 8, device="cuda")
    y, total, rstd = P.rms_norm(x, g)
    assert total is x
    full = P.rms_norm_backward(y, x, g, rstd)
    only_x = P.rms_norm_backward(y, x, g, rstd, want_gamma=False)
    only_g = P.rms_norm_backward(y, x, g, rstd, want_dx=False)
    assert only_x[1] is None and only_g[0] is None
    assert torch.equal(full[0], only_x[0]) and torch.equal(full[1], only_g[1])


@pytest.mark.parametrize("q8", [False, True])
def test_rms_norm_rows_of_zeros_and_nan(q8):
    x = torch.randn(9, 64, device="cuda")
    x[2] = 0.0
    x[5, 40] = math.nan
    g = torch.ones(64, device="cuda")
    y, _, rstd = P.rms_norm(x, g, eps=1e-6, q8=q8)
    v = P.q8_values(y) if q8 else y
    assert not v[2].any() and abs(rstd[2].item() - 1e3) < 1e-2
    assert v[5].isnan().all() and not v[[0, 1, 2, 3, 4, 6, 7, 8]].isnan().any()


@pytest.mark.parametrize("dim,dtype", [(128, "bf16"), (128, "f32"), (97, "f32"), (1500, "f32")])
def test_rms_norm_in_8_bits_where_the_squares_pass_fp32(dim, dtype):
    """Rows with rstd 0 are zeros, and NaN in a block with an infinity, whichever rows lie
    beside them: among so many some have codes near a border, for which a wave forms
    its rows once more."""
    n = 20_000 if dim < 1000 else 4000
    x = torch.randn((n, dim), generator=torch.Generator().manual_seed(3))
    x[1::4] = 1e25
    x[3::8] = 1.0
    x[3::8, 40] = math.inf
    x = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()
    g = torch.linspace(0.5, 1.5, dim, device="cuda")
    y, _, rstd = P.rms_norm(x, g, q8=True)
    codes, scales = y.codes.view(torch.uint8), y.scales
    for rows in (slice(1, None, 4), slice(3, None, 8)):
        assert not rstd[rows].any()
        kept = [b for b in range(scales.shape[1]) if b != 1 or rows.start == 1]
        assert (scales[rows][:, kept] == 127 - 100).all()
        for b in kept:
            assert not codes[rows, 32 * b:32 * b + 32].any()
    assert (scales[3::8, 1] == 255).all()
    assert torch.isnan(P.q8_values(y)[3::8, 32:64]).all()
    few, _, _ = P.rms_norm(x[::2].contiguous(), g, q8=True)  # the others, without them
    assert torch.equal(few.codes.view(torch.uint8), codes[::2])
    assert torch.equal(few.scales, scales[::2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [96, 97, 1500])
def test_rms_norm_in_place(dim, dtype):
    """The sum over either input, the norm over its rows, the gradient over either's."""
    x, r, dy, dt = (torch.randn(300, dim, device="cuda").to(TYPES[dtype]) for _ in range(4))
    g = torch.rand(dim, device="cuda")
    code = B.HUGE_DTYPE_BF16 if dtype == "bf16" else B.HUGE_DTYPE_F32
    y, total, rstd = P.rms_norm(x, g, r)
    L = P.load()
    for into in (0, 1):
        a, b, out = x.clone(), r.clone(), torch.empty_like(y)
        t = (a, b)[into]
        assert L.huge_rms_norm(a.data_ptr(), dim, b.data_ptr(), dim, 300, dim, code, g.data_ptr(),
                               1e-5, t.data_ptr(), dim, out.data_ptr(), dim, None, 0, None, 0, None,
                               None) == 0
        torch.cuda.synchronize()
        assert torch.equal(t, total) and torch.equal(out, y)
    a = total.clone()
    assert L.huge_rms_norm(a.data_ptr(), dim, None, 0, 300, dim, code, g.data_ptr(), 1e-5, None, 0,
                           a.data_ptr(), dim, None, 0, None, 0, None, None) == 0
    torch.cuda.synchronize()
    assert torch.equal(a, y)
    want = P.rms_norm_backward(dy, total, g, rstd, dt, want_gamma=False)[0]
    for into in (0, 1):
        a, b = dy.clone(), dt.clone()
        assert L.huge_rms_norm_backward(a.data_ptr(), dim, total.data_ptr(), dim, b.data_ptr(), dim,
                                        300, dim, code, g.data_ptr(), rstd.data_ptr(),
                                        (a, b)[into].data_ptr(), dim, None, None, 0, None) == 0
        torch.cuda.synchronize()
        assert torch.equal((a, b)[into], want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_q8_rows_are_the_oracle_s(dtype):
    rng = np.random.default_rng(5)
    for n, dim, pad, offset in ((1, 1, 0, 0), (3, 31, 0, 0), (40, 32, 0, 0), (33, 100, 4, 0),
                                (60, 257, 3, 1), (7, 1028, 0, 0)):
        x = rng.normal(size=(n, dim)) * 10.0 ** rng.integers(-12, 12, size=(n, 1))
        x[rng.random((n, dim)) < 0.1] = 0.0
        x[:, ::7] *= 1e-3
        x[0] = 0.0
        t, v = rows(x, dtype, pad, offset)
        q = P.q8_rows(t)
        codes, scales = ref.q8_rows(v)
        np.testing.assert_array_equal(q.scales.cpu().numpy(), scales)
        np.testing.assert_array_equal(q.codes.view(torch.uint8).cpu().numpy(), codes)
        np.testing.assert_array_equal(P.q8_values(q).double().cpu().numpy(),
                                      ref.q8_values(codes, scales))


def test_q8_rows_at_the_ends_of_the_range():
    """The largest of a type, its smallest, exact borders of a scale, infinities and NaN."""
    big = torch.finfo(torch.float32).max
    x = torch.zeros(9, 64, device="cuda")
    x[0, 3] = big
    x[1, 3] = -big
    x[2, 3] = 448.0
    x[3, 3] = 448.0 * (1 + 2.0 ** -23)
    x[4, 3] = 1e-38
    x[5, 3] = math.inf
    x[6, 3] = -math.nan
    x[7, 3] = 2.0 ** -100 * 2.0 ** -9
    x[8, 40] = -0.0
    q = P.q8_rows(x)
    v = P.q8_values(q)
    s = q.scales.cpu().numpy()[:, 0].tolist()
    assert s == [127 + 120, 127 + 120, 127, 128, 27, 255, 255, 27, 27]
    # the largest float is 255.99 2^120, whose nearest code is 256: 2^128 in 32 bits is infinite
    assert (q.codes[:2, 3].double() * 2.0 ** 120).tolist() == [2.0 ** 128, -2.0 ** 128]
    want = [math.inf, -math.inf, 448.0, 448.0, 0.0]
    assert v[:5, 3].double().tolist() == want and v[7, 3].item() == 2.0 ** -109
    assert v[5, :32].isnan().all() and v[6, :32].isnan().all() and not v[5:, 32:].any()


# --------------------------------------------------------------------------- #
# Log probabilities
# --------------------------------------------------------------------------- #
def case(n, classes, dim, dtype, rng, pad=0, offset=0, bias=True, masked=0.0, unlabelled=0.2,
         size=1.5, labels=True):
    kind = "bf16" if dtype == "q8" else dtype
    h, hv = rows(rng.normal(size=(n, dim)), kind, pad, offset)
    w, wv = rows(rng.normal(size=(classes, dim)) * size / math.sqrt(dim), kind, pad, offset)
    k = dict(h=h, w=w, hv=hv, wv=wv, b=None, tb=None, labels=None, tl=None, dtype=dtype)
    if dtype == "q8":
        codes, scales = ref.q8_rows(wv)
        flat = torch.full((offset + classes * (dim + pad) + 1,), 127, dtype=torch.uint8,
                          device="cuda")
        c = flat[offset:offset + classes * (dim + pad)].view(classes, dim + pad)[:, :dim]
        c.copy_(torch.from_numpy(codes))
        more = torch.full((classes, scales.shape[1] + pad), 255, dtype=torch.uint8, device="cuda")
        s = more[:, :scales.shape[1]]
        s.copy_(torch.from_numpy(scales))
        k["w"], k["wv"] = P.Q8Rows(c.view(torch.float8_e4m3fn), s), ref.q8_values(codes, scales)
    if bias:
        k["b"] = rng.normal(size=classes).astype(np.float32)
        k["b"][rng.random(classes) < masked] = -np.inf
        k["tb"] = vec(k["b"])
    if labels:
        k["labels"] = rng.integers(0, classes, n)
        k["labels"][rng.random(n) < unlabelled] = -1
        k["tl"] = torch.from_numpy(k["labels"].astype(np.int32)).cuda()
    return k


def check(k, top=0, grad=True, max_rows=None, op=None):
    n, dim = k["hv"].shape
    classes, dtype = len(k["wv"]), k["dtype"]
    grad = grad and dtype != "q8"
    op = op or P.LogProbs(max_rows or max(1, n), classes, dim, dtype=dtype, top=top, grad=grad)
    a = op.log_probs(k["h"], k["w"], k["tl"], k["tb"])
    logp, entropy, lse, ids, best = ref.log_probs(k["hv"], k["wv"], k["labels"], k["b"], top)
    hs, ws = (np.where(np.isfinite(t), t, 0.0) for t in (k["hv"], k["wv"]))
    b = np.zeros(classes) if k["b"] is None else np.where(k["b"] < -1e28, 0, k["b"])
    # a logit's error, as for the loss
    e = (dim + 8) * U * (np.abs(hs) @ np.abs(ws).T + np.abs(b))
    el = e.max(1) if n else np.zeros(0)
    mag = np.where(np.isfinite(lse), np.abs(lse), 0.0)
    depth = 64 + classes / 16  # tiles added in sequence, if one wave has them all
    elow = el + depth * U + 8 * U * mag
    within(a.lse, lse, elow + 1e-30, "lse")
    # d entropy = - sum p (log p + entropy) dx; u = x - top is rounded, at u, as the sums are
    x = ref.logits(hs, ws, k["b"])
    lp = np.where(np.isfinite(x) & np.isfinite(lse)[:, None], x - np.where(
        np.isfinite(lse), lse, 0.0)[:, None], 0.0)
    p = np.where(np.isfinite(x), np.exp(lp), 0.0)
    h0 = np.nan_to_num(entropy)
    far = (p * (np.abs(lp) + h0[:, None])).sum(1)
    u = np.abs(lp) + h0[:, None] + 4  # |x - top| is at most |log p| + |log sum| + a rise
    eh = 2 * el * far + 4 * U * (p * u * (np.abs(lp) + h0[:, None])).sum(1) \
        + (depth + 8) * U * ((p * u).sum(1) + np.log1p(classes) + 4)
    within(a.entropy, entropy, eh + 1e-30, "entropy")
    if k["tl"] is None:
        assert a.logp is None
    else:
        within(a.logp, logp, elow + 4 * U * (mag + np.nan_to_num(np.abs(logp), posinf=0)) + 1e-30,
               "logp")
    if top:
        np.testing.assert_array_equal(a.ids.cpu().numpy(), ids)
        within(a.top_logp, best, elow[:, None] + 4 * U * (mag[:, None] + np.nan_to_num(
            np.abs(best), posinf=0)) + 1e-30, "top_logp")
    else:
        assert a.ids is None and a.top_logp is None
    again = op.log_probs(k["h"], k["w"], k["tl"], k["tb"])
    for s, t in zip(a, again):
        assert s is None or torch.equal(s, t) or torch.equal(s.isnan(), t.isnan())
    if grad:
        check_grad(k, op, a, el, elow, eh, lp, h0)
    op.check()
    return a


def check_grad(k, op, a, el, elow, eh, lp, h0):
    n, dim = k["hv"].shape
    classes, dtype = len(k["wv"]), k["dtype"]
    rng = np.random.default_rng(n + classes)
    for has_l, has_e in ((True, True), (True, False), (False, True)):
        if has_l and k["tl"] is None:
            continue
        dl = vec(rng.normal(size=n) * 0.5) if has_l else None
        de = vec(rng.normal(size=n) * 0.3) if has_e else None
        if has_l and n > 3:
            dl[1] = 0.0
        val = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
        got = op.grad(k["h"], k["w"], a, k["tl"] if has_l else None, dl, de, k["tb"])
        wants, size, soft, hc, wc = ref.log_probs_grad(
            k["hv"], k["wv"], k["labels"] if has_l else None, val(dl), val(de), k["b"])
        # an element: p is off by the logit's and lse's errors (relatively), its logarithm
        # and the entropy by theirs, its factor and product by roundings
        rel = (el + elow + 16 * U)[:, None] + 4 * U * np.abs(lp)
        eg = size * rel + soft * (el + elow + eh)[:, None] + soft * 4 * U * (np.abs(lp) + h0[:, None])
        half = BF if dtype == "bf16" else 0.0
        # an element is held in fp16, half a step of 2^-10 off (fp32 rows: in two parts, within
        # 2^-21 of its row's (column's) largest)
        part, split = (2.0 ** -11, 2.0 ** -24) if dtype == "bf16" else (0.0, 2.0 ** -21)
        eh_, ew_ = (eg + part * size + split * size.max(ax, keepdims=True) for ax in (1, 0)) \
            if n else (eg, eg)
        s = size @ np.abs(wc)
        within(got[0], wants[0], eh_ @ np.abs(wc) + (classes ** 0.5 + 64) * U * s
               + half * np.abs(wants[0]) + 1e-30, "dh")
        s = size.T @ np.abs(hc)
        within(got[1], wants[1], ew_.T @ np.abs(hc) + (n ** 0.5 + 64) * U * s
               + half * np.abs(wants[1]) + 1e-30, "dw")
        within(got[2], wants[2], eg.sum(0) + (n ** 0.5 + 64) * U * size.sum(0) + 1e-30, "db")
        again = op.grad(k["h"], k["w"], a, k["tl"] if has_l else None, dl, de, k["tb"])
        for x, y in zip(got, again):
            assert torch.equal(x, y)


SIZES = [(1, 1, 4), (1, 2, 8), (2, 33, 4), (5, 31, 36), (33, 32, 32), (32, 65, 64), (100, 257, 100),
         (129, 1000, 128), (300, 10, 128), (64, 511, 160), (70, 300, 224), (31, 999, 256),
         (40, 333, 260), (65, 130, 384), (17, 70, 516), (90, 200, 300), (100, 99, 420),
         (70, 150, 772), (66, 90, 900), (67, 301, 188), (40, 64, 1024), (1000, 5, 32),
         (1, 5000, 64), (7, 3001, 24), (513, 700, 68)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "q8"])
@pytest.mark.parametrize("n,classes,dim", SIZES)
def test_log_probs_and_their_gradient(n, classes, dim, dtype):
    say(f"log probs {n} x {classes} x {dim} {dtype}")
    rng = np.random.default_rng(n * 7919 + classes * 31 + dim)
    check(case(n, classes, dim, dtype, rng), top=min(classes, 10))
    check(case(n, classes, dim, dtype, rng, pad=3, offset=1, bias=False, unlabelled=0.0),
          top=min(classes, 1))
    check(case(n, classes, dim, dtype, rng, pad=4, masked=0.3, labels=False), top=0)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "q8"])
@pytest.mark.parametrize("top", [1, 7, 33, 64])
def test_many_best_classes(top, dtype):
    """Few tiles and many of them, for few rows and for more."""
    rng = np.random.default_rng(top)
    for n, classes, dim in ((3, 64, 32), (3, 6000, 32), (70, 64, 36), (70, 5000, 64), (70, 2200, 128)):
        say(f"best {top} of {n} x {classes} x {dim} {dtype}")
        check(case(n, classes, dim, dtype, rng, bias=dim != 128, masked=0.2), top=top, grad=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "q8"])
@pytest.mark.parametrize("n", [5, 80])
def test_equal_logits_give_the_lowest_classes(n, dtype):
    """Rows of zeros, and classes that repeat: every logit has many equals."""
    rng = np.random.default_rng(n)
    k = case(n, 3000, 32, dtype, rng, bias=False)
    k["h"][::2] = 0
    k["hv"][::2] = 0
    if dtype == "q8":
        for t in k["w"]:
            t[100:] = t[:100].repeat(29, 1)
    else:
        k["w"][100:] = k["w"][:100].repeat(29, 1)
    k["wv"][100:] = np.tile(k["wv"][:100], (29, 1))
    a = check(k, top=20, grad=False)
    assert a.ids[0].tolist() == list(range(20))


@pytest.mark.parametrize("top", [1, 20, 64])
@pytest.mark.parametrize("n", [3, 40, 70])
def test_more_tiles_above_the_bar_than_a_list_holds(n, top):
    """Rows of zeros whose logits are the bias alone: all equal, rising, falling, and
    nearly all classes out."""
    classes, dim = 60_000, 8
    op = P.LogProbs(n, classes, dim, dtype="bf16", top=top)
    h = torch.zeros(n, dim, device="cuda", dtype=torch.bfloat16)
    w = torch.randn(classes, dim, device="cuda").to(torch.bfloat16)
    up = torch.arange(classes, device="cuda", dtype=torch.float32) * 2.0 ** -12
    few = torch.full((classes,), -math.inf, device="cuda")
    few[59_000:59_000 + 3 * top:3] = up[:top]
    for name, b, ids in (("equal", torch.zeros_like(up), torch.arange(top)),
                         ("rising", up, classes - 1 - torch.arange(top)),
                         ("falling", up.flip(0), torch.arange(top)),
                         ("few in", few, 59_000 + 3 * torch.arange(top).flip(0))):
        say(f"{name}, {n} rows, best {top}")
        a = op.log_probs(h, w, bias=b)
        assert (a.ids.cpu() == ids.to(torch.int32)).all()
        want = torch.log_softmax(b.double(), 0)[ids.cuda()]
        assert (a.top_logp - want).abs().max().item() <= 1e-5
        op.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "q8"])
@pytest.mark.parametrize("n", [6, 75])
@pytest.mark.parametrize("lowest", [-math.inf, -3.4e38, -1e29])
def test_classes_that_are_out(n, dtype, lowest):
    """A mask by -inf or by a type's lowest value: their rows of w may hold anything.  Few
    classes that are left, one, and none."""
    rng = np.random.default_rng(n)
    for left in (150, 3, 1, 0):
        say(f"{left} classes left, mask {lowest}, {n} rows of {dtype}")
        k = case(n, 300, 48, dtype, rng)
        out = rng.permutation(300)[left:]
        k["b"][out] = lowest
        k["tb"] = vec(k["b"])
        at = torch.from_numpy(out).cuda()
        if dtype == "q8":
            k["w"].scales[at[::2]] = 255
            k["w"].codes.view(torch.uint8)[at[1::2]] = 127
        else:
            k["w"][at[::2]] = math.nan
            k["w"][at[1::2]] = math.inf
        k["wv"][out] = math.nan
        a = check(k, top=5)
        if left == 0:
            assert (a.lse == -math.inf).all() and not a.entropy.any() and (a.ids == -1).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [6, 75])
def test_nan_stays_in_its_row(n, dtype):
    rng = np.random.default_rng(n)
    k = case(n, 100, 32, dtype, rng, unlabelled=0.0)
    op = P.LogProbs(n, 100, 32, dtype=dtype, top=3, grad=True)
    clean = op.log_probs(k["h"], k["w"], k["tl"], k["tb"])
    k["h"][2, 5] = math.nan
    a = op.log_probs(k["h"], k["w"], k["tl"], k["tb"])
    keep = [i for i in range(n) if i != 2]
    for x, y in zip(a, clean):
        assert torch.equal(x[keep], y[keep])
    assert all(t[2].isnan().all() for t in (a.logp, a.entropy, a.lse, a.top_logp))
    assert (a.ids[2] == -1).all()
    dl = torch.ones(n, device="cuda")
    dh = op.grad(k["h"], k["w"], a, k["tl"], dl, dl, k["tb"])[0]
    assert dh[2].isnan().all() and not dh[keep].isnan().any()
    dl[2] = 0  # a row whose weights are 0 is not read
    dh, dw, db = op.grad(k["h"], k["w"], a, k["tl"], dl, dl, k["tb"])
    assert not dh[2].any() and not dw.isnan().any() and not db.isnan().any()
    k["w"][9, 0] = math.nan  # in a class that counts: in every row
    a = op.log_probs(k["h"], k["w"], k["tl"], k["tb"])
    assert a.lse.isnan().all() and (a.ids == -1).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "q8"])
@pytest.mark.parametrize("size", [8.0, 60.0, 1e5])
def test_confident_rows(size, dtype):
    """Logits of tens, hundreds and a million: entropies near 0, probabilities that vanish."""
    rng = np.random.default_rng(12)
    for n in (30, 200):
        check(case(n, 90, 64, dtype, rng, size=size), top=3)


def test_labels_out_of_range_are_reported():
    rng = np.random.default_rng(1)
    for n in (4, 80):
        k = case(n, 30, 16, "f32", rng, unlabelled=0.0)
        op = P.LogProbs(n, 30, 16, top=2, grad=True)
        k["tl"][1] = 30
        a = op.log_probs(k["h"], k["w"], k["tl"], k["tb"])
        assert a.logp.isnan().nonzero().flatten().tolist() == [1] and not a.lse.isnan().any()
        with pytest.raises(P.HugeError) as e:
            op.check()
        assert e.value.status == B.HUGE_ERR_ID_OUT_OF_RANGE
        op.check()
        ones = torch.ones(n, device="cuda")
        dh = op.grad(k["h"], k["w"], a, k["tl"], dlogp=ones, bias=k["tb"])[0]
        assert not dh[1].any() and dh[0].any()
        with pytest.raises(P.HugeError):
            op.check()


def on_device(h, w, labels, bias, top, dl=None, de=None):
    """In float64 on the GPU, for sizes beyond the oracle's."""
    h, w = h.double(), w.double()
    x = h @ w.t() + (0 if bias is None else bias.double())
    lse = torch.logsumexp(x, 1)
    lp = x - lse[:, None]
    p = lp.exp()
    entropy = -(p * lp).sum(1)
    logp = lp.gather(1, labels.long()[:, None])[:, 0]
    out = [logp, entropy, lse]
    if top:
        v, at = lp.sort(dim=1, descending=True, stable=True)
        out += [at[:, :top], v[:, :top]]
    if dl is not None:
        g = p * (-dl.double()[:, None] - de.double()[:, None] * (lp + entropy[:, None]))
        g[torch.arange(len(h), device="cuda"), labels.long()] += dl.double()
        out += [g @ w, g.t().contiguous() @ h, g.sum(0)]
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16", "q8"])
@pytest.mark.parametrize("n,classes,dim,top", [(70, 140_003, 32, 10), (96, 150_001, 100, 5),
                                               (9_001, 3_001, 256, 3), (2, 200_003, 64, 64),
                                               (60, 100_001, 48, 12), (20_011, 37, 32, 2),
                                               (4_100, 9_001, 384, 4), (333, 64_000, 128, 10)])
def test_many_tiles(n, classes, dim, top, dtype):
    say(f"log probs {n} x {classes} x {dim} {dtype}, best {top}")
    g = torch.Generator(device="cuda").manual_seed(n + dim)
    new = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    kind = TYPES["bf16" if dtype == "q8" else dtype]
    h = new(n, dim).to(kind)
    w = (new(classes, dim) * 1.5 / math.sqrt(dim)).to(kind)
    labels = torch.randint(0, classes, (n,), device="cuda", generator=g).to(torch.int32)
    bias = None if dim == 128 else new(classes)
    table = w
    if dtype == "q8":
        table = P.q8_rows(w)
        w = P.q8_values(table)
    grad = dtype != "q8"
    op = P.LogProbs(n, classes, dim, dtype=dtype, top=top, grad=grad)
    a = op.log_probs(h, table, labels, bias)
    dl, de = new(n), 0.1 * new(n)
    want = on_device(h, w, labels, bias, top, dl if grad else None, de)
    assert torch.equal(a.ids.long(), want[3])
    got = [a.logp, a.entropy, a.lse, None, a.top_logp]
    if grad:
        got += op.grad(h, table, a, labels, dl, de, bias)
    # norms here: fp32 sums of many terms about 1e-6, a rounding to bf16 and one of the
    # elements before it 2^-8 each at most
    for k, (x, y) in enumerate(zip(got, want)):
        if x is None:
            continue
        tol = 2.0 ** -8 if dtype == "bf16" and k in (5, 6) else 3e-6
        err = ((x.double() - y).norm() / y.norm()).item()
        far = ((x.double() - y).abs().max() / y.abs().max()).item()
        say(f"  output {k}: {err:.3g} of the norm, {far:.3g} of the largest")
        assert err <= tol and far <= 4 * tol, k
    op.check()


def test_fewer_rows_than_planned():
    """One workspace serves every number of rows up to the largest."""
    rng = np.random.default_rng(3)
    for dtype in ("f32", "bf16", "q8"):
        op = P.LogProbs(300, 500, 64, dtype=dtype, top=4, grad=dtype != "q8")
        for n in (300, 1, 16, 17, 33, 64, 65, 128, 299, 0):
            k = case(n, 500, 64, dtype, rng)
            check(k, top=4, op=op, grad=n > 0)


# --------------------------------------------------------------------------- #
# Norms of gradients
# --------------------------------------------------------------------------- #
LISTS = [[1], [5, 0, 3], [16384], [16383, 16385, 2], [40_000, 7, 100_003], [33] * 200,
         [1_000_003, 1], [16384 * 5, 16384 * 3 + 8]]


def gradients(sizes, dtype, rng, offset=0):
    out = []
    for k, n in enumerate(sizes):
        t = TYPES[["f32", "bf16"][k % 2] if dtype == "mixed" else dtype]
        buf = torch.from_numpy(rng.normal(size=n + offset) * 10.0 ** rng.integers(-3, 3)).to(t).cuda()
        out.append(buf[offset:])
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("which", range(len(LISTS)))
def test_grad_norm_and_clipping(which, dtype):
    rng = np.random.default_rng(which)
    for offset in (0, 1):
        gs = gradients(LISTS[which], dtype, rng, offset)
        vals = [g.double().cpu().numpy() for g in gs]
        want = ref.grad_norm(vals)
        norm = P.grad_norm(gs)
        assert norm.shape == (1,) and norm.dtype is torch.float32
        assert abs(norm.item() - want) <= 2 * U * want  # rounded once, from sums in fp64
        for most in (want * 2, want * 0.3, math.inf):
            cs = [g.clone() for g in gs]
            assert torch.equal(P.clip_grads(cs, most), norm)
            f = min(1.0, most / want)
            for c, g, v in zip(cs, gs, vals):
                if f == 1.0:
                    assert torch.equal(c, g)
                    continue
                half = BF if c.dtype is torch.bfloat16 else U
                err = np.abs(c.double().cpu().numpy() - v * f)
                assert (err <= (half + 4 * U) * np.abs(v * f) + 1e-45).all()


def test_grad_norm_at_the_ends_of_the_range():
    """Squares that fp32 does not hold, nothing, zeros, infinities and NaN."""
    one = lambda *v: torch.tensor(v, device="cuda")  # noqa: E731
    assert P.grad_norm([one(3e38, 0.0)]).item() == pytest.approx(3e38, rel=1e-6)
    assert P.grad_norm([one(1e-38, 0.0)]).item() == pytest.approx(1e-38, rel=1e-6)
    assert P.grad_norm([one(3e38, 3e38)]).item() == math.inf
    assert P.grad_norm([torch.empty(0, device="cuda")]).item() == 0
    assert P.grad_norm([torch.zeros(99, device="cuda")]).item() == 0
    g = torch.zeros(99, device="cuda")
    assert P.clip_grads([g], 1e-3).item() == 0 and not g.any()
    g = one(3e38, 3e38)
    P.clip_grads([g], 1.0)
    assert g.tolist() == pytest.approx([0.5 ** 0.5] * 2, rel=1e-6)
    for bad in (math.nan, math.inf):
        g = one(1.0, bad)
        assert not math.isfinite(P.clip_grads([g], 0.5).item())
        assert g[0].item() == 1.0


@pytest.mark.parametrize("states", ["f32", "q8"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "mixed"])
def test_clipped_step_is_a_step_with_scaled_gradients(dtype, states):
    """Bit for bit that of grad_scale = factor, and with a norm below the largest that
    of no clipping."""
    rng = np.random.default_rng(6)
    sizes = [300, 5000, 16385, 1]
    params = [torch.from_numpy(rng.normal(size=n)).float().cuda() for n in sizes]
    gs = gradients(sizes, dtype, rng)
    before = [g.clone() for g in gs]
    norm = P.grad_norm(gs).double().item()
    for most, scale in ((norm * 10, 1.0), (norm * 0.25, 1.0), (norm * 0.25, -2.0), (math.inf, 0.5)):
        a, b = (P.AdamW([p.clone() for p in params], states=states) for _ in range(2))
        for _ in range(3):
            got = a.step(gs, max_norm=most, grad_scale=scale)
            full = abs(scale) * ref.grad_norm([g.double().cpu().numpy() for g in gs])
            factor = scale * min(1.0, most / full)
            assert got.item() == pytest.approx(full, rel=2 * U)
            assert b.step(gs, grad_scale=float(np.float32(factor))) is None
        for x, y in zip(a.params, b.params):
            # the factor is rounded once from fp64 sums in another order: one step apart at most
            assert (x - y).abs().max().item() <= 1e-6
        m, v = a.values()
        m2, v2 = b.values()
        for x, y in zip(m + v, m2 + v2):
            if states == "f32":
                assert ((x - y).abs() <= 32 * U * y.abs()).all()
        a.check()
    for g, h in zip(gs, before):
        assert torch.equal(g, h)


@pytest.mark.parametrize("states", ["f32", "q8"])
def test_clipped_step_without_a_finite_norm_moves_nothing(states):
    for bad in (math.nan, math.inf):
        p = torch.randn(1000, device="cuda")
        opt = P.AdamW([p], states=states)
        g = torch.randn(1000, device="cuda")
        opt.step([g], max_norm=1.0)
        keep, m, v = p.clone(), *([t.clone() for t in ts] for ts in opt.values())
        g[7] = bad
        assert not math.isfinite(opt.step([g], max_norm=1.0).item())
        assert torch.equal(p, keep)
        for x, y in zip(opt.values()[0] + opt.values()[1], m + v):
            assert torch.equal(x, y)
        with pytest.raises(P.HugeError) as e:
            opt.check()
        assert e.value.status == B.HUGE_ERR_NOT_FINITE
