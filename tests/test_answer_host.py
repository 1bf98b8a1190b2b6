"""Host-side checks of RMS norm, rows in 8 bits, log probabilities and clipped
gradients (no GPU): sizes, and arguments that are refused before any launch."""
import ctypes
import math

import pytest

import paper_2307_14490_amd as P
from paper_2307_14490_amd import binding as B

PTR = 1 << 20  # never followed: every call here is refused
NONE = None
F32, BF16, Q8 = B.HUGE_DTYPE_F32, B.HUGE_DTYPE_BF16, B.HUGE_DTYPE_Q8


def _rms(x=PTR, ld_x=32, res=PTR, ld_res=32, n=8, dim=32, dtype=F32, gamma=PTR, eps=1e-5,
         total=PTR, ld_total=32, y=PTR, ld_y=32, codes=NONE, ld_codes=0, scales=NONE, ld_scales=0,
         rstd=PTR):
    return P.load().huge_rms_norm(x, ld_x, res, ld_res, n, dim, dtype, gamma, eps, total, ld_total,
                                  y, ld_y, codes, ld_codes, scales, ld_scales, rstd, None)


EIGHT = dict(y=NONE, codes=PTR, ld_codes=32, scales=PTR, ld_scales=1)


@pytest.mark.parametrize("kw", [
    dict(x=NONE), dict(gamma=NONE), dict(y=NONE), dict(total=NONE), dict(res=NONE), dict(dim=0),
    dict(dim=8193), dict(n=-1), dict(n=2**31), dict(dtype=2), dict(dtype=-1), dict(eps=0.0),
    dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(ld_x=31), dict(ld_res=31),
    dict(ld_total=31), dict(ld_y=31), dict(x=PTR + 2), dict(res=PTR + 1), dict(total=PTR + 2),
    dict(y=PTR + 2), dict(gamma=PTR + 2), dict(rstd=PTR + 2), {**EIGHT, "y": PTR},
    {**EIGHT, "scales": NONE}, {**EIGHT, "codes": NONE}, {**EIGHT, "ld_codes": 31},
    {**EIGHT, "ld_scales": 0}, {**EIGHT, "dim": 33, "ld_x": 33, "ld_res": 33, "ld_total": 33,
                                "ld_codes": 33},
    dict(x=NONE, n=1, res=NONE, total=NONE),
])
def test_rms_norm_refuses(kw):
    assert _rms(**kw) == B.HUGE_ERR_INVALID_ARG


def test_rms_norm_of_no_rows_needs_no_rows():
    assert _rms(n=0, x=NONE, y=NONE, res=NONE, total=NONE, rstd=NONE) == B.HUGE_OK


def test_rms_norm_backward_refuses():
    L = P.load()

    def call(dy=PTR, total=PTR, dt=PTR, ld=32, n=8, dim=32, dtype=0, gamma=PTR, rstd=PTR, dx=PTR,
             dg=PTR, ws=PTR, size=1 << 30):
        return L.huge_rms_norm_backward(dy, ld, total, ld, dt, ld, n, dim, dtype, gamma, rstd, dx,
                                        ld, dg, ws, size, None)

    for kw in (dict(dy=NONE), dict(total=NONE), dict(rstd=NONE), dict(gamma=NONE), dict(dim=8193),
               dict(dim=0), dict(n=-1), dict(ws=PTR + 4), dict(ld=31), dict(dtype=2),
               dict(dt=PTR + 2), dict(dx=PTR + 2), dict(dg=PTR + 2), dict(rstd=PTR + 1)):
        assert call(**kw) == B.HUGE_ERR_INVALID_ARG, kw
    assert call(size=10) == B.HUGE_ERR_WORKSPACE
    assert call(ws=NONE) == B.HUGE_ERR_WORKSPACE
    assert call(dg=NONE, dx=NONE) == B.HUGE_OK  # nothing is wanted
    assert L.huge_rms_norm_workspace_bytes(-1, 32) == 0
    assert L.huge_rms_norm_workspace_bytes(5, 0) == 0
    assert L.huge_rms_norm_workspace_bytes(0, 32) > 0


@pytest.mark.parametrize("kw", [
    dict(x=NONE), dict(codes=NONE), dict(scales=NONE), dict(ld_x=31), dict(ld_codes=31),
    dict(ld_scales=0), dict(dim=33), dict(dim=0), dict(dim=8193), dict(n=-1), dict(dtype=2),
    dict(x=PTR + 2),
])
def test_rows_in_8_bits_refuse(kw):
    a = dict(x=PTR, ld_x=32, n=4, dim=32, dtype=F32, codes=PTR, ld_codes=32, scales=PTR,
             ld_scales=1)
    a.update(kw)
    L = P.load()
    assert L.huge_quantise_rows(a["x"], a["ld_x"], a["n"], a["dim"], a["dtype"], a["codes"],
                                a["ld_codes"], a["scales"], a["ld_scales"],
                                None) == B.HUGE_ERR_INVALID_ARG
    assert L.huge_dequantise_rows(a["codes"], a["ld_codes"], a["scales"], a["ld_scales"], a["n"],
                                  a["dim"], a["x"], a["ld_x"], a["dtype"],
                                  None) == B.HUGE_ERR_INVALID_ARG


def _cfg(**kw):
    base = dict(num_classes=1000, max_rows=64, dim=32, dtype=F32, table_dtype=F32, top=5, grad=1)
    base.update(kw)
    return B.HugeLogProbsConfig(**base)


def _size(**kw):
    return P.load().huge_log_probs_workspace_bytes(ctypes.byref(_cfg(**kw)))


@pytest.mark.parametrize("kw", [
    dict(num_classes=0), dict(num_classes=2**31), dict(max_rows=0), dict(max_rows=2**31),
    dict(dim=0), dict(dim=6), dict(dim=1028), dict(dtype=2), dict(dtype=-1), dict(grad=2),
    dict(top=-1), dict(top=65), dict(top=11, num_classes=10), dict(table_dtype=BF16),
    dict(table_dtype=Q8), dict(table_dtype=Q8, dtype=BF16), dict(table_dtype=3),
])
def test_invalid_configs_have_no_workspace(kw):
    assert _size(**kw) == 0


@pytest.mark.parametrize("dtype,table", [(F32, F32), (BF16, BF16), (BF16, Q8)])
def test_workspace_never_shrinks_with_rows(dtype, table):
    """A call of fewer rows than planned needs no more."""
    for dim in (4, 32, 128, 260, 388, 1024):
        for classes in (1, 33, 50_021, 3_000_000):
            for top in (0, min(classes, 10), min(classes, 64)):
                last = 0
                for rows in (1, 15, 16, 17, 32, 33, 48, 64, 65, 96, 4096, 8192, 9000, 131072,
                             200_000):
                    now = _size(dtype=dtype, table_dtype=table, grad=0, dim=dim, max_rows=rows,
                                num_classes=classes, top=top)
                    assert now >= last > -1 and now > 0
                    last = now
                if table != Q8:
                    assert _size(dtype=dtype, table_dtype=table, grad=1, dim=dim, max_rows=rows,
                                 num_classes=classes, top=top) >= last


def test_workspace_stays_bounded():
    """The tiles' largest logits take 1 GiB at most, the table's copy 2."""
    for rows in (1, 64, 65, 4096, 100_000):
        for dim in (4, 128, 1024):
            assert _size(num_classes=2**31 - 1, max_rows=rows, dim=dim, grad=0, top=64) < 2**32
    # few rows keep no copy of the table
    assert _size(num_classes=1_000_000, dim=128, max_rows=16, grad=0, top=0) < 1 << 23
    assert _size(num_classes=2**31 - 1, max_rows=2**31 - 1, dim=1024) > 2**42  # no wrap


def _call(cfg=None, h=PTR, ld_h=32, n=8, w=PTR, ld_w=32, scales=NONE, ld_scales=0, bias=NONE,
          labels=PTR, logp=PTR, entropy=PTR, lse=PTR, ids=PTR, best=PTR, status=PTR, ws=PTR,
          ws_bytes=1 << 40):
    c = _cfg() if cfg is None else cfg
    return P.load().huge_log_probs(ctypes.byref(c), h, ld_h, n, w, ld_w, scales, ld_scales, bias,
                                   labels, logp, entropy, lse, ids, best, status, ws, ws_bytes,
                                   None)


EIGHT_BITS = _cfg(dtype=BF16, table_dtype=Q8, grad=0)


@pytest.mark.parametrize("kw", [
    dict(cfg=_cfg(dim=30)), dict(h=NONE), dict(w=NONE), dict(lse=NONE), dict(status=NONE),
    dict(logp=NONE), dict(labels=NONE), dict(ids=NONE), dict(best=NONE), dict(n=-1), dict(n=65),
    dict(ld_h=31), dict(ld_w=31), dict(h=PTR + 2), dict(w=PTR + 2), dict(labels=PTR + 2),
    dict(entropy=PTR + 2), dict(ws=PTR + 128), dict(scales=PTR), dict(bias=PTR + 1),
    dict(cfg=_cfg(top=0)), dict(cfg=EIGHT_BITS), dict(cfg=EIGHT_BITS, scales=PTR, ld_scales=0),
    dict(cfg=EIGHT_BITS, scales=PTR, ld_scales=1, ld_w=31),
])
def test_log_probs_refuses(kw):
    assert _call(**kw) == B.HUGE_ERR_INVALID_ARG


def test_log_probs_refuses_a_small_workspace():
    assert _call(ws_bytes=1000) == B.HUGE_ERR_WORKSPACE
    assert _call(ws=NONE) == B.HUGE_ERR_WORKSPACE
    assert _call(n=0, h=NONE, labels=NONE, logp=NONE, lse=NONE, ids=NONE, best=NONE) == B.HUGE_OK


@pytest.mark.parametrize("kw", [
    dict(grad=0), dict(dh=PTR + 2), dict(lse=NONE), dict(labels=NONE), dict(entropy=NONE),
    dict(dl=PTR + 2), dict(de=PTR + 1), dict(db=PTR + 2), dict(h=NONE),
])
def test_log_probs_grad_refuses(kw):
    c = _cfg(grad=kw.get("grad", 1))
    g = lambda k: kw.get(k, PTR)  # noqa: E731
    st = P.load().huge_log_probs_grad(ctypes.byref(c), g("h"), 32, 8, PTR, 32, None, g("labels"),
                                      g("lse"), g("entropy"), g("dl"), g("de"), g("dh"), PTR,
                                      g("db"), PTR, PTR, 1 << 40, None)
    assert st == B.HUGE_ERR_INVALID_ARG


def _tensors(*ts):
    out = (B.HugeGradTensor * len(ts))()
    for t, (p, n, d) in zip(out, ts):
        t.d_grad, t.n, t.dtype = p, n, d
    return out


@pytest.mark.parametrize("bad", [(NONE, 5, 0), (PTR + 2, 5, 0), (PTR + 1, 5, 1), (PTR, -1, 0),
                                 (PTR, (1 << 40) + 1, 0), (PTR, 5, 2)])
def test_norms_refuse_bad_tensors(bad):
    L = P.load()
    ts = _tensors((PTR, 5, 0), bad)
    assert L.huge_grad_norm(ts, 2, PTR, PTR, 1 << 30, None) == B.HUGE_ERR_INVALID_ARG
    assert L.huge_clip_grads(ts, 2, 1.0, PTR, PTR, 1 << 30, None) == B.HUGE_ERR_INVALID_ARG


def test_norms_refuse():
    L = P.load()
    ts = _tensors((PTR, 5, 0))
    for call in (lambda n=1, t=ts, norm=PTR, ws=PTR, size=1 << 30: L.huge_grad_norm(
            t, n, norm, ws, size, None),
            lambda n=1, t=ts, norm=PTR, ws=PTR, size=1 << 30: L.huge_clip_grads(
                t, n, 1.0, norm, ws, size, None)):
        assert call(n=-1) == B.HUGE_ERR_INVALID_ARG
        assert call(t=None) == B.HUGE_ERR_INVALID_ARG
        assert call(norm=PTR + 2) == B.HUGE_ERR_INVALID_ARG
        assert call(ws=NONE) == B.HUGE_ERR_WORKSPACE
        assert call(size=100) == B.HUGE_ERR_WORKSPACE
        assert call(ws=PTR + 8) == B.HUGE_ERR_INVALID_ARG
    assert L.huge_grad_norm(ts, 1, None, PTR, 1 << 30, None) == B.HUGE_ERR_INVALID_ARG
    for most in (0.0, -1.0, math.nan):
        assert L.huge_clip_grads(ts, 1, most, PTR, PTR, 1 << 30, None) == B.HUGE_ERR_INVALID_ARG
    assert L.huge_grad_norm_workspace_bytes(-1) == 0
    sizes = [L.huge_grad_norm_workspace_bytes(n) for n in (0, 1, 64, 65, 1000)]
    assert sizes == sorted(sizes) and sizes[0] > 0


def test_clipped_step_refuses():
    L = P.load()
    ts = (B.HugeAdamwTensor * 1)()
    ts[0].d_param = ts[0].d_grad = ts[0].d_state = PTR
    ts[0].n = 5

    def call(most=1.0, norm=PTR, ws=PTR, size=1 << 30, count=1, status=PTR, step=1):
        c = B.HugeAdamwConfig(1e-3, 0.9, 0.999, 1e-8, 0.0, 1.0, step, 0)
        return L.huge_adamw_step_clipped(ctypes.byref(c), ts, count, most, norm, status, ws, size,
                                         None)

    for kw in (dict(most=0.0), dict(most=-1.0), dict(most=math.nan), dict(norm=PTR + 2),
               dict(count=-1), dict(status=NONE), dict(step=0), dict(ws=PTR + 8)):
        assert call(**kw) == B.HUGE_ERR_INVALID_ARG, kw
    assert call(size=100) == call(ws=NONE) == B.HUGE_ERR_WORKSPACE


def test_python_refuses_what_is_no_gpu_tensor():
    torch = pytest.importorskip("torch")
    x, g = torch.zeros(4, 32), torch.ones(32)
    for call in (lambda: P.rms_norm(x, g), lambda: P.q8_rows(x), lambda: P.grad_norm([x]),
                 lambda: P.clip_grads([x], 1.0), lambda: P.q8_values(x), lambda: P.q8_values((x, x)),
                 lambda: P.rms_norm_backward(x, x, g, g)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: P.grad_norm([]), lambda: P.clip_grads([], 1.0)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(P.HugeError):
        P.LogProbs(4, 10, 6)
    with pytest.raises(P.HugeError):
        P.LogProbs(4, 10, 8, dtype="q8", grad=True)
