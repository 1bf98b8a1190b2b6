"""Host-side checks of the softmax head's C ABI (no GPU): sizes, and arguments that
are refused before any launch."""
import ctypes
import math

import pytest

import paper_2307_14490_amd as P
from paper_2307_14490_amd import binding as B

PTR = 1 << 20  # never followed: every call here is refused
NONE = None


def _soft(**kw):
    base = dict(num_classes=1000, max_rows=64, dim=32, dtype=B.HUGE_DTYPE_F32, grad=1)
    base.update(kw)
    return B.HugeSoftmaxConfig(**base)


def test_new_status_has_a_string():
    assert B.status_string(B.HUGE_ERR_NOT_FINITE) not in ("", "unknown status")


@pytest.mark.parametrize("kw", [
    dict(num_classes=0), dict(num_classes=2**31), dict(max_rows=0), dict(max_rows=2**31),
    dict(dim=0), dict(dim=6), dict(dim=1028), dict(dtype=2), dict(dtype=-1), dict(grad=2),
])
def test_invalid_softmax_configs_have_no_workspace(kw):
    assert P.load().huge_softmax_workspace_bytes(ctypes.byref(_soft(**kw))) == 0


def test_softmax_workspace_grows_with_rows_and_stays_bounded_in_classes():
    size = lambda **kw: P.load().huge_softmax_workspace_bytes(ctypes.byref(_soft(**kw)))  # noqa: E731
    assert 0 < size(grad=0) < size() <= size(max_rows=1 << 17) < size(max_rows=1 << 20)
    assert size(num_classes=10_000_000, dim=128) == pytest.approx(
        size(num_classes=2**31 - 1, dim=128), rel=0.01)
    # the largest sizes do not wrap
    assert size(num_classes=2**31 - 1, max_rows=2**31 - 1, dim=1024) > 2**42


def _loss(cfg=None, h=PTR, ld_h=32, n=8, w=PTR, ld_w=32, bias=NONE, labels=PTR, weight=NONE,
          loss=PTR, lse=PTR, total=NONE, status=PTR, ws=PTR, ws_bytes=1 << 40):
    c = _soft() if cfg is None else cfg
    return P.load().huge_softmax_loss(ctypes.byref(c), h, ld_h, n, w, ld_w, bias, labels, weight,
                                      loss, lse, total, status, ws, ws_bytes, None)


@pytest.mark.parametrize("kw", [
    dict(cfg=_soft(dim=30)), dict(h=NONE), dict(w=NONE), dict(labels=NONE), dict(loss=NONE),
    dict(lse=NONE), dict(status=NONE), dict(n=-1), dict(n=65), dict(ld_h=31), dict(ld_w=31),
    dict(h=PTR + 2), dict(labels=PTR + 2), dict(total=PTR + 4), dict(ws=PTR + 128),
])
def test_softmax_loss_refuses(kw):
    assert _loss(**kw) == B.HUGE_ERR_INVALID_ARG


def test_softmax_refuses_a_small_workspace():
    assert _loss(ws_bytes=1000) == B.HUGE_ERR_WORKSPACE
    assert _loss(ws=NONE) == B.HUGE_ERR_WORKSPACE


@pytest.mark.parametrize("kw", [dict(scale=math.nan), dict(scale=math.inf), dict(grad=0),
                                dict(dh=PTR + 2), dict(lse=NONE)])
def test_softmax_grad_refuses(kw):
    c = _soft(grad=kw.get("grad", 1))
    st = P.load().huge_softmax_grad(ctypes.byref(c), PTR, 32, 8, PTR, 32, None, PTR, None,
                                    kw.get("lse", PTR), kw.get("scale", 1.0), kw.get("dh", PTR),
                                    PTR, PTR, PTR, PTR, 1 << 40, None)
    assert st == B.HUGE_ERR_INVALID_ARG


def _norm(x=PTR, ld_x=32, n=8, dim=32, dtype=0, gamma=PTR, beta=PTR, eps=1e-5, y=PTR, ld_y=32,
          mean=PTR, rstd=PTR):
    return P.load().huge_layer_norm(x, ld_x, n, dim, dtype, gamma, beta, eps, y, ld_y, mean, rstd,
                                    None)


@pytest.mark.parametrize("kw", [
    dict(x=NONE), dict(y=NONE), dict(gamma=NONE), dict(beta=NONE), dict(dim=0), dict(dim=8193),
    dict(n=-1), dict(n=2**31), dict(dtype=3), dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan),
    dict(eps=math.inf), dict(ld_x=31), dict(ld_y=31), dict(mean=NONE), dict(rstd=NONE),
    dict(x=PTR + 2), dict(gamma=PTR + 1),
])
def test_layer_norm_refuses(kw):
    assert _norm(**kw) == B.HUGE_ERR_INVALID_ARG


def test_layer_norm_backward_refuses():
    L = P.load()

    def call(dy=PTR, x=PTR, n=8, dim=32, dx=PTR, dg=PTR, db=PTR, ws=PTR, size=1 << 30, mean=PTR):
        return L.huge_layer_norm_backward(dy, 32, x, 32, n, dim, 0, PTR, mean, PTR, dx, 32, dg, db,
                                          ws, size, None)

    for kw in (dict(dy=NONE), dict(x=NONE), dict(mean=NONE), dict(dim=8193), dict(dg=NONE),
               dict(db=NONE), dict(ws=PTR + 4), dict(n=-1)):
        assert call(**kw) == B.HUGE_ERR_INVALID_ARG, kw
    assert call(size=10) == B.HUGE_ERR_WORKSPACE
    assert call(ws=NONE) == B.HUGE_ERR_WORKSPACE
    assert L.huge_layer_norm_workspace_bytes(-1, 32) == 0
    assert L.huge_layer_norm_workspace_bytes(5, 0) == 0
    assert L.huge_layer_norm_workspace_bytes(0, 32) > 0


def test_adamw_state_sizes():
    L = P.load()
    assert L.huge_adamw_state_bytes(0, B.HUGE_STATE_F32) == 0
    assert L.huge_adamw_state_bytes(1, B.HUGE_STATE_F32) == 8 * 256
    assert L.huge_adamw_state_bytes(257, B.HUGE_STATE_Q8) == 2 * 512 + 2 * 8
    assert L.huge_adamw_state_bytes(5, 2) == 0
    assert L.huge_adamw_state_bytes(-1, 0) == 0
    assert L.huge_adamw_state_bytes((1 << 40) + 1, 0) == 0


@pytest.mark.parametrize("kw", [
    dict(lr=-1.0), dict(lr=math.nan), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0),
    dict(beta2=math.nan), dict(eps=0.0), dict(eps=-1.0), dict(eps=1e-31), dict(weight_decay=-1.0),
    dict(grad_scale=math.inf), dict(step=0), dict(state_kind=2),
])
def test_adamw_refuses_bad_settings(kw):
    base = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, grad_scale=1.0,
                step=1, state_kind=0)
    base.update(kw)
    c = B.HugeAdamwConfig(**base)
    assert P.load().huge_adamw_step(ctypes.byref(c), None, 0, PTR, None) == B.HUGE_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [
    dict(d_param=NONE), dict(d_grad=NONE), dict(d_state=NONE), dict(n=-1), dict(n=(1 << 40) + 1),
    dict(param_dtype=2), dict(grad_dtype=-1), dict(d_state=PTR + 8), dict(d_param=PTR + 2),
])
def test_adamw_refuses_bad_tensors(kw):
    base = dict(d_param=PTR, d_grad=PTR, d_state=PTR, n=10, param_dtype=0, grad_dtype=0)
    c = B.HugeAdamwConfig(1e-3, 0.9, 0.999, 1e-8, 0.0, 1.0, 1, 0)
    ts = (B.HugeAdamwTensor * 2)()
    for t, d in zip(ts, (base, {**base, **kw})):
        for k, v in d.items():
            setattr(t, k, v)
    L = P.load()
    assert L.huge_adamw_step(ctypes.byref(c), ts, 2, PTR, None) == B.HUGE_ERR_INVALID_ARG
    assert L.huge_adamw_step(ctypes.byref(c), ts, -1, PTR, None) == B.HUGE_ERR_INVALID_ARG
    assert L.huge_adamw_step(ctypes.byref(c), None, 2, PTR, None) == B.HUGE_ERR_INVALID_ARG
    assert L.huge_adamw_step(ctypes.byref(c), ts, 2, None, None) == B.HUGE_ERR_INVALID_ARG


def test_adamw_state_calls_refuse():
    L = P.load()
    ts = (B.HugeAdamwTensor * 1)()
    ts[0].d_state, ts[0].n = PTR, 5
    good, bad = (ctypes.c_void_p * 1)(PTR), (ctypes.c_void_p * 1)(None)
    for fn in (L.huge_adamw_get_state, L.huge_adamw_set_state):
        assert fn(ts, 1, 0, good, bad, None) == B.HUGE_ERR_INVALID_ARG
        assert fn(ts, 1, 0, bad, good, None) == B.HUGE_ERR_INVALID_ARG
        assert fn(ts, 1, 7, good, good, None) == B.HUGE_ERR_INVALID_ARG
        assert fn(ts, 1, 0, None, good, None) == B.HUGE_ERR_INVALID_ARG
        assert fn(None, 1, 0, good, good, None) == B.HUGE_ERR_INVALID_ARG


@pytest.mark.parametrize("dtype,rows,dim", [(0, 1, 128), (0, 64, 512), (0, 16, 1024), (1, 64, 448),
                                            (1, 1, 1024)])
def test_losses_of_few_rows_keep_no_copy_of_the_table(dtype, rows, dim):
    """They read it as it lies: what is left are the partial sums."""
    size = lambda **kw: P.load().huge_softmax_workspace_bytes(  # noqa: E731
        ctypes.byref(_soft(num_classes=1_000_000, dim=dim, dtype=dtype, **kw)))
    assert 0 < size(max_rows=rows, grad=0) <= 8 * 131072
    assert size(max_rows=65, grad=0) > 2 * 10 ** 8 < size(max_rows=rows, grad=1)


@pytest.mark.parametrize("dtype", [0, 1])
def test_softmax_workspace_never_shrinks_with_rows(dtype):
    """A call of fewer rows than planned needs no more, a loss no more than a gradient."""
    for dim in (4, 32, 128, 260, 384, 388, 512, 772, 1024):
        for classes in (1, 50_021, 3_000_000):
            last = {0: 0, 1: 0}
            for rows in (1, 16, 17, 32, 33, 64, 65, 4096, 131072, 200_000):
                for grad in (0, 1):
                    now = P.load().huge_softmax_workspace_bytes(ctypes.byref(
                        _soft(num_classes=classes, dim=dim, dtype=dtype, max_rows=rows, grad=grad)))
                    assert now >= last[grad]
                    last[grad] = now
                assert last[0] <= last[1]
