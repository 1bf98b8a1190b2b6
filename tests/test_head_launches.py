"""The launches of the softmax head's calls at sizes that take minutes or most of the
card: the host layer and the kernels' objects are linked with a stand-in for the HIP
runtime that writes launches down (launches/record.cpp).  No GPU."""
import ctypes
import os
import shutil
import subprocess

import pytest

import paper_2307_14490_amd as P
from paper_2307_14490_amd import binding as B
from paper_2307_14490_amd import build as b

HERE = os.path.dirname(os.path.abspath(__file__))
PTR = 1 << 20
CARD = 288 * 10 ** 9  # bytes


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    objs = [os.path.join(b.BUILD, s + ".o")
            for s in ("api_head.hip", "k_norm.hip", "k_softmax.hip", "k_adamw.hip")]
    newest = max(os.path.getmtime(os.path.join(b.CSRC, f)) for f in os.listdir(b.CSRC))
    if not all(os.path.exists(o) and os.path.getmtime(o) >= newest for o in objs):
        b.build()
    out = str(tmp_path_factory.mktemp("launches") / "librecord.so")
    r = subprocess.run(["g++", "-shared", "-fPIC", "-O1", "-std=c++17", "-Wl,-Bsymbolic",
                        os.path.join(HERE, "launches", "record.cpp"), *objs, "-o", out],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    real, L = P.load(), ctypes.CDLL(out)
    for name in B.EXPORTED:
        if hasattr(L, name):
            fn = getattr(L, name)
            fn.argtypes, fn.restype = getattr(real, name).argtypes, getattr(real, name).restype
    L.record_launch.restype = ctypes.c_char_p
    L.record_launch.argtypes = [ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p]
    return L


def launches(L, call, *args):
    """(kernel, workgroups, threads of one, bytes of LDS) of each launch of a call."""
    L.record_clear()
    assert call(*args) == B.HUGE_OK
    out = []
    for k in range(L.record_count()):
        dims, lds = (ctypes.c_uint32 * 6)(), ctypes.c_uint64()
        name = L.record_launch(k, dims, ctypes.byref(lds)).decode()
        for d in range(3):  # a launch has fewer than 2^32 threads in a direction
            assert 0 < dims[d] and 0 < dims[d] * dims[3 + d] < 2 ** 32, (name, list(dims))
        out.append((name, dims[0], dims[3], lds.value))
    return out


def softmax(L, n, classes, dim, dtype, grad, want=(True, True, True), bias=PTR):
    """Launches of a loss, or of a gradient, whose arrays fit the card."""
    cfg = B.HugeSoftmaxConfig(classes, n, dim, dtype, int(grad))
    ws = L.huge_softmax_workspace_bytes(ctypes.byref(cfg))
    size = 2 if dtype == B.HUGE_DTYPE_BF16 else 4
    rows = (n + classes) * dim * size * (2 if grad else 1)
    assert 0 < ws and ws + rows + 12 * n < CARD
    a = (ctypes.byref(cfg), PTR, dim, n, PTR, dim, bias, PTR, None)
    if not grad:
        return launches(L, L.huge_softmax_loss, *a, PTR, PTR, PTR, PTR, PTR, ws, None)
    out = [PTR if w else None for w in want]
    return launches(L, L.huge_softmax_grad, *a, PTR, 1.0, *out, PTR, PTR, ws, None)


def blocks(found, kernel):
    return sum(grid for name, grid, _, _ in found if kernel in name)


@pytest.mark.parametrize("dtype", [B.HUGE_DTYPE_F32, B.HUGE_DTYPE_BF16])
@pytest.mark.parametrize("n", [1, 64, 65, 4095, 4096, 2 ** 28 - 1, 2 ** 28, 2 ** 29 + 77])
def test_losses_of_many_rows(lib, n, dtype):
    found = softmax(lib, n, 5, 4, dtype, grad=False)
    assert blocks(found, "k_sm_loss") * 256 >= n * (64 if n < 4096 else 16)
    if n > 64:
        assert blocks(found, "k_sm_pack") == -(-n // 32) + 1


@pytest.mark.parametrize("n", [100, 2 ** 28, 2 ** 29 + 77])
def test_gradients_of_many_rows(lib, n):
    found = softmax(lib, n, 5, 4, B.HUGE_DTYPE_BF16, grad=True)
    assert blocks(found, "k_sm_pack") == -(-n // 32) + 1
    assert blocks(found, "k_sm_grad") > 0


def test_joined_sums_of_many_wide_rows(lib):
    """The table is in pieces, so that every row's sums are joined."""
    n, classes, dim = 2 ** 24 + 9, 600_000, 1024
    found = softmax(lib, n, classes, dim, B.HUGE_DTYPE_BF16, grad=True, want=(True, False, False))
    assert blocks(found, "k_sm_join") * 256 >= n * (dim // 4)
