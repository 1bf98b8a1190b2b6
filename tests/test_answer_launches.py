"""The launches of what normalises, answers and clips, at sizes that take minutes or most
of the card: as in test_head_launches, with a stand-in for the HIP runtime.  No GPU."""
import ctypes
import os
import shutil
import subprocess

import pytest

import paper_2307_14490_amd as P
from paper_2307_14490_amd import binding as B
from paper_2307_14490_amd import build as b
from test_head_launches import CARD, HERE, PTR, blocks, launches

OBJECTS = ("api_head.hip", "k_norm.hip", "k_softmax.hip", "k_adamw.hip", "api_answer.hip",
           "k_rms.hip", "k_answer.hip", "k_clip.hip")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    objs = [os.path.join(b.BUILD, s + ".o") for s in OBJECTS]
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


KINDS = {"f32": (0, 0), "bf16": (1, 1), "q8": (1, 2)}


def answers(L, n, classes, dim, kind, top, bias=PTR, labels=PTR):
    dtype, table = KINDS[kind]
    cfg = B.HugeLogProbsConfig(classes, n, dim, dtype, table, top, 0)
    ws = L.huge_log_probs_workspace_bytes(ctypes.byref(cfg))
    size = 2 if dtype else 4
    assert 0 < ws and ws + n * dim * size + classes * dim * (1 if kind == "q8" else size) < CARD
    scales = PTR if kind == "q8" else None
    found = PTR if top else None
    return launches(L, L.huge_log_probs, ctypes.byref(cfg), PTR, dim, n, PTR, dim, scales,
                    -(-dim // 32), bias, labels, PTR if labels else None, PTR, PTR, found, found,
                    PTR, PTR, ws, None)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("n", [1, 64, 65, 4095, 4096, 32768, 2 ** 28 - 1, 2 ** 28, 2 ** 29 + 77])
def test_answers_of_many_rows(lib, n, kind):
    found = answers(lib, n, 5, 4, kind, 0)
    if n >= 32768:
        assert blocks(found, "k_lp_rows") * 32 >= n
    assert not blocks(found, "k_lp_select") and not blocks(found, "k_lp_top")


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("n,classes,dim,top", [
    (1, 1, 4, 1), (64, 10, 4, 10), (65, 33, 4, 33), (2 ** 22 + 5, 5, 4, 5), (2 ** 24 + 9, 64, 4, 64),
    (100, 2 ** 31 - 1, 4, 64), (48, 2 ** 31 - 1, 8, 1), (4096, 3_000_000, 128, 10),
    (70_000, 2_000_000, 64, 7), (16, 100_000_000, 128, 10), (9000, 20_000_000, 1024, 64)])
def test_best_classes_of_many_rows_and_classes(lib, n, classes, dim, top, kind):
    found = answers(lib, n, classes, dim, kind, top)
    assert blocks(found, "k_lp_top") == n  # a workgroup a row
    tiles = -(-classes // (16 if blocks(found, "k_sm_few") else 32))
    pieces = sum("k_lp_select" in f[0] for f in found)
    assert sum("k_lp_merge" in f[0] for f in found) in (0, pieces)
    assert pieces >= tiles * n // 2 ** 28
    for name, _, threads, lds in found:
        assert lds <= 160 * 1024 and threads <= 1024, name


def rms(L, n, dim, dtype, eight=False, grad=False):
    if grad:
        ws = L.huge_rms_norm_workspace_bytes(n, dim)
        return launches(L, L.huge_rms_norm_backward, PTR, dim, PTR, dim, PTR, dim, n, dim, dtype,
                        PTR, PTR, PTR, dim, PTR, PTR, ws, None)
    y = (None, 0, PTR, dim, PTR, -(-dim // 32)) if eight else (PTR, dim, None, 0, None, 0)
    return launches(L, L.huge_rms_norm, PTR, dim, PTR, dim, n, dim, dtype, PTR, 1e-5, PTR, dim, *y,
                    PTR, None)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("n,dim", [(1, 1), (2 ** 31 - 1, 1), (2 ** 31 - 1, 8), (2 ** 24, 8192),
                                   (2 ** 20, 2052), (2 ** 28, 96)])
def test_norms_of_many_rows(lib, n, dim, dtype):
    assert rms(lib, n, dim, dtype) and rms(lib, n, dim, dtype, eight=True)
    assert rms(lib, n, dim, dtype, grad=True)
    assert launches(lib, lib.huge_quantise_rows, PTR, dim, n, dim, dtype, PTR, dim, PTR,
                    -(-dim // 32), None)
    assert launches(lib, lib.huge_dequantise_rows, PTR, dim, PTR, -(-dim // 32), n, dim, PTR, dim,
                    dtype, None)


def tensors(*sizes):
    out = (B.HugeGradTensor * len(sizes))()
    for k, (t, n) in enumerate(zip(out, sizes)):
        t.d_grad, t.n, t.dtype = PTR, n, k % 2
    return out


@pytest.mark.parametrize("sizes", [(1,), (0, 0), (2 ** 40,) * 3, (5,) * 149, (5,) * 150, (5,) * 151,
                                   (2 ** 40,) * 70, (0, 7) * 200, (2 ** 33, 1, 0, 2 ** 36)])
def test_norms_of_many_and_of_large_tensors(lib, sizes):
    ts, count = tensors(*sizes), len(sizes)
    ws = lib.huge_grad_norm_workspace_bytes(count)
    found = launches(lib, lib.huge_grad_norm, ts, count, PTR, PTR, ws, None)
    # each launch leaves a partial sum per workgroup behind the factor
    assert 16 + 8 * blocks(found, "k_squares") <= ws
    assert blocks(found, "k_norm_factor") + blocks(found, "k_norm_small") == 1
    clipped = launches(lib, lib.huge_clip_grads, ts, count, 1.0, PTR, PTR, ws, None)
    assert clipped[:len(found)] == found
    assert (blocks(clipped, "k_scale") > 0) == (sum(sizes) > 0)
