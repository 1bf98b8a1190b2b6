"""Workspace of the log probabilities: what the best classes add to it is bounded.  No GPU."""
import ctypes

import pytest

import paper_2307_14490_amd as P
from paper_2307_14490_amd import binding as B

KINDS = {"f32": (0, 0), "bf16": (1, 1), "q8": (1, 2)}


def bytes_of(classes, n, dim, kind, top):
    cfg = B.HugeLogProbsConfig(classes, n, dim, *KINDS[kind], top, 0)
    ws = P.load().huge_log_probs_workspace_bytes(ctypes.byref(cfg))
    assert ws > 0
    return ws


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("classes,n,dim,top", [
    (2208, 3_800_000, 32, 64), (1000, 4_000_000, 32, 20), (64, 2 ** 24, 4, 64), (33, 2 ** 26, 4, 1),
    (1_000_000, 4096, 128, 10), (1_000_000, 8192, 128, 64), (2 ** 31 - 1, 8192, 64, 64),
    (2 ** 31 - 1, 64, 8, 64), (100_000_000, 16, 128, 10), (10, 5, 4, 10)])
def test_what_the_best_classes_add(classes, n, dim, top, kind):
    """Tile maxima and lists take 1 GiB, lists of splits 8 bytes of each of 68 tiles of 32768
    rows; few rows have entries of more pieces."""
    lists = 8 * 32768 * 68
    more = bytes_of(classes, n, dim, kind, top) - bytes_of(classes, n, dim, kind, 0)
    parts = 0 if n > 64 else 16 * 2048 * 64 * -(-classes // (1 << 25))
    assert more <= (1 << 30) + lists + parts + 1024


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("top", [1, 20, 64])
@pytest.mark.parametrize("classes,dim", [(64, 4), (5000, 128), (1_100_000, 32), (40_000_000, 256)])
def test_fewer_rows_need_no_more(classes, dim, top, kind):
    sizes = [bytes_of(classes, n, dim, kind, top)
             for n in (1, 16, 17, 48, 64, 65, 4096, 8192, 8193, 100_000, 3_000_000, 2 ** 22 + 33)]
    assert sizes == sorted(sizes)
