"""ocs_cache_read refuses outputs in which two vectors would lie on each other, and takes every nesting of tokens and heads (no
GPU needed: nothing is launched)."""
import ctypes

import pytest
import torch

import paper_1901_09504_b200 as ocs
from paper_1901_09504_b200.binding import _CacheDesc

INVALID, SHAPE = 1, 2
P = 1 << 20            # a well-aligned address that is never dereferenced
HEADS, DIM, ROWS = 3, 32, 5


def read(ld, heads=HEADS, rows=ROWS, Y2=None, ld2=None, dim=DIM, y_type=0):
    d = _CacheDesc(4, 8, heads, dim, ocs.MX4_E4M3)
    return ocs.lib().ocs_cache_read(ctypes.byref(d), P, P if Y2 else None, P, 4, 4, P, 2, rows, P, *ld, Y2, *(ld2 or ld), y_type, None, None)


def taken(status):
    """What follows the checks of the arguments: a launch, which this test leaves to machines without a GPU."""
    return status in (4, 5)


@pytest.mark.parametrize("ld,heads,rows,ok", [
    ((32, 32), 3, 5, False), ((32, 32), 2, 2, False), ((64, 32), 3, 5, False), ((95, 32), 3, 5, False), ((96, 32), 3, 5, True),
    ((32, 159), 3, 5, False), ((32, 160), 3, 5, True), ((48, 48), 3, 5, False), ((200, 64), 3, 5, True), ((40, 192), 3, 5, True),
    ((40, 191), 3, 5, False), ((32, 32), 1, 5, True), ((32, 0), 1, 5, True), ((0, 32), 3, 1, True), ((31, 32), 1, 5, False),
    ((0, 31), 3, 1, False), ((0, 0), 1, 1, True), ((-96, 32), 3, 5, False), ((96, -32), 3, 5, False),
    ((2 ** 62, 2 ** 62), 3, 5, False), ((2 ** 62, 32), 3, 5, True), ((32, 2 ** 62), 3, 5, True), ((2 ** 62, 2 ** 61), 3, 5, False),
])
def test_vectors_of_one_output(ld, heads, rows, ok):
    if ok and torch.cuda.is_available():
        pytest.skip("would launch")
    got = read(ld, heads, rows)
    assert taken(got) if ok else got == SHAPE


def lies_on(ld, ld2, d, heads, rows, dim):
    at = {t * ld[0] + h * ld[1] + e for t in range(rows) for h in range(heads) for e in range(dim)}
    return any(d + t * ld2[0] + h * ld2[1] + e in at for t in range(rows) for h in range(heads) for e in range(dim))


@pytest.mark.parametrize("ld", [(12, 4), (19, 4), (19, 5), (4, 20), (5, 26), (24, 8), (31, 9)])
@pytest.mark.parametrize("heads,rows", [(3, 5), (1, 5), (3, 1), (1, 1), (2, 2)])
def test_two_outputs_of_the_same_strides(ld, heads, rows):
    """Every distance between them, against the set of elements: next to each other, between each other's vectors, on them."""
    if torch.cuda.is_available():
        pytest.skip("would launch")
    for d in range(-150, 151):
        got = read(ld, heads, rows, Y2=P + 4 * d, dim=4)
        want = INVALID if d == 0 else (SHAPE if lies_on(ld, ld, d, heads, rows, 4) else None)
        assert taken(got) if want is None else got == want, (d, got, want)


def test_the_same_output_twice():
    assert read((96, 32), Y2=P) == INVALID
    assert read((96, 32), Y2=P, ld2=(32, 160)) == INVALID
    assert read((64, 32), Y2=P + 4096, ld2=(96, 32)) == SHAPE          # the second one's own vectors are fine, the first one's are not
    assert read((96, 32), Y2=P + 4096, ld2=(64, 32)) == SHAPE
    assert read((96, 32), Y2=P + 2 * 32, y_type=1) == SHAPE             # 16-bit elements: a vector further
