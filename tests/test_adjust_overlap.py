"""laq_adjust_logits_f16 refuses logits and out that share some elements, and
only those.  Checked on the host before any HIP call: the sizes here are all too
many for one launch, which is asked after the overlap, so that an answer names
which of the two it was and no GPU is needed."""
import numpy as np
import pytest

from paper_2605_08755_amd import laq
from test_serving8_abi import adjust

V, ROWS = 1 << 24, 4200


@pytest.fixture(scope="module")
def L():
    return laq.lib()


def shares(L, offset, stride, out_stride, rows=ROWS, v=V):
    """What the library says of out `offset` elements from the logits."""
    at = 1 << 50
    assert adjust(L, logits=at, out=at + 2 * offset, stride=stride, out_stride=out_stride, rows=rows, V=v) == laq.LAQ_ERR_BAD_SHAPE
    said = L.laq_last_error()
    assert (b"out must be" in said) != (b"too many" in said), said
    return b"out must be" in said


def want(offset, stride, out_stride, rows=ROWS, v=V):
    """Rows are [i stride, + v): each against the row of out that begins last before its end."""
    i = np.arange(rows, dtype=np.int64) * stride
    j = offset + np.arange(rows, dtype=np.int64) * out_stride
    k = np.searchsorted(j, i + v, side="left") - 1  # the last of out's that begins before the row's end
    return bool(((k >= 0) & (j[np.maximum(k, 0)] + v > i)).any())


def test_columns_of_one_array(L):
    """The two halves of rows of 2 V and more, either first; one element over the border."""
    for stride in (2 * V, 2 * V + 13):
        for offset, over in ((V, False), (-V, False), (V - 1, True), (1 - V, True), (stride - V, False),
                             (stride - V + 1, True), (5 * stride + V, False), (5 * stride + V - 1, True), (0, False)):
            if offset == 0:  # in place
                assert not shares(L, 0, stride, stride)
            else:
                assert shares(L, offset, stride, stride) == over == want(offset, stride, stride), (stride, offset)
    # rows one after another: out before, behind, and by one row over it
    for offset, over in ((ROWS * V, False), (-ROWS * V, False), (V, True), (-V, True), (ROWS * V - 1, True), (1, True)):
        assert shares(L, offset, V, V) == over == want(offset, V, V), offset


def test_strides_that_differ(L):
    rng = np.random.default_rng(0)
    seen = set()
    cases = [(V, 4 * V, 2 * V), (V, 2 * V, 4 * V), (0, 2 * V, 2 * V + 1), (V, 2 * V, 2 * V + 1),
             (V, V + V // 2, 3 * V), ((ROWS - 1) * V + V, V, 2 * V), ((ROWS - 1) * V + V - 1, V, 2 * V)]
    for _ in range(200):
        s, o = (int(x) for x in rng.integers(V, 6 * V, 2))
        if rng.random() < 0.5:
            o = s * int(rng.integers(1, 4))
        cases.append((int(rng.integers(-3 * ROWS * V, 3 * ROWS * V)) if rng.random() < 0.7 else int(rng.integers(-4 * V, 4 * V)), s, o))
    for c in cases:
        got = shares(L, *c)
        assert got == want(*c), c
        seen.add(got)
    assert seen == {True, False}


def test_most_rows(L):
    """The most rows that a call takes: a step a row."""
    rows = (1 << 22) - 1
    assert not shares(L, V, 2 * V, 2 * V, rows)
    assert shares(L, V - 1, 2 * V, 2 * V, rows)
    assert not shares(L, V, 2 * V, 4 * V, rows)
