"""Limits of the batched serving entry points, checked on the host: no GPU is
needed, and the pointers used here are never dereferenced.  And the oracle of
sampling at the limit of its uniform numbers."""
import numpy as np
import pytest

from oracle import serving as OS
from paper_2605_08755_amd import laq
from test_serving_abi import append


@pytest.fixture(scope="module")
def L():
    return laq.lib()


@pytest.mark.parametrize("below", [1, 2, 3])
def test_append_of_2_32_threads_is_refused(L, below):
    """Four rows a block of 256 threads: the last block of 2^26 - 3 rows makes
    it 2^32 threads, more than one launch may have."""
    assert append(L, Hq=1, Hkv=1, stride=3 * 128, T=(1 << 26) - below) == laq.LAQ_ERR_BAD_SHAPE
    assert b"too many rows" in L.laq_last_error()


def test_oracle_sample_at_one():
    """From u = 1 on the last token kept, also where the running sum of the
    weights before it is rounded above their exact sum."""
    rng = np.random.default_rng(5)
    for _ in range(200):
        x = (5 * rng.standard_normal(64)).astype(np.float16)
        last = max(range(64), key=lambda i: (-x[i], i))
        for u in (1.0, 7.0):
            assert OS.sample_row(x, u, temperature=0.08)[0] == last
