"""Limits of the batched serving entry points, checked on the host: no GPU is
needed, and the pointers used here are never dereferenced."""
import pytest

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
