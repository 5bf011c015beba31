"""More of the serving calls' checks on the host: calls that are in order are not refused, nothing here runs on a GPU (each call ends
at a later refusal)."""
import ctypes

import pytest

GOOD, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1001)       # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    from paper_2410_02367_amd import binding
    return binding.load()


def test_an_eviction_into_another_pool_may_have_the_same_table(lib):
    other = ctypes.c_void_p(0x2000)

    def call(out_cache, out_pages, kept):
        return lib.sage_cache4_evict(GOOD, 8, GOOD, 4, GOOD, GOOD, 64, out_cache, 8, out_pages, 4, other, 32, kept, other, 1, 1, 64, 16, 32, 20, 4, None)
    assert call(GOOD, GOOD, GOOD) == 7                      # in place
    assert call(GOOD, other, ODD) == 5 and call(other, other, ODD) == 5
    assert call(other, GOOD, ODD) == 5                      # past the check of values, up to that of alignment
