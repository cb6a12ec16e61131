"""Host-side behaviour of the layer operators at the ends of their ranges (CPU)."""
import pytest

from paper_2607_25234_gb300 import build as libbuild
from paper_2607_25234_gb300 import whtmix


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return whtmix.library()


def test_nothing_is_asked_of_an_empty_batch(lib):
    """The gradient of no rows has no address: with dx alone there is nothing to do, with rows there is nothing to write to."""
    def call(T, act=0, dtype=1):
        return lib.whtmix_linear_backward(None, None, None, None, None, None, None, T, 8, 16, 16, 16, 8, 8, 16, act, dtype, None)
    assert call(0) == 0 and call(0, act=2) == 0
    assert call(4) == 1
    assert call(0, act=9) == 1 and call(0, dtype=3) == 3 and call(-1) == 1
