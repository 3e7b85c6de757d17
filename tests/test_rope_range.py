"""Arguments of the rotation at the ends of their ranges (host only)."""
import pytest

from paper_2608_01718_gb300 import build
from paper_2608_01718_gb300 import lacache as L


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build()


@pytest.mark.parametrize("args", [(64, 0, 1e4, L.LACACHE_ROPE_LINEAR, 1e-310),
                                  (64, 0, 1e4, L.LACACHE_ROPE_BANDED, 1e-310, 1.0, 1.0, 4.0),
                                  (64, 0, 1e4, L.LACACHE_ROPE_BANDED, 8.0, 1e308, -1e308, 1e308),
                                  (64, 0, 1e4, L.LACACHE_ROPE_BASE, 1e-320)])
def test_frequencies_that_are_not_finite_are_refused(args):
    with pytest.raises(L.LacacheError) as e:
        L.lacache_rope_init(*args)
    assert e.value.status == L.LACACHE_ERR_INVALID_ARG


@pytest.mark.parametrize("args", [(64, 0, 1e4, L.LACACHE_ROPE_LINEAR, 1e-30), (64, 0, 1e4, L.LACACHE_ROPE_LINEAR, 1e300),
                                  (64, 0, 1e4, L.LACACHE_ROPE_BASE, 1e-3), (2, 0, 1e300), (256, 0, 1.0 + 2.0 ** -50)])
def test_extreme_frequencies_are_taken(args):
    plan = L.lacache_rope_init(*args)
    assert plan.rot_dim == args[0]
