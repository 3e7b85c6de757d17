"""Arguments of the rotation and of the cache's write at the ends of their ranges (host only)."""
import ctypes

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


def test_counts_of_heads_past_32_bits():
    # rows of a token are counted in 32 bits, with room for a pass
    lib, plan = L.load(), L.lacache_rope_init(64)
    rows = L.lacache_rows(1 << 20, 0, 0)
    ref = ctypes.addressof

    def rotate(heads):
        return lib.lacache_rope_apply(ref(plan), 0, heads, 64, L.LACACHE_BF16, ref(rows), 1 << 20, 0, ref(rows), None)

    for heads in ((1 << 31) - 1, (1 << 30) + 1):
        assert rotate(heads) == L.LACACHE_ERR_UNSUPPORTED
    assert rotate(1 << 30) == L.LACACHE_OK           # (no tokens: nothing is launched)
