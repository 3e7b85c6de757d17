"""Pins of the gathered attention weights and the eviction by them, and what their calls refuse (no GPU)."""
import ctypes

import numpy as np
import pytest

from oracle import decode
from paper_2608_01718_gb300 import build
from paper_2608_01718_gb300 import lacache as L


def test_shares_of_a_query_add_up_to_one():
    rng = np.random.default_rng(0)
    lengths, T = [9, 0, 3, 1], 2
    k = [rng.normal(size=(n, 2, 8)) for n in lengths]
    q = rng.normal(size=(8, 4, 8))
    _, lse, _, _ = decode.attend(q, k, k, lengths, T, 0.5)
    got = decode.weigh(q, k, lengths, T, 0.5, lse)
    for (w, _, _), n in zip(got, lengths):
        # two queries a kv head, T positions of which the last min(T, n) are there
        assert np.allclose(w.sum(1), 2 * min(T, n))
    assert got[0][0].shape == (2, 9)


def test_the_past_fades_and_new_tokens_start_from_nothing():
    k = [np.zeros((4, 1, 8))]
    q, lse = np.zeros((2, 1, 8)), np.log([[3.0], [4.0]])
    (w, _, _), = decode.weigh(q, k, [4], 2, 1.0, lse, past=[np.array([[10.0, 20.0, 99.0, 99.0]])], decay=0.5)
    assert np.allclose(w, [[5 + 1 / 3 + 1 / 4, 10 + 1 / 3 + 1 / 4, 1 / 3 + 1 / 4, 1 / 4]])


def test_kept_positions():
    w = [np.array([[1.0, 5.0, 5.0, 0.0, 5.0, 2.0, 0.0]])]
    assert decode.evict(w, [7], 3, 1) == [[[1, 2, 6]]]                    # of equal weights the earlier
    assert decode.evict(w, [7], 3, 3) == [[[4, 5, 6]]]
    assert decode.evict(w, [7], 3, 0, [2]) == [[[2, 4, 5]]]
    assert decode.evict(w, [7], 9, 0, [5]) == [[[5, 6]]]
    assert decode.evict(w, [0], 3, 1) == [[[]]]
    nan = [np.array([[np.nan, -np.inf, -0.0, 0.0, np.inf]])]
    assert decode.evict(nan, [5], 2, 0) == [[[2, 4]]] and decode.evict(nan, [5], 4, 0) == [[[1, 2, 3, 4]]]


def test_refusals_need_no_device():
    build.build()
    lib, ref = L.load(), ctypes.addressof
    table = L.lacache_kv_table(256, 4, 1, 4)
    w = L.lacache_weights(256, 64, 64, 64)
    assert lib.lacache_kv_weigh(None, 0, ref(table), ref(L.lacache_weighing()), None) == L.LACACHE_ERR_INVALID_ARG
    assert lib.lacache_kv_weigh(None, 0, ref(table), None, None) == L.LACACHE_ERR_INVALID_ARG
    assert lib.lacache_kv_evict(None, 0, ref(table), 256, None, ref(w), 4, 0, ref(table), 256, 256, None, None) == \
        L.LACACHE_ERR_INVALID_ARG
    assert ctypes.sizeof(L.lacache_weights) == 32 and ctypes.sizeof(L.lacache_weighing) == 136


@pytest.mark.parametrize("field", ["data_dev", "seq_stride", "head_stride", "width"])
def test_struct_fields(field):
    assert [f for f, _ in L.lacache_weights._fields_][["data_dev", "seq_stride", "head_stride", "width"].index(field)] == field
