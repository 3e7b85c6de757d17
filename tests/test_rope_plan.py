"""The rotation's plan (host only): phases as fractions of 2^64, and the refusals of lacache_rope_init."""
import math

import numpy as np
import pytest

from oracle import decode
from paper_2608_01718_gb300 import build
from paper_2608_01718_gb300 import lacache as L


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build()


@pytest.mark.parametrize("kw", [dict(), dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0),
                                dict(scaling="banded", factor=8.0, original_len=8192.0), dict(base=1e6),
                                dict(scaling="linear", factor=0.01)])
def test_phases(kw):
    plan = L.Rope(96, **kw).plan
    got = np.array([plan.turn[i] / 2.0 ** 64 for i in range(48)])
    want = decode.rope_frequencies(96, **kw) / (2 * math.pi)
    want = want - np.floor(want)
    assert np.all(np.abs(got - want) <= 2.0 ** -48 * np.maximum(1, want))
    assert all(plan.turn[i] == 0 for i in range(48, 128))
    assert plan.rot_dim == 96 and plan.layout == L.LACACHE_ROPE_HALF and plan.amplitude == 1.0


@pytest.mark.parametrize("args", [(0,), (3,), (258,), (-2,), (64, 2), (64, 0, 1.0), (64, 0, float("nan")), (64, 0, math.inf),
                                  (64, 0, 1e4, 4), (64, 0, 1e4, -1), (64, 0, 1e4, 1, 0.0), (64, 0, 1e4, 1, math.inf),
                                  (2, 0, 1e4, 2, 2.0), (64, 0, 1e4, 3, 2.0, 0.0), (64, 0, 1e4, 3, 2.0, 100.0, 4.0, 4.0),
                                  (64, 0, 1e4, 0, 1.0, 0.0, 1.0, 4.0, math.inf)])
def test_refused_plans(args):
    with pytest.raises(L.LacacheError) as e:
        L.lacache_rope_init(*args)
    assert e.value.status == L.LACACHE_ERR_INVALID_ARG


def test_refused_names():
    with pytest.raises(ValueError):
        L.Rope(64, scaling="other")
    with pytest.raises(ValueError):
        L.KVCache(1, 64, 4, format="fp4")


@pytest.mark.parametrize("field,value,status", [
    ("layers", 0, 1), ("kv_heads", 0, 1), ("head_dim", 0, 1), ("page_size", 0, 1), ("pages", 0, 1), ("pages", 1 << 31, 1),
    ("format", 4, 1), ("format", -1, 1), ("device", -1, 1), ("head_dim", 72, 6), ("head_dim", 272, 6), ("page_size", 24, 6),
    ("kv_heads", 1 << 16, 6), ("pages", (1 << 31) - 1, 3)])
def test_refused_caches(field, value, status):
    # before any device is touched; the last would hold more than 2^46 bytes
    cfg = L.lacache_kv_config(64, 64, 128, 64, 4, 0, 0)
    setattr(cfg, field, value)
    with pytest.raises(L.LacacheError) as e:
        L.lacache_kv_create(cfg)
    assert e.value.status == status
    assert L.load().lacache_kv_destroy(None) == L.LACACHE_OK
    assert L.load().lacache_kv_sync(None) == L.LACACHE_ERR_INVALID_ARG
