"""The decoding calls' arguments: what is refused, strides and numbers at the edges, streams and gradients."""
import pytest
import torch

from kv_cases import Filled
from paper_2608_01718_gb300 import build
from paper_2608_01718_gb300 import lacache as L

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    build.build()
    L.load()


def test_outputs_over_the_queries_are_refused():
    # the many-row kernel may read a row of q again after it has written that row of out
    c = Filled("bf16", [40], 1, 64, seed=33)
    for new in (1, 20):
        q = torch.randn(new, 1, 64, device="cuda").bfloat16()
        kept = q.clone()
        with pytest.raises(L.LacacheError) as e:
            c.kv.attend(q, c.table, c.len_dev, new_tokens=new, out=q)
        assert e.value.status == L.LACACHE_ERR_INVALID_ARG and torch.equal(q, kept)
    c.kv.sync()


def test_numbers_past_32_bits_are_refused_or_mean_what_they_say():
    # a window of 2^32 + 5 is no window of 5
    c = Filled("bf16", [40], 1, 64, seed=35)
    q = torch.randn(1, 1, 64, device="cuda").bfloat16()
    want = c.kv.attend(q, c.table, c.len_dev)
    for window in ((1 << 32) + 5, 1 << 31, 1 << 62):
        assert torch.equal(c.kv.attend(q, c.table, c.len_dev, window=window), want)
    for window in (-1, -(1 << 32) + 5):
        with pytest.raises((ValueError, L.LacacheError)):
            c.kv.attend(q, c.table, c.len_dev, window=window)
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    for layer in (1 << 32, -(1 << 32)):
        with pytest.raises((ValueError, L.LacacheError)):
            c.kv.attend(q, c.table, c.len_dev, layer=layer)
        with pytest.raises((ValueError, L.LacacheError)):
            c.kv.append(q, q, one, one, c.table, layer=layer)
        with pytest.raises((ValueError, L.LacacheError)):
            c.kv.read(one, one, c.table, layer=layer)
        with pytest.raises((ValueError, L.LacacheError)):
            c.kv.pool(layer)
    c.kv.sync()
