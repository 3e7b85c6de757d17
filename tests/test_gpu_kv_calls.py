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
