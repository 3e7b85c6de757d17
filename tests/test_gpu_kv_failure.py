"""Failure detection of the many-row attention without a fault: a wait that runs out is reported, not hung, and leaves nothing behind.

lacache_kv_inject_stall makes the block that holds the first keys withhold its loads, so that its bounded waits for them run
out (about a second). The block records the timeout, stops its roles and still arrives at the counters of the triples that it shares
with other blocks: a later call, even one before the next sync, is not affected."""
import pytest
import torch

from kv_cases import Filled, TORCH
from paper_2608_01718_gb300 import build
from paper_2608_01718_gb300 import lacache as L

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    build.build()
    L.load()


# one sequence, which half of the blocks share a head of; several, shared by few
@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("lengths", [[20_000], [9_000, 300, 0, 20_000, 2_000]])
def test_a_wait_that_runs_out_is_reported_and_later_calls_are_right(fmt, dtype, lengths):
    new, group = 9, 4
    c = Filled(fmt, lengths, 2, 128, seed=30)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(31)
    first, second = (torch.randn(len(lengths) * new, 2 * group, 128, generator=gen, device="cuda").to(TORCH[dtype]) for _ in range(2))
    want = [c.kv.attend(q, c.table, c.len_dev, new_tokens=new) for q in (first, second)]
    few = c.kv.attend(first[: len(lengths)], c.table, c.len_dev)
    c.kv.sync()
    L.lacache_kv_inject_stall(c.kv.h, 1)
    c.kv.attend(first, c.table, c.len_dev, new_tokens=new)
    after = c.kv.attend(second, c.table, c.len_dev, new_tokens=new)       # before the sync
    few_after = c.kv.attend(first[: len(lengths)], c.table, c.len_dev)    # the few-row kernel uses the same counters
    with pytest.raises(L.LacacheError) as e:
        c.kv.sync()
    assert e.value.status == L.LACACHE_ERR_DEVICE_TIMEOUT
    assert torch.equal(after, want[1]) and torch.equal(few_after, few)
    c.kv.sync()                                                           # reported once
    assert torch.equal(c.kv.attend(first, c.table, c.len_dev, new_tokens=new), want[0])
    c.kv.sync()


def test_refusals():
    c = Filled("bf16", [20], 1, 64, seed=32)
    for h, n in ((None, 1), (c.kv.h, -1)):
        with pytest.raises(L.LacacheError) as e:
            L.lacache_kv_inject_stall(h, n)
        assert e.value.status == L.LACACHE_ERR_INVALID_ARG
    L.lacache_kv_inject_stall(c.kv.h, 1)
    L.lacache_kv_inject_stall(c.kv.h, 0)                                  # taken back
    c.kv.attend(torch.randn(20, 1, 64, device="cuda").bfloat16(), c.table, c.len_dev, new_tokens=20)
    c.kv.sync()
