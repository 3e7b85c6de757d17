"""Shared prefixes: what the rows of the table have to name."""
import pytest
import torch

from test_gpu_kv_shared import check, filled, ints, library, queries  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("e4m3", "f16")])
@pytest.mark.parametrize("head_dim,q_heads", [(64, 2), (64, 8), (256, 2)])
def test_sequences_that_see_nothing_ask_for_no_pages(fmt, dtype, head_dim, q_heads):
    """A batch padded with empty sequences, and one that is all before its start, behind a prefix whose first pages have left every
    sequence's window."""
    c = filled(fmt, [(700, [760, 0, 730, 745, 0, 710, 90, 701])], 2, head_dim, seed=31)
    starts = [0, 0, 0, 0, 0, 0, 90, 0]
    q = queries(c, dtype, q_heads, 1)
    kw = dict(starts=ints(starts), window=300)
    want, _ = check(c, dtype, q_heads, starts=starts, window=300)
    c.table[:, :(701 - 300) // c.page] = 1 << 29
    lse = torch.empty(q.shape[:2], device="cuda")
    got = c.kv.attend_shared(q, c.table, c.len_dev, ints(c.common), bounds=ints(c.bounds), lse=lse, **kw)
    c.kv.sync()
    assert torch.equal(got, want)
    assert bool(torch.isneginf(lse[ints([1, 4, 6]).long()]).all())


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("f16", "f16"), ("int8", "bf16")])
@pytest.mark.parametrize("head_dim,q_heads,new", [(64, 2, 1), (128, 8, 3), (64, 8, 9), (192, 4, 2)])
@pytest.mark.parametrize("length", [0, 1, 50, 399])
def test_a_first_sequence_that_ends_before_the_common_positions(fmt, dtype, head_dim, q_heads, new, length):
    """Its row of the table names their pages all the same."""
    c = filled(fmt, [(400, [420, 410, 401, 450]), (90, [100, 95])], 2, head_dim, seed=32)
    for s in (0, 4):
        c.lengths[s] = min(length, c.common[s // 4] - 1)
        c.len_dev[s] = c.lengths[s]
    check(c, dtype, q_heads, new)
    check(c, dtype, q_heads, new, window=100)


def test_no_workspace_for_arguments_outside_their_ranges():
    from paper_2608_01718_gb300 import lacache as L
    c = filled("bf16", [(20, [40, 30])], 2, 64, seed=33)
    t = c.kv._table(c.table)
    size = lambda groups=1, new=1, heads=4: L.lacache_kv_attend_shared_workspace_bytes(c.kv.h, t, groups, new, heads)
    assert size() > 0 and size(new=512) > 0 and size(heads=1 << 16) > 0
    for kw in (dict(new=513), dict(heads=3), dict(heads=(1 << 16) + 2), dict(heads=-2), dict(groups=-1)):
        assert size(**kw) == 0, kw
