"""Shared prefixes whose later keys outscore the earlier ones by more than a power of two that fp32 holds: the common part's kernel
for many rows keeps a reference that it moves after the keys that ask for it."""
import pytest
import torch

from test_gpu_kv_shared import check, filled, ints, library  # noqa: F401 (the fixture)
from kv_cases import TORCH

pytestmark = pytest.mark.gpu

FORMATS = [("bf16", "bf16"), ("e4m3", "bf16"), ("int8", "f16"), ("f16", "f16")]


def along(c, dtype, q_heads, new, seed):
    """A direction per kv head, and queries near it."""
    D, H, n = c.kv.cfg.head_dim, c.kv.cfg.kv_heads, len(c.lengths) * new
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    base = torch.randn(H, D, generator=gen, device="cuda")
    q = base.repeat_interleave(q_heads // H, 0) + torch.randn(n, q_heads, D, generator=gen, device="cuda") / 32
    return base, q.to(TORCH[dtype])


def raise_keys(c, dtype, base, group, at, powers):
    """Keys at common positions `at` of a group whose scores with the queries are near powers[i], in powers of two; their values are 1
    to len(at), so that whose they are shows."""
    D, first = c.kv.cfg.head_dim, c.bounds[group]
    a = torch.tensor(powers, device="cuda") * 0.6931471805599453 * D ** 0.5
    k = (base[None] / base.square().sum(-1)[None, :, None] * a[:, None, None]).to(TORCH[dtype])
    v = torch.arange(1, len(at) + 1, device="cuda").view(-1, 1, 1).expand(k.shape).to(TORCH[dtype]).contiguous()
    seq, page = ints([first] * len(at)), c.page
    full = c.common[group] // page * page
    assert all(p < full for p in at)                         # in pages that the sequences share
    c.kv.append(k, v, seq, ints(at), c.table, layer=c.layer)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("power", [14, 60, 99, 101, 119, 122, 130, 300])
@pytest.mark.parametrize("at", [[128], [300], [640], [127, 128, 500], [5, 260, 650]])
def test_scores_that_rise_within_a_block(fmt, dtype, power, at):
    """Eighty pairs of a group and a kv head: most lie within one block's keys whole, the others are cut."""
    groups = [(672 + i % 3, [680 + (i * 7 + s) % 40 for s in range(3)]) for i in range(20)]
    c = filled(fmt, groups, 4, 64, seed=21)
    base, q = along(c, dtype, 32, 1, 22)
    for g in range(len(groups)):
        raise_keys(c, dtype, base, g, at, [power * (i + 1) / len(at) for i in range(len(at))])
    check(c, dtype, 32, q=q)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("power", [100, 125, 250])
def test_scores_that_rise_over_many_blocks(fmt, dtype, head_dim, power):
    """One group, its 157 units over all blocks; the keys before the rise weigh nothing after it."""
    c = filled(fmt, [(20_001, [20_010 + s for s in range(6)])], 1, head_dim, seed=23)
    base, q = along(c, dtype, 4, 5, 24)
    raise_keys(c, dtype, base, 0, [200, 9000, 9130, 19_900], [power / 2, power / 2 + 3, power, power - 1])
    check(c, dtype, 4, 5, q=q)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("window", [0, 500])
def test_low_scores_first(fmt, dtype, window):
    """The first two units score 200 powers of two below all others, which are of plain size (window: its first unit is half of one
    and half of the other)."""
    groups = [(672 + i % 3, [680 + (i * 7 + s) % 40 for s in range(3)]) for i in range(20)]
    c = filled(fmt, groups, 4, 64, seed=25)
    base, q = along(c, dtype, 32, 1, 26)
    for g in range(len(groups)):
        raise_keys(c, dtype, base, g, list(range(256)), [-200.0] * 256)
    check(c, dtype, 32, q=q, window=window)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
def test_a_score_that_is_infinite(fmt, dtype):
    """In the last unit of three: the rows that see it are NaN, as the ordinary attention's, the others what they were."""
    c = filled(fmt, [(384, [386 + s for s in range(20)])], 1, 64, seed=27)
    base, q = along(c, dtype, 2, 1, 28)
    raise_keys(c, dtype, base, 0, [370], [1.0])
    starts = ints([0, 380] * 10)
    kw = dict(starts=starts)
    clean = c.kv.attend_shared(q, c.table, c.len_dev, ints(c.common), **kw)
    pool = c.kv.pool()
    page, slot = int(c.host_table[0, 370 // c.page]), 370 % c.page
    if "ks" in pool:
        pool["ks"][page, :, slot] = float("inf")
    else:
        most = int(base[0].abs().argmax())                   # (where every query has the same sign)
        pool["k"][page, :, slot, most] = float("inf") * float(base[0, most].sign())
    got = c.kv.attend_shared(q, c.table, c.len_dev, ints(c.common), **kw)
    want = c.kv.attend(q, c.table, c.len_dev, **kw)
    c.kv.sync()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and bool(torch.isnan(got[::2]).all())
    assert torch.allclose(got[1::2].float(), clean[1::2].float(), rtol=2.0 ** -7, atol=2.0 ** -9)
