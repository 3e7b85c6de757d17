"""Attention over the paged cache where groups of sequences have their first positions in common, against the fp64 oracle of whole
sequences."""
import numpy as np
import pytest
import torch

from kv_cases import Filled, TORCH, bounds as tolerances
from oracle import decode
from paper_2608_01718_gb300 import build
from paper_2608_01718_gb300 import lacache as L

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    build.build()
    L.load()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def filled(fmt, groups, kv_heads, head_dim, page=16, seed=0, alone=(), small=False, **kw):
    """groups: (common positions, [lengths of its sequences, whole]); `alone`: lengths of sequences of no group, after them. A table
    as wide as one that serves long sequences too (unless `small`), or the call would read each sequence for itself."""
    lengths = [n for _, ns in groups for n in ns] + list(alone)
    c = Filled(fmt, lengths, kv_heads, head_dim, page, seed=seed, **kw)
    c.bounds = np.cumsum([0] + [len(ns) for _, ns in groups]).tolist()
    c.common = [p for p, _ in groups]
    pool = c.kv.pool(c.layer)
    for g, (p, ns) in enumerate(groups):
        first = c.bounds[g]
        if not ns or lengths[first] < min(p, max(ns)):
            assert not ns, "the first sequence holds what is common"
            continue
        for s in range(first + 1, c.bounds[g + 1]):
            full, rest = min(p, lengths[s]) // page, min(p, lengths[s]) % page
            c.host_table[s, :full] = c.host_table[first, :full]
            if rest:      # the page that the common part ends in is the sequence's own, with a copy
                a, b = int(c.host_table[first, full]), int(c.host_table[s, full])
                for t in pool.values():
                    x = t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t
                    x[b, :, :rest] = x[a, :, :rest].clone()
    row = 2 * kv_heads * head_dim * (1 if fmt in ("e4m3", "int8") else 2)
    width = c.host_table.shape[1] if small else max(c.host_table.shape[1], 80_000_000 // (row * page * len(lengths)) + 1)
    wide = np.full((len(lengths), width), 1 << 29, dtype=np.int32)
    wide[:, :c.host_table.shape[1]] = c.host_table
    c.table = torch.from_numpy(wide).cuda()
    return c


def queries(c, dtype, q_heads, new, seed=1):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randn(len(c.lengths) * new, q_heads, c.kv.cfg.head_dim, generator=gen, device="cuda").to(TORCH[dtype])


def check(c, dtype, q_heads, new=1, window=0, starts=None, scale=None, seed=1, q=None, none_bounds=False):
    D, n = c.kv.cfg.head_dim, len(c.lengths) * new
    q = queries(c, dtype, q_heads, new, seed) if q is None else q
    out = torch.full((n, q_heads, D), float("nan"), dtype=TORCH[dtype], device="cuda")
    lse = torch.full((n, q_heads), float("nan"), device="cuda")
    st = None if starts is None else ints(starts)
    kw = dict(bounds=None if none_bounds else ints(c.bounds), new_tokens=new, layer=c.layer, starts=st, window=window, scale=scale)
    got = c.kv.attend_shared(q, c.table, c.len_dev, ints(c.common), out=out, lse=lse, **kw)
    c.kv.sync()
    assert got is out
    k, v = c.values()
    f = D ** -0.5 if scale is None else scale
    hq = q.double().cpu().numpy()
    want, want_lse, mass, span = decode.attend(hq, k, v, c.lengths, new, f, starts, window)
    tol, tol_lse = tolerances(want, mass, span, want_lse, hq, k, f, dtype)
    hg, hl = out.double().cpu().numpy(), lse.double().cpu().numpy()
    empty = np.isinf(want_lse)
    assert np.array_equal(np.isneginf(hl), empty) and np.all(hg[empty] == 0.0)
    assert np.all(np.abs(hg - want) <= tol), float(np.nanmax(np.abs(hg - want) / tol))
    assert np.all(np.abs(hl[~empty] - want_lse[~empty]) <= tol_lse[~empty])
    again = c.kv.attend_shared(q, c.table, c.len_dev, ints(c.common), **kw)
    assert torch.equal(again.view(torch.int16), out.view(torch.int16))        # the same bits every time
    return out, lse


FORMATS = [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16"), ("e4m3", "f16"), ("int8", "bf16"), ("int8", "f16")]
MIXED = [(300, [301, 417, 300, 299, 5, 0, 333]), (0, [40, 1]), (64, [65]), (17, []), (33, [50, 60, 70, 34])]


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("kv_heads,group,head_dim,page,new", [(2, 1, 64, 16, 1), (1, 4, 128, 32, 1), (3, 5, 80, 16, 3), (2, 2, 256, 48, 2),
                                                             (1, 7, 192, 16, 1), (2, 4, 128, 16, 17), (1, 2, 16, 16, 1), (1, 8, 96, 64, 5)])
def test_against_the_oracle(fmt, dtype, kv_heads, group, head_dim, page, new):
    c = filled(fmt, MIXED, kv_heads, head_dim, page, seed=head_dim + new, alone=[0, 77])
    check(c, dtype, kv_heads * group, new)


@pytest.mark.parametrize("fmt,dtype", FORMATS[:1] + FORMATS[2:3])
@pytest.mark.parametrize("kw", [dict(window=1), dict(window=40), dict(window=320), dict(scale=-0.25), dict(scale=0.0),
                                dict(starts=[0, 10, 299, 300, 4, 0, 320, 45, 0, 64, 1, 60, 3, 34]),
                                dict(starts=[5, 10, 17, 1, 4, 0, 30, 2, 0, 70, 1, 60, 3, 34], window=50)])
@pytest.mark.parametrize("head_dim,q_heads,new", [(64, 2, 1), (64, 8, 1), (64, 4, 9), (144, 4, 2)])
def test_masks(fmt, dtype, kw, head_dim, q_heads, new):
    c = filled(fmt, MIXED, 2, head_dim, seed=3)
    check(c, dtype, q_heads, new, **kw)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("head_dim", [64, 128, 256])
def test_one_group_of_all_and_many_rows(fmt, head_dim):
    """Rows of a kv head over several tiles of 128, in sequences that end all over them."""
    c = filled(fmt, [(700, [701 + (i * 37) % 90 for i in range(40)])], 1, head_dim, 32, seed=4)
    check(c, "bf16", 7, 1, none_bounds=True)


@pytest.mark.parametrize("fmt,dtype", FORMATS[:3])
def test_long_common_part_of_few_rows(fmt, dtype):
    """One triple over all blocks, and its joins."""
    for heads, new in ((1, 1), (4, 9)):
        c = filled(fmt, [(20_001, [20_040, 20_001 + new])], 1, 64, 16, seed=5)
        check(c, dtype, heads, new)


def test_groups_of_one_and_many_groups():
    c = filled("bf16", [(16 * (i % 5) + i % 3, [16 * (i % 5) + i % 3 + 1 + i % 20]) for i in range(150)], 1, 64, seed=6)
    check(c, "bf16", 2)
    c = filled("f16", [(200, [201])], 2, 64, seed=7)
    check(c, "f16", 4, none_bounds=True)


@pytest.mark.parametrize("fmt,head_dim", [("bf16", 80), ("e4m3", 64), ("f16", 128)])
def test_blocks_with_one_and_two_tiles_of_rows(fmt, head_dim):
    """Groups of 100 and of 140 rows a kv head in turn: a block has units of one tile of rows, then units of two."""
    groups = [(700 - i, [701 + (i * 7 + s) % 40 for s in range(5 if i % 2 else 7)]) for i in range(20)]
    c = filled(fmt, groups, 8, head_dim, seed=17)
    check(c, fmt if fmt == "f16" else "bf16", 32, 5)


@pytest.mark.parametrize("fmt,dtype", FORMATS[:3])
def test_rows_that_see_nothing_of_their_first_units(fmt, dtype):
    """Windows and starts that begin some hundred positions into a block's keys, and rows that see nothing at all."""
    groups = [(900 - 9 * i, [901 + (i * 7 + s * 29) % 60 for s in range(9)] + [0, 500]) for i in range(12)]
    starts = [(s * 97) % 1000 for s in range(12 * 11)]
    c = filled(fmt, groups, 4, 64, seed=18)
    check(c, dtype, 16, 3, window=333)
    check(c, dtype, 16, 3, starts=starts)
    check(c, dtype, 16, 3, starts=starts, window=450, scale=-0.25)


def test_own_parts_of_a_draft_window():
    c = filled("bf16", [(500, [517, 600, 530, 560])], 2, 128, seed=8)
    check(c, "bf16", 8, 17)                                   # the own part on tcgen05 too
    c = filled("int8", [(500, [517, 600, 530, 560])], 1, 64, seed=9)
    check(c, "bf16", 8, 17)


@pytest.mark.parametrize("fmt", ["bf16", "f16"])
@pytest.mark.parametrize("q_heads,new", [(1, 1), (8, 4)])
def test_values_that_are_not_finite_keep_to_the_rows_that_see_them(fmt, q_heads, new):
    """Infinities and NaN among the common values, seen by the sequences whose start lies before them only."""
    c = filled(fmt, [(100, [120, 130, 140, 125])], 1, 64, seed=10)
    q = queries(c, fmt, q_heads, new)
    starts = ints([0, 60, 60, 41])
    kw = dict(bounds=ints(c.bounds), new_tokens=new, starts=starts)
    clean = c.kv.attend_shared(q, c.table, c.len_dev, ints(c.common), **kw)
    pool, at = c.kv.pool(), 40
    for value in (float("inf"), float("nan")):
        pool["v"][int(c.host_table[0, at // 16]), :, at % 16] = value
        got = c.kv.attend_shared(q, c.table, c.len_dev, ints(c.common), **kw)
        assert torch.allclose(got[new:].float(), clean[new:].float(), rtol=2.0 ** -7, atol=2.0 ** -7)   # (weights of another reference)
        rows = got[:new].float()
        assert bool(torch.isposinf(rows).all() if value > 0 else torch.isnan(rows).all())
    c.kv.sync()


def test_bad_groups_are_reported():
    c = filled("bf16", [(100, [120, 130, 140, 125])], 1, 64, seed=11)
    q = queries(c, "bf16", 4, 1)
    want = c.kv.attend(q, c.table, c.len_dev)
    for bounds in ([0, 5], [-1, 4], [3, 1], [0, 3, 2, 4]):
        got = c.kv.attend_shared(q, c.table, c.len_dev, ints([100] * (len(bounds) - 1)), bounds=ints(bounds))
        with pytest.raises(L.LacacheError) as e:
            c.kv.sync()
        assert e.value.status == L.LACACHE_ERR_INVALID_ARG
        assert torch.equal(got, want)                         # without groups: every sequence for itself
    c.kv.attend_shared(q, c.table, c.len_dev, ints([-5]))
    with pytest.raises(L.LacacheError):
        c.kv.sync()
    c.kv.attend_shared(q, c.table, c.len_dev, ints([(1 << 31) - 1]))   # past the table: cut; nothing is left of any sequence's own
    with pytest.raises(L.LacacheError):
        c.kv.sync()
    table = c.table.clone()
    table[0, 2] = c.kv.cfg.pages                              # a page of the common part
    c.kv.attend_shared(q, table, c.len_dev, ints([100]))
    with pytest.raises(L.LacacheError):
        c.kv.sync()
    c.kv.attend_shared(q, c.table, c.len_dev, ints([100]))
    c.kv.sync()


@pytest.mark.parametrize("fmt,dtype", FORMATS[:3])
def test_small_calls_are_the_ordinary_attention(fmt, dtype):
    c = filled(fmt, [(100, [120, 130, 99, 125]), (20, [21])], 2, 64, seed=16, small=True)
    for new in (1, 9):
        out, lse = check(c, dtype, 4, new, window=70)
        q = queries(c, dtype, 4, new)
        want_lse = torch.empty_like(lse)
        want = c.kv.attend(q, c.table, c.len_dev, new_tokens=new, window=70, lse=want_lse)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_strided_rows():
    c = filled("f16", [(90, [100, 95, 121])], 2, 64, seed=12)
    q = queries(c, "f16", 4, 3)
    want = c.kv.attend_shared(q, c.table, c.len_dev, ints([90]), new_tokens=3)
    wide = torch.full((9, 9, 64), float("nan"), dtype=torch.float16, device="cuda")
    wide[:, 1:8:2] = q
    store = torch.full((4, 9, 128), 5.0, dtype=torch.float16, device="cuda")
    out = store.transpose(0, 1)[..., 64:]
    c.kv.attend_shared(wide[:, 1:8:2], c.table, c.len_dev, ints([90]), new_tokens=3, out=out)
    assert torch.equal(out, want) and float(store[..., :64].min()) == 5.0
    c.kv.sync()


def test_two_captured_graphs_and_another_stream():
    c = filled("bf16", [(200, [260, 230, 300]), (32, [64, 50])], 2, 64, seed=13)
    q, lengths, common = queries(c, "bf16", 8, 1), c.len_dev.clone(), ints(c.common)
    bounds, table = ints(c.bounds), c.table.clone()
    outs = [torch.empty_like(q) for _ in range(3)]
    first = ints([210, 201, 205, 40, 33])
    lengths.copy_(first)

    def step(out, stream=None):
        c.kv.attend_shared(q, table, lengths, common, bounds=bounds, out=out, cuda_stream=stream)

    step(outs[2])
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g, out in zip(graphs, outs):
        with torch.cuda.graph(g):
            step(out)
    lengths.copy_(c.len_dev)
    for _ in range(3):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    step(outs[2])
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[2])
    side = torch.cuda.Stream()
    got = torch.empty_like(q)
    torch.cuda.synchronize()
    step(got, side)
    side.synchronize()
    assert torch.equal(got, outs[2])
    check(c, "bf16", 8)


def test_a_wait_that_runs_out_is_reported():
    c = filled("bf16", [(400, [401 + i for i in range(12)])], 2, 64, seed=14)
    q = queries(c, "bf16", 8, 1)
    want = c.kv.attend_shared(q, c.table, c.len_dev, ints([400]))
    L.load().lacache_kv_inject_stall(c.kv.h, 1)
    c.kv.attend_shared(q, c.table, c.len_dev, ints([400]))
    with pytest.raises(L.LacacheError) as e:
        c.kv.sync()
    assert e.value.status == L.LACACHE_ERR_DEVICE_TIMEOUT
    assert torch.equal(c.kv.attend_shared(q, c.table, c.len_dev, ints([400])), want)
    c.kv.sync()


def test_refusals():
    import ctypes
    c = filled("bf16", [(20, [40, 30])], 2, 64, seed=15)
    q, common = queries(c, "bf16", 4, 1), ints([20])
    for args, kw in (((common[:0],), {}), ((common[0],), {}), ((common.long(),), {}), ((ints([20, 5]),), {}), ((common,), dict(bounds=ints([0, 1, 2]))),
                     ((common,), dict(bounds=torch.tensor([0, 2], dtype=torch.int32))), ((common,), dict(window=-1)),
                     ((common,), dict(lse=torch.empty(2, 4)))):
        with pytest.raises(ValueError):
            c.kv.attend_shared(q, c.table, c.len_dev, *args, **kw)
    with pytest.raises(L.LacacheError) as e:
        c.kv.attend_shared(q, c.table, c.len_dev, common, out=q)
    assert e.value.status == L.LACACHE_ERR_INVALID_ARG
    assert c.kv.attend_shared(q[:0], c.table[:0], c.len_dev[:0], common).shape == (0, 4, 64)
    t, a, out = c.kv._attention(q, c.table, c.len_dev, 1, None, 0, None, None, None, None)
    lib, at = L.load(), ctypes.addressof
    size = L.lacache_kv_attend_shared_workspace_bytes(c.kv.h, t, 1, 1, 4)
    assert size > 0 and L.lacache_kv_attend_shared_workspace_bytes(c.kv.h, L.lacache_kv_table(None, 0, 2, 9), 1, 1, 4) == 0
    ws = torch.empty(size + 16, dtype=torch.uint8, device="cuda")
    groups = L.lacache_shared(1, None, common.data_ptr())

    def call(shared=groups, p=ws.data_ptr(), n=size):
        return lib.lacache_kv_attend_shared(c.kv.h, 0, at(t), at(a), at(shared), p, n, torch.cuda.current_stream().cuda_stream)

    assert call() == L.LACACHE_OK
    for bad in (dict(p=None), dict(p=ws.data_ptr() + 8), dict(n=size - 1), dict(shared=L.lacache_shared(0, None, common.data_ptr())),
                dict(shared=L.lacache_shared(2, None, common.data_ptr())), dict(shared=L.lacache_shared(1, None, None))):
        assert call(**bad) == L.LACACHE_ERR_INVALID_ARG, bad
    for bad in ((None, 1, 1, 4), (L.lacache_kv_table(None, 0, -1, 1 << 20), 1, 1, 4), (t, 0, 1, 4), (t, 1, 0, 4), (t, 1, 1, 0)):
        assert L.lacache_kv_attend_shared_workspace_bytes(c.kv.h, *bad) == 0
    c.kv.sync()
