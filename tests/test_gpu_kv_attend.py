"""Attention over the paged cache against the fp64 oracle."""
import math

import numpy as np
import pytest
import torch

from kv_cases import Filled, TORCH, bounds
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


def check(c, dtype, q_heads, new=1, window=0, starts=None, scale=None, seed=1, q=None, q_scale=1.0):
    """One call against the oracle; returns (out, lse)."""
    D, n = c.kv.cfg.head_dim, len(c.lengths) * new
    if q is None:
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        q = (torch.randn(n, q_heads, D, generator=gen, device="cuda") * q_scale).to(TORCH[dtype])
    out = torch.full((n, q_heads, D), float("nan"), dtype=TORCH[dtype], device="cuda")
    lse = torch.full((n, q_heads), float("nan"), device="cuda")
    st = None if starts is None else torch.tensor(starts, dtype=torch.int32, device="cuda")
    c.kv.attend(q, c.table, c.len_dev, new_tokens=new, layer=c.layer, starts=st, window=window, scale=scale, out=out, lse=lse)
    c.kv.sync()
    k, v = c.values()
    f = D ** -0.5 if scale is None else scale
    hq = q.double().cpu().numpy()
    want, want_lse, mass, span = decode.attend(hq, k, v, c.lengths, new, f, starts, window)
    tol, tol_lse = bounds(want, mass, span, want_lse, hq, k, f, dtype)
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.all(np.abs(got - want) <= tol), float((np.abs(got - want) / tol).max())
    empty = np.isinf(want_lse)
    assert np.array_equal(np.isneginf(got_lse), empty) and np.all(got[empty] == 0.0)
    assert np.all(np.abs(got_lse[~empty] - want_lse[~empty]) <= tol_lse[~empty])
    return out, lse


FORMATS = [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16"), ("e4m3", "f16"), ("int8", "bf16"), ("int8", "f16")]


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("head_dim", [16, 64, 80, 128, 208, 256])
def test_one_new_token(fmt, dtype, head_dim):
    c = Filled(fmt, [1, 0, 15, 16, 17, 63, 64, 65, 200, 333], 2, head_dim, seed=head_dim)
    check(c, dtype, 2)
    check(c, dtype, 10)


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("e4m3", "f16"), ("int8", "bf16")])
@pytest.mark.parametrize("group,new", [(1, 2), (1, 8), (3, 3), (8, 1), (4, 4), (16, 1), (5, 6), (8, 5), (17, 2), (4, 17), (1, 70)])
def test_rows_a_kv_head(fmt, dtype, group, new):
    # every number of rows from 2 to 70 or so that share a kv head, drafts masked among themselves; a sequence shorter
    # than its drafts has rows that see nothing
    c = Filled(fmt, [0, 1, new, new + 1, 40, 130, 257], 2, 64, seed=group * 100 + new)
    check(c, dtype, 2 * group, new=new)


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("head_dim", [128, 256])
@pytest.mark.parametrize("new,group", [(3, 4), (9, 4), (33, 1)])
def test_wide_heads_with_drafts(fmt, dtype, head_dim, new, group):
    check(Filled(fmt, [5, 100, 301], 1, head_dim, seed=head_dim + new), dtype, group, new=new)


@pytest.mark.parametrize("fmt,dtype", [("f16", "f16"), ("e4m3", "bf16")])
@pytest.mark.parametrize("page", [16, 48, 64, 4096])
def test_page_sizes(fmt, dtype, page):
    check(Filled(fmt, [1, 47, 48, 49, 500], 3, 96, page=page, seed=page), dtype, 6, new=2)


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("int8", "bf16")])
@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 100, 1 << 30])
def test_windows_and_starts(fmt, dtype, window):
    lengths = [0, 1, 16, 33, 150, 290]
    c = Filled(fmt, lengths, 2, 64, seed=window % 1000)
    check(c, dtype, 4, window=window)
    check(c, dtype, 4, new=4, window=window)
    check(c, dtype, 4, new=4, window=window, starts=[0, 1, 15, 40, 16, 100])      # starts past the end among them
    check(c, dtype, 4, starts=[5, 0, 15, 32, 149, 290])                           # rows of one key, and of none
    check(c, dtype, 4, new=3, starts=[-7, -1, 14, 31, 149, 289])                  # a negative start masks nothing


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16")])
def test_one_long_sequence(fmt, dtype):
    # all the work along one axis: split over the GPU and joined
    check(Filled(fmt, [20_011], 2, 64, page=32, seed=5), dtype, 8)
    check(Filled(fmt, [20_011, 3, 9_000], 1, 128, page=16, seed=6), dtype, 2, new=5)


def test_many_short_sequences():
    rng = np.random.default_rng(3)
    c = Filled("bf16", [int(n) for n in rng.integers(0, 40, 700)], 1, 64, seed=7)
    check(c, "bf16", 3)


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("f16", "f16"), ("int8", "f16")])
def test_large_scores_and_a_late_maximum(fmt, dtype):
    # scores of hundreds: one key takes all; keys in rising order of score move the running maximum at every tile
    c = Filled(fmt, [600, 37], 1, 64, spread=6.0, seed=8)
    check(c, dtype, 4, new=2, q_scale=4.0)
    c = Filled(fmt, [512], 1, 64, seed=9)
    ramp = torch.linspace(-4, 4, 512, device="cuda").view(-1, 1, 1).to(c.k_rows.dtype)
    c.kv.append(torch.ones_like(c.k_rows) * ramp, c.v_rows, c.seq, c.pos, c.table)
    check(c, dtype, 2, q=torch.ones(1, 2, 64, device="cuda", dtype=TORCH[dtype]))
    check(c, dtype, 2, q=-torch.ones(1, 2, 64, device="cuda", dtype=TORCH[dtype]))


@pytest.mark.parametrize("scale", [0.0, -0.25, 3.0])
def test_scales(scale):
    check(Filled("bf16", [100, 7], 1, 64, seed=10), "bf16", 2, scale=scale)


def test_tiny_and_huge_queries_on_an_8_bit_cache():
    # rows of q far outside f16's range, and rows of zeros
    for fmt in ("e4m3", "int8"):
        c = Filled(fmt, [90], 1, 64, seed=11)
        q = torch.randn(1, 4, 64, device="cuda").to(torch.bfloat16)
        q[0, 0] *= 1e30
        q[0, 1] *= 1e-30
        q[0, 2] = 0
        # the huge row's scores are scaled back by the caller's factor
        check(c, "bf16", 4, q=q, scale=1e-29)


def test_tokens_of_very_different_magnitude():
    # the scales of v span 2^60: a weight is held relative to the largest weight times scale
    for fmt in ("e4m3", "int8"):
        c = Filled(fmt, [200, 64], 1, 64, seed=12)
        v = c.v_rows.clone()
        v[::3] *= 2.0 ** 30
        v[1::3] *= 2.0 ** -30
        v[7] = 0
        c.kv.append(c.k_rows, v, c.seq, c.pos, c.table)
        check(c, "bf16", 4)
        c.kv.append(c.k_rows, torch.zeros_like(v), c.seq, c.pos, c.table)
        check(c, "bf16", 4)


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_masked_tokens_hold_stays_out(fmt, dtype, bad):
    # the last draft's key and value are not finite: only its own row may show it
    c = Filled(fmt, [50, 18], 1, 64, seed=13)
    k, v = c.k_rows.clone(), c.v_rows.clone()
    for last in (49, 67):
        k[last], v[last] = bad, bad
    c.kv.append(k, v, c.seq, c.pos, c.table)
    # the oracle cannot see the last token either: compare with a cache that is one token shorter
    short = Filled(fmt, [49, 17], 1, 64, seed=14)
    keep = torch.tensor([i for i in range(68) if i not in (49, 67)], device="cuda")
    short.kv.append(k[keep], v[keep], short.seq, short.pos, short.table)
    q = torch.randn(2 * 3, 4, 64, device="cuda").to(TORCH[dtype])
    out = c.kv.attend(q, c.table, c.len_dev, new_tokens=3)
    pick = torch.tensor([0, 1, 3, 4], device="cuda")
    want, _ = check(short, dtype, 4, new=2, q=q[pick].contiguous())
    assert torch.isfinite(out[pick].float()).all()
    assert np.allclose(out[pick].float().cpu(), want.float().cpu(), rtol=2 ** -7, atol=2 ** -9 * float(v[keep].abs().max()))
    assert torch.isnan(out[torch.tensor([2, 5], device="cuda")].float()).all()
    # the same below a window and before a start
    k, v = c.k_rows.clone(), c.v_rows.clone()
    k[:20], v[:20] = bad, bad
    c.kv.append(k, v, c.seq, c.pos, c.table)
    starts = torch.tensor([20, 0], dtype=torch.int32, device="cuda")
    out = c.kv.attend(q, c.table, c.len_dev, new_tokens=3, starts=starts)
    assert torch.isfinite(out[:3].float()).all()
    out = c.kv.attend(q, c.table, c.len_dev, new_tokens=3, window=28)      # the first draft sees position 20 at the earliest
    assert torch.isfinite(out[:3].float()).all()
    out = c.kv.attend(q, c.table, c.len_dev, new_tokens=3, window=29)      # the first sees position 19, the others do not
    assert torch.isnan(out[0].float()).all() and torch.isfinite(out[1:3].float()).all()


def test_strides_layers_and_shared_pages():
    c = Filled("bf16", [70, 33], 2, 64, layers=3, layer=1, seed=15)
    c.table[1, 0] = c.table[0, 0]                 # a shared prefix
    c.host_table[1, 0] = c.host_table[0, 0]
    want, _ = check(c, "bf16", 8, new=2)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    q = torch.randn(4, 8, 64, generator=gen, device="cuda").bfloat16()
    wide = torch.zeros(4, 3, 8, 96, device="cuda", dtype=torch.bfloat16)
    wide[:, 1, :, 16:80] = q
    into = torch.zeros(8, 4, 72, device="cuda", dtype=torch.bfloat16)
    out = into.transpose(0, 1)[:, :, 8:72]        # heads outermost
    table = torch.full((2, 40), 1 << 29, dtype=torch.int32, device="cuda")
    table[:, : c.table.shape[1]] = c.table
    got = c.kv.attend(wide[:, 1, :, 16:80], table[:, : c.table.shape[1]], c.len_dev, new_tokens=2, layer=1, out=out)
    assert torch.equal(got, want) and float(into[:, :, :8].abs().max()) == 0.0


def test_repeated_calls_agree_to_the_bit():
    c = Filled("e4m3", [5000, 100, 0, 3000], 2, 128, seed=16)
    first, lse = check(c, "bf16", 8)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    q = torch.randn(4, 8, 128, generator=gen, device="cuda").bfloat16()
    for _ in range(20):
        again = torch.empty_like(lse)
        assert torch.equal(c.kv.attend(q, c.table, c.len_dev, lse=again), first) and torch.equal(again, lse)


def test_another_stream_and_a_graph():
    c = Filled("bf16", [300, 20], 2, 64, seed=17)
    q = torch.randn(2, 4, 64, device="cuda").bfloat16()
    want = c.kv.attend(q, c.table, c.len_dev).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = c.kv.attend(q, c.table, c.len_dev)
    side.synchronize()
    assert torch.equal(got, want)
    lengths, static_q = c.len_dev.clone(), q.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = c.kv.attend(static_q, c.table, lengths)
    graph.replay()
    assert torch.equal(out, want)
    lengths.copy_(torch.tensor([299, 1], device="cuda"))     # replays read the lengths anew
    graph.replay()
    assert torch.equal(out, c.kv.attend(q, c.table, lengths))
    c.kv.sync()


def test_a_cache_whose_offsets_pass_32_bits():
    # 2^31 elements a pool and more: the last pages lie past every 32-bit offset
    kv = L.KVCache(8, 128, pages=140_000, page_size=16, format="e4m3")
    pool = kv.pool()
    assert pool["k"].numel() > 2 ** 31
    table = torch.tensor([[139_999, 0, 139_998]], dtype=torch.int32, device="cuda")
    k, v = (torch.randn(40, 8, 128, device="cuda").bfloat16() for _ in range(2))
    seq, pos = torch.zeros(40, dtype=torch.int32, device="cuda"), torch.arange(40, dtype=torch.int32, device="cuda")
    kv.append(k, v, seq, pos, table)
    q = torch.randn(1, 8, 128, device="cuda").bfloat16()
    out = kv.attend(q, table, torch.tensor([40], dtype=torch.int32, device="cuda"))
    kv.sync()
    bk, bv = kv.read(seq, pos, table, dtype=torch.float32)
    hk, hv, hq = (x.double().cpu().numpy() for x in (bk, bv, q))
    want, lse, mass, span = decode.attend(hq, [hk], [hv], [40], 1, 128 ** -0.5)
    tol, _ = bounds(want, mass, span, lse, hq, [hk], 128 ** -0.5, "bf16")
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol)
    kv.close()


def test_bad_indices_are_masked_and_reported():
    c = Filled("bf16", [64, 40], 1, 64, seed=18)
    q = torch.randn(2, 1, 64, device="cuda").bfloat16()
    c.table[0, 1] = 1 << 28
    out = c.kv.attend(q, c.table, c.len_dev)
    with pytest.raises(L.LacacheError) as e:
        c.kv.sync()
    assert e.value.status == L.LACACHE_ERR_INVALID_ARG
    c.kv.sync()                                     # reported once
    k, v = c.values()                               # positions 16 to 31 of the first sequence are masked
    k[0], v[0] = np.delete(k[0], np.s_[16:32], 0), np.delete(v[0], np.s_[16:32], 0)
    hq = q.double().cpu().numpy()
    want, lse, mass, span = decode.attend(hq, k, v, [48, 40], 1, 0.125)
    tol, _ = bounds(want, mass, span, lse, hq, k, 0.125, "bf16")
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol)
    c.table[0, 1] = -1
    c.kv.attend(q, c.table, c.len_dev)
    with pytest.raises(L.LacacheError):
        c.kv.sync()
    c.table[0, 1] = int(c.host_table[0, 1])
    too_long = torch.tensor([10 ** 9, -3], dtype=torch.int32, device="cuda")
    whole = torch.tensor([[*c.host_table[0, :4]], [*c.host_table[1, :3], c.host_table[0, 0]]], dtype=torch.int32,
                         device="cuda")
    got = c.kv.attend(q, whole, too_long)
    with pytest.raises(L.LacacheError):
        c.kv.sync()
    assert torch.equal(got[0], c.kv.attend(q, whole, c.len_dev)[0])      # as long as the table allows
    assert float(got[1].abs().max()) == 0.0
    c.kv.sync()


def test_refusals():
    c = Filled("bf16", [20], 2, 64, seed=19)
    q = torch.randn(1, 4, 64, device="cuda").bfloat16()
    lib, stream = L.load(), torch.cuda.current_stream().cuda_stream
    import ctypes

    def attention(**kw):
        a = L.lacache_attention(1, 4, 0, L.LACACHE_BF16, 0.125, c.len_dev.data_ptr(), None,
                                L.lacache_rows(q.data_ptr(), 256, 64), L.lacache_rows(q.data_ptr(), 256, 64), None)
        for name, value in kw.items():
            setattr(a, name, value)
        return a

    def status(a, layer=0, table=None):
        t = table or L.lacache_kv_table(c.table.data_ptr(), c.table.stride(0), 1, c.table.shape[1])
        return lib.lacache_kv_attend(c.kv.h, layer, ctypes.byref(t), ctypes.byref(a), stream)

    bad, no = L.LACACHE_ERR_INVALID_ARG, L.LACACHE_ERR_UNSUPPORTED
    for kw, want in [(dict(new_tokens=0), bad), (dict(new_tokens=513), no), (dict(q_heads=3), bad), (dict(q_heads=0), bad),
                     (dict(window=-1), bad), (dict(scale=float("nan")), bad), (dict(scale=math.inf), bad),
                     (dict(dtype=L.LACACHE_F32), bad), (dict(dtype=L.LACACHE_F16), no), (dict(lengths_dev=None), bad),
                     (dict(q=L.lacache_rows(q.data_ptr() + 2, 256, 64)), bad),
                     (dict(q=L.lacache_rows(q.data_ptr(), 255, 64)), bad),
                     (dict(out=L.lacache_rows(q.data_ptr(), 256, 60)), bad),
                     (dict(out=L.lacache_rows(None, 256, 64)), bad)]:
        assert status(attention(**kw)) == want, kw
    assert status(attention(), layer=1) == bad and status(attention(), layer=-1) == bad
    assert status(attention(), table=L.lacache_kv_table(None, 4, 1, 4)) == bad
    assert status(attention(), table=L.lacache_kv_table(c.table.data_ptr(), 4, -1, 4)) == bad
    assert status(attention(), table=L.lacache_kv_table(c.table.data_ptr(), 4, 1, 0)) == bad
    assert status(attention(), table=L.lacache_kv_table(None, 4, 0, 4)) == L.LACACHE_OK      # no sequence: nothing to do
    for kw in [dict(q=q[:, :, :32]), dict(q=q.float()), dict(lengths=c.len_dev.long()), dict(table=c.table.long()),
               dict(lse=torch.empty(1, 3, device="cuda")), dict(q=q.cpu()), dict(lengths=c.len_dev.cpu())]:
        args = dict(q=q, table=c.table, lengths=c.len_dev)
        args.update(kw)
        with pytest.raises((ValueError, L.LacacheError)):
            c.kv.attend(args.pop("q"), args.pop("table"), args.pop("lengths"), **args)
    c.kv.sync()
