"""Attention of many rows a kv head (a window of drafts times a group of heads) against the fp64 oracle: the kernel that takes
more than 16 rows, or more than 32 over an 8-bit cache with heads of up to 64."""
import numpy as np
import pytest
import torch

from kv_cases import Filled, TORCH
from paper_2608_01718_gb300 import build
from paper_2608_01718_gb300 import lacache as L
from test_gpu_kv_attend import FORMATS, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    build.build()
    L.load()


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("head_dim", [16, 48, 64, 80, 112, 128])
@pytest.mark.parametrize("group,new", [(3, 11), (2, 9), (8, 16), (1, 129)])
def test_head_dims(fmt, dtype, head_dim, group, new):
    # 33, 18, 128 and 129 rows; keys that end inside a tile of 128, at it and past it; sequences shorter than their drafts
    c = Filled(fmt, [0, 1, new, 100, 128, 129, 300], 2, head_dim, seed=head_dim + new)
    check(c, dtype, 2 * group, new=new)


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "f16"), ("int8", "bf16")])
@pytest.mark.parametrize("rows", [(1, 33), (33, 1), (40, 1), (5, 13), (7, 18), (17, 8), (16, 17), (1, 512)])
def test_row_counts(fmt, dtype, rows):
    # one tile of rows and several, with warps that hold none; groups from 1 to 40
    group, new = rows
    check(Filled(fmt, [40, 0, 513, 259], 1, 64, seed=group + new), dtype, group, new=new)


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("window", [1, 16, 100, 127, 128, 129])
def test_windows_and_starts(fmt, dtype, window):
    c = Filled(fmt, [0, 1, 16, 33, 150, 290], 1, 128, seed=window)
    check(c, dtype, 4, new=10, window=window)
    check(c, dtype, 4, new=10, window=window, starts=[0, 1, 15, 40, 16, 280])
    check(c, dtype, 4, new=10, starts=[-7, 0, 12, 31, 149, 290])


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16")])
@pytest.mark.parametrize("page", [16, 48, 4096])
def test_long_and_ragged(fmt, dtype, page):
    # split over the GPU and joined; many triples a block; pages of other sizes
    check(Filled(fmt, [15_001, 3, 6_000], 2, 64, page=page, seed=page), dtype, 16, new=5)
    rng = np.random.default_rng(page)
    check(Filled(fmt, [int(n) for n in rng.integers(0, 200, 200)], 2, 128, page=page, seed=page + 1), dtype, 12, new=6)


@pytest.mark.parametrize("scale", [0.0, -0.25, 3.0])
@pytest.mark.parametrize("fmt,dtype", [("f16", "f16"), ("int8", "bf16")])
def test_scales(fmt, dtype, scale):
    check(Filled(fmt, [200, 7], 1, 64, seed=10), dtype, 10, new=4, scale=scale)


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "f16")])
def test_large_scores_and_a_late_maximum(fmt, dtype):
    c = Filled(fmt, [600, 137], 1, 64, spread=6.0, seed=8)
    check(c, dtype, 8, new=5, q_scale=4.0)
    c = Filled(fmt, [900], 1, 64, seed=9)
    ramp = torch.linspace(-4, 4, 900, device="cuda").view(-1, 1, 1).to(c.k_rows.dtype)
    c.kv.append(torch.ones_like(c.k_rows) * ramp, c.v_rows, c.seq, c.pos, c.table)
    ones = torch.ones(40, 1, 64, device="cuda", dtype=TORCH[dtype])
    check(c, dtype, 1, new=40, q=ones)
    check(c, dtype, 1, new=40, q=-ones)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_tokens_of_very_different_magnitude(fmt):
    c = Filled(fmt, [200, 64], 1, 128, seed=12)
    v = c.v_rows.clone()
    v[::3] *= 2.0 ** 30
    v[1::3] *= 2.0 ** -30
    v[7] = 0
    c.kv.append(c.k_rows, v, c.seq, c.pos, c.table)
    check(c, "bf16", 8, new=5)
    c.kv.append(c.k_rows, torch.zeros_like(v), c.seq, c.pos, c.table)
    check(c, "bf16", 8, new=5)


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_masked_tokens_hold_stays_out(fmt, dtype, bad):
    # the last two drafts' keys and values are not finite: only their own rows may show it
    new, group = 9, 4
    c = Filled(fmt, [250, 18], 1, 128, seed=13)
    k, v = c.k_rows.clone(), c.v_rows.clone()
    for last in (248, 249, 266, 267):
        k[last], v[last] = bad, bad
    c.kv.append(k, v, c.seq, c.pos, c.table)
    short = Filled(fmt, [248, 16], 1, 128, seed=14)       # the cache without them
    keep = torch.tensor([i for i in range(268) if i not in (248, 249, 266, 267)], device="cuda")
    short.kv.append(k[keep], v[keep], short.seq, short.pos, short.table)
    q = torch.randn(2 * new, group, 128, device="cuda").to(TORCH[dtype])
    out = c.kv.attend(q, c.table, c.len_dev, new_tokens=new)
    pick = torch.tensor([i for i in range(2 * new) if i % new < new - 2], device="cuda")
    want, _ = check(short, dtype, group, new=new - 2, q=q[pick].contiguous())
    assert torch.isfinite(out[pick].float()).all()
    assert np.allclose(out[pick].float().cpu(), want.float().cpu(), rtol=2 ** -7, atol=2 ** -9 * float(v[keep].abs().max()))
    others = torch.tensor([i for i in range(2 * new) if i % new >= new - 2], device="cuda")
    assert torch.isnan(out[others].float()).all()


def test_an_infinite_value_that_is_seen():
    # the weights' second terms may be zero: an infinity in V is an infinity in the output, not a NaN
    for new, group in ((1, 4), (9, 4)):
        c = Filled("bf16", [300], 1, 64, seed=15)
        v = c.v_rows.clone()
        v[5, 0, 3], v[6, 0, 9] = float("inf"), -float("inf")
        c.kv.append(c.k_rows, v, c.seq, c.pos, c.table)
        q = torch.randn(new, group, 64, device="cuda").bfloat16()
        out = c.kv.attend(q, c.table, c.len_dev, new_tokens=new).float()
        assert (out[..., 3] == float("inf")).all() and (out[..., 9] == -float("inf")).all()
        rest = [d for d in range(64) if d not in (3, 9)]
        assert torch.isfinite(out[..., rest]).all()


def test_repeated_calls_agree_to_the_bit_and_bad_pages_are_masked():
    c = Filled("f16", [5000, 100, 0, 3000], 2, 128, seed=16)
    first, lse = check(c, "f16", 16, new=5)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    q = torch.randn(20, 16, 128, generator=gen, device="cuda").half()
    for _ in range(20):
        again = torch.empty_like(lse)
        assert torch.equal(c.kv.attend(q, c.table, c.len_dev, new_tokens=5, lse=again), first) and torch.equal(again, lse)
    c.kv.sync()
    c.table[1, 2] = -1
    out = c.kv.attend(q, c.table, c.len_dev, new_tokens=5)
    with pytest.raises(L.LacacheError) as e:
        c.kv.sync()
    assert e.value.status == L.LACACHE_ERR_INVALID_ARG
    assert torch.isfinite(out.float()).all() and torch.equal(out[:5], first[:5]) and torch.equal(out[15:], first[15:])
    assert not torch.equal(out[5:10], first[5:10])
