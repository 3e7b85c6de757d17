"""Attention over values that are not finite, very large, or of very different magnitudes, against the fp64 oracle: what only
some rows see, what a weight rounded to fewer bits would lose, and what an unnormalised sum would."""
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


def rows_along_first(scores, head_dim, dtype):
    """Rows whose product with (1, 0, 0, ...) is `scores` [n x heads]; their other elements are small and random."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    s = torch.as_tensor(scores, dtype=torch.float32, device="cuda")
    x = torch.randn(*s.shape, head_dim, generator=gen, device="cuda") / 64
    x[..., 0] = s
    return x.to(dtype)


def first(n, heads, head_dim, dtype):
    q = torch.zeros(n, heads, head_dim, device="cuda", dtype=dtype)
    q[..., 0] = 1
    return q


# rows a kv head: eight, nine to sixteen, and the many-row kernel's
ROWS = [(1, 4), (3, 4), (9, 4)]


@pytest.mark.parametrize("new,group", ROWS)
@pytest.mark.parametrize("head_dim", [64, 128])
def test_an_infinity_under_a_weight_that_f16_rounds_to_zero(new, group, head_dim):
    # its weight is 2^-43 of the largest: below f16's range, but not zero, so the output is an infinity and not 0 x inf
    c = Filled("f16", [290], 1, head_dim, seed=20)
    scores = torch.zeros(290, 1)
    scores[5] = -30.0
    v = c.v_rows.clone()
    v[5, 0, 3], v[5, 0, 9] = float("inf"), -float("inf")
    c.kv.append(rows_along_first(scores, head_dim, torch.float16), v, c.seq, c.pos, c.table)
    out = c.kv.attend(first(new, group, head_dim, torch.float16), c.table, c.len_dev, new_tokens=new, scale=1.0)
    c.kv.sync()
    assert (out[..., 3] == float("inf")).all() and (out[..., 9] == -float("inf")).all()
    rest = [d for d in range(head_dim) if d not in (3, 9)]
    k, vv = c.values()
    vv[0][5, 0, [3, 9]] = 0.0
    q = first(new, group, head_dim, torch.float64).cpu().numpy()
    want, lse, mass, span = decode.attend(q, k, vv, c.lengths, new, 1.0)
    tol, _ = bounds(want, mass, span, lse, q, k, 1.0, "f16")
    assert np.all((np.abs(out.double().cpu().numpy() - want) <= tol)[..., rest])


@pytest.mark.parametrize("new,group", ROWS)
@pytest.mark.parametrize("head_dim", [64, 128])
def test_weights_keep_their_bits_beside_an_infinity(new, group, head_dim):
    """bf16: one dimension of one value is an infinity; the other dimensions are as exact as without it. A weight's two bf16
    terms leave 2^-18 of it, the scores' error delta (kv_cases.bounds) 4 delta; the output rounds to within 2^-8 of itself."""
    c = Filled("bf16", [290], 1, head_dim, seed=21)
    v = c.v_rows.clone()
    v[100, 0, 3] = float("inf")
    c.kv.append(c.k_rows, v, c.seq, c.pos, c.table)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    q = torch.randn(new, group, head_dim, generator=gen, device="cuda").bfloat16()
    out = c.kv.attend(q, c.table, c.len_dev, new_tokens=new, scale=head_dim ** -0.5)
    c.kv.sync()
    assert (out[..., 3] == float("inf")).all()
    k, vv = c.values()
    vv[0][100, 0, 3] = 0.0
    hq = q.double().cpu().numpy()
    want, lse, mass, span = decode.attend(hq, k, vv, c.lengths, new, head_dim ** -0.5)
    delta = 2.0 ** -19 * span
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -17 + 4 * delta)[..., None] * mass
    rest = [d for d in range(head_dim) if d != 3]
    assert np.all((np.abs(out.double().cpu().numpy() - want) <= tol)[..., rest])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new,group", [(2, 1), (4, 2), (4, 4), (8, 4), (9, 4)])
@pytest.mark.parametrize("head_dim", [48, 64, 80, 128, 256])
def test_codes_that_are_no_numbers_stay_in_the_rows_that_see_them(dtype, new, group, head_dim):
    """e4m3: NaN codes in V (0x7f and 0xff; a pool filled by a page copy or another quantiser may hold them) of the last two
    tokens, in dimensions of their own. A row shows NaN where it sees the token and nowhere else."""
    c = Filled("e4m3", [150, new + 1], 2, head_dim, seed=22)
    bad = {1: [0, 17, head_dim - 1], 2: [5, 30, head_dim - 10]}      # tokens from the end: dimensions
    pool = c.kv.pool()["v"].view(torch.uint8)
    seen = np.zeros((2 * new, 2 * group, head_dim), dtype=bool)
    for s, n in enumerate(c.lengths):
        for back, dims in bad.items():
            p = n - back
            for i, d in enumerate(dims):
                pool[int(c.host_table[s, p // 16]), :, p % 16, d] = 0x7f if i % 2 else 0xff
                for t in range(new):
                    if n - new + t >= p:
                        seen[s * new + t, :, d] = True
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    q = torch.randn(2 * new, 2 * group, head_dim, generator=gen, device="cuda").to(TORCH[dtype])
    out = c.kv.attend(q, c.table, c.len_dev, new_tokens=new)
    c.kv.sync()
    got = out.double().cpu().numpy()
    k, v = c.values()
    v = [np.nan_to_num(x, nan=0.0) for x in v]
    hq = q.double().cpu().numpy()
    want, lse, mass, span = decode.attend(hq, k, v, c.lengths, new, head_dim ** -0.5)
    tol, _ = bounds(want, mass, span, lse, hq, k, head_dim ** -0.5, dtype)
    assert np.array_equal(np.isnan(got), seen)
    assert np.all((np.abs(got - want) <= tol)[~seen])


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("new,group", [(1, 1), (2, 4), (3, 4), (9, 4)])
@pytest.mark.parametrize("head_dim", [64, 128, 256])
@pytest.mark.parametrize("gap", [20.0, 60.0, 95.0])
def test_large_values_of_small_weight_before_small_values_of_large_weight(fmt, new, group, head_dim, gap):
    """8-bit caches, whose scales multiply the weights: the first token's value is 2^40 times the others' (at 20 nats 2^12), the
    last ones' scores are `gap` nats above its, the rest's far below both. The late tokens decide the output. Enough
    sequences that a block has whole ones, so that a warp meets both."""
    c = Filled(fmt, [300], 8, head_dim, seed=23)
    scores = torch.full((300, 8), -gap - 90.0)
    scores[0] = -gap
    scores[-76 - new:] = torch.linspace(-1, 0, 76 + new).unsqueeze(1)
    v = c.v_rows.clone()
    v[0] *= 2.0 ** (40 if gap > 20 else 12)
    c.kv.append(rows_along_first(scores, head_dim, torch.bfloat16), v, c.seq, c.pos, c.table)
    seqs = 128                                       # of one table row each, all the same
    q = first(seqs * new, 8 * group, head_dim, torch.bfloat16)
    table, lengths = c.table.expand(seqs, -1), c.len_dev.expand(seqs).contiguous()
    out = c.kv.attend(q, table, lengths, new_tokens=new, scale=1.0)
    c.kv.sync()
    k, vv = c.values()
    hq = q[:new].double().cpu().numpy()
    want, lse, mass, span = decode.attend(hq, k, vv, [300], new, 1.0)
    tol, _ = bounds(want, mass, span, lse, hq, k, 1.0, "bf16")
    got = out.view(seqs, new, -1, head_dim).double().cpu().numpy()
    assert np.all(np.abs(got - want) <= tol), float((np.abs(got - want) / tol).max())


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("new,group", [(1, 1), (1, 4), (3, 4), (9, 4)])
@pytest.mark.parametrize("head_dim", [64, 128, 256])
def test_values_near_the_largest_float(fmt, new, group, head_dim):
    """V of 2^119 and scores that rise: weights taken relative to less than the largest would bring the sums past fp32's range
    (290 of them by their softmax weights stay within it)."""
    c = Filled(fmt, [290], 2, head_dim, seed=24)
    scores = torch.linspace(-9, 0, 290).unsqueeze(1).expand(-1, 2)
    v = (c.v_rows.float().clamp(-1, 1) * 2.0 ** 119).to(torch.bfloat16)
    c.kv.append(rows_along_first(scores, head_dim, torch.bfloat16), v, c.seq, c.pos, c.table)
    q = first(new, 2 * group, head_dim, torch.bfloat16)
    out = c.kv.attend(q, c.table, c.len_dev, new_tokens=new, scale=1.0)
    c.kv.sync()
    k, vv = c.values()
    hq = q.double().cpu().numpy()
    want, lse, mass, span = decode.attend(hq, k, vv, c.lengths, new, 1.0)
    tol, _ = bounds(want, mass, span, lse, hq, k, 1.0, "bf16")
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all() and np.all(np.abs(got - want) <= tol)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("new,group", [(1, 4), (3, 4), (9, 4)])
def test_partial_sums_whose_join_would_leave_the_range(fmt, new, group):
    # equal weights, one value everywhere: every part's sum is finite, and the parts' total is not
    c = Filled(fmt, [384], 2, 64, seed=25)
    v = torch.full_like(c.v_rows, 2.0 ** 113)
    c.kv.append(rows_along_first(torch.zeros(384, 2), 64, torch.bfloat16), v, c.seq, c.pos, c.table)
    out = c.kv.attend(first(new, 2 * group, 64, torch.bfloat16), c.table, c.len_dev, new_tokens=new, scale=1.0)
    c.kv.sync()
    assert ((out.double() / 2.0 ** 113 - 1).abs() <= 2.0 ** -8).all()


@pytest.mark.parametrize("where,n", [("k", 300_000), ("v", 1_200_000)])
def test_a_long_sequence_that_is_not_finite_leaves_the_others_alone(where, n):
    """Many rows: outputs that are not finite are computed again key by key, which over 1,200,000 keys takes longer than the bound of
    the kernel's waits. That is no timeout, and the sequences that share the blocks are as without it."""
    new, D, page, seqs = 32, 16, 64, 200
    used = -(-n // page)
    kv = L.KVCache(1, D, 2 * used, page, "bf16")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(26)
    pool = kv.pool()
    for name in "kv":
        half = torch.randn(used, 1, page, D, generator=gen, device="cuda").bfloat16()
        pool[name][:used] = half
        pool[name][used:] = half
    if where == "k":
        pool["k"][used, 0, 5, 2] = float("nan")                  # sequence 1's token 5
    else:
        pool["v"][used, 0, 5, 3], pool["v"][used, 0, 7, 5] = float("inf"), float("nan")
    table = torch.arange(used, dtype=torch.int32, device="cuda").repeat(seqs, 1)
    table[1] += used
    q = torch.randn(new, 1, D, generator=gen, device="cuda").bfloat16()
    lengths = torch.full((seqs,), n, dtype=torch.int32, device="cuda")
    lse = torch.empty(seqs * new, 1, device="cuda")
    out = kv.attend(q.repeat(seqs, 1, 1), table, lengths, new_tokens=new, lse=lse).view(seqs, new, 1, D)
    kv.sync()
    rows = [pool[name][:used].transpose(1, 2).reshape(-1, 1, D)[:n].double().cpu().numpy() for name in "kv"]
    hq = q.double().cpu().numpy()
    want, want_lse, mass, span = decode.attend(hq, rows[:1], rows[1:], [n], new, D ** -0.5)
    tol, tol_lse = bounds(want, mass, span, want_lse, hq, rows[:1], D ** -0.5, "bf16")
    got, got_lse = out.double().cpu().numpy(), lse.view(seqs, new, 1).double().cpu().numpy()
    healthy = [s for s in range(seqs) if s != 1]
    assert np.all(np.abs(got[healthy] - want) <= tol) and np.all(np.abs(got_lse[healthy] - want_lse) <= tol_lse)
    if where == "k":
        assert np.isnan(got[1]).all() and np.isnan(got_lse[1]).all()
    else:
        rest = [d for d in range(D) if d not in (3, 5)]
        assert np.isposinf(got[1, ..., 3]).all() and np.isnan(got[1, ..., 5]).all()
        assert np.all((np.abs(got[1] - want) <= tol)[..., rest]) and np.all(np.abs(got_lse[1] - want_lse) <= tol_lse)
    kv.close()


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("new,group", [(1, 3), (3, 2), (4, 4), (7, 4), (10, 12)])
@pytest.mark.parametrize("head_dim,window", [(64, 0), (80, 37), (128, 150), (256, 0)])
def test_scattered_values_that_are_not_finite(fmt, dtype, new, group, head_dim, window):
    """Infinities and NaN here and there in V, and NaN in K, of many ragged sequences, most of which are finite: every output is what the
    oracle's is, finite, infinite or NaN. (8-bit caches: NaN codes of e4m3, NaN scales of both.)"""
    rng = np.random.default_rng(new * 1000 + head_dim + window)
    lengths = [int(n) for n in rng.integers(0, 260, 30)] + [1500, new, new + 1]
    c = Filled(fmt, lengths, 2, head_dim, seed=27)
    pool = c.kv.pool()
    bad = {"bf16": [np.inf, -np.inf, np.nan], "f16": [np.inf, -np.inf, np.nan]}.get(fmt, [])
    for s in range(0, len(lengths), 2):
        for _ in range(int(rng.integers(1, 6))):
            n = lengths[s]
            if n == 0:
                continue
            p = int(rng.integers(max(0, n - 2 * new), n)) if rng.random() < 0.6 else int(rng.integers(0, n))
            page, at, h, d = int(c.host_table[s, p // c.page]), p % c.page, int(rng.integers(0, 2)), int(rng.integers(0, head_dim))
            kind = rng.random()
            if kind < 0.15:                                                    # K: the whole row for those who see it
                if fmt in ("bf16", "f16"):
                    pool["k"][page, h, at, d] = float("nan")
                else:
                    pool["ks"][page, h, at] = float("nan")
            elif fmt in ("bf16", "f16"):
                pool["v"][page, h, at, d] = float(bad[int(rng.integers(0, 3))])
            elif fmt == "e4m3" and kind < 0.8:
                pool["v"].view(torch.uint8)[page, h, at, d] = 0x7f
            else:
                pool["vs"][page, h, at] = float("nan")
    starts = [int(rng.integers(0, n + 1)) if rng.random() < 0.3 else 0 for n in lengths]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(28)
    q = torch.randn(len(lengths) * new, 2 * group, head_dim, generator=gen, device="cuda").to(TORCH[dtype])
    out = c.kv.attend(q, c.table, c.len_dev, new_tokens=new, window=window,
                      starts=torch.tensor(starts, dtype=torch.int32, device="cuda"))
    c.kv.sync()
    k, v = c.values()
    hq = q.double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        want, _, _, _ = decode.attend(hq, k, v, lengths, new, head_dim ** -0.5, starts, window)
        got = out.double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(want).any()
        assert np.array_equal(np.isposinf(got), np.isposinf(want)) and np.array_equal(np.isneginf(got), np.isneginf(want))
        # what is finite, against the same without them
        k, v = [[np.nan_to_num(x, nan=0.0, posinf=0.0, neginf=0.0) for x in rows] for rows in (k, v)]
        clean, lse, mass, span = decode.attend(hq, k, v, lengths, new, head_dim ** -0.5, starts, window)
        tol, _ = bounds(clean, mass, span, lse, hq, k, head_dim ** -0.5, dtype)
        fine = np.isfinite(want)
        assert np.all((np.abs(got - want) <= tol)[fine])
