"""The attention weight that cached tokens gather, against the fp64 oracle."""
import numpy as np
import pytest
import torch

from kv_cases import Filled, TORCH
from oracle import decode
from paper_2608_01718_gb300 import build
from paper_2608_01718_gb300 import lacache as L

pytestmark = pytest.mark.gpu
MARK = 12345.0


@pytest.fixture(scope="module", autouse=True)
def library():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    build.build()
    L.load()


def queries(c, dtype, q_heads, new, seed=1, spread=1.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return (torch.randn(len(c.lengths) * new, q_heads, c.kv.cfg.head_dim, generator=gen, device="cuda") * spread).to(TORCH[dtype])


def tolerance(c, q, k, lse, parts, past, decay, scale, rows):
    """A score is off by at most delta, 2^-19 of the sum of |q k| * scale and what a q scaled into f16 loses (2^-24 of its row's
    largest against any key): a share by 2 delta of itself. Its exponent x, in powers of two, is made of lse log2(e), the score and their
    difference, each rounded to 2^-24 of itself (the score, which is below |lse log2(e)| + |x|, up to three times): 2^-22 |lse| +
    2^-22.5 |x| of the share. Shares with |x| <= 8 are covered by 2^-20 (1 + |lse|); smaller ones are below 2^-8, and down to 2^-120
    |x| 2^-22.5 is below 2^-15. The exponential itself is within 2^-22. Sums of `rows` shares and the past round 2^-24 of the whole each."""
    w, by_span, by_lse = parts
    q_top = np.abs(q).max() if q.size else 0.0
    k_sum = np.abs(k).sum(-1).max() if k.size else 0.0
    delta = 2.0 ** -19 * by_span + 2.0 ** -24 * q_top * k_sum * abs(scale) * w
    return 2 * delta + 2.0 ** -20 * (by_lse + w) + 2.0 ** -15 * np.minimum(w, 2.0 ** -8 * rows) + (rows + 4) * 2.0 ** -24 * w + rows * 2.0 ** -120


def check(c, dtype, q_heads, new=1, window=0, starts=None, scale=None, past=True, decay=1.0, wide=0, seed=1, inplace=False, lse=None,
          spread=1.0):
    """One call, after the attention whose lse it takes, against the oracle; returns the weights."""
    B, H, D = len(c.lengths), c.kv.cfg.kv_heads, c.kv.cfg.head_dim
    q = queries(c, dtype, q_heads, new, seed, spread)
    st = None if starts is None else torch.tensor(starts, dtype=torch.int32, device="cuda")
    kw = dict(new_tokens=new, layer=c.layer, starts=st, window=window, scale=scale)
    if lse is None:
        lse = torch.empty(q.shape[:2], device="cuda")
        c.kv.attend(q, c.table, c.len_dev, lse=lse, **kw)
    W = max(c.lengths + [1]) + wide
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 100)
    before = torch.rand(B, H, W, generator=gen, device="cuda") * 5 if past else None
    out = before if inplace else torch.full((B, H, W), MARK, device="cuda")
    kept = None if before is None else before.clone()
    got = c.kv.weigh(q, c.table, c.len_dev, lse, weights=before, decay=decay, out=None if inplace else out, **kw)
    assert got.data_ptr() == out.data_ptr()
    c.kv.sync()
    f = D ** -0.5 if scale is None else scale
    k, _ = c.values()
    hq, hl = q.double().cpu().numpy(), lse.double().cpu().numpy()
    hp = None if kept is None else kept.cpu().numpy()
    want = decode.weigh(hq, k, c.lengths, new, f, hl, hp, decay, starts, window)
    rows = new * q_heads // H
    hg = got.double().cpu().numpy()
    for s, n in enumerate(c.lengths):
        w = want[s][0]
        tol = tolerance(c, hq[s * new:(s + 1) * new], k[s], hl, want[s], hp, decay, f, rows)
        assert np.all(np.abs(hg[s, :, :n] - w) <= tol), (s, float((np.abs(hg[s, :, :n] - w) / np.maximum(tol, 1e-300)).max()))
        rest = hp[s, :, n:] if inplace else MARK
        assert np.all(hg[s, :, n:] == rest)          # what lies behind a sequence stays as it was
    return got


FORMATS = [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16"), ("e4m3", "f16"), ("int8", "bf16"), ("int8", "f16")]


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("kv_heads,group,head_dim,page,new", [(2, 1, 64, 16, 1), (1, 4, 128, 32, 1), (3, 5, 80, 16, 3), (2, 8, 256, 48, 2),
                                                             (1, 7, 192, 16, 11), (2, 4, 128, 16, 17), (1, 2, 16, 16, 1),
                                                             (1, 1, 48, 64, 130)])
def test_against_the_oracle(fmt, dtype, kv_heads, group, head_dim, page, new):
    c = Filled(fmt, [300, 0, 1, 15, 16, 17, 257, 512, 2], kv_heads, head_dim, page, seed=head_dim + new)
    check(c, dtype, kv_heads * group, new)


@pytest.mark.parametrize("fmt,dtype", FORMATS[:1] + FORMATS[2:3])
@pytest.mark.parametrize("kw", [dict(window=40), dict(window=1), dict(window=300, starts=[10, 0, 0, 3, 400, 40]),
                                dict(starts=[0, 5, 1, 16, 17, 39]), dict(scale=0.5), dict(scale=-0.125), dict(scale=0.0),
                                dict(decay=0.25), dict(decay=0.0), dict(past=False), dict(inplace=True, decay=0.5), dict(wide=37)])
def test_masks_and_the_past(fmt, dtype, kw):
    c = Filled(fmt, [333, 5, 0, 100, 257, 40], 2, 64, 16, seed=3)
    for new in (1, 6):
        check(c, dtype, 4, new, **kw)


@pytest.mark.parametrize("fmt,dtype", FORMATS[:3])
def test_many_rows(fmt, dtype):
    c = Filled(fmt, [700, 512, 3, 1100], 1, 128, 32, seed=4)
    check(c, dtype, 2, 512)
    check(c, dtype, 2, 300, window=64)


def test_long_and_sharp():
    """Scores so far apart that most shares underflow, and a long sequence over many blocks."""
    c = Filled("bf16", [40_000, 17], 1, 64, 16, seed=5, spread=4.0)
    check(c, "bf16", 2, 1, spread=4.0)


def test_many_short_sequences():
    c = Filled("f16", [(i * 7) % 41 for i in range(300)], 2, 64, 16, seed=6)
    check(c, "f16", 4, 1)


def test_queries_that_saw_nothing_add_nothing():
    c = Filled("bf16", [50], 1, 64, seed=7)
    lse = torch.full((1, 2), float("-inf"), device="cuda")
    lse[0, 1] = 3.0
    check(c, "bf16", 2, lse=lse)
    got = c.kv.weigh(queries(c, "bf16", 2, 1), c.table, c.len_dev, torch.full((1, 2), float("-inf"), device="cuda"))
    assert float(got.abs().max()) == 0.0


@pytest.mark.parametrize("fmt", ["bf16", "f16", "e4m3", "int8"])
def test_a_key_that_is_not_finite_keeps_to_itself(fmt):
    dtype = fmt if fmt in TORCH else "bf16"
    c = Filled(fmt, [100, 60], 1, 64, seed=8)
    q = queries(c, dtype, 4, 2)
    lse = torch.empty(4, 4, device="cuda")
    c.kv.attend(q, c.table, c.len_dev, new_tokens=2, lse=lse)
    clean = c.kv.weigh(q, c.table, c.len_dev, lse, new_tokens=2)
    bad = torch.zeros(2, 1, 64, device="cuda").to(TORCH[dtype])
    bad[0] = float("nan")
    bad[1] = float("inf")
    at = torch.tensor([37, 99], dtype=torch.int32, device="cuda")        # 99: seen by the last query only
    c.kv.append(bad, bad, torch.zeros(2, dtype=torch.int32, device="cuda"), at, c.table)
    got = c.kv.weigh(q, c.table, c.len_dev, lse, new_tokens=2)
    other = torch.ones(112, dtype=torch.bool, device="cuda")
    other[at.long()] = False
    assert torch.equal(got[0, 0, :112][other], clean[0, 0, :112][other]) and torch.equal(got[1], clean[1])
    assert torch.isnan(got[0, 0, 37])
    c.kv.sync()


def test_bad_pages_and_lengths_are_reported():
    c = Filled("bf16", [100, 60], 1, 64, seed=9)
    q = queries(c, "bf16", 2, 1)
    lse = torch.zeros(2, 2, device="cuda")
    want = c.kv.weigh(q, c.table, c.len_dev, lse)
    c.kv.sync()
    table = c.table.clone()
    table[0, 2] = c.kv.cfg.pages
    table[1, 0] = -5
    got = c.kv.weigh(q, table, c.len_dev, lse)
    with pytest.raises(L.LacacheError) as e:
        c.kv.sync()
    assert e.value.status == L.LACACHE_ERR_INVALID_ARG
    want[0, 0, 32:48] = 0.0
    want[1, 0, :16] = 0.0
    assert torch.equal(got, want)
    short = torch.full((2, 1, 80), MARK, device="cuda")                  # narrower than the first sequence
    c.kv.weigh(q, c.table, c.len_dev, lse, out=short)
    with pytest.raises(L.LacacheError):
        c.kv.sync()
    assert float(short[1, 0, 60:].min()) == MARK
    c.kv.weigh(q, c.table, torch.tensor([-3, 60], dtype=torch.int32, device="cuda"), lse)
    with pytest.raises(L.LacacheError):
        c.kv.sync()


def test_strided_weights_and_queries():
    c = Filled("f16", [90, 33], 2, 64, seed=10)
    q = queries(c, "f16", 4, 2)
    lse = torch.empty(4, 4, device="cuda")
    c.kv.attend(q, c.table, c.len_dev, new_tokens=2, lse=lse)
    past = torch.rand(2, 2, 90, device="cuda")
    want = c.kv.weigh(q, c.table, c.len_dev, lse, weights=past, out=torch.zeros(2, 2, 90, device="cuda"), new_tokens=2)
    wide = torch.full((4, 7, 64), float("nan"), dtype=torch.float16, device="cuda")
    wide[:, 2:6] = q
    store, old = torch.full((2, 2, 2, 131), MARK, device="cuda"), torch.full((3, 2, 95), MARK, device="cuda")
    out = store[:, :, 1, 3:93]
    old.transpose(0, 1)[:, :2, 5:] = past
    c.kv.weigh(wide[:, 2:6], c.table, c.len_dev, lse, weights=old.transpose(0, 1)[:, :2, 5:], out=out, new_tokens=2)
    assert torch.equal(out[0], want[0]) and torch.equal(out[1, :, :33], want[1, :, :33]) and float(out[1, :, 33:].min()) == MARK
    assert float(store[:, :, 0].min()) == MARK and float(store[:, :, 1, :3].min()) == MARK
    c.kv.sync()


def test_replays_read_lengths_anew():
    c = Filled("bf16", [300, 300], 1, 64, seed=11)
    q = queries(c, "bf16", 2, 1)
    lengths, lse = torch.tensor([40, 7], dtype=torch.int32, device="cuda"), torch.empty(2, 2, device="cuda")
    weights = torch.zeros(2, 1, 300, device="cuda")

    def step():
        c.kv.attend(q, c.table, lengths, lse=lse)
        c.kv.weigh(q, c.table, lengths, lse, weights=weights)

    step()
    torch.cuda.synchronize()
    weights.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(5):
        graph.replay()
        lengths += 50 if int(lengths[0]) < 240 else 0
    torch.cuda.synchronize()
    want = torch.zeros(2, 1, 300, device="cuda")
    lengths.copy_(torch.tensor([40, 7], dtype=torch.int32))
    for i in range(5):
        c.kv.attend(q, c.table, lengths, lse=lse)
        c.kv.weigh(q, c.table, lengths, lse, weights=want)
        lengths += 50 if int(lengths[0]) < 240 else 0
    assert torch.equal(weights, want)
    assert abs(float(weights.sum()) - 2 * 2 * 5) < 1e-3                  # every query's shares add up to 1, 5 times
    c.kv.sync()


def test_another_stream_and_layers():
    c = Filled("bf16", [120, 33], 2, 64, seed=12, layers=2, layer=1)
    want = check(c, "bf16", 4, 1)
    q, lse = queries(c, "bf16", 4, 1), torch.empty(2, 4, device="cuda")
    c.kv.attend(q, c.table, c.len_dev, layer=1, lse=lse)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = c.kv.weigh(q, c.table, c.len_dev, lse, layer=1, cuda_stream=side)
    side.synchronize()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(101)
    past = torch.rand(2, 2, 120, generator=gen, device="cuda") * 5
    past[0, :, 119] = 0
    past[1, :, 32] = 0
    for s, n in enumerate(c.lengths):
        assert torch.allclose(got[s, :, :n] + past[s, :, :n], want[s, :, :n], rtol=2 ** -22, atol=2 ** -22)


def test_a_wait_that_runs_out_is_reported():
    c = Filled("bf16", [400, 90], 2, 64, seed=14)
    q, lse = queries(c, "bf16", 8, 9), torch.empty(18, 8, device="cuda")
    c.kv.attend(q, c.table, c.len_dev, new_tokens=9, lse=lse)
    want = c.kv.weigh(q, c.table, c.len_dev, lse, new_tokens=9)
    L.load().lacache_kv_inject_stall(c.kv.h, 1)
    c.kv.weigh(q, c.table, c.len_dev, lse, new_tokens=9)
    with pytest.raises(L.LacacheError) as e:
        c.kv.sync()
    assert e.value.status == L.LACACHE_ERR_DEVICE_TIMEOUT
    assert torch.equal(c.kv.weigh(q, c.table, c.len_dev, lse, new_tokens=9), want)
    c.kv.sync()


@pytest.mark.parametrize("head_dim", [256, 144])
def test_a_wait_that_runs_out_in_wide_heads(head_dim):
    c = Filled("f16", [400, 90], 1, head_dim, seed=15)
    q, lse = queries(c, "f16", 8, 9), torch.zeros(18, 8, device="cuda")
    L.load().lacache_kv_inject_stall(c.kv.h, 1)
    c.kv.weigh(q, c.table, c.len_dev, lse, new_tokens=9)
    with pytest.raises(L.LacacheError) as e:
        c.kv.sync()
    assert e.value.status == L.LACACHE_ERR_DEVICE_TIMEOUT
    check(c, "f16", 8, 9)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("head_dim", [48, 64, 80, 128, 144, 256])
@pytest.mark.parametrize("group,new", [(3, 6), (1, 33), (7, 15), (2, 97)])
def test_rows_of_every_tile(fmt, dtype, head_dim, group, new):
    """From 18 to 200 rows a kv head: tiles that are full, and not."""
    c = Filled(fmt, [530, 128, 1, 0, 255, 257, new, new + 1], 2, head_dim, 16, seed=head_dim + new)
    check(c, dtype, 2 * group, new)
    check(c, dtype, 2 * group, new, window=100, starts=[0, 3, 0, 0, 200, 100, 5, 0], decay=0.5)


def test_refusals():
    c = Filled("bf16", [40], 2, 64, seed=13)
    q, lse = queries(c, "bf16", 4, 1), torch.zeros(1, 4, device="cuda")
    ok = torch.zeros(1, 2, 64, device="cuda")
    for kw in (dict(out=ok[0]), dict(out=ok.double()), dict(out=ok[:, :1]), dict(out=ok.cpu()), dict(out=ok[:, :, ::2]),
               dict(weights=ok[:, :, :39], out=ok), dict(window=-1), dict(layer=1), dict(new_tokens=2)):
        with pytest.raises(ValueError):
            c.kv.weigh(q, c.table, c.len_dev, lse, **kw)
    for bad in (lse.double(), lse[:, :3], lse.T.contiguous()):
        with pytest.raises(ValueError):
            c.kv.weigh(q, c.table, c.len_dev, bad)
    for kw, status in ((dict(decay=float("nan")), L.LACACHE_ERR_INVALID_ARG), (dict(scale=float("inf")), L.LACACHE_ERR_INVALID_ARG)):
        with pytest.raises(L.LacacheError) as e:
            c.kv.weigh(q, c.table, c.len_dev, lse, **kw)
        assert e.value.status == status
    # rows that share memory, and in place with other strides
    for kw in (dict(out=ok[:, :1].expand(1, 2, 64)), dict(weights=torch.zeros(1, 3, 64, device="cuda")[:, ::2], out=ok)):
        if "weights" in kw:
            kw["out"] = kw["weights"].as_strided((1, 2, 64), (192, 64, 1))
        with pytest.raises(L.LacacheError) as e:
            c.kv.weigh(q, c.table, c.len_dev, lse, **kw)
        assert e.value.status == L.LACACHE_ERR_INVALID_ARG
    with pytest.raises(L.LacacheError) as e:
        c.kv.weigh(q.half(), c.table, c.len_dev, lse)
    assert e.value.status == L.LACACHE_ERR_UNSUPPORTED
    assert c.kv.weigh(q[:0], c.table[:0], c.len_dev[:0], lse[:0]).shape == (0, 2, c.table.shape[1] * 16)
    c.kv.sync()


@pytest.mark.parametrize("fmt", ["bf16", "f16", "e4m3", "int8"])
@pytest.mark.parametrize("head_dim,q_heads,new", [(64, 2, 1), (64, 16, 2), (128, 8, 9), (256, 16, 3)])
def test_pages_that_no_query_sees_need_not_be_there(fmt, head_dim, q_heads, new):
    """A window's older pages, and those before a start, may have been given to others: as for the attention, no page of theirs is
    looked at."""
    dtype = fmt if fmt in TORCH else "bf16"
    c = Filled(fmt, [300, 90, 33, 0, 513], 2, head_dim, 16, seed=17)
    q = queries(c, dtype, q_heads, new)
    lse = torch.empty(q.shape[:2], device="cuda")
    past = torch.rand(5, 2, 513, device="cuda")
    for kw, first in ((dict(window=40), [max(0, n - new + 1 - 40) for n in c.lengths]),
                      (dict(starts=torch.tensor([299, 17, 33, 0, 512], dtype=torch.int32, device="cuda")), [299, 17, 33, 0, 512])):
        c.kv.attend(q, c.table, c.len_dev, new_tokens=new, lse=lse, **kw)
        want = c.kv.weigh(q, c.table, c.len_dev, lse, weights=past, out=past.clone(), new_tokens=new, **kw)
        c.kv.sync()
        table = c.table.clone()
        for s, x in enumerate(first):
            # (no key of the third is seen from its start on)
            table[s, :x // 16 if x < c.lengths[s] else table.shape[1]] = -1 if s % 2 else 1 << 29
        again = torch.empty_like(lse)
        if "window" in kw:
            c.kv.attend(q, table, c.len_dev, new_tokens=new, lse=again, **kw)
            assert torch.equal(again, lse)
        got = c.kv.weigh(q, table, c.len_dev, lse, weights=past, out=past.clone(), new_tokens=new, **kw)
        c.kv.sync()
        assert torch.equal(got, want)
