"""Eviction by weight against the oracle: kept positions, and every bit of what is copied."""
import numpy as np
import pytest
import torch

from kv_cases import Filled
from oracle import decode
from paper_2608_01718_gb300 import build
from paper_2608_01718_gb300 import lacache as L

pytestmark = pytest.mark.gpu
MARK = 777.0


@pytest.fixture(scope="module", autouse=True)
def library():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    build.build()
    L.load()


def filled(fmt, lengths, kv_heads, head_dim, page, keep, seed=0, **kw):
    """A cache, and a table of spare pages for what is kept."""
    each = -(-keep // page)
    c = Filled(fmt, lengths, kv_heads, head_dim, page, seed=seed, spare=each * len(lengths) + 2, **kw)
    used = sum(-(-n // page) for n in lengths)
    taken = {int(c.host_table[s, i]) for s, n in enumerate(lengths) for i in range(-(-n // page))}
    free = [p for p in range(c.kv.cfg.pages) if p not in taken]
    assert len(taken) == used
    rng = np.random.default_rng(seed + 1)
    to = rng.permutation(free)[:each * len(lengths)].reshape(len(lengths), each).astype(np.int32)
    return c, to


def bits(t):
    return t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()]).cpu().numpy()


def check(c, to, weights, keep, recent=0, starts=None, lengths=None):
    B, H, page = len(c.lengths), c.kv.cfg.kv_heads, c.page
    lengths = c.lengths if lengths is None else lengths
    st = None if starts is None else torch.tensor(starts, dtype=torch.int32, device="cuda")
    kept = torch.full((B, H, keep), -9, dtype=torch.int32, device="cuda")
    new_w = torch.full((B, H, keep + 3), MARK, device="cuda")
    before = {n: bits(t).copy() for n, t in c.kv.pool(c.layer).items()}
    new_lengths, got, nw = c.kv.evict(c.table, c.len_dev, weights, keep, torch.from_numpy(to).cuda(), recent=recent, layer=c.layer,
                                      starts=st, kept=kept, new_weights=new_w)
    c.kv.sync()
    assert got is kept and nw is new_w
    w = weights.cpu().numpy()
    want = decode.evict([w[s, :, :n] for s, n in enumerate(lengths)], lengths, keep, recent, starts)
    assert new_lengths.tolist() == [len(rows[0]) for rows in want]
    hk, hw = kept.cpu().numpy(), new_w.cpu().numpy()
    for name, old in before.items():
        expect = old.copy()
        for s, rows in enumerate(want):
            for h, pos in enumerate(rows):
                for i, j in enumerate(pos):
                    expect[to[s, i // page], h, i % page] = old[c.host_table[s, j // page], h, j % page]
        assert np.array_equal(bits(c.kv.pool(c.layer)[name]), expect), name
    for s, rows in enumerate(want):
        for h, pos in enumerate(rows):
            assert hk[s, h].tolist() == pos + [-1] * (keep - len(pos))
            assert np.array_equal(hw[s, h, :len(pos)], w[s, h, pos], equal_nan=True) and np.all(hw[s, h, len(pos):] == MARK)
    return kept


def random_weights(c, seed, wide=0, levels=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    w = torch.rand(len(c.lengths), c.kv.cfg.kv_heads, max(c.lengths) + wide, generator=gen, device="cuda")
    return (w * levels).floor() if levels else w ** 8 * 100


@pytest.mark.parametrize("fmt", ["bf16", "f16", "e4m3", "int8"])
@pytest.mark.parametrize("kv_heads,head_dim,page,keep,recent", [(2, 64, 16, 20, 4), (1, 128, 32, 100, 0), (3, 80, 16, 33, 33), (2, 256, 48, 7, 1),
                                                               (1, 16, 16, 64, 10), (2, 192, 16, 1, 0)])
def test_against_the_oracle(fmt, kv_heads, head_dim, page, keep, recent):
    c, to = filled(fmt, [150, 0, 1, keep, keep + 1, 40, 513], kv_heads, head_dim, page, keep, seed=head_dim)
    check(c, to, random_weights(c, 1), keep, recent)


@pytest.mark.parametrize("keep,recent", [(1, 0), (1, 1), (31, 0), (200, 50), (200, 200), (599, 0), (600, 0), (1000, 3)])
def test_budgets(keep, recent):
    c, to = filled("bf16", [600, 333], 2, 16, 16, keep, seed=2)
    check(c, to, random_weights(c, 2), keep, recent)


@pytest.mark.parametrize("levels", [1, 2, 5])
def test_equal_weights_go_to_the_earlier_positions(levels):
    c, to = filled("bf16", [3000, 70], 2, 16, 16, 300, seed=3)
    check(c, to, random_weights(c, 3, levels=levels), 300, 20)


def test_weights_that_are_no_plain_numbers():
    c, to = filled("f16", [400, 90], 1, 16, 16, 60, seed=4)
    w = random_weights(c, 4) - 1.0
    special = torch.tensor([float("nan"), float("inf"), float("-inf"), 0.0, -0.0, 1e-45, -1e-45, 3e38], device="cuda")
    w[:, :, ::3] = special[torch.arange(w[:, :, ::3].shape[-1], device="cuda") % 8]
    check(c, to, w, 60, 5)
    w[0, 0, :350] = float("nan")
    check(c, to, w, 60, 5)
    w[:] = float("nan")
    check(c, to, w, 60, 0)
    w.view(torch.int32)[0, 0, ::2] = -1                              # another NaN: the same rank
    check(c, to, w, 60, 0)


def test_padding_goes_first():
    c, to = filled("bf16", [200, 64, 30, 5], 2, 64, 16, 50, seed=5)
    w = random_weights(c, 5)
    w[:, :, :20] = 1000.0
    check(c, to, w, 50, 10, starts=[17, 20, 3, 9])
    check(c, to, w, 50, 50, starts=[199, 64, -4, 0])


def test_long_sequences():
    c, to = filled("bf16", [70_001, 20_000], 1, 16, 16, 5000, seed=6)
    check(c, to, random_weights(c, 6), 5000, 100)


def test_more_positions_than_shared_memory_holds():
    c, to = filled("bf16", [450_001, 9], 1, 16, 128, 700, seed=12)
    check(c, to, random_weights(c, 12), 700, 100)
    check(c, to, random_weights(c, 13, levels=40), 700, 0)


@pytest.mark.parametrize("kv_heads,lengths", [(3, [9000] * 40), (1, [5000, 4097, 12_288, 2048]), (8, [20_000, 11])])
def test_clusters_of_every_size(kv_heads, lengths):
    c, to = filled("bf16", lengths, kv_heads, 16, 64, 900, seed=13)
    check(c, to, random_weights(c, 14, levels=1000), 900, 77)


def test_strided_weights_and_layers():
    c, to = filled("bf16", [100, 44], 2, 64, 16, 30, seed=7, layers=2, layer=1)
    w = random_weights(c, 7, wide=9)
    store = torch.full((2, 3, 2, 117), float("nan"), device="cuda")
    store[:, 1, :, 5:114] = w
    a = check(c, to, store[:, 1, :, 5:114], 30, 4)
    assert torch.equal(a, check(c, to, w, 30, 4))


def test_bad_pages_and_lengths_are_reported():
    c, to = filled("bf16", [100, 60], 1, 64, 16, 48, seed=8)
    w = random_weights(c, 8)
    target = torch.from_numpy(to).cuda()
    before = bits(c.kv.pool()["k"]).copy()
    c.table[0, 1] = c.kv.cfg.pages + 5
    target[1, 2] = -1
    lengths, kept, _ = c.kv.evict(c.table, c.len_dev, w, 48, target)
    with pytest.raises(L.LacacheError) as e:
        c.kv.sync()
    assert e.value.status == L.LACACHE_ERR_INVALID_ARG
    want = decode.evict([w[s, :, :n].cpu().numpy() for s, n in enumerate(c.lengths)], c.lengths, 48, 0)
    assert lengths.tolist() == [48, 48] and kept.tolist() == want
    expect = before.copy()
    for s in range(2):
        for i, j in enumerate(want[s][0]):
            if not (s == 0 and j // 16 == 1) and not (s == 1 and i // 16 == 2):
                expect[to[s, i // 16], 0, i % 16] = before[c.host_table[s, j // 16], 0, j % 16]
    assert np.array_equal(bits(c.kv.pool()["k"]), expect)
    c, to = filled("bf16", [100, 60], 1, 64, 16, 48, seed=8)
    target = torch.from_numpy(to).cuda()
    for lengths_bad, narrow in (([100, 60], 90), ([100, -1], 100)):      # cut to the weights' width; negative: empty
        cut = [min(max(n, 0), narrow) for n in lengths_bad]
        ln = torch.tensor(lengths_bad, dtype=torch.int32, device="cuda")
        new_lengths, kept, _ = c.kv.evict(c.table, ln, w[:, :, :narrow], 48, target)
        with pytest.raises(L.LacacheError):
            c.kv.sync()
        assert new_lengths.tolist() == [min(48, n) for n in cut]
        want = decode.evict([w[s, :, :n].cpu().numpy() for s, n in enumerate(cut)], cut, 48, 0)
        assert [[x for x in r if x >= 0] for r in kept[:, 0].tolist()] == [r[0] for r in want]


def test_capture_and_another_stream():
    c, to = filled("e4m3", [300, 90], 2, 64, 16, 64, seed=9)
    w, target = random_weights(c, 9), torch.from_numpy(to).cuda()
    lengths = torch.tensor([100, 20], dtype=torch.int32, device="cuda")
    out = [torch.empty(2, dtype=torch.int32, device="cuda"), torch.empty(2, 2, 64, dtype=torch.int32, device="cuda"),
           torch.zeros(2, 2, 64, device="cuda")]

    def step(stream=None):
        c.kv.evict(c.table, lengths, w, 64, target, recent=8, kept=out[1], new_lengths=out[0], new_weights=out[2], cuda_stream=stream)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    lengths.copy_(c.len_dev)
    w.copy_(random_weights(c, 10))
    graph.replay()
    torch.cuda.synchronize()
    want = decode.evict([w[s, :, :n].cpu().numpy() for s, n in enumerate(c.lengths)], c.lengths, 64, 8)
    assert out[0].tolist() == [64, 64] and out[1].tolist() == want
    side = torch.cuda.Stream()
    replayed = [t.clone() for t in out]
    torch.cuda.synchronize()
    for t in out:
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, replayed))
    c.kv.sync()


def test_refusals():
    c, to = filled("bf16", [40, 9], 2, 64, 16, 20, seed=10)
    w, target = random_weights(c, 10), torch.from_numpy(to).cuda()
    for kw in (dict(keep=0), dict(keep=20, recent=21), dict(keep=20, recent=-1), dict(keep=1 << 31),
               dict(keep=20, new_weights=w[:, :, :19]), dict(keep=20, kept=torch.zeros(2, 2, 19, dtype=torch.int32, device="cuda")),
               dict(keep=20, new_lengths=torch.zeros(3, dtype=torch.int32, device="cuda")), dict(keep=20, layer=1)):
        with pytest.raises(ValueError):
            c.kv.evict(c.table, c.len_dev, w, to=target, **kw)
    for weights, ln, to_bad in ((w.double(), c.len_dev, target), (w[:1], c.len_dev, target), (w, c.len_dev.long(), target), (w, c.len_dev, target.long()),
                                (w[:, :, ::2], c.len_dev, target)):
        with pytest.raises(ValueError):
            c.kv.evict(c.table, ln, weights, 20, to_bad)
    for to_bad in (target[:1], target[:, :1]):                       # too few sequences, too few pages
        with pytest.raises(L.LacacheError) as e:
            c.kv.evict(c.table, c.len_dev, w, 20, to_bad)
        assert e.value.status == L.LACACHE_ERR_INVALID_ARG
    # tables and weights in place, and rows that share memory
    wide = torch.zeros(2, 1, 64, device="cuda")
    for to_bad, new_weights in ((c.table, None), (target, w), (target, wide.expand(2, 2, 64)), (target, wide[:1].expand(2, 2, 64))):
        with pytest.raises(L.LacacheError) as e:
            c.kv.evict(c.table, c.len_dev, w, 20, to_bad, new_weights=new_weights)
        assert e.value.status == L.LACACHE_ERR_INVALID_ARG
    assert c.kv.evict(c.table[:0], c.len_dev[:0], w[:0], 20, target[:0])[1].shape == (0, 2, 20)
    c.kv.sync()


def test_decoding_goes_on_after_an_eviction():
    """Weights gathered over steps, an eviction, and tokens written and attended to behind what was kept."""
    c, to = filled("bf16", [120, 77], 2, 64, 16, 48, seed=11)
    q = torch.randn(2, 4, 64, device="cuda").bfloat16()
    lse = torch.empty(2, 4, device="cuda")
    c.kv.attend(q, c.table, c.len_dev, lse=lse)
    weights = c.kv.weigh(q, c.table, c.len_dev, lse)
    target = torch.cat((torch.from_numpy(to).cuda(), c.table.new_zeros(2, 1)), 1)
    target[:, 3] = torch.from_numpy(np.setdiff1d(np.arange(c.kv.cfg.pages), np.concatenate((to.ravel(), c.host_table.ravel())))[:2]).cuda()
    new_lengths, kept, new_weights = c.kv.evict(c.table, c.len_dev, weights, 48, target, recent=8)
    x = torch.randn(2, 2, 64, device="cuda").bfloat16()
    seq = torch.arange(2, dtype=torch.int32, device="cuda")
    rope = L.Rope(64)
    c.kv.append(x, x, seq, new_lengths, target, rope=rope, rope_pos=c.len_dev)
    out = c.kv.attend(q, target, new_lengths + 1)
    c.kv.sync()
    k, v = c.values()
    rows = [[np.stack([np.concatenate((src[s][kept[s, h].cpu().numpy(), h], extra[s, h][None])) for h in range(2)], 1) for s in range(2)]
            for src, extra in ((k, rope.apply(x, c.len_dev).double().cpu().numpy()), (v, x.double().cpu().numpy()))]
    want, _, mass, _ = decode.attend(q.double().cpu().numpy(), *rows, [49, 49], 1, 64 ** -0.5)
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -9 * mass)
    assert float(new_weights.sum()) <= float(weights.sum())


def test_lengths_are_not_written_over_themselves():
    c, to = filled("bf16", [40, 9, 30], 2, 64, 16, 20, seed=16)
    w, target = random_weights(c, 16), torch.from_numpy(to).cuda()
    store = torch.tensor([40, 9, 30, 0, 0, 0], dtype=torch.int32, device="cuda")
    starts = torch.zeros(3, dtype=torch.int32, device="cuda")
    for kw in (dict(new_lengths=store[:3]), dict(new_lengths=store[2:5]), dict(starts=starts, new_lengths=starts)):
        with pytest.raises(L.LacacheError) as e:
            c.kv.evict(c.table, store[:3], w, 20, target, **kw)
        assert e.value.status == L.LACACHE_ERR_INVALID_ARG
    new_lengths, _, _ = c.kv.evict(c.table, store[:3], w, 20, target, starts=starts, new_lengths=store[3:])
    assert new_lengths.tolist() == [20, 9, 20] and store[:3].tolist() == [40, 9, 30]
    c.kv.sync()
