"""The paged cache's write and read back: codes to the bit, values against the fp64 oracle, and what a call leaves alone."""
import ctypes

import numpy as np
import pytest
import torch

from kv_cases import Filled, TORCH
from oracle import decode
from paper_2608_01718_gb300 import build
from paper_2608_01718_gb300 import lacache as L

pytestmark = pytest.mark.gpu

TOP = {"e4m3": 448.0, "int8": 127.0}


@pytest.fixture(scope="module", autouse=True)
def library():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    build.build()
    L.load()


def codes(x, fmt):
    """Codes and scales of fp32 rows by IEEE fp32 division on the CPU."""
    with np.errstate(all="ignore"):
        scale = (np.abs(x).max(-1) / np.float32(TOP[fmt])).astype(np.float32)
        u = np.where(scale[..., None] > 0, x / scale[..., None], np.float32(0)).astype(np.float32)
    u = np.clip(u, -TOP[fmt], TOP[fmt])
    if fmt == "int8":
        return np.rint(u), scale
    return torch.from_numpy(u).to(torch.float8_e4m3fn).float().numpy(), scale


def placed(c, name, layer=None):
    """A pool's rows in the order of the cache's tokens, as fp32."""
    x = c.kv.pool(c.layer if layer is None else layer)[name].float().cpu().numpy()
    seq, pos = c.seq.cpu().numpy(), c.pos.cpu().numpy()
    return x[c.host_table[seq, pos // c.page], :, pos % c.page]


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("head_dim", [16, 48, 64, 128, 176, 256])
def test_codes_to_the_bit(fmt, dtype, head_dim):
    c = Filled(fmt, [5, 0, 33, 16], 3, head_dim, page=32, dtype=dtype, seed=head_dim)
    for name, rows in (("k", c.k_rows), ("v", c.v_rows)):
        want, scale = codes(rows.float().cpu().numpy(), fmt)
        assert np.array_equal(placed(c, name), want)
        assert np.array_equal(placed(c, name + "s"), scale)
        back = c.kv.read(c.seq, c.pos, c.table, dtype=torch.float32)[0 if name == "k" else 1].cpu().numpy()
        assert np.array_equal(back, (want * scale[..., None]).astype(np.float32))
    c.kv.sync()


@pytest.mark.parametrize("fmt", ["bf16", "f16"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_16_bit_formats_round_once(fmt, dtype):
    c = Filled(fmt, [20, 7], 2, 80, dtype=dtype, seed=2)
    for i, rows in enumerate((c.k_rows, c.v_rows)):
        want = rows.float().to(TORCH[fmt])
        assert np.array_equal(placed(c, "kv"[i]), want.float().cpu().numpy())
        for back in ("bf16", "f16", "f32"):
            got = c.kv.read(c.seq, c.pos, c.table, dtype=TORCH[back])[i]
            assert torch.equal(got, want.float().to(TORCH[back]))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_rows_at_the_edges(fmt):
    # zeros, one value, the largest and smallest magnitudes, ties, infinities and NaN
    c = Filled(fmt, [16], 1, 32, dtype="f32", seed=3)
    x = np.zeros((16, 1, 32), dtype=np.float32)
    x[1, 0, 5] = -2.5
    x[2] = 3.0e38
    x[3] = 1e-44
    x[4, 0] = np.arange(32) - 15.5
    x[5, 0, 0], x[5, 0, 1:9] = TOP[fmt], np.arange(8) + 0.5       # scale 1: halves tie to even
    x[6, 0, 3] = np.inf
    x[7, 0, 3] = -np.inf
    x[8, 0, 31] = np.nan
    x[9] = -0.0
    x[10, 0, 0], x[10, 0, 1] = 1.0, 2.0 ** -30
    x[11:] = np.random.default_rng(0).standard_normal((5, 1, 32))
    t = torch.from_numpy(x).cuda()
    c.kv.append(t, t, c.seq, c.pos, c.table)
    c.kv.sync()
    fine = [i for i in range(16) if i not in (6, 7, 8)]
    want, scale = codes(x[fine], fmt)
    for name in "kv":
        assert np.array_equal(placed(c, name)[fine], want) and np.array_equal(placed(c, name + "s")[fine], scale)
        assert np.isnan(placed(c, name + "s")[[6, 7, 8]]).all() and not placed(c, name)[[6, 7, 8]].any()
    back = c.kv.read(c.seq, c.pos, c.table, dtype=torch.float32)[0].cpu().numpy()
    assert np.isnan(back[[6, 7, 8]]).all() and np.isfinite(back[fine]).all() and not back[[0, 9]].any()
    # half a step: relative to the value (e4m3, 3 bits after the point) or to the largest (int8)
    err = np.abs(back[fine].astype(np.float64) - x[fine])
    step = 2.0 ** -4 * np.abs(x[fine].astype(np.float64)) if fmt == "e4m3" else 0.0
    least = scale.astype(np.float64)[..., None] * (2.0 ** -10 if fmt == "e4m3" else 0.5)
    normal = scale >= 2.0 ** -126     # a subnormal scale is itself rounded coarsely
    assert np.all((err <= np.maximum(step, least) * (1 + 2.0 ** -10))[normal])


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("interleaved,rot,head_dim", [(False, 128, 128), (True, 64, 128), (False, 32, 80), (True, 256, 256),
                                                      (False, 20, 64)])
def test_rotation_and_write_in_one_pass(fmt, interleaved, rot, head_dim):
    c = Filled(fmt, [9, 21], 2, head_dim, seed=rot)
    rope = L.Rope(rot, interleaved=interleaved, scaling="linear", factor=2.0, amplitude=1.25)
    n = 30
    qkv = torch.randn(n, 9, head_dim, device="cuda").bfloat16()
    q, k, v = qkv[:, :5], qkv[:, 5:7], qkv[:, 7:]
    at = (c.pos + 1000).to(torch.int32)
    rotated = c.kv.append(k, v, c.seq, c.pos, c.table, rope=rope, rope_pos=at, q=q)
    assert torch.equal(rotated, rope.apply(q, at))
    got_k, got_v = c.kv.read(c.seq, c.pos, c.table, dtype=torch.float32)
    freq = decode.rope_frequencies(rot, scaling="linear", factor=2.0)
    want = decode.rotate(k.double().cpu().numpy(), at.cpu().numpy(), freq, interleaved, 1.25)
    top = np.abs(want).max(-1, keepdims=True)
    # half a step of the format, and the rotation's own error
    step = {"bf16": 2.0 ** -8 * np.abs(want), "int8": top / 127 * 0.5, "e4m3": np.maximum(2.0 ** -4 * np.abs(want), top / 448 * 2.0 ** -10)}[fmt]
    assert np.all(np.abs(got_k.double().cpu().numpy() - want) <= step * (1 + 2.0 ** -9) + 2.0 ** -18 * top)
    plain = Filled(fmt, [9, 21], 2, head_dim, seed=rot)
    plain.kv.append(k, v, plain.seq, plain.pos, plain.table)
    assert torch.equal(got_v, plain.kv.read(plain.seq, plain.pos, plain.table, dtype=torch.float32)[1])
    # positions of the cache where no others are given; in place; no q
    c.kv.append(k, v, c.seq, c.pos, c.table, rope=rope)
    want = rope.apply(q, c.pos)
    c.kv.append(k, v, c.seq, c.pos, c.table, rope=rope, q=q, q_out=q)
    assert torch.equal(q, want)
    # without a rotation q is copied
    assert torch.equal(c.kv.append(k, v, c.seq, c.pos, c.table, q=q), q)
    c.kv.sync()


def test_only_the_named_slots_change():
    c = Filled("e4m3", [40, 20], 2, 64, layers=2, layer=1, seed=5)
    before = [{n: t.view(torch.uint8).clone() for n, t in c.kv.pool(i).items()} for i in range(2)]
    k = torch.randn(4, 2, 64, device="cuda").bfloat16()
    seq = torch.tensor([0, -1, 1, 0], dtype=torch.int32, device="cuda")      # one token skipped
    pos = torch.tensor([17, 3, 19, 39], dtype=torch.int32, device="cuda")
    q = torch.zeros(4, 1, 64, device="cuda").bfloat16()
    q_out = torch.full_like(q, 7.0)
    c.kv.append(k, k, seq, pos, c.table, layer=1, q=q, q_out=q_out)
    c.kv.sync()
    assert float(q_out[1].min()) == 7.0 and float(q_out[[0, 2, 3]].abs().max()) == 0.0
    for i in range(2):
        for name, t in c.kv.pool(i).items():
            same = (t.view(torch.uint8) == before[i][name]).view(t.shape[0], 2, 16, -1).all(-1).all(1)
            changed = {(int(a), int(b)) for a, b in (~same).nonzero().cpu()}
            named = {(int(c.host_table[s, p // 16]), p % 16) for s, p in ((0, 17), (1, 19), (0, 39))} if i == 1 else set()
            assert changed <= named and (name in ("ks", "vs") or changed == named)


def test_bad_places_are_skipped_and_reported():
    c = Filled("int8", [40], 1, 64, seed=6)
    before = c.kv.pool()["k"].clone()
    k = torch.randn(1, 1, 64, device="cuda").bfloat16()
    out = torch.full((1, 1, 64), 3.0, device="cuda").bfloat16()
    i32 = dict(dtype=torch.int32, device="cuda")
    width = c.table.shape[1]
    for seq, pos in [(1, 0), (-2, 0), (0, -1), (0, 16 * width), (0, 2 ** 31 - 1), (0, 16 * (width - 1))]:   # the last page id is no page
        s, p = torch.tensor([seq], **i32), torch.tensor([pos], **i32)
        c.kv.append(k, k, s, p, c.table)
        with pytest.raises(L.LacacheError) as e:
            c.kv.sync()
        assert e.value.status == L.LACACHE_ERR_INVALID_ARG
        c.kv.read(s, p, c.table, k_out=out)
        with pytest.raises(L.LacacheError):
            c.kv.sync()
    c.kv.sync()
    assert torch.equal(c.kv.pool()["k"], before) and float(out.min()) == 3.0


def test_strided_rows_and_one_output():
    c = Filled("f16", [30, 18], 3, 64, seed=7)
    heads_first = torch.zeros(3, 48, 72, device="cuda", dtype=torch.float16)
    k, v = c.kv.read(c.seq, c.pos, c.table, dtype=torch.float16)
    got, none = c.kv.read(c.seq, c.pos, c.table, k_out=heads_first.transpose(0, 1)[:, :, 8:])
    assert none is None and torch.equal(got, k) and not heads_first[:, :, :8].any()
    other = Filled("f16", [30, 18], 3, 64, seed=8)
    other.kv.append(heads_first.transpose(0, 1)[:, :, 8:], v.flip(0).flip(0), other.seq, other.pos, other.table)
    again = other.kv.read(other.seq, other.pos, other.table, dtype=torch.float16)
    assert torch.equal(again[0], k) and torch.equal(again[1], v)


def test_no_tokens_and_many():
    c = Filled("bf16", [1], 1, 16, seed=9)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    rows = torch.empty(0, 1, 16, device="cuda").bfloat16()
    c.kv.append(rows, rows, none, none, c.table)
    c.kv.read(none, none, c.table)
    big = Filled("bf16", [70_000], 1, 16, page=64, seed=10)       # more tokens than a grid's blocks
    back = big.kv.read(big.seq, big.pos, big.table)
    assert torch.equal(back[0], big.k_rows) and torch.equal(back[1], big.v_rows)
    big.kv.sync()


def test_written_under_a_graph_and_on_a_side_stream():
    c = Filled("e4m3", [33, 20], 2, 64, seed=11)
    rope = L.Rope(64)
    k, q = torch.randn(53, 2, 64, device="cuda").bfloat16(), torch.randn(53, 4, 64, device="cuda").bfloat16()
    want_q = c.kv.append(k, k, c.seq, c.pos, c.table, rope=rope, q=q).clone()
    want = c.kv.read(c.seq, c.pos, c.table)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got_q = c.kv.append(k, k, c.seq, c.pos, c.table, rope=rope, q=q)
        got = c.kv.read(c.seq, c.pos, c.table)
    c.poison(0)
    graph.replay()
    assert torch.equal(got_q, want_q) and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_refusals():
    lib = L.load()
    c = Filled("bf16", [20], 2, 64, seed=12)
    x = torch.randn(20, 2, 64, device="cuda").bfloat16()
    ok = L.lacache_rows(x.data_ptr(), 128, 64)
    off = L.lacache_rows(x.data_ptr() + 2, 128, 64)
    odd = L.lacache_rows(x.data_ptr(), 129, 64)
    table = L.lacache_kv_table(c.table.data_ptr(), c.table.stride(0), 1, c.table.shape[1])
    wide = L.Rope(96).plan
    ref = ctypes.addressof

    def append(layer=0, t=table, n=20, seq=c.seq.data_ptr(), pos=c.pos.data_ptr(), rope=None, dtype=0, k=ok, v=ok, heads=0,
               q=None, q_out=None, h=c.kv.h):
        return lib.lacache_kv_append(h, layer, ref(t), n, seq, pos, rope, None, dtype, ref(k) if k else None,
                                     ref(v) if v else None, heads, q, q_out, None)

    bad = L.LACACHE_ERR_INVALID_ARG
    for kw in [dict(h=None), dict(layer=1), dict(n=-1), dict(seq=None), dict(pos=None), dict(dtype=5), dict(k=None), dict(v=None),
               dict(k=off), dict(v=odd), dict(heads=2, q=ref(ok)), dict(heads=0, q=ref(ok), q_out=ref(ok)),
               dict(heads=2, q=ref(off), q_out=ref(ok)), dict(rope=ref(wide)),
               dict(t=L.lacache_kv_table(None, 4, 1, 4)), dict(t=L.lacache_kv_table(c.table.data_ptr(), 4, 1, 0))]:
        assert append(**kw) == bad, kw
    assert append(n=0, k=None) == L.LACACHE_OK
    assert lib.lacache_kv_read(c.kv.h, 0, ref(table), 20, None, c.pos.data_ptr(), 0, ref(ok), None, None) == bad
    assert lib.lacache_kv_read(c.kv.h, 0, ref(table), 20, c.seq.data_ptr(), c.pos.data_ptr(), 7, ref(ok), None, None) == bad
    assert lib.lacache_kv_read(c.kv.h, 0, ref(table), 20, c.seq.data_ptr(), c.pos.data_ptr(), 0, ref(off), None, None) == bad
    assert lib.lacache_kv_read(c.kv.h, 2, ref(table), 20, c.seq.data_ptr(), c.pos.data_ptr(), 0, ref(ok), None, None) == bad
    pool = L.lacache_kv_pool()
    assert lib.lacache_kv_get_pool(c.kv.h, -1, ctypes.byref(pool)) == bad
    for kw in [dict(k=x.float()), dict(k=x[:, :1]), dict(v=x[:10]), dict(seq=c.seq.long()), dict(pos=c.pos[:5]),
               dict(table=c.table.cpu()), dict(q=x.float()), dict(rope_pos=c.pos[:1]), dict(k=x.cpu())]:
        args = dict(k=x, v=x, seq=c.seq, pos=c.pos, table=c.table)
        args.update(kw)
        with pytest.raises((ValueError, L.LacacheError)):
            c.kv.append(**args)
    c.kv.sync()
