"""The decoding calls' arguments: what is refused, numbers at the edges, streams and gradients."""
import ctypes

import pytest
import torch

from kv_cases import Filled
from paper_2608_01718_gb300 import build
from paper_2608_01718_gb300 import lacache as L

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    build.build()
    L.load()


def test_outputs_over_the_queries_are_refused():
    # the many-row kernel may read a row of q again after it has written that row of out
    c = Filled("bf16", [40], 1, 64, seed=33)
    for new in (1, 20):
        q = torch.randn(new, 1, 64, device="cuda").bfloat16()
        kept = q.clone()
        with pytest.raises(L.LacacheError) as e:
            c.kv.attend(q, c.table, c.len_dev, new_tokens=new, out=q)
        assert e.value.status == L.LACACHE_ERR_INVALID_ARG and torch.equal(q, kept)
    c.kv.sync()


def test_numbers_past_32_bits_are_refused_or_mean_what_they_say():
    # a window of 2^32 + 5 is no window of 5
    c = Filled("bf16", [40], 1, 64, seed=35)
    q = torch.randn(1, 1, 64, device="cuda").bfloat16()
    want = c.kv.attend(q, c.table, c.len_dev)
    for window in ((1 << 32) + 5, 1 << 31, 1 << 62):
        assert torch.equal(c.kv.attend(q, c.table, c.len_dev, window=window), want)
    for window in (-1, -(1 << 32) + 5):
        with pytest.raises((ValueError, L.LacacheError)):
            c.kv.attend(q, c.table, c.len_dev, window=window)
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    for layer in (1 << 32, -(1 << 32)):
        with pytest.raises((ValueError, L.LacacheError)):
            c.kv.attend(q, c.table, c.len_dev, layer=layer)
        with pytest.raises((ValueError, L.LacacheError)):
            c.kv.append(q, q, one, one, c.table, layer=layer)
        with pytest.raises((ValueError, L.LacacheError)):
            c.kv.read(one, one, c.table, layer=layer)
        with pytest.raises((ValueError, L.LacacheError)):
            c.kv.pool(layer)
    c.kv.sync()


class Slow:
    """Work for the current stream that takes some ten milliseconds."""

    def __init__(self):
        self.x = torch.randn(4096, 4096, device="cuda")

    def __call__(self):
        for _ in range(20):
            self.x @ self.x


@pytest.mark.parametrize("call", ["rotate", "append", "read", "attend"])
def test_results_made_on_another_stream_take_no_memory_of_this_one(call):
    """A call on a given stream allocates its result from that stream's memory: a block that was freed while the current stream still
    works on it must not be written from the other."""
    c = Filled("bf16", [500] * 8, 32, 64, seed=36)           # results of 16 MB: a block of memory of their own
    x = torch.randn(4000, 32, 64, device="cuda").bfloat16()
    rope, at = L.Rope(64), torch.arange(4000, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    slow = Slow()

    def run(stream):
        if call == "rotate":
            return rope.apply(x, at, cuda_stream=stream)
        if call == "append":
            return c.kv.append(x, x, c.seq, c.pos, c.table, q=x, cuda_stream=stream)
        if call == "read":
            return c.kv.read(c.seq, c.pos, c.table, cuda_stream=stream)[0]
        return c.kv.attend(x, c.table, c.len_dev, new_tokens=500, cuda_stream=stream)

    for stream in (side, side.cuda_stream):
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        old = torch.full((4000, 32, 64), 3.0, device="cuda", dtype=torch.bfloat16)
        kept = torch.empty_like(old)
        torch.cuda.synchronize()
        slow()
        kept.copy_(old)              # queued behind the slow work
        where = old.data_ptr()
        del old
        got = run(stream)
        assert got.data_ptr() != where
        torch.cuda.synchronize()
        assert float(kept.float().min()) == 3.0 == float(kept.float().max())
        assert torch.equal(got, run(None))
    c.kv.sync()


def test_a_lookup_on_another_stream_allocates_there():
    x = torch.nn.functional.normalize(torch.randn(4, 64, device="cuda"), dim=-1).bfloat16()
    ids = torch.zeros(4, 8, dtype=torch.int32, device="cuda")
    with L.LaCache(d=64, k=8, capacity=64, tau_c=0.9, tau_a=0.8, top_c=2, max_batch=4) as cache:
        cache.insert(x, x, ids)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        for stream, handle in ((side, side.cuda_stream), (side.cuda_stream, side.cuda_stream), (0, 0), (None, 0)):
            out = cache.lookup(x, x, ids, cuda_stream=stream)
            torch.cuda.synchronize()
            at = out["entry_id"].data_ptr()
            (where,) = [s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] <= at < s["address"] + s["total_size"]]
            assert where == handle and out["entry_id"].tolist() == [0, 1, 2, 3]


def test_autograd_goes_through_the_rotation():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    pos = torch.arange(100, 107, dtype=torch.int32, device="cuda")
    for rope in (L.Rope(32, interleaved=True, amplitude=1.5), L.Rope(48), L.Rope(20)):
        for inverse in (False, True):
            x, g = (torch.randn(7, 3, 64, generator=gen, device="cuda") for _ in range(2))
            x.requires_grad_(True)
            y = rope.apply(x, pos, inverse=inverse)
            with torch.no_grad():
                plain = rope.apply(x, pos, inverse=inverse)
                want = rope.apply(g, pos, inverse=not inverse)
            assert y.requires_grad and not plain.requires_grad and torch.equal(y, plain)
            (got,) = torch.autograd.grad(y, x, g)
            assert torch.equal(got, want)
            # against differences: f(x) = <g, y> is linear
            d = torch.randn(7, 3, 64, generator=gen, device="cuda")
            with torch.no_grad():
                up, down = ((g.double() * rope.apply(x + e * 0.5 * d, pos, inverse=inverse).double()).sum() for e in (1, -1))
            assert abs(float(up - down) - float((got.double() * d.double()).sum())) < 1e-4


def test_autograd_of_shared_and_strided_rows():
    # a gradient that autograd expands (a sum's: strides of zero), and a leaf that is used twice
    rope, pos = L.Rope(64), torch.arange(5, dtype=torch.int32, device="cuda")
    x = torch.randn(5, 2, 64, device="cuda").bfloat16().requires_grad_(True)
    (rope.apply(x, pos).float().sum() + rope.apply(x, pos, inverse=True).float().sum()).backward()
    ones = torch.ones(5, 2, 64, device="cuda").bfloat16()
    want = rope.apply(ones, pos, inverse=True).float() + rope.apply(ones, pos).float()
    assert torch.allclose(x.grad.float(), want, atol=2 ** -6)
    stored = torch.empty(5, 2, 64, device="cuda").bfloat16()
    for out in (stored, x):          # autograd cannot follow a given output
        with pytest.raises(ValueError):
            rope.apply(x, pos, out=out)
    with torch.no_grad():
        rope.apply(x, pos, out=stored)


def test_counts_of_query_heads_past_32_bits():
    c = Filled("bf16", [16], 1, 64, seed=37)
    lib, ref = L.load(), ctypes.addressof
    rows = L.lacache_rows(c.k_rows.data_ptr(), 64, 64)
    table = L.lacache_kv_table(c.table.data_ptr(), c.table.stride(0), 1, c.table.shape[1])
    for heads, n, want in (((1 << 31) - 1, 16, L.LACACHE_ERR_UNSUPPORTED), ((1 << 30) + 1, 16, L.LACACHE_ERR_UNSUPPORTED),
                           (1 << 30, 0, L.LACACHE_OK)):
        assert lib.lacache_kv_append(c.kv.h, 0, ref(table), n, c.seq.data_ptr(), c.pos.data_ptr(), None, None, L.LACACHE_BF16,
                                     ref(rows), ref(rows), heads, ref(rows), ref(rows), None) == want
    c.kv.sync()
