"""Attention over shared prefixes, the weights of its tokens, eviction by them and attention over what is left: one after another,
eager and as replays of two captured graphs, against the fp64 oracle of each step."""
import numpy as np
import pytest
import torch

import test_gpu_kv_shared as shared
import test_gpu_kv_weigh as weigh
from kv_cases import bounds as tolerances
from oracle import decode
from paper_2608_01718_gb300 import build
from paper_2608_01718_gb300 import lacache as L

pytestmark = pytest.mark.gpu
GROUPS = [(300, [301, 417, 300, 340]), (64, [90]), (33, [50, 60, 70, 34])]
KEEP, RECENT = 80, 16


@pytest.fixture(scope="module", autouse=True)
def library():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    build.build()
    L.load()


class Chain:
    """The four calls on tensors that stay; `run` can be captured."""

    def __init__(self, fmt, dtype, kv_heads, q_heads, head_dim, new, small=False):
        pages = -(-KEEP // 16)
        n = sum(len(ns) for _, ns in GROUPS)
        self.c = c = shared.filled(fmt, GROUPS, kv_heads, head_dim, seed=head_dim, small=small, spare=pages * n + 1)
        taken = {int(p) for s, m in enumerate(c.lengths) for p in c.host_table[s, :-(-m // 16)]}
        self.to = np.array([p for p in range(c.kv.cfg.pages) if p not in taken][:n * pages], dtype=np.int32).reshape(n, pages)
        self.to_dev = torch.from_numpy(self.to).cuda()
        self.new, self.dtype, self.q_heads = new, dtype, q_heads
        self.bounds, self.common = shared.ints(c.bounds), shared.ints(c.common)
        self.q = shared.queries(c, dtype, q_heads, new, seed=5)
        self.lse = torch.empty(self.q.shape[:2], device="cuda")
        self.past = torch.rand(n, kv_heads, max(c.lengths) + 5, device="cuda") * 0.1
        self.weights = torch.zeros_like(self.past)

    def run(self):
        c = self.c
        self.out = c.kv.attend_shared(self.q, c.table, c.len_dev, self.common, bounds=self.bounds, new_tokens=self.new, lse=self.lse)
        c.kv.weigh(self.q, c.table, c.len_dev, self.lse, weights=self.past, decay=0.5, out=self.weights, new_tokens=self.new)
        self.lengths, self.kept, self.kept_weights = c.kv.evict(c.table, c.len_dev, self.weights, KEEP, self.to_dev, recent=RECENT)
        self.after = c.kv.attend(self.q, self.to_dev, self.lengths, new_tokens=self.new)

    def check(self):
        c, new = self.c, self.new
        c.kv.sync()
        f = c.kv.cfg.head_dim ** -0.5
        k, v = c.values()
        hq, hl = self.q.double().cpu().numpy(), self.lse.double().cpu().numpy()
        want, want_lse, mass, span = decode.attend(hq, k, v, c.lengths, new, f)
        tol, tol_lse = tolerances(want, mass, span, want_lse, hq, k, f, self.dtype)
        assert np.all(np.abs(self.out.double().cpu().numpy() - want) <= tol) and np.all(np.abs(hl - want_lse) <= tol_lse)
        past, got = self.past.cpu().numpy(), self.weights.double().cpu().numpy()
        parts = decode.weigh(hq, k, c.lengths, new, f, hl, past, 0.5)
        rows = new * self.q_heads // c.kv.cfg.kv_heads
        for s, n in enumerate(c.lengths):
            tol = weigh.tolerance(c, hq[s * new:(s + 1) * new], k[s], hl, parts[s], past, 0.5, f, rows)
            assert np.all(np.abs(got[s, :, :n] - parts[s][0]) <= tol)
        # what is kept, by the weights as they are
        kept = decode.evict([got[s, :, :n] for s, n in enumerate(c.lengths)], c.lengths, KEEP, RECENT)
        sizes = [len(rows[0]) for rows in kept]
        assert self.lengths.tolist() == sizes
        for s, rows in enumerate(kept):
            assert self.kept[s, :, :sizes[s]].tolist() == rows
        # and the attention over it: a head's tokens are those it kept, in order
        few = [[np.stack([x[s][rows[h], h] for h in range(len(rows))], 1) for s, rows in enumerate(kept)] for x in (k, v)]
        want, want_lse, mass, span = decode.attend(hq, few[0], few[1], sizes, new, f)
        tol, _ = tolerances(want, mass, span, want_lse, hq, few[0], f, self.dtype)
        assert np.all(np.abs(self.after.double().cpu().numpy() - want) <= tol)


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("kv_heads,q_heads,head_dim,new", [(2, 8, 64, 1), (1, 4, 128, 17), (2, 2, 256, 2)])
def test_one_after_another(fmt, dtype, kv_heads, q_heads, head_dim, new):
    for small in (False, True):
        chain = Chain(fmt, dtype, kv_heads, q_heads, head_dim, new, small)
        chain.run()
        chain.check()


def test_two_graphs_in_turn():
    """Two captured chains of different sizes, replayed in turn and both again with other queries and lengths."""
    chains = [Chain("e4m3", "bf16", 2, 8, 128, 3), Chain("bf16", "bf16", 1, 8, 64, 1)]
    graphs = []
    for chain in chains:
        chain.run()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            chain.run()
    for turn in range(3):
        for chain, graph in zip(chains, graphs):
            if turn:
                c = chain.c
                chain.q.copy_(shared.queries(c, chain.dtype, chain.q_heads, chain.new, seed=20 + turn))
                c.lengths = [n - 1 if n > 300 else n for n in c.lengths]
                c.len_dev.copy_(shared.ints(c.lengths))
            graph.replay()
        for chain in chains:
            chain.check()
