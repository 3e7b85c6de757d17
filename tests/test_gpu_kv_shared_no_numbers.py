"""Shared prefixes that hold keys, values or scales that are no finite numbers, in any of a block's units: rows that do not see them
are what they were, rows that do are as the ordinary attention gives them."""
import numpy as np
import pytest
import torch

from test_gpu_kv_shared import filled, ints, library, queries  # noqa: F401 (the fixture)
from kv_cases import TORCH, bounds as tolerances
from oracle import decode

pytestmark = pytest.mark.gpu

FORMATS = [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16"), ("int8", "f16")]
CUT = [(700, [720 + 3 * i for i in range(8)])]
WHOLE = [(680 + i % 3, [700 + (i * 7 + s) % 40 for s in range(4)]) for i in range(20)]


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("groups,kv_heads,head_dim", [(CUT, 2, 128), (WHOLE, 4, 64)], ids=["cut", "whole"])
@pytest.mark.parametrize("at", [3, 300, 660])
@pytest.mark.parametrize("what", ["k", "v", "both"])
def test_rows_that_do_not_see_them(fmt, dtype, groups, kv_heads, head_dim, at, what):
    new, q_heads = 2, 4 * kv_heads
    c = filled(fmt, groups, kv_heads, head_dim, seed=41)
    q = queries(c, dtype, q_heads, new)
    B = len(c.lengths)
    starts = [at + 1 if s % 2 else 0 for s in range(B)]      # (a sequence of every group sees it, another does not)
    kw = dict(new_tokens=new, starts=ints(starts))
    k, v = c.values()
    f, hq = head_dim ** -0.5, q.double().cpu().numpy()
    want, want_lse, mass, span = decode.attend(hq, k, v, c.lengths, new, f, starts)
    tol, tol_lse = tolerances(want, mass, span, want_lse, hq, k, f, dtype)
    blind = np.repeat(np.arange(B) % 2 == 1, new)
    firsts, where = ints([c.bounds[g] for g in range(len(groups))]), ints([at] * len(groups))
    old = c.kv.read(firsts, where, c.table, dtype=TORCH[dtype])
    for value in (float("nan"), float("inf"), float("-inf")):
        bad = torch.randn(len(groups), kv_heads, head_dim, device="cuda").to(TORCH[dtype])
        bad[..., ::head_dim if what == "k" else 5] = value
        c.kv.append(bad if what != "v" else old[0], bad if what != "k" else old[1], firsts, where, c.table)
        out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        c.kv.attend_shared(q, c.table, c.len_dev, ints(c.common), bounds=ints(c.bounds), out=out, lse=lse, **kw)
        plain = c.kv.attend(q, c.table, c.len_dev, **kw)
        c.kv.sync()
        got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        assert np.all(np.abs(got[blind] - want[blind]) <= tol[blind])
        assert np.all(np.abs(got_lse[blind] - want_lse[blind]) <= tol_lse[blind])
        seen, theirs = out[~torch.from_numpy(blind)], plain[~torch.from_numpy(blind)]
        assert torch.equal(torch.isnan(seen), torch.isnan(theirs)) and torch.equal(torch.isposinf(seen), torch.isposinf(theirs))
        assert torch.equal(torch.isneginf(seen), torch.isneginf(theirs)) and not bool(torch.isfinite(theirs).all())
