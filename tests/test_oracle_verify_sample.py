"""Pins of verification by random numbers, and what its call refuses (no GPU)."""
import ctypes

import numpy as np
import pytest

import oracle
from oracle import HIT, MISS_KEY
from paper_2608_01718_gb300 import build
from paper_2608_01718_gb300 import lacache as L


def test_acceptance_and_the_refused_position():
    target = [[[0.5, 0.25, 0.25], [0.25, 0.25, 0.5], [0.25, 0.5, 0.25]]]
    draft = [[[0.25, 0.5, 0.25], [0.5, 0.25, 0.25]]]
    # token 0: u * 0.25 < 0.5 always; token 0 again: u * 0.5 < 0.25 for u < 0.5
    assert [int(x[0]) for x in oracle.verify_sample(target, draft, [[0, 0]], [[0.99, 0.25, 0.5]])] == [2, 1]
    # u = 0.5 is refused (not below); only token 2 has p > q there
    assert [int(x[0]) for x in oracle.verify_sample(target, draft, [[0, 0]], [[0.0, 0.5, 0.0]])] == [1, 2]
    # -1 ends the window: the token is drawn from p itself
    assert [int(x[0]) for x in oracle.verify_sample(target, draft, [[0, -1]], [[0.0, 0.0, 0.25]])] == [1, 1]


def test_ties_and_the_ends_of_the_draw():
    assert oracle.speculative.draw([1, 1, 1, 1], 0.5) == 2       # C_1 = 2 does not exceed 2
    assert oracle.speculative.draw([0, 0, 1, 0], 0.0) == 2
    assert oracle.speculative.draw([1, 0, 1, 0], 1.0) == 2       # none exceeds: the last of any weight
    assert oracle.speculative.draw([0, 0], 0.3) == -1


def test_likeliest_drafts_leave_themselves_out():
    target = [[[0.25, 0.5, 0.25], [1.0, 0.0, 0.0]]]
    assert [int(x[0]) for x in oracle.verify_sample(target, None, [[1]], [[0.5, 0.4]])] == [0, 0]
    assert [int(x[0]) for x in oracle.verify_sample(target, None, [[1]], [[0.5, 0.6]])] == [0, 2]
    assert [int(x[0]) for x in oracle.verify_sample(target, None, [[1]], [[0.4, 0.6]])] == [1, 0]


def test_served_queries_get_neither():
    target = np.full((2, 2, 4), 0.25)
    got = oracle.verify_sample(target, target[:, :1], [[1], [1]], np.zeros((2, 2)), [HIT, MISS_KEY])
    assert [x.tolist() for x in got] == [[-1, 1], [-1, 0]]


def test_the_pair_is_distributed_as_the_target():
    # one position, three tokens, every draft and a fine grid of random numbers: the emitted first token's distribution is p
    p, q = np.array([0.5, 0.125, 0.375], np.float32), np.array([0.25, 0.5, 0.25], np.float32)
    grid = (np.arange(64) + 0.5) / 64
    mass = np.zeros(3)
    for x in range(3):
        B = 64 * 64
        u = np.stack(np.meshgrid(grid, grid, indexing="ij"), -1).reshape(B, 2)
        n, token = oracle.verify_sample(np.broadcast_to(np.stack([p, p]), (B, 2, 3)), np.broadcast_to(q, (B, 1, 3)),
                                        np.full((B, 1), x), u)
        first = np.where(n == 1, x, token)
        mass += q[x] * np.bincount(first, minlength=3) / B
    assert np.abs(mass - p).max() <= 1 / 64


def test_refusals_need_no_device():
    build.build()
    lib, ref = L.load(), ctypes.addressof
    one = L.lacache_probs(256, 4, 2)
    none = L.lacache_probs(None, 4, 2)

    def call(B=1, k=1, vocab=2, target=one, draft=one, drafts=256, u=256, accepted=256, token=256):
        return lib.lacache_verify_sample(B, k, vocab, target and ref(target), draft and ref(draft), drafts, u, None, accepted,
                                         token, None)

    for bad in (dict(B=0), dict(B=-1), dict(k=-1), dict(k=257), dict(vocab=0), dict(target=None), dict(target=none),
                dict(draft=none), dict(drafts=None), dict(u=None), dict(accepted=None), dict(token=None)):
        assert call(**bad) == L.LACACHE_ERR_INVALID_ARG, bad
    assert call(vocab=(1 << 30) + 1) == L.LACACHE_ERR_UNSUPPORTED
    assert ctypes.sizeof(L.lacache_probs) == 24


@pytest.mark.parametrize("name", ["target", "u"])
def test_host_tensors_are_refused(name):
    import torch
    x = torch.zeros(1, 2, 4)
    with pytest.raises(ValueError):
        L.lacache_verify_sample(x, None, torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, 2), torch.zeros(1, dtype=torch.int32),
                                torch.zeros(1, dtype=torch.int32))


def test_outputs_over_each_other_or_the_inputs_are_refused():
    build.build()
    lib, ref = L.load(), ctypes.addressof
    rows = L.lacache_probs(1 << 20, 12, 4)
    good = dict(drafts=1024, u=2048, status=4096, accepted=8192, token=8192 + 12)      # three queries, two drafts

    def call(**kw):
        a = {**good, **kw}
        return lib.lacache_verify_sample(3, 2, 4, ref(rows), None, a["drafts"], a["u"], a["status"], a["accepted"], a["token"], None)

    for bad in (dict(token=8192), dict(token=8192 + 8), dict(accepted=1024), dict(accepted=1024 + 20), dict(token=1024 - 8),
                dict(token=2048 + 32), dict(accepted=4096), dict(token=4096 - 8)):
        assert call(**bad) == L.LACACHE_ERR_INVALID_ARG, bad
