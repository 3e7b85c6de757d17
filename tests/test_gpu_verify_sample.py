"""Verification by given random numbers against the oracle's exact rational arithmetic: whole numbers, which must agree.

The drawn token depends on cumulative weights that the kernel holds to within 2^-40 of their total. With at most 10^5 tokens
and u of 24 bits, fewer than one seeded draw in 2^20 could meet a border that near."""
import numpy as np
import pytest
import torch

import oracle
from paper_2608_01718_gb300 import build
from paper_2608_01718_gb300 import lacache as L

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def library():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    build.build()
    L.load()


def inputs(B, k, V, seed, spread=2.5, likeliest=False):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    logits = torch.randn(B, k + 1, V, generator=gen, device="cuda") * spread
    target = torch.softmax(logits, -1)
    draft = torch.softmax(logits[:, :k] + 0.5 * torch.randn(B, k, V, generator=gen, device="cuda"), -1)
    if likeliest:
        drafts = draft.argmax(-1).int()
    else:
        at = torch.rand(B, k, 1, generator=gen, device="cuda")
        drafts = (draft.cumsum(-1) <= at).sum(-1).clamp(max=V - 1).int()
    return target, None if likeliest else draft, drafts.view(B, k), torch.rand(B, k + 1, generator=gen, device="cuda")


def call(target, draft, drafts, u, status=None, stream=None):
    accepted = torch.full((target.shape[0],), -7, dtype=torch.int32, device="cuda")
    token = torch.full_like(accepted, -7)
    L.lacache_verify_sample(target, draft, drafts, u, accepted, token, status=status, cuda_stream=stream)
    return accepted, token


def host(*tensors):
    return [None if t is None else t.cpu().numpy() for t in tensors]


def check(target, draft, drafts, u, status=None):
    got = call(target, draft, drafts, u, status)
    torch.cuda.synchronize()
    want = oracle.verify_sample(*host(target, draft, drafts, u, status))
    assert got[0].tolist() == want[0].tolist()
    assert got[1].tolist() == want[1].tolist()
    return want


@pytest.mark.parametrize("likeliest", [False, True])
@pytest.mark.parametrize("B,k,V", [(1, 0, 1), (1, 1, 1), (3, 2, 2), (5, 1, 31), (2, 31, 32), (4, 32, 33), (2, 33, 257),
                                   (300, 3, 300), (9, 5, 2047), (7, 5, 2048), (3, 4, 8193), (40, 6, 5000), (2, 2, 100_003),
                                   (3, 256, 40)])
def test_against_the_oracle(B, k, V, likeliest):
    accepted, _ = check(*inputs(B, k, V, seed=B + k + V, likeliest=likeliest))
    if B >= 40:
        assert accepted.min() == 0 and accepted.max() >= (1 if likeliest else 2)


def test_more_queries_than_clusters_of_one():
    check(*inputs(1500, 1, 64, seed=5))
    check(*inputs(700, 1, 4000, seed=6, spread=0.5))


@pytest.mark.parametrize("V", [50, 4096, 30_001])
def test_borders_that_are_exact(V):
    """Uniform target, a dyadic u: C_i = u C exactly, which is not past it; and the two ends."""
    n = 1 << (V.bit_length() - 1)
    target = torch.zeros(6, 1, V, device="cuda")
    target[:, :, :n] = 1.0 / n
    target[5, 0, :] = 0.0
    u = torch.tensor([[0.0], [0.5], [0.25], [1 - 2.0 ** -24], [1.0], [0.5]], device="cuda")
    _, token = check(target, None, torch.zeros(6, 0, dtype=torch.int32, device="cuda"), u)
    assert token.tolist() == [0, n // 2, n // 4, n - 1, n - 1, -1]


def test_acceptance_at_the_border():
    # u q against p where fp32's product would round onto p
    p, q, u = np.float32(0.3), np.float32(0.6000001), np.float32(0.49999994)
    target = torch.tensor([[[float(p), 0.7], [1.0, 0.0]]] * 3, device="cuda")
    draft = torch.tensor([[[float(q), 0.4]]] * 3, device="cuda")
    us = torch.tensor([[float(u), 0.0], [0.5, 0.0], [float(np.nextafter(u, np.float32(0))), 0.0]], device="cuda")
    check(target, draft, torch.zeros(3, 1, dtype=torch.int32, device="cuda"), us)


def test_refusals_that_leave_no_weight_draw_from_the_target():
    same = torch.full((2, 1, 8), 0.125, device="cuda")
    target = torch.cat((same, same), 1).contiguous()
    target[1] = 0.0
    draft = same * 2                                     # p - q is nowhere positive
    drafts = torch.full((2, 1), 3, dtype=torch.int32, device="cuda")
    u = torch.tensor([[0.75, 0.5], [0.75, 0.5]], device="cuda")
    accepted, token = check(target, draft, drafts, u)
    assert accepted.tolist() == [0, 0] and token.tolist() == [4, -1]


def test_small_differences_of_large_rows():
    """p and q agree but for their last bits: the weights are some 2^-24 of the row, and still those of the real numbers."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(11)
    target = torch.softmax(torch.randn(4, 2, 50_000, generator=gen, device="cuda"), -1)
    bits = target[:, :1].contiguous().view(torch.int32)
    draft = (bits + torch.randint(-2, 3, bits.shape, generator=gen, device="cuda", dtype=torch.int32)).view(torch.float32)
    drafts = (draft > target[:, :1]).int().argmax(-1).int()           # a draft that can be refused
    u = torch.full((4, 2), 1 - 2.0 ** -24, device="cuda")
    u[:, 1] = torch.tensor([0.1, 0.4, 0.7, 0.99], device="cuda")
    accepted, _ = check(target, draft, drafts, u)
    assert accepted.tolist() == [0] * 4


def test_windows_that_end_early_and_served_queries():
    target, draft, drafts, u = inputs(40, 7, 500, seed=8)
    drafts[::3, 2:] = -1
    drafts[1::3, 4] = 500
    drafts[2::9, 0] = -(1 << 31)
    status = torch.randint(0, 3, (40,), dtype=torch.uint8, device="cuda")
    accepted, token = check(target, draft, drafts, u, status)
    served = status.cpu().numpy() == L.LACACHE_HIT
    assert (accepted[served] == -1).all() and (token[served] == -1).all()


def test_numbers_that_are_none_have_no_weight():
    target, draft, drafts, u = inputs(12, 1, 3000, seed=9)
    target[:, :, ::7] = float("nan")
    draft[:, :, ::11] = float("nan")
    check(target, draft, drafts, u)


def test_strided_probabilities():
    target, draft, drafts, u = inputs(6, 4, 1001, seed=10)
    wide = torch.full((5, 6, 1003), float("nan"), device="cuda")      # positions first, rows apart and off 16 bytes
    wide[:, :, 1:1002] = target.transpose(0, 1)
    thin = torch.full((6, 9, 1001), float("nan"), device="cuda")
    thin[:, ::2][:, :4] = draft
    views = wide[:, :, 1:1002].transpose(0, 1), thin[:, ::2][:, :4]
    assert [x.tolist() for x in call(*views, drafts, u)] == [x.tolist() for x in call(target, draft, drafts, u)]
    check(target, draft, drafts, u)


def test_rows_past_32_bits():
    """A query whose rows lie beyond 2^31 elements."""
    V = 1 << 20
    flat = torch.empty((1 << 31) + 4 * V, device="cuda")
    target = flat.as_strided((2, 2, V), ((1 << 31) + V, V, 1))
    target.zero_()
    target[1, 0, V - 3] = 1.0
    target[0, 0, 5] = 1.0
    drafts = torch.tensor([[6], [V - 4]], dtype=torch.int32, device="cuda")
    accepted, token = call(target, None, drafts, torch.full((2, 2), 0.5, device="cuda"))
    assert accepted.tolist() == [0, 0] and token.tolist() == [5, V - 3]


def test_capture_and_another_stream():
    target, draft, drafts, u = inputs(20, 5, 2500, seed=12)
    want = call(target, draft, drafts, u)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = call(target, draft, drafts, u, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    accepted, token = torch.empty_like(want[0]), torch.empty_like(want[1])
    with torch.cuda.graph(graph):
        L.lacache_verify_sample(target, draft, drafts, u, accepted, token)
    other = inputs(20, 5, 2500, seed=13)
    for a, b in zip((target, draft, drafts, u), other):
        a.copy_(b)
    graph.replay()
    torch.cuda.synchronize()
    want = oracle.verify_sample(*host(target, draft, drafts, u))
    assert accepted.tolist() == want[0].tolist() and token.tolist() == want[1].tolist()


def test_wrong_tensors_are_refused():
    target, draft, drafts, u = inputs(2, 3, 40, seed=14)
    out = [torch.zeros(2, dtype=torch.int32, device="cuda") for _ in range(2)]
    good = [target, draft, drafts, u, *out]
    for i, bad in ((0, target.double()), (0, target[0]), (0, target.transpose(1, 2).contiguous().transpose(1, 2)), (1, draft[:, :2]), (1, draft[:, :, :39]),
                   (2, drafts.long()), (2, drafts[:, :2]), (3, u[:, :3]), (3, u.double()), (4, out[0][:1]), (5, out[0].float())):
        args = list(good)
        args[i] = bad
        with pytest.raises(ValueError):
            L.lacache_verify_sample(*args)
    with pytest.raises(ValueError):
        L.lacache_verify_sample(*good, status=torch.zeros(2, dtype=torch.int32, device="cuda"))


def near_borders(V, count, seed, head):
    """A row of V multiples of 2^-42 (fp32 values), one of 0.7 at `head`, the last 0, the others alike, each 6.45 times the last bit of
    0.7, and `count` u's whose borders lie 9 to 10 multiples before or behind u C, which is 2^-39 C: (row, u, tokens)."""
    rng = np.random.default_rng(seed)
    n = np.full(V, 6 * 2 ** 18 + 117_963)
    n[head], n[V - 1] = int(np.float32(0.7) * 2.0 ** 42), 0
    upto, total = np.cumsum(n), int(n.sum())
    u, tokens = [], []
    for x, i in enumerate(np.sort(rng.choice(V // 3 - 2, count, replace=False)).tolist()):
        i = 3 * i + 1                                        # (pairs i, i + 1 that share no token)
        if i in (head - 1, head):
            i = head + 1
        U = max(1, round(int(upto[i]) * 2 ** 24 / total))
        past = U * total >> 24                               # u C, rounded down
        below = x % 2 == 0                                   # C_i below u C: the token is the next
        shift = (past - 9 if below else past + 10) - int(upto[i])
        n[i] += shift
        n[i + 1] -= shift
        u.append(U * 2.0 ** -24)
        tokens.append(i + below)
    row = (n * 2.0 ** -42).astype(np.float32)
    assert int(n.sum()) == total and n[:-1].min() > 0 and np.array_equal(row.astype(np.float64) * 2.0 ** 42, n)
    upto = np.cumsum(n)                                      # in 2^-42, and u C in 2^-66
    for x, i in zip(u, tokens):
        assert (i == 0 or int(upto[i - 1]) << 24 <= int(x * 2 ** 24) * total) and int(upto[i]) << 24 > int(x * 2 ** 24) * total
    return row, u, tokens


@pytest.mark.parametrize("V,copies", [(262_147, 1), (131_072, 16), (262_147, 16), (1 << 20, 1), (1 << 20, 16)])
@pytest.mark.parametrize("head", [0, 77_777])
@pytest.mark.parametrize("residual", [False, True])
def test_borders_nearer_than_a_running_sum_holds(V, copies, head, residual):
    """One token of 0.7 and a flat tail: what a long sum and its rounding errors lose at every term shows. Both signs of a border 2^-39 C
    away, which errors of 2^-40 in C_i and in C do not reach; with few queries (eight blocks each) and with many (one)."""
    row, u, tokens = near_borders(V, 40, V + head, head)
    B = len(tokens) * copies
    assert (B > 608) == (copies > 1)
    target = torch.from_numpy(row).cuda()
    us = torch.tensor(u, dtype=torch.float32, device="cuda").repeat(copies).view(-1, 1)
    if residual:                                             # the same weights as differences, after a draft of weight 0 was refused
        less = torch.randint(0, 1 << 22, (V,), device="cuda").double() * 2.0 ** -42
        less[head] = 0.125
        p = target.double() + less
        less[V - 1] += 2.0 ** -21
        q = less.float()
        assert torch.equal(p.float().double(), p) and torch.equal(q.double(), less)
        got = call(p.float().expand(B, 2, V), q.expand(B, 1, V), torch.full((B, 1), V - 1, dtype=torch.int32, device="cuda"),
                   torch.cat((torch.full_like(us, 1 - 2.0 ** -24), us), 1))
    else:
        got = call(target.expand(B, 1, V), None, torch.zeros(B, 0, dtype=torch.int32, device="cuda"), us)
    assert got[0].tolist() == [0] * B
    assert got[1].tolist() == tokens * copies


@pytest.mark.parametrize("V", [33, 97, 3611, 40_000])
@pytest.mark.parametrize("k", [0, 2])
def test_the_last_token_of_any_weight_at_u_of_one(V, k):
    """Rows whose last tokens weigh less than the last bits of the whole: at u >= 1 none qualifies, however the sums round."""
    target, draft, drafts, u = inputs(40, k, V, seed=V, spread=10.0)
    target[::3, :, -2:] = 0.0
    u[:, -1] = torch.tensor([1.0, 1.5, 2.0, float("inf")], device="cuda").repeat(10)
    got = call(target, draft, drafts, u)
    finite = u.clone()
    finite[:, -1] = 1.0                                      # (a rational one, for the oracle)
    want = oracle.verify_sample(*host(target, draft, drafts, finite))
    assert got[0].tolist() == want[0].tolist() and got[1].tolist() == want[1].tolist()
    u[:, -1] = 1.0
    check(target, draft, drafts, u)
